// Attention of a step's rows over the paged cache (abq_attn.hip has the rules; abq_attn_d*.hip instantiate the kernels).
//
// Mathematics.  With c = scale * log2 e, a row's result is sum_t 2^(c q.k_t - m) v_t / sum_t 2^(c q.k_t - m) for any m; m follows
// the running maximum, and what was summed before is multiplied by 2^(old m - new m) when it moves.  Codes: the score is
// c * ks_t * (q . (code - zero)), whose inner product takes the exact differences; the value's scale goes into the exponent,
// 2^(c q.k_t + log2 vs_t - m) (code - zero), so that the weight is rounded to binary16 once, scale included, and a weight times its
// scale falls into binary16's range whatever the scale; the denominator adds the weight divided by its scale again.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T: a lane of the first product's result holds several tokens of one row, which
// is, with the tokens in that order, what the second product wants as its operand: the weights never leave the lane.  V^T comes
// from row-major V in LDS by the transposing LDS read.  m moves only when a score passes it by 2^8 (a weight of up to 256 loses
// nothing in binary16), so that most steps need no exchange between lanes and no pass over the sums.
//
// Roundings: the second product takes the weights as halves.  Few rows wait for memory, and take what that leaves of a weight as a second
// half: 22 bits for up to 2 % of the time (32 sequences of 2000 tokens 34.1 and 34.4 us; codes, 4 of 32768, 42.5 and 43.4).  Many rows
// take one half: the matrix pipe is what they wait for, and the second one's registers are not there (two groups of waves with heads of
// 128 go to scratch).  A weight is then off by 2^-11 of itself at most, either way, which over many tokens averages out below the result's
// own rounding.
#pragma once
#include "abq_kv.h"

#include <type_traits>

namespace abq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kManyRows = 128;    // rows of a workgroup of the kernel for many rows
constexpr int kManyTokens = 64;   // tokens of one of its steps
constexpr int kFewTokens = 32;    // tokens of a wave's step of the kernel for few rows
// Tokens of a part at least, where a sequence is shared out.  (Many rows at 384, 512, 768: 64 over 1000, 8 key heads, 20, 21, 25 us, 256 over
// 1000 27, 27, 29.5, a prompt of 512 20, 16, 16.)
constexpr int kFewLeast = 256, kManyLeast = 512;

struct AttnArgs {
    abq_kv_cache c;
    abq_batch b;
    int heads_q, group, page_shift;
    const uint16_t* q;
    int ldq;
    float scale2;        // scale * log2 e
    bool causal;
    uint16_t* y;
    int few, few_parts, many_parts;   // sequences of up to `few` rows (tokens * group) are the business of the part for few rows; parts at most
    int few_rows;        // and have at most so many rows
    unsigned many_wgs;   // workgroups of the part for many rows, per part of the tokens
    float *few_o, *many_o;      // results of parts, not yet divided by the sum: [seqs][heads][few_rows][few_parts][head_dim], [rows][heads_q][many_parts][head_dim]
    float2 *few_ml, *many_ml;   // their (m, sum)
    // number of the first part of row R (token * group + query head) of a sequence
    __device__ __forceinline__ int64_t few_part(int seq, int head, int R) const { return (((int64_t)seq * c.heads + head) * few_rows + R) * few_parts; }
    __device__ __forceinline__ int64_t many_part(int64_t yrow) const { return yrow * many_parts; }
};

// A sequence's rows and tokens within all bounds.
struct Sequence {
    int first, tokens, before, length;   // first row; new tokens that are handled; position of the first; tokens held
    __device__ __forceinline__ Sequence() : first(0), tokens(0), before(0), length(0) {}
    __device__ __forceinline__ Sequence(const AttnArgs& a, int seq)
    {
        const int r0 = a.b.row_start[seq], r1 = a.b.row_start[seq + 1], len = a.b.lens[seq];
        first = min(max(r0, 0), a.b.rows);
        const int n = min(max(r1, first), a.b.rows) - first;
        tokens = min(n, a.b.max_new);
        before = (int)min(max((int64_t)len - n, (int64_t)-INT32_MAX), (int64_t)INT32_MAX);
        const int64_t room = (int64_t)a.b.max_pages << a.page_shift;
        length = (int)min((int64_t)max(min(len, a.b.max_len), 0), room);
    }
    // tokens that new token i sees
    __device__ __forceinline__ int seen(int i, bool causal) const
    {
        return causal ? (int)min((int64_t)max((int64_t)before + i + 1, (int64_t)0), (int64_t)length) : length;
    }
};

// Up to half as much again as the least tokens of a part stay whole: joining costs as much as two steps of a lone workgroup.  (One
// token, 32 heads, context of 400: 9.9 us whole, 11.2 in two parts; of 512: 12.9 whole, 10.7 in three.  A prompt of 700 on 8 key heads:
// 19.0 whole, 22.6 where parts are launched.)
__host__ __device__ __forceinline__ bool stays_whole(int top, int least) { return top <= least + least / 2; }
// Tokens of one part of `top` when up to `parts` share them, in whole steps, at least `least`; the number of parts is then what covers top.
__device__ __forceinline__ int part_tokens(int top, int parts, int step, int least)
{
    if (stays_whole(top, least)) return max(top, 1);
    const int per = (int)(((int64_t)top + parts - 1) / parts);
    return (max(per, least) + step - 1) / step * step;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, h2)); }
__device__ __forceinline__ bool any(bool p) { return __ballot(p) != 0; }

// Four code bytes -> code - zero as four halves, exactly: 0x6400 | byte is 1024 + byte; `bias` holds -(1024 + zero) twice.
__device__ __forceinline__ void codes_to_halves(uint32_t codes, h2 bias, uint32_t* out)
{
    const uint32_t lo = __builtin_amdgcn_perm(0x64646464u, codes, 0x04010400u), hi = __builtin_amdgcn_perm(0x64646464u, codes, 0x04030402u);
    out[0] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, lo) + bias);
    out[1] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2, hi) + bias);
}
__device__ __forceinline__ h2 code_bias(int zero)
{
    const _Float16 v = (_Float16)(float)(-1024 - zero);
    return h2{v, v};
}

typedef __fp16 g4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) g4 lds_g4;
// Four rows of row-major halves, transposed: of each sixteen lanes, lane i gives the address of the (i % 4)-th four columns of row
// i / 4 and gets column i of the four rows.
__device__ __forceinline__ h4 read_transposed(const uint16_t* p)
{
    return __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_g4*)p));
}
__device__ __forceinline__ h8 join(h4 a, h4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }
// Halves that are infinite or NaN become zero; whether there was one.
__device__ __forceinline__ bool drop_not_finite(u4& x)
{
    uint32_t out = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t lo = (x[j] & 0x7C00u) == 0x7C00u ? 0xFFFFu : 0u, hi = (x[j] & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u;
        x[j] &= ~(lo | hi);
        out |= lo | hi;
    }
    return out != 0;
}
// A half that is infinite or NaN as a float; zero for any other.
__device__ __forceinline__ float only_not_finite(const uint16_t* p)
{
    const uint16_t h = *p;
    return (h & 0x7C00u) == 0x7C00u ? __half2float(__ushort_as_half(h)) : 0.0f;
}

// A value that is infinite or NaN in a step that some rows see only in part: 0 times it is none, so it stays out of the product
// there, and the tokens that hold one (not those without a page, for which another's is loaded) are kept track of ...
struct OddTokens {
    int first, last;
    __device__ __forceinline__ void clear() { first = INT32_MAX; last = -1; }
    __device__ __forceinline__ void found(int t, int to)
    {
        if (t < to) { atomicMin(&first, t); atomicMax(&last, t); }
    }
    __device__ __forceinline__ bool any() const { return last >= 0; }
};
// ... and what they hold is added to the results of the rows that see them, behind the stores of rows R0 .. R1 - 1.  (Whatever positive
// weight it has, it makes the sum infinite or NaN; what has gone through the product is so already.)
template <class F>   // part_of(R, yrow): where the part's result of a row is, null when the row's result is whole
__device__ __forceinline__ void add_not_finite(const AttnArgs& a, const Sequence& sq, int seq, int head, int R0, int R1, int first, int last, F&& part_of)
{
    __syncthreads();
    const int D = a.c.head_dim;
    for (int i = threadIdx.x; i < (R1 - R0) * D; i += blockDim.x) {
        const int R = R0 + i / D, d = i % D, end = min(last + 1, sq.seen(R / a.group, a.causal));
        float x = 0.0f;
        for (int t = first; t < end; ++t) {
            const int page = page_of(a.b, a.c, a.page_shift, seq, t);
            if (page < 0) t |= a.c.page_size - 1;   // (the next page's first comes then)
            else x += only_not_finite((const uint16_t*)a.c.v + vector_of(a.c, page, head, t & (a.c.page_size - 1)) * D + d);
        }
        if (x == 0.0f) continue;
        const int64_t yrow = (int64_t)(sq.first + R / a.group) * a.heads_q + head * a.group + R % a.group;
        if (float* const o = part_of(R, yrow)) {
            o[d] += x;
        } else {
            uint16_t* const y = a.y + yrow * D + d;
            *y = __half_as_ushort(__float2half_rn(__half2float(__ushort_as_half(*y)) + x));
        }
    }
}

// Each element of a row whose weights add up to nothing: zero if it sees no token; else its scores are all minus infinity, and it is 0 / 0.
__device__ __forceinline__ float without_weight(const AttnArgs& a, const Sequence& sq, int seq, int i)
{
    const int seen = sq.seen(i, a.causal), pages = (int)(((int64_t)seen + a.c.page_size - 1) >> a.page_shift);
    for (int p = 0; p < pages; ++p)
        if (page_of(a.b, a.c, a.page_shift, seq, p << a.page_shift) >= 0) return __builtin_nanf("");
    return 0.0f;
}

// Columns of the DP that a kernel goes over which every head that comes to it has.
template <int DP>
constexpr int kSureColumns = DP == 64 ? 16 : DP / 2 + 16;

constexpr float kFloor = -3.40282347e+38f;   // m of a row that has seen nothing, the lowest number: any other score passes it, and 2^(floor - m) is 0
// Scores from here on are rounded before m is taken from them.  2^(c x - m) of one operation has the product unrounded, which lies up to
// |m| 2^-24 above an m that is rounded: beyond the 2^8 that a weight may reach, and at 2^28 beyond binary16.
constexpr float kFarScore = 0x1p22f;
// Whether a row's largest score makes its m move, and m after it.  Each row decides for itself: were m raised along with another row's, a
// token that only that one sees would change how this one's weights are rounded.
__device__ __forceinline__ bool passes(float m, float score) { return score > m + 8.0f; }
__device__ __forceinline__ float moved(float m, float score) { return passes(m, score) ? score : m; }

// ---- few rows ------------------------------------------------------------------------------------
// One workgroup per sequence, key head and part of the tokens; NR tiles of sixteen rows (token * group + query head).  Its
// WAVES waves take 32 tokens in turn, each with a maximum, sums and an LDS region of its own (no barrier in the loop), and are
// joined at the end.  K goes from memory straight into the matrix operand's registers, V through LDS for the transposition.
// What bounds it: memory.  A wave has 16 KB in flight (32 tokens of K and V, 128 halves each) from the moment it has used the
// last ones, and two to four workgroups share a compute unit.  32 sequences of 1..2 thousand tokens, 32 heads on 32 of 128, 814 MB:
// 148 us, 5.5 TB/s (a large copy: 5.1); as codes, four of 19..32 thousand, 103088 tokens on 8 heads, 219 MB: 41 us, 5.3 TB/s, and 5 for
// the joining.  One sequence of 513 on 32 heads is latency: 7.5 us, and 3.2 for the joining.
template <int DP, int WAVES>
constexpr int kFewLds = WAVES * kFewTokens * (DP + 16);   // halves
template <int DP, bool CODES, int NR, int WAVES>
__device__ __forceinline__ void attn_few(const AttnArgs& a, uint16_t* lds, int head, int seq, int part)
{
    constexpr int DT = DP / 16;                      // tiles of sixteen columns
    constexpr int QS = DP / 32;                      // steps of the first product
    constexpr int KV = CODES ? DP / 64 : DP / 32;    // 16-byte loads of a lane per sixteen tokens of K
    constexpr int LPT = CODES ? DP / 16 : DP / 8;    // lanes that hold a token of V
    constexpr int TPL = 64 / LPT;                    // tokens of V per load of a wave
    constexpr int VV = kFewTokens / TPL;             // 16-byte loads of a lane per step's V
    constexpr int VS = DP + 16;                      // halves of a row of V in LDS: eight banks on, sixteen lanes of a transposing read take all
    constexpr int OS = DP + 4;                       // floats of a row when the waves are joined
    __shared__ float2 s_ml[WAVES][16];
    __shared__ OddTokens s_odd;
    static_assert(kFewLds<DP, WAVES> == WAVES * kFewTokens * VS && kFewLds<DP, WAVES> * 2 >= WAVES * 16 * OS * 4, "the waves are joined in the memory of V");

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, g = lane >> 4, D = a.c.head_dim;
    const Sequence sq(a, seq);
    const int nrows = sq.tokens * a.group;
    if (nrows <= 0 || nrows > a.few) return;
    const int top = sq.seen(sq.tokens - 1, a.causal), least = sq.seen(0, a.causal);
    const int per = part_tokens(top, a.few_parts, kFewTokens, kFewLeast), nparts = max(1, (top + per - 1) / per);
    if (part >= nparts) return;
    const int from = part * per, to = min(top, from + per);
    if (tid == 0) s_odd.clear();
    __syncthreads();

    // queries: row n16 of each tile, the columns that this lane's loads of K hold
    h8 qv[NR][QS];
    int vis[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        const int R = 16 * t + n16, tok = R / a.group, hq = head * a.group + R % a.group;
        vis[t] = R < nrows ? sq.seen(tok, a.causal) : 0;
        const uint16_t* row = a.q + (size_t)(sq.first + (R < nrows ? tok : 0)) * a.ldq + (size_t)hq * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            const int d = CODES ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
            u4 v = {0, 0, 0, 0};
            if (R < nrows && d < D) v = *reinterpret_cast<const u4*>(row + d);
            qv[t][s] = __builtin_bit_cast(h8, v);
        }
    }

    f4 o[NR][DT];
    float m[NR], l[NR];
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        m[t] = kFloor;
        l[t] = 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) o[t][i] = f4{0, 0, 0, 0};
    }

    u4 kr[2][KV], vr[VV];
    f4 ks[2], vs[2];        // codes: scales of the lane's tokens in the order of the scores
    uint32_t kz[2], vz[VV];
    uint16_t* const lv = lds + wave * kFewTokens * VS;

    int pages_at = 0, table = -1;   // the pages of the wave's next 32 steps, two to a step: lane 2 i + j holds step i's j-th
    auto fetch_pages = [&](int i) {
        pages_at = i;
        const int t = from + ((i + (lane >> 1)) * WAVES + wave) * kFewTokens + 16 * (lane & 1);
        table = t < to ? page_of(a.b, a.c, a.page_shift, seq, t) : -1;
    };
    int pg[2];   // (of the step that is loaded)
    auto load = [&](int i) {
        if (i - pages_at >= 32) fetch_pages(i);
        const int t0 = from + (i * WAVES + wave) * kFewTokens;
        int64_t vec[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            pg[j] = __builtin_amdgcn_readlane(table, 2 * (i - pages_at) + j);
            vec[j] = vector_of(a.c, max(pg[j], 0), head, (t0 + 16 * j) & (a.c.page_size - 1));   // (no page: the first one's, masked)
#pragma unroll
            for (int u = 0; u < KV; ++u) {
                int d = CODES ? 64 * u + 16 * g : 32 * u + 8 * g;
                if (d >= D) d = 0;   // (codes: the queries are zero there)
                kr[j][u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.k + ((vec[j] + n16) * D + d) * (CODES ? 1 : 2));
            }
            if constexpr (CODES) {
                kz[j] = a.c.k_zero[vec[j] + n16];
                ks[j] = *reinterpret_cast<const f4*>(a.c.k_scale + vec[j] + 4 * g);
                vs[j] = *reinterpret_cast<const f4*>(a.c.v_scale + vec[j] + 4 * g);
            }
        }
#pragma unroll
        for (int u = 0; u < VV; ++u) {
            int d = (lane % LPT) * (CODES ? 16 : 8);
            if (d >= D) d = 0;   // (columns that are not stored)
            const int64_t at = (u * TPL < 16 ? vec[0] : vec[1]) + ((u * TPL + lane / LPT) & 15);
            if constexpr (CODES) vz[u] = a.c.v_zero[at];
            vr[u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.v + (at * D + d) * (CODES ? 1 : 2));
        }
    };

    const int steps = to > from + wave * kFewTokens ? (to - from - wave * kFewTokens + WAVES * kFewTokens - 1) / (WAVES * kFewTokens) : 0;
    if (steps) {
        fetch_pages(0);
        load(0);
    }
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        const int t0 = from + (i * WAVES + wave) * kFewTokens;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const bool masked = t0 + kFewTokens > least || pg[0] < 0 || pg[1] < 0;
        const bool gone0 = pg[0] < 0, gone1 = pg[1] < 0;
        // V to LDS
#pragma unroll
        for (int u = 0; u < VV; ++u) {
            uint16_t* dst = lv + (u * TPL + lane / LPT) * VS + (lane % LPT) * (CODES ? 16 : 8);
            if constexpr (CODES) {
                const h2 bias = code_bias((int)vz[u]);
                u4 w[2];
#pragma unroll
                for (int j = 0; j < 4; ++j) codes_to_halves(vr[u][j], bias, (uint32_t*)&w[j >> 1] + 2 * (j & 1));
                *reinterpret_cast<u4*>(dst) = w[0];
                *reinterpret_cast<u4*>(dst + 8) = w[1];
            } else {
                u4 v = vr[u];
                if (masked && drop_not_finite(v) && !(u * TPL < 16 ? gone0 : gone1)) s_odd.found(t0 + u * TPL + lane / LPT, to);
                *reinterpret_cast<u4*>(dst) = v;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (other lanes' rows are read below)
        if (!CODES && DP != D) {   // zero queries do not rid the sum of an infinity in the columns behind the head
            asm volatile("");      // (a branch, not a selection that heads of DP go through too)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int u = 0; u < KV; ++u)
                    if (32 * u + 32 > kSureColumns<DP> && 32 * u + 8 * g >= D) kr[j][u] = u4{0, 0, 0, 0};
        }
        // scores
        f4 s[NR][2];
#pragma unroll
        for (int t = 0; t < NR; ++t) s[t][0] = s[t][1] = f4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int u = 0; u < KV; ++u) {
                if constexpr (CODES) {
                    const h2 bias = code_bias((int)kz[j]);
                    u4 w[2];
#pragma unroll
                    for (int e = 0; e < 4; ++e) codes_to_halves(kr[j][u][e], bias, (uint32_t*)&w[e >> 1] + 2 * (e & 1));
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int t = 0; t < NR; ++t) s[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w[e]), qv[t][2 * u + e], s[t][j], 0, 0, 0);
                } else {
#pragma unroll
                    for (int t = 0; t < NR; ++t) s[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, kr[j][u]), qv[t][u], s[t][j], 0, 0, 0);
                }
            }
        }
        f4 inv[2];   // codes: 1 / scale of the values
        if constexpr (CODES) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    inv[j][r] = __builtin_amdgcn_rcpf(vs[j][r]);
                    const float lg = __builtin_amdgcn_logf(vs[j][r]), c = ks[j][r] * a.scale2;
#pragma unroll
                    for (int t = 0; t < NR; ++t) s[t][j][r] = fmaf(s[t][j][r], c, lg);
                }
        } else {
#pragma unroll
            for (int t = 0; t < NR; ++t) { s[t][0] *= a.scale2; s[t][1] *= a.scale2; }
        }
        if (masked) {
#pragma unroll
            for (int t = 0; t < NR; ++t)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if ((j ? gone1 : gone0) || t0 + 16 * j + 4 * g + r >= vis[t]) s[t][j][r] = -INFINITY;
        }
        if (i + 1 < steps) load(i + 1);

#pragma unroll
        for (int t = 0; t < NR; ++t) {
            float lm = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])), fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
            if (any(passes(m[t], lm))) {
                lm = fmaxf(lm, __shfl_xor(lm, 16, 64));
                lm = moved(m[t], fmaxf(lm, __shfl_xor(lm, 32, 64)));
                const float fade = __builtin_amdgcn_exp2f(m[t] - lm);
                m[t] = lm;
                l[t] *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[t][d] *= fade;
            }
            float w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                w[e] = __builtin_amdgcn_exp2f(s[t][e >> 2][e & 3] - m[t]);
                if constexpr (CODES) l[t] += w[e] != 0.0f || !masked ? w[e] * inv[e >> 2][e & 3] : 0.0f;   // (a masked token's scale may be anything)
                else l[t] += w[e];
            }
            const u4 pw = {pack2(w[0], w[1]), pack2(w[2], w[3]), pack2(w[4], w[5]), pack2(w[6], w[7])};
            const h8 p = __builtin_bit_cast(h8, pw);
            // what the rounding left is a second operand: the matrix pipe has room for it beside the loads
#pragma unroll
            for (int e = 0; e < 8; ++e) w[e] -= (float)p[e];
            const u4 rw = {pack2(w[0], w[1]), pack2(w[2], w[3]), pack2(w[4], w[5]), pack2(w[6], w[7])};
            const h8 rest = __builtin_bit_cast(h8, rw);
            const uint16_t* src = lv + (4 * g + (n16 >> 2)) * VS + 4 * (n16 & 3);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const h8 v = join(read_transposed(src + 16 * d), read_transposed(src + 16 * VS + 16 * d));
                o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p, o[t][d], 0, 0, 0);
                o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, rest, o[t][d], 0, 0, 0);
            }
        }
    }

    // the waves' sums as one, a tile of rows at a time, 4 WAVES threads to a row
    float* const so = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int t = 0; t < NR; ++t) {
        l[t] += __shfl_xor(l[t], 16, 64);
        l[t] += __shfl_xor(l[t], 32, 64);
        __syncthreads();   // (V is used up; the tile before is stored)
        if (g == 0) s_ml[wave][n16] = float2{m[t], l[t]};
#pragma unroll
        for (int d = 0; d < DT; ++d) *reinterpret_cast<f4*>(so + (wave * 16 + n16) * OS + 16 * d + 4 * g) = o[t][d];
        __syncthreads();
        constexpr int TPR = 4 * WAVES;
        const int r = tid / TPR, R = 16 * t + r;
        if (R < nrows) {
            float top_m = kFloor, sum = 0.0f, f[WAVES];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top_m = fmaxf(top_m, s_ml[w][r].x);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                f[w] = __builtin_amdgcn_exp2f(s_ml[w][r].x - top_m);
                sum += f[w] * s_ml[w][r].y;
            }
            const int64_t yrow = (int64_t)(sq.first + R / a.group) * a.heads_q + head * a.group + R % a.group;
            for (int d = 4 * (tid % TPR); d < D; d += 4 * TPR) {
                f4 v = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) v += f[w] * *reinterpret_cast<const f4*>(so + (w * 16 + r) * OS + d);
                if (nparts > 1) {
                    *reinterpret_cast<f4*>(a.few_o + (a.few_part(seq, head, R) + part) * D + d) = v;
                } else {
                    const float inv_sum = sum == 0.0f ? 1.0f : 1.0f / sum;
                    if (sum == 0.0f) v = f4{} + without_weight(a, sq, seq, R / a.group);
                    *reinterpret_cast<uint2*>(a.y + yrow * D + d) = uint2{pack2(v[0] * inv_sum, v[1] * inv_sum), pack2(v[2] * inv_sum, v[3] * inv_sum)};
                }
            }
            if (nparts > 1 && tid % TPR == 0) a.few_ml[a.few_part(seq, head, R) + part] = float2{top_m, sum};
        }
    }
    if constexpr (!CODES) {
        if (s_odd.any()) add_not_finite(a, sq, seq, head, 0, nrows, s_odd.first, s_odd.last, [&](int R, int64_t) { return nparts > 1 ? a.few_o + (a.few_part(seq, head, R) + part) * D : nullptr; });
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// The sequence and tile of a workgroup: tiles of the sequences with more than `few` rows, in order; within a sequence the last
// tile (the longest under the causal mask) first.  false: there is none.
__device__ __forceinline__ bool many_tile(const AttnArgs& a, int index, int* seq, int* tile, Sequence* sq)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.b.seqs; s0 += 64) {
        Sequence mine;
        if (s0 + lane < a.b.seqs) mine = Sequence(a, s0 + lane);
        const int nrows = mine.tokens * a.group, nt = nrows > a.few ? (nrows + kManyRows - 1) / kManyRows : 0;
        int sum = nt;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(sum, off, 64);
            if (lane >= off) sum += up;
        }
        const uint64_t past = __ballot(sum > index);
        if (past) {
            const int at = __builtin_amdgcn_readfirstlane(__builtin_ctzll(past));
            *seq = s0 + at;
            *tile = __builtin_amdgcn_readlane(sum, at) - 1 - index;
            sq->first = __builtin_amdgcn_readlane(mine.first, at);
            sq->tokens = __builtin_amdgcn_readlane(mine.tokens, at);
            sq->before = __builtin_amdgcn_readlane(mine.before, at);
            sq->length = __builtin_amdgcn_readlane(mine.length, at);
            return true;
        }
        index -= __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The waves' LDS work done and seen by the workgroup.  (Loads from memory stay in flight: a workgroup fence would wait for them.)
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// N loads of sixteen bytes a lane from base + offset[i] + 1024 i to LDS, a wave's N KB in a row from LDS address `to` on (the immediate
// offset counts on both sides); complete when the wave's vmcnt says so.
template <int N>
__device__ __forceinline__ void lds_load(const uint8_t* base, const uint32_t* offset, uint32_t to)
{
    static_assert(N == 2 || N == 4);
    if constexpr (N == 4)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                     "global_load_lds_dwordx4 %3, %5 offset:2048\n\tglobal_load_lds_dwordx4 %4, %5 offset:3072"
                     : : "s"(to), "v"(offset[0]), "v"(offset[1]), "v"(offset[2]), "v"(offset[3]), "s"(base) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024"
                     : : "s"(to), "v"(offset[0]), "v"(offset[1]), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ uint32_t lds_address(const uint16_t* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint16_t*)p; }

// One workgroup per key head, 128 rows (token * group + query head) and part of the tokens.  GROUPS groups of four waves, a
// wave for 32 of the rows in each; the groups take the steps of 64 tokens in turn and are joined at the end.  A step of a group has two
// halves with a barrier behind each: the matrix instructions (scores of this step, and the weights of the last one times
// its values), and everything else (softmax, loads; of codes also the next step's way through registers to LDS).  The second group runs
// half a step behind the first, so that of the two waves of a SIMD one has matrix and the other vector work.  Each group has two
// buffers for K and two for V, of steps in turn; binary16 goes into them straight from memory, the next but one while this is used.
// What bounds it: of a step's 3400 clocks the matrix half takes 1500 and the rest 1900 (1150 of them softmax),
// which the other group's matrix half hides all but 400 of.  1024 tokens over 15360, 32 heads on 8 of 128: 272 us (980 TFLOP/s; one
// group alone 370), as codes 363 (735), both 6 % longer on some cards.
// A prompt of 2048, 32 heads, takes 54..57 us (600..640 TFLOP/s): two workgroups a unit, one after the other, 17 rounds of two steps at
// 1.6 us together, and about 12 us for each one's start and end (a prompt of 128, one round, takes 13; 16 heads, one workgroup a unit of
// up to 16 rounds, 37).
template <int DP, bool CODES, int GROUPS>
constexpr int kManyLds = GROUPS * 2 * kManyTokens * (CODES ? 2 * DP + 40 : 2 * DP);   // halves
template <int DP, bool CODES, int GROUPS>
__device__ __forceinline__ void attn_many(const AttnArgs& a, uint16_t* lds, unsigned index, int part)
{
    constexpr int DT = DP / 32;                       // tiles of 32 columns of the result
    constexpr int QS = DP / 16;                       // steps of the first product
    constexpr int LPT = CODES ? DP / 16 : DP / 8;     // lanes that hold a token
    constexpr int TPL = 64 / LPT;                     // tokens per load of a wave
    constexpr int LV = 16 / TPL;                      // 16-byte loads of a lane per step, of K and of V: wave w loads the step's w-th sixteen tokens
    constexpr int BYTES = CODES ? 1 : 2;
    constexpr bool DIRECT = !CODES;                   // binary16 goes from memory to LDS directly, codes through registers
    // Halves of a row in LDS.  Codes: 4 banks on from row to row for the reads of K, 16 for the transposing ones of V.  The direct loads
    // write rows as they are; there the 16-byte pieces of row r change places, piece c lying in place c ^ turn(r).
    constexpr int KS = DIRECT ? DP : DP + 8, VS = DIRECT ? DP : DP + 32;
    constexpr int KL = kManyTokens * KS, VL = kManyTokens * VS;   // halves of a buffer
    constexpr int GL = 2 * (KL + VL);                 // of a group
    static_assert(GROUPS == 1 || GROUPS * GL * 2 >= kManyRows * DP * 4, "the groups are joined in the memory of K and V");
    static_assert(kManyLds<DP, CODES, GROUPS> == GROUPS * GL);
    __shared__ __align__(16) float s_par[CODES ? GROUPS : 1][2][3][CODES ? kManyTokens : 4];   // codes, of two steps: scales of K, logarithms and reciprocals of those of V
    __shared__ float2 s_ml[GROUPS == 1 ? 1 : kManyRows];
    __shared__ OddTokens s_odd;

    const int head = index % a.c.heads, tid = threadIdx.x & 255, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int grp = GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8);
    const int n32 = lane & 31, hh = lane >> 5, D = a.c.head_dim;
    int seq, tile;
    Sequence sq;
    if (!many_tile(a, index / a.c.heads, &seq, &tile, &sq)) return;
    const int nrows = sq.tokens * a.group, R0 = tile * kManyRows;
    const int top = sq.seen((min(nrows, R0 + kManyRows) - 1) / a.group, a.causal);
    const int per = part_tokens(top, a.many_parts, kManyTokens, kManyLeast), nparts = max(1, (top + per - 1) / per);
    if (part >= nparts) return;
    const int from = part * per, to = min(top, from + per), all_steps = (to - from + kManyTokens - 1) / kManyTokens;
    const int steps = (all_steps - grp + GROUPS - 1) / GROUPS, rounds = (all_steps + GROUPS - 1) / GROUPS;   // this group's; the most of any group

    // this lane's row, and what the wave's rows and the tile's see at least and at most
    const int W0 = R0 + 32 * wave, R = W0 + n32, tok = R / a.group, hq = head * a.group + R % a.group;
    const int vis = R < nrows ? sq.seen(tok, a.causal) : 0, tile_least = sq.seen(R0 / a.group, a.causal);
    const int wave_least = W0 < nrows ? sq.seen(W0 / a.group, a.causal) : 0, wave_top = W0 < nrows ? sq.seen((min(nrows, W0 + 32) - 1) / a.group, a.causal) : 0;
    // A negative scale is the queries' sign; the scale itself is kept above 0, so that a masked score stays minus infinity under it.
    const float scale2 = fmaxf(fabsf(a.scale2), 1e-37f);
    h8 qv[QS];
    {
        const uint32_t sign = a.scale2 < 0.0f ? 0x80008000u : 0u;
        const uint16_t* row = a.q + (size_t)(sq.first + (R < nrows ? tok : 0)) * a.ldq + (size_t)hq * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            u4 v = {0, 0, 0, 0};
            if (R < nrows && 16 * s + 8 * hh < D) v = *reinterpret_cast<const u4*>(row + 16 * s + 8 * hh) ^ sign;
            qv[s] = __builtin_bit_cast(h8, v);
        }
    }
    f16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f16{};
    float m = kFloor, l = 0.0f;

    uint16_t *const lk = lds + grp * GL, *const lv = lk + 2 * KL;   // two buffers each, a step's in number step % 2
    auto t_of = [&](int j) { return from + (j * GROUPS + grp) * kManyTokens; };   // first token of the group's step j

    // Where the group's steps lie: lane 4 i + q holds the q-th sixteen tokens of step at + i, as the number of sixteens in front of them
    // (0 where there is no page, and a bit of `gone`).  Sixteen steps to a window; the next one, fourteen steps on, is fetched ahead,
    // so that step j's window always holds steps j + 1 and j + 2.
    const int per_head = a.c.page_size >> 4, per_page = per_head * a.c.heads;
    struct Window { uint32_t sixteens; uint64_t gone; };
    auto fetch = [&](int j) {
        const int t = t_of(j + (lane >> 2)) + 16 * (lane & 3), page = t < to ? page_of(a.b, a.c, a.page_shift, seq, t) : -1;
        return page < 0 ? -1 : page * per_page + head * per_head + ((t & (a.c.page_size - 1)) >> 4);
    };
    auto window = [&](int fetched) { return Window{(uint32_t)max(fetched, 0), __ballot(fetched < 0)}; };
    int at = 0, ahead = -1;
    Window win{};
    // Reads of K: eight rows, one piece of each, sixteen rows with one turn each (two rows of up to 64 columns fill the banks: one turn for
    // both).  Transposing reads of V: of four rows four neighbouring pieces each, which have to lie in four different quarters of the banks.
    auto turn_k = [](int r) { return !DIRECT ? 0 : DP == 64 ? (r >> 1) & 7 : r & 15; };
    auto turn_v = [](int r) { return !DIRECT ? 0 : DP == 64 ? ((r >> 1) & 1) << 2 : (r & 3) << 2 | ((r >> 2) & 3); };
    // this lane's places from the first byte of its wave's sixteen tokens (direct loads: less what lds_load adds, on kBias)
    constexpr uint32_t kBias = DIRECT ? 3072 : 0;
    uint32_t place_k[LV], place_v[LV];
#pragma unroll
    for (int u = 0; u < LV; ++u) {
        const int r = u * TPL + lane / LPT;
        int dk = ((lane % LPT) ^ turn_k(r)) * (CODES ? 16 : 8), dv = ((lane % LPT) ^ turn_v(r)) * (CODES ? 16 : 8);
        if (dk >= D) dk = 0;   // (K: left out of the product, or of codes against zero queries; V: columns that are not stored)
        if (dv >= D) dv = 0;
        const uint32_t less = DIRECT ? kBias - 1024u * (u & 3) : 0u;
        place_k[u] = (uint32_t)(r * D + dk) * BYTES + less;
        place_v[u] = (uint32_t)(r * D + dv) * BYTES + less;
    }
    const uint32_t stride = 16u * D * BYTES;
    uint32_t next = 0;   // the wave's sixteen tokens of the step whose K is loaded, and the byte they begin with
    uint64_t next_byte = 0;
    auto locate = [&](int j) {
        next = __builtin_amdgcn_readlane(win.sixteens, 4 * (j - at) + wave);
        next_byte = (uint64_t)next * stride - kBias;
    };
    const uint32_t lk_to = __builtin_amdgcn_readfirstlane(lds_address(lk + 16 * wave * KS)), lv_to = __builtin_amdgcn_readfirstlane(lds_address(lv + 16 * wave * VS));
    auto load_zero = [&](const uint8_t* base, int u) { return (uint32_t)(base + (uint64_t)next * 16)[(uint32_t)(u * TPL + lane / LPT)]; };
    u4 kr[CODES ? LV : 1], vr[CODES ? LV : 1];
    uint32_t kz[LV], vz[LV];
    float t_ks = 0.0f, t_vs = 1.0f;   // codes: scales of the step's token `lane` (the group's first wave)
    auto load_k = [&](int u) {   // codes, of the step that `next` tells of
        kr[u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.k + next_byte + place_k[u]);
        kz[u] = load_zero(a.c.k_zero, u);
    };
    auto load_v = [&](int u) {
        vr[u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.v + next_byte + place_v[u]);
        vz[u] = load_zero(a.c.v_zero, u);
    };
    auto load_scales = [&](int j) {
        if (CODES && wave == 0) {
            const uint32_t mine = __shfl(win.sixteens, 4 * (j - at) + (lane >> 4), 64);
            const uint64_t vec = (uint64_t)mine * 16 + (lane & 15);
            t_ks = a.c.k_scale[vec];
            t_vs = a.c.v_scale[vec];
        }
    };
    auto gone_at = [&](int j) { return (unsigned)(win.gone >> (4 * (j - at))) & 15u; };   // sixteens of a step that have no page
    const int row_at = 16 * wave + lane / LPT, col_at = (lane % LPT) * (CODES ? 16 : 8);
    auto store = [&](uint16_t* dst, const u4& v, uint32_t z) {
        const h2 bias = code_bias((int)z);
        uint32_t x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) codes_to_halves(v[e], bias, x + 2 * e);
        *reinterpret_cast<u4*>(dst) = u4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<u4*>(dst + 8) = u4{x[4], x[5], x[6], x[7]};
    };
    auto store_k = [&](int u, int j) { store(lk + (j & 1) * KL + (u * TPL + row_at) * KS + col_at, kr[u], kz[u]); };
    auto store_v = [&](int u, int j) { store(lv + (j & 1) * VL + (u * TPL + row_at) * VS + col_at, vr[u], vz[u]); };
    // Direct loads, in the second half, where they hold up no matrix instruction: V of the next step and K of the one behind it, into the
    // buffers that the first half has read.
    auto send_v = [&](int j) {
        if constexpr (DIRECT) {
            constexpr int N = LV < 4 ? LV : 4;
#pragma unroll
            for (int u = 0; u < LV; u += N) lds_load<N>((const uint8_t*)a.c.v + next_byte, place_v + u, lv_to + (j & 1) * VL * 2 + u * 1024);
        }
    };
    auto send_k = [&](int j) {
        if constexpr (DIRECT) {
            constexpr int N = LV < 4 ? LV : 4;
#pragma unroll
            for (int u = 0; u < LV; u += N) lds_load<N>((const uint8_t*)a.c.k + next_byte, place_k + u, lk_to + (j & 1) * KL * 2 + u * 1024);
        }
    };
    auto send = [&](int j) {
        if (DIRECT && j + 1 < steps) {
            send_v(j + 1);
            if (j + 2 < steps) {
                locate(j + 2);
                send_k(j + 2);
            }
        }
    };
    // Those of the second half before have arrived (V of this step, K of the next; all but this half's own), V of a masked step without what
    // is not finite.  (A thread looks after what it has loaded.)
    auto arrive = [&](int j) {
        if constexpr (DIRECT) {
            __builtin_amdgcn_sched_barrier(0);
            if (j + 2 < steps) __builtin_amdgcn_s_waitcnt(0x0F70 | (2 * LV & 15) | (2 * LV >> 4) << 14);   // vmcnt(2 LV)
            else __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
            asm volatile("" ::: "memory");
            if (j < steps && (t_of(j) + kManyTokens > tile_least || gone_at(j) != 0)) {
#pragma unroll
                for (int u = 0; u < LV; ++u) {
                    u4* const p = reinterpret_cast<u4*>(lv + (j & 1) * VL + (u * TPL + row_at) * VS + col_at);
                    u4 v = *p;
                    if (drop_not_finite(v)) {
                        if (!(gone_at(j) >> wave & 1u)) s_odd.found(t_of(j) + u * TPL + row_at, to);
                        *p = v;
                    }
                }
            }
        }
    };
    auto store_scales = [&](int j) {
        if (CODES && wave == 0) {
            s_par[grp][j & 1][0][lane] = t_ks * scale2;
            s_par[grp][j & 1][1][lane] = __builtin_amdgcn_logf(t_vs);
            s_par[grp][j & 1][2][lane] = __builtin_amdgcn_rcpf(t_vs);
        }
    };

    h8 w[4];   // a step's weights in the order of the second product: of s[c / 2][8 (c % 2) ..] in w[c]
    // this lane's place in the operands' rows, in bytes; of another piece of the row: the turned place
    const uint32_t k_at = (n32 * KS + (hh ^ turn_k(n32)) * 8) * 2;
    const int v_row = 4 * hh + ((lane & 15) >> 2);
    const uint32_t v_at = (v_row * VS + ((2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) ^ turn_v(v_row)) * 8 + 4 * (lane & 1)) * 2;
    // First half of step j: the matrix instructions in QS slots of two of each product, their operands read one slot ahead; and between
    // them, of codes, V of this step and K of the next from registers to LDS and the loads behind those.  The scores of token 32 k + 8
    // (e / 4) + 4 hh + e % 4 come to s[k][e].
    auto matrix = [&](int j, auto with_scores, auto with_values, f16* s) {
        constexpr bool S = decltype(with_scores)::value, V = decltype(with_values)::value;
        const uint8_t *const kp = (const uint8_t*)(lk + (j & 1) * KL), *const vp = (const uint8_t*)(lv + ((j & 1) ^ 1) * VL);
        const bool v_here = j < steps, k_here = j + 1 < steps, k_next = j + 2 < steps;
        if (j + 2 - at >= 16) {
            at += 14;
            win = window(ahead);
            ahead = fetch(at + 14);
        }
        h8 ko[2][2], vo[2][2];
        auto read = [&](int st) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (S) ko[st & 1][k] = *reinterpret_cast<const h8*>(kp + (DIRECT ? k_at ^ (uint32_t)(32 * st) : k_at + 32 * st) + 32 * k * KS * 2);
                if constexpr (V) {
                    const int c = (2 * st + k) / DT, d = (2 * st + k) % DT;
                    const uint8_t *const p0 = vp + (DIRECT ? v_at ^ (uint32_t)(64 * d) : v_at + 64 * d) + 16 * c * VS * 2;
                    const uint8_t *const p1 = vp + (DIRECT ? v_at ^ (uint32_t)(64 * d + (DP == 64 ? 0 : 32)) : v_at + 64 * d) + (16 * c + 8) * VS * 2;
                    vo[st & 1][k] = join(read_transposed((const uint16_t*)p0), read_transposed((const uint16_t*)p1));
                }
            }
        };
        read(0);
#pragma unroll
        for (int st = 0; st < QS; ++st) {
            __builtin_amdgcn_sched_barrier(0);
            if (st + 1 < QS) read(st + 1);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (CODES) {
#pragma unroll
                for (int i = st * 2 * LV / QS; i < (st + 1) * 2 * LV / QS; ++i) {   // V first: it is loaded first
                    if (i < LV) {
                        if (v_here) store_v(i, j);
                        if (k_here) load_v(i);
                    } else {
                        if (i == LV && k_next) locate(j + 2);
                        if (k_here) store_k(i - LV, j + 1);
                        if (k_next) load_k(i - LV);
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                if constexpr (S) {
                    // Binary16: zero queries do not rid the sum of an infinity in the columns behind the head.  The product stops there; of the
                    // widest heads, which have no register for what a branch keeps apart, it goes over zeros.  (1024 tokens over 15360, 32 heads
                    // on 8: of 80, 255 us with all columns, 239 so, 256 over zeros; of 256, 581 with all columns, 582 so, 991 with the branch.)
                    const bool behind = !CODES && 16 * st >= kSureColumns<DP> && 16 * st >= D;
                    u4 kv = __builtin_bit_cast(u4, ko[st & 1][k]);
                    if (GROUPS == 1 && behind) kv = u4{0, 0, 0, 0};
                    if (GROUPS == 1 || !behind) s[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, kv), qv[st], st ? s[k] : f16{}, 0, 0, 0);
                }
                if constexpr (V) o[(2 * st + k) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vo[st & 1][k], w[(2 * st + k) / DT], o[(2 * st + k) % DT], 0, 0, 0);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (k_here) store_scales(j + 1);
        if (k_next) load_scales(j + 2);
    };
    auto softmax = [&](int j, f16* s) {
        const int t0 = t_of(j);
        const unsigned gone = gone_at(j);
        const bool masked = t0 + kManyTokens > wave_least || gone != 0;
        const float* par = &s_par[CODES ? grp : 0][j & 1][0][0];
        if constexpr (CODES) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f4 c = *reinterpret_cast<const f4*>(par + 32 * k + 8 * e + 4 * hh), lg = *reinterpret_cast<const f4*>(par + kManyTokens + 32 * k + 8 * e + 4 * hh);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s[k][4 * e + r] = fmaf(s[k][4 * e + r], c[r], lg[r]);
                }
        }
        if (masked) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = 32 * k + 8 * (e >> 2) + 4 * hh + (e & 3);
                    if (t0 + t >= vis || (gone >> (2 * k + (e >> 3)) & 1u)) s[k][e] = -INFINITY;
                }
        }
        float lm = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int e = 1; e < 16; ++e) lm = fmaxf(fmaxf(lm, s[0][e]), s[1][e]);
        if constexpr (!CODES) lm *= scale2;
        if (any(passes(m, lm))) {
            lm = moved(m, fmaxf(lm, __shfl_xor(lm, 32, 64)));
            const float fade = __builtin_amdgcn_exp2f(m - lm);
            m = lm;
            l *= fade;
#pragma unroll
            for (int d = 0; d < DT; ++d) o[d] *= fade;
        }
        float factor = scale2, base = m;
        if constexpr (!CODES) {
            const bool far = fabsf(m) >= kFarScore && m != kFloor;   // (each row for itself)
            if (any(far)) {
                asm volatile("");   // (a branch)
                factor = far ? 1.0f : scale2;
                base = far ? 0.0f : m;
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[k][e] = far ? s[k][e] * scale2 - m : s[k][e];
            }
        }
        float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            u4 pw;
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                float x[4];
                f4 inv = {0, 0, 0, 0};
                if constexpr (CODES) inv = *reinterpret_cast<const f4*>(par + 2 * kManyTokens + 16 * c + 4 * e + 4 * hh);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = s[c >> 1][8 * (c & 1) + 2 * e + r];
                    x[r] = __builtin_amdgcn_exp2f(CODES ? v - m : fmaf(v, factor, -base));
                    const float part = !CODES ? x[r] : x[r] != 0.0f || !masked ? x[r] * inv[r] : 0.0f;   // (a masked token's scale may be anything)
                    (r & 1 ? sum1 : sum0) += part;
                }
                pw[e] = pack2(x[0], x[1]);
                pw[e + 1] = pack2(x[2], x[3]);
            }
            w[c] = __builtin_bit_cast(h8, pw);
        }
        l += sum0 + sum1;
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]), "+v"(l));   // (all of it in this half of the step)
    };

    if (threadIdx.x == 0) s_odd.clear();
    if (steps) {   // K of step 0 to LDS, V of step 0 and K of step 1 on their way
        win = window(fetch(0));
        ahead = fetch(14);
        locate(0);
        load_scales(0);
        if constexpr (CODES) {
#pragma unroll
            for (int u = 0; u < LV; ++u) load_k(u);
#pragma unroll
            for (int u = 0; u < LV; ++u) load_v(u);
#pragma unroll
            for (int u = 0; u < LV; ++u) store_k(u, 0);
            store_scales(0);
            if (steps > 1) {
                locate(1);
                load_scales(1);
#pragma unroll
                for (int u = 0; u < LV; ++u) load_k(u);
            }
        } else {
            send_k(0);
            send(-1);
        }
    }
    if constexpr (DIRECT) __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
    lds_barrier();
    if (GROUPS == 2 && grp == 1) lds_barrier();   // half a step behind
    // the steps that this wave's rows see anything of; it takes part in the others' staging and barriers
    const int mine = min(steps, max(0, (wave_top - from - grp * kManyTokens + GROUPS * kManyTokens - 1) / (GROUPS * kManyTokens)));
    const std::true_type yes;
    const std::false_type no;
    int j = 0;
    if (mine > 0) {
        {
            f16 s[2];
            matrix(0, yes, no, s);
            lds_barrier();
            send(0);
            softmax(0, s);
            arrive(0);
            lds_barrier();
        }
#pragma unroll 1
        for (j = 1; j < mine; ++j) {
            f16 s[2];
            __builtin_amdgcn_s_setprio(2);   // (ahead of the other group's wave, which has more to choose from)
            matrix(j, yes, yes, s);
            __builtin_amdgcn_s_setprio(0);
            lds_barrier();
            send(j);
            softmax(j, s);
            arrive(j);
            lds_barrier();
        }
        matrix(j, no, yes, nullptr);
        lds_barrier();
        send(j);
        arrive(j++);
        lds_barrier();
    }
#pragma unroll 1
    for (; j <= rounds; ++j) {
        matrix(j, no, no, nullptr);
        lds_barrier();
        send(j);
        arrive(j);
        lds_barrier();
    }
    if (GROUPS == 2 && grp == 0) lds_barrier();   // (as many as the other group's)

    l += __shfl_xor(l, 32, 64);
    if constexpr (GROUPS == 2) {   // the second group's sums into the first's, lane by lane
        f4* const so = reinterpret_cast<f4*>(lds) + (wave * DT * 4) * 64 + lane;
        if (grp == 1) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) so[(d * 4 + e) * 64] = f4{o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
            if (hh == 0) s_ml[32 * wave + n32] = float2{m, l};
        }
        lds_barrier();
        if (grp == 0) {
            const float2 other = s_ml[32 * wave + n32];
            const float both = fmaxf(m, other.x), f0 = __builtin_amdgcn_exp2f(m - both), f1 = __builtin_amdgcn_exp2f(other.x - both);
            m = both;
            l = l * f0 + other.y * f1;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f4 v = so[(d * 4 + e) * 64];
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[d][4 * e + r] = fmaf(o[d][4 * e + r], f0, v[r] * f1);
                }
        }
    }
    if (grp == 0 && R < nrows) {
        const int64_t yrow = (int64_t)(sq.first + tok) * a.heads_q + hq;
        const float inv = l == 0.0f ? 1.0f : 1.0f / l, otherwise = nparts == 1 && l == 0.0f ? without_weight(a, sq, seq, tok) : 0.0f;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = 32 * d + 8 * e + 4 * hh;
                if (DP != D && at >= D) continue;
                f4 v = {o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
                if (nparts > 1) {
                    *reinterpret_cast<f4*>(a.many_o + (a.many_part(yrow) + part) * D + at) = v;
                } else {
                    if (l == 0.0f) v = f4{} + otherwise;
                    *reinterpret_cast<uint2*>(a.y + yrow * D + at) = uint2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
                }
            }
        if (nparts > 1 && hh == 0) a.many_ml[a.many_part(yrow) + part] = float2{m, l};
    }
    if constexpr (!CODES) {
        if (s_odd.any()) add_not_finite(a, sq, seq, head, R0, min(nrows, R0 + kManyRows), s_odd.first, s_odd.last, [&](int, int64_t yrow) { return nparts > 1 ? a.many_o + (a.many_part(yrow) + part) * D : nullptr; });
    }
}

// ---- kernels and launches (one file per head size) ---------------------------------------------------
template <int DP, bool CODES, int NR>
__global__ __launch_bounds__(256) void attn_few_kernel(AttnArgs a)
{
    __shared__ __align__(16) uint16_t lds[kFewLds<DP, 4>];
    attn_few<DP, CODES, NR, 4>(a, lds, blockIdx.x, blockIdx.y, blockIdx.z);
}
template <int DP, bool CODES, int GROUPS>
__global__ __launch_bounds__(256 * GROUPS, GROUPS) void attn_many_kernel(AttnArgs a)
{
    __shared__ __align__(16) uint16_t lds[kManyLds<DP, CODES, GROUPS>];
    attn_many<DP, CODES, GROUPS>(a, lds, blockIdx.x, blockIdx.y);
}
// Prompts beside single tokens: the workgroups of both parts in one launch, the longer ones (of many rows) first; one after the
// other they would each leave the chip half empty (a chunk of 333 tokens and eight decoding requests: 24 us together, 24 + 9 in two launches).
template <int DP, bool CODES>
__global__ __launch_bounds__(512, 2) void attn_both_kernel(AttnArgs a)
{
    __shared__ __align__(16) uint16_t lds[kManyLds<DP, CODES, 2> > kFewLds<DP, 8> ? kManyLds<DP, CODES, 2> : kFewLds<DP, 8>];
    const unsigned many = a.many_wgs * a.many_parts;
    if (blockIdx.x < many) {
        attn_many<DP, CODES, 2>(a, lds, blockIdx.x % a.many_wgs, blockIdx.x / a.many_wgs);
    } else {
        const unsigned i = blockIdx.x - many, pair = i / a.few_parts;
        attn_few<DP, CODES, 1, 8>(a, lds, pair % a.c.heads, pair / a.c.heads, i % a.few_parts);
    }
}

template <int DP>
void launch_attn_few(const AttnArgs& a, int nr, hipStream_t s);
template <int DP>
void launch_attn_many(const AttnArgs& a, hipStream_t s);
template <int DP>
void launch_attn_both(const AttnArgs& a, hipStream_t s);   // up to 128 columns, one tile of few rows

#define ABQ_ATTN_INSTANTIATE(DP)                                                                                     \
    namespace abq {                                                                                                  \
    template <>                                                                                                      \
    void launch_attn_few<DP>(const AttnArgs& a, int nr, hipStream_t s)                                               \
    {                                                                                                                \
        const dim3 grid(a.c.heads, a.b.seqs, a.few_parts);                                                           \
        if (a.c.kv_bits == 8) {                                                                                      \
            if (nr == 1) attn_few_kernel<DP, true, 1><<<grid, 256, 0, s>>>(a);                                       \
            else attn_few_kernel<DP, true, 2><<<grid, 256, 0, s>>>(a);                                               \
        } else {                                                                                                     \
            if (nr == 1) attn_few_kernel<DP, false, 1><<<grid, 256, 0, s>>>(a);                                      \
            else attn_few_kernel<DP, false, 2><<<grid, 256, 0, s>>>(a);                                              \
        }                                                                                                            \
    }                                                                                                                \
    template <>                                                                                                      \
    void launch_attn_many<DP>(const AttnArgs& a, hipStream_t s)                                                      \
    {                                                                                                                \
        constexpr int G = DP > 128 ? 1 : 2; /* (two groups of the widest heads run out of registers) */                 \
        const dim3 grid(a.many_wgs, a.many_parts);                                                                   \
        if (a.c.kv_bits == 8) attn_many_kernel<DP, true, G><<<grid, 256 * G, 0, s>>>(a);                             \
        else attn_many_kernel<DP, false, G><<<grid, 256 * G, 0, s>>>(a);                                             \
    }                                                                                                                \
    }
#define ABQ_ATTN_INSTANTIATE_BOTH(DP)                                                                                \
    namespace abq {                                                                                                  \
    template <>                                                                                                      \
    void launch_attn_both<DP>(const AttnArgs& a, hipStream_t s)                                                      \
    {                                                                                                                \
        const dim3 grid(a.many_wgs * a.many_parts + (unsigned)a.c.heads * a.b.seqs * a.few_parts);                   \
        if (a.c.kv_bits == 8) attn_both_kernel<DP, true><<<grid, 512, 0, s>>>(a);                                    \
        else attn_both_kernel<DP, false><<<grid, 512, 0, s>>>(a);                                                    \
    }                                                                                                                \
    }

}  // namespace abq
