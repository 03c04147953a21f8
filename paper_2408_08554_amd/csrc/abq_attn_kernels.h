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
#pragma once
#include "abq_kv.h"

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
constexpr int kFewLeast = 256, kManyLeast = 512;   // tokens of a part at least, where a sequence is shared out

struct AttnArgs {
    abq_kv_cache c;
    abq_batch b;
    int heads_q, group, page_shift;
    const uint16_t* q;
    int ldq;
    float scale2;        // scale * log2 e
    bool causal;
    uint16_t* y;
    float* part_o;       // [rows][heads_q][parts][head_dim], not yet divided by the sum
    float2* part_ml;     // [rows][heads_q][parts]: (m, sum)
    int parts;           // places per row and head there
    int few, few_parts;  // sequences of up to `few` rows (tokens * group) go to the kernel for few rows, in so many parts at most
    int many_parts;
};

// A sequence's rows and tokens within all bounds.
struct Sequence {
    int first, tokens, before, length;   // first row; new tokens that are handled; position of the first; tokens held
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

// Tokens of one part of `top` when up to `parts` share them, in whole steps; the number of parts is then what covers top.
__host__ __device__ __forceinline__ int part_tokens(int top, int parts, int step, int least)
{
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
// there, and the tokens that hold one are kept track of ...
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
__device__ __forceinline__ void add_not_finite(const AttnArgs& a, const Sequence& sq, int seq, int head, int R0, int R1, int first, int last, int part, int nparts)
{
    __syncthreads();
    const int D = a.c.head_dim;
    for (int i = threadIdx.x; i < (R1 - R0) * D; i += 256) {
        const int R = R0 + i / D, d = i % D, end = min(last + 1, sq.seen(R / a.group, a.causal));
        float x = 0.0f;
        for (int t = first; t < end; ++t) {
            const int page = page_of(a.b, a.c, a.page_shift, seq, t);
            if (page >= 0) x += only_not_finite((const uint16_t*)a.c.v + vector_of(a.c, page, head, t & (a.c.page_size - 1)) * D + d);
        }
        if (x == 0.0f) continue;
        const int64_t yrow = (int64_t)(sq.first + R / a.group) * a.heads_q + head * a.group + R % a.group;
        if (nparts > 1) {
            a.part_o[(yrow * a.parts + part) * D + d] += x;
        } else {
            uint16_t* const y = a.y + yrow * D + d;
            *y = __half_as_ushort(__float2half_rn(__half2float(__ushort_as_half(*y)) + x));
        }
    }
}

constexpr float kFloor = -1e30f;   // m of a row that has seen nothing: any score passes it, and 2^(floor - m) is 0

// ---- few rows ------------------------------------------------------------------------------------
// One workgroup per sequence, key head and part of the tokens; NR tiles of sixteen rows (token * group + query head).  Its
// four waves take 32 tokens in turn, each with a maximum, sums and an LDS region of its own (no barrier in the loop), and are
// joined at the end.  K goes from memory straight into the matrix operand's registers, V through LDS for the transposition.
// What bounds it: memory.  A wave has 16 KB in flight (32 tokens of K and V, 128 halves each) from the moment it has used the
// last ones, and three or four workgroups share a compute unit.
template <int DP, bool CODES, int NR>
__global__ __launch_bounds__(256) void attn_few_kernel(AttnArgs a)
{
    constexpr int DT = DP / 16;                      // tiles of sixteen columns
    constexpr int QS = DP / 32;                      // steps of the first product
    constexpr int KV = CODES ? DP / 64 : DP / 32;    // 16-byte loads of a lane per sixteen tokens of K
    constexpr int LPT = CODES ? DP / 16 : DP / 8;    // lanes that hold a token of V
    constexpr int TPL = 64 / LPT;                    // tokens of V per load of a wave
    constexpr int VV = kFewTokens / TPL;             // 16-byte loads of a lane per step's V
    constexpr int VS = DP + 16;                      // halves of a row of V in LDS: eight banks on, sixteen lanes of a transposing read take all
    constexpr int OS = DP + 4;                       // floats of a row when the waves are joined
    __shared__ __align__(16) uint16_t lds[4 * kFewTokens * VS];
    __shared__ float2 s_ml[4][16];
    __shared__ OddTokens s_odd;
    static_assert(sizeof(lds) >= 4 * 16 * OS * sizeof(float), "the waves are joined in the memory of V");

    const int head = blockIdx.x, seq = blockIdx.y, part = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
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
        const int t = from + ((i + (lane >> 1)) * 4 + wave) * kFewTokens + 16 * (lane & 1);
        table = t < to ? page_of(a.b, a.c, a.page_shift, seq, t) : -1;
    };
    int pg[2];   // (of the step that is loaded)
    auto load = [&](int i) {
        if (i - pages_at >= 32) fetch_pages(i);
        const int t0 = from + (i * 4 + wave) * kFewTokens;
        int64_t vec[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            pg[j] = __builtin_amdgcn_readlane(table, 2 * (i - pages_at) + j);
            vec[j] = vector_of(a.c, max(pg[j], 0), head, (t0 + 16 * j) & (a.c.page_size - 1));   // (no page: the first one's, masked)
#pragma unroll
            for (int u = 0; u < KV; ++u) {
                int d = CODES ? 64 * u + 16 * g : 32 * u + 8 * g;
                if (d >= D) d = 0;   // (the queries are zero there)
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

    const int steps = to > from + wave * kFewTokens ? (to - from - wave * kFewTokens + 4 * kFewTokens - 1) / (4 * kFewTokens) : 0;
    if (steps) {
        fetch_pages(0);
        load(0);
    }
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        const int t0 = from + (i * 4 + wave) * kFewTokens;
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
                if (masked && drop_not_finite(v)) s_odd.found(t0 + u * TPL + lane / LPT, to);
                *reinterpret_cast<u4*>(dst) = v;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (other lanes' rows are read below)
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
            if (any(lm > m[t] + 8.0f)) {
                lm = fmaxf(lm, __shfl_xor(lm, 16, 64));
                lm = fmaxf(fmaxf(lm, __shfl_xor(lm, 32, 64)), m[t]);
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
            const uint16_t* src = lv + (4 * g + (n16 >> 2)) * VS + 4 * (n16 & 3);
#pragma unroll
            for (int d = 0; d < DT; ++d)
                o[t][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(read_transposed(src + 16 * d), read_transposed(src + 16 * VS + 16 * d)), p, o[t][d], 0, 0, 0);
        }
    }

    // the four waves' sums as one, a tile of rows at a time
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
        const int r = tid >> 4, R = 16 * t + r;
        if (R < nrows) {
            float top_m = kFloor, sum = 0.0f, f[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) top_m = fmaxf(top_m, s_ml[w][r].x);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f[w] = __builtin_amdgcn_exp2f(s_ml[w][r].x - top_m);
                sum += f[w] * s_ml[w][r].y;
            }
            const int64_t yrow = (int64_t)(sq.first + R / a.group) * a.heads_q + head * a.group + R % a.group;
            for (int d = 4 * (tid & 15); d < D; d += 64) {
                f4 v = {0, 0, 0, 0};
#pragma unroll
                for (int w = 0; w < 4; ++w) v += f[w] * *reinterpret_cast<const f4*>(so + (w * 16 + r) * OS + d);
                if (nparts > 1) {
                    *reinterpret_cast<f4*>(a.part_o + (yrow * a.parts + part) * D + d) = v;
                } else {
                    const float inv_sum = sum == 0.0f ? 0.0f : 1.0f / sum;
                    if (sum == 0.0f) v = f4{0, 0, 0, 0};
                    *reinterpret_cast<uint2*>(a.y + yrow * D + d) = uint2{pack2(v[0] * inv_sum, v[1] * inv_sum), pack2(v[2] * inv_sum, v[3] * inv_sum)};
                }
            }
            if (nparts > 1 && (tid & 15) == 0) a.part_ml[yrow * a.parts + part] = float2{top_m, sum};
        }
    }
    if constexpr (!CODES) {
        if (s_odd.any()) add_not_finite(a, sq, seq, head, 0, nrows, s_odd.first, s_odd.last, part, nparts);
    }
}

// ---- many rows -----------------------------------------------------------------------------------
// The sequence and tile of a workgroup: tiles of the sequences with more than `few` rows, in order; within a sequence the last
// tile (the longest under the causal mask) first.  false: there is none.
__device__ __forceinline__ bool many_tile(const AttnArgs& a, int index, int* seq, int* tile)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.b.seqs; s0 += 64) {
        int nt = 0;
        if (s0 + lane < a.b.seqs) {
            const int nrows = Sequence(a, s0 + lane).tokens * a.group;
            nt = nrows > a.few ? (nrows + kManyRows - 1) / kManyRows : 0;
        }
        int sum = nt;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int up = __shfl_up(sum, off, 64);
            if (lane >= off) sum += up;
        }
        const uint64_t past = __ballot(sum > index);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            *seq = s0 + at;
            *tile = __shfl(sum, at, 64) - 1 - index;
            return true;
        }
        index -= __shfl(sum, 63, 64);
    }
    return false;
}

// One workgroup per key head, 128 rows (token * group + query head) and part of the tokens: four waves of 32 rows, which share 64
// tokens of K and V at a time in LDS, two buffers, one barrier a step; the next step's loads are in flight meanwhile.
template <int DP, bool CODES>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void attn_many_kernel(AttnArgs a)
{
    constexpr int DT = DP / 32;                       // tiles of 32 columns of the result
    constexpr int QS = DP / 16;                       // steps of the first product
    constexpr int LPT = CODES ? DP / 16 : DP / 8;     // lanes that hold a token
    constexpr int TPP = 256 / LPT;                    // tokens per load of the workgroup
    constexpr int LV = kManyTokens / TPP;             // 16-byte loads of a thread per step, of K and of V
    constexpr int KS = DP + 8, VS = DP + 32;          // halves of a row in LDS: 4 banks on for the reads of K, 16 for the transposing ones of V
    constexpr int NB = DP > 128 ? 1 : 2;              // buffers
    __shared__ __align__(16) uint16_t lk[NB][kManyTokens * KS], lv[NB][kManyTokens * VS];
    __shared__ __align__(16) float s_ks[CODES ? NB : 1][kManyTokens], s_lg[CODES ? NB : 1][kManyTokens], s_inv[CODES ? NB : 1][kManyTokens];
    __shared__ OddTokens s_odd;

    const int head = blockIdx.x % a.c.heads, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n32 = lane & 31, hh = lane >> 5, D = a.c.head_dim;
    int seq, tile;
    if (!many_tile(a, blockIdx.x / a.c.heads, &seq, &tile)) return;
    seq = __builtin_amdgcn_readfirstlane(seq);
    tile = __builtin_amdgcn_readfirstlane(tile);
    const Sequence sq(a, seq);
    const int nrows = sq.tokens * a.group, R0 = tile * kManyRows;
    const int top = sq.seen((min(nrows, R0 + kManyRows) - 1) / a.group, a.causal);
    const int per = part_tokens(top, a.many_parts, kManyTokens, kManyLeast), nparts = max(1, (top + per - 1) / per), part = blockIdx.y;
    if (part >= nparts) return;
    const int from = part * per, to = min(top, from + per), steps = (to - from + kManyTokens - 1) / kManyTokens;

    // this lane's row, and what the wave's rows see at least and at most
    const int W0 = R0 + 32 * wave, R = W0 + n32, tok = R / a.group, hq = head * a.group + R % a.group;
    const int vis = R < nrows ? sq.seen(tok, a.causal) : 0;
    const int wave_least = W0 < nrows ? sq.seen(W0 / a.group, a.causal) : 0, wave_top = W0 < nrows ? sq.seen((min(nrows, W0 + 32) - 1) / a.group, a.causal) : 0;
    h8 qv[QS];
    {
        const uint16_t* row = a.q + (size_t)(sq.first + (R < nrows ? tok : 0)) * a.ldq + (size_t)hq * D;
#pragma unroll
        for (int s = 0; s < QS; ++s) {
            u4 v = {0, 0, 0, 0};
            if (R < nrows && 16 * s + 8 * hh < D) v = *reinterpret_cast<const u4*>(row + 16 * s + 8 * hh);
            qv[s] = __builtin_bit_cast(h8, v);
        }
    }
    f16 o[DT];
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = f16{};
    float m = kFloor, l = 0.0f;

    u4 kr[LV], vr[LV];
    uint32_t kz[LV], vz[LV];
    float t_ks = 0.0f, t_vs = 1.0f;   // codes: scales of token tid of the step (threads 0..63)
    int pages_at = 0, table = -1;     // the pages of the next 16 steps, four to a step
    auto fetch_pages = [&](int i) {
        pages_at = i;
        const int t = from + i * kManyTokens + 16 * lane;
        table = t < to ? page_of(a.b, a.c, a.page_shift, seq, t) : -1;
    };
    auto page_at = [&](int i, int sixteenth) { return __builtin_amdgcn_readlane(table, 4 * (i - pages_at) + sixteenth); };
    unsigned gone_next = 0;           // sixteens of the loaded step that have no page
    auto load = [&](int i) {
        if (i - pages_at >= 16) fetch_pages(i);
        const int t0 = from + i * kManyTokens;
        gone_next = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) gone_next |= (page_at(i, j) < 0 ? 1u : 0u) << j;
#pragma unroll
        for (int u = 0; u < LV; ++u) {
            int d = (tid % LPT) * (CODES ? 16 : 8);
            if (d >= D) d = 0;   // (the queries are zero there, and the columns of V are not stored)
            const int sixteenth = __builtin_amdgcn_readfirstlane((u * TPP + (wave * 64) / LPT) >> 4);   // (a wave's tokens of one load lie in one)
            const int page = page_at(i, sixteenth);
            const int64_t at = vector_of(a.c, max(page, 0), head, (t0 + u * TPP + tid / LPT) & (a.c.page_size - 1));   // (no page: the first one's, masked)
            kr[u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.k + (at * D + d) * (CODES ? 1 : 2));
            vr[u] = *reinterpret_cast<const u4*>((const uint8_t*)a.c.v + (at * D + d) * (CODES ? 1 : 2));
            if constexpr (CODES) {
                kz[u] = a.c.k_zero[at];
                vz[u] = a.c.v_zero[at];
            }
        }
        if constexpr (CODES) {
            if (wave == 0) {
                int page = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int pj = page_at(i, j);
                    if ((lane >> 4) == j) page = pj;
                }
                t_ks = 0.0f;
                t_vs = 1.0f;
                if (t0 + lane < to && page >= 0) {
                    const int64_t at = vector_of(a.c, page, head, (t0 + lane) & (a.c.page_size - 1));
                    t_ks = a.c.k_scale[at];
                    t_vs = a.c.v_scale[at];
                }
            }
        }
    };
    const int tile_least = sq.seen(R0 / a.group, a.causal);
    auto store = [&](int i) {   // what load(i) has brought, to its buffer
        const int buf = NB == 2 ? i & 1 : 0;
        const bool masked = from + (i + 1) * kManyTokens > tile_least || gone_next != 0;
#pragma unroll
        for (int u = 0; u < LV; ++u) {
            const int t = u * TPP + tid / LPT, d = (tid % LPT) * (CODES ? 16 : 8);
            uint16_t *dk = lk[buf] + t * KS + d, *dv = lv[buf] + t * VS + d;
            if constexpr (CODES) {
                const h2 kb = code_bias((int)kz[u]), vb = code_bias((int)vz[u]);
                uint32_t w[8];
#pragma unroll
                for (int j = 0; j < 4; ++j) codes_to_halves(kr[u][j], kb, w + 2 * j);
                *reinterpret_cast<u4*>(dk) = u4{w[0], w[1], w[2], w[3]};
                *reinterpret_cast<u4*>(dk + 8) = u4{w[4], w[5], w[6], w[7]};
#pragma unroll
                for (int j = 0; j < 4; ++j) codes_to_halves(vr[u][j], vb, w + 2 * j);
                *reinterpret_cast<u4*>(dv) = u4{w[0], w[1], w[2], w[3]};
                *reinterpret_cast<u4*>(dv + 8) = u4{w[4], w[5], w[6], w[7]};
            } else {
                u4 v = vr[u];
                if (masked && drop_not_finite(v)) s_odd.found(from + i * kManyTokens + t, to);
                *reinterpret_cast<u4*>(dk) = kr[u];
                *reinterpret_cast<u4*>(dv) = v;
            }
        }
        if constexpr (CODES) {
            if (wave == 0) {
                s_ks[buf][lane] = t_ks * a.scale2;
                s_lg[buf][lane] = __builtin_amdgcn_logf(t_vs);
                s_inv[buf][lane] = __builtin_amdgcn_rcpf(t_vs);
            }
        }
    };

    if (tid == 0) s_odd.clear();
    if (steps) {
        fetch_pages(0);
        load(0);
    }
    __syncthreads();
    unsigned gone = gone_next;
    if (steps) store(0);
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < steps; ++i) {
        const int t0 = from + i * kManyTokens, buf = NB == 2 ? i & 1 : 0;
        if (i + 1 < steps) load(i + 1);
        if (t0 < wave_top) {
            const bool masked = t0 + kManyTokens > wave_least || gone != 0;
            f16 s[2] = {f16{}, f16{}};
#pragma unroll
            for (int st = 0; st < QS; ++st)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const u4 kv = *reinterpret_cast<const u4*>(lk[buf] + (32 * kt + n32) * KS + 16 * st + 8 * hh);
                    s[kt] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, kv), qv[st], s[kt], 0, 0, 0);
                }
            if constexpr (CODES) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f4 c = *reinterpret_cast<const f4*>(&s_ks[buf][32 * kt + 8 * e + 4 * hh]), lg = *reinterpret_cast<const f4*>(&s_lg[buf][32 * kt + 8 * e + 4 * hh]);
#pragma unroll
                        for (int r = 0; r < 4; ++r) s[kt][4 * e + r] = fmaf(s[kt][4 * e + r], c[r], lg[r]);
                    }
            } else {
                s[0] *= a.scale2;
                s[1] *= a.scale2;
            }
            if (masked) {
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int t = 32 * kt + 8 * (e >> 2) + 4 * hh + (e & 3);
                        if (t0 + t >= vis || (gone >> (2 * kt + (e >> 3)) & 1u)) s[kt][e] = -INFINITY;
                    }
            }
            float lm = s[0][0];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 16; ++e) lm = fmaxf(lm, s[kt][e]);
            if (any(lm > m + 8.0f)) {
                lm = fmaxf(fmaxf(lm, __shfl_xor(lm, 32, 64)), m);
                const float fade = __builtin_amdgcn_exp2f(m - lm);
                m = lm;
                l *= fade;
#pragma unroll
                for (int d = 0; d < DT; ++d) o[d] *= fade;
            }
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f4 inv = {1, 1, 1, 1};
                    if constexpr (CODES) inv = *reinterpret_cast<const f4*>(&s_inv[buf][32 * kt + 8 * e + 4 * hh]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float w = __builtin_amdgcn_exp2f(s[kt][4 * e + r] - m);
                        s[kt][4 * e + r] = w;
                        if constexpr (CODES) l += w != 0.0f || !masked ? w * inv[r] : 0.0f;   // (a masked token's scale may be anything)
                        else l += w;
                    }
                }
            const uint16_t* const src = lv[buf] + (4 * hh + ((lane & 15) >> 2)) * VS + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                u4 pw;
#pragma unroll
                for (int e = 0; e < 4; ++e) pw[e] = pack2(s[c >> 1][8 * (c & 1) + 2 * e], s[c >> 1][8 * (c & 1) + 2 * e + 1]);
                const h8 p = __builtin_bit_cast(h8, pw);
#pragma unroll
                for (int d = 0; d < DT; ++d) {
                    const h8 v = join(read_transposed(src + 16 * c * VS + 32 * d), read_transposed(src + (16 * c + 8) * VS + 32 * d));
                    o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p, o[d], 0, 0, 0);
                }
            }
        }
        if constexpr (NB == 1) __syncthreads();
        if (i + 1 < steps) store(i + 1);
        gone = gone_next;
        __syncthreads();
    }

    l += __shfl_xor(l, 32, 64);
    if (R < nrows) {
        const int64_t yrow = (int64_t)(sq.first + tok) * a.heads_q + hq;
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = 32 * d + 8 * e + 4 * hh;
                if (DP != D && at >= D) continue;
                f4 v = {o[d][4 * e], o[d][4 * e + 1], o[d][4 * e + 2], o[d][4 * e + 3]};
                if (nparts > 1) {
                    *reinterpret_cast<f4*>(a.part_o + (yrow * a.parts + part) * D + at) = v;
                } else {
                    if (l == 0.0f) v = f4{0, 0, 0, 0};
                    *reinterpret_cast<uint2*>(a.y + yrow * D + at) = uint2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
                }
            }
        if (nparts > 1 && hh == 0) a.part_ml[yrow * a.parts + part] = float2{m, l};
    }
    if constexpr (!CODES) {
        if (s_odd.any()) add_not_finite(a, sq, seq, head, R0, min(nrows, R0 + kManyRows), s_odd.first, s_odd.last, part, nparts);
    }
}

// ---- launches (one file per head size) --------------------------------------------------------------
template <int DP>
void launch_attn_few(const AttnArgs& a, int nr, const dim3& grid, hipStream_t s);
template <int DP>
void launch_attn_many(const AttnArgs& a, const dim3& grid, hipStream_t s);

#define ABQ_ATTN_INSTANTIATE(DP)                                                                                     \
    namespace abq {                                                                                                  \
    template <>                                                                                                      \
    void launch_attn_few<DP>(const AttnArgs& a, int nr, const dim3& grid, hipStream_t s)                             \
    {                                                                                                                \
        if (a.c.kv_bits == 8) {                                                                                      \
            if (nr == 1) attn_few_kernel<DP, true, 1><<<grid, 256, 0, s>>>(a);                                       \
            else attn_few_kernel<DP, true, 2><<<grid, 256, 0, s>>>(a);                                               \
        } else {                                                                                                     \
            if (nr == 1) attn_few_kernel<DP, false, 1><<<grid, 256, 0, s>>>(a);                                      \
            else attn_few_kernel<DP, false, 2><<<grid, 256, 0, s>>>(a);                                              \
        }                                                                                                            \
    }                                                                                                                \
    template <>                                                                                                      \
    void launch_attn_many<DP>(const AttnArgs& a, const dim3& grid, hipStream_t s)                                    \
    {                                                                                                                \
        if (a.c.kv_bits == 8) attn_many_kernel<DP, true><<<grid, 256, 0, s>>>(a);                                    \
        else attn_many_kernel<DP, false><<<grid, 256, 0, s>>>(a);                                                    \
    }                                                                                                                \
    }

}  // namespace abq
