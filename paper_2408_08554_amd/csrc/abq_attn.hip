// Attention of a step's rows over the paged cache: which kernel takes a sequence, how its tokens are shared out, and the joining
// of the parts.
#include "abq_attn_kernels.h"

#include <algorithm>

namespace abq {

template <>
void launch_attn_few<64>(const AttnArgs&, int, hipStream_t);
template <>
void launch_attn_many<64>(const AttnArgs&, hipStream_t);
template <>
void launch_attn_few<128>(const AttnArgs&, int, hipStream_t);
template <>
void launch_attn_many<128>(const AttnArgs&, hipStream_t);
template <>
void launch_attn_few<256>(const AttnArgs&, int, hipStream_t);
template <>
void launch_attn_many<256>(const AttnArgs&, hipStream_t);
template <>
void launch_attn_both<64>(const AttnArgs&, hipStream_t);
template <>
void launch_attn_both<128>(const AttnArgs&, hipStream_t);

// The parts of a row and head that was shared out as one.  What bounds it is latency (sequence, maxima and sums, parts: three
// dependent loads).  LP lanes take a row and head, four columns each, and hold its parts' maxima and sums, one each.  WAVES = 4:
// many parts, which the waves of a workgroup take in turn, four at a time; else a workgroup has 256 / LP heads, and a wave one of
// up to 64 / LP of them.  (341 rows, 32 heads of 128 in up to two parts: 5.9 us, 9.4 with a wave for each head.)
template <int WAVES, int LP>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    static_assert(WAVES == 1 || LP == 64);
    __shared__ __align__(16) f4 s_o[WAVES][64];
    const int lane = threadIdx.x & 63, wave = WAVES == 4 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0, D = a.c.head_dim;
    const int sl = lane & (LP - 1), group0 = lane & ~(LP - 1);
    const int row = blockIdx.x, hq = WAVES == 4 ? blockIdx.y : blockIdx.y * (256 / LP) + threadIdx.x / LP;
    int seq = 0;
    for (int s0 = 0; s0 < a.b.seqs; s0 += 64) {
        const int s = s0 + lane;
        seq += __popcll(__ballot(s < a.b.seqs && a.b.row_start[s + 1] <= row));
    }
    if (seq >= a.b.seqs) return;
    const Sequence sq(a, seq);
    const int i = row - sq.first;
    if (i < 0 || i >= sq.tokens) return;
    const int nrows = sq.tokens * a.group;
    const bool few = nrows <= a.few;
    const int last = few ? nrows : min(nrows, ((i * a.group + hq % a.group) / kManyRows + 1) * kManyRows);
    const int top = sq.seen((last - 1) / a.group, a.causal);
    const int per = few ? part_tokens(top, a.few_parts, kFewTokens, kFewLeast) : part_tokens(top, a.many_parts, kManyTokens, kManyLeast);
    int nparts = (top + per - 1) / per;
    if (nparts <= 1 || hq >= a.heads_q) nparts = 0;   // (written by its workgroup)
    if (!any(nparts != 0)) return;
    const int64_t yrow = (int64_t)row * a.heads_q + hq;
    const int64_t place = few ? a.few_part(seq, hq / a.group, i * a.group + hq % a.group) : a.many_part(yrow);
    const float* const o = (few ? a.few_o : a.many_o) + place * D + 4 * sl;
    const float2 ml = sl < nparts ? (few ? a.few_ml : a.many_ml)[place + sl] : float2{kFloor, 0.0f};
    const bool mine = 4 * sl < D;
    // this wave's parts: its first four are on their way before their weights are known
    f4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = mine && wave + WAVES * u < nparts ? *reinterpret_cast<const f4*>(o + (int64_t)(wave + WAVES * u) * D) : f4{0, 0, 0, 0};
    float m = ml.x;
#pragma unroll
    for (int off = LP / 2; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    float l = f * ml.y;
#pragma unroll
    for (int off = LP / 2; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
    f4 v = {0, 0, 0, 0};
    for (int p0 = wave; any(p0 < nparts); p0 += 4 * WAVES) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float w = __shfl(f, (group0 + p0 + WAVES * u) & 63, 64);
            if (p0 + WAVES * u < nparts) v += w * x[u];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (mine && p0 + WAVES * (4 + u) < nparts) x[u] = *reinterpret_cast<const f4*>(o + (int64_t)(p0 + WAVES * (4 + u)) * D);
    }
    if constexpr (WAVES == 4) {
        s_o[wave][lane] = v;
        __syncthreads();
        if (wave != 0) return;
        v = s_o[0][lane] + s_o[1][lane] + (s_o[2][lane] + s_o[3][lane]);
    }
    if (!mine || nparts == 0) return;
    const float inv = l == 0.0f ? 1.0f : 1.0f / l;
    if (l == 0.0f) v = f4{} + without_weight(a, sq, seq, i);
    *reinterpret_cast<uint2*>(a.y + yrow * D + 4 * sl) = uint2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
}

// Which kernels a step needs, and into how many parts sequences are cut at most; from the sizes that the host knows alone, so that a
// captured launch serves whatever lengths the arrays hold later.
struct AttnPlan {
    int nr, few, few_parts, few_rows, many_parts;
    int64_t many_wgs;
    bool both;   // one launch for the two parts
    size_t few_places, many_places;   // of results of parts
};
static AttnPlan attn_plan(const abq_kv_cache& c, const abq_batch& b, int heads_q)
{
    AttnPlan p{};
    const int group = heads_q / c.heads;
    const int64_t most = (int64_t)b.max_new * group, all = (int64_t)b.rows * group;
    // Up to 32 rows of a sequence belong to the part for few rows; beside longer ones up to sixteen, so that one launch can take both.
    // (24 rows each, 16 sequences of 1000, 4 heads: 16 us there, 22 as many rows; a group of 32, four of 1000: 14 and 20, and 32 of 2000
    // 20.5 and 21.  33 requests, one of them a prompt of 100 tokens: 26 us in one launch, 46 as 32 rows and two launches.)
    p.nr = most <= 16 || (group <= 16 && most > 32) ? 1 : 2;
    p.few = group <= 32 && (b.seqs > 1 || most <= 32) ? 16 * p.nr : 0;
    p.few_rows = (int)std::min<int64_t>(p.few, most);
    p.both = p.few && most > p.few && p.nr == 1 && c.head_dim <= 128;
    const int tokens = (int)std::min<int64_t>(b.max_len, (int64_t)b.max_pages * c.page_size);
    p.few_parts = p.many_parts = 1;
    // Parts until each compute unit has a workgroup (of codes two, which have half the bytes in flight); beside prompts half of them
    // have one.  More parts balance better but have to be joined.  us, heads of 128, n sequences of two thirds of L to L tokens on h key heads:
    //   binary16, at 128, 256, 512 workgroups: 4 of 32000 on 8 106, 90, 89; 4 of 8000 on 8 29, 28, 26; 16 of 1000 on 8 17, 18, 18; 32 of 2000 on
    //     8 38, 38, 42; 8 of 2000 on 32 38, 38, 42; 8 of 8000 on 32 162, 162, 167
    //   codes, at 256, 512, 1024: 4 of 32000 on 8 54, 47, 48; 4 of 8000 on 8 23, 20, 22; 1 of 32000 on 32 56, 50, 52; 8 of 2000 on 8 15.0,
    //     15.5, 15.3; 32 of 2000 on 8 27, 28, 29; 8 of 2000 on 32 28, 30, 31
    //   beside a prompt's chunk of 333 over 1000, at 128, 256, 512: 8 of 1000 on 8 30, 32, 33 (codes 35, 37, 38); 2 of 4000 on 8 37, 55, 59;
    //     32 of 2000 on 32 166, 167, 166; beside a prompt of 1000: 2 of 4000 on 8 35, 67, 68; but few long ones would have more:
    //     4 of 16000 on 32 229, 193, 191
    if (p.few && !stays_whole(tokens, kFewLeast)) {
        const int64_t wgs = (int64_t)b.seqs * c.heads, want = p.both ? 128 : c.kv_bits == 8 ? 512 : 256;
        p.few_parts = (int)std::min<int64_t>({(want + wgs - 1) / wgs, (tokens + kFewLeast - 1) / kFewLeast, 64});
    }
    if (most > p.few) {   // a workgroup to a compute unit (256 tokens over 4096, 8 heads: 37 us; of two, 47)
        p.many_wgs = (all / kManyRows + std::min<int64_t>(b.seqs, all / (p.few + 1))) * c.heads;
        if (!stays_whole(tokens, kManyLeast)) p.many_parts = (int)std::min<int64_t>({(256 + p.many_wgs - 1) / p.many_wgs, (tokens + kManyLeast - 1) / kManyLeast, 32});
    }
    p.few_places = p.few_parts > 1 ? (size_t)b.seqs * c.heads * p.few_rows * p.few_parts : 0;
    p.many_places = p.many_parts > 1 ? (size_t)b.rows * heads_q * p.many_parts : 0;
    return p;
}

size_t attn_workspace_bytes(const abq_kv_cache& c, const abq_batch& b, int heads_q)
{
    const AttnPlan p = attn_plan(c, b, heads_q);
    return (p.few_places + p.many_places) * (c.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_attn_paged(const abq_kv_cache& c, const abq_batch& b, int heads_q, const uint16_t* q, int ldq, float scale, bool causal,
                             uint16_t* y, void* workspace, hipStream_t s)
{
    const AttnPlan p = attn_plan(c, b, heads_q);
    AttnArgs a{};
    a.c = c;
    a.b = b;
    a.b.max_len = std::min(b.max_len, 1 << 30);   // (steps, and windows of steps, are counted past a sequence's end in 32 bits)
    a.heads_q = heads_q;
    a.group = heads_q / c.heads;
    a.page_shift = __builtin_ctz(c.page_size);
    a.q = q;
    a.ldq = ldq;
    a.scale2 = (float)((double)scale * 1.44269504088896340736);
    a.causal = causal;
    a.y = y;
    a.few = p.few;
    a.few_parts = p.few_parts;
    a.many_parts = p.many_parts;
    a.few_rows = p.few_rows;
    a.many_wgs = (unsigned)p.many_wgs;
    a.few_o = (float*)workspace;   // (16-byte vectors first, the pairs behind them)
    a.many_o = a.few_o + p.few_places * c.head_dim;
    a.few_ml = (float2*)(a.many_o + p.many_places * c.head_dim);
    a.many_ml = a.few_ml + p.few_places;
    if (p.both) {
        c.head_dim <= 64 ? launch_attn_both<64>(a, s) : launch_attn_both<128>(a, s);
    } else {
        if (p.many_wgs) c.head_dim <= 64 ? launch_attn_many<64>(a, s) : c.head_dim <= 128 ? launch_attn_many<128>(a, s) : launch_attn_many<256>(a, s);
        if (p.few) c.head_dim <= 64 ? launch_attn_few<64>(a, p.nr, s) : c.head_dim <= 128 ? launch_attn_few<128>(a, p.nr, s) : launch_attn_few<256>(a, p.nr, s);
    }
    const int parts = std::max(p.few_parts, p.many_parts);
    // (A prompt's rows fill the chip with less than a wave for each head; where a few rows have many parts, four waves share one.  One
    // request of 32000 tokens: 44 us with one, 29 with four; a prompt of 256 over 4096 in up to eight parts: 37 and 49.)
    if (parts > 8) attn_join_kernel<4, 64><<<dim3(b.rows, heads_q), 256, 0, s>>>(a);
    else if (parts > 1 && c.head_dim <= 64) attn_join_kernel<1, 16><<<dim3(b.rows, (heads_q + 15) / 16), 256, 0, s>>>(a);
    else if (parts > 1 && c.head_dim <= 128) attn_join_kernel<1, 32><<<dim3(b.rows, (heads_q + 7) / 8), 256, 0, s>>>(a);
    else if (parts > 1) attn_join_kernel<1, 64><<<dim3(b.rows, (heads_q + 3) / 4), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace abq
