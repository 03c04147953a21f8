// Attention of a step's rows over the paged cache: which kernel takes a sequence, how its tokens are shared out, and the joining
// of the parts.
#include "abq_attn_kernels.h"

#include <algorithm>

namespace abq {

template <>
void launch_attn_few<64>(const AttnArgs&, int, const dim3&, hipStream_t);
template <>
void launch_attn_few<128>(const AttnArgs&, int, const dim3&, hipStream_t);
template <>
void launch_attn_few<256>(const AttnArgs&, int, const dim3&, hipStream_t);
template <>
void launch_attn_many<64>(const AttnArgs&, const dim3&, hipStream_t);
template <>
void launch_attn_many<128>(const AttnArgs&, const dim3&, hipStream_t);
template <>
void launch_attn_many<256>(const AttnArgs&, const dim3&, hipStream_t);

// The parts of a row and head that was shared out as one.  What bounds it is latency (sequence, maxima and sums, parts: three
// dependent loads), so WAVES waves of a workgroup take the parts in turn, four at a time (few parts: a wave for each of four heads); a
// wave holds up to 64 parts' maxima and sums in its lanes.
template <int WAVES>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    __shared__ __align__(16) f4 s_o[WAVES][64];
    const int lane = threadIdx.x & 63, nth = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = WAVES == 4 ? nth : 0, D = a.c.head_dim;
    const int row = blockIdx.x, hq = WAVES == 4 ? blockIdx.y : 4 * blockIdx.y + nth;
    if (hq >= a.heads_q) return;
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
    const int nparts = (top + per - 1) / per;
    if (nparts <= 1) return;   // (written by its workgroup)
    const int64_t yrow = (int64_t)row * a.heads_q + hq;
    const float* const o = a.part_o + yrow * a.parts * D + 4 * lane;
    const float2 ml = lane < nparts ? a.part_ml[yrow * a.parts + lane] : float2{kFloor, 0.0f};
    const bool mine = 4 * lane < D;
    // this wave's parts: its first four are on their way before their weights are known
    f4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) x[u] = mine && wave + WAVES * u < nparts ? *reinterpret_cast<const f4*>(o + (int64_t)(wave + WAVES * u) * D) : f4{0, 0, 0, 0};
    float m = ml.x;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 64));
    const float f = __builtin_amdgcn_exp2f(ml.x - m);
    float l = f * ml.y;
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
    f4 v = {0, 0, 0, 0};
    for (int p0 = wave; p0 < nparts; p0 += 4 * WAVES) {
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p0 + WAVES * u < nparts) v += __shfl(f, p0 + WAVES * u, 64) * x[u];
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
    if (!mine) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (l == 0.0f) v = f4{0, 0, 0, 0};
    *reinterpret_cast<uint2*>(a.y + yrow * D + 4 * lane) = uint2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
}

// Which kernels a step needs, and into how many parts sequences are cut at most; from the sizes that the host knows alone, so that a
// captured launch serves whatever lengths the arrays hold later.
struct AttnPlan {
    int nr, few, few_parts, many_parts, parts;
    int64_t many_tiles;
};
static AttnPlan attn_plan(const abq_kv_cache& c, const abq_batch& b, int heads_q)
{
    AttnPlan p{};
    const int group = heads_q / c.heads;
    const int64_t most = (int64_t)b.max_new * group, all = (int64_t)b.rows * group;
    p.nr = most <= 16 || (group <= 16 && most > 32) ? 1 : 2;
    p.few = group <= 32 && (b.seqs > 1 || most <= 32) ? 16 * p.nr : 0;
    const int tokens = (int)std::min<int64_t>(b.max_len, (int64_t)b.max_pages * c.page_size);
    p.few_parts = p.many_parts = 1;
    if (p.few) {
        const int64_t wgs = (int64_t)b.seqs * c.heads;
        p.few_parts = (int)std::min<int64_t>({(1024 + wgs - 1) / wgs, (tokens + kFewLeast - 1) / kFewLeast, 64});
    }
    if (most > p.few) {
        p.many_tiles = all / kManyRows + std::min<int64_t>(b.seqs, all / (p.few + 1));
        const int64_t wgs = p.many_tiles * c.heads;
        p.many_parts = (int)std::min<int64_t>({(256 + wgs - 1) / wgs, (tokens + kManyLeast - 1) / kManyLeast, 32});
    }
    p.parts = std::max(p.few_parts, p.many_parts);
    return p;
}

size_t attn_workspace_bytes(const abq_kv_cache& c, const abq_batch& b, int heads_q)
{
    const AttnPlan p = attn_plan(c, b, heads_q);
    return p.parts == 1 ? 0 : (size_t)b.rows * heads_q * p.parts * (c.head_dim * sizeof(float) + sizeof(float2));
}

hipError_t launch_attn_paged(const abq_kv_cache& c, const abq_batch& b, int heads_q, const uint16_t* q, int ldq, float scale, bool causal,
                             uint16_t* y, void* workspace, hipStream_t s)
{
    const AttnPlan p = attn_plan(c, b, heads_q);
    AttnArgs a{c, b, heads_q, heads_q / c.heads, __builtin_ctz(c.page_size), q, ldq, (float)((double)scale * 1.44269504088896340736), causal, y, nullptr, nullptr,
               p.parts, p.few, p.few_parts, p.many_parts};
    if (p.parts > 1) {
        a.part_o = (float*)workspace;
        a.part_ml = (float2*)(a.part_o + (size_t)b.rows * heads_q * p.parts * c.head_dim);
    }
    if (p.many_tiles * c.heads > INT32_MAX) return hipErrorInvalidConfiguration;
    if (p.many_tiles) {
        const dim3 grid((unsigned)(p.many_tiles * c.heads), p.many_parts);
        if (c.head_dim <= 64) launch_attn_many<64>(a, grid, s);
        else if (c.head_dim <= 128) launch_attn_many<128>(a, grid, s);
        else launch_attn_many<256>(a, grid, s);
    }
    if (p.few) {
        const dim3 grid(c.heads, b.seqs, p.few_parts);
        if (c.head_dim <= 64) launch_attn_few<64>(a, p.nr, grid, s);
        else if (c.head_dim <= 128) launch_attn_few<128>(a, p.nr, grid, s);
        else launch_attn_few<256>(a, p.nr, grid, s);
    }
    if (p.parts > 1) {
        if (p.parts > 8) attn_join_kernel<4><<<dim3(b.rows, heads_q), 256, 0, s>>>(a);
        else attn_join_kernel<1><<<dim3(b.rows, (heads_q + 3) / 4), 256, 0, s>>>(a);
    }
    return hipGetLastError();
}

}  // namespace abq
