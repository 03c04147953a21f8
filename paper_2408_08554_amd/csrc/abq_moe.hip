// A layer of experts: the router's choice and the sorting of its rows, the host side of the products with the experts' weights
// (kernels: abq_moe_rows_kernels.h, abq_block_kernels.h), and the weighted sum of each token's rows.
#include "abq_block_kernels.h"
#include "abq_moe_rows_kernels.h"
#include "../../include/abq.h"

#include <algorithm>

namespace abq {

// ---- the router -----------------------------------------------------------------------------------
struct RouteParams {
    MoeRouteArgs g;
    int chunk, chunks, bits;   // tokens of a workgroup, workgroups, bits of an expert's number
    int32_t* hist;             // [chunks][experts] (more than one chunk)
};

// Reductions over the 16 lanes of a row, every lane gets the result: two exchanges inside the quads, then the half row and the row mirrored.
template <int CTRL>
__device__ __forceinline__ uint32_t row_move(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xF, 0xF, true); }
template <int CTRL>
__device__ __forceinline__ uint64_t row_move(uint64_t x)
{
    return (uint64_t)row_move<CTRL>((uint32_t)(x >> 32)) << 32 | row_move<CTRL>((uint32_t)x);
}
template <int CTRL>
__device__ __forceinline__ float row_move(float x) { return __uint_as_float(row_move<CTRL>(__float_as_uint(x))); }
template <int CTRL>
__device__ __forceinline__ double row_move(double x) { return __builtin_bit_cast(double, row_move<CTRL>(__builtin_bit_cast(uint64_t, x))); }

template <int LPT, class T, class F>
__device__ __forceinline__ T reduce(T x, F f)
{
    x = f(x, row_move<0xB1>(x));    // quad_perm 1,0,3,2
    x = f(x, row_move<0x4E>(x));    // quad_perm 2,3,0,1
    x = f(x, row_move<0x141>(x));   // row_half_mirror
    x = f(x, row_move<0x140>(x));   // row_mirror
    if constexpr (LPT == 64) {
        T a;
        static_assert(sizeof(T) == 4 || sizeof(T) == 8, "words");
        if constexpr (sizeof(T) == 4) {
            a = __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, x), 16));
            x = f(x, a);
            a = __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, x), 32));
        } else {
            a = __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(long long, x), 16));
            x = f(x, a);
            a = __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(long long, x), 32));
        }
        x = f(x, a);
    }
    return x;
}

// Keys: whole numbers in the order of the values, all above that of minus infinity, which like NaN is 0: an expert that is not there.
__device__ __forceinline__ uint32_t key_of(float x)
{
    if (!(x > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(x + 0.0f);   // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t key_of(double x)
{
    if (!(x > -(double)INFINITY)) return 0;
    const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);
    return b >> 63 ? ~b : b | 1ull << 63;
}

__device__ __forceinline__ float logit(const MoeRouteArgs& g, int64_t token, int e)
{
    const int64_t at = token * g.ld + e;
    return g.logits_bits == 16 ? __half2float(__ushort_as_half(((const unsigned short*)g.logits)[at])) : ((const float*)g.logits)[at];
}

// What decides between two experts, by KIND.  0: a binary16 logit's key and, in its last 13 bits, 0x1FFF - expert: one word whose maximum is the
// choice, ties to the lowest expert.  1: the same of a binary32 logit in two words.  2: score + bias in binary64 (the expert's number is looked for afterwards).
template <int KIND> struct KeyType { typedef uint64_t type; };
template <> struct KeyType<0> { typedef uint32_t type; };

// The choice of one token by LPT lanes, lane l holding experts VPL l .. + VPL - 1.  Lane j gets choice j: its expert, or -1, and weight.
template <int LPT, int VPL, int KIND>
__device__ __forceinline__ void route_token(const MoeRouteArgs& g, int64_t token, int l, int* id_out, float* weight_out)
{
    typedef typename KeyType<KIND>::type Key;
    Key key[VPL];
    const auto larger = [](auto a, auto b) { return a > b ? a : b; };
    const auto sum = [](auto a, auto b) { return a + b; };
    float x[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = VPL * l + i < g.experts ? logit(g, token, VPL * l + i) : -INFINITY;
    if constexpr (KIND == 2) {
        float top = -INFINITY;
        double total = 0;
        if (!g.sigmoid) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) top = fmaxf(top, x[i]);
            top = reduce<LPT>(top, larger);
#pragma unroll
            for (int i = 0; i < VPL; ++i) total += x[i] > -INFINITY ? exp((double)x[i] - (double)top) : 0.0;
            total = reduce<LPT>(total, sum);
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            key[i] = 0;
            if (x[i] > -INFINITY) {
                const double s = g.sigmoid ? 1.0 / (1.0 + exp(-(double)x[i])) : exp((double)x[i] - (double)top) / total;
                key[i] = key_of(s + (double)g.bias[VPL * l + i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint32_t k = key_of(x[i]), e = VPL * l + i;
            // (a binary16 value's binary32 form has thirteen zeros at its end, ones where the key is its complement)
            if constexpr (KIND == 0) key[i] = k ? (k & 0xFFFFE000u) | (0x1FFFu - e) : 0;
            else key[i] = k ? (uint64_t)k << 32 | (0xFFFFFFFFu - e) : 0;
        }
    }
    int id = -1;
    for (int j = 0; j < g.top; ++j) {
        Key best = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) best = larger(best, key[i]);
        best = reduce<LPT>(best, larger);
        int e;
        if constexpr (KIND == 0) e = 0x1FFF - (int)(best & 0x1FFFu);
        else if constexpr (KIND == 1) e = (int)(0xFFFFFFFFu - (uint32_t)best);
        else {
            uint32_t low = 0xFFFFFFFFu;
#pragma unroll
            for (int i = VPL - 1; i >= 0; --i) low = key[i] == best ? (uint32_t)(VPL * l + i) : low;
            e = (int)reduce<LPT>(low, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
        }
        if (best == 0) e = -1;
#pragma unroll
        for (int i = 0; i < VPL; ++i) key[i] = VPL * l + i == e ? 0 : key[i];
        if (l == j) id = e;
    }
    // weights: the chosen experts' scores, over their sum where that is asked for (the largest logit taken out of all of them first)
    const float v = id >= 0 ? logit(g, token, id) : -INFINITY;
    float w;
    if (g.sigmoid) {
        const float c = g.renormalize ? fminf(reduce<LPT>(v, larger), 0.0f) : 0.0f;
        w = v >= 0.0f ? 1.0f / (1.0f + expf(-v)) : expf(v - c) / (1.0f + expf(v));
        if (id < 0) w = 0.0f;
        if (g.renormalize) w /= reduce<LPT>(w, sum);
    } else {
        float top = v, total;
        if (!g.renormalize) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) top = fmaxf(top, x[i]);   // (fmaxf leaves a NaN out)
        }
        top = reduce<LPT>(top, larger);
        w = id >= 0 ? expf(v - top) : 0.0f;
        if (g.renormalize) total = reduce<LPT>(w, sum);
        else {
            total = 0.0f;
#pragma unroll
            for (int i = 0; i < VPL; ++i) total += x[i] > -INFINITY ? expf(x[i] - top) : 0.0f;
            total = reduce<LPT>(total, sum);
        }
        w /= total;
    }
    *id_out = id;
    *weight_out = id >= 0 ? w * g.scale : 0.0f;
}

// Lanes of the wave that hold the same number as this one; 0 for lanes without one.
__device__ __forceinline__ uint64_t same_number(int id, int bits)
{
    uint64_t m = __ballot(id >= 0);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((id >> b) & 1);
        m &= (id >> b) & 1 ? set : ~set;
    }
    return id >= 0 ? m : 0;
}

// Places of a chunk's rows.  counts: LDS [waves][experts], all zero; base: LDS [experts], the place of the chunk's first row of each expert.  Every
// wave takes a run of the rows in order, so that the rows of one expert stay in theirs.
__device__ __forceinline__ void place_rows(const RouteParams& prm, int64_t slot0, int slots, int32_t* counts, const int32_t* base)
{
    const MoeRouteArgs& g = prm.g;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int run = (slots + 64 * waves - 1) / (64 * waves) * 64, from = wave * run, to = min(from + run, slots);
    int32_t* mine = counts + wave * g.experts;
    for (int i = from; i < to; i += 64) {
        const int id = i + lane < to ? g.ids[slot0 + i + lane] : -1;
        const uint64_t same = same_number(id, prm.bits);
        if (same && lane == __ffsll((unsigned long long)same) - 1) mine[id] += __popcll(same);
    }
    __syncthreads();
    for (int e = tid; e < g.experts; e += blockDim.x) {
        int32_t at = base[e];
        for (int w = 0; w < waves; ++w) {
            const int32_t n = counts[w * g.experts + e];
            counts[w * g.experts + e] = at;
            at += n;
        }
    }
    __syncthreads();
    for (int i = from; i < to; i += 64) {
        const bool there = i + lane < to;
        const int id = there ? g.ids[slot0 + i + lane] : -1;
        const uint64_t same = same_number(id, prm.bits);
        int place = -1;
        if (id >= 0) {
            place = mine[id] + __popcll(same & ((1ull << lane) - 1));
            g.order[place] = (int32_t)(slot0 + i + lane);
        }
        if (there) g.places[slot0 + i + lane] = place;
        __builtin_amdgcn_wave_barrier();
        if (same && lane == __ffsll((unsigned long long)same) - 1) mine[id] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
}

// Sums of totals[0..experts-1] (LDS) before each expert, by the first wave; returns (to that wave) the sum of all.  Ends with a barrier.
__device__ __forceinline__ void expert_starts(const RouteParams& prm, const int32_t* totals, int32_t* before, int32_t* all, bool store)
{
    const MoeRouteArgs& g = prm.g;
    if (threadIdx.x < 64) {
        int run = 0;
        for (int e0 = 0; e0 < g.experts; e0 += 64) {
            const int e = e0 + threadIdx.x, n = e < g.experts ? totals[e] : 0, upto = moe_scan(n);
            if (e < g.experts) {
                before[e] = run + upto - n;
                if (store) g.starts[e] = run + upto - n;
            }
            run += __builtin_amdgcn_readlane(upto, 63);
        }
        if (threadIdx.x == 0) {
            *all = run;
            if (store) g.starts[g.experts] = run;
        }
    }
    __syncthreads();
}

// What bounds it: one token is latency (a launch, the logits, `top` rounds of a maximum over 16 lanes); many tokens are the vector ALU: a
// round is some 3 VPL + 10 operations for the four tokens of a wave.  Up to kRouteOne tokens are one launch of one workgroup, which also sorts
// the rows; more are a launch that chooses and counts, a workgroup per chunk, and a second one whose workgroups add the counts of the chunks before
// theirs and place their rows (no atomics on memory: the same rows in the same order every time).
template <int LPT, int VPL, int KIND>
__global__ __launch_bounds__(1024) void moe_route_kernel(RouteParams prm)
{
    extern __shared__ __align__(16) int32_t lds[];   // [experts] totals, [experts] before, [waves][experts] counts (one chunk: the place of its rows)
    __shared__ int32_t all;
    const MoeRouteArgs& g = prm.g;
    const int tid = threadIdx.x, l = tid % LPT, E = g.experts;
    const bool alone = prm.chunks == 1;
    const int64_t t0 = (int64_t)blockIdx.x * prm.chunk, t1 = min(t0 + prm.chunk, (int64_t)g.tokens);
    for (int i = tid; i < (alone ? 2 + (int)(blockDim.x >> 6) : 1) * E; i += blockDim.x) lds[i] = 0;
    __syncthreads();
    for (int64_t t = t0 + tid / LPT; t < t1; t += blockDim.x / LPT) {
        int id;
        float w;
        route_token<LPT, VPL, KIND>(g, t, l, &id, &w);
        if (l < g.top) {
            g.ids[t * g.top + l] = id;
            g.weights[t * g.top + l] = w;
            if (id >= 0) atomicAdd(&lds[id], 1);
        }
    }
    __syncthreads();
    if (!alone) {
        for (int e = tid; e < E; e += blockDim.x) prm.hist[(size_t)blockIdx.x * E + e] = lds[e];
        return;
    }
    expert_starts(prm, lds, lds + E, &all, true);
    place_rows(prm, 0, g.tokens * g.top, lds + 2 * E, lds + E);
    for (int i = all + tid; i < g.tokens * g.top; i += blockDim.x) g.order[i] = -1;
}

__global__ __launch_bounds__(1024) void moe_place_kernel(RouteParams prm)
{
    extern __shared__ __align__(16) int32_t lds[];   // [experts] totals, [experts] before, [waves][experts] counts
    __shared__ int32_t all;
    const MoeRouteArgs& g = prm.g;
    const int tid = threadIdx.x, E = g.experts, c = blockIdx.x, waves = blockDim.x >> 6;
    int32_t *totals = lds, *before = lds + E, *counts = lds + 2 * E;
    for (int i = tid; i < (2 + waves) * E; i += blockDim.x) lds[i] = 0;
    __syncthreads();
    // the chunks' counts: threads side by side along the experts, groups of them along the chunks (sums of whole numbers: any order)
    const int wide = min(E, (int)blockDim.x), groups = blockDim.x / wide, group = tid / wide;
    if (group < groups)
        for (int e = tid % wide; e < E; e += wide) {
            int32_t sum = 0, pre = 0;
#pragma unroll 8
            for (int k = group; k < prm.chunks; k += groups) {
                const int32_t n = prm.hist[(size_t)k * E + e];
                sum += n;
                pre += k < c ? n : 0;
            }
            atomicAdd(&totals[e], sum);
            atomicAdd(&counts[e], pre);
        }
    __syncthreads();
    expert_starts(prm, totals, before, &all, c == 0);
    for (int e = tid; e < E; e += blockDim.x) { before[e] += counts[e]; counts[e] = 0; }
    __syncthreads();
    const int64_t t0 = (int64_t)c * prm.chunk, t1 = min(t0 + prm.chunk, (int64_t)g.tokens);
    place_rows(prm, t0 * g.top, (int)(t1 - t0) * g.top, counts, before);
    for (int64_t i = all + (int64_t)c * blockDim.x + tid; i < (int64_t)g.tokens * g.top; i += (int64_t)prm.chunks * blockDim.x) g.order[i] = -1;
}

constexpr int kRouteOne = 256, kRouteChunks = 256;   // tokens of a single launch; chunks of two, at most

static void route_chunks(int tokens, int* chunk, int* chunks)
{
    *chunk = tokens <= kRouteOne ? tokens : std::max(64, (tokens + kRouteChunks - 1) / kRouteChunks);
    *chunks = (tokens + *chunk - 1) / *chunk;
}

size_t moe_route_workspace_bytes(int tokens, int experts)
{
    int chunk, chunks;
    route_chunks(tokens, &chunk, &chunks);
    return chunks == 1 ? 0 : (size_t)chunks * experts * sizeof(int32_t);
}

template <int LPT, int VPL>
static void route_go(const RouteParams& prm, unsigned threads, size_t lds_bytes, hipStream_t s)
{
    const unsigned grid = (unsigned)prm.chunks;
    if (prm.g.bias) moe_route_kernel<LPT, VPL, 2><<<grid, threads, lds_bytes, s>>>(prm);
    else if (prm.g.logits_bits == 16) moe_route_kernel<LPT, VPL, 0><<<grid, threads, lds_bytes, s>>>(prm);
    else moe_route_kernel<LPT, VPL, 1><<<grid, threads, lds_bytes, s>>>(prm);
}

hipError_t launch_moe_route(const MoeRouteArgs& g, hipStream_t s)
{
    RouteParams prm;
    prm.g = g;
    route_chunks(g.tokens, &prm.chunk, &prm.chunks);
    prm.hist = (int32_t*)g.workspace;
    prm.bits = 32 - __builtin_clz((unsigned)g.experts);
    const int E = g.experts, lpt = E <= 256 ? 16 : 64;
    const int64_t lanes = (int64_t)prm.chunk * lpt;
    const unsigned most = E <= 512 ? 1024u : 512u;                               // (counts of every wave in 64 KiB of LDS)
    const unsigned threads = lanes >= most ? most : (unsigned)((lanes + 63) / 64 * 64);
    const size_t place_lds = (size_t)(2 + threads / 64) * E * sizeof(int32_t);
    const size_t route_lds = prm.chunks == 1 ? place_lds : (size_t)E * sizeof(int32_t);
    if (E <= 16) route_go<16, 1>(prm, threads, route_lds, s);
    else if (E <= 32) route_go<16, 2>(prm, threads, route_lds, s);
    else if (E <= 64) route_go<16, 4>(prm, threads, route_lds, s);
    else if (E <= 128) route_go<16, 8>(prm, threads, route_lds, s);
    else if (E <= 256) route_go<16, 16>(prm, threads, route_lds, s);
    else if (E <= 512) route_go<64, 8>(prm, threads, route_lds, s);
    else route_go<64, 16>(prm, threads, route_lds, s);
    if (hipError_t e = hipGetLastError()) return e;
    if (prm.chunks > 1) moe_place_kernel<<<(unsigned)prm.chunks, most, (size_t)(2 + most / 64) * E * sizeof(int32_t), s>>>(prm);
    return hipGetLastError();
}

// ---- the products: choice of kernel --------------------------------------------------------------
// Workgroup shapes of the block kernel: 0 (256 x 256), 3 (128 x 128), 4 (64 x 128).
static int expert_bm(int shape) { return shape == 0 ? 256 : (shape == 3 ? 128 : 64); }
static int expert_bn(int p, int shape) { return shape == 0 ? 64 * bk_expert_nt(p) : 128; }

// Groups of `per` rows that `rows` rows of `experts` experts can make at most.
static int most_groups(int rows, int experts, int per)
{
    return (int)(((int64_t)rows + (int64_t)std::min(experts, rows) * (per - 1)) / per);
}

struct MoePlan {
    bool few;                    // the few-rows kernel, else the block kernel
    int R, MT, kparts, tgroups;  // few
    int shape;                   // block
};

static bool rows_plan(int p, int K, int MT, MoePlan* pl)
{
    const int nsuper = (K + kSuperK - 1) / kSuperK;
    for (int R = 1; R <= 4; ++R) {
        const int most = moe_max_waves(p, R, MT);
        if (most == 0 || nsuper > R * most) continue;
        pl->few = true;
        pl->R = R;
        pl->MT = MT;
        pl->kparts = (nsuper + R - 1) / R;
        pl->tgroups = std::max(1, 8 / pl->kparts);
        return true;
    }
    return false;
}

static MoePlan moe_plan(int p, int q, int rows, int N, int K, int tokens, int experts)
{
    MoePlan pl{};
    const double mean = (double)rows / std::min(experts, rows);   // rows of an expert
    if (K >= 16 && mean <= 32 && rows_plan(p, K, mean <= 16 ? 1 : 2, &pl)) return pl;
    pl.shape = mean >= 192 ? 0 : (mean >= 80 ? 3 : 4);
    return pl;
}

size_t moe_gemm_workspace_bytes(int p, int q, int rows, int N, int K, int tokens, int experts)
{
    if (moe_plan(p, q, rows, N, K, tokens, experts).few) return 0;
    ActLayout A;
    make_act_layout(q, tokens, K, ABQ_LAYOUT_FIELDS, &A);
    return A.total;
}

static MoeGroups groups_of(const MoeGemmArgs& g) { return MoeGroups{g.starts, g.order, g.experts, g.rows, g.tokens, g.top}; }

hipError_t launch_moe_gemm(const MoeGemmArgs& g, const WeightLayout& W, hipStream_t s)
{
    const MoePlan pl = moe_plan(g.p, g.q, g.rows, g.N, g.K, g.tokens, g.experts);
    if (pl.few) {
        MoeRowsParams prm{};
        prm.w = g.w_blobs;
        prm.w_stride = g.w_stride;
        prm.off_params = W.off_params;
        for (int i = 0; i < 3; ++i) prm.off_fields[i] = W.off_fields[i];
        prm.a = g.a_codes; prm.a_scale = g.a_scale; prm.a_zero = g.a_zero;
        prm.y = g.y;
        prm.g = groups_of(g);
        prm.N = g.N; prm.K = g.K;
        prm.nsuper = (g.K + kSuperK - 1) / kSuperK;
        prm.ntiles = W.NT;
        prm.oa = g.q == 8 ? 128 : 0;
        prm.ow = g.p == 8 ? 128 : 0;
        prm.a_mask = (uint32_t)((1 << g.q) - 1) * 0x01010101u;
        prm.kparts = pl.kparts; prm.tgroups = pl.tgroups;
        prm.batch = pl.kparts >= 4 ? moe_batch(pl.MT) : 2;
        prm.groups_n = (W.NT + pl.tgroups - 1) / pl.tgroups;
        prm.most = most_groups(g.rows, g.experts, 16 * pl.MT);
        const int waves = pl.kparts * pl.tgroups, room = moe_max_waves(g.p, pl.R, pl.MT);   // (waves a unit holds)
        const unsigned grid = (unsigned)std::min<int64_t>((int64_t)num_cus() * std::max(1, room / waves), (int64_t)prm.most * prm.groups_n);
        switch (g.p) {
            case 1: return moe_rows_launch_p1(prm, pl.R, pl.MT, grid, s);
            case 2: return moe_rows_launch_p2(prm, pl.R, pl.MT, grid, s);
            case 3: return moe_rows_launch_p3(prm, pl.R, pl.MT, grid, s);
            case 4: return moe_rows_launch_p4(prm, pl.R, pl.MT, grid, s);
            case 5: return moe_rows_launch_p5(prm, pl.R, pl.MT, grid, s);
            case 6: return moe_rows_launch_p6(prm, pl.R, pl.MT, grid, s);
            case 7: return moe_rows_launch_p7(prm, pl.R, pl.MT, grid, s);
            default: return moe_rows_launch_p8(prm, pl.R, pl.MT, grid, s);
        }
    }
    ActLayout A;
    make_act_layout(g.q, g.tokens, g.K, ABQ_LAYOUT_FIELDS, &A);
    uint8_t* packed = (uint8_t*)g.workspace;
    if (hipError_t e = launch_pack_act_codes(A, g.a_codes, g.a_scale, g.a_zero, packed, s)) return e;
    const int bm = expert_bm(pl.shape), bn = expert_bn(g.p, pl.shape);
    BlockExpertParams prm{};
    for (int i = 0; i < 3; ++i) prm.fields[i] = g.w_blobs + W.off_fields[i];
    prm.a = packed + A.off_codes;
    prm.aparams = (const RowParams*)(packed + A.off_params);
    prm.wparams = (const RowParams*)(g.w_blobs + W.off_params);
    prm.y = g.y;
    prm.M = g.tokens; prm.N = g.N; prm.K = g.K;
    prm.lda = A.Kp;
    prm.nsuper = A.Kp / kSuperK;
    prm.ntiles = W.NT;
    prm.oa = g.q == 8 ? 128 : 0;
    prm.ow = g.p == 8 ? 128 : 0;
    prm.narrow_sums = ((long)g.K * ((1 << g.p) - 1) < (1L << 23) && (long)g.K * ((1 << g.q) - 1) < (1L << 23)) ? 1 : 0;
    prm.tiles_m = most_groups(g.rows, g.experts, bm);
    prm.tiles_n = (g.N + bn - 1) / bn;
    prm.band_m = 1024 / bm;
    prm.g = groups_of(g);
    prm.w_stride = g.w_stride;
    switch (g.p) {
        case 1: return block_experts_launch_p1(prm, pl.shape, s);
        case 2: return block_experts_launch_p2(prm, pl.shape, s);
        case 3: return block_experts_launch_p3(prm, pl.shape, s);
        case 4: return block_experts_launch_p4(prm, pl.shape, s);
        case 5: return block_experts_launch_p5(prm, pl.shape, s);
        case 6: return block_experts_launch_p6(prm, pl.shape, s);
        case 7: return block_experts_launch_p7(prm, pl.shape, s);
        default: return block_experts_launch_p8(prm, pl.shape, s);
    }
}

// ---- back to one row a token ----------------------------------------------------------------------
struct CombineParams {
    int N, rows, top;
    const uint16_t* y;
    int64_t ldy;
    const int32_t* places;
    const float* weights;
    const uint16_t* add;
    int64_t ldadd;
    uint16_t* out;
    int64_t ldout;
};

// One workgroup per token and run of 256 eights of its row; the terms are added in the order of the choices, in binary32.
__global__ __launch_bounds__(256) void moe_combine_kernel(CombineParams prm)
{
    const int64_t t = blockIdx.x;
    const int v = blockIdx.y * 256 + threadIdx.x;
    if (8 * v >= prm.N) return;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    uint32_t h[4];
    if (prm.add) {
        load_half8<true>(prm.add + t * prm.ldadd, v, prm.N, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = __half2float(__ushort_as_half((unsigned short)(h[e >> 1] >> (16 * (e & 1)))));
    }
    const int32_t* places = prm.places + t * prm.top;
    const float* weights = prm.weights + t * prm.top;
#pragma unroll 4
    for (int j = 0; j < prm.top; ++j) {
        const int place = places[j];
        if ((unsigned)place >= (unsigned)prm.rows) continue;
        const float w = weights[j];
        load_half8<true>(prm.y + place * prm.ldy, v, prm.N, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] = fmaf(w, __half2float(__ushort_as_half((unsigned short)(h[e >> 1] >> (16 * (e & 1))))), sum[e]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        h[j] = (uint32_t)__half_as_ushort(__float2half_rn(sum[2 * j])) | ((uint32_t)__half_as_ushort(__float2half_rn(sum[2 * j + 1])) << 16);
    store_half8<true>(prm.out + t * prm.ldout, v, prm.N, h);
}

hipError_t launch_moe_combine(int tokens, int N, int rows, int top, const uint16_t* y, int ldy, const int32_t* places, const float* weights,
                              const uint16_t* add, int ldadd, uint16_t* out, int ldout, hipStream_t s)
{
    const CombineParams prm{N, rows, top, y, ldy, places, weights, add, ldadd, out, ldout};
    moe_combine_kernel<<<dim3((unsigned)tokens, (unsigned)((N + 2047) / 2048)), 256, 0, s>>>(prm);
    return hipGetLastError();
}

}  // namespace abq
