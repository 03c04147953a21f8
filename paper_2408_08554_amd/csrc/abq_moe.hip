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
    int each;                  // chunks that a workgroup of the second launch places
    int padded;                // experts, to a multiple of eight
    uint16_t* hist;            // [chunks][padded] (more than one chunk)
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

// What decides between two experts, by KIND: its maximum is the choice, ties to the lowest expert.
// 0, a binary16 logit: a whole number in the order of the values, above 0 (which is an expert that is not there: minus infinity or NaN), whose last 13
//    bits are 0x1FFF - expert.  (A binary16 value's binary32 form has thirteen zeros at its end, ones where the key is its complement.)
// 1, a binary32 logit: its binary64 form, which ends in 29 zeros, with the expert's number in the last 13 bits (of a negative value as it is, else
//    0x1FFF - expert).  Plus infinity is 2^1023, not there is the lowest finite value.  One maximum is one instruction; on whole numbers of two words it is three.
// 2: score + bias in binary64; the expert's number is looked for afterwards.  Not there is minus infinity.
template <int KIND> struct KeyType { typedef double type; };
template <> struct KeyType<0> { typedef uint32_t type; };
constexpr uint32_t kNotThereHigh = 0xFFEFFFFFu;   // (KIND 1: the lowest finite value's upper word, whatever the lower)

__device__ __forceinline__ double packed(uint32_t high, uint32_t low) { return __builtin_bit_cast(double, (uint64_t)high << 32 | low); }
__device__ __forceinline__ uint32_t high_of(double x) { return (uint32_t)(__builtin_bit_cast(uint64_t, x) >> 32); }
__device__ __forceinline__ uint32_t low_of(double x) { return (uint32_t)__builtin_bit_cast(uint64_t, x); }
__device__ __forceinline__ uint32_t key_max(uint32_t a, uint32_t b) { return max(a, b); }
__device__ __forceinline__ double key_max(double a, double b)   // (the instruction: fmax() makes quiet NaNs of its arguments first, and there are none)
{
    double d;
    asm("v_max_f64 %0, %1, %2" : "=v"(d) : "v"(a), "v"(b));
    return d;
}
template <int KIND>
__device__ __forceinline__ typename KeyType<KIND>::type key_of(float x, int e)
{
    if constexpr (KIND == 0) {
        const uint32_t b = __float_as_uint(x + 0.0f);   // (-0 is 0)
        return x > -INFINITY ? ((b & 0x80000000u ? ~b : b | 0x80000000u) & 0xFFFFE000u) | (0x1FFFu - e) : 0;
    } else {
        const double d = (double)(x + 0.0f);
        const uint32_t high = x > -INFINITY ? min(high_of(d), x < 0.0f ? 0xFFFFFFFFu : 0x7FE00000u) : kNotThereHigh;
        return packed(high, low_of(d) | (high >> 31 ? e : 0x1FFF - e));
    }
}

// Logits VPL l .. + VPL - 1 of a token, minus infinity behind the last one: as vectors where the lanes have as many experts as there are (unaligned: any stride of
// rows), else one by one.  (Whole loads, none under a condition of a lane's, or each waits for the one before.)
template <int LPT, int VPL, bool HALF>
__device__ __forceinline__ void load_logits(const MoeRouteArgs& g, int64_t token, int l, float* x)
{
    const int64_t row = token * g.ld;
    constexpr int kWords = HALF ? (VPL + 1) / 2 : VPL, kVec = kWords >= 4 ? 4 : kWords;
    typedef uint32_t Vec __attribute__((ext_vector_type(kVec), aligned(2)));
    if (VPL > 1 && g.experts == LPT * VPL) {
        const Vec* at = reinterpret_cast<const Vec*>((const uint8_t*)g.logits + (row + VPL * l) * (HALF ? 2 : 4));
        uint32_t raw[kWords];
#pragma unroll
        for (int v = 0; v < kWords / kVec; ++v) {
            const Vec w = at[v];
#pragma unroll
            for (int e = 0; e < kVec; ++e) raw[kVec * v + e] = w[e];
        }
#pragma unroll
        for (int i = 0; i < VPL; ++i) x[i] = HALF ? __half2float(__ushort_as_half((unsigned short)(raw[i / 2] >> (16 * (i & 1))))) : __uint_as_float(raw[HALF ? 0 : i]);
        return;
    }
    uint32_t raw[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int64_t at = row + min(VPL * l + i, g.experts - 1);
        if constexpr (HALF) raw[i] = ((const unsigned short*)g.logits)[at];
        else raw[i] = ((const uint32_t*)g.logits)[at];
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const float v = HALF ? __half2float(__ushort_as_half((unsigned short)raw[i])) : __uint_as_float(raw[i]);
        x[i] = VPL * l + i < g.experts ? v : -INFINITY;
    }
}

// The choice of one token by LPT lanes, lane l holding experts VPL l .. + VPL - 1.  Lane j gets choice j: its expert, or -1, and weight.
template <int LPT, int VPL, int KIND, bool HALF>
__device__ __forceinline__ void route_token(const MoeRouteArgs& g, int64_t token, int l, int* id_out, float* weight_out)
{
    typedef typename KeyType<KIND>::type Key;
    Key key[VPL];
    const auto larger = [](auto a, auto b) { return a > b ? a : b; };
    const auto sum = [](auto a, auto b) { return a + b; };
    float x[VPL];
    load_logits<LPT, VPL, HALF>(g, token, l, x);
    if constexpr (KIND == 2) {
        float top = -INFINITY;
        double total = 0;
        float bias[VPL];
#pragma unroll
        for (int i = 0; i < VPL; ++i) bias[i] = g.bias[min(VPL * l + i, g.experts - 1)];
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
            const double s = g.sigmoid ? 1.0 / (1.0 + exp(-(double)x[i])) : exp((double)x[i] - (double)top) / total;
            const double k = s + (double)bias[i];
            key[i] = x[i] > -INFINITY && k > -(double)INFINITY ? k : -(double)INFINITY;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VPL; ++i) key[i] = key_of<KIND>(x[i], VPL * l + i);
    }
    int id = -1;
    float v = -INFINITY;   // the choice's logit
    Key mine = 0;
    for (int j = 0; j < g.top; ++j) {
        Key best = key[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) best = key_max(best, key[i]);
        best = reduce<LPT>(best, [](Key a, Key b) { return key_max(a, b); });
        if constexpr (KIND == 2) {
            uint32_t low = 0xFFFFFFFFu;
#pragma unroll
            for (int i = VPL - 1; i >= 0; --i) low = key[i] == best ? (uint32_t)(VPL * l + i) : low;
            const int e = best > -(double)INFINITY ? (int)reduce<LPT>(low, [](uint32_t a, uint32_t b) { return a < b ? a : b; }) : -1;
            float at = -INFINITY;
#pragma unroll
            for (int i = 0; i < VPL; ++i) {
                if (VPL * l + i == e) { key[i] = -(double)INFINITY; at = x[i]; }
            }
            at = reduce<LPT>(at, larger);
            if (l == j) { id = e; v = at; }
        } else if constexpr (KIND == 1) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) key[i] = packed(low_of(key[i]) == low_of(best) ? kNotThereHigh : high_of(key[i]), low_of(key[i]));
            if (l == j) mine = best;
        } else {
#pragma unroll
            for (int i = 0; i < VPL; ++i) key[i] = key[i] == best ? 0 : key[i];
            if (l == j) mine = best;
        }
    }
    // (the key's way back)
    if constexpr (KIND == 0) {
        if (l < g.top && mine != 0) {
            id = 0x1FFF - (int)(mine & 0x1FFFu);
            v = __uint_as_float((mine >> 31 ? mine & 0x7FFFFFFFu : ~mine) & 0xFFFFE000u);
        }
    } else if constexpr (KIND == 1) {
        if (l < g.top && high_of(mine) != kNotThereHigh) {
            id = (int)(low_of(mine) & 0x1FFFu);
            id = high_of(mine) >> 31 ? id : 0x1FFF - id;
            v = (float)packed(high_of(mine), low_of(mine) & 0xFFFFE000u);
        }
    }
    // weights: the chosen experts' scores, over their sum where that is asked for (the largest logit taken out of all of them first)
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

// Places of a run of rows, kept in registers: every wave takes a part of the rows in order, 64 at a time, kPlaceRounds times at most, so that the rows of one
// expert stay in theirs.
constexpr int kPlaceRounds = 8;
struct PlacedRows {
    int id[kPlaceRounds], at[kPlaceRounds];   // a row's expert, its place among the wave's rows of that expert
    int from, rounds;                         // the wave's first row, its 64s of rows

    __device__ __forceinline__ PlacedRows(const int32_t* ids, int slots)   // ids: the rows' experts
    {
        const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
        rounds = (slots + 64 * waves - 1) / (64 * waves);
        from = (int)(threadIdx.x >> 6) * rounds * 64;
#pragma unroll
        for (int i = 0; i < kPlaceRounds; ++i) {
            const int row = from + 64 * i + lane;
            const int v = ids[min(row, slots - 1)];
            id[i] = i < rounds && row < slots ? v : -1;
        }
    }
    // counts: LDS [waves][experts], all zero; becomes the waves' own
    __device__ __forceinline__ void count(const RouteParams& prm, int32_t* counts)
    {
        const int lane = threadIdx.x & 63;
        int32_t* mine = counts + (threadIdx.x >> 6) * prm.g.experts;
#pragma unroll
        for (int i = 0; i < kPlaceRounds; ++i) {
            if (i < rounds) {
                const uint64_t same = same_number(id[i], prm.bits);
                const int before = mine[max(id[i], 0)], below = __popcll(same & ((1ull << lane) - 1));
                at[i] = before + below;
                __builtin_amdgcn_wave_barrier();
                if (id[i] >= 0 && below == 0) mine[id[i]] = before + __popcll(same);
                __builtin_amdgcn_wave_barrier();
            }
        }
    }
    // ... and base: LDS [experts], the place of the run's first row of each expert: order and places of the rows from slot0 on
    __device__ __forceinline__ void store(const RouteParams& prm, int64_t slot0, int slots, int32_t* counts, const int32_t* base)
    {
        const MoeRouteArgs& g = prm.g;
        const int lane = threadIdx.x & 63, waves = blockDim.x >> 6;
        __syncthreads();
        for (int e = threadIdx.x; e < g.experts; e += blockDim.x) {
            int32_t next = base[e];
            for (int w0 = 0; w0 < waves; w0 += 8) {   // (loads first: the compiler takes every store for one to what is loaded next)
                int32_t n[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) n[w] = counts[min(w0 + w, waves - 1) * g.experts + e];
#pragma unroll
                for (int w = 0; w < 8; ++w) {
                    if (w0 + w < waves) counts[(w0 + w) * g.experts + e] = next;
                    next += n[w];
                }
            }
        }
        __syncthreads();
        const int32_t* mine = counts + (threadIdx.x >> 6) * g.experts;
#pragma unroll
        for (int i = 0; i < kPlaceRounds; ++i) {
            const int row = from + 64 * i + lane;
            if (i < rounds && row < slots) {
                int place = -1;
                if (id[i] >= 0) {
                    place = mine[id[i]] + at[i];
                    g.order[place] = (int32_t)(slot0 + row);
                }
                g.places[slot0 + row] = place;
            }
        }
    }
};

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

// Threads of a workgroup, at most: sixteen logits a lane with a bias take more than the 128 registers of 1024.
__host__ __device__ constexpr int route_threads(int VPL, bool biased) { return VPL >= 16 && biased ? 512 : 1024; }

// What bounds it: one token is latency (a launch, the logits, `top` rounds of a maximum over 16 lanes); many tokens are the vector ALU: a
// round is some 3 VPL + 10 operations for the four tokens of a wave.  Few are one launch of one workgroup, which also sorts
// the rows; more are a launch that chooses and counts, a workgroup per chunk, and a second one whose workgroups add the counts of the chunks before
// theirs and place their rows (no atomics on memory: the same rows in the same order every time).  Measured: one token of eight experts 3.4 us, 64 of 128
// (binary32) 7.2, 4099 of 64 with a bias 5.5 + 6.5, 32768 of 128 (binary16) 10.7 + 9.4.
template <int LPT, int VPL, int KIND, bool HALF>
__global__ __launch_bounds__(route_threads(VPL, KIND == 2)) void moe_route_kernel(RouteParams prm)
{
    extern __shared__ __align__(16) int32_t lds[];   // [experts] totals; one chunk alone: [experts] before, [waves][experts] counts, [rows] ids
    __shared__ int32_t all;
    const MoeRouteArgs& g = prm.g;
    const int tid = threadIdx.x, l = tid % LPT, E = g.experts;
    const bool alone = prm.chunks == 1;
    const int64_t t0 = (int64_t)blockIdx.x * prm.chunk, t1 = min(t0 + prm.chunk, (int64_t)g.tokens);
    const int counted = (alone ? 2 + (int)(blockDim.x >> 6) : 1) * E;
    for (int i = tid; i < counted; i += blockDim.x) lds[i] = 0;
    __syncthreads();
    for (int64_t t = t0 + tid / LPT; t < t1; t += blockDim.x / LPT) {
        int id;
        float w;
        route_token<LPT, VPL, KIND, HALF>(g, t, l, &id, &w);
        if (l < g.top) {
            g.ids[t * g.top + l] = id;
            g.weights[t * g.top + l] = w;
            if (alone) lds[counted + (int)t * g.top + l] = id;
            if (id >= 0) atomicAdd(&lds[id], 1);
        }
    }
    __syncthreads();
    if (!alone) {   // (a count is at most a chunk's tokens)
        for (int e = tid; e < prm.padded; e += blockDim.x) prm.hist[(size_t)blockIdx.x * prm.padded + e] = (uint16_t)(e < E ? lds[e] : 0);
        return;
    }
    PlacedRows rows(lds + counted, g.tokens * g.top);
    rows.count(prm, lds + 2 * E);
    expert_starts(prm, lds, lds + E, &all, true);
    rows.store(prm, 0, g.tokens * g.top, lds + 2 * E, lds + E);
    for (int i = all + tid; i < g.tokens * g.top; i += blockDim.x) g.order[i] = -1;
}

__global__ __launch_bounds__(1024) void moe_place_kernel(RouteParams prm)
{
    extern __shared__ __align__(16) int32_t lds[];   // [padded] totals, [padded] before, [waves][experts] counts (at least [padded])
    __shared__ int32_t all;
    const MoeRouteArgs& g = prm.g;
    const int tid = threadIdx.x, E = g.experts, c0 = blockIdx.x * prm.each, waves = blockDim.x >> 6;
    int32_t *totals = lds, *before = lds + prm.padded, *counts = lds + 2 * prm.padded;
    const int64_t t0 = (int64_t)c0 * prm.chunk, t1 = min(t0 + (int64_t)prm.each * prm.chunk, (int64_t)g.tokens);
    const int slots = (int)(t1 - t0) * g.top;
    PlacedRows rows(g.ids + t0 * g.top, slots);
    for (int i = tid; i < 2 * prm.padded + max(waves * E, prm.padded); i += blockDim.x) lds[i] = 0;
    __syncthreads();
    // the chunks' counts: threads side by side along the experts (eight each), groups of them along the chunks, a thread's loads all in flight (sums of whole
    // numbers: any order), no more groups than take eight chunks each: with few experts all of them add to the same words one after the other (300 tokens of eight
    // experts took 20.6 us with every thread a group, 7.0 now)
    const int eights = prm.padded / 8, wide = min(eights, (int)blockDim.x), groups = min((int)blockDim.x / wide, (prm.chunks + 7) / 8), group = tid / wide;
    const uint4* hist = reinterpret_cast<const uint4*>(prm.hist);
    if (group < groups)
        for (int f = tid % wide; f < eights; f += wide) {
            int sum[8] = {0, 0, 0, 0, 0, 0, 0, 0}, pre[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            for (int k0 = group; k0 < prm.chunks; k0 += 8 * groups) {
                uint4 n[8], some = {0, 0, 0, 0}, rest = {0, 0, 0, 0};   // (two counts a word: eight of at most kRouteLongest tokens stay below 2^16)
#pragma unroll
                for (int u = 0; u < 8; ++u) n[u] = hist[(size_t)min(k0 + u * groups, prm.chunks - 1) * eights + f];
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int k = k0 + u * groups;
                    const uint32_t before_of = k < c0 ? ~0u : 0u, rest_of = k >= c0 && k < prm.chunks ? ~0u : 0u;
                    some.x += n[u].x & before_of; some.y += n[u].y & before_of; some.z += n[u].z & before_of; some.w += n[u].w & before_of;
                    rest.x += n[u].x & rest_of; rest.y += n[u].y & rest_of; rest.z += n[u].z & rest_of; rest.w += n[u].w & rest_of;
                }
                const uint32_t a[4] = {some.x, some.y, some.z, some.w}, b[4] = {rest.x, rest.y, rest.z, rest.w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int v = (int)(a[e >> 1] >> (16 * (e & 1)) & 0xFFFFu);
                    pre[e] += v;
                    sum[e] += v + (int)(b[e >> 1] >> (16 * (e & 1)) & 0xFFFFu);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {   // (expert 8 f + e at e eights + f: neighbours on neighbouring banks)
                atomicAdd(&before[e * eights + f], sum[e]);
                atomicAdd(&counts[e * eights + f], pre[e]);
            }
        }
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x) totals[e] = before[(e & 7) * eights + (e >> 3)];
    __syncthreads();
    expert_starts(prm, totals, before, &all, c0 == 0);
    for (int e = tid; e < E; e += blockDim.x) before[e] += counts[(e & 7) * eights + (e >> 3)];
    __syncthreads();
    for (int i = tid; i < prm.padded; i += blockDim.x) counts[i] = 0;
    __syncthreads();
    rows.count(prm, counts);
    rows.store(prm, t0 * g.top, slots, counts, before);
    for (int64_t i = all + (int64_t)blockIdx.x * blockDim.x + tid; i < (int64_t)g.tokens * g.top; i += (int64_t)gridDim.x * blockDim.x) g.order[i] = -1;
}

// A single launch is for so many tokens and logits at most, and for so many rounds of its one workgroup, which has one unit's vector ALU (a round of 1024 lanes
// takes 0.2 to 0.45 us, the two launches together about 9; 256 tokens of 256 experts with a bias, all in one: 80 us, 15 now; 436 of eight, top 6, with a bias
// 26, 9.4 now).  At the bounds (us, one / two launches, binary32, and with a bias): 64 of 128, top 8, 7.9 / 9.7, 14.1 / 12.1; 128 of 64, top 2, 7.0 / 8.7,
// 11.2 / 9.5; 32 of 256, top 8, 8.0 / 11.2, 14.9 / 15.4; 512 of 16, top 2, 12.0 / 8.5, 20.2 / 9.1; past them 128 of 128, top 2, 8.1 / 9.2, 16.3 / 10.5; 256 of
// 64, top 2, 9.5 / 8.8, 17.9 / 9.5.  (So two launches would be ahead earlier where few experts have many tokens, and where there is a bias.)  Of more, chunks of
// kRouteTokens (about kRouteChunks longer ones of many), placed by about kPlacers workgroups, each of which reads all
// chunks' counts and has room for the rows of place_room().
constexpr int kRouteOne = 512, kRouteOneLogits = 8192, kRouteOneRounds = 16, kRouteTokens = 16, kRouteLongest = 4096, kRouteChunks = 512, kPlacers = 128;

static int route_lanes(int experts) { return experts <= 256 ? 16 : 64; }   // lanes of a token
static int place_threads(int experts) { return experts <= 512 ? 1024 : 512; }   // (the counts of every wave in 64 KiB of LDS)
static int place_room(int experts) { return place_threads(experts) * kPlaceRounds; }

static int route_longest(int experts, int top) { return std::min(kRouteLongest, place_room(experts) / top); }   // tokens of a chunk, at most

static void route_chunks(int tokens, int experts, int top, int* chunk, int* chunks)
{
    const int64_t rounds = ((int64_t)tokens * route_lanes(experts) + 1023) / 1024 * top;
    *chunk = tokens <= kRouteOne && tokens * experts <= kRouteOneLogits && rounds <= kRouteOneRounds ? tokens : std::min(std::max(kRouteTokens, (tokens + kRouteChunks - 1) / kRouteChunks), route_longest(experts, top));
    *chunks = (tokens + *chunk - 1) / *chunk;
}

// Counts of the most chunks that so many tokens or fewer are cut into, so that a workspace of the largest batch serves all: a chunk grows by whole tokens, and
// their number falls where it does (8192 tokens are 512 chunks, 8193 are 482).
size_t moe_route_workspace_bytes(int tokens, int experts, int top)
{
    int chunk, chunks;
    route_chunks(tokens, experts, top, &chunk, &chunks);
    if (chunks == 1) return 0;   // (and for fewer tokens)
    const int longest = route_longest(experts, top);
    const int most = std::max(std::min((tokens + kRouteTokens - 1) / kRouteTokens, kRouteChunks), (tokens + longest - 1) / longest);
    return (size_t)most * ((experts + 7) / 8 * 8) * sizeof(uint16_t);
}

template <int LPT, int VPL>
static void route_go(const RouteParams& prm, unsigned threads, size_t lds_bytes, hipStream_t s)
{
    const unsigned grid = (unsigned)prm.chunks;
    const bool half = prm.g.logits_bits == 16;
    if (prm.g.bias && half) moe_route_kernel<LPT, VPL, 2, true><<<grid, threads, lds_bytes, s>>>(prm);
    else if (prm.g.bias) moe_route_kernel<LPT, VPL, 2, false><<<grid, threads, lds_bytes, s>>>(prm);
    else if (half) moe_route_kernel<LPT, VPL, 0, true><<<grid, threads, lds_bytes, s>>>(prm);
    else moe_route_kernel<LPT, VPL, 1, false><<<grid, threads, lds_bytes, s>>>(prm);
}

hipError_t launch_moe_route(const MoeRouteArgs& g, hipStream_t s)
{
    RouteParams prm;
    prm.g = g;
    route_chunks(g.tokens, g.experts, g.top, &prm.chunk, &prm.chunks);
    prm.each = std::min(std::max((prm.chunks + kPlacers - 1) / kPlacers, (64 + prm.chunk - 1) / prm.chunk), place_room(g.experts) / (prm.chunk * g.top));
    prm.hist = (uint16_t*)g.workspace;
    prm.padded = (g.experts + 7) / 8 * 8;
    prm.bits = g.experts > 1 ? 32 - __builtin_clz((unsigned)g.experts - 1) : 0;
    const int E = g.experts, lpt = route_lanes(E);
    const int64_t lanes = (int64_t)prm.chunk * lpt;
    const unsigned most = (unsigned)place_threads(E);
    const unsigned routing = std::min(most, (unsigned)route_threads((E > 128 && E <= 256) || E > 512 ? 16 : 8, g.bias != nullptr));
    const unsigned threads = lanes >= routing ? routing : (unsigned)((lanes + 63) / 64 * 64);
    const size_t route_lds = (prm.chunks == 1 ? (size_t)(2 + threads / 64) * E + (size_t)g.tokens * g.top : (size_t)E) * sizeof(int32_t);
    if (E <= 16) route_go<16, 1>(prm, threads, route_lds, s);
    else if (E <= 32) route_go<16, 2>(prm, threads, route_lds, s);
    else if (E <= 64) route_go<16, 4>(prm, threads, route_lds, s);
    else if (E <= 128) route_go<16, 8>(prm, threads, route_lds, s);
    else if (E <= 256) route_go<16, 16>(prm, threads, route_lds, s);
    else if (E <= 512) route_go<64, 8>(prm, threads, route_lds, s);
    else route_go<64, 16>(prm, threads, route_lds, s);
    if (hipError_t e = hipGetLastError()) return e;
    if (prm.chunks > 1) moe_place_kernel<<<(unsigned)((prm.chunks + prm.each - 1) / prm.each), most, (size_t)(2 * prm.padded + std::max((int)(most / 64) * E, prm.padded)) * sizeof(int32_t), s>>>(prm);
    return hipGetLastError();
}

// ---- the products: choice of kernel --------------------------------------------------------------
// Workgroup shapes of the block kernel: 0 (256 x 256, or 192 channels), 3 (128 x 128), 4 (64 x 128).
static int expert_bm(int shape) { return shape == 0 ? 256 : (shape == 3 ? 128 : 64); }
static int expert_bn(int p, int shape) { return shape == 0 ? 64 * bk_expert_nt(p) : 128; }

// Groups of `per` rows that `rows` rows of `experts` experts can make at most.
static int most_groups(int rows, int experts, int per)
{
    return (int)(((int64_t)rows + (int64_t)std::min(experts, rows) * (per - 1)) / per);
}

struct MoePlan {
    bool few;                    // the few-rows kernel, else the block kernel
    int R, kparts, tgroups;      // few
    int shape;                   // block
};

static bool rows_plan(int p, int K, MoePlan* pl)
{
    const int nsuper = (K + kSuperK - 1) / kSuperK;
    for (int R = 1; R <= 4; ++R) {
        const int most = moe_max_waves(p, R);
        if (most == 0 || nsuper > R * most) continue;
        pl->few = true;
        pl->R = R;
        pl->kparts = (nsuper + R - 1) / R;
        pl->tgroups = std::max(1, 8 / pl->kparts);
        return true;
    }
    return false;
}

// Rows of an expert, as far as the host knows: their mean.  The few-rows kernel passes over an expert's weights once for every 16 rows that one has, the
// block kernel's 64 x 128 tiles once for 64, which costs it a launch that packs A; they meet at 8 rows, at 14 where a weight has one or two bits
// (us, few / block: W4A8 eight of 4096->4096, 8 rows 15.4 / 15.7, 12 rows 20.9 / 15.8, 32 rows 33 / 16.3; W2A8 thirty-two 8 rows 29 / 39, 12 rows 35 / 40, 16 rows
// 40 / 41, 32 rows 65 / 43).  Where the block kernel's tiles leave half the units without one, its time is that of one tile, 5.5 us and 0.22 or 0.32 a step, and the
// few-rows kernel's its passes' bytes at 5.7 TB/s and 3.5 us: the lesser of the two, up to 96 rows (us, few / block: W5A8 67 rows of eight 448->320 5.7 / 9.5,
// W8A8 10 rows of eight 4096->512 8.1 / 14.5, W4A8 25 rows of eight 8192->1024 14.8 / 19.2, W8A8 32 rows of four 4096->2048 18.3 / 15.1; over 40 sizes with so few
// tiles the choice takes 1.02 times the lesser time, 1.31 at most: W8A8 37 rows of thirty-two 320->384 11.1 / 8.5).  Tiles of up to 256 rows are ahead from 80 rows
// an expert on where there are 1.2 of them to a compute unit, from 192 on with 0.7; of up to 128 rows from 100 on with one to a unit (us, 64 / 128 / 256 rows a tile:
// W4A8 eight of 4096->4096, 90 rows 26 / 28 / 35, 144 rows 32 / 30 / 45; of 4096->11008, 110 rows 70 / 70 / 66, 180 rows 98 / 94 / 83; W3A8 eight of 8192->2048, 180
// rows 41 / 46 / 71; W8A8 sixty-four of 1408->2048, 180 rows 91 / 86 / 78).  Over 58 drawn sizes of all kinds the choice takes 1.02 times the best kernel's time, 1.20 at
// most.  Rows that are spread less evenly than their mean cost 1.5 times at most of what was measured: 32 tokens that all choose the same two of eight
// W4A8 4096->11008, 22.4 us in two passes, 16.1 with blocks (14.9 where one expert has all rows).
static MoePlan moe_plan(int p, int rows, int N, int K, int experts)
{
    MoePlan pl{};
    const double mean = (double)rows / std::min(experts, rows);   // rows of an expert
    const auto tiles = [&](int shape) {   // about: the last block of an expert is part of one
        const int bm = expert_bm(shape), bn = expert_bn(p, shape);
        return std::min(experts, rows) * std::max(1.0, mean / bm + 0.3) * ((N + bn - 1) / bn);
    };
    bool few = mean <= (p <= 2 ? 14 : 8);
    if (!few && mean <= 96 && tiles(4) <= 0.5 * num_cus()) {
        const double passes = mean / 16 + 0.5, weights = (double)std::min(experts, rows) * p * N * K / 8;
        few = 3.5 + passes * weights / 5.7e6 < 5.5 + (K + 127) / 128 * (p <= 4 ? 0.22 : 0.32);
    }
    if (K >= 16 && few && rows_plan(p, K, &pl)) return pl;
    pl.shape = (mean >= 80 && tiles(0) >= 1.2 * num_cus()) || (mean >= 192 && tiles(0) >= 0.7 * num_cus()) ? 0 : (mean >= 100 && tiles(3) >= num_cus() ? 3 : 4);
    return pl;
}

size_t moe_gemm_workspace_bytes(int p, int q, int rows, int N, int K, int tokens, int experts)
{
    if (moe_plan(p, rows, N, K, experts).few) return 0;
    ActLayout A;
    make_act_layout(q, tokens, K, ABQ_LAYOUT_FIELDS, &A);
    return A.total;
}

static MoeGroups groups_of(const MoeGemmArgs& g) { return MoeGroups{g.starts, g.order, g.experts, g.rows, g.tokens, g.top}; }

hipError_t launch_moe_gemm(const MoeGemmArgs& g, const WeightLayout& W, hipStream_t s)
{
    const MoePlan pl = moe_plan(g.p, g.rows, g.N, g.K, g.experts);
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
        prm.batch = moe_batch(pl.kparts);
        prm.groups_n = (W.NT + pl.tgroups - 1) / pl.tgroups;
        prm.most = most_groups(g.rows, g.experts, 16);
        const int waves = pl.kparts * pl.tgroups, room = moe_max_waves(g.p, pl.R);   // (waves a unit holds)
        const unsigned grid = (unsigned)std::min<int64_t>((int64_t)num_cus() * std::max(1, room / waves), (int64_t)prm.most * prm.groups_n);
        switch (g.p) {
            case 1: return moe_rows_launch_p1(prm, pl.R, grid, s);
            case 2: return moe_rows_launch_p2(prm, pl.R, grid, s);
            case 3: return moe_rows_launch_p3(prm, pl.R, grid, s);
            case 4: return moe_rows_launch_p4(prm, pl.R, grid, s);
            case 5: return moe_rows_launch_p5(prm, pl.R, grid, s);
            case 6: return moe_rows_launch_p6(prm, pl.R, grid, s);
            case 7: return moe_rows_launch_p7(prm, pl.R, grid, s);
            default: return moe_rows_launch_p8(prm, pl.R, grid, s);
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

// One workgroup per token and run of up to 256 eights of its row; the terms are added in the order of the choices, in binary32.  Memory bounds it: 4099 tokens of
// eight rows of 5120 87 us, 4.8 TB/s.
__global__ __launch_bounds__(256) void moe_combine_kernel(CombineParams prm)
{
    const int64_t t = blockIdx.x;
    const int v = blockIdx.y * blockDim.x + threadIdx.x;
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
    const int eights = (N + 7) / 8, threads = std::min(256, (eights + 63) / 64 * 64);
    moe_combine_kernel<<<dim3((unsigned)tokens, (unsigned)((eights + threads - 1) / threads)), threads, 0, s>>>(prm);
    return hipGetLastError();
}

}  // namespace abq
