// A layer of experts as the kernels see it: rows sorted by expert, in ragged groups that only device memory knows.
#pragma once
#include "abq_internal.h"

namespace abq {

struct MoeGemmArgs {
    int p, q, rows, N, K, tokens, experts, top;
    const uint8_t* a_codes;
    const float* a_scale;
    const int32_t* a_zero;
    const uint8_t* w_blobs;
    size_t w_stride;          // bytes from one expert's blob to the next
    const int32_t *starts, *order;
    uint16_t* y;
    void* workspace;
};
size_t moe_gemm_workspace_bytes(int p, int q, int rows, int N, int K, int tokens, int experts);
hipError_t launch_moe_gemm(const MoeGemmArgs& g, const WeightLayout& W, hipStream_t s);

struct MoeRouteArgs {
    int tokens, experts, top, logits_bits, ld;
    const void* logits;
    const float* bias;
    bool sigmoid, renormalize;
    float scale;
    int32_t* ids;
    float* weights;
    int32_t *starts, *order, *places;
    void* workspace;
};
size_t moe_route_workspace_bytes(int tokens, int experts, int top);
hipError_t launch_moe_route(const MoeRouteArgs& g, hipStream_t s);
hipError_t launch_moe_combine(int tokens, int N, int rows, int top, const uint16_t* y, int ldy, const int32_t* places, const float* weights,
                              const uint16_t* add, int ldadd, uint16_t* out, int ldout, hipStream_t s);

// ---- the few-rows kernel and the block kernel of experts: parameters, entry points of the per-width translation units --------------
struct MoeGroups {            // the groups of rows
    const int32_t *starts, *order;
    int experts, rows, tokens, top;
};
struct MoeRowsParams {
    const uint8_t* w;         // blob of expert 0
    size_t w_stride, off_params, off_fields[3];
    const uint8_t* a;         // codes [tokens][K]
    const float* a_scale;
    const int32_t* a_zero;
    uint16_t* y;
    MoeGroups g;
    int N, K, nsuper, ntiles;
    int oa, ow;
    uint32_t a_mask;
    int kparts, tgroups;      // waves of a workgroup: parts of K, tiles side by side
    int batch;                // tiles between two barriers
    int groups_n;             // tile groups of an expert
    int most;                 // groups of 16 rows there can be
};
struct BlockExpertParams;     // (abq_block_kernels.h)

// Units of `per` rows of the experts, for a whole wave: how many there are, and which expert a unit belongs to.  What `starts` holds is taken
// into 0..rows first, so that nothing outside the rows is ever touched.
struct ExpertAt { int expert, before, first, rows; };   // the expert, the units of those before it, its first row, its rows

__device__ __forceinline__ void moe_expert_rows(const MoeGroups& g, int e, int* first, int* rows)
{
    const int a = g.starts[min(e, g.experts)], b = g.starts[min(e + 1, g.experts)];   // (no expert: none between them)
    const int lo = min(max(a, 0), g.rows), hi = min(max(b, 0), g.rows);
    *first = lo;
    *rows = max(hi - lo, 0);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int moe_moved(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, true); }
__device__ __forceinline__ int moe_scan(int x)   // sums over this lane and those before it
{
    x += moe_moved<0x111, 0xF>(x);   // inside the rows of sixteen, from 1, 2, 4 and 8 lanes before
    x += moe_moved<0x112, 0xF>(x);
    x += moe_moved<0x114, 0xF>(x);
    x += moe_moved<0x118, 0xF>(x);
    x += moe_moved<0x142, 0xA>(x);   // the last lane of the first and third row to the row behind
    x += moe_moved<0x143, 0xC>(x);   // lane 31 to the upper half
    return x;
}
// UNITS: how many units so many rows are.
template <class UNITS>
struct ExpertUnits {
    UNITS of;
    int first0, rows0, sum0, total;   // of lane's expert among the first 64: first row, rows, units up to and with it; all units
    // at most `most` units (starts that do not ascend could name more)
    __device__ __forceinline__ ExpertUnits(const MoeGroups& g, UNITS of, int most) : of(of)
    {
        const int lane = threadIdx.x & 63;
        moe_expert_rows(g, lane, &first0, &rows0);
        sum0 = moe_scan(of(rows0));
        total = min(__builtin_amdgcn_readlane(sum0, 63), most);
        for (int e0 = 64; e0 < g.experts; e0 += 64) {
            int first, rows;
            moe_expert_rows(g, e0 + lane, &first, &rows);
            total = min(total + __builtin_amdgcn_readlane(moe_scan(of(rows)), 63), most);
        }
    }
    // u < total
    __device__ __forceinline__ ExpertAt find(const MoeGroups& g, int u) const
    {
        const int lane = threadIdx.x & 63;
        int first = first0, rows = rows0, sum = sum0, before = 0;
        for (int e0 = 0;; e0 += 64) {
            const int at = __popcll(__ballot(before + sum <= u));   // experts that end at or before it
            if (at < 64 || e0 + 64 >= g.experts) {
                const int l = min(at, 63);
                ExpertAt r;
                r.expert = min(e0 + l, g.experts - 1);
                r.before = before + (l ? __builtin_amdgcn_readlane(sum, l - 1) : 0);
                r.first = __builtin_amdgcn_readlane(first, l);
                r.rows = __builtin_amdgcn_readlane(rows, l);
                return r;
            }
            before += __builtin_amdgcn_readlane(sum, 63);
            moe_expert_rows(g, e0 + 64 + lane, &first, &rows);
            sum = moe_scan(of(rows));
        }
    }
};
// Blocks of `per` rows, the last one with what is left.
struct BlocksOf {
    static constexpr bool kLast = false;
    int per;
    __device__ __forceinline__ int operator()(int rows) const { return (rows + per - 1) / per; }
};
// Of those with LO + 1 .. HI rows.
template <int PER, int LO, int HI>
struct BlocksBetween {
    static constexpr bool kLast = HI != PER;   // an expert has one at most, its last
    __device__ __forceinline__ int operator()(int rows) const { return (HI == PER ? rows / PER : 0) + (rows % PER > LO && rows % PER <= HI ? 1 : 0); }
};

// Row of A of a sorted row (an entry of `order` that names none takes the nearest there is): what there is to load, and what it says.
__device__ __forceinline__ int moe_order(const MoeGroups& g, int row) { return g.order ? g.order[row] : row; }
__device__ __forceinline__ int moe_row(const MoeGroups& g, int entry) { return min((int)((unsigned)max(entry, 0) / (unsigned)g.top), g.tokens - 1); }
__device__ __forceinline__ int moe_row_of(const MoeGroups& g, int row) { return moe_row(g, moe_order(g, row)); }

}  // namespace abq
