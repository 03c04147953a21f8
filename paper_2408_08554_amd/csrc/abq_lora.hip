// Low-rank adapters of many requests beside a shared projection: out = y + scale_i B_i (A_i x), i the row's adapter.
//
// Two kernels, both on tiles of sixteen rows: u = A_i x (parts of K side by side, binary32), then the rows of the output.  A tile goes
// through the distinct adapters of its rows one after the other: each adapter's matrices are read once per tile, whatever the order of
// the rows, and a row takes the result of its own adapter alone (the others' are discarded lane by lane, not multiplied by zero, so that
// an infinity in one request's adapter stays there).
//
// What bounds it: one token is latency (two launches and what each waits for), many adapters are their matrices, a prompt is
// reading and writing y.
#include "abq_kv.h"
#include "abq_rows.h"

#include <algorithm>

namespace abq {

typedef _Float16 lh8 __attribute__((ext_vector_type(8)));
typedef float lf4 __attribute__((ext_vector_type(4)));
typedef uint32_t lu4 __attribute__((ext_vector_type(4)));

// Eight halves of a row of n from element k on, zeros behind its end.
__device__ __forceinline__ lu4 load_eight(const uint16_t* row, int k, int n)
{
    if (k + 8 <= n) {
        const u32x4_half v = *reinterpret_cast<const u32x4_half*>(row + k);
        return lu4{v.x, v.y, v.z, v.w};
    }
    lu4 v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 7; ++e)
        if (k + e < n) v[e >> 1] |= (uint32_t)row[k + e] << (16 * (e & 1));
    return v;
}

// The distinct adapters of sixteen rows, one after the other (lane l: row l % 16).
struct Adapters {
    int id;          // of the lane's row, -1 for none
    uint32_t left;   // rows whose adapter has not had its turn
    __device__ __forceinline__ Adapters(const int32_t* ids, int m, int M, int adapters)
    {
        const int v = m < M ? ids[m] : -1;
        id = (unsigned)v < (unsigned)adapters ? v : -1;
        left = (uint32_t)__ballot(id >= 0) & 0xFFFFu;
    }
    __device__ __forceinline__ int next()   // -1: all had theirs
    {
        if (!left) return -1;
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(left));
        left &= ~(uint32_t)__ballot(id == a);
        return a;
    }
};

// u[part][m][r] = sum over a part of K of A_i[r][k] x[m][k].  A workgroup: sixteen rows, a part of K (its four waves a quarter each),
// the adapters number blockIdx.y, blockIdx.y + gridDim.y, ... of the tile.  RT tiles of sixteen ranks share a load of x.
template <int RT>
__global__ __launch_bounds__(256) void lora_shrink_kernel(int M, int K, int rank, int adapters, int slice, const uint16_t* __restrict__ x, int ldx, const int32_t* __restrict__ ids,
                                                          const uint16_t* __restrict__ a, float* __restrict__ u)
{
    __shared__ lf4 part[4][RT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int m = blockIdx.z * 16 + n16, quarter = slice >> 2;
    Adapters turn(ids, m, M, adapters);
    const uint16_t* const xr = x + (size_t)min(m, M - 1) * ldx;
    const int k0 = blockIdx.x * slice + wave * quarter, k1 = min(K, k0 + quarter);   // (quarters are whole steps of 32)
    int nth = 0;
    for (int i = turn.next(); i >= 0; i = turn.next(), ++nth) {
        if (nth % (int)gridDim.y != (int)blockIdx.y) continue;
        const uint16_t* row[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) row[t] = a + ((size_t)i * rank + min(16 * t + n16, rank - 1)) * K;
        lf4 acc[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = lf4{0, 0, 0, 0};
        int k = k0;
        constexpr int AHEAD = RT <= 2 ? 4 : RT <= 4 ? 2 : 1;   // steps whose loads are in flight together
        for (; k + 32 * AHEAD <= k1; k += 32 * AHEAD) {
            lu4 xv[AHEAD], av[AHEAD][RT];
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
                const u32x4_half v = *reinterpret_cast<const u32x4_half*>(xr + k + 32 * s + 8 * g);
                xv[s] = lu4{v.x, v.y, v.z, v.w};
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    const u32x4_half w = *reinterpret_cast<const u32x4_half*>(row[t] + k + 32 * s + 8 * g);
                    av[s][t] = lu4{w.x, w.y, w.z, w.w};
                }
            }
#pragma unroll
            for (int s = 0; s < AHEAD; ++s)
#pragma unroll
                for (int t = 0; t < RT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lh8, av[s][t]), __builtin_bit_cast(lh8, xv[s]), acc[t], 0, 0, 0);
        }
        for (; k < k1; k += 32) {
            const lu4 xv = load_eight(xr, k + 8 * g, K);
#pragma unroll
            for (int t = 0; t < RT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lh8, load_eight(row[t], k + 8 * g, K)), __builtin_bit_cast(lh8, xv), acc[t], 0, 0, 0);
        }
        __syncthreads();   // (the adapter before is stored)
#pragma unroll
        for (int t = 0; t < RT; ++t) part[wave][t][lane] = acc[t];
        __syncthreads();
        // a lane's four values: ranks 16 t + 4 g .. of row n16
        if (turn.id == i) {
            float* const dst = u + ((size_t)blockIdx.x * M + m) * rank;
            for (int t = wave; t < RT; t += 4) {
                const lf4 v = part[0][t][lane] + part[1][t][lane] + (part[2][t][lane] + part[3][t][lane]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (16 * t + 4 * g + e < rank) dst[16 * t + 4 * g + e] = v[e];
            }
        }
    }
}

// The rows of the output.  A workgroup: sixteen rows, `blocks` blocks of 256 columns (its waves 64 each).  u enters the product as two
// halves, hi + lo, of u over the power of two above its row's largest element: 22 bits of it, for one matrix instruction per sixteen ranks
// (16 k of hi, 16 of lo).  The rows of B are dealt to the operand's rows so that a lane ends with sixteen neighbouring columns of one row.
__global__ __launch_bounds__(256) void lora_expand_kernel(int M, int N, int rank, int adapters, int parts, int blocks, const int32_t* __restrict__ ids, const uint16_t* __restrict__ b,
                                                          const float* __restrict__ scale, const float* __restrict__ u, const uint16_t* y, int ldy, uint16_t* out, int ldout)
{
    constexpr int US = 256 + 8;   // halves of a row of u in LDS
    __shared__ __align__(16) uint16_t hi[16 * US], lo[16 * US];
    __shared__ float factor[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.y * 16, m = m0 + n16, RT = (rank + 15) >> 4;
    const Adapters rows(ids, m, M, adapters);

    {   // sixteen threads a row: its parts added, the largest element, the two halves
        const int r = tid >> 4, c = tid & 15, row = min(m0 + r, M - 1), id = ids[row];
        const bool there = m0 + r < M && (unsigned)id < (unsigned)adapters;
        float v[16], top = 0.0f;
        const float* src = u + (size_t)row * rank;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            v[t] = 0.0f;
            if (t < RT && there && 16 * t + c < rank) {
                for (int p = 0; p < parts; ++p) v[t] += src[(size_t)p * M * rank + 16 * t + c];
                top = fmaxf(top, fabsf(v[t]));
            }
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        int e = 0;
        if (top > 0.0f && top < INFINITY) (void)frexpf(top, &e);
        if (c == 0) factor[r] = there ? ldexpf(scale[id], e) : 0.0f;
#pragma unroll
        for (int t = 0; t < 16; ++t)
            if (t < RT) {
                const float w = ldexpf(v[t], -e);
                const __half h = __float2half_rn(w);
                hi[r * US + 16 * t + c] = __half_as_ushort(h);
                lo[r * US + 16 * t + c] = __half_as_ushort(__float2half_rn(w - __half2float(h)));
            }
    }
    __syncthreads();
    const float f = factor[n16];
    const uint16_t* const us = (g < 2 ? hi : lo) + n16 * US + 8 * (g & 1);

    for (int blk = 0; blk < blocks; ++blk) {
        const int n0 = (blockIdx.x * blocks + blk) * 256 + wave * 64;
        if (n0 >= N) return;
        // y of this lane's columns
        const int n = n0 + 16 * g;
        const uint16_t* const yr = y + (size_t)min(m, M - 1) * ldy;
        lu4 yv[2] = {lu4{0, 0, 0, 0}, lu4{0, 0, 0, 0}};
        if (m < M) {
            yv[0] = load_eight(yr, n, N);
            yv[1] = load_eight(yr, n + 8, N);
        }
        lf4 res[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) res[t] = lf4{0, 0, 0, 0};
        // operand row n16 of tile t: column n0 + 16 (n16 / 4) + 4 t + n16 % 4
        int nb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) nb[t] = min(n0 + 16 * (n16 >> 2) + 4 * t + (n16 & 3), N - 1);
        auto load = [&](int i, int rt, lu4* v) {
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = load_eight(b + ((size_t)i * N + nb[t]) * rank, 16 * rt + 8 * (g & 1), rank);
        };
        Adapters turn = rows;
        int i = turn.next();
        lu4 bv[4];
        if (i >= 0) load(i, 0, bv);
        while (i >= 0) {
            const int then = turn.next();
            lf4 acc[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = lf4{0, 0, 0, 0};
            for (int rt = 0; rt < RT; ++rt) {
                lu4 nv[4];   // the next sixteen ranks, or the next adapter's first
                const bool more = rt + 1 < RT;
                if (more || then >= 0) load(more ? i : then, more ? rt + 1 : 0, nv);
                const lh8 uv = *reinterpret_cast<const lh8*>(us + 16 * rt);
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lh8, bv[t]), uv, acc[t], 0, 0, 0);
#pragma unroll
                for (int t = 0; t < 4; ++t) bv[t] = nv[t];
            }
            if (rows.id == i) {
#pragma unroll
                for (int t = 0; t < 4; ++t) res[t] = acc[t];
            }
            i = then;
        }
        if (m < M) {
            if (rows.id >= 0) {   // (a row without an adapter keeps its bits)
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint32_t w = yv[e >> 3][(e & 7) >> 1];
                    const float v0 = fmaf(f, res[e >> 2][e & 3], __half2float(__ushort_as_half((unsigned short)w)));
                    const float v1 = fmaf(f, res[e >> 2][(e & 3) + 1], __half2float(__ushort_as_half((unsigned short)(w >> 16))));
                    yv[e >> 3][(e & 7) >> 1] = (uint32_t)__half_as_ushort(__float2half_rn(v0)) | (uint32_t)__half_as_ushort(__float2half_rn(v1)) << 16;
                }
            }
            uint16_t* const dst = out + (size_t)m * ldout;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (n + 8 * h < N) store_row_part8(dst + n + 8 * h, n + 8 * h, N, yv[h][0], yv[h][1], yv[h][2], yv[h][3]);
        }
    }
}

// Parts of K, each a whole number of steps for four waves: few tiles of rows leave the chip idle and want many short parts, but the
// second kernel adds them up once per workgroup.
struct LoraPlan { int slice, parts; };
static LoraPlan lora_plan(int M, int K)
{
    const int tiles = (M + 15) / 16, wgs = tiles * std::min(M, 8);   // (a tile of a few requests has as many adapters)
    const int want = std::max(1, std::min({256 / std::max(wgs, 1), (K + 255) / 256, 16}));
    LoraPlan p;
    p.slice = ((K + want - 1) / want + 127) / 128 * 128;
    p.parts = (K + p.slice - 1) / p.slice;
    return p;
}

size_t lora_workspace_bytes(int M, int, int K, int rank) { return (size_t)lora_plan(M, K).parts * M * rank * sizeof(float); }

hipError_t launch_lora_add(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a,
                           const uint16_t* b, const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout, void* workspace,
                           hipStream_t s)
{
    const LoraPlan p = lora_plan(M, K);
    const int tiles = (M + 15) / 16;
    float* const u = (float*)workspace;
    // distinct adapters of a tile side by side where the tiles alone are few
    const dim3 grid(p.parts, tiles <= 16 ? std::min({M, adapters, 16}) : 1, tiles);
#define ABQ_LORA_SHRINK(RT) lora_shrink_kernel<RT><<<grid, 256, 0, s>>>(M, K, rank, adapters, p.slice, x, ldx, ids, a, u)
    if (rank <= 16) ABQ_LORA_SHRINK(1);
    else if (rank <= 32) ABQ_LORA_SHRINK(2);
    else if (rank <= 64) ABQ_LORA_SHRINK(4);
    else if (rank <= 128) ABQ_LORA_SHRINK(8);
    else ABQ_LORA_SHRINK(16);
#undef ABQ_LORA_SHRINK
    const int64_t columns = ((int64_t)N + 255) / 256;
    const int blocks = columns * tiles >= 2048 ? 4 : 1;
    lora_expand_kernel<<<dim3((unsigned)((columns + blocks - 1) / blocks), tiles), 256, 0, s>>>(M, N, rank, adapters, p.parts, blocks, ids, b, scale, u, y, ldy, out, ldout);
    return hipGetLastError();
}

}  // namespace abq
