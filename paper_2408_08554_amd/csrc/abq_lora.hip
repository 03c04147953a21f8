// Low-rank adapters of many requests beside a shared projection: out = y + scale_i B_i (A_i x), i the row's adapter.
//
// Two kernels, both on tiles of sixteen rows: u = A_i x (parts of K side by side, binary32), then the rows of the output.  A tile goes
// through the distinct adapters of its rows one after the other: each adapter's matrices are read once per tile, whatever the order of
// the rows, and a row takes the result of its own adapter alone (the others' are discarded lane by lane, not multiplied by zero, so that
// an infinity in one request's adapter stays there).
//
// What bounds it: one token is latency (two launches and what each waits for: rank 16, 4096 to 4096, 3.3 + 4.1 us); 64 rows of 32
// adapters too, though less (rank 16, 4096 to 11008: 18.8 MB in 5.3 + 7.7 us, 1.4 TB/s); a prompt is reading and writing y, at 3 TB/s
// (2048 rows, rank 64, 5120 to 13824: 113 MB of y in 37 us, u in 12 + 4): a workgroup's waves wait for ids, u and B
// before their y can leave, and the accumulators of 64 x 64 leave room for two of them on a unit.
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

// The same where all eight are there.  (No branch: a load that only some lanes take makes every later one wait for it.)
__device__ __forceinline__ lu4 load_whole(const uint16_t* p)
{
    const u32x4_half v = *reinterpret_cast<const u32x4_half*>(p);
    return lu4{v.x, v.y, v.z, v.w};
}

// The distinct adapters of up to 64 rows (lane l: row l), one after the other.
struct Adapters {
    int id;          // of the lane's row, -1 for none
    uint64_t left;   // rows whose adapter has not had its turn
    __device__ __forceinline__ Adapters(const int32_t* ids, int m, int M, int adapters, bool mine)
    {
        const int v = mine && m < M ? ids[m] : -1;
        id = (unsigned)v < (unsigned)adapters ? v : -1;
        left = __ballot(id >= 0);
    }
    __device__ __forceinline__ int next(uint64_t* rows)   // its rows; -1: all had theirs
    {
        if (!left) return -1;
        const int a = __builtin_amdgcn_readlane(id, __builtin_ctzll(left));
        *rows = __ballot(id == a);
        left &= ~*rows;
        return a;
    }
};

// u[part][m][r] = sum over a part of K of A_i[r][k] x[m][k].  A workgroup: MT tiles of sixteen rows, a part of K (its four waves a
// quarter each), the adapters number blockIdx.y, blockIdx.y + gridDim.y, ... of its rows.  RT tiles of sixteen ranks share a load of x,
// the tiles of rows one of A (a tile without rows of the adapter goes through it all the same: prompts have few adapters to a tile).
template <int RT, int MT>
__global__ __launch_bounds__(256) void lora_shrink_kernel(int M, int K, int rank, int adapters, int slice, const uint16_t* __restrict__ x, int ldx, const int32_t* __restrict__ ids,
                                                          const uint16_t* __restrict__ a, float* __restrict__ u)
{
    __shared__ lf4 part[4][RT * MT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.z * 16 * MT, quarter = slice >> 2;
    Adapters turn(ids, m0 + lane, M, adapters, lane < 16 * MT);
    const uint16_t* xr[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) xr[j] = x + (size_t)min(m0 + 16 * j + n16, M - 1) * ldx;
    const int k0 = blockIdx.x * slice + wave * quarter, k1 = min(K, k0 + quarter);   // (quarters are whole steps of 32)
    int nth = 0;
    uint64_t rows = 0;
    for (int i = turn.next(&rows); i >= 0; i = turn.next(&rows), ++nth) {
        if (nth % (int)gridDim.y != (int)blockIdx.y) continue;
        const uint16_t* row[RT];
#pragma unroll
        for (int t = 0; t < RT; ++t) row[t] = a + ((size_t)i * rank + min(16 * t + n16, rank - 1)) * K;
        lf4 acc[RT][MT];
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int j = 0; j < MT; ++j) acc[t][j] = lf4{0, 0, 0, 0};
        auto step = [&](const lu4* av, const lu4* xv) {
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int j = 0; j < MT; ++j) acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lh8, av[t]), __builtin_bit_cast(lh8, xv[j]), acc[t][j], 0, 0, 0);
        };
        int k = k0;
        constexpr int AHEAD = RT + MT <= 3 ? 4 : RT + MT <= 9 ? 2 : 1;   // steps whose loads are in flight together
        for (; k + 32 * AHEAD <= k1; k += 32 * AHEAD) {
            lu4 xv[AHEAD][MT], av[AHEAD][RT];
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) {
#pragma unroll
                for (int j = 0; j < MT; ++j) xv[s][j] = load_whole(xr[j] + k + 32 * s + 8 * g);
#pragma unroll
                for (int t = 0; t < RT; ++t) av[s][t] = load_whole(row[t] + k + 32 * s + 8 * g);
            }
#pragma unroll
            for (int s = 0; s < AHEAD; ++s) step(av[s], xv[s]);
        }
        for (; k < k1; k += 32) {
            lu4 xv[MT], av[RT];
#pragma unroll
            for (int j = 0; j < MT; ++j) xv[j] = load_eight(xr[j], k + 8 * g, K);
#pragma unroll
            for (int t = 0; t < RT; ++t) av[t] = load_eight(row[t], k + 8 * g, K);
            step(av, xv);
        }
        __syncthreads();   // (the adapter before is stored)
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int j = 0; j < MT; ++j) part[wave][t * MT + j][lane] = acc[t][j];
        __syncthreads();
        // a lane's four values: ranks 16 t + 4 g .. of row 16 j + n16
        for (int q = wave; q < RT * MT; q += 4) {
            const int t = q / MT, j = q % MT;
            if (!(rows >> (16 * j + n16) & 1)) continue;
            const lf4 v = part[0][q][lane] + part[1][q][lane] + (part[2][q][lane] + part[3][q][lane]);
            float* const dst = u + ((size_t)blockIdx.x * M + m0 + 16 * j + n16) * rank + 16 * t + 4 * g;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (16 * t + 4 * g + e < rank) dst[e] = v[e];
        }
    }
}

// u enters the second product as two halves, hi + lo, of u over the power of two above its row's largest element: 22 bits of it, for one
// matrix instruction per sixteen ranks (16 k of hi, 16 of lo).
__device__ __forceinline__ void split_u(float v, int e, uint16_t* hi, uint16_t* lo)
{
    const float w = ldexpf(v, -e);
    const __half h = __float2half_rn(w);
    *hi = __half_as_ushort(h);
    *lo = __half_as_ushort(__float2half_rn(w - __half2float(h)));
}
__device__ __forceinline__ int exponent_above(float top) { return top > 0.0f && top < INFINITY ? __builtin_amdgcn_frexp_expf(top) : 0; }

// Many rows: the parts of u added up and split once, a wave a row, where every workgroup of the second kernel would do it over.
// halves [M][2][padded]: hi, lo, zeros behind the rank; factor [M]: the adapter's scale times the row's power of two.
__global__ __launch_bounds__(256) void lora_split_kernel(int M, int rank, int padded, int adapters, int parts, const int32_t* __restrict__ ids, const float* __restrict__ scale,
                                                         const float* __restrict__ u, uint16_t* __restrict__ halves, float* __restrict__ factor)
{
    const int m = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (m >= M) return;
    const int id = ids[m];
    const bool there = (unsigned)id < (unsigned)adapters;
    float v[4], top = 0.0f;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v[q] = 0.0f;
        if (64 * q >= rank) continue;
        const int r = min(64 * q + lane, rank - 1);
        float w[16];
#pragma unroll
        for (int p = 0; p < 16; ++p) w[p] = u[((size_t)min(p, parts - 1) * M + m) * rank + r];
#pragma unroll
        for (int p = 0; p < 16; ++p) v[q] += p < parts ? w[p] : 0.0f;
        if (!there || 64 * q + lane >= rank) v[q] = 0.0f;
        top = fmaxf(top, fabsf(v[q]));
    }
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
    const int e = exponent_above(top);
    if (lane == 0) factor[m] = there ? ldexpf(scale[id], e) : 0.0f;
    uint16_t* const dst = halves + (size_t)m * 2 * padded;
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (64 * q + lane < padded) split_u(v[q], e, dst + 64 * q + lane, dst + padded + 64 * q + lane);
}

// The rows of the output.  A workgroup: MT tiles of sixteen rows; its waves take blocks of 64 columns, `blocks` each (SPREAD: one block
// for all four, and every fourth adapter each).  The rows of B are dealt to the operand's rows so that a lane ends with twice eight
// neighbouring columns of one row, and four lanes with twice 32.  FAST: a rank of whole eights, columns of whole blocks; the branches that the others need for their
// ends cost a third of the time.  SPLIT: u comes split, else in parts.
template <int RT, int MT, bool SPREAD, bool FAST, bool SPLIT>
__global__ __launch_bounds__(256, MT == 4 && FAST ? 2 : 1) void lora_expand_kernel(int M, int N, int rank, int adapters, int parts, int blocks, const int32_t* __restrict__ ids, const uint16_t* __restrict__ b,
                                                          const float* __restrict__ scale, const float* __restrict__ u, const uint16_t* __restrict__ halves, const float* __restrict__ factors,
                                                          const uint16_t* y, int ldy, uint16_t* out, int ldout)
{
    constexpr int RP = 16 * RT, US = 2 * RP + 8;   // halves of a row of u, hi and lo, in LDS
    __shared__ __align__(16) uint16_t us[16 * MT * US];
    __shared__ float factor[16 * MT];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, g = lane >> 4;
    const int m0 = blockIdx.y * 16 * MT;
    Adapters all(ids, m0 + lane, M, adapters, lane < 16 * MT);
    const int n0 = SPREAD ? blockIdx.x * 64 : (blockIdx.x * 4 * blocks + wave) * 64;   // the wave's first block

    // y of the first block, on its way early
    lu4 yv[MT][2];
    auto load_y = [&](int at) {
        const int n = at + 8 * g;
#pragma unroll
        for (int j = 0; j < MT; ++j) {
            const uint16_t* const yr = y + (size_t)min(m0 + 16 * j + n16, M - 1) * ldy;
            if (FAST || at + 64 <= N) {
                yv[j][0] = load_whole(yr + n);
                yv[j][1] = load_whole(yr + n + 32);
            } else {
                yv[j][0] = load_eight(yr, n, N);
                yv[j][1] = load_eight(yr, n + 32, N);
            }
        }
    };
    if constexpr (SPLIT) {
        constexpr int EACH = 2 * RP / 8, ALL = 16 * MT * EACH, VT = (ALL + 255) / 256;   // vectors of eight halves
        lu4 v[VT];
#pragma unroll
        for (int i = 0; i < VT; ++i) {
            const int at = min(i * 256 + tid, ALL - 1);
            v[i] = *reinterpret_cast<const lu4*>(halves + (size_t)min(m0 + at / EACH, M - 1) * 2 * RP + 8 * (at % EACH));
        }
        const float f = factors[min(m0 + tid % (16 * MT), M - 1)];
        if (n0 < N) load_y(n0);   // (behind what is waited for)
#pragma unroll
        for (int i = 0; i < VT; ++i) {
            const int at = i * 256 + tid;
            if (ALL % 256 == 0 || at < ALL) *reinterpret_cast<lu4*>(us + at / EACH * US + 8 * (at % EACH)) = v[i];
        }
        if (tid < 16 * MT) factor[tid] = f;
    } else {
        if (n0 < N) load_y(n0);
#pragma unroll
        for (int j = 0; j < MT; ++j) {   // sixteen threads a row: its parts added, the largest element, the two halves
            const int r = 16 * j + (tid >> 4), c = tid & 15, row = min(m0 + r, M - 1);
            constexpr int PB = RT <= 4 ? 16 / RT : 4;   // parts whose loads are in flight together
            float v[RT], top = 0.0f;
#pragma unroll
            for (int t = 0; t < RT; ++t) v[t] = 0.0f;
            for (int p0 = 0; p0 < parts; p0 += PB) {
                float w[PB][RT];
#pragma unroll
                for (int p = 0; p < PB; ++p)
#pragma unroll
                    for (int t = 0; t < RT; ++t) w[p][t] = u[((size_t)min(p0 + p, parts - 1) * M + row) * rank + min(16 * t + c, rank - 1)];
#pragma unroll
                for (int p = 0; p < PB; ++p)
#pragma unroll
                    for (int t = 0; t < RT; ++t) v[t] += p0 + p < parts ? w[p][t] : 0.0f;
            }
            const int mine = __shfl(all.id, r, 64);
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if (mine < 0 || 16 * t + c >= rank) v[t] = 0.0f;
                top = fmaxf(top, fabsf(v[t]));
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
            const int e = exponent_above(top);
            if (c == 0) factor[r] = mine >= 0 ? ldexpf(scale[mine], e) : 0.0f;
#pragma unroll
            for (int t = 0; t < RT; ++t) split_u(v[t], e, us + r * US + 16 * t + c, us + r * US + RP + 16 * t + c);
        }
    }
    __syncthreads();
    const uint16_t* const mine = us + n16 * US + (g < 2 ? 0 : RP) + 8 * (g & 1);

    for (int blk = 0; blk < blocks; ++blk) {
        const int at = n0 + blk * 256, n = at + 8 * g;
        if (at >= N) return;
        if (blk) load_y(at);
        auto store = [&](int j) {
            uint16_t* const dst = out + (size_t)(m0 + 16 * j + n16) * ldout;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (FAST) *reinterpret_cast<u32x4_half*>(dst + n + 32 * h) = u32x4_half{yv[j][h][0], yv[j][h][1], yv[j][h][2], yv[j][h][3]};
                else if (n + 32 * h < N) store_row_part8(dst + n + 32 * h, n + 32 * h, N, yv[j][h][0], yv[j][h][1], yv[j][h][2], yv[j][h][3]);
            }
        };
        // operand row n16 of tile t: column at + 32 (t / 2) + 8 (n16 / 4) + 4 (t % 2) + n16 % 4
        int nb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) nb[t] = min(at + 32 * (t >> 1) + 8 * (n16 >> 2) + 4 * (t & 1) + (n16 & 3), N - 1);
        auto load = [&](int i, int rt, lu4* v) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint16_t* const row = b + ((size_t)i * N + nb[t]) * rank;
                const int r = 16 * rt + 8 * (g & 1);
                if constexpr (FAST) {
                    v[t] = load_whole(row + min(r, rank - 8));
                    if (r >= rank) v[t] = lu4{0, 0, 0, 0};
                } else {
                    v[t] = load_eight(row, r, rank);
                }
            }
        };
        Adapters turn = all;
        uint64_t rows = 0, then_rows = 0;
        int nth = 0;
        auto next = [&](uint64_t* r) {
            for (;;) {
                const int i = turn.next(r);
                if (!SPREAD || i < 0 || (nth++ & 3) == wave) return i;
            }
        };
        // An adapter's operands on their way together as far as registers go: up to two tiles of ranks, the next adapter's too.
        constexpr int LOADED = RT <= 4 ? RT : 2;
        constexpr bool NEXT = RT <= 2;
        int i = next(&rows);
        lu4 bv[LOADED][4];
        auto load_first = [&](int of, lu4 (*v)[4]) {
#pragma unroll
            for (int rt = 0; rt < LOADED; ++rt) load(of, rt, v[rt]);
        };
        if (i >= 0 && NEXT) load_first(i, bv);
        while (i >= 0) {
            const int then = next(&then_rows);
            lu4 nv[NEXT ? LOADED : 1][4];
            if constexpr (NEXT) load_first(then >= 0 ? then : i, nv);
            else load_first(i, bv);
            lf4 acc[MT][4];
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[j][t] = lf4{0, 0, 0, 0};
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                lu4 now[4];
#pragma unroll
                for (int t = 0; t < 4; ++t) now[t] = bv[rt % LOADED][t];
                if (rt + LOADED < RT) load(i, rt + LOADED, bv[rt % LOADED]);
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    const lh8 uv = *reinterpret_cast<const lh8*>(mine + 16 * j * US + 16 * rt);
#pragma unroll
                    for (int t = 0; t < 4; ++t) acc[j][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(lh8, now[t]), uv, acc[j][t], 0, 0, 0);
                }
            }
            if constexpr (NEXT) {
#pragma unroll
                for (int rt = 0; rt < LOADED; ++rt)
#pragma unroll
                    for (int t = 0; t < 4; ++t) bv[rt][t] = nv[rt][t];
            }
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                if (!(rows >> (16 * j + n16) & 1)) continue;   // (a row takes its own adapter's result alone)
                const float f = factor[16 * j + n16];
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const uint32_t w = yv[j][e >> 3][(e & 7) >> 1];
                    const float v0 = fmaf(f, acc[j][e >> 2][e & 3], __half2float(__ushort_as_half((unsigned short)w)));
                    const float v1 = fmaf(f, acc[j][e >> 2][(e & 3) + 1], __half2float(__ushort_as_half((unsigned short)(w >> 16))));
                    yv[j][e >> 3][(e & 7) >> 1] = (uint32_t)__half_as_ushort(__float2half_rn(v0)) | (uint32_t)__half_as_ushort(__float2half_rn(v1)) << 16;
                }
                store(j);
            }
            rows = then_rows;
            i = then;
        }
        if (!SPREAD || wave == 0) {   // a row without an adapter keeps its bits
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                const int id = __shfl(all.id, 16 * j + n16, 64);
                if (id < 0 && m0 + 16 * j + n16 < M) store(j);
            }
        }
    }
}

// Tiles of rows that share a workgroup: many rows (prompts, whose tiles have one or few adapters) as many as the accumulators allow.
// (Rank 16, 4096 to 4096, one tile against four: 160 rows of 2 adapters 9.7 and 12.3 us, of 64 adapters 14 and 31; 320 rows 15.1 and 12.4,
// of 64 adapters 43 and 24.)
static int lora_tiles(int M, int rank) { return M < 256 || rank > 128 ? 1 : rank > 64 ? 2 : 4; }

// Parts of K, each a whole number of steps for four waves: few tiles of rows leave the chip idle and want many short parts, but the
// second kernel adds them up once per workgroup.  (A workgroup to a compute unit: 160 rows 9.7 us, half as many 14.0, twice as many 8.9;
// 2048 rows of rank 64, 5120 to 13824, half as many 53.6, 56.1, 58.3.)
struct LoraPlan { int slice, parts; };
static LoraPlan lora_plan(int M, int K, int rank)
{
    const int each = 16 * lora_tiles(M, rank), tiles = (M + each - 1) / each, wgs = M < 256 ? tiles * std::min(M, 8) : tiles;   // (a tile of a few requests has as many adapters)
    const int want = std::max(1, std::min({256 / wgs, (K + 255) / 256, 16}));
    LoraPlan p;
    p.slice = ((K + want - 1) / want + 127) / 128 * 128;
    p.parts = (K + p.slice - 1) / p.slice;
    return p;
}

// The workspace: the parts of u, and for many rows u split.
static bool lora_split(int M) { return M >= 256; }
static int lora_padded(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : rank <= 128 ? 128 : 256; }
size_t lora_workspace_bytes(int M, int, int K, int rank)
{
    const size_t parts = align_up((size_t)lora_plan(M, K, rank).parts * M * rank * sizeof(float), 16);
    return lora_split(M) ? parts + (size_t)M * (4 * lora_padded(rank) + sizeof(float)) : parts;
}

template <int RT, int MT>
static void launch_lora(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a, const uint16_t* b,
                        const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout, float* u, hipStream_t s)
{
    const LoraPlan p = lora_plan(M, K, rank);
    const int tiles = (M + 16 * MT - 1) / (16 * MT);
    // distinct adapters of a tile side by side where the tiles alone are few
    lora_shrink_kernel<RT, MT><<<dim3(p.parts, tiles <= 16 ? std::min({M, adapters, 16}) : 1, tiles), 256, 0, s>>>(M, K, rank, adapters, p.slice, x, ldx, ids, a, u);
    uint16_t* const halves = (uint16_t*)((uint8_t*)u + align_up((size_t)p.parts * M * rank * sizeof(float), 16));
    float* const factors = (float*)(halves + (size_t)M * 2 * 16 * RT);
    const int64_t columns = ((int64_t)N + 63) / 64;
    const bool fast = rank % 8 == 0 && N % 64 == 0;
    auto expand = [&](auto kernel, unsigned wgs, int blocks) {
        kernel<<<dim3(wgs, tiles), 256, 0, s>>>(M, N, rank, adapters, p.parts, blocks, ids, b, scale, u, halves, factors, y, ldy, out, ldout);
    };
    if (lora_split(M)) {
        lora_split_kernel<<<(M + 3) / 4, 256, 0, s>>>(M, rank, 16 * RT, adapters, p.parts, ids, scale, u, halves, factors);
        // two blocks a wave where that leaves two workgroups to a compute unit (4096 rows, rank 64, 11008 columns: 79 us, with one 84, with
        // four 92; 1024 rows, 4096 columns: 29 us, with one 26), but not with shorter tiles (rank 128, 2048 rows: 100 us, with one 94)
        const int blocks = MT == 4 && columns * tiles >= 4096 ? 2 : 1;
        expand(!fast ? lora_expand_kernel<RT, MT, false, false, true> : lora_expand_kernel<RT, MT, false, true, true>, (unsigned)((columns + 4 * blocks - 1) / (4 * blocks)), blocks);
    } else if constexpr (MT == 1) {
        // (16 rows of as many adapters, rank 64: 18 us, 38 with the adapters one after the other; two adapters in 160 rows: 9.7 and 9.3)
        if (M > 1 && adapters > 1) expand(!fast ? lora_expand_kernel<RT, 1, true, false, false> : lora_expand_kernel<RT, 1, true, true, false>, (unsigned)columns, 1);
        else expand(!fast ? lora_expand_kernel<RT, 1, false, false, false> : lora_expand_kernel<RT, 1, false, true, false>, (unsigned)((columns + 3) / 4), 1);
    }
}

hipError_t launch_lora_add(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a,
                           const uint16_t* b, const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout, void* workspace,
                           hipStream_t s)
{
    const int mt = lora_tiles(M, rank);
    auto go = [&](auto rt, auto tiles) {
        launch_lora<decltype(rt)::value, decltype(tiles)::value>(M, N, K, rank, adapters, x, ldx, ids, a, b, scale, y, ldy, out, ldout, (float*)workspace, s);
    };
    using std::integral_constant;
    const integral_constant<int, 1> one;
    const integral_constant<int, 2> two;
    const integral_constant<int, 4> four;
    if (rank <= 16) mt == 1 ? go(one, one) : go(one, four);
    else if (rank <= 32) mt == 1 ? go(two, one) : go(two, four);
    else if (rank <= 64) mt == 1 ? go(four, one) : go(four, four);
    else if (rank <= 128) mt == 1 ? go(integral_constant<int, 8>{}, one) : go(integral_constant<int, 8>{}, two);
    else go(integral_constant<int, 16>{}, one);
    return hipGetLastError();
}

}  // namespace abq
