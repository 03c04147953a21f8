// Device code of the few-rows kernel of experts, and the templates that launch its variants.
//
// Each expert's weights are multiplied by the few rows that chose it, 16 MT of them at a time.  What bounds it is the stream of the
// weights.  The work is a list of units (expert, its 16 MT rows, a group of output tiles), dealt out in even runs to a grid that fills the chip,
// whatever the groups are: one token's two experts take as many compute units as sixty-four experts do.  Inside a workgroup the waves are a
// grid of (part of K) x (tile of the group).  A wave keeps its part of A in registers, as operands, for as long as a run stays with the same rows
// (unpacked codes are masked and made signed once, the sums of the codes are taken on the way), and streams weights past it: as a super-chunk
// has been multiplied, the next tile's is asked for.  The parts of K of a tile meet in LDS, and one wave after the other adds a tile up and stores it
// while the rest go on.
#pragma once
#include "abq_moe.h"
#include "abq_rows.h"

namespace abq {

typedef int mv4i __attribute__((ext_vector_type(4)));

__host__ __device__ constexpr int moe_load_base(int p, int g) { return g == 0 ? 0 : (g == 1 ? group_width(p, 0) : group_width(p, 0) + group_width(p, 1)); }

// Operand dword j of slice SL (0..7) of a super-chunk, all plane groups merged into a byte per weight.  w: the super-chunk's chunks, lane's part.
template <int P, int SL, int G0 = 0>
__device__ __forceinline__ uint32_t moe_dword(const mv4i* w, int j)
{
    constexpr int b = group_width(P, G0), shift = group_shift(P, G0), t = SL % (8 / b), sh = b * t - shift;
    const uint32_t x = (uint32_t)w[moe_load_base(P, G0) + SL * b / 8][j];
    if constexpr (P == 8) return x;
    constexpr uint32_t mask = (((1u << b) - 1u) * 0x01010101u) << shift;
    uint32_t v;
    if constexpr (sh > 0) v = (x >> sh) & mask;
    else if constexpr (sh < 0) v = (x << (-sh)) & mask;
    else v = x & mask;
    if constexpr (G0 + 1 < group_count(P)) v |= moe_dword<P, SL, G0 + 1>(w, j);
    return v;
}

template <int P, int MT, int SL = 0>
__device__ __forceinline__ void moe_super_chunk(const mv4i* w, const mv4i (*a)[8], mv4i* acc)
{
    if constexpr (SL < 8) {
        mv4i b;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = (int)moe_dword<P, SL>(w, j);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt] = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[mt][SL], b, acc[mt], 0, 0, 0);
        moe_super_chunk<P, MT, SL + 1>(w, a, acc);
    }
}

// Sixteen codes of a row as operand bytes, and their sum on the way.
__device__ __forceinline__ void moe_operand(mv4i& v, uint32_t mask, uint32_t flip, uint32_t& sum)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t c = (uint32_t)v[j] & mask;
        sum = __builtin_amdgcn_udot4(c, 0x01010101u, sum, false);
        v[j] = (int)(c ^ flip);
    }
}
// The same from k on where the row of K ends among them or before: zeros behind its end (the weights there are those of code 0, which
// eight-bit blobs hold as -128).  They were loaded from `at`, or from the tensor's last sixteen bytes if those come first.
__device__ __forceinline__ void moe_operand_at_end(mv4i& v, uint32_t mask, uint32_t flip, uint32_t& sum, int k, int K, uint32_t at, uint32_t last)
{
    uint64_t lo = (uint32_t)v[0] | (uint64_t)(uint32_t)v[1] << 32, hi = (uint32_t)v[2] | (uint64_t)(uint32_t)v[3] << 32;
    const uint32_t back = at > last ? min(at - last, 16u) : 0u;   // bytes that it was moved back
    if (back >= 8) { lo = hi; hi = 0; }
    const uint32_t sh = 8 * (back & 7);
    if (sh) { lo = lo >> sh | hi << (64 - sh); hi >>= sh; }
    const int n = min(max(K - k, 0), 16);                         // codes of the row
    const uint64_t in_lo = n >= 8 ? ~0ull : ~(~0ull << (8 * n)), in_hi = n >= 16 ? ~0ull : (n <= 8 ? 0ull : ~(~0ull << (8 * (n - 8))));
    lo &= in_lo;
    hi &= in_hi;
    v = mv4i{(int)(uint32_t)lo, (int)(uint32_t)(lo >> 32), (int)(uint32_t)hi, (int)(uint32_t)(hi >> 32)};
    moe_operand(v, mask, flip, sum);
    v = mv4i{v[0] & (int)(uint32_t)in_lo, v[1] & (int)(uint32_t)(in_lo >> 32), v[2] & (int)(uint32_t)in_hi, v[3] & (int)(uint32_t)(in_hi >> 32)};
}

// Waves a workgroup can have with R super-chunks a wave, 0 where the variant is not built: what the registers leave (A takes 32 MT R of
// them, the weights in flight 4 P R, the rest 35 to 55; variants that spill are not built).
__host__ __device__ constexpr int moe_max_waves(int P, int R, int MT)
{
    if (MT == 2) return R == 1 ? 12 : (R == 2 ? 8 : 0);
    return R == 1 ? 16 : (R == 2 ? (P <= 6 ? 12 : 0) : (R == 3 ? (P >= 7 ? 8 : 0) : (R == 4 && P <= 4 ? 8 : 0)));
}

template <int P, int R, int MT>
__global__ __launch_bounds__(64 * moe_max_waves(P, R, MT)) void moe_rows_kernel(MoeRowsParams prm)
{
    constexpr int kMax = moe_max_waves(P, R, MT);
    __shared__ __align__(16) mv4i red[2][kMax][MT][64];
    __shared__ int32_t part_sum[kMax][16 * MT];
    __shared__ __align__(16) RowParams par_a[16 * MT];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, G = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tg = wave / prm.kparts, kpart = wave - tg * prm.kparts;   // (blockDim = 64 kparts tgroups)
    const int k0 = kpart * R * kSuperK;

    const ExpertUnits units(prm.g, 16 * MT, prm.most);
    // this workgroup's run: all units are dealt out evenly
    const int64_t all = (int64_t)units.total * prm.groups_n;
    int64_t u = all * blockIdx.x / gridDim.x;
    const int64_t end = all * (blockIdx.x + 1) / gridDim.x;
    const uint32_t flip = prm.oa ? 0x80808080u : 0u;

    while (u < end) {
        const int block = (int)(u / prm.groups_n), g0 = (int)(u - (int64_t)block * prm.groups_n);
        const int count = (int)min(end - u, (int64_t)(prm.groups_n - g0));
        const ExpertAt at = units.find(prm.g, 16 * MT, block);
        const int local = (block - at.before) * 16 * MT;
        const int row0 = at.first + local, nrow = min(max(at.rows - local, 0), 16 * MT);
        const uint8_t* blob = prm.w + (size_t)at.expert * prm.w_stride;
        const RowParams* wparams = reinterpret_cast<const RowParams*>(blob + prm.off_params);
        u += count;

        // ---- A: lane (r, G) holds bytes 16 G .. of slice s of rows r, r + 16; rows past the group's are its last one again.  Vectors past a row's
        // end hold what follows in memory; those past the last row's end are moved back.  Both are put right below.
        mv4i a[R][MT][8];
        uint32_t off[MT];
        const uint32_t a_end = (uint32_t)prm.g.tokens * (uint32_t)prm.K - 16u;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
            off[mt] = (uint32_t)moe_row_of(prm.g, min(row0 + min(16 * mt + r, max(nrow - 1, 0)), prm.g.rows - 1)) * (uint32_t)prm.K + G * 16u;
        const int last_slice = (prm.K - 1) / 64 * 64;
#pragma unroll
        for (int rr = 0; rr < R; ++rr)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const uint32_t ks = (uint32_t)min(k0 + rr * kSuperK + s * 64, last_slice);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    const u32x4_byte v = *reinterpret_cast<const u32x4_byte*>(prm.a + ks + min(off[mt], a_end - ks));
                    a[rr][mt][s] = mv4i{(int)v.x, (int)v.y, (int)v.z, (int)v.w};
                }
            }
        // ---- weights of the run's first tile
        mv4i w[R][P];
        RowParams pw, pw_next;
        auto load_super = [&](int rr, int tile) {
            const int sc = min(kpart * R + rr, prm.nsuper - 1);
#pragma unroll
            for (int g = 0; g < group_count(P); ++g) {
                const int b = group_width(P, g);
                const mv4i* base = reinterpret_cast<const mv4i*>(blob + prm.off_fields[g]) + ((size_t)tile * prm.nsuper + sc) * (b * 64) + lane;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < b) w[rr][moe_load_base(P, g) + i] = __builtin_nontemporal_load(base + i * 64);
            }
        };
        auto tile_of = [&](int i) { return min((g0 + i) * prm.tgroups + tg, prm.ntiles - 1); };
        auto load_params = [&](int tile) { return wparams[min(tile * kTileN + r, prm.N - 1)]; };
        pw = load_params(tile_of(0));
#pragma unroll
        for (int rr = 0; rr < R; ++rr) load_super(rr, tile_of(0));
        __syncthreads();   // (the tiles before are done with the row parameters)
        if (tid < 16 * MT) {
            const int row = moe_row_of(prm.g, min(row0 + min(tid, max(nrow - 1, 0)), prm.g.rows - 1));
            par_a[tid] = RowParams{0, prm.a_scale[row], prm.a_zero[row], 0};
        }
        int K = prm.K, k_lane = G * 16;
        asm volatile("" : "+s"(K), "+v"(k_lane));   // (or every slice's masks are made ahead of the loop over the runs, and spilled)
        uint32_t sums[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sums[mt] = 0;
#pragma unroll
        for (int rr = 0; rr < R; ++rr)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int ks = k0 + rr * kSuperK + s * 64;
                if (ks >= K) {                             // (the same for every lane; past the last super-chunk the weights are its own again)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) a[rr][mt][s] = mv4i{0, 0, 0, 0};
                    continue;
                }
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (ks + 64 > K) moe_operand_at_end(a[rr][mt][s], prm.a_mask, flip, sums[mt], ks + k_lane, K, off[mt], a_end - ks);
                    else moe_operand(a[rr][mt][s], prm.a_mask, flip, sums[mt]);
                }
            }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            sums[mt] += __shfl_xor(sums[mt], 16);
            sums[mt] += __shfl_xor(sums[mt], 32);
            if (lane < 16) part_sum[wave][16 * mt + lane] = (int32_t)sums[mt];
        }

        // ---- the tiles
        int buf = 0, turn = 0;
        auto tile_step = [&](int i, auto more) {
            mv4i acc[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) acc[mt] = mv4i{0, 0, 0, 0};
            if constexpr (decltype(more)::value) pw_next = load_params(tile_of(i + 1));
#pragma unroll
            for (int rr = 0; rr < R; ++rr) {
                moe_super_chunk<P, MT>(w[rr], a[rr], acc);
                if constexpr (decltype(more)::value) load_super(rr, tile_of(i + 1));
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) red[buf][wave][mt][lane] = acc[mt];
            // every wave's parts are written; loads stay in flight (a workgroup fence would wait for them)
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            if (kpart == turn) {
                int own = lane;
                asm volatile("" : "+v"(own));   // (or every address below is made ahead of the loop, in registers that the operands need)
                const int tile = (g0 + i) * prm.tgroups + tg, n = tile * kTileN + (own & 15);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mv4i sum = mv4i{0, 0, 0, 0};
                    for (int k = 0; k < prm.kparts; ++k) sum += red[buf][tg * prm.kparts + k][mt][own];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int m = 16 * mt + 4 * (own >> 4) + e;
                        RowParams pa = par_a[m];
                        for (int k = 0; k < prm.kparts; ++k) pa.sum += part_sum[k][m];
                        int32_t raw;
                        const uint16_t h = epilogue_value(sum[e], prm.oa, prm.ow, prm.K, pa, pw, &raw);
                        if (m < nrow && n < prm.N) prm.y[(size_t)(row0 + m) * prm.N + n] = h;
                    }
                }
            }
            buf ^= 1;
            turn = turn + 1 == prm.kparts ? 0 : turn + 1;
            if constexpr (decltype(more)::value) pw = pw_next;
        };
        for (int i = 0; i + 1 < count; ++i) tile_step(i, std::true_type{});
        tile_step(count - 1, std::false_type{});
    }
}

template <int P, int R, int MT>
static hipError_t moe_rows_go(const MoeRowsParams& prm, unsigned grid, hipStream_t s)
{
    moe_rows_kernel<P, R, MT><<<grid, 64 * prm.kparts * prm.tgroups, 0, s>>>(prm);
    return hipGetLastError();
}

template <int P, int R = 1, int MT = 1>
static hipError_t moe_rows_launch(const MoeRowsParams& prm, int Rwant, int MTwant, unsigned grid, hipStream_t s)
{
    if constexpr (moe_max_waves(P, R, MT) > 0)
        if (Rwant == R && MTwant == MT) return moe_rows_go<P, R, MT>(prm, grid, s);
    if constexpr (R < 4) return moe_rows_launch<P, R + 1, MT>(prm, Rwant, MTwant, grid, s);
    else if constexpr (MT < 2) return moe_rows_launch<P, 1, MT + 1>(prm, Rwant, MTwant, grid, s);
    else return hipErrorInvalidValue;
}

#define ABQ_MOE_ROWS_LAUNCH(P) hipError_t moe_rows_launch_p##P(const MoeRowsParams& prm, int R, int MT, unsigned grid, hipStream_t s)
ABQ_MOE_ROWS_LAUNCH(1);
ABQ_MOE_ROWS_LAUNCH(2);
ABQ_MOE_ROWS_LAUNCH(3);
ABQ_MOE_ROWS_LAUNCH(4);
ABQ_MOE_ROWS_LAUNCH(5);
ABQ_MOE_ROWS_LAUNCH(6);
ABQ_MOE_ROWS_LAUNCH(7);
ABQ_MOE_ROWS_LAUNCH(8);

}  // namespace abq
