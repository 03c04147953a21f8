// Device code of the few-rows kernel of experts, and the templates that launch its variants.
//
// Each expert's weights are multiplied by the few rows that chose it, 16 of them at a time.  What bounds it is the stream of the
// weights.  The work is a list of units (expert, its 16 rows, a group of output tiles), dealt out in even runs to a grid that fills the chip,
// whatever the groups are: one token's two experts take as many compute units as sixty-four experts do.  Inside a workgroup the waves are a
// grid of (part of K) x (tile of the group).  A wave keeps its part of A in registers, as operands, for as long as a run stays with the same rows
// (unpacked codes are masked and made signed once, the sums of the codes are taken on the way), and streams weights past it: as a super-chunk
// has been multiplied, the next tile's is asked for.  The parts of K of up to four tiles meet in LDS, and all waves add them up and store them: one barrier
// to four tiles.  (With a barrier to every tile and its sum left to one wave, W2A8 64 rows of eight 11008->4096 took 30 us; now 20.8 to 25, differing from run to
// run of the same binary, 3.7 to 4.4 TB/s of weights; W4A8 one token's two experts 4096->11008 14.4 and now 11.4.)
// A whole row of A is in one workgroup's registers, which bounds K (moe_max_waves): 16384 up to four bits, 12288 from five on.
#pragma once
#include "abq_moe.h"
#include "abq_rows.h"

#include <atomic>

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

template <int P, int SL = 0>
__device__ __forceinline__ void moe_super_chunk(const mv4i* w, const mv4i* a, mv4i& acc)
{
    if constexpr (SL < 8) {
        mv4i b;
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = (int)moe_dword<P, SL>(w, j);
        acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(a[SL], b, acc, 0, 0, 0);
        moe_super_chunk<P, SL + 1>(w, a, acc);
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
// eight-bit blobs hold as -128).  They were loaded from `at`, or from `last`, the tensor's last sixteen bytes, if those come first.
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

// Waves a workgroup can have with R super-chunks a wave, 0 where the variant is not built: what the registers leave (A takes 32 R of
// them, the weights in flight 4 P R, the rest 35 to 55; variants that spill are not built).
__host__ __device__ constexpr int moe_max_waves(int P, int R)
{
    return R == 1 ? 16 : (R == 2 ? (P <= 6 ? 12 : 0) : (R == 3 ? (P >= 7 ? 8 : 0) : (R == 4 && P <= 4 ? 8 : 0)));
}

// Tiles in flight.
__host__ __device__ constexpr int moe_depth(int P, int R) { return P * R <= 4 ? 2 : 1; }

// Every wave's LDS accesses are done; loads stay in flight (a workgroup fence would wait for them).
__device__ __forceinline__ void moe_barrier()
{
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// Tiles between two barriers: their parts of K meet in LDS together, and the waves share the work of adding them up (where few parts share it, two).
static int moe_batch(int kparts) { return kparts >= 4 ? 4 : 2; }
// LDS: [2][batch][waves][64] parts of tiles, [3][tgroups][64] channels' parameters.
static size_t moe_rows_lds_bytes(const MoeRowsParams& prm) { return (size_t)(2 * prm.batch * prm.kparts + 3) * prm.tgroups * 1024; }

template <int P, int R>
__global__ __launch_bounds__(64 * moe_max_waves(P, R)) void moe_rows_kernel(MoeRowsParams prm)
{
    constexpr int D = moe_depth(P, R);
    extern __shared__ __align__(16) mv4i lds[];
    __shared__ int32_t row_sum[2][16];
    __shared__ __align__(16) RowParams par_a[16];
    const int tid = threadIdx.x, lane = tid & 63, r = lane & 15, G = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tg = wave / prm.kparts, kpart = wave - tg * prm.kparts;   // (blockDim = 64 kparts tgroups)
    const int k0 = kpart * R * kSuperK, waves = prm.kparts * prm.tgroups;
    mv4i* const red = lds;                                               // part of tile b, buffer f: at ((f batch + b) waves + wave) 64
    mv4i* const par_w = lds + 2 * prm.batch * waves * 64;

    const ExpertUnits<BlocksOf> units(prm.g, BlocksOf{16}, prm.most);
    // this workgroup's run: all units are dealt out evenly
    const unsigned all = (unsigned)units.total * (unsigned)prm.groups_n, per = all / gridDim.x, rest = all - per * gridDim.x;   // (below 2^30)
    unsigned u = blockIdx.x * per + min(blockIdx.x, rest);
    const unsigned end = u + per + (blockIdx.x < rest ? 1u : 0u);
    const uint32_t flip = prm.oa ? 0x80808080u : 0u;
    if (tid < 16) row_sum[0][tid] = 0;
    int sums_at = 0, buf = 0, par_at = 0;   // buffers in turn: the runs' row sums, the batches' parts, their parameters

    while (u < end) {
        const int block = (int)(u / (unsigned)prm.groups_n), g0 = (int)u - block * prm.groups_n;
        const int count = min((int)(end - u), prm.groups_n - g0);
        const ExpertAt at = units.find(prm.g, block);
        const int local = (block - at.before) * 16;
        const int row0 = at.first + local, nrow = min(max(at.rows - local, 0), 16);
        const uint8_t* blob = prm.w + (size_t)at.expert * prm.w_stride;
        const RowParams* wparams = reinterpret_cast<const RowParams*>(blob + prm.off_params);
        u += count;

        // ---- loads.  The rows' numbers first, then the weights of the run's first tiles, which need the expert alone, then what waits for the numbers.
        const int entry = moe_order(prm.g, min(row0 + min(r, max(nrow - 1, 0)), prm.g.rows - 1));
        __builtin_amdgcn_sched_barrier(0);
        mv4i w[D][R][P];
        // (past the run's end a load goes to the blob's first KiB, for nobody: a load under a condition would make every wait one for all)
        auto load_super = [&](int d, int rr, int i) {
            const int tile = min((g0 + i) * prm.tgroups + tg, prm.ntiles - 1), sc = min(kpart * R + rr, prm.nsuper - 1);
            const size_t at = i < count ? (size_t)tile * prm.nsuper + sc : 0;
#pragma unroll
            for (int g = 0; g < group_count(P); ++g) {
                const int b = group_width(P, g);
                const mv4i* base = reinterpret_cast<const mv4i*>(blob + prm.off_fields[g]) + at * (b * 64) + lane;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (c < b) w[d][rr][moe_load_base(P, g) + c] = __builtin_nontemporal_load(base + c * 64);
            }
        };
        // The channels' parameters of four tiles from i on, straight into LDS, by the first wave of a tile group.  A batch's are asked for a batch ahead and
        // before that batch's refills: loads return in order, so they are there once the weights of the batch's last tile are.  (Written as the
        // instruction: the compiler would wait for the builtin at every LDS access.)
        auto load_params = [&](int i, int place) {
            if (kpart != 0 || i >= count) return;   // (the same for the wave; what is asked for is always waited for)
            const unsigned n = (unsigned)min(((g0 + i + G) * prm.tgroups + tg) * kTileN + r, prm.N - 1) * 16u;
            const unsigned dst = (unsigned)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)(par_w + (place * prm.tgroups + tg) * 64);
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(dst), "v"(n), "s"(wparams) : "memory", "m0");
        };
        auto load_tile = [&](int d) {
#pragma unroll
            for (int rr = 0; rr < R; ++rr) load_super(d, rr, d);
            __builtin_amdgcn_sched_barrier(0);
        };
        load_params(0, par_at);
        load_tile(0);
        // A: lane (r, G) holds bytes 16 G .. of slice s of row r; rows past the group's are its last one again.  Vectors past a row's
        // end hold what follows in memory; those past the last row's end are moved back.  Both are put right below.
        mv4i a[R][8];
        const int row = moe_row(prm.g, entry);
        const uint32_t a_end = (uint32_t)prm.g.tokens * (uint32_t)prm.K - 16u, off = (uint32_t)row * (uint32_t)prm.K + G * 16u;
        const int last_slice = (prm.K - 1) / 64 * 64;
#pragma unroll
        for (int rr = 0; rr < R; ++rr)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const uint32_t ks = min((uint32_t)min(k0 + rr * kSuperK + s * 64, last_slice), a_end);   // (a single row's last slice may begin behind a_end)
                const u32x4_byte v = *reinterpret_cast<const u32x4_byte*>(prm.a + ks + min(off, a_end - ks));
                a[rr][s] = mv4i{(int)v.x, (int)v.y, (int)v.z, (int)v.w};
            }
        const float par_scale = prm.a_scale[row];
        const int32_t par_zero = prm.a_zero[row];
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (D == 2) load_tile(1);
        moe_barrier();   // (every wave is done with the run before: its rows' parameters and sums)
        int K = prm.K, k_lane = G * 16;
        asm volatile("" : "+s"(K), "+v"(k_lane));   // (or every slice's masks are made ahead of the loop over the runs, and spilled)
        uint32_t sum_a = 0;
#pragma unroll
        for (int rr = 0; rr < R; ++rr)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const int ks = k0 + rr * kSuperK + s * 64;
                if (ks >= K) a[rr][s] = mv4i{0, 0, 0, 0};   // (the same for every lane; past the last super-chunk the weights are its own again)
                else if (ks + 64 > K) {
                    const uint32_t from = min((uint32_t)ks, a_end);
                    moe_operand_at_end(a[rr][s], prm.a_mask, flip, sum_a, ks + k_lane, K, ks - from + off, a_end - from);
                }
                else moe_operand(a[rr][s], prm.a_mask, flip, sum_a);
            }
        if (tg == 0) {   // (the waves of the other tile groups hold the same parts of A)
            sum_a += __shfl_xor(sum_a, 16);
            sum_a += __shfl_xor(sum_a, 32);
            if (lane < 16) atomicAdd(&row_sum[sums_at][lane], (int32_t)sum_a);   // (whole numbers: any order)
        }
        if (tid < 16) {
            row_sum[sums_at ^ 1][tid] = 0;
            par_a[tid] = RowParams{0, par_scale, par_zero, 0};
        }

        // ---- the tiles, D of them in flight, a batch of them to a barrier
        auto tile_step = [&](auto DC, int i, int b) {
            constexpr int d = decltype(DC)::value;
            mv4i acc = mv4i{0, 0, 0, 0};
#pragma unroll
            for (int rr = 0; rr < R; ++rr) {
                moe_super_chunk<P>(w[d][rr], a[rr], acc);
                load_super(d, rr, i + D);
            }
            red[((buf * prm.batch + b) * waves + wave) * 64 + lane] = acc;
        };
        for (int i0 = 0; i0 < count; i0 += prm.batch) {
            const int nb = min(prm.batch, count - i0), par_next = par_at == 2 ? 0 : par_at + 1;
            load_params(i0 + prm.batch, par_next);
            int b = 0;
            for (; b + D <= nb; b += D) {   // (whole rounds: a step that may be left out would make every wait one for all loads)
                tile_step(std::integral_constant<int, 0>{}, i0 + b, b);
                if constexpr (D == 2) tile_step(std::integral_constant<int, 1>{}, i0 + b + 1, b + 1);
            }
            if constexpr (D == 2) { if (b < nb) tile_step(std::integral_constant<int, 0>{}, i0 + b, b); }
            moe_barrier();
            for (int t = kpart; t < nb; t += prm.kparts) {   // tiles of this tile group: its waves in turn
                int own = lane;
                asm volatile("" : "+v"(own));   // (or every address below is made ahead of the loop, in registers that the operands need)
                const mv4i* part = red + ((buf * prm.batch + t) * waves + tg * prm.kparts) * 64 + own;
                mv4i sum = mv4i{0, 0, 0, 0};
                for (int k = 0; k < prm.kparts; k += 4) {
                    mv4i v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] = part[min(k + j, prm.kparts - 1) * 64];
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum += v[j] & (k + j < prm.kparts ? -1 : 0);
                }
                const RowParams pw = reinterpret_cast<const RowParams*>(par_w)[(par_at * prm.tgroups + tg) * 64 + t * 16 + (own & 15)];
                const int n = ((g0 + i0 + t) * prm.tgroups + tg) * kTileN + (own & 15);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int m = 4 * (own >> 4) + e;
                    RowParams pa = par_a[m];
                    pa.sum = row_sum[sums_at][m];
                    int32_t raw;
                    const uint16_t h = epilogue_value(sum[e], prm.oa, prm.ow, prm.K, pa, pw, &raw);
                    if (m < nrow && n < prm.N) prm.y[(size_t)(row0 + m) * prm.N + n] = h;
                }
            }
            buf ^= 1;
            par_at = par_next;
        }
        sums_at ^= 1;
    }
}

template <int P, int R>
static hipError_t moe_rows_go(const MoeRowsParams& prm, unsigned grid, hipStream_t s)
{
    static std::atomic<bool> attr_set{false};   // (an idempotent call: a lost race only repeats it)
    if (!attr_set.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute((const void*)moe_rows_kernel<P, R>, hipFuncAttributeMaxDynamicSharedMemorySize, 159 * 1024);
        if (e != hipSuccess) return e;
        attr_set.store(true, std::memory_order_release);
    }
    moe_rows_kernel<P, R><<<grid, 64 * prm.kparts * prm.tgroups, moe_rows_lds_bytes(prm), s>>>(prm);
    return hipGetLastError();
}

template <int P, int R = 1>
static hipError_t moe_rows_launch(const MoeRowsParams& prm, int Rwant, unsigned grid, hipStream_t s)
{
    if constexpr (moe_max_waves(P, R) > 0)
        if (Rwant == R) return moe_rows_go<P, R>(prm, grid, s);
    if constexpr (R < 4) return moe_rows_launch<P, R + 1>(prm, Rwant, grid, s);
    else return hipErrorInvalidValue;
}

#define ABQ_MOE_ROWS_LAUNCH(P) hipError_t moe_rows_launch_p##P(const MoeRowsParams& prm, int R, unsigned grid, hipStream_t s)
ABQ_MOE_ROWS_LAUNCH(1);
ABQ_MOE_ROWS_LAUNCH(2);
ABQ_MOE_ROWS_LAUNCH(3);
ABQ_MOE_ROWS_LAUNCH(4);
ABQ_MOE_ROWS_LAUNCH(5);
ABQ_MOE_ROWS_LAUNCH(6);
ABQ_MOE_ROWS_LAUNCH(7);
ABQ_MOE_ROWS_LAUNCH(8);

}  // namespace abq
