// Appending keys and values to a paged cache, with the rotation to their positions and, for a cache of codes, the quantizer
// on the way; and the way back.
//
// What bounds it: a step of few rows is latency (row -> sequence -> position -> page -> store, three dependent loads beside
// the operands' own): one row of 32 heads of 128 takes 3.0 us, 64 rows with 8 key heads as codes 4.3, reading them back 2.7.  A prompt is
// the copy of its vectors: two prompts of up to 2048 tokens, 40 heads on 40, 213 MB in 48 us, 4.4 TB/s (a large copy: 5.1; 34 us where
// the last-level cache holds them).
#include "abq_kv.h"
#include "abq_rows.h"

namespace abq {

struct KvAppendArgs {
    abq_kv_cache c;
    abq_batch b;
    int heads_q, rotary_dim, page_shift;
    bool interleaved;
    const float* inv_freq;
    const uint16_t *q, *k, *v;
    int ldq, ldk, ldv;
    uint16_t* q_out;
};

// The sequence that a row belongs to: as many end at or before it.  (One load for 64 sequences, no search.)
__device__ __forceinline__ int sequence_of_row(const abq_batch& b, int row)
{
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int s0 = 0; s0 < b.seqs; s0 += 64) {
        const int s = s0 + lane;
        n += __popcll(__ballot(s < b.seqs && b.row_start[s + 1] <= row));
    }
    return n;
}

// Sine and cosine of position * frequency.  The angle in quarter turns and its distance from the nearest whole one are formed in
// binary64 (a position of 2^20 at frequency 1 would lose all but four bits of the fraction in binary32), the angle and the quotient
// each with what its rounding left (55 bits of product, 2 / pi in two parts: at a position of 2^31 the roundings alone are 2^-22); the
// remaining eighth of a turn goes through the Taylor polynomials of sine and cosine in binary32, whose first missing terms are below
// 2^-28 there.
__device__ __forceinline__ float2 sine_cosine(int position, float frequency)
{
    constexpr double kTwoByPi = 0.63661977236758134308, kRest = -3.935735335036497e-17;   // (their sum is 2 / pi to 2^-108)
    const double angle = (double)position * (double)frequency, quarters = angle * kTwoByPi, whole = rint(quarters);
    const double left = fma(fma((double)position, (double)frequency, -angle), kTwoByPi, fma(angle, kRest, fma(angle, kTwoByPi, -quarters)));
    const float x = (float)(quarters - whole + left) * 1.57079632679489661923f, z = x * x;
    const int quadrant = (int)(whole - 4.0 * floor(whole * 0.25));
    float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);
    s = fmaf(fmaf(fmaf(s, z, 8.33333333e-3f), z, -1.66666667e-1f) * z, x, x);
    float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);
    c = fmaf(fmaf(fmaf(fmaf(c, z, -1.38888889e-3f), z, 4.16666667e-2f), z, -0.5f), z, 1.0f);
    const float sv = quadrant & 1 ? c : s, cv = quadrant & 1 ? s : c;
    return float2{quadrant & 2 ? -sv : sv, (quadrant + 1) & 2 ? -cv : cv};
}

__device__ __forceinline__ void to_float8(const uint32_t* h, float* f)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __half2float(__ushort_as_half((unsigned short)(h[j] & 0xFFFFu)));
        f[2 * j + 1] = __half2float(__ushort_as_half((unsigned short)(h[j] >> 16)));
    }
}
__device__ __forceinline__ void to_half8(const float* f, uint32_t* h)
{
#pragma unroll
    for (int j = 0; j < 4; ++j)
        h[j] = (uint32_t)__half_as_ushort(__float2half_rn(f[2 * j])) | ((uint32_t)__half_as_ushort(__float2half_rn(f[2 * j + 1])) << 16);
}

// One workgroup per row (and part of its heads: blockIdx.y); LG lanes hold one head's vector, 16 elements each as two runs of
// eight: inside the rotated part runs r/2 apart, so that a lane holds both members of its pairs.
template <int LG, bool CODES>
__global__ __launch_bounds__(256) void kv_append_kernel(KvAppendArgs a)
{
    __shared__ float2 angle[128];   // (sine, cosine)
    const int row = blockIdx.x, tid = threadIdx.x, D = a.c.head_dim, r = a.rotary_dim;
    const int seq = sequence_of_row(a.b, row);
    if (seq >= a.b.seqs) return;   // behind the last sequence
    const int64_t pos64 = (int64_t)a.b.lens[seq] - ((int64_t)a.b.row_start[seq + 1] - row);
    const int pos = (int)min(max(pos64, (int64_t)INT32_MIN), (int64_t)INT32_MAX);   // (below 0: more rows than tokens; rotated, not appended)
    if (tid < r / 2) angle[tid] = sine_cosine(pos, a.inv_freq[tid]);
    __syncthreads();
    const int page = page_of(a.b, a.c, a.page_shift, seq, pos), offset = pos & (a.c.page_size - 1);

    const int lane = tid % LG, per = 256 / LG;
    const int nq = a.q ? a.heads_q : 0, units = nq + 2 * a.c.heads;
    const bool inside = 16 * lane < D, turned = 16 * lane < r;
    const int at0 = !turned ? 16 * lane : a.interleaved ? 16 * lane : 8 * lane;
    const int at1 = !turned || a.interleaved ? at0 + 8 : at0 + r / 2;
    for (int u = blockIdx.y * per + tid / LG; u < units; u += gridDim.y * per) {
        const bool is_q = u < nq, is_v = u >= nq + a.c.heads;
        const int head = is_q ? u : is_v ? u - nq - a.c.heads : u - nq;
        const uint16_t* src = is_q ? a.q + (size_t)row * a.ldq : is_v ? a.v + (size_t)row * a.ldv : a.k + (size_t)row * a.ldk;
        src += (size_t)head * D;
        uint32_t h[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (inside) {
            load_half8<false>(src + at0, 0, 8, h);
            load_half8<false>(src + at1, 0, 8, h + 4);
            if (turned && !is_v) {
                float x[16], y[16];
                to_float8(h, x);
                to_float8(h + 4, x + 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) {   // eight pairs
                    const int i0 = a.interleaved ? 2 * e : e, i1 = a.interleaved ? 2 * e + 1 : e + 8;
                    const float2 sc = angle[8 * lane + e];
                    y[i0] = fmaf(x[i0], sc.y, -(x[i1] * sc.x));
                    y[i1] = fmaf(x[i1], sc.y, x[i0] * sc.x);
                }
                to_half8(y, h);
                to_half8(y + 8, h + 4);
            }
        }
        if (is_q) {
            if (inside) {
                uint16_t* dst = a.q_out + ((size_t)row * nq + head) * D;
                store_half8<false>(dst + at0, 0, 8, h);
                store_half8<false>(dst + at1, 0, 8, h + 4);
            }
            continue;
        }
        if (page < 0) continue;
        const int64_t vec = vector_of(a.c, page, head, offset);
        if constexpr (!CODES) {
            if (inside) {
                uint16_t* dst = (uint16_t*)(is_v ? a.c.v : a.c.k) + vec * D;
                store_half8<false>(dst + at0, 0, 8, h);
                store_half8<false>(dst + at1, 0, 8, h + 4);
            }
        } else {
            float x[16], lo = 0.0f, hi = 0.0f;
            to_float8(h, x);
            to_float8(h + 4, x + 8);
#pragma unroll
            for (int e = 0; e < 16; ++e) { lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]); }
#pragma unroll
            for (int off = LG / 2; off > 0; off >>= 1) {
                lo = fminf(lo, __shfl_xor(lo, off, 64));
                hi = fmaxf(hi, __shfl_xor(hi, off, 64));
            }
            const TokenQuantizer tq(lo, hi, 255);
            if (lane == 0) {
                // (zeros take the quantizer's smallest scale: attention's weights carry the scale of V into binary16, where a token that
                // adds nothing must not push out the others)
                (is_v ? a.c.v_scale : a.c.k_scale)[vec] = hi == lo ? 0x1p-32f : tq.delta;
                (is_v ? a.c.v_zero : a.c.k_zero)[vec] = (uint8_t)tq.z;
            }
            if (inside) {
                uint8_t* dst = (uint8_t*)(is_v ? a.c.v : a.c.k) + vec * D;
                uint32_t o[2];
                tq.codes8(h, o);
                store_bytes8<false>(dst + at0, 0, 8, o);
                tq.codes8(h + 4, o);
                store_bytes8<false>(dst + at1, 0, 8, o);
            }
        }
    }
}

template <bool CODES>
static void append(const KvAppendArgs& a, hipStream_t s)
{
    const int D = a.c.head_dim, lg = D <= 64 ? 4 : D <= 128 ? 8 : 16;
    const int passes = ((a.q ? a.heads_q : 0) + 2 * a.c.heads) * lg;   // threads that a row's vectors take
    // few rows: as many workgroups as it takes for one pass each; from 256 rows on there is a workgroup for every unit, and the angles
    // are formed once a row
    const int parts = a.b.rows <= 256 ? (passes + 255) / 256 : 1;
    const dim3 grid(a.b.rows, parts);
    if (lg == 4) kv_append_kernel<4, CODES><<<grid, 256, 0, s>>>(a);
    else if (lg == 8) kv_append_kernel<8, CODES><<<grid, 256, 0, s>>>(a);
    else kv_append_kernel<16, CODES><<<grid, 256, 0, s>>>(a);
}

hipError_t launch_kv_append(const abq_kv_cache& c, const abq_batch& b, int heads_q, int rotary_dim, bool interleaved, const float* inv_freq,
                            const uint16_t* q, int ldq, const uint16_t* k, int ldk, const uint16_t* v, int ldv, uint16_t* q_out, hipStream_t s)
{
    const KvAppendArgs a{c, b, heads_q, rotary_dim, __builtin_ctz(c.page_size), interleaved, inv_freq, q, k, v, ldq, ldk, ldv, q_out};
    if (c.kv_bits == 8) append<true>(a, s);
    else append<false>(a, s);
    return hipGetLastError();
}

// One workgroup per slot (and run of 256 eights of its vectors): codes back to values, binary16 values as they are.
__global__ __launch_bounds__(256) void kv_read_kernel(abq_kv_cache c, const int32_t* slots, uint16_t* k_out, uint16_t* v_out, int page_shift)
{
    const int D = c.head_dim, per_vector = D / 8, n = c.heads * per_vector;
    const int i = blockIdx.y * 256 + threadIdx.x;
    if (i >= 2 * n) return;
    const bool is_v = i >= n;
    const int head = (is_v ? i - n : i) / per_vector, at = 8 * ((is_v ? i - n : i) % per_vector);
    const int slot = slots[blockIdx.x], page = slot >> page_shift;
    uint32_t h[4] = {0, 0, 0, 0};
    if (slot >= 0 && page < c.num_pages) {
        const int64_t vec = vector_of(c, page, head, slot & (c.page_size - 1));
        if (c.kv_bits == 16) {
            load_half8<false>((const uint16_t*)(is_v ? c.v : c.k) + vec * D + at, 0, 8, h);
        } else {
            const uint2 codes = *reinterpret_cast<const uint2*>((const uint8_t*)(is_v ? c.v : c.k) + vec * D + at);
            const float scale = (is_v ? c.v_scale : c.k_scale)[vec];
            const int zero = (is_v ? c.v_zero : c.k_zero)[vec];
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = scale * (float)((int)(((e < 4 ? codes.x : codes.y) >> (8 * (e & 3))) & 255u) - zero);
            to_half8(f, h);
        }
    }
    store_half8<false>((is_v ? v_out : k_out) + ((size_t)blockIdx.x * c.heads + head) * D + at, 0, 8, h);
}

hipError_t launch_kv_read(const abq_kv_cache& c, int count, const int32_t* slots, uint16_t* k_out, uint16_t* v_out, hipStream_t s)
{
    const dim3 grid(count, (c.heads * c.head_dim / 4 + 255) / 256);
    kv_read_kernel<<<grid, 256, 0, s>>>(c, slots, k_out, v_out, __builtin_ctz(c.page_size));
    return hipGetLastError();
}

}  // namespace abq
