// Attention of a step's rows over the paged cache: one wave per row and query head, 64 tokens at a time, running maximum and
// sum in binary32.
#include "abq_kv.h"

namespace abq {

__device__ __forceinline__ float cache_value(const abq_kv_cache& c, bool is_v, int64_t vec, int d)
{
    if (c.kv_bits == 16) return __half2float(__ushort_as_half(((const uint16_t*)(is_v ? c.v : c.k))[vec * c.head_dim + d]));
    const int code = ((const uint8_t*)(is_v ? c.v : c.k))[vec * c.head_dim + d], zero = (is_v ? c.v_zero : c.k_zero)[vec];
    return (is_v ? c.v_scale : c.k_scale)[vec] * (float)(code - zero);
}

__global__ __launch_bounds__(64) void attn_rows_kernel(abq_kv_cache c, abq_batch b, int heads_q, const uint16_t* q, int ldq, float scale, bool causal,
                                                       uint16_t* y, int page_shift)
{
    __shared__ float sq[256], sp[64];
    __shared__ int64_t sv[64];
    const int row = blockIdx.x, hq = blockIdx.y, lane = threadIdx.x, D = c.head_dim, head = hq / (heads_q / c.heads);
    int seq = 0;
    while (seq < b.seqs && b.row_start[seq + 1] <= row) ++seq;
    if (seq >= b.seqs || row - b.row_start[seq] >= b.max_new) return;
    const int len = min(max(b.lens[seq], 0), b.max_len);
    const int64_t pos = (int64_t)b.lens[seq] - ((int64_t)b.row_start[seq + 1] - row);
    const int seen = causal ? (int)min((int64_t)len, max(pos + 1, (int64_t)0)) : len;
    for (int d = lane; d < D; d += 64) sq[d] = __half2float(__ushort_as_half(q[(size_t)row * ldq + (size_t)hq * D + d]));
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
    for (int t0 = 0; t0 < seen; t0 += 64) {
        const int t = t0 + lane, page = t < seen ? page_of(b, c, page_shift, seq, t) : -1;
        const int64_t vec = page < 0 ? -1 : vector_of(c, page, head, t & (c.page_size - 1));
        float s = -INFINITY;
        if (vec >= 0) {
            s = 0.0f;
            for (int d = 0; d < D; ++d) s = fmaf(sq[d], cache_value(c, false, vec, d), s);
            s *= scale;
        }
        float top = s;
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float next = fmaxf(m, top), base = next == -INFINITY ? 0.0f : next;
        const float fade = expf(m - base), p = vec >= 0 ? expf(s - base) : 0.0f;
        sp[lane] = p;
        sv[lane] = vec;
        float sum = p;
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
        l = l * fade + sum;
        m = next;
        __syncthreads();
        for (int i = 0; i < 4; ++i) {
            const int d = lane + 64 * i;
            if (d >= D) break;
            float acc = o[i] * fade;
            for (int j = 0; j < 64; ++j)
                if (sv[j] >= 0) acc = fmaf(sp[j], cache_value(c, true, sv[j], d), acc);
            o[i] = acc;
        }
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int d = lane + 64 * i;
        if (d < D) y[((size_t)row * heads_q + hq) * D + d] = __half_as_ushort(__float2half_rn(l == 0.0f ? 0.0f : o[i] / l));
    }
}

size_t attn_workspace_bytes(const abq_kv_cache&, const abq_batch&, int) { return 0; }

hipError_t launch_attn_paged(const abq_kv_cache& c, const abq_batch& b, int heads_q, const uint16_t* q, int ldq, float scale, bool causal,
                             uint16_t* y, void*, hipStream_t s)
{
    attn_rows_kernel<<<dim3(b.rows, heads_q), 64, 0, s>>>(c, b, heads_q, q, ldq, scale, causal, y, __builtin_ctz(c.page_size));
    return hipGetLastError();
}

}  // namespace abq
