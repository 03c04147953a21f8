// Low-rank adapters of many requests beside a shared projection: out = y + scale_i B_i (A_i x), i the row's adapter.
// Two kernels: u = A_i x for every row, then the rows of the output.
#include "abq_kv.h"

namespace abq {

// one wave per row and element of u
__global__ __launch_bounds__(64) void lora_shrink_kernel(int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a, float* u)
{
    const int m = blockIdx.x, r = blockIdx.y, lane = threadIdx.x, id = ids[m];
    if ((unsigned)id >= (unsigned)adapters) return;
    const uint16_t *xr = x + (size_t)m * ldx, *ar = a + ((size_t)id * rank + r) * K;
    float s = 0.0f;
    for (int k = lane; k < K; k += 64) s = fmaf(__half2float(__ushort_as_half(xr[k])), __half2float(__ushort_as_half(ar[k])), s);
    for (int off = 32; off > 0; off >>= 1) s += __shfl_xor(s, off, 64);
    if (lane == 0) u[(size_t)m * rank + r] = s;
}

__global__ __launch_bounds__(256) void lora_expand_kernel(int N, int rank, int adapters, const int32_t* ids, const uint16_t* b, const float* scale, const float* u,
                                                          const uint16_t* y, int ldy, uint16_t* out, int ldout)
{
    const int m = blockIdx.x, n = blockIdx.y * 256 + threadIdx.x, id = ids[m];
    if (n >= N) return;
    uint16_t v = y[(size_t)m * ldy + n];
    if ((unsigned)id < (unsigned)adapters) {
        float s = 0.0f;
        for (int r = 0; r < rank; ++r) s = fmaf(u[(size_t)m * rank + r], __half2float(__ushort_as_half(b[((size_t)id * N + n) * rank + r])), s);
        v = __half_as_ushort(__float2half_rn(fmaf(scale[id], s, __half2float(__ushort_as_half(v)))));
    }
    out[(size_t)m * ldout + n] = v;
}

size_t lora_workspace_bytes(int M, int, int, int rank) { return (size_t)M * rank * sizeof(float); }

hipError_t launch_lora_add(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a,
                           const uint16_t* b, const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout, void* workspace,
                           hipStream_t s)
{
    lora_shrink_kernel<<<dim3(M, rank), 64, 0, s>>>(K, rank, adapters, x, ldx, ids, a, (float*)workspace);
    lora_expand_kernel<<<dim3(M, (N + 255) / 256), 256, 0, s>>>(N, rank, adapters, ids, b, scale, (const float*)workspace, y, ldy, out, ldout);
    return hipGetLastError();
}

}  // namespace abq
