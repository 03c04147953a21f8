// The paged cache and the batch as the kernels see them (append, read back, attention).
#pragma once
#include "abq_internal.h"
#include "../../include/abq.h"

namespace abq {

hipError_t launch_kv_append(const abq_kv_cache& c, const abq_batch& b, int heads_q, int rotary_dim, bool interleaved, const float* inv_freq,
                            const uint16_t* q, int ldq, const uint16_t* k, int ldk, const uint16_t* v, int ldv, uint16_t* q_out, hipStream_t s);
hipError_t launch_kv_read(const abq_kv_cache& c, int count, const int32_t* slots, uint16_t* k_out, uint16_t* v_out, hipStream_t s);
size_t attn_workspace_bytes(const abq_kv_cache& c, const abq_batch& b, int heads_q);
hipError_t launch_attn_paged(const abq_kv_cache& c, const abq_batch& b, int heads_q, const uint16_t* q, int ldq, float scale, bool causal,
                             uint16_t* y, void* workspace, hipStream_t s);
size_t lora_workspace_bytes(int M, int N, int K, int rank);
hipError_t launch_lora_add(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids, const uint16_t* a,
                           const uint16_t* b, const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout, void* workspace,
                           hipStream_t s);

// Page of token t of a sequence, -1 where there is none: t outside the table, or an entry that names no page.
__device__ __forceinline__ int page_of(const abq_batch& b, const abq_kv_cache& c, int page_shift, int seq, int t)
{
    const int at = t >> page_shift;
    if (t < 0 || at >= b.max_pages) return -1;
    const int page = b.pages[(size_t)seq * b.max_pages + at];
    return (unsigned)page < (unsigned)c.num_pages ? page : -1;
}

// Vector number of (page, head, offset); element offsets pass 32 bits in a long cache, so everything that multiplies it does so in 64.
__device__ __forceinline__ int64_t vector_of(const abq_kv_cache& c, int page, int head, int offset)
{
    return ((int64_t)page * c.heads + head) * c.page_size + offset;
}

}  // namespace abq
