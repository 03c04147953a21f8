// Attention over the paged cache, heads of up to 64.
#include "abq_attn_kernels.h"

ABQ_ATTN_INSTANTIATE(64)
ABQ_ATTN_INSTANTIATE_BOTH(64)
