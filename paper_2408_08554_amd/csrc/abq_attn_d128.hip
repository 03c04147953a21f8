// Attention over the paged cache, heads of 65 to 128.
#include "abq_attn_kernels.h"

ABQ_ATTN_INSTANTIATE(128)
ABQ_ATTN_INSTANTIATE_BOTH(128)
