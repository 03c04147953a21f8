// Attention over the paged cache, heads of 129 to 256.
#include "abq_attn_kernels.h"

ABQ_ATTN_INSTANTIATE(256)
