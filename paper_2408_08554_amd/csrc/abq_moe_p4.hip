// Products with experts' weights: the variants of 4-bit weights.
#include "abq_block_kernels.h"
#include "abq_moe_rows_kernels.h"

namespace abq {
ABQ_MOE_ROWS_LAUNCH(4) { return moe_rows_launch<4>(prm, R, grid, s); }
ABQ_BLOCK_EXPERTS_LAUNCH(4) { return block_experts_launch<4>(prm, shape, s); }
}  // namespace abq
