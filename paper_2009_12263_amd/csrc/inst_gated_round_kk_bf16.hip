// Gated feed-forward block, bfloat16: rounded products, A and B contiguous along K (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_round_kk_bf16, GATED_ROUND_KK, true, true, true, "gated_round_kk_bf16")
}
