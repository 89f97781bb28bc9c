// Gated feed-forward block, bfloat16: rounded products, neither operand contiguous along K (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_round_nn_bf16, GATED_ROUND_NN, false, false, true, "gated_round_nn_bf16")
}
