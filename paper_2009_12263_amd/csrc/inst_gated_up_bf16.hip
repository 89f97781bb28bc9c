// Gated feed-forward block, bfloat16: X W_in^T becomes h (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_up_bf16, GATED_UP, true, true, true, "gated_up_bf16")
}
