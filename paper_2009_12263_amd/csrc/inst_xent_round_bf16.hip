// Linear cross entropy, bfloat16: rows of dw (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_round_bf16, XENT_ROUND, false, false, true, "xent_round_bf16")
}
