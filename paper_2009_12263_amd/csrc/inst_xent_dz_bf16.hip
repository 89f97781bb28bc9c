// Linear cross entropy, bfloat16: logits become dz (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_dz_bf16, XENT_DZ, true, true, true, "xent_dz_bf16")
}
