// Linear cross entropy, binary16: logits become dz (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_dz_f16, XENT_DZ, true, true, false, "xent_dz_f16")
}
