// Linear cross entropy, binary16: rows of dw (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_round_f16, XENT_ROUND, false, false, false, "xent_round_f16")
}
