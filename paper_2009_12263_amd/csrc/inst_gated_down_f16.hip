// Gated feed-forward block, binary16: dY W_out becomes dg, du and h (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_down_f16, GATED_DOWN, true, false, false, "gated_down_f16")
}
