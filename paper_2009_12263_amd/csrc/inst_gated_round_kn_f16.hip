// Gated feed-forward block, binary16: rounded products, A contiguous along K (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_round_kn_f16, GATED_ROUND_KN, true, false, false, "gated_round_kn_f16")
}
