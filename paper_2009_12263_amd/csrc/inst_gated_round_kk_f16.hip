// Gated feed-forward block, binary16: rounded products, A and B contiguous along K (gated_kernel.hpp).
#include "gated_kernel.hpp"
namespace fg {
FG_GATED_TABLE(kernel_table_gated_round_kk_f16, GATED_ROUND_KK, true, true, false, "gated_round_kk_f16")
}
