// Linear cross entropy, binary16: logits become their rows' statistics (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_stats_f16, XENT_STATS, true, true, false, "xent_stats_f16")
}
