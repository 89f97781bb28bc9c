// Linear cross entropy, bfloat16: logits become their rows' statistics (xent_kernel.hpp).
#include "xent_kernel.hpp"
namespace fg {
FG_XENT_TABLE(kernel_table_xent_stats_bf16, XENT_STATS, true, true, true, "xent_stats_bf16")
}
