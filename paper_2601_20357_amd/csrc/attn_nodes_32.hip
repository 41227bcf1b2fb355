// Attention over trees, heads of 32 dims.
#include "attn_nodes.h"
namespace tabed {
TABED_NODES_HD(32)
}
