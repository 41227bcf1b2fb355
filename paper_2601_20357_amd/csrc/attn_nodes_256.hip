// Attention over trees, heads of 256 dims.
#include "attn_nodes.h"
namespace tabed {
TABED_NODES_HD(256)
}
