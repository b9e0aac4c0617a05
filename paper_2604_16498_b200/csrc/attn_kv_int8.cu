// Attention over a KV cache, format FORGE_KV_INT8.  The kernel is in attn_kv.cuh.
#include "attn_kv.cuh"

namespace forge {
FORGE_ATTN_KV_FORMAT(FORGE_KV_INT8)
}
