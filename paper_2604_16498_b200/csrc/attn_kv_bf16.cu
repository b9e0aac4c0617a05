// Attention over a KV cache, format FORGE_KV_BF16.  The kernels are in attn_kv_narrow.cuh and attn_kv_rows.cuh.
#include "attn_kv.cuh"

namespace forge {
FORGE_ATTN_KV_FORMAT(FORGE_KV_BF16)
}
