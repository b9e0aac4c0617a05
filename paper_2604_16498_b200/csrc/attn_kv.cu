// C entry points of the attention over a KV cache of any format.  The kernels are in attn_kv_narrow.cuh and attn_kv_rows.cuh.
#include "attn_kv.cuh"

namespace forge {
template <> int run_attn_kv<FORGE_KV_BF16>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t);
template <> int run_attn_kv<FORGE_KV_F16>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t);
template <> int run_attn_kv<FORGE_KV_INT8>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t);
template <> int run_attn_kv<FORGE_KV_E4M3>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t);

namespace {

// How the G T rows of a KV head form tiles: of as many whole heads as 128 rows hold.
struct RowSplit { int tiles, heads; };
RowSplit split_rows(int G, int T) {
    RowSplit s;
    s.heads = 128 / T < G ? 128 / T : G;
    s.tiles = (G + s.heads - 1) / s.heads;
    return s;
}
// What a workspace has for counters: kKvCounterBytes, and for more (sequence, KV head, row tile) items than that has counters four bytes for each, which
// nothing uses any more (workspaces keep the sizes that they had when each item had a counter of its own).
size_t counter_bytes(size_t items) {
    const size_t n = items * sizeof(unsigned int);
    return ((n > kKvCounterBytes ? n : kKvCounterBytes) + 255) & ~(size_t)255;
}

// Floats of what a CTA leaves of an item: O, m and l of the rows that its kernel works on.
size_t part_floats(long long rows, int D) { return (size_t)(rows <= kNarrowRows ? 8 : 128) * ((D <= 64 ? 64 : 128) + 4); }

int attn_kv(const forge_kv_cache* cache, const void* q, void* out, int dtype, int Hq, int T, bool own_rows, const int64_t* q_strides,
            const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B, float scale, void* workspace,
            size_t workspace_bytes, void* stream) {
    int st = check_cache(cache, dtype);
    if (st != FORGE_OK) return st;
    if (!q || !out || !lens || Hq <= 0 || T <= 0 || Hq % cache->Hkv != 0) return FORGE_ERR_INVALID_ARG;
    if (!aligned16(q) || !aligned16(out) || (reinterpret_cast<uintptr_t>(lens) & 3u)) return FORGE_ERR_INVALID_ARG;
    if (tree && ((reinterpret_cast<uintptr_t>(tree) & 7u) || (tree_B != 1 && tree_B != cache->B))) return FORGE_ERR_INVALID_ARG;
    if (!workspace || !aligned16(workspace)) return FORGE_ERR_INVALID_ARG;
    const float scale_log2 = scale * 1.4426950408889634f;
    if (T > kKvMaxTokens || Hq > 65535 || !(scale_log2 - scale_log2 == 0.f)) return FORGE_ERR_UNSUPPORTED;
    KvAttnArgs a = {};
    if ((st = check_strides(q_strides, Hq, T, cache->D, &a.qs)) != FORGE_OK) return st;
    if ((st = check_strides(out_strides, Hq, T, cache->D, &a.os)) != FORGE_OK) return st;
    if (workspace_bytes < forge_attn_kv_workspace_bytes(cache->B, Hq, cache->Hkv, T, cache->D)) return FORGE_ERR_WORKSPACE;
    const int G = Hq / cache->Hkv;
    const RowSplit rs = split_rows(G, T);
    const long long items = (long long)cache->B * cache->Hkv * rs.tiles;
    const long long tiles = items * (((long long)cache->Smax + 15) / 16);  // of the smallest size
    if (tiles >= (1LL << 31)) return FORGE_ERR_UNSUPPORTED;  // counted in 32 bits
    a.q = q;
    a.v = cache->v;
    a.out = out;
    a.lens = lens;
    a.tree = reinterpret_cast<const unsigned long long*>(tree);
    a.tree_stride = tree_B == 1 ? 0 : T;
    a.T = own_rows ? T : 0;
    a.B = cache->B; a.Hkv = cache->Hkv; a.G = G; a.Smax = cache->Smax; a.D = cache->D;
    a.rows = G * T;
    a.row_tiles = rs.tiles;
    a.tile_heads = rs.heads;
    a.tile_rows = rs.heads * T;
    a.tile_stride = (a.tile_rows + 31) / 32 * 32;
    a.q_f16 = dtype == FORGE_DTYPE_F16;
    a.scale_log2 = scale_log2;
    a.counters = static_cast<unsigned int*>(workspace);
    a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace) + kKvCounterBytes);
    a.status = device_status_word();
    const int sms = sm_count();
    if (!a.status || sms <= 0) return FORGE_ERR_CUDA;
    int ctas = sms < kKvMaxCtas ? sms : kKvMaxCtas;
    if (tiles < ctas) ctas = (int)tiles;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    switch (cache->format) {
        case FORGE_KV_BF16: return run_attn_kv<FORGE_KV_BF16>(*cache, a, ctas, s);
        case FORGE_KV_F16: return run_attn_kv<FORGE_KV_F16>(*cache, a, ctas, s);
        case FORGE_KV_INT8: return run_attn_kv<FORGE_KV_INT8>(*cache, a, ctas, s);
        default: return run_attn_kv<FORGE_KV_E4M3>(*cache, a, ctas, s);
    }
}

}  // namespace
}  // namespace forge

extern "C" size_t forge_attn_kv_workspace_bytes(int B, int Hq, int Hkv, int T, int D) {
    using namespace forge;
    if (B <= 0 || Hq <= 0 || Hkv <= 0 || T <= 0 || D <= 0 || Hq % Hkv != 0) return 0;
    if (T > kKvMaxTokens) return 0;
    const long long rows = (long long)Hq / Hkv * T;
    const RowSplit rs = split_rows(Hq / Hkv, T);
    return counter_bytes((size_t)B * Hkv * rs.tiles) + (size_t)kKvMaxCtas * 2 * part_floats(rows, D) * sizeof(float);
}

extern "C" int forge_attn_kv_workspace_init(void* workspace, size_t workspace_bytes, void* stream) {
    return forge_attn_decode_workspace_init(workspace, workspace_bytes, stream);
}

extern "C" int forge_attn_decode_kv(const forge_kv_cache* cache, const void* q, void* out, int dtype, int Hq, const int32_t* lens,
                                    float scale, void* workspace, size_t workspace_bytes, void* stream) {
    return forge::attn_kv(cache, q, out, dtype, Hq, 1, false, nullptr, nullptr, lens, nullptr, 1, scale, workspace, workspace_bytes, stream);
}

extern "C" int forge_attn_tree(const forge_kv_cache* cache, const void* q, void* out, int dtype, int Hq, int T, const int64_t* q_strides,
                               const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B, float scale,
                               void* workspace, size_t workspace_bytes, void* stream) {
    return forge::attn_kv(cache, q, out, dtype, Hq, T, true, q_strides, out_strides, lens, tree, tree_B, scale, workspace,
                          workspace_bytes, stream);
}
