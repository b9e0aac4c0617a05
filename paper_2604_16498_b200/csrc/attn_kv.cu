// C entry points of the attention over a KV cache of any format, in one block or in pages.  The kernels are in attn_kv_narrow.cuh and attn_kv_rows.cuh.
#include "attn_kv.cuh"

namespace forge {
#define FORGE_RUN_ATTN_KV(fmt)                                                               \
    template <> int run_attn_kv<fmt, false>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t); \
    template <> int run_attn_kv<fmt, true>(const forge_kv_cache&, const KvAttnArgs&, int, cudaStream_t)
FORGE_RUN_ATTN_KV(FORGE_KV_BF16);
FORGE_RUN_ATTN_KV(FORGE_KV_F16);
FORGE_RUN_ATTN_KV(FORGE_KV_INT8);
FORGE_RUN_ATTN_KV(FORGE_KV_E4M3);

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

// A cache in pages: the query heads of a KV head that are worked on in parts of up to 8 rows each, on the kernel for those, although it then reads K
// and V once for each part (all but the first from L2): how many parts, 1 where the other kernel is the one.  How long the requests are is not known here, so
// the rule goes by the number of parts and the rows' type alone.  Measured with 1 to 512 KV heads in all, 256 to 65,536 rows each (and down to a quarter of
// that), single tokens of 12 to 32 heads to a KV head and trees of 4 to 8 tokens; the tile of 128 rows takes, in times of what the parts take (means are geometric):
//   8-bit rows of 64     2 parts 1.02 .. 3.9, 3 parts 1.03 .. 2.6, 4 parts 0.89 .. 2.4 (mean 1.41)
//   8-bit rows of 128    2 parts 1.03 .. 2.7, 3 parts 1.06 .. 2.3, 4 parts 0.82 .. 2.1 (mean 1.21; below 1 from 8 KV heads of long requests on: 64 x 32/1 heads,
//     1024 rows, 20.5 us in parts and 19.3; 32, 4096 rows 28.5 and 27.0; but 512, 1024 rows 89 and 107, 1, 4096 rows 14.8 and 20.7)
//   16-bit rows of 64    2 parts 0.88 .. 2.4 (mean 1.40); 4 parts 0.59 .. 1.9 (mean 1.04)
//   16-bit rows of 128   2 parts 0.83 .. 2.2 (mean 1.31; below 1 from 16,384 rows and 32 KV heads on, whose K and V leave L2 between the parts: 32 x 16/1 heads,
//     16,384 rows 50.9 us in parts and 42.4; but 64, 4096 rows 28.3 and 35.7, 128, 4096 rows 38.6 and 59.4, 1, 4096 rows 10.3 and 18.8); 4 parts 0.47 .. 1.8 (mean 0.98)
int narrow_parts(const forge_kv_cache& c, int G, int T) {
    if (G * T <= kNarrowRows) return 1;
    const int most = eight_bit(c.format) ? 4 : 2;
    for (int parts = 2; parts <= most; ++parts)
        if (G % parts == 0 && G / parts * T <= kNarrowRows) return parts;
    return 1;
}

// Floats of what a CTA leaves of an item: O, m and l of the rows that its kernel works on.
size_t part_floats(long long rows, int D) { return (size_t)(rows <= kNarrowRows ? 8 : 128) * ((D <= 64 ? 64 : 128) + 4); }

template <bool PAGED>
int run_format(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {
    switch (cache.format) {
        case FORGE_KV_BF16: return run_attn_kv<FORGE_KV_BF16, PAGED>(cache, a, ctas, s);
        case FORGE_KV_F16: return run_attn_kv<FORGE_KV_F16, PAGED>(cache, a, ctas, s);
        case FORGE_KV_INT8: return run_attn_kv<FORGE_KV_INT8, PAGED>(cache, a, ctas, s);
        default: return run_attn_kv<FORGE_KV_E4M3, PAGED>(cache, a, ctas, s);
    }
}

// cache: as the tokens see it.  pages: the memory, where that is in pages that `table` puts in order.
int attn_kv(const forge_kv_cache* cache, const forge_kv_pages* pages, const int32_t* table, const void* q, void* out, int dtype, int Hq, int T,
            bool own_rows, const int64_t* q_strides, const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B, float scale,
            void* workspace, size_t workspace_bytes, void* stream) {
    int st;
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
    const int most = sms < kKvMaxCtas ? sms : kKvMaxCtas;
    auto ctas_for = [&](long long n) { return n < most ? (int)n : most; };
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (!pages) return run_format<false>(*cache, a, ctas_for(tiles), s);
    a.page_heads = cache->Hkv;
    int parts = narrow_parts(*cache, G, T);
    if (tiles * parts >= (1LL << 31)) parts = 1;
    if (parts > 1) {
        a.Hkv *= parts;
        a.G /= parts;
        a.rows /= parts;
        a.part_mul = (unsigned)(((1ULL << 32) + parts - 1) / parts);
    }
    a.table = table;
    a.num_pages = pages->num_pages;
    a.max_pages = cache->Smax / pages->page_size;
    a.page_shift = log2_of(pages->page_size);
    const forge_kv_cache memory = {pages->k, pages->v, pages->k_scale, pages->v_scale, pages->num_pages, pages->Hkv, pages->page_size, pages->D, pages->format};
    return run_format<true>(memory, a, ctas_for(tiles * parts), s);
}

int attn_cache(const forge_kv_cache* cache, const void* q, void* out, int dtype, int Hq, int T, bool own_rows, const int64_t* q_strides,
               const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B, float scale, void* workspace,
               size_t workspace_bytes, void* stream) {
    const int st = check_cache(cache, dtype);
    if (st != FORGE_OK) return st;
    return attn_kv(cache, nullptr, nullptr, q, out, dtype, Hq, T, own_rows, q_strides, out_strides, lens, tree, tree_B, scale, workspace,
                   workspace_bytes, stream);
}
int attn_pages(const forge_kv_pages* pages, const int32_t* table, int B, int max_pages, const void* q, void* out, int dtype, int Hq, int T,
               bool own_rows, const int64_t* q_strides, const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B,
               float scale, void* workspace, size_t workspace_bytes, void* stream) {
    int st = check_pages(pages, dtype), rows = 0;
    if (st != FORGE_OK) return st;
    if ((st = check_table(table, B, max_pages, pages->page_size, &rows)) != FORGE_OK) return st;
    const forge_kv_cache seen = {pages->k, pages->v, pages->k_scale, pages->v_scale, B, pages->Hkv, rows, pages->D, pages->format};
    return attn_kv(&seen, pages, table, q, out, dtype, Hq, T, own_rows, q_strides, out_strides, lens, tree, tree_B, scale, workspace,
                   workspace_bytes, stream);
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
    return forge::attn_cache(cache, q, out, dtype, Hq, 1, false, nullptr, nullptr, lens, nullptr, 1, scale, workspace, workspace_bytes, stream);
}

extern "C" int forge_attn_tree(const forge_kv_cache* cache, const void* q, void* out, int dtype, int Hq, int T, const int64_t* q_strides,
                               const int64_t* out_strides, const int32_t* lens, const int64_t* tree, int tree_B, float scale,
                               void* workspace, size_t workspace_bytes, void* stream) {
    return forge::attn_cache(cache, q, out, dtype, Hq, T, true, q_strides, out_strides, lens, tree, tree_B, scale, workspace,
                             workspace_bytes, stream);
}

extern "C" int forge_attn_decode_pages(const forge_kv_pages* cache, const int32_t* table, int B, int max_pages, const void* q, void* out,
                                       int dtype, int Hq, const int32_t* lens, float scale, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    return forge::attn_pages(cache, table, B, max_pages, q, out, dtype, Hq, 1, false, nullptr, nullptr, lens, nullptr, 1, scale, workspace,
                             workspace_bytes, stream);
}

extern "C" int forge_attn_tree_pages(const forge_kv_pages* cache, const int32_t* table, int B, int max_pages, const void* q, void* out,
                                     int dtype, int Hq, int T, const int64_t* q_strides, const int64_t* out_strides, const int32_t* lens,
                                     const int64_t* tree, int tree_B, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    return forge::attn_pages(cache, table, B, max_pages, q, out, dtype, Hq, T, true, q_strides, out_strides, lens, tree, tree_B, scale,
                             workspace, workspace_bytes, stream);
}
