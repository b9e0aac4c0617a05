// Attention of a few query rows per (sequence, KV head) over a KV cache of 16-bit or 8-bit rows.
//
// A (sequence, KV head) has R = G T query rows: its G heads for each of T tokens (T = 1: the decode step; more: a tree of drafted
// tokens whose own rows are the last of the cache).  With p_j = exp2(scale log2(e) q.k_j - m) and running m,
//     l = sum_j p_j        O = sum_j p_j v_j        out = O / l,
// and what is computed over different keys is merged with the usual 2^(m - M) weights.  8-bit rows enter the products as codes
// (exact in fp16); their scales multiply the score and the probability: q.k_j = ks_j (q.kc_j), p_j v_j = (p_j vs_j) vc_j.
//
// The work is bound by reading K and V once, and with many rows by the tensor cores.  One CTA per SM; a long sequence is shared by several, and
// what they have of it is merged by the one that finishes last (arrival counters).  Up to 8 rows run on attn_kv_narrow.cuh (warp-level
// products with the keys as the 16-row operand), more on attn_kv_rows.cuh (tcgen05, a tile of 128 rows).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_math.cuh"
#include "kv_cache.cuh"
#include "mma_16816.cuh"
#include "sm100_ptx.cuh"
#include "tmap.cuh"

namespace forge {

constexpr int kKvMaxCtas = 160;         // what the workspace has room for
constexpr int kKvMaxTokens = 64;
// The workspace: arrival counters, one for each part of an item that several CTAs share (that of the item's first part is used), then the parts.  The
// counters' place does not depend on the shape, so that calls of any shapes leave each other's at zero.
constexpr size_t kKvCounterBytes = 65536 * sizeof(unsigned int);
static_assert(kKvMaxCtas * 2 * sizeof(unsigned int) <= kKvCounterBytes, "a counter for each part");

struct KvAttnArgs {
    const void* q;
    const void* v;                   // the cache's
    void* out;
    Strides qs, os;
    const int32_t* lens;
    const unsigned long long* tree;  // NULL: a chain
    int tree_stride;                 // of a sequence in `tree`
    int T;                           // tokens; their rows are the last ones of the cache (0: one token that has none)
    int B, Hkv, G, Smax, D;
    int rows, row_tiles, tile_rows;  // G * T; groups of rows (of tile_heads whole heads), and how many a group has
    int tile_heads, tile_stride;     // rows between the columns of a part in the workspace
    bool q_f16;
    float scale_log2;
    unsigned int* counters;
    float* parts;                    // [cta][2]: what a CTA leaves of the items at the ends of its run
    int* status;
    // a cache in pages: the rows of a sequence are those of the pages that its row of the table names, in that order
    const int32_t* table;            // [B, max_pages]
    int max_pages, num_pages, page_shift;
    // The heads of a KV head may be worked on as those of several KV heads with the same rows: Hkv, G and rows count these parts then.
    int page_heads;                  // KV heads that a page has
    unsigned part_mul;               // 2^32 / parts of a KV head, rounded up; 0: one part
};

namespace {

// A cache in pages.  Copies take boxes of rows that lie in one page: as many as a page has, up to the rows of a block.  An entry of the table that names
// no page, and one behind the sequence's last row, becomes box -1, which the copy engine fills with zeros.
__device__ __forceinline__ int page_entry(const KvAttnArgs& a, int b, int page) {
    return page < a.max_pages ? __ldcg(a.table + (int64_t)b * a.max_pages + page) : -1;  // L2's: the kernel before this one may have had old ones in L1
}
__device__ __forceinline__ int page_box(const KvAttnArgs& a, int entry, int kvh) {
    if (a.part_mul) kvh = (int)__umulhi((unsigned)kvh, a.part_mul);
    return (unsigned)entry < (unsigned)a.num_pages ? entry * a.page_heads + kvh : -1;
}

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void lds4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void lds2(uint32_t addr, uint32_t& a, uint32_t& b) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(addr) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_dst), "l"(src), "r"(bytes), "r"(ptx::smem_u32(bar))
                 : "memory");
}

// From L2, like the table: the kernels before this one, which may have made room for more rows, may still run while its CTAs already do, and a read of constant
// data (0.1 to 0.6 us less for a call) may give what they had not written yet, or leave before they are waited for.
__device__ __forceinline__ int kv_past(const KvAttnArgs& a, int b) { return min(max(__ldcg(a.lens + b), 0), a.Smax); }
// Rows that any token of the sequence may see.
__device__ __forceinline__ int kv_rows(const KvAttnArgs& a, int past) { return min(past + a.T, a.Smax); }
// Tiles of KEYS keys of a (sequence, KV head): one at least, so that a sequence without rows gets its zeros.
template <int KEYS>
__device__ __forceinline__ int kv_tiles(const KvAttnArgs& a, int past) { return max((kv_rows(a, past) + KEYS - 1) / KEYS, 1); }

// A sequence of the call: its number, its first tile (of all its KV heads), its past and the tiles of one (KV head, row tile).
struct KvCursor {
    int b, base, past, tiles;
};

__device__ __forceinline__ int kv_scan(int v, int lane) {  // inclusive sum over lanes
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += t;
    }
    return v;
}
__device__ __forceinline__ int kv_sum(int v) { return __reduce_add_sync(0xffffffffu, v); }  // over all lanes
__device__ __forceinline__ int kv_max(int v) { return __reduce_max_sync(0xffffffffu, v); }

// 8-bit rows of V: the products' operand is p vs (vs the row's scale) in fp16, and what a query row has of it may be anything: scales differ by
// up to 2^230, and a row of any size may have next to no weight.  So each query row has a unit of its own, a power of two by which its
// p vs are divided and in which its O is kept.  It follows the largest p vs that the row has met, seen rows alone: raised where one would pass 2^14 in
// fp16 (so that the largest comes to 2^5 .. 2^6: what is more than 2^30 smaller than the largest is lost, and no more), and lowered with p when the
// reference m is raised.  Units are 2^kUnitLow to 2^122: the smallest scale that a cache has is 2^-109, and p at least 2^-9 for the largest.
// unit_inv holds 1 / unit.  p is at most 1 there, so that p vs stays finite.
constexpr int kUnitLow = -125, kUnitHigh = 122;
constexpr float kUnitTop = 16384.f;
__device__ __forceinline__ float kv_pow2(int n) { return __int_as_float(max(n + 127, 0) << 23); }  // n <= 127; 0 below 2^-126
__device__ __forceinline__ int kv_log2(float pow2) { return (__float_as_int(pow2) >> 23) - 127; }
__device__ __forceinline__ float kv_unit(float unit_inv) { return kv_pow2(-kv_log2(unit_inv)); }
// Both return what O is multiplied by.  p becomes 2^by times what it was (by: a whole number, at most 0): so does the unit, as far down as it goes.
__device__ __forceinline__ float kv_lower_unit(float& unit_inv, float by) {
    const int unit = -kv_log2(unit_inv) + (int)fmaxf(by, -300.f), now = max(unit, kUnitLow);
    unit_inv = kv_pow2(-now);
    return kv_pow2(unit - now);
}
// `most`: the largest |p vs| of the row that is about to enter O.
__device__ __forceinline__ float kv_raise_unit(float& unit_inv, float most) {
    if (!(most * unit_inv > kUnitTop)) return 1.f;
    const int unit = -kv_log2(unit_inv), now = min(kv_log2(most) + 1 - 6, kUnitHigh);
    unit_inv = kv_pow2(-now);
    return kv_pow2(unit - now);
}

// Two elements of P as the operand of the product with V, and what that leaves of them, for a second product.  16-bit rows may hold infinities, and times
// a rest of zero or below they would become NaN: P is rounded towards zero there, and the rest is above zero where P is (bf16: 2^-23 of P at
// least; fp16: its smallest number).
template <bool F16, bool INFINITIES>
__device__ __forceinline__ uint32_t kv_operand(float x, float y) {
    if constexpr (!INFINITIES) {
        return pack16<F16>(x, y);
    } else if constexpr (F16) {
        uint32_t p;
        asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(p) : "f"(y), "f"(x));
        return p;
    } else {
        return __byte_perm(__float_as_uint(x), __float_as_uint(y), 0x7632);
    }
}
template <bool F16, bool INFINITIES>
__device__ __forceinline__ uint32_t kv_rest(float x, float y, uint32_t p) {
    float2 was;
    if constexpr (F16) was = __half22float2(*reinterpret_cast<const __half2*>(&p));
    else was = make_float2(__uint_as_float(p << 16), __uint_as_float(p & 0xffff0000u));
    if constexpr (!INFINITIES) {
        return pack16<F16>(x - was.x, y - was.y);
    } else if constexpr (F16) {
        constexpr float kLeast = 5.9604644775390625e-8f;  // 2^-24
        return pack16<true>(fmaxf(x - was.x, fminf(x, kLeast)), fmaxf(y - was.y, fminf(y, kLeast)));
    } else {
        constexpr float kMore = 1.00000011920928955078125f;  // 1 + 2^-23
        return pack16<false>(fmaf(x, kMore, -was.x), fmaf(y, kMore, -was.y));
    }
}

// n / d for quotients up to a few thousand: the float quotient is off by one at most.
__device__ __forceinline__ int kv_small_quotient(int n, int d) {
    const int q = (int)__fdividef((float)n, (float)d), rest = n - q * d;
    return q + (rest >= d ? 1 : rest < 0 ? -1 : 0);
}
// Whole numbers 0 .. n - 1 shared evenly by `by` (at most n) of them, in order: the first n % by get one more than the others.
struct KvShares {
    int by, each, more;
    __device__ __forceinline__ KvShares(int n, int by_) : by(by_), each(n / by_), more(n - each * by_) {}
    __device__ __forceinline__ int first(int i) const { return i * each + min(i, more); }
    __device__ __forceinline__ int of(int u) const {  // who has u
        const int low = more * (each + 1);
        return u < low ? kv_small_quotient(u, each + 1) : more + kv_small_quotient(u - low, max(each, 1));
    }
};

// The call's tiles of up to 8 rows, which W CTAs share (at least LEAST each; or one item each, if the longest then has at most MERGE tiles
// more than an even share, which is what joining parts of several CTAs takes), and the sequence in which tile u lies.  Lane l keeps what there
// is to know of sequence l, so that up to 32 sequences are read once.
template <int KEYS, int LEAST, int MERGE>
struct KvSchedule {
    int N, W;
    bool whole;                    // CTA i has item i, all of it
    int past0, tiles0, incl0;
    __device__ __forceinline__ KvSchedule(const KvAttnArgs& a, int lane) {
        past0 = lane < a.B ? kv_past(a, lane) : 0;
        tiles0 = lane < a.B ? kv_tiles<KEYS>(a, past0) : 0;
        incl0 = kv_scan(tiles0, lane);
        int total = tiles0, most = tiles0;
        for (int b = 32 + lane; b < a.B; b += 32) {
            const int tiles = kv_tiles<KEYS>(a, kv_past(a, b));
            total += tiles;
            most = max(most, tiles);
        }
        N = kv_sum(total) * a.Hkv;
        most = kv_max(most);
        // Adding one part to a merge takes as long as a tile: n + most / n is smallest at sqrt(most).  8/1 heads of 128, one sequence, with 8 tiles at
        // least and with this: 32,000 int8 rows 24.8 and 16.7 us, 8000 11.4 and 11.3; 8000 bf16 rows 14.7 and 10.8.
        const int least = max(LEAST, (int)__fsqrt_rn((float)most));
        W = min((int)gridDim.x, (N + least - 1) / least);
        const int items = a.B * a.Hkv;
        whole = items <= (int)gridDim.x && most <= N / W + MERGE;
        if (whole) W = items;
    }
    // The first tile of item i, and (whole) where the CTA's share ends.
    __device__ __forceinline__ int item_at(const KvAttnArgs& a, int i, int lane, int* end) const {
        const int b = i / a.Hkv, kvh = i - b * a.Hkv;
        int before = 0, tiles = tiles0, incl = incl0;
#pragma unroll 1
        for (int b0 = 32; b0 <= b; b0 += 32) {
            before += __shfl_sync(0xffffffffu, incl, 31);
            tiles = b0 + lane < a.B ? kv_tiles<KEYS>(a, kv_past(a, b0 + lane)) : 0;
            incl = kv_scan(tiles, lane);
        }
        const int n = __shfl_sync(0xffffffffu, tiles, b & 31);
        const int first = (before + __shfl_sync(0xffffffffu, incl, b & 31) - n) * a.Hkv + kvh * n;
        *end = first + n;
        return first;
    }
    __device__ __forceinline__ int past_of(const KvAttnArgs& a, int b) const {  // the same b in all lanes
        return b < 32 ? __shfl_sync(0xffffffffu, past0, b) : kv_past(a, b);
    }
    __device__ __forceinline__ void at(const KvAttnArgs& a, int u, KvCursor& cur, int lane) const {
        const int per = a.Hkv;
        int before = 0, past = past0, tiles = tiles0, incl = incl0;
#pragma unroll 1
        for (int b0 = 0;; b0 += 32) {
            const unsigned hit = __ballot_sync(0xffffffffu, u < (before + incl) * per);
            if (hit || b0 + 32 >= a.B) {
                const int src = hit ? __ffs(hit) - 1 : 0;
                cur.b = b0 + src;
                cur.tiles = __shfl_sync(0xffffffffu, tiles, src);
                cur.past = __shfl_sync(0xffffffffu, past, src);
                cur.base = (before + __shfl_sync(0xffffffffu, incl, src) - cur.tiles) * per;
                return;
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
            past = b0 + 32 + lane < a.B ? kv_past(a, b0 + 32 + lane) : 0;
            tiles = b0 + 32 + lane < a.B ? kv_tiles<KEYS>(a, past) : 0;
            incl = kv_scan(tiles, lane);
        }
    }
};

}  // namespace
}  // namespace forge

#include "attn_kv_narrow.cuh"
#include "attn_kv_rows.cuh"

namespace forge {

// One per format, each in a file of its own (they compile side by side).
// PAGED: `cache` has the pages as its sequences, of a page's rows each.
template <int FMT, bool PAGED>
int run_attn_kv(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s);
#define FORGE_ATTN_KV_FORMAT(fmt, paged)                                                                  \
    template <>                                                                                           \
    int run_attn_kv<fmt, paged>(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) { \
        if (a.rows <= kNarrowRows)                                                                        \
            return cache.D <= 64 ? launch_attn_kv_narrow<64, fmt, paged>(cache, a, ctas, s) : launch_attn_kv_narrow<128, fmt, paged>(cache, a, ctas, s); \
        return cache.D <= 64 ? launch_attn_kv_rows<64, fmt, paged>(cache, a, ctas, s) : launch_attn_kv_rows<128, fmt, paged>(cache, a, ctas, s); \
    }

}  // namespace forge
