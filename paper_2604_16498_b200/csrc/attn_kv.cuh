// Attention of a few query rows per (sequence, KV head) over a KV cache of 16-bit or 8-bit rows.
//
// A (sequence, KV head) has R = G T query rows: its G heads for each of T tokens (T = 1: the decode step; more: a tree of drafted
// tokens whose own rows are the last of the cache).  With p_j = exp2(scale log2(e) q.k_j - m) and running m,
//     l = sum_j p_j        O = sum_j p_j v_j        out = O / l,
// and what is computed over different keys is merged with the usual 2^(m - M) weights.  8-bit rows enter the products as codes
// (exact in fp16); their scales multiply the score and the probability: q.k_j = ks_j (q.kc_j), p_j v_j = (p_j vs_j) vc_j.
//
// The work is bound by reading K and V once, up to about 64 rows; beyond, by the warp-level matrix instructions.  All CTAs
// (one per SM) share the 128-key tiles of the whole call evenly: tiles are numbered through sequences, KV heads and row
// groups, and each CTA takes a run of them.  What a cut leaves in two CTAs is merged by the one that finishes
// last (arrival counters); a CTA has at most two such parts.  Within a CTA a producer warp keeps a ring of whole tiles
// filled by TMA (the scales by 4-byte copies), and eight warps work on every tile: RG of them on different groups of 16 rows,
// 8 / RG on different keys of it, merged when the CTA's part of the sequence ends.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_math.cuh"
#include "kv_cache.cuh"
#include "sm100_ptx.cuh"
#include "tmap.cuh"

namespace forge {

constexpr int kKvMaxCtas = 160;         // what the workspace has room for
constexpr int kKvMaxRows = 128;         // rows of a group of warps: more take further tiles of their own
constexpr int kKvMaxTokens = 64;
constexpr int kMidRows = 8;
constexpr size_t kKvMinCounters = 65536;

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
    int rows, row_tiles, tile_rows;  // G * T; groups of rows, and how many a group has
    int least;                       // rows <= 8: blocks of keys that a CTA has at least
    int RG;                          // warps over the rows: 16 RG >= tile_rows, 1, 2, 4 or 8
    bool q_f16;
    float scale_log2;
    unsigned int* counters;
    float* parts;                    // [cta][2][RG][DW / 2 + 1][32]: fragments of O, then m and l of the 16 rows
    int* status;
};

namespace {

constexpr int kKvWarps = 8;
constexpr int kKvThreads = (kKvWarps + 1) * 32;
constexpr int kTileKeys = 128;
constexpr int kBoxKeys = 64;

template <int DW, int FMT>
struct KvShape {
    static constexpr bool kEight = FMT == FORGE_KV_INT8 || FMT == FORGE_KV_E4M3;
    static constexpr int kKBytes = kTileKeys * DW * (kEight ? 1 : 2);
    static constexpr int kScaleBytes = kEight ? 2 * kTileKeys * 4 : 0;
    static constexpr int kTileBytes = 2 * kKBytes + kScaleBytes;
    static constexpr int kFrag = (DW / 2 + 1) * 32;              // floats of a warp's O, then m and l of its 16 rows
    static constexpr int kMergeBytes = 4 * kFrag * 4;            // half of the warps hand theirs over at a time
    static constexpr int kRoom = 232448 - 1024 - 256 - kMergeBytes;
    static constexpr int kStages = kRoom / kTileBytes < 8 ? kRoom / kTileBytes : 8;
    static constexpr int kSmem = 1024 + kStages * kTileBytes + kMergeBytes;
    static_assert(kStages >= 3, "ring size");
};

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
__device__ __forceinline__ float2 lds_f2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void copy4(uint32_t smem, const float* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem), "l"(src) : "memory");
}
// One of the barrier's counted arrivals, once this thread's copies so far have landed.
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(ptx::smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// D(16 x 8, fp32) += A(16 x 16) B(16 x 8); lane = (g = lane / 4, c = lane % 4) holds of A rows g, g + 8 and k 2c, 2c+1, 2c+8, 2c+9;
// of B column g and the same k; of D rows g, g + 8 and columns 2c, 2c + 1.
template <bool F16>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ int kv_past(const KvAttnArgs& a, int b) { return min(max(__ldg(a.lens + b), 0), a.Smax); }
// Rows that any token of the sequence may see.
__device__ __forceinline__ int kv_rows(const KvAttnArgs& a, int past) { return min(past + a.T, a.Smax); }
// Tiles of KEYS keys of a (sequence, KV head, row group): one at least, so that a sequence without rows gets its zeros.
template <int KEYS>
__device__ __forceinline__ int kv_tiles(const KvAttnArgs& a, int past) { return max((kv_rows(a, past) + KEYS - 1) / KEYS, 1); }

// Where a CTA is in the call's tiles.  Every warp walks through the CTA's share by itself; all lanes hold the same.
struct KvCursor {
    int u, end;          // tiles of the call: the next one, and the end of this CTA's share
    int b, base;         // sequence, and its first tile
    int past, tiles;     // of sequence b
};

// Whole numbers 0 .. n - 1 shared evenly by `by` (at most n) of them, in order: the first n % by get one more than the others.
struct KvShares {
    int by, each, more;
    __device__ __forceinline__ KvShares(int n, int by_) : by(by_), each(n / by_), more(n - each * by_) {}
    __device__ __forceinline__ int first(int i) const { return i * each + min(i, more); }
    __device__ __forceinline__ int of(int u) const {  // who has u
        const int low = more * (each + 1);
        return u < low ? u / (each + 1) : more + (u - low) / max(each, 1);
    }
};

// The call's tiles, which W CTAs share (at least `least` each), and the sequence in which tile u lies: `at(...)` leaves its b, base, past and
// tiles in the cursor.  Lane l keeps what there is to know of sequence l, so that up to 32 sequences are read once.
template <int KEYS>
struct KvSchedule {
    int N, W;
    int past0, tiles0, incl0;
    __device__ __forceinline__ KvSchedule(const KvAttnArgs& a, int least, int lane) {
        past0 = lane < a.B ? kv_past(a, lane) : 0;
        tiles0 = lane < a.B ? kv_tiles<KEYS>(a, past0) : 0;
        incl0 = scan(tiles0, lane);
        int total = tiles0;
        for (int b = 32 + lane; b < a.B; b += 32) total += kv_tiles<KEYS>(a, kv_past(a, b));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        N = total * a.Hkv * a.row_tiles;
        W = min((int)gridDim.x, (N + least - 1) / least);
    }
    static __device__ __forceinline__ int scan(int v, int lane) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, v, o);
            if (lane >= o) v += t;
        }
        return v;
    }
    __device__ __forceinline__ int past_of(const KvAttnArgs& a, int b) const {  // the same b in all lanes
        return b < 32 ? __shfl_sync(0xffffffffu, past0, b) : kv_past(a, b);
    }
    __device__ __forceinline__ void at(const KvAttnArgs& a, int u, KvCursor& cur, int lane) const {
        const int per = a.Hkv * a.row_tiles;
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
            incl = scan(tiles, lane);
        }
    }
};

// The CTA's part of one (sequence, KV head, row group).
struct KvPart {
    int b, kvh, rt, item;      // item: number of the (sequence, KV head, row group)
    int first, tiles, of;      // tiles of it in this CTA, out of how many
    int start;                 // the item's first tile in the call
    int past, rows;
};
__device__ __forceinline__ KvPart kv_part(const KvAttnArgs& a, const KvCursor& cur) {
    KvPart p;
    const int in = cur.u - cur.base, item = in / cur.tiles;
    p.b = cur.b;
    p.kvh = item / a.row_tiles;
    p.rt = item - p.kvh * a.row_tiles;
    p.item = cur.b * a.Hkv * a.row_tiles + item;
    p.first = in - item * cur.tiles;
    p.of = cur.tiles;
    p.tiles = min(cur.tiles - p.first, cur.end - cur.u);
    p.start = cur.u - p.first;
    p.past = cur.past;
    p.rows = kv_rows(a, cur.past);
    return p;
}
template <int KEYS>
__device__ __forceinline__ void kv_advance(const KvAttnArgs& a, KvCursor& cur, int tiles) {
    cur.u += tiles;
    if (cur.u < cur.end && cur.u - cur.base >= cur.tiles * a.Hkv * a.row_tiles) {
        cur.base += cur.tiles * a.Hkv * a.row_tiles;
        cur.past = kv_past(a, ++cur.b);
        cur.tiles = kv_tiles<KEYS>(a, cur.past);
    }
}

// State of a warp's 16 rows: this lane holds rows g and g + 8.
template <int DW>
struct KvState {
    float m[2], l[2], o[DW / 8][4];
    __device__ __forceinline__ void clear() {
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int t = 0; t < DW / 8; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][i] = 0.f;
    }
    // Merges what was computed over other keys: (m2, l2) and a fragment of O behind `src` (floats, 32 apart).
    template <typename Load>
    __device__ __forceinline__ void merge(const float (&m2)[2], const float (&l2)[2], Load load) {
        float wa[2], wb[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float M = fmaxf(m[r], m2[r]);
            const float ref = M == -INFINITY ? 0.f : M;
            wa[r] = ex2(m[r] - ref);
            wb[r] = ex2(m2[r] - ref);
            // a side without keys has nothing to say, whatever the weight (2^-inf is 0, but 0 x inf is NaN)
            l[r] = fmaf(l[r], wa[r], l2[r] * wb[r]);
            m[r] = M;
        }
#pragma unroll
        for (int t = 0; t < DW / 8; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][i] = fmaf(o[t][i], wa[i >> 1], load(t * 4 + i) * wb[i >> 1]);
    }
};

// Which of the 16 rows of V from key0 on (the first `rows` of them) hold something that is not a finite number: bits 2 k and 2 k + 1 for
// row k, whose halves two lanes look through.
template <int DW, bool F16>
__device__ __forceinline__ uint32_t odd_rows(uint32_t vb, int key0, int rows, int lane) {
    constexpr uint32_t kExp = F16 ? 0x7c00u : 0x7f80u;
    const int k = lane >> 1, row = key0 + k;
    bool found = false;
#pragma unroll
    for (int i = 0; i < DW / 16; ++i) {
        const int piece = (lane & 1) * (DW / 16) + i;
        uint32_t w[4];
        lds4(vb + (piece >> 3) * (kTileKeys * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4), w);
#pragma unroll
        for (int x = 0; x < 4; ++x) found |= (w[x] & kExp) == kExp || (w[x] >> 16 & kExp) == kExp;
    }
    return __ballot_sync(0xffffffffu, found && k < rows);
}

template <int DW, int FMT>
__global__ void __launch_bounds__(kKvThreads, 1)
attn_kv_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
               const float* __restrict__ k_scale, const float* __restrict__ v_scale, const KvAttnArgs a) {
    using S = KvShape<DW, FMT>;
    constexpr bool kEight = S::kEight, kE4m3 = FMT == FORGE_KV_E4M3;
    constexpr bool kF16 = FMT != FORGE_KV_BF16;  // operands of the products
    constexpr int NT = DW / 8;                   // 8-wide column tiles of O
    constexpr int KS = DW / 16;                  // 16-wide steps of the scores' contraction
    extern __shared__ __align__(128) uint8_t smem_raw[];
    __shared__ uint64_t full[8], empty[8];
    __shared__ unsigned int arrived_all;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t ring = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    float* merge_buf = reinterpret_cast<float*>(smem_raw + (ring - ptx::smem_u32(smem_raw)) + S::kStages * S::kTileBytes);
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            ptx::mbar_init(&full[i], kEight ? 33 : 1);
            ptx::mbar_init(&empty[i], kKvWarps);
        }
        ptx::fence_mbar_init();
        ptx::prefetch_tmap(&tmap_k);
        ptx::prefetch_tmap(&tmap_v);
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();

    const KvSchedule<kTileKeys> sched(a, 1, lane);
    const KvShares shares(sched.N, sched.W);
    if ((int)blockIdx.x >= sched.W) return;
    KvCursor cur;
    cur.u = shares.first(blockIdx.x);
    cur.end = shares.first(blockIdx.x + 1);
    sched.at(a, cur.u, cur, lane);
    bool failed = false;

    if (warp == kKvWarps) {
        // ------------------------------------------------------------------------ producer
        int n = 0;
        const uint64_t policy = ptx::l2_policy_evict_first();
        while (cur.u < cur.end && !failed) {
            const KvPart p = kv_part(a, cur);
            const int bk = p.b * a.Hkv + p.kvh;
            for (int t = 0; t < p.tiles; ++t, ++n) {
                const int st = n % S::kStages;
                if (n >= S::kStages && !ptx::warp_wait_relaxed(&empty[st], (n / S::kStages - 1) & 1)) { failed = true; break; }
                const int j0 = (p.first + t) * kTileKeys;
                const int rows = min(p.rows - j0, kTileKeys);  // not above 0 for a sequence without rows
                const uint32_t dst = ring + st * S::kTileBytes;
                if (lane == 0) {
                    const int boxes = rows > kBoxKeys ? 2 : rows > 0 ? 1 : 0;
                    ptx::mbar_expect_tx(&full[st], boxes * (S::kKBytes / (kTileKeys / kBoxKeys)) * 2);
                    for (int x = 0; x < boxes; ++x) {
                        if constexpr (kEight) {
                            ptx::tma_load_3d_addr_hint(dst + x * kBoxKeys * DW, &tmap_k, &full[st], 0, j0 + x * kBoxKeys, bk, policy);
                            ptx::tma_load_3d_addr_hint(dst + S::kKBytes + x * kBoxKeys * DW, &tmap_v, &full[st], 0, j0 + x * kBoxKeys, bk, policy);
                        } else {
#pragma unroll
                            for (int cb = 0; cb < DW / 64; ++cb) {
                                const uint32_t at = dst + cb * (kTileKeys * 128) + x * (kBoxKeys * 128);
                                ptx::tma_load_3d_addr_hint(at, &tmap_k, &full[st], cb * 64, j0 + x * kBoxKeys, bk, policy);
                                ptx::tma_load_3d_addr_hint(at + S::kKBytes, &tmap_v, &full[st], cb * 64, j0 + x * kBoxKeys, bk, policy);
                            }
                        }
                    }
                }
                if constexpr (kEight) {
                    const uint32_t sc = dst + 2 * S::kKBytes;
                    const int64_t row0 = (int64_t)bk * a.Smax + j0;
#pragma unroll
                    for (int i = 0; i < kTileKeys / 32; ++i) {
                        const int r = i * 32 + lane;
                        if (r < rows) {
                            copy4(sc + r * 4, k_scale + row0 + r);
                            copy4(sc + (kTileKeys + r) * 4, v_scale + row0 + r);
                        }
                    }
                    copies_arrive(&full[st]);
                }
            }
            kv_advance<kTileKeys>(a, cur, p.tiles);
        }
        if (failed) {
            if (lane == 0) atomicExch(a.status, 1);
            // copies in flight land before the ring goes away
            for (int i = n > S::kStages ? n - S::kStages : 0; i < n; ++i) ptx::warp_wait_relaxed(&full[i % S::kStages], (i / S::kStages) & 1);
        }
        return;
    }

    // ---------------------------------------------------------------------------- consumers
    const int g = lane >> 2, c = lane & 3;
    const int RG = a.RG, KG = kKvWarps / RG, rg = warp & (RG - 1), kg = warp / RG;
    const int warp_keys = 16 * RG;  // of a tile
    KvState<DW> st;
    int n = 0;

    auto put_ml = [&](float* ml) {
#pragma unroll
        for (int r = 0; r < 2; ++r) { ml[8 * r + g] = st.m[r]; ml[16 + 8 * r + g] = st.l[r]; }
    };
    // Hands the upper half of the key groups' states to the lower half until one is left, in the warps of key group 0.
    auto merge_cta = [&]() {
        for (int half = KG >> 1; half > 0; half >>= 1) {
            if (kg >= half && kg < 2 * half) {
                float* dst = merge_buf + ((kg - half) * RG + rg) * S::kFrag + lane;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) dst[(t * 4 + i) * 32] = st.o[t][i];
                if (c == 0) put_ml(dst - lane + NT * 128);
            }
            consumers_sync();
            if (kg < half) {
                const float* src = merge_buf + (kg * RG + rg) * S::kFrag + lane;
                const float* ml = src - lane + NT * 128;
                const float m2[2] = {ml[g], ml[8 + g]}, l2[2] = {ml[16 + g], ml[24 + g]};
                st.merge(m2, l2, [&](int i) { return src[i * 32]; });
            }
            consumers_sync();
        }
    };

    while (cur.u < cur.end) {
        const KvPart p = kv_part(a, cur);
        // ---- this lane's two rows: query rows p.rt * tile_rows + rg * 16 + g (+ 8) of the KV head
        const int local = rg * 16 + g;
        int64_t q_at[2], o_at[2];
        unsigned long long sees[2];
        bool row_ok[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = p.rt * a.tile_rows + local + 8 * r;
            row_ok[r] = local + 8 * r < a.tile_rows && row < a.rows;
            const int T = max(a.T, 1), h = row / T, t = row - h * T;
            q_at[r] = p.b * a.qs.b + (int64_t)(p.kvh * a.G + h) * a.qs.h + t * a.qs.s;
            o_at[r] = p.b * a.os.b + (int64_t)(p.kvh * a.G + h) * a.os.h + t * a.os.s;
            sees[r] = 0;
            if (a.T > 0 && row_ok[r]) sees[r] = a.tree ? a.tree[(int64_t)p.b * a.tree_stride + t] : (2ull << t) - 1ull;
        }
        // ---- Q as the A operand of the scores
        uint32_t qf[KS][4];
        float row_mul[2];
        const uint16_t* q16 = static_cast<const uint16_t*>(a.q);
        if constexpr (!kEight) {
            row_mul[0] = row_mul[1] = a.scale_log2;
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = s * 16 + (i >> 1) * 8 + 2 * c;
                    qf[s][i] = row_ok[i & 1] && d < a.D ? *reinterpret_cast<const uint32_t*>(q16 + q_at[i & 1] + d) : 0u;
                }
        } else {
            // The contraction may run through the head in any order: step s of lane c takes elements c DW/4 + 4 s .. + 3, which is
            // how the codes lie in their 16-byte pieces.  Each row is scaled by a power of two to where fp16 keeps bf16's 8 bits
            // exactly over 2^28 below the row's largest magnitude.
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float x[DW / 4];
                float big = 0.f;
#pragma unroll
                for (int i = 0; i < DW / 4; i += 8) {
                    const int d = c * (DW / 4) + i;
                    uint4 raw = make_uint4(0, 0, 0, 0);
                    if (row_ok[r] && d < a.D) raw = *reinterpret_cast<const uint4*>(q16 + q_at[r] + d);
                    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (a.q_f16) {
                            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[k]));
                            x[i + 2 * k] = t.x;
                            x[i + 2 * k + 1] = t.y;
                        } else {
                            x[i + 2 * k] = __uint_as_float(w[k] << 16);
                            x[i + 2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
                        }
                        big = fmaxf(big, fmaxf(fabsf(x[i + 2 * k]), fabsf(x[i + 2 * k + 1])));
                    }
                }
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                // exponent e of the largest: it goes to [2^14, 2^15); none for rows of zeros or with infinities
                const int e = (int)(__float_as_uint(big) >> 23) - 127;
                const int up = big == 0.f || e == 128 ? 0 : min(max(14 - e, -110), 110);
                const float f = __int_as_float((127 + up) << 23);
                row_mul[r] = a.scale_log2 * __int_as_float((127 - up) << 23);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    qf[s][r] = pack16<true>(x[4 * s] * f, x[4 * s + 1] * f);
                    qf[s][2 + r] = pack16<true>(x[4 * s + 2] * f, x[4 * s + 3] * f);
                }
            }
        }

        st.clear();
        float unit = 1.17549435e-38f;  // 8-bit: power of two that P is divided by, at least the largest scale of V so far
        for (int t = 0; t < p.tiles; ++t, ++n) {
            const int stage = n % S::kStages;
            if (!failed && !ptx::warp_wait(&full[stage], (n / S::kStages) & 1)) failed = true;
            const int j_warp = (p.first + t) * kTileKeys + kg * warp_keys;
            const uint32_t kb = ring + stage * S::kTileBytes, vb = kb + S::kKBytes;
            const uint32_t ksb = kb + 2 * S::kKBytes, vsb = ksb + kTileKeys * 4;
            const bool cut = (p.first + t + 1) * kTileKeys > p.past;  // keys beyond the past: not everyone sees them
#pragma unroll 1
            for (int blk = 0; blk < RG; ++blk) {
                const int j0 = j_warp + blk * 16;
                if (j0 >= p.rows || failed) break;
                const int key0 = kg * warp_keys + blk * 16;  // within the tile
                // ---- scores of 16 rows x 16 keys: s[u] are keys j0 + 8 u + 2 c + {0, 1}
                float s[2][4], s2[2][4];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[u][i] = s2[u][i] = 0.f;
                if constexpr (!kEight) {
                    const int row = key0 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                    for (int k = 0; k < KS; ++k) {
                        uint32_t b[4];
                        const int piece = (k & 3) * 2 + ((lane >> 3) & 1);
                        ldsm4(kb + (k >> 2) * (kTileKeys * 128) + row * 128 + ((piece ^ (row & 7)) << 4), b);
                        mma_16816<kF16>((k & 1) ? s2[0] : s[0], qf[k], b[0], b[1]);
                        mma_16816<kF16>((k & 1) ? s2[1] : s[1], qf[k], b[2], b[3]);
                    }
                } else {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row = key0 + u * 8 + g;
#pragma unroll
                        for (int h = 0; h < KS / 4; ++h) {
                            uint32_t w[4];
                            const int piece = DW == 128 ? (2 * c + h) ^ (row & 7) : c ^ ((row >> 1) & 3);
                            lds4(kb + row * DW + (piece << 4), w);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t f = flip_codes<kE4m3>(w[i]);
                                mma_16816<true>((i & 1) ? s2[u] : s[u], qf[h * 4 + i], codes_to_half2<kE4m3, false>(f), codes_to_half2<kE4m3, true>(f));
                            }
                        }
                    }
                }
                float2 vs[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float2 ks = make_float2(1.f, 1.f);
                    if constexpr (kEight) {
                        ks = lds_f2(ksb + (key0 + 8 * u + 2 * c) * 4);
                        vs[u] = lds_f2(vsb + (key0 + 8 * u + 2 * c) * 4);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        s[u][i] += s2[u][i];
                        if constexpr (kEight) s[u][i] *= (i & 1) ? ks.y : ks.x;
                        s[u][i] *= row_mul[i >> 1];
                    }
                }
                uint32_t there = 0xffffffffu;  // cut: bit 4 u + i, whether the row of s[u][i] sees its key
                if (cut) {
                    there = 0;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = j0 + 8 * u + 2 * c + (i & 1);
                            const bool ok = j < p.past || (j < p.rows && ((sees[i >> 1] >> (j - p.past)) & 1ull));
                            there |= (uint32_t)ok << (4 * u + i);
                            if (!ok) s[u][i] = -INFINITY;
                        }
                }
                // ---- online softmax; p reaches 2^14, where fp16 has the most room below it
                float alpha[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float mx = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const float m_new = fmaxf(st.m[r], mx);
                    const float ref = m_new == -INFINITY ? 0.f : m_new;
                    alpha[r] = ex2(st.m[r] - ref);
                    st.m[r] = m_new;
                    const float ref14 = ref - 14.f;
                    float sum = 0.f;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            s[u][2 * r + i] = ex2(s[u][2 * r + i] - ref14);
                            sum += s[u][2 * r + i];
                        }
                    st.l[r] = fmaf(st.l[r], alpha[r], sum);
                }
                if constexpr (kEight) {
                    float big = 0.f;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int j = j0 + 8 * u + 2 * c;
                        if (!cut || j < p.rows) big = fmaxf(big, vs[u].x);
                        if (!cut || j + 1 < p.rows) big = fmaxf(big, vs[u].y);
                    }
                    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                    if (big > unit) {  // the same in all lanes
                        const float next = __uint_as_float(min((__float_as_uint(big) + 0x007fffffu) & 0x7f800000u, 0x7e800000u));
                        const float f = unit / next;
                        alpha[0] *= f;
                        alpha[1] *= f;
                        unit = next;
                    }
                    const float inv = 1.f / unit;
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float w = s[u][i] * (((i & 1) ? vs[u].y : vs[u].x) * inv);
                            s[u][i] = !cut || (there >> (4 * u + i) & 1u) ? w : 0.f;
                        }
                }
                if (__any_sync(0xffffffffu, alpha[0] != 1.f || alpha[1] != 1.f)) {
#pragma unroll
                    for (int t8 = 0; t8 < NT; ++t8) {
                        st.o[t8][0] *= alpha[0]; st.o[t8][1] *= alpha[0];
                        st.o[t8][2] *= alpha[1]; st.o[t8][3] *= alpha[1];
                    }
                }
                // ---- O += P V, P as the A operand straight from the scores' registers
                const uint32_t pf[4] = {pack16<kF16>(s[0][0], s[0][1]), pack16<kF16>(s[0][2], s[0][3]),
                                        pack16<kF16>(s[1][0], s[1][1]), pack16<kF16>(s[1][2], s[1][3])};
                if constexpr (!kEight) {
                    const int row = key0 + (lane & 7) + (((lane >> 3) & 1) << 3);
                    // A row past the sequence's end holds whatever the cache holds there: it must not reach the MMA.  Nor must a NaN or
                    // infinity of a row that only some of the tokens see (0 x NaN is NaN): such rows are added one by one below.
                    uint32_t keep[2] = {0xffffffffu, 0xffffffffu}, odd = 0;
                    if (cut && j0 + 16 > p.past) {
                        odd = odd_rows<DW, kF16>(vb, key0, p.rows - j0, lane);
                        if (odd != 0 || j0 + 16 > p.rows) {
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const int j = j0 + 8 * u + 2 * c;
                                const uint32_t x = odd >> (2 * (8 * u + 2 * c));
                                keep[u] = (j < p.rows && (x & 3u) == 0 ? 0xffffu : 0u) | (j + 1 < p.rows && (x & 12u) == 0 ? 0xffff0000u : 0u);
                            }
                        }
                    }
#pragma unroll
                    for (int t16 = 0; t16 < NT / 2; ++t16) {
                        uint32_t b[4];
                        const int piece = (t16 & 3) * 2 + (lane >> 4);
                        ldsm4_t(vb + (t16 >> 2) * (kTileKeys * 128) + row * 128 + ((piece ^ (row & 7)) << 4), b);
                        mma_16816<kF16>(st.o[2 * t16], pf, b[0] & keep[0], b[1] & keep[1]);
                        mma_16816<kF16>(st.o[2 * t16 + 1], pf, b[2] & keep[0], b[3] & keep[1]);
                    }
                    if (odd != 0) {
#pragma unroll 1
                        for (int k = 0; k < 16; ++k) {
                            if ((odd >> (2 * k) & 3u) == 0) continue;
                            const int from = (lane & ~3) + ((k & 7) >> 1), bit = (k >> 3) * 4 + (k & 1);
                            const float p0 = __shfl_sync(0xffffffffu, k & 8 ? (k & 1 ? s[1][1] : s[1][0]) : (k & 1 ? s[0][1] : s[0][0]), from);
                            const float p1 = __shfl_sync(0xffffffffu, k & 8 ? (k & 1 ? s[1][3] : s[1][2]) : (k & 1 ? s[0][3] : s[0][2]), from);
                            const uint32_t seen = __shfl_sync(0xffffffffu, there, from) >> bit;
                            const int kr = key0 + k;
#pragma unroll
                            for (int t8 = 0; t8 < NT; ++t8) {
                                uint32_t v;
                                asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(vb + (t8 >> 3) * (kTileKeys * 128) + kr * 128 + (((t8 & 7) ^ (kr & 7)) << 4) + c * 4) : "memory");
                                const float2 x = kF16 ? __half22float2(*reinterpret_cast<const __half2*>(&v)) : make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
                                if (seen & 1u) { st.o[t8][0] = fmaf(p0, x.x, st.o[t8][0]); st.o[t8][1] = fmaf(p0, x.y, st.o[t8][1]); }
                                if (seen & 4u) { st.o[t8][2] = fmaf(p1, x.x, st.o[t8][2]); st.o[t8][3] = fmaf(p1, x.y, st.o[t8][3]); }
                            }
                        }
                    }
                } else {
                    // rows 2c, 2c+1, 2c+8, 2c+9; lane g has DW / 8 elements of each, one for every column tile
                    uint32_t w[4][NT / 4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int row = key0 + 2 * c + (i & 1) + (i >> 1) * 8;
                        if constexpr (DW == 128) {
                            uint32_t t4[4];
                            lds4(vb + row * 128 + ((g ^ (row & 7)) << 4), t4);
#pragma unroll
                            for (int k = 0; k < 4; ++k) w[i][k] = flip_codes<kE4m3>(t4[k]);
                        } else {
                            uint32_t x, y;
                            lds2(vb + row * 64 + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8, x, y);
                            w[i][0] = flip_codes<kE4m3>(x);
                            w[i][1] = flip_codes<kE4m3>(y);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < NT / 4; ++k)
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi) {
                            const uint32_t ab = __byte_perm(w[0][k], w[1][k], hi ? 0x7362 : 0x5140);
                            const uint32_t cd = __byte_perm(w[2][k], w[3][k], hi ? 0x7362 : 0x5140);
                            auto finite = [](uint32_t x) { return kE4m3 ? e4m3_finite(x) : x; };
                            mma_16816<true>(st.o[4 * k + 2 * hi], pf, finite(codes_to_half2<kE4m3, false>(ab)), finite(codes_to_half2<kE4m3, false>(cd)));
                            mma_16816<true>(st.o[4 * k + 2 * hi + 1], pf, finite(codes_to_half2<kE4m3, true>(ab)), finite(codes_to_half2<kE4m3, true>(cd)));
                        }
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&empty[stage]);
        }

        // ---- the CTA's part is done: merge its key groups
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            st.l[r] += __shfl_xor_sync(0xffffffffu, st.l[r], 1);
            st.l[r] += __shfl_xor_sync(0xffffffffu, st.l[r], 2);
        }
        if constexpr (kEight) {
            const float f = unit;
#pragma unroll
            for (int t8 = 0; t8 < NT; ++t8)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[t8][i] *= f;
        }
        merge_cta();

        bool write = true;
        if (p.tiles < p.of) {
            // ---- other CTAs have parts of it: leave this one in the workspace, merge all of them if it is the last to arrive
            const int cta0 = shares.of(p.start), ctas = shares.of(p.start + p.of - 1) - cta0 + 1;
            auto slot = [&](int cta) {  // an item that covers a CTA's first tile has its first slot
                const int which = p.start > shares.first(cta) ? 1 : 0;
                return a.parts + ((size_t)(cta * 2 + which) * RG + rg) * S::kFrag + lane;
            };
            if (kg == 0) {
                float* dst = slot(blockIdx.x);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (row_ok[i >> 1]) {
#pragma unroll
                        for (int t8 = 0; t8 < NT; ++t8) dst[(t8 * 4 + i) * 32] = st.o[t8][i];
                    }
                if (c == 0) put_ml(dst - lane + NT * 128);
            }
            consumers_sync();  // the warps' stores happen before the arrival
            if (threadIdx.x == 0) {
                unsigned int before;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.counters + p.item) : "memory");
                arrived_all = before;
                if (before + 1 == (unsigned)ctas) a.counters[p.item] = 0;  // as the next call expects it
            }
            consumers_sync();
            write = arrived_all + 1 == (unsigned)ctas;
            if (write) {  // the same for all warps
                st.clear();
                for (int i = kg; i < ctas; i += KG) {
                    const float* src = slot(cta0 + i);
                    const float* ml = src - lane + NT * 128;
                    const float m2[2] = {__ldcg(ml + g), __ldcg(ml + 8 + g)}, l2[2] = {__ldcg(ml + 16 + g), __ldcg(ml + 24 + g)};
                    float part[NT * 4];
#pragma unroll
                    for (int k = 0; k < NT * 4; ++k) part[k] = row_ok[(k >> 1) & 1] ? __ldcg(src + k * 32) : 0.f;
                    st.merge(m2, l2, [&](int k) { return part[k]; });
                }
                merge_cta();
            }
        }
        if (write && kg == 0 && !failed) {
            uint16_t* out = static_cast<uint16_t*>(a.out);
            const bool f16 = kEight ? a.q_f16 : kF16;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                if (!row_ok[r]) continue;
                const float inv = st.l[r] == 0.f ? 0.f : 1.f / st.l[r];  // no key seen: zeros
                auto pair = [&](float x, float y) { return f16 ? pack16<true>(x * inv, y * inv) : pack16<false>(x * inv, y * inv); };
                if constexpr (!kEight) {
#pragma unroll
                    for (int t8 = 0; t8 < NT; ++t8)
                        if (t8 * 8 < a.D) *reinterpret_cast<uint32_t*>(out + o_at[r] + t8 * 8 + 2 * c) = pair(st.o[t8][2 * r], st.o[t8][2 * r + 1]);
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {  // column 2c + e of every column tile: consecutive elements
                        const int d0 = (2 * c + e) * NT;
#pragma unroll
                        for (int t8 = 0; t8 < NT; t8 += 8)
                            if (d0 + t8 < a.D)
                                *reinterpret_cast<uint4*>(out + o_at[r] + d0 + t8) =
                                    make_uint4(pair(st.o[t8][2 * r + e], st.o[t8 + 1][2 * r + e]), pair(st.o[t8 + 2][2 * r + e], st.o[t8 + 3][2 * r + e]),
                                               pair(st.o[t8 + 4][2 * r + e], st.o[t8 + 5][2 * r + e]), pair(st.o[t8 + 6][2 * r + e], st.o[t8 + 7][2 * r + e]));
                    }
                }
            }
        }
        kv_advance<kTileKeys>(a, cur, p.tiles);
    }
    if (failed) {
        if (lane == 0) atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies in flight land before the ring goes away
    }
}

template <int DW, int FMT>
int launch_attn_kv(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {
    using S = KvShape<DW, FMT>;
    CUtensorMap tk, tv;
    const uint64_t es = S::kEight ? 1 : 2;
    const uint32_t box[3] = {S::kEight ? (uint32_t)DW : 64u, (uint32_t)kBoxKeys, 1};
    // rows of D <= DW elements: the TMA unit fills the columns up to DW with zeros
    const uint64_t dims[3] = {(uint64_t)cache.D, (uint64_t)cache.Smax, (uint64_t)cache.B * cache.Hkv};
    const uint64_t strides[2] = {(uint64_t)cache.D * es, (uint64_t)cache.Smax * cache.D * es};
    const auto encode = !S::kEight ? encode_tmap_bf16_sw128 : DW == 128 ? encode_tmap_u8_sw128 : encode_tmap_u8_sw64;
    if (!encode(&tk, cache.k, 3, dims, strides, box) || !encode(&tv, cache.v, 3, dims, strides, box)) return FORGE_ERR_CUDA;
    auto kernel = attn_kv_kernel<DW, FMT>;
    FORGE_SET_SMEM_ONCE(kernel, S::kSmem);
    FORGE_CUDA_TRY(launch_pdl(kernel, dim3(ctas), dim3(kKvThreads), S::kSmem, s, tk, tv, cache.k_scale, cache.v_scale, a));
    return finish_launch(1);
}

}  // namespace

}  // namespace forge

#include "attn_kv_narrow.cuh"
#include "attn_kv_rows.cuh"

namespace forge {

// One per format, each in a file of its own (they compile side by side).
template <int FMT>
int run_attn_kv(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s);
#define FORGE_ATTN_KV_FORMAT(fmt)                                                                         \
    template <>                                                                                           \
    int run_attn_kv<fmt>(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {    \
        if (a.rows <= kNarrowRows) return cache.D <= 64 ? launch_attn_kv_narrow<64, fmt>(cache, a, ctas, s) : launch_attn_kv_narrow<128, fmt>(cache, a, ctas, s); \
        if (a.rows > kMidRows) return cache.D <= 64 ? launch_attn_kv_rows<64, fmt>(cache, a, ctas, s) : launch_attn_kv_rows<128, fmt>(cache, a, ctas, s); \
        return cache.D <= 64 ? launch_attn_kv<64, fmt>(cache, a, ctas, s) : launch_attn_kv<128, fmt>(cache, a, ctas, s); \
    }

}  // namespace forge
