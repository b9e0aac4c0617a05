// Attention over a KV cache for up to 8 query rows per (sequence, KV head): the decode step, and short drafts of few heads.
// Included by attn_kv.cuh.
//
// Keys are the rows of both matrix products' 16-row operands, so none of the instructions' work goes to rows that do not exist:
//     S^T(16 keys x 8 rows) = K(16 x 16 dims) Q^T,    O^T(16 dims x 8 rows) += V^T(16 x 16 keys) P^T,
// with P^T brought from the first product's layout to the second's by two 8 x 8 transposes.  Eight warps per SM stream
// blocks (32 keys of 8-bit rows, 16 of 16-bit ones) through rings of their own, filled by TMA as soon as the fragments of a block are in
// registers.  A CTA's share of the call's blocks is cut into eight runs, one per warp, and no warp waits for another until all have
// finished theirs: only then, once per CTA, are the warps' results merged (through the rings, which are free by then).  The running
// reference of a row is raised only where a score exceeds it by 2^8, so that an ordinary block needs no exchange between
// lanes but a vote (8-bit rows: two, the other on the unit of P).
//
// What bounds it: the copies' latency times the 128 KB of them that an SM has in flight while it streams, and before and after that some 5 us of
// dependent steps (lengths, shares and queries; the warps' merge; the CTAs').  int8 rows, heads of 128: 16 x 32/8 x 1024 .. 4096 rows (87 MB)
// 24.8 us, 1 x 32/8 x 32,768 e4m3 rows (69 MB) 23.2; 12/12 heads of 64, 40 x up to 1000 rows (34 MB) 19.7; bf16 rows, the first of these (168 MB) 32.0.
// Over a cache in pages (PAGED) the same within 5 %, and 0.5 us more for a small call: the table is one more dependent read at the start, and none after.
// Twelve warps with smaller rings took 31.9 us for the first when eight took 27.3; a warp that only copies would leave the others 168 registers of the 246 they use.
#pragma once

namespace forge {
namespace {

// What the instructions have room for.  With few rows this kernel is the faster one: 16 sequences of 32/8 heads of 128, 8 rows (4 heads x 2 tokens), 4000
// cached rows: int8 31.7 us, on the other kernel 94; bf16 47.9 and 52.0, 1000 bf16 rows 14.1 and 18.8.
constexpr int kNarrowRows = 8;
constexpr int kNarrowWarps = 8;
constexpr int kNarrowThreads = kNarrowWarps * 32;
// Blocks that joining the parts of several CTAs is worth.  int8 rows of 128, 32/8 heads: 16 x 1000 rows take 16.8 us in even shares and 12.6
// as whole items (5 blocks more than the share), 8 x 1000 rows 13.3 and 12.0 (19 more), 2 x 1000 rows 8.6 and 11.7 (25 more).
constexpr int kNarrowMerge = 20;
// The scales of a block of 32 keys, copied from the 16-byte boundary at or before the first: up to 3 others come first.
constexpr int kScaleKeys = 36, kScaleBox = 256;

template <int DW, int FMT>
struct NarrowShape {
    static constexpr bool kEight = FMT == FORGE_KV_INT8 || FMT == FORGE_KV_E4M3;
    static constexpr int kKeys = kEight ? 32 : 16;                 // of a block
    static constexpr int kKBytes = kKeys * DW * (kEight ? 1 : 2);
    static constexpr int kStageBytes = 2 * kKBytes;
    static constexpr int kStages = 16384 / kStageBytes;            // 2 for DW = 128, 4 for 64
    static constexpr int kRingBytes = kStages * kStageBytes;
    static constexpr int kScaleBytes = kEight ? kStages * 2 * kScaleBox : 0;
    static constexpr int kFrag = (DW / 4 + 1) * 32;                // floats of a warp's O^T, then m and l of its 8 rows
    static constexpr int kSmem = 1024 + kNarrowWarps * (kRingBytes + kScaleBytes + kFrag * 4);
    static_assert(kSmem <= 232448 - 1024 && kFrag * 4 <= kRingBytes, "shared memory");
};

__device__ __forceinline__ void tma_load_1d(uint32_t smem_dst, const void* tmap, uint64_t* bar, int x) {
    asm volatile("cp.async.bulk.tensor.1d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3}], [%2];"
                 ::"r"(smem_dst), "l"(reinterpret_cast<uint64_t>(tmap)), "r"(ptx::smem_u32(bar)), "r"(x)
                 : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}

// int8 codes as fp16: x + 1152 (the exponent of 1024, and the byte with its top bit flipped), two at a time; sub_1152 takes the offset away before the
// products, in whose fp32 sums 1152 times the sum of a query would leave the scores 8 bits less (16 x 32/8 x 1024 .. 4096 rows 24.1 us with it in the sums, 24.3).
__device__ __forceinline__ uint32_t even_bytes(uint32_t w) { return (w & 0x00ff00ffu) ^ 0x64806480u; }
// A word of K: its four codes as two pairs (int8: bytes 0, 2 and 1, 3).
template <bool E4M3>
__device__ __forceinline__ void key_codes(uint32_t w, uint32_t& x, uint32_t& y) {
    if constexpr (E4M3) {
        x = e4m3_pair(w);
        y = e4m3_pair(w >> 16);
    } else {
        x = sub_1152(even_bytes(w));
        y = sub_1152(even_bytes(w >> 8));
    }
}
// Words of two rows of V: the codes of elements 0, 1 (hi: 2, 3), those of the two rows side by side.
template <bool E4M3>
__device__ __forceinline__ void value_codes(uint32_t a, uint32_t b, int hi, uint32_t& x, uint32_t& y) {
    if constexpr (E4M3) {
        const uint32_t t = __byte_perm(a, b, hi ? 0x7362 : 0x5140);
        x = e4m3_finite(e4m3_pair(t));
        y = e4m3_finite(e4m3_pair(t >> 16));
    } else {
        const uint32_t t = __byte_perm(a, b, hi ? 0x7632 : 0x5410);
        x = sub_1152(even_bytes(t));
        y = sub_1152(even_bytes(t >> 8));
    }
}

// The state of up to 8 rows: this lane holds of rows 2c, 2c + 1 the running reference, its share of the sum (the keys with index g of each 8)
// and of O^T the column tile's dims (see the fragments below).
template <int DW>
struct NarrowState {
    float m[2], l[2], o[DW / 16][4];
    __device__ __forceinline__ void clear() {
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
#pragma unroll
        for (int t = 0; t < DW / 16; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[t][i] = 0.f;
    }
};

template <int KEYS>
using NarrowSchedule = KvSchedule<KEYS, kNarrowWarps, kNarrowMerge>;
// A warp's run of blocks.
struct NarrowWalk {
    int u, end;                          // blocks of the call
    int b, kvh, tile, tiles, past;       // the next one is block `tile` of `tiles` of (b, kvh)
    template <int KEYS>
    __device__ __forceinline__ void step(const KvAttnArgs& a, const NarrowSchedule<KEYS>& sched, int n) {
        u += n;
        tile += n;
        if (tile == tiles && u < end) {
            tile = 0;
            if (++kvh == a.Hkv) {
                kvh = 0;
                ++b;
                past = sched.past_of(a, b);
                tiles = kv_tiles<KEYS>(a, past);
            }
        }
    }
};

template <int DW, int FMT, bool PAGED>
__global__ void __launch_bounds__(kNarrowThreads, 1)
attn_kv_narrow_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const __grid_constant__ CUtensorMap tmap_ks, const __grid_constant__ CUtensorMap tmap_vs, const KvAttnArgs a) {
    using S = NarrowShape<DW, FMT>;
    constexpr bool kEight = S::kEight, kE4m3 = FMT == FORGE_KV_E4M3;
    constexpr bool kF16 = FMT != FORGE_KV_BF16;  // operands of the products
    constexpr int KEYS = S::kKeys;
    constexpr int KG = KEYS / 16;                // groups of 16 keys in a block
    constexpr int KS = DW / 16;                  // 16-wide steps over the head: of the scores' contraction, and of O^T's rows
    // 16-bit rows: p reaches 2^14, 2^8 above what the reference m stands for.  8-bit rows: m is a whole number, p is 2^(x - m - 8), at most 1.
    constexpr float kTop = kEight ? 0.f : 14.f, kLift = kEight ? -8.f : 6.f;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    __shared__ uint64_t full_all[kNarrowWarps][S::kStages];
    // What a warp leaves of an item that it did not have all of: where it lies, how many blocks and which rows of the cache; 0 blocks: nothing.
    struct Left { int start, blocks, b, kvh; };
    __shared__ Left tails[kNarrowWarps];                       // ... whose run ends in it (the rest, if any, is the next warp's)
    __shared__ Left cuts[2];                                   // what the CTA has of the items at the ends of its share
    __shared__ int cut_last[2];                                // CTAs with parts of that item, if this one was the last to arrive
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, c = lane & 3;
    const uint32_t base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* base_ptr = smem_raw + (base - ptx::smem_u32(smem_raw));
    const uint32_t ring = base + warp * S::kRingBytes;
    const uint32_t scales = base + kNarrowWarps * S::kRingBytes + warp * S::kScaleBytes;
    float* heads = reinterpret_cast<float*>(base_ptr + kNarrowWarps * (S::kRingBytes + S::kScaleBytes));  // [warp]: what it has of an item that ends within its run
    uint64_t* full = full_all[warp];
    if (lane == 0) {
        for (int i = 0; i < S::kStages; ++i) ptx::mbar_init(&full[i], 1);
        ptx::fence_mbar_init();
        tails[warp].blocks = 0;
        if (warp < 2) cuts[warp].blocks = 0;
        if (warp == 0) {
            ptx::prefetch_tmap(&tmap_k);
            ptx::prefetch_tmap(&tmap_v);
            if (kEight) {
                ptx::prefetch_tmap(&tmap_ks);
                ptx::prefetch_tmap(&tmap_vs);
            }
        }
    }
    __syncwarp();
    pdl_launch_dependents();
    pdl_wait();

    const NarrowSchedule<KEYS> sched(a, lane);
    if ((int)blockIdx.x >= sched.W) return;
    const KvShares shares(sched.N, sched.W);
    int u0 = shares.first(blockIdx.x), u1 = shares.first(blockIdx.x + 1);
    if (sched.whole) u0 = sched.item_at(a, blockIdx.x, lane, &u1);
    const KvShares runs(u1 - u0, kNarrowWarps);
    NarrowWalk cur;
    cur.u = u0 + runs.first(warp);
    cur.end = u0 + runs.first(warp + 1);
    if (cur.u < cur.end) {
        KvCursor at;
        sched.at(a, cur.u, at, lane);
        cur.b = at.b;
        cur.past = at.past;
        cur.tiles = at.tiles;
        cur.kvh = (cur.u - at.base) / at.tiles;
        cur.tile = cur.u - at.base - cur.kvh * at.tiles;
    }
    bool failed = false;

    // ---- Q's row g of an item, as loaded: 16-bit rows for the steps of the contraction in turn, 8-bit ones as the codes lie
    uint32_t q_raw[KS * 2];
    auto row_at = [&](int b, int kvh, int row, const Strides& s, int* t) {
        const int T = max(a.T, 1), h = row / T;
        *t = row - h * T;
        return b * s.b + (int64_t)(kvh * a.G + h) * s.h + *t * s.s;
    };
    auto load_q = [&](int b, int kvh) {
        int t;
        const uint16_t* src = static_cast<const uint16_t*>(a.q) + row_at(b, kvh, g, a.qs, &t);
        const bool ok = g < a.rows;
#pragma unroll
        for (int i = 0; i < KS * 2; i += kEight ? 4 : 1) {
            if constexpr (kEight) {
                const int d = c * (DW / 4) + 2 * i;
                uint4 raw = make_uint4(0, 0, 0, 0);
                if (ok && d < a.D) raw = *reinterpret_cast<const uint4*>(src + d);
                q_raw[i] = raw.x; q_raw[i + 1] = raw.y; q_raw[i + 2] = raw.z; q_raw[i + 3] = raw.w;
            } else {
                const int d = i * 8 + 2 * c;
                q_raw[i] = ok && d < a.D ? *reinterpret_cast<const uint32_t*>(src + d) : 0u;
            }
        }
    };
    if (cur.u < cur.end) load_q(cur.b, cur.kvh);

    // ---- the warp's copies run ahead of its products, across the ends of sequences
    NarrowWalk ahead = cur;
    int issued = 0;
    // rows that several parts of a KV head's query heads read stay in L2 for the next one
    const uint64_t policy = PAGED && a.part_mul ? ptx::l2_policy_evict_normal() : ptx::l2_policy_evict_first();
    // PAGED: 32 entries of the table, one in each lane, those of the item's pages from entries0 on; and the ones that come after them in the run, asked
    // for when the first of these is used: behind the copies in flight they are long in coming.
    int entries = -1, entries0 = 0, entries_then = -1;
    auto ask_entries = [&]() {
        int b = ahead.b, from = entries0 + 32;
        if ((int64_t)from << a.page_shift >= kv_rows(a, ahead.past)) {  // the item after this one
            from = 0;
            b += ahead.kvh + 1 == a.Hkv;
        }
        entries_then = b < a.B ? page_entry(a, b, from + lane) : -1;
    };
    const int sub = PAGED ? min(1 << a.page_shift, KEYS) : KEYS;  // rows of a copy
    if constexpr (PAGED) {
        if (cur.u < cur.end) {
            entries0 = (cur.tile * KEYS) >> a.page_shift;
            entries = page_entry(a, cur.b, entries0 + lane);
            ask_entries();
        }
    }
    auto issue_paged = [&]() {
        if (ahead.u >= ahead.end) return;
        const int j0 = ahead.tile * KEYS, rows = kv_rows(a, ahead.past), st = issued % S::kStages;
        const int page = j0 >> a.page_shift;
        const bool item = issued > 0 && ahead.tile == 0;
        if (item || page >= entries0 + 32) {
            entries = entries_then;
            entries0 = item ? 0 : entries0 + 32;
            ask_entries();
        }
        const uint32_t dst = ring + st * S::kStageBytes;
        if (j0 >= rows) {  // a sequence without rows
            if (lane == 0) ptx::mbar_arrive(&full[st]);
        } else {
            if (lane == 0) ptx::mbar_expect_tx(&full[st], S::kStageBytes + (kEight ? 2 * KEYS * 4 : 0));
#pragma unroll
            for (int i = 0; i < KG; ++i) {  // KG copies of 16 rows, or one of all
                if (i * sub >= KEYS) break;
                const int entry = __shfl_sync(0xffffffffu, entries, (page + i - entries0) & 31);
                const int box = j0 + i * sub < rows ? page_box(a, entry, ahead.kvh) : -1, y = (j0 + i * sub) & ((1 << a.page_shift) - 1);
                if (lane != 0) continue;
                if constexpr (kEight) {
                    ptx::tma_load_2d_addr(scales + st * (2 * kScaleBox) + i * 128, &tmap_ks, &full[st], y, box);
                    ptx::tma_load_2d_addr(scales + st * (2 * kScaleBox) + kScaleBox + i * 128, &tmap_vs, &full[st], y, box);
                    ptx::tma_load_3d_addr_hint(dst + i * (16 * DW), &tmap_k, &full[st], 0, y, box, policy);
                    ptx::tma_load_3d_addr_hint(dst + S::kKBytes + i * (16 * DW), &tmap_v, &full[st], 0, y, box, policy);
                } else {
#pragma unroll
                    for (int cb = 0; cb < DW / 64; ++cb) {
                        ptx::tma_load_3d_addr_hint(dst + cb * (KEYS * 128), &tmap_k, &full[st], cb * 64, y, box, policy);
                        ptx::tma_load_3d_addr_hint(dst + S::kKBytes + cb * (KEYS * 128), &tmap_v, &full[st], cb * 64, y, box, policy);
                    }
                }
            }
        }
        ++issued;
        ahead.step<KEYS>(a, sched, 1);
    };
    auto issue = [&]() {
        if constexpr (PAGED) {
            issue_paged();
            return;
        }
        if (ahead.u >= ahead.end) return;
        const int j0 = ahead.tile * KEYS, bk = ahead.b * a.Hkv + ahead.kvh, rows = kv_rows(a, ahead.past) - j0;
        const int st = issued % S::kStages;
        const uint32_t dst = ring + st * S::kStageBytes;
        if (lane == 0) {
            if (rows > 0) {
                ptx::mbar_expect_tx(&full[st], S::kStageBytes + (kEight ? 2 * kScaleKeys * 4 : 0));
                if constexpr (kEight) {
                    const int x = (bk * a.Smax + j0) & ~3;
                    tma_load_1d(scales + st * (2 * kScaleBox), &tmap_ks, &full[st], x);
                    tma_load_1d(scales + st * (2 * kScaleBox) + kScaleBox, &tmap_vs, &full[st], x);
                    ptx::tma_load_3d_addr_hint(dst, &tmap_k, &full[st], 0, j0, bk, policy);
                    ptx::tma_load_3d_addr_hint(dst + S::kKBytes, &tmap_v, &full[st], 0, j0, bk, policy);
                } else {
#pragma unroll
                    for (int cb = 0; cb < DW / 64; ++cb) {
                        ptx::tma_load_3d_addr_hint(dst + cb * (KEYS * 128), &tmap_k, &full[st], cb * 64, j0, bk, policy);
                        ptx::tma_load_3d_addr_hint(dst + S::kKBytes + cb * (KEYS * 128), &tmap_v, &full[st], cb * 64, j0, bk, policy);
                    }
                }
            } else {  // a sequence without rows
                ptx::mbar_arrive(&full[st]);
            }
        }
        ++issued;
        ahead.step<KEYS>(a, sched, 1);
    };
#pragma unroll 1
    for (int i = 0; i < S::kStages; ++i) issue();

    NarrowState<DW> st;
    int n = 0;  // blocks consumed

    // A fragment of O^T in memory: [KS * 4][32 lanes], then m and l of the 8 rows.
    constexpr int kMl = (DW / 4) * 32;
    auto put_ml = [&](float* f) {
        if (g == 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r) { f[kMl + 2 * c + r] = st.m[r]; f[kMl + 8 + 2 * c + r] = st.l[r]; }
        }
    };
    auto put = [&](float* f) {
#pragma unroll
        for (int t = 0; t < KS; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) f[(t * 4 + i) * 32 + lane] = st.o[t][i];
        put_ml(f);
    };
    auto part_of = [&](int cta, int item_start) {  // an item that covers a CTA's first block has its first place
        return a.parts + (size_t)(cta * 2 + (item_start > shares.first(cta) ? 1 : 0)) * S::kFrag;
    };
    const bool out_f16 = kEight ? a.q_f16 : kF16;
    auto pack = [&](float y, float z) { return out_f16 ? pack16<true>(y, z) : pack16<false>(y, z); };
    // Registers 4 s .. 4 s + 3 of O^T (rows 2c, 2c + 1 of one dim, then of another), normalised, to the output.
    auto write4 = [&](uint16_t* out0, uint16_t* out1, int s, const float (&y)[4], float inv0, float inv1) {
        const uint32_t y0 = pack(y[0] * inv0, y[2] * inv0), y1 = pack(y[1] * inv1, y[3] * inv1);
        const bool has0 = 2 * c < a.rows && !failed, has1 = 2 * c + 1 < a.rows && !failed;
        if constexpr (kEight) {  // dims side by side
            const int d = g * (DW / 8) + 2 * s;
            if (has0 && d < a.D) *reinterpret_cast<uint32_t*>(out0 + d) = y0;
            if (has1 && d < a.D) *reinterpret_cast<uint32_t*>(out1 + d) = y1;
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int d = 16 * s + 8 * i + g;
                if (has0 && d < a.D) out0[d] = (uint16_t)(y0 >> (16 * i));
                if (has1 && d < a.D) out1[d] = (uint16_t)(y1 >> (16 * i));
            }
        }
    };
    auto rows_of_item = [&](int b, int kvh, uint16_t** out0, uint16_t** out1) {
        int t;
        *out0 = static_cast<uint16_t*>(a.out) + row_at(b, kvh, 2 * c, a.os, &t);
        *out1 = static_cast<uint16_t*>(a.out) + row_at(b, kvh, 2 * c + 1, a.os, &t);
    };
    auto inverse = [](float l) { return l == 0.f ? 0.f : 1.f / l; };  // no key seen: zeros
    while (cur.u < cur.end) {
        struct { int b, kvh, past, rows; } p = {cur.b, cur.kvh, cur.past, kv_rows(a, cur.past)};
        const int item_start = cur.u - cur.tile, item_end = item_start + cur.tiles;
        const int blocks = min(cur.tiles - cur.tile, cur.end - cur.u);
        // ---- the rows: Q^T as the B operand (row g), and what the rows 2c, 2c + 1 of the scores and outputs need
        uint32_t qf[KS][2], w[KS * 2];
#pragma unroll
        for (int i = 0; i < KS * 2; ++i) w[i] = q_raw[i];
        {  // those of the run's next item are asked for now: behind the copies in flight they would be long in coming
            NarrowWalk then = cur;
            then.step<KEYS>(a, sched, blocks);
            if (then.u < then.end) load_q(then.b, then.kvh);
        }
        float q_mul = a.scale_log2;  // of row g
        {
            if constexpr (!kEight) {
#pragma unroll
                for (int s = 0; s < KS; ++s) { qf[s][0] = w[2 * s]; qf[s][1] = w[2 * s + 1]; }
            } else {
                // Step s of lane c takes elements c DW/4 + 4 s .. + 3, as the codes lie in their 16-byte pieces; the row is scaled by a power
                // of two to where fp16 keeps bf16's 8 bits exactly over 2^28 below the row's largest magnitude.
                // the largest magnitude's bits: those of two elements side by side compare as 16-bit numbers
                uint32_t big = 0;
#pragma unroll
                for (int i = 0; i < DW / 8; ++i) big = __vmaxu2(big, w[i] & 0x7fff7fffu);
                big = max(big & 0xffffu, big >> 16);
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const float top = a.q_f16 ? __half2float(__ushort_as_half((unsigned short)big)) : __uint_as_float(big << 16);
                // the largest goes to [2^14, 2^15) (bf16's goes up to 2^127; one below 2^-96 stays smaller); rows of zeros or with infinities stay
                const int e = (int)(__float_as_uint(top) >> 23) - 127;
                const int up = top == 0.f || e == 128 ? 0 : min(max(14 - e, -113), 110);
                const float f = __int_as_float((127 + up) << 23);
                q_mul = a.scale_log2 * __int_as_float((127 - up) << 23);
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    float2 x, y;
                    if (a.q_f16) {
                        x = __half22float2(*reinterpret_cast<const __half2*>(&w[2 * s]));
                        y = __half22float2(*reinterpret_cast<const __half2*>(&w[2 * s + 1]));
                    } else {
                        x = make_float2(__uint_as_float(w[2 * s] << 16), __uint_as_float(w[2 * s] & 0xffff0000u));
                        y = make_float2(__uint_as_float(w[2 * s + 1] << 16), __uint_as_float(w[2 * s + 1] & 0xffff0000u));
                    }
                    if constexpr (kE4m3) {  // as the codes of a word come in pairs
                        qf[s][0] = pack16<true>(x.x * f, x.y * f);
                        qf[s][1] = pack16<true>(y.x * f, y.y * f);
                    } else {
                        qf[s][0] = pack16<true>(x.x * f, y.x * f);
                        qf[s][1] = pack16<true>(x.y * f, y.y * f);
                    }
                }
            }
        }
        float row_mul[2];
        unsigned long long sees[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = 2 * c + r;
            row_mul[r] = __shfl_sync(0xffffffffu, q_mul, row * 4);
            int t;
            sees[r] = 0;
            if (a.T > 0) t = row % a.T;
            if (a.T > 0 && row < a.rows) sees[r] = a.tree ? a.tree[(int64_t)p.b * a.tree_stride + t] : (2ull << t) - 1ull;
        }

        st.clear();
        float ref[2] = {-INFINITY, -INFINITY};  // reference - kLift; -infinity: none yet
        // 8-bit rows: O^T of each row is kept in units of a power of two, with which p vs goes into the products' fp16 (see kv_unit)
        float unit_inv[2] = {kv_pow2(-kUnitLow), kv_pow2(-kUnitLow)};
        for (int blk = 0; blk < blocks; ++blk, ++n) {
            const int stage = n % S::kStages;
            if (!failed && !ptx::warp_wait(&full[stage], (n / S::kStages) & 1)) failed = true;
            if (failed) continue;
            const uint32_t kb = ring + stage * S::kStageBytes, vb = kb + S::kKBytes;
            const int j0 = (cur.tile + blk) * KEYS;
            // ---- fragments: K's raw rows g, g + 8 of each group of 16; V's rows 2c, 2c + 1, 2c + 8, 2c + 9, elements by lane g
            uint32_t kr[kEight ? KG * 2 : KG * KS][kEight ? DW / 16 : 4], vr[kEight ? KG * 4 : KG * KS][kEight ? DW / 32 : 4];
            float ks[KG][2], vs[KG][2];
            if constexpr (kEight) {
#pragma unroll
                for (int i = 0; i < KG * 2; ++i) {
                    const int row = i * 8 + g;
#pragma unroll
                    for (int h = 0; h < DW / 64; ++h) {
                        uint32_t w[4];
                        const int piece = DW == 128 ? (2 * c + h) ^ (row & 7) : c ^ ((row >> 1) & 3);
                        lds4(kb + row * DW + (piece << 4), w);
#pragma unroll
                        for (int x = 0; x < 4; ++x) kr[i][h * 4 + x] = w[x];
                    }
                    const uint32_t sc = scales + stage * (2 * kScaleBox) +
                                        (PAGED ? (i >> 1) * (sub == 16 ? 128 : 64) + (row & 15) * 4
                                               : (((p.b * a.Hkv + p.kvh) * a.Smax + j0) & 3) * 4 + row * 4);
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(ks[i >> 1][i & 1]) : "r"(sc) : "memory");
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(vs[i >> 1][i & 1]) : "r"(sc + kScaleBox) : "memory");
                }
#pragma unroll
                for (int i = 0; i < KG * 4; ++i) {
                    const int row = (i >> 2) * 16 + 2 * c + (i & 1) + ((i >> 1) & 1) * 8;
                    if constexpr (DW == 128) {
                        uint32_t w[4];
                        lds4(vb + row * 128 + ((g ^ (row & 7)) << 4), w);
#pragma unroll
                        for (int x = 0; x < 4; ++x) vr[i][x] = w[x];
                    } else {
                        lds2(vb + row * 64 + (((g >> 1) ^ ((row >> 1) & 3)) << 4) + (g & 1) * 8, vr[i][0], vr[i][1]);
                    }
                }
            } else {
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    // K: (keys 0-7, dims 0-7), (keys 8-15, dims 0-7), (keys 0-7, dims 8-15), (keys 8-15, dims 8-15) of step s
                    const int krow = (lane & 7) + ((lane >> 3) & 1) * 8, kpiece = (s & 3) * 2 + (lane >> 4);
                    ldsm4(kb + (s >> 2) * (KEYS * 128) + krow * 128 + ((kpiece ^ (krow & 7)) << 4), kr[s]);
                    // V transposed: (dims 0-7, keys 0-7), (dims 8-15, keys 0-7), (dims 0-7, keys 8-15), (dims 8-15, keys 8-15)
                    const int vrow = (lane & 7) + (lane >> 4) * 8, vpiece = (s & 3) * 2 + ((lane >> 3) & 1);
                    ldsm4_t(vb + (s >> 2) * (KEYS * 128) + vrow * 128 + ((vpiece ^ (vrow & 7)) << 4), vr[s]);
                }
            }
            __syncwarp();                   // all fragment reads done before this stage is refilled ...
            ptx::fence_proxy_async_smem();  // ... by the copy engine
            issue();

            // ---- scores: x[k][i]: key j0 + 16 k + g + 8 (i >> 1), row 2c + (i & 1)
            float x[KG][4];
#pragma unroll
            for (int k = 0; k < KG; ++k) {
                float even[4] = {0.f, 0.f, 0.f, 0.f}, odd[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    uint32_t f[4];
                    if constexpr (kEight) {
                        key_codes<kE4m3>(kr[2 * k][s], f[0], f[2]);
                        key_codes<kE4m3>(kr[2 * k + 1][s], f[1], f[3]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i) f[i] = kr[s][i];
                    }
                    mma_16816<kF16>(s & 1 ? odd : even, f, qf[s][0], qf[s][1]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[k][i] = even[i] + odd[i];
                    // the factors first: each may be as far from 1 as the other makes up for
                    x[k][i] *= kEight ? ks[k][i >> 1] * row_mul[i & 1] : row_mul[i & 1];
                }
            }
            const bool cut = j0 + KEYS > p.past;  // keys beyond the past: not everyone sees them
            uint32_t there = 0xffffffffu;         // bit 4 k + i
            if (cut) {
                there = 0;
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = j0 + 16 * k + g + 8 * (i >> 1);
                        const bool ok = j < p.past || (j < p.rows && ((sees[i & 1] >> (j - p.past)) & 1ull));
                        there |= (uint32_t)ok << (4 * k + i);
                        if (!ok) x[k][i] = -INFINITY;
                        if (kEight && j >= p.rows) vs[k][i >> 1] = 0.f;
                    }
            }
            // ---- references: raised where a score passes them by 2^8 (the first of a row always does)
            float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int k = 0; k < KG; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i) mx[i & 1] = fmaxf(mx[i & 1], x[k][i]);
            const bool lift = mx[0] > ref[0] + kTop || mx[1] > ref[1] + kTop;
            if (__any_sync(0xffffffffu, lift)) {
                float alpha[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], o));
                    const float m_new = fmaxf(st.m[r], kEight ? ceilf(mx[r]) : mx[r]);
                    alpha[r] = m_new == -INFINITY ? 1.f : ex2(st.m[r] - m_new);
                    if constexpr (kEight) {
                        const float by = st.m[r] == -INFINITY ? 0.f : st.m[r] - m_new;
                        st.l[r] *= alpha[r];
                        alpha[r] = kv_lower_unit(unit_inv[r], by);
                    } else {
                        st.l[r] *= alpha[r];
                    }
                    st.m[r] = m_new;
                    ref[r] = m_new - kLift;  // -infinity stays
                }
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) st.o[s][i] *= alpha[i & 1];
            }
            // ---- probabilities, and P^T as the B operand: keys 2c, 2c + 1 (and + 8) of row g
            const float sub[2] = {ref[0] == -INFINITY ? 0.f : ref[0], ref[1] == -INFINITY ? 0.f : ref[1]};
            // P is rounded once to the products' type, and what that leaves is multiplied too (pl), so that outputs are off by their own rounding alone: fp16 ones
            // by 2.1e-4 of their size instead of 2.9e-4, bf16 ones of 8-bit rows by 1.67e-3 instead of 1.69e-3, for 1 to 3 % of the time.
            uint32_t pf[KG][2], pl[KG][2];
            float pr[KG][4];
#pragma unroll
            for (int k = 0; k < KG; ++k) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float w = ex2(x[k][i] - sub[i & 1]);
                    st.l[i & 1] += w;
                    if constexpr (kEight) {
                        w *= vs[k][i >> 1];
                        if (cut && !(there >> (4 * k + i) & 1u)) w = 0.f;
                    }
                    pr[k][i] = w;
                }
            }
            if constexpr (kEight) {
                float most[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) most[i & 1] = fmaxf(most[i & 1], fabsf(pr[k][i]));
                if (__any_sync(0xffffffffu, most[0] * unit_inv[0] > kUnitTop || most[1] * unit_inv[1] > kUnitTop)) {
                    float alpha[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
#pragma unroll
                        for (int o = 4; o < 32; o <<= 1) most[r] = fmaxf(most[r], __shfl_xor_sync(0xffffffffu, most[r], o));
                        alpha[r] = kv_raise_unit(unit_inv[r], most[r]);
                    }
#pragma unroll
                    for (int s = 0; s < KS; ++s)
#pragma unroll
                        for (int i = 0; i < 4; ++i) st.o[s][i] *= alpha[i & 1];
                }
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) pr[k][i] *= unit_inv[i & 1];
            }
#pragma unroll
            for (int k = 0; k < KG; ++k) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t p16 = kv_operand<kF16, !kEight>(pr[k][2 * u], pr[k][2 * u + 1]);
                    pf[k][u] = transpose8x8(p16);
                    pl[k][u] = transpose8x8(kv_rest<kF16, !kEight>(pr[k][2 * u], pr[k][2 * u + 1], p16));
                }
            }
            // ---- O^T += V^T P^T
            if constexpr (kEight) {
                // step s: rows g and g + 8 of the fragment are elements (DW / 8) g + 2 s and + 1; byte pairs of two keys side by side
#pragma unroll
                for (int k = 0; k < KG; ++k)
#pragma unroll
                    for (int w4 = 0; w4 < DW / 32; ++w4) {
#pragma unroll
                        for (int hi = 0; hi < 2; ++hi) {
                            uint32_t f[4];
                            value_codes<kE4m3>(vr[4 * k][w4], vr[4 * k + 1][w4], hi, f[0], f[1]);
                            value_codes<kE4m3>(vr[4 * k + 2][w4], vr[4 * k + 3][w4], hi, f[2], f[3]);
                            mma_16816<true>(st.o[2 * w4 + hi], f, pf[k][0], pf[k][1]);
                            mma_16816<true>(st.o[2 * w4 + hi], f, pl[k][0], pl[k][1]);
                        }
                    }
            } else {
                // what must not reach the product: rows past the end, and NaN or infinities of rows that only some of the tokens see
                uint32_t keep[2] = {0xffffffffu, 0xffffffffu}, odd = 0;
                if (cut) {
                    uint32_t lo = 0, hi = 0;
                    constexpr uint32_t kExp = kF16 ? 0x7c00u : 0x7f80u;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        bool b0 = false, b1 = false;
#pragma unroll
                        for (int s = 0; s < KS; ++s)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                b0 |= (vr[s][2 * u + i] & kExp) == kExp;
                                b1 |= (vr[s][2 * u + i] >> 16 & kExp) == kExp;
                            }
                        const uint32_t v0 = __ballot_sync(0xffffffffu, b0), v1 = __ballot_sync(0xffffffffu, b1);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {  // lanes with c = q: keys 8 u + 2 q and + 1
                            if (v0 & (0x11111111u << q)) lo |= 1u << (8 * u + 2 * q);
                            if (v1 & (0x11111111u << q)) hi |= 1u << (8 * u + 2 * q + 1);
                        }
                    }
                    odd = lo | hi;
                    const int have = p.rows - j0;  // keys from here on are not there
                    odd &= have >= 16 ? 0xffffu : (1u << max(have, 0)) - 1u;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int k0 = 8 * u + 2 * c;
                        keep[u] = (k0 < have && !(odd >> k0 & 1u) ? 0xffffu : 0u) | (k0 + 1 < have && !(odd >> (k0 + 1) & 1u) ? 0xffff0000u : 0u);
                    }
                }
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const uint32_t f[4] = {vr[s][0] & keep[0], vr[s][1] & keep[0], vr[s][2] & keep[1], vr[s][3] & keep[1]};
                    mma_16816<kF16>(st.o[s], f, pf[0][0], pf[0][1]);
                    mma_16816<kF16>(st.o[s], f, pl[0][0], pl[0][1]);
                }
                if (odd != 0) {  // those rows one by one, for the rows that see them; this lane has elements 16 s + g (+ 8) of O^T
#pragma unroll 1
                    for (int k = 0; k < 16; ++k) {
                        if (!(odd >> k & 1u)) continue;
                        const int p_from = (k & 7) * 4 + c;  // holds key k of rows 2c, 2c + 1
                        const float p0 = __shfl_sync(0xffffffffu, k & 8 ? pr[0][2] : pr[0][0], p_from);
                        const float p1 = __shfl_sync(0xffffffffu, k & 8 ? pr[0][3] : pr[0][1], p_from);
                        const uint32_t seen = __shfl_sync(0xffffffffu, there, p_from) >> (k & 8 ? 2 : 0);
                        const int v_from = g * 4 + ((k & 7) >> 1);  // holds element g (+ 8) of key k
#pragma unroll
                        for (int s = 0; s < KS; ++s)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                uint32_t v = __shfl_sync(0xffffffffu, k & 8 ? vr[s][2 + i] : vr[s][i], v_from);
                                v = k & 1 ? v >> 16 : v & 0xffffu;
                                const float e = kF16 ? __half2float(__ushort_as_half((unsigned short)v)) : __uint_as_float(v << 16);
                                if (seen & 1u) st.o[s][2 * i] = fmaf(p0, e, st.o[s][2 * i]);
                                if (seen & 2u) st.o[s][2 * i + 1] = fmaf(p1, e, st.o[s][2 * i + 1]);
                            }
                    }
                }
            }
        }

        // ---- the warp's blocks of this item are done
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) st.l[r] += __shfl_xor_sync(0xffffffffu, st.l[r], o);
        if constexpr (kEight) {
            const float unit[2] = {kv_unit(unit_inv[0]), kv_unit(unit_inv[1])};
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[s][i] *= unit[i & 1];
        }
        const Left left = {item_start, cur.tiles, p.b, p.kvh};
        if (blocks == cur.tiles) {  // all of it
            uint16_t *out0, *out1;
            rows_of_item(p.b, p.kvh, &out0, &out1);
            const float inv0 = inverse(st.l[0]), inv1 = inverse(st.l[1]);
#pragma unroll
            for (int s = 0; s < KS; ++s) write4(out0, out1, s, st.o[s], inv0, inv1);
        } else if (item_end < cur.end) {  // its end: warp 0 has all that the CTA has of it, the others' joins what the warps before have
            put(warp == 0 ? part_of(blockIdx.x, item_start) : heads + warp * S::kFrag);
            if (lane == 0 && warp == 0) cuts[0] = left;
        } else {  // to the end of the run: into the ring, whose copies have all been consumed
            put(reinterpret_cast<float*>(base_ptr + warp * S::kRingBytes));
            if (lane == 0) tails[warp] = left;
        }
        cur.step<KEYS>(a, sched, blocks);
    }

    // kMine registers of a fragment of O^T from kMine warp on in this lane, summed over several fragments; a few at a time, and the loads of three
    // times as many leave together (1 x 32/8 heads x 32,000 bf16 rows, 19 parts to an item: 28.5 and 26.8 us).  of(i): the i-th.
    constexpr int kMine = KS * 4 / kNarrowWarps;
    float sum[kMine], M[2], L[2];
    auto sum_over = [&](int n_of, auto of) {
        constexpr int kAtOnce = 4, kLoads = 3 * kAtOnce;
        M[0] = M[1] = -INFINITY;
        L[0] = L[1] = 0.f;
#pragma unroll
        for (int k = 0; k < kMine; ++k) sum[k] = 0.f;
#pragma unroll 1
        for (int i0 = 0; i0 < n_of; i0 += kLoads) {
            float2 m[kLoads], l[kLoads];
            float x[kLoads][kMine];
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const float* f = of(min(i0 + i, n_of - 1));
                m[i] = make_float2(-INFINITY, -INFINITY);
                l[i] = make_float2(0.f, 0.f);
#pragma unroll
                for (int k = 0; k < kMine; ++k) x[i][k] = 0.f;
                if (i0 + i < n_of) {
                    m[i] = *reinterpret_cast<const float2*>(f + kMl + 2 * c);
                    l[i] = *reinterpret_cast<const float2*>(f + kMl + 8 + 2 * c);
#pragma unroll
                    for (int k = 0; k < kMine; ++k) x[i][k] = f[(warp * kMine + k) * 32 + lane];
                }
            }
#pragma unroll
            for (int j = 0; j < kLoads; j += kAtOnce) {
                if (i0 + j >= n_of) break;
                float old[2] = {M[0], M[1]};
#pragma unroll
                for (int i = j; i < j + kAtOnce; ++i) { M[0] = fmaxf(M[0], m[i].x); M[1] = fmaxf(M[1], m[i].y); }
                const float ref0 = M[0] == -INFINITY ? 0.f : M[0], ref1 = M[1] == -INFINITY ? 0.f : M[1];
                const float a0 = ex2(old[0] - ref0), a1 = ex2(old[1] - ref1);
                L[0] *= a0;
                L[1] *= a1;
#pragma unroll
                for (int k = 0; k < kMine; ++k) sum[k] *= k & 1 ? a1 : a0;
#pragma unroll
                for (int i = j; i < j + kAtOnce; ++i) {
                    const float w0 = ex2(m[i].x - ref0), w1 = ex2(m[i].y - ref1);
                    L[0] = fmaf(w0, l[i].x, L[0]);
                    L[1] = fmaf(w1, l[i].y, L[1]);
#pragma unroll
                    for (int k = 0; k < kMine; ++k) sum[k] = fmaf(k & 1 ? w1 : w0, x[i][k], sum[k]);
                }
            }
        }
    };
    auto write_sum = [&](int b, int kvh) {  // normalised, to the output
        uint16_t *out0, *out1;
        rows_of_item(b, kvh, &out0, &out1);
        const float inv0 = inverse(L[0]), inv1 = inverse(L[1]);
        if constexpr (kMine == 4) {
            write4(out0, out1, warp, sum, inv0, inv1);
        } else {  // one dim of both rows
            static_assert(kMine == 2);
            const int s = warp >> 1, i = warp & 1, d = kEight ? g * (DW / 8) + 2 * s + i : 16 * s + 8 * i + g;
            if (d >= a.D || failed) return;
            if (2 * c < a.rows) out0[d] = (uint16_t)pack(sum[0] * inv0, 0.f);
            if (2 * c + 1 < a.rows) out1[d] = (uint16_t)pack(sum[1] * inv1, 0.f);
        }
    };
    __syncthreads();

    // ---- once per CTA: what several of its warps have of an item is merged by those whose runs end in it, each some of the fragment's
    // registers, all items of the CTA at a time
    if (tails[warp].blocks > 0) {
        const Left left = tails[warp];
        const int end = left.start + left.blocks, to = min(end, u1), w0 = runs.of(max(left.start, u0) - u0), w1 = runs.of(to - 1 - u0);
        const bool head = u0 + runs.first(w1 + 1) > to;  // the last of the warps has other items after it
        const int n_of = w1 - w0 + 1, helpers = n_of - head;
        constexpr int kNext = S::kRingBytes / 4;  // floats from a warp's ring to the next one's
        const float* const first = reinterpret_cast<const float*>(base_ptr + w0 * S::kRingBytes);
        const float* const last = head ? heads + w1 * S::kFrag : first + (n_of - 1) * kNext;
        // lane (g, c): the weights of rows 2c, 2c + 1 of warp w0 + g; from there to all lanes with this c
        const float* const ml = (g < n_of - 1 ? first + g * kNext : last) + kMl + 2 * c;
        float2 m = make_float2(-INFINITY, -INFINITY), l = make_float2(0.f, 0.f);
        if (g < n_of) {
            m = *reinterpret_cast<const float2*>(ml);
            l = *reinterpret_cast<const float2*>(ml + 8);
        }
        M[0] = m.x;
        M[1] = m.y;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
            for (int r = 0; r < 2; ++r) M[r] = fmaxf(M[r], __shfl_xor_sync(0xffffffffu, M[r], o));
        const float w0_ = ex2(m.x - (M[0] == -INFINITY ? 0.f : M[0])), w1_ = ex2(m.y - (M[1] == -INFINITY ? 0.f : M[1]));
        L[0] = w0_ * l.x;
        L[1] = w1_ * l.y;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1)
#pragma unroll
            for (int r = 0; r < 2; ++r) L[r] += __shfl_xor_sync(0xffffffffu, L[r], o);
        float wt[kNarrowWarps][2];
#pragma unroll
        for (int i = 0; i < kNarrowWarps; ++i) {  // the last one's come last
            const int from = (i < kNarrowWarps - 1 ? i : n_of - 1) * 4 + c;
            wt[i][0] = __shfl_sync(0xffffffffu, w0_, from);
            wt[i][1] = __shfl_sync(0xffffffffu, w1_, from);
        }
        const bool whole = left.start >= u0 && end <= u1;
        float* part = part_of(blockIdx.x, left.start);
        const float inv0 = inverse(L[0]), inv1 = inverse(L[1]);
        uint16_t *out0, *out1;
        rows_of_item(left.b, left.kvh, &out0, &out1);
#pragma unroll 1
        for (int s = warp - w0; s < KS; s += helpers) {
            const int at = s * 128 + lane;
            float y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = wt[kNarrowWarps - 1][k & 1] * last[at + 32 * k];
#pragma unroll
            for (int i = 0; i < kNarrowWarps - 1; ++i)
                if (i < n_of - 1) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[k] = fmaf(wt[i][k & 1], first[i * kNext + at + 32 * k], y[k]);
                }
            if (whole) {
                write4(out0, out1, s, y, inv0, inv1);
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) part[at + 32 * k] = y[k];
            }
        }
        if (!whole && warp == w0) {
            st.m[0] = M[0]; st.m[1] = M[1]; st.l[0] = L[0]; st.l[1] = L[1];
            put_ml(part);
            if (lane == 0) cuts[left.start > u0 ? 1 : 0] = left;
        }
    }
    __syncthreads();

    // ---- items that other CTAs have parts of: the CTA that arrives last merges all of them
    if (lane == 0 && warp < 2) {
        const Left left = cuts[warp];
        cut_last[warp] = 0;
        if (left.blocks > 0) {
            const int cta0 = shares.of(left.start), ctas = shares.of(left.start + left.blocks - 1) - cta0 + 1;
            unsigned int* counter = a.counters + cta0 * 2 + (left.start > shares.first(cta0) ? 1 : 0);  // that of its first part
            unsigned int before;
            asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
            if (before + 1 == (unsigned)ctas) {
                *counter = 0;  // as the next call expects it
                cut_last[warp] = ctas;
            }
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int e = 0; e < 2; ++e) {
        if (cut_last[e] == 0) continue;
        const Left left = cuts[e];
        const int cta0 = shares.of(left.start);
        sum_over(cut_last[e], [&](int i) -> const float* { return part_of(cta0 + i, left.start); });
        write_sum(left.b, left.kvh);
    }
    if (failed) {
        if (lane == 0) atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies in flight land before the ring goes away
    }
}

template <int DW, int FMT, bool PAGED>
int launch_attn_kv_narrow(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {
    using S = NarrowShape<DW, FMT>;
    CUtensorMap tk, tv;
    const uint64_t es = S::kEight ? 1 : 2;
    const uint32_t keys = PAGED && cache.Smax < S::kKeys ? cache.Smax : S::kKeys;
    const uint32_t box[3] = {S::kEight ? (uint32_t)DW : 64u, keys, 1};
    const uint64_t dims[3] = {(uint64_t)cache.D, (uint64_t)cache.Smax, (uint64_t)cache.B * cache.Hkv};
    const uint64_t strides[2] = {(uint64_t)cache.D * es, (uint64_t)cache.Smax * cache.D * es};
    const auto encode = !S::kEight ? encode_tmap_bf16_sw128 : DW == 128 ? encode_tmap_u8_sw128 : encode_tmap_u8_sw64;
    if (!encode(&tk, cache.k, 3, dims, strides, box) || !encode(&tv, cache.v, 3, dims, strides, box)) return FORGE_ERR_CUDA;
    CUtensorMap tks = {}, tvs = {};
    if (S::kEight) {
        const uint32_t sbox[2] = {PAGED ? keys : (uint32_t)kScaleKeys, 1};
        const uint64_t n[2] = {PAGED ? (uint64_t)cache.Smax : (uint64_t)cache.B * cache.Hkv * cache.Smax, (uint64_t)cache.B * cache.Hkv};
        const uint64_t row[1] = {(uint64_t)cache.Smax * 4};
        if (!encode_tmap_f32_plain(&tks, cache.k_scale, PAGED ? 2 : 1, n, PAGED ? row : nullptr, sbox) ||
            !encode_tmap_f32_plain(&tvs, cache.v_scale, PAGED ? 2 : 1, n, PAGED ? row : nullptr, sbox))
            return FORGE_ERR_CUDA;
    }
    auto kernel = attn_kv_narrow_kernel<DW, FMT, PAGED>;
    FORGE_SET_SMEM_ONCE(kernel, S::kSmem);
    FORGE_CUDA_TRY(launch_pdl(kernel, dim3(ctas), dim3(kNarrowThreads), S::kSmem, s, tk, tv, tks, tvs, a));
    return finish_launch(1);
}

}  // namespace
}  // namespace forge
