// Attention over a KV cache for more than 8 query rows per (sequence, KV head): trees of drafted tokens, and single tokens of large head
// groups.  Included by attn_kv.cuh.
//
// The rows (up to 128: several tokens of several heads that share K and V) are one tile of the tensor cores: per step of 128 keys (16-bit rows;
// a product 128 x 64 would read Q from shared memory twice as often as the tensor cores need it) or 64 (8-bit)
//     S[128 x keys] = Q K^T  and  O[128 x DW] += P V   by tcgen05.mma, with S (two steps' worth), P and O in tensor memory,
// and thread = row does the softmax in between.  Each half of a step's keys belongs to a group of softmax threads with references, sums and an O
// of its own; the two are merged when a piece ends.  Every item (sequence, KV head, row tile) is cut into pieces of C steps, with one C for the
// call, so that a CTA has one piece, if that can be had: changing the item costs as much as three steps, and a second merge
// as much as four (with the steps shared out evenly, the runs of most CTAs going over the end of an item, 4 x 32/8 x 64 tokens took
// 36 us).  The pieces of an item are merged by the CTA that finishes last, after all its pieces: loads between them would wait behind
// the copies in flight.
//   warps 0-7   softmax (two groups of 128 threads), O out      warp 8  TMA      warp 9  tcgen05.mma
//   warps 10-13 8-bit rows only: codes of K and V to fp16, from the copies' ring into operands
// 8-bit rows stay codes in the products (exact in fp16; int8 elements come in the order 0 2 1 3 of each four, in Q and O too); their scales
// multiply the scores and the probabilities.  Q comes by TMA, an item ahead: plain loads would wait behind the copies in flight.
//
// What bounds it: the chain of a step (scores, softmax of a row per thread, P into tensor memory, product with V; 1.23 us for 128 keys of 16-bit rows,
// where the tensor cores need 0.8, and 1.33 for 64 of 8-bit ones), and some 8 us around the steps: start, first copies, the output and the merge of pieces.
// 4 x 32/8 heads x 64 tokens behind 1024 .. 4096 16-bit rows take 30.3 us, 8 x 28/4 x 16 behind 600 .. 2400 int8 rows 24.0, 1 x 32/8 x 5 behind some 600 12.9.
#pragma once

namespace forge {
namespace {

// Steps that joining the pieces of an item is worth.  Whole and cut: 8 x 32/8 heads x 16 tokens over int8 rows, 400 rows of the past 17.4 and 17.1 us (3 steps
// more), 480 18.6 and 17.1 (4 more); over 16-bit rows 4 x 32/8 x 64 tokens, 640 rows 16.1 and 17.8 (3 more), 1 x 32/8 x 5, 470 rows 11.5 and 11.2 (3 more),
// 600 12.9 and 11.5 (4 more), 800 16.8 and 13.5 (6 more).
constexpr int kRowsMerge = 3;
// p reaches 2^8 above what the reference m stands for.  16-bit rows: that is 2^14.  8-bit rows: 1, and m is a whole number.
constexpr float kRowsAbove = 8.f;

template <int DW, int FMT>
struct RowsShape {
    static constexpr bool kEight = FMT == FORGE_KV_INT8 || FMT == FORGE_KV_E4M3;
    static constexpr int kStep = kEight ? 64 : 128, kHalf = kStep / 2;  // keys; of a group
    static constexpr int kConvWarps = kEight ? 4 : 0;
    static constexpr int kThreads = (10 + kConvWarps) * 32;
    static constexpr int kQChunk = 128 * 128;                        // 128 rows x 64 elements
    static constexpr int kQBytes = DW / 64 * kQChunk;
    static constexpr int kOpChunk = kStep * 128;                     // a step's keys x 64 elements
    static constexpr int kOpBytes = DW / 64 * kOpChunk;              // K, or V
    static constexpr int kRawBytes = kStep * DW;                     // 8-bit: the codes of K, or V
    static constexpr int kScaleBox = 512;                            // scales from the 16-byte boundary at or before the first
    static constexpr int kScaleKeys = kStep + 4;
    // 16-bit: rings of K and of V; K's is longer, a step's scores being asked for two steps before its product with V.
    // 8-bit: a ring of codes, of K and V together, and operand buffers, K then V.
    static constexpr int kLoadBytes = 2 * kRawBytes + 2 * kScaleBox;
    static constexpr int kLoads = kEight ? (DW == 128 ? 4 : 8) : 0;
    static constexpr int kOps = kEight ? 3 : 0;
    static constexpr int kKBufs = kEight ? kOps : DW == 128 ? 3 : 4, kVBufs = kEight ? kOps : DW == 128 ? 2 : 4;
    static constexpr int kKOff = kQBytes, kKEach = kEight ? 2 * kOpBytes : kOpBytes;
    static constexpr int kVOff = kEight ? kKOff + kOpBytes : kKOff + kKBufs * kOpBytes, kVEach = kKEach;
    static constexpr int kLoadOff = kEight ? kKOff + kOps * 2 * kOpBytes : kVOff + kVBufs * kOpBytes;
    static constexpr int kScaleOff = kLoadOff + kLoads * kLoadBytes; // 8-bit: of each operand buffer, scales of K and V
    static constexpr int kScaleBytes = 2 * kStep * 4;
    static constexpr int kOutOff = (kScaleOff + kOps * kScaleBytes + 127) / 128 * 128;  // of each softmax warp, 32 rows x 32 elements on their way out
    static constexpr int kSmem = 1024 + kOutOff + 8 * 2048;
    static_assert(kSmem <= 232448 - 6144, "shared memory");
    static constexpr int kPart = 128 * DW + 256;                     // floats of a CTA's part: [DW / 4][rows] of four, then m and l; at most 128 rows
    static constexpr int kRing = (kEight ? kScaleOff : kLoadOff) - kKOff;  // bytes of rings and operands: free at the end of a run
};

// The call's pieces: those of items with several come first, and number i of them has place i in the workspace.
template <int STEP>
struct RowsPieces {
    int C, cut, all;               // steps of a piece; pieces of items with several, and of all
    int past0, tiles0;             // of sequence `lane`
    static __device__ __forceinline__ int pieces(int tiles, int C) { return (tiles + C - 1) / C; }
    // The smallest C that gives each CTA its share of the steps and no item too many pieces; up to twice that if then no CTA has two pieces, and a few steps more if then
    // nothing is cut.
    __device__ __forceinline__ RowsPieces(const KvAttnArgs& a, int ctas, int lane) {
        const int per = a.Hkv * a.row_tiles;
        past0 = lane < a.B ? kv_past(a, lane) : 0;
        tiles0 = lane < a.B ? kv_tiles<STEP>(a, past0) : 0;
        int total = tiles0, most = tiles0;
        for (int b = 32 + lane; b < a.B; b += 32) {
            const int tiles = kv_tiles<STEP>(a, kv_past(a, b));
            total += tiles;
            most = max(most, tiles);
        }
        most = kv_max(most);
        // Adding one part to a merge takes as long as half a step: C + most / C / 2 is smallest at sqrt(most / 2).  16/1 heads of 128 over int8 rows of
        // one sequence, with as many pieces as CTAs and with this: 1000 rows 16.5 and 14.9 us, 4000 36.9 and 21.7, 8000 63.2 and 27.2, 32,000 67.6 and 47.2.
        const int N = kv_sum(total) * per, low = max((N + ctas - 1) / ctas, (int)__fsqrt_rn(0.5f * most));
        C = a.B * per <= ctas && most <= low + kRowsMerge ? most : low;
        count(a, lane);
        for (int c = low; all > ctas && c < 2 * low;) {
            c += max(c >> 4, 1);
            C = c;
            count(a, lane);
        }
        if (all > ctas && C > low) {
            C = low;
            count(a, lane);
        }
    }
    __device__ __forceinline__ void count(const KvAttnArgs& a, int lane) {
        const int per = a.Hkv * a.row_tiles;
        int n = lane < a.B ? pieces(tiles0, C) : 0, m = n > 1 ? n : 0;
        for (int b = 32 + lane; b < a.B; b += 32) {
            const int x = pieces(kv_tiles<STEP>(a, kv_past(a, b)), C);
            n += x;
            m += x > 1 ? x : 0;
        }
        all = kv_sum(n) * per;
        cut = kv_sum(m) * per;
    }
};
// Piece number idx.
struct RowsPiece {
    int b, kvh, rt;
    int first, tiles;              // its steps
    int start, of;                 // the item's pieces: number of the first, and how many
    int past, rows;
};
template <int STEP>
__device__ __forceinline__ RowsPiece rows_piece(const KvAttnArgs& a, const RowsPieces<STEP>& ps, int idx, int lane) {
    const int per = a.Hkv * a.row_tiles;
    const bool is_cut = idx < ps.cut;
    const int at = is_cut ? idx : idx - ps.cut;  // among those with several pieces, or among the others
    RowsPiece p;
    int before = 0, past = ps.past0, tiles = ps.tiles0;
#pragma unroll 1
    for (int b0 = 0;; b0 += 32) {
        int n = b0 + lane < a.B ? RowsPieces<STEP>::pieces(tiles, ps.C) : 0;
        if ((n > 1) != is_cut) n = 0;
        const int incl = kv_scan(n, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, at < (before + incl) * per);
        if (hit || b0 + 32 >= a.B) {
            const int src = hit ? __ffs(hit) - 1 : 0;
            p.b = b0 + src;
            p.of = __shfl_sync(0xffffffffu, n, src);
            p.past = __shfl_sync(0xffffffffu, past, src);
            const int first = (before + __shfl_sync(0xffffffffu, incl, src) - p.of) * per, in = at - first, item = in / p.of;
            p.kvh = item / a.row_tiles;
            p.rt = item - p.kvh * a.row_tiles;
            p.start = first + item * p.of;  // (of items with several)
            p.first = (in - item * p.of) * ps.C;
            p.tiles = min(ps.C, __shfl_sync(0xffffffffu, tiles, src) - p.first);
            p.rows = kv_rows(a, p.past);
            return p;
        }
        before += __shfl_sync(0xffffffffu, incl, 31);
        past = b0 + 32 + lane < a.B ? kv_past(a, b0 + 32 + lane) : 0;
        tiles = b0 + 32 + lane < a.B ? kv_tiles<STEP>(a, past) : 0;
    }
}

// Where element 8 i of row r of a [rows][64] chunk lies: 16-byte pieces swizzled over 128-byte lines.
__device__ __forceinline__ uint32_t sw128(int r, int piece) { return r * 128 + ((piece ^ (r & 7)) << 4); }

template <int DW, int FMT>
__global__ void __launch_bounds__(RowsShape<DW, FMT>::kThreads, 1)
attn_kv_rows_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ CUtensorMap tmap_ks, const __grid_constant__ CUtensorMap tmap_vs, const KvAttnArgs a) {
    using S = RowsShape<DW, FMT>;
    using namespace ptx;
    constexpr int kLoads = S::kLoads ? S::kLoads : 1, kConvThreads = S::kConvWarps ? S::kConvWarps * 32 : 32;
    constexpr bool kEight = S::kEight, kE4m3 = FMT == FORGE_KV_E4M3;
    constexpr bool kF16 = FMT != FORGE_KV_BF16;
    constexpr float kLift = kEight ? -8.f : 6.f;
    constexpr int kColS = 0, kColO = 2 * S::kStep;  // S of step n at kStep (n % 2), O of group h at kColO + DW h
    constexpr int kTmemCols = kColO + 2 * DW <= 256 ? 256 : 512;
    constexpr int kMaxOdd = 2 * kKvMaxTokens;
    extern __shared__ uint8_t smem_raw[];
    // codes (8-bit); operands of the scores and of the product with V (8-bit: complete together, k_full and k_empty serve for both)
    __shared__ uint64_t load_full[kLoads], load_empty[kLoads], k_full[S::kKBufs], k_empty[S::kKBufs], v_full[S::kVBufs], v_empty[S::kVBufs];
    constexpr int kMergeSlots = 4;
    __shared__ uint64_t merge_full[kMergeSlots];
    __shared__ uint64_t q_full, q_empty, q_ready, s_full[2], p_ready[2][2], pv_done[2][2];  // the last two: [step % 2][group]
    __shared__ uint32_t tmem_slot;
    // items that the CTA had a piece of several of; whether it was the last to arrive
    struct Cut { int start, of, b, kvh, rt; };
    __shared__ Cut cuts[2];
    __shared__ int cut_last[2];
    // halves of rows of V with elements that are not finite numbers, which some of the tokens see (twice the token's number, and which half);
    // pieces count in turns (see where they are cleared)
    __shared__ int odd_keys[kMaxOdd], odd_count[2];
    __shared__ float q_mul[128];                  // 8-bit: what a row's scores are multiplied by
    __shared__ float4 group_state[2][128];        // m, l and the unit of O
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    if (threadIdx.x == 0) {
        for (int i = 0; i < kLoads; ++i) { mbar_init(&load_full[i], 1); mbar_init(&load_empty[i], kEight ? S::kConvWarps : 1); }
        for (int i = 0; i < S::kKBufs; ++i) { mbar_init(&k_full[i], kEight ? S::kConvWarps : 1); mbar_init(&k_empty[i], 1); }
        for (int i = 0; i < S::kVBufs; ++i) { mbar_init(&v_full[i], 1); mbar_init(&v_empty[i], 1); }
        mbar_init(&q_full, 1);
        for (int i = 0; i < kMergeSlots; ++i) mbar_init(&merge_full[i], 1);
        mbar_init(&q_empty, 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s_full[i], 1);
            for (int h = 0; h < 2; ++h) { mbar_init(&p_ready[i][h], 4); mbar_init(&pv_done[i][h], 1); }
        }
        mbar_init(&q_ready, 4);
        fence_mbar_init();
        prefetch_tmap(&tmap_q);
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
        odd_count[0] = odd_count[1] = 0;
        cuts[0].of = cuts[1].of = 0;
    }
    if (warp == 9) {
        tmem_alloc(&tmem_slot, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();
    pdl_wait();

    const int ctas = gridDim.x;
    const RowsPieces<S::kStep> pieces(a, ctas, lane);
    bool failed = false;

    if (warp == 8) {
        // ------------------------------------------------------------------ copies
        // rows that only one row tile reads are marked first to go from L2
        const uint64_t policy = a.row_tiles == 1 ? l2_policy_evict_first() : l2_policy_evict_normal();
        int n = 0, parts = 0;
        for (int idx = blockIdx.x; idx < pieces.all; idx += ctas) {
            const RowsPiece p = rows_piece(a, pieces, idx, lane);
            if (elect_one()) {
                const int bk = p.b * a.Hkv + p.kvh;
                if (parts > 0 && !failed && !mbar_wait_relaxed(&q_empty, (parts - 1) & 1)) failed = true;
                if (!failed) mbar_expect_tx(&q_full, a.tile_rows * (DW * 2));
#pragma unroll
                for (int c = 0; c < DW / 64 && !failed; ++c)
                    tma_load_4d(smem + c * S::kQChunk, &tmap_q, &q_full, c * 64, 0, p.kvh * a.G + p.rt * a.tile_heads, p.b);
                for (int t = 0; t < p.tiles && !failed; ++t) {
                    const int j0 = (p.first + t) * S::kStep;
                    const bool none = j0 >= p.rows;  // a sequence without rows
                    if constexpr (kEight) {
                        const int pos = n + t, st = pos % kLoads;
                        if (pos >= kLoads && !mbar_wait_relaxed(&load_empty[st], (pos / kLoads - 1) & 1)) { failed = true; break; }
                        if (none) { mbar_arrive(&load_full[st]); continue; }
                        const uint32_t dst = smem_u32(smem + S::kLoadOff + st * S::kLoadBytes);
                        const int x = (bk * a.Smax + j0) & ~3;
                        mbar_expect_tx(&load_full[st], 2 * S::kRawBytes + 2 * S::kScaleKeys * 4);
                        tma_load_3d_addr_hint(dst, &tmap_k, &load_full[st], 0, j0, bk, policy);
                        tma_load_1d(dst + 2 * S::kRawBytes, &tmap_ks, &load_full[st], x);
                        tma_load_3d_addr_hint(dst + S::kRawBytes, &tmap_v, &load_full[st], 0, j0, bk, policy);
                        tma_load_1d(dst + 2 * S::kRawBytes + S::kScaleBox, &tmap_vs, &load_full[st], x);
                    } else {
                        const int pos = n + t, kb = pos % S::kKBufs, vb = pos % S::kVBufs;
                        if (pos >= S::kKBufs && !mbar_wait_relaxed(&k_empty[kb], (pos / S::kKBufs - 1) & 1)) { failed = true; break; }
                        if (none) {
                            mbar_arrive(&k_full[kb]);
                        } else {
                            mbar_expect_tx(&k_full[kb], S::kOpBytes);
#pragma unroll
                            for (int c = 0; c < DW / 64; ++c)
                                tma_load_3d_addr_hint(smem_u32(smem + S::kKOff + kb * S::kKEach + c * S::kOpChunk), &tmap_k, &k_full[kb], c * 64, j0, bk, policy);
                        }
                        if (pos >= S::kVBufs && !mbar_wait_relaxed(&v_empty[vb], (pos / S::kVBufs - 1) & 1)) { failed = true; break; }
                        if (none) {
                            mbar_arrive(&v_full[vb]);
                        } else {
                            mbar_expect_tx(&v_full[vb], S::kOpBytes);
#pragma unroll
                            for (int c = 0; c < DW / 64; ++c)
                                tma_load_3d_addr_hint(smem_u32(smem + S::kVOff + vb * S::kVEach + c * S::kOpChunk), &tmap_v, &v_full[vb], c * 64, j0, bk, policy);
                        }
                    }
                }
            }
            __syncwarp();
            n += p.tiles;
            ++parts;
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ products
        constexpr uint32_t idesc_s = kF16 ? make_idesc_f16(128, S::kStep, false, false) : make_idesc_bf16(128, S::kStep, false, false);
        constexpr uint32_t idesc_o = kF16 ? make_idesc_f16(128, DW, false, true) : make_idesc_bf16(128, DW, false, true);
        int base = 0, parts = 0;  // steps and pieces before this one
        for (int idx = blockIdx.x; idx < pieces.all; idx += ctas) {
            const RowsPiece p = rows_piece(a, pieces, idx, lane);
            const int n = p.tiles;
            if (elect_one() && !failed) {
                const uint64_t qd = make_smem_desc(smem_u32(smem), 16, 1024);
                auto issue_qk = [&](int g) -> bool {
                    const int pos = base + g, buf = pos % S::kKBufs;
                    if (!mbar_wait(&k_full[buf], (pos / S::kKBufs) & 1)) return false;
                    tc_fence_after_sync();
                    const uint64_t kd = make_smem_desc(smem_u32(smem + S::kKOff + buf * S::kKEach), 16, 1024);
#pragma unroll
                    for (int k = 0; k < DW / 16; ++k)
                        mma_ss(tmem + kColS + (pos & 1) * S::kStep, qd + (((k / 4) * S::kQChunk + (k % 4) * 32) >> 4),
                               kd + (((k / 4) * S::kOpChunk + (k % 4) * 32) >> 4), idesc_s, k != 0);
                    mma_commit(&s_full[pos & 1]);
                    if (!kEight) mma_commit(&k_empty[buf]);
                    if (g == n - 1) mma_commit(&q_empty);
                    return true;
                };
                const bool have_q = kEight ? mbar_wait(&q_ready, parts & 1) : mbar_wait(&q_full, parts & 1);
                failed = !have_q;
                for (int g = 0; g < n && g < 2 && !failed; ++g) failed = !issue_qk(g);
                for (int g = 0; g < n && !failed; ++g) {
                    const int pos = base + g, buf = pos % S::kVBufs;
                    if (!kEight && !mbar_wait(&v_full[buf], (pos / S::kVBufs) & 1)) { failed = true; break; }
                    const uint64_t vd = make_smem_desc(smem_u32(smem + S::kVOff + buf * S::kVEach), S::kOpChunk, 1024);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {  // P of group h in the first columns of its half of S
                        if (!mbar_wait(&p_ready[pos & 1][h], (pos / 2) & 1)) { failed = true; break; }
                        tc_fence_after_sync();
#pragma unroll
                        for (int k = 0; k < S::kHalf / 16; ++k)
                            mma_ts(tmem + kColO + h * DW, tmem + kColS + (pos & 1) * S::kStep + h * S::kHalf + k * 8,
                                   vd + (h * (S::kHalf / 16) + k) * (2048 >> 4), idesc_o, g > 0 || k != 0);
#pragma unroll
                        for (int k = 0; k < S::kHalf / 16; ++k)  // what rounding P left
                            mma_ts(tmem + kColO + h * DW, tmem + kColS + (pos & 1) * S::kStep + h * S::kHalf + S::kHalf / 2 + k * 8,
                                   vd + (h * (S::kHalf / 16) + k) * (2048 >> 4), idesc_o, 1);
                        mma_commit(&pv_done[pos & 1][h]);
                    }
                    if (failed) break;
                    mma_commit(kEight ? &k_empty[buf] : &v_empty[buf]);
                    if (g + 2 < n && !issue_qk(g + 2)) { failed = true; break; }
                }
            }
            __syncwarp();
            base += n;
            ++parts;
        }
    } else if (kEight && warp >= 10) {
        // ------------------------------------------------------------------ codes to fp16
        constexpr int kOps = S::kOps ? S::kOps : 1;
        const int t = threadIdx.x - 10 * 32;
        int n = 0;
        for (int idx = blockIdx.x; idx < pieces.all && !failed; idx += ctas) {
            const RowsPiece p = rows_piece(a, pieces, idx, lane);
            for (int i = 0; i < p.tiles; ++i, ++n) {
                const int st = n % kLoads, buf = n % kOps, j0 = (p.first + i) * S::kStep;
                if (!warp_wait(&load_full[st], (n / kLoads) & 1)) { failed = true; break; }
                if (n >= kOps && !warp_wait(&k_empty[buf], (n / kOps - 1) & 1)) { failed = true; break; }
                const uint32_t raw = smem_u32(smem + S::kLoadOff + st * S::kLoadBytes);
                uint8_t* op = smem + S::kKOff + buf * S::kKEach;
                // a thread's 16-byte pieces of codes: K's, then V's (16 codes become 32 bytes: two pieces of the operand)
                constexpr int kPerRow = DW / 16, kPieces = S::kStep * kPerRow / kConvThreads;
#pragma unroll
                for (int mat = 0; mat < 2; ++mat)
#pragma unroll 4
                    for (int x = 0; x < kPieces; ++x) {
                        const int at = x * kConvThreads + t, row = at / kPerRow, piece = at % kPerRow;
                        uint32_t w[4], o[8];
                        lds4(raw + mat * S::kRawBytes + row * DW + ((DW == 128 ? piece ^ (row & 7) : piece ^ ((row >> 1) & 3)) << 4), w);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if constexpr (kE4m3) {
                                o[2 * k] = e4m3_pair(w[k]);
                                o[2 * k + 1] = e4m3_pair(w[k] >> 16);
                                if (mat) { o[2 * k] = e4m3_finite(o[2 * k]); o[2 * k + 1] = e4m3_finite(o[2 * k + 1]); }
                            } else {
                                o[2 * k] = sub_1152(even_bytes(w[k]));
                                o[2 * k + 1] = sub_1152(even_bytes(w[k] >> 8));
                            }
                        }
                        uint8_t* dst = op + mat * S::kOpBytes + (piece >> 2) * S::kOpChunk;
                        *reinterpret_cast<uint4*>(dst + sw128(row, (piece & 3) * 2)) = make_uint4(o[0], o[1], o[2], o[3]);
                        *reinterpret_cast<uint4*>(dst + sw128(row, (piece & 3) * 2 + 1)) = make_uint4(o[4], o[5], o[6], o[7]);
                    }
                // scales (warp 10: of K, warp 11: of V): those of rows that are not there count as zero
                if (warp < 12) {
                    float* sc = reinterpret_cast<float*>(smem + S::kScaleOff + buf * S::kScaleBytes) + (warp - 10) * S::kStep;
                    const float* from = reinterpret_cast<const float*>(smem + S::kLoadOff + st * S::kLoadBytes + 2 * S::kRawBytes + (warp - 10) * S::kScaleBox) +
                                        (((p.b * a.Hkv + p.kvh) * a.Smax + j0) & 3);
                    const float x0 = j0 + lane < p.rows ? from[lane] : 0.f, x1 = j0 + 32 + lane < p.rows ? from[32 + lane] : 0.f;
                    sc[lane] = x0;
                    sc[32 + lane] = x1;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&k_full[buf]);
                    mbar_arrive(&load_empty[st]);
                }
            }
        }
    } else if (warp < 8) {
        // ------------------------------------------------------------------ softmax, O
        const int group = warp >> 2, row = threadIdx.x & 127;
        const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        auto slot = [&](int piece) { return a.parts + (size_t)piece * S::kPart; };
        const bool out_f16 = kEight ? a.q_f16 : kF16;
        constexpr int kCols = DW / 2;
        const int col0 = (warp >> 2) * kCols;  // a group of threads writes a half of O's columns
        auto out_row = [&](int b, int kvh, int h, int tok) {
            return static_cast<uint16_t*>(a.out) + b * a.os.b + (int64_t)(kvh * a.G + h) * a.os.h + tok * a.os.s;
        };
        // Elements d .. d + 31 of this thread's row, scaled: through shared memory, so that a warp's store covers 8 rows' 64 bytes each (16 bytes of
        // 32 rows each take four times as long).  All lanes of the warp take part.
        uint8_t* out_stage = smem + S::kOutOff + warp * 2048;
        auto write_out = [&](const uint16_t* orow, bool live, int d, const float (&x)[32], float scale) {
            auto pair = [&](float y, float z) { return out_f16 ? pack16<true>(y * scale, z * scale) : pack16<false>(y * scale, z * scale); };
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint4*>(out_stage + lane * 64 + ((i ^ (lane >> 1 & 3)) << 4)) =
                    make_uint4(pair(x[i * 8], x[i * 8 + 1]), pair(x[i * 8 + 2], x[i * 8 + 3]), pair(x[i * 8 + 4], x[i * 8 + 5]), pair(x[i * 8 + 6], x[i * 8 + 7]));
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = i * 8 + (lane >> 2), piece = lane & 3;
                const unsigned long long to = __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(orow), r);
                const bool there = __shfl_sync(0xffffffffu, live, r);
                if (there && d + piece * 8 < a.D)
                    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(to) + d + piece * 8) =
                        *reinterpret_cast<const uint4*>(out_stage + r * 64 + ((piece ^ (r >> 1 & 3)) << 4));
            }
        };
        // Waits for this group's product of a step whose scores it has seen.  A wait tells a phase from the next one only, and the tensor cores may be a step behind
        // this group where the other one's P is late: so steps take two barriers in turns.  The phase before, of step pos - 2, is over then: the scores of
        // step pos were asked for behind that product, or it was one of the piece before.
        auto product_done = [&](int pos) { return warp_wait(&pv_done[pos & 1][group], (pos / 2) & 1); };
        auto rows_sync = [] { asm volatile("bar.sync 1, 256;" ::: "memory"); };
        int base = 0, parts = 0;  // steps and pieces before this one
        unsigned long long next_sees = 0;
        for (int idx = blockIdx.x; idx < pieces.all; idx += ctas) {
            const RowsPiece p = rows_piece(a, pieces, idx, lane);
            const int at = p.rt * a.tile_rows + row;                  // row of the KV head
            const bool live = row < a.tile_rows && at < a.rows;
            const bool idle = (warp & 3) * 32 >= min(a.tile_rows, a.rows - p.rt * a.tile_rows);  // the whole warp has no row
            const int T = max(a.T, 1), h = at / T, tok = at - h * T;
            // the mask of this row's token, and that of the next piece: asked for now, behind the copies in flight it is long in coming
            auto mask_of = [&](const RowsPiece& of) -> unsigned long long {
                const int r = of.rt * a.tile_rows + row, t = r - r / T * T;
                if (a.T == 0 || row >= a.tile_rows || r >= a.rows) return 0;
                return a.tree ? a.tree[(int64_t)of.b * a.tree_stride + t] : (2ull << t) - 1ull;
            };
            const unsigned long long sees = parts == 0 ? mask_of(p) : next_sees;
            if (idx + ctas < pieces.all) next_sees = mask_of(rows_piece(a, pieces, idx + ctas, lane));
            float mul = a.scale_log2;
            if constexpr (kEight) {
                // ---- group 0: the row of Q, in place, to fp16 in the codes' order, scaled by a power of two that puts its largest into
                // [2^14, 2^15): fp16 keeps bf16's bits
                if (group == 0) {
                    uint8_t* sq = smem;
                    if (!failed && !warp_wait(&q_full, parts & 1)) failed = true;
                    uint32_t big = 0;
#pragma unroll
                    for (int i = 0; i < DW / 8; ++i) {
                        const uint4 w = *reinterpret_cast<const uint4*>(sq + (i >> 3) * S::kQChunk + sw128(row, i & 7));
                        big = __vmaxu2(__vmaxu2(big, __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu)), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
                    }
                    big = max(big & 0xffffu, big >> 16);
                    const float top = a.q_f16 ? __half2float(__ushort_as_half((unsigned short)big)) : __uint_as_float(big << 16);
                    const int e = (int)(__float_as_uint(top) >> 23) - 127;
                    const int up = top == 0.f || e == 128 ? 0 : min(max(14 - e, -113), 110);
                    const float f = __int_as_float((127 + up) << 23);
                    q_mul[row] = a.scale_log2 * __int_as_float((127 - up) << 23);
#pragma unroll 4
                    for (int i = 0; i < DW / 8; ++i) {
                        uint4* at16 = reinterpret_cast<uint4*>(sq + (i >> 3) * S::kQChunk + sw128(row, i & 7));
                        const uint32_t in[4] = {at16->x, at16->y, at16->z, at16->w};
                        uint32_t out[4];
#pragma unroll
                        for (int k = 0; k < 4; k += 2) {
                            float2 x, y;
                            if (a.q_f16) {
                                x = __half22float2(*reinterpret_cast<const __half2*>(&in[k]));
                                y = __half22float2(*reinterpret_cast<const __half2*>(&in[k + 1]));
                            } else {
                                x = make_float2(__uint_as_float(in[k] << 16), __uint_as_float(in[k] & 0xffff0000u));
                                y = make_float2(__uint_as_float(in[k + 1] << 16), __uint_as_float(in[k + 1] & 0xffff0000u));
                            }
                            out[k] = kE4m3 ? pack16<true>(x.x * f, x.y * f) : pack16<true>(x.x * f, y.x * f);
                            out[k + 1] = kE4m3 ? pack16<true>(y.x * f, y.y * f) : pack16<true>(x.y * f, y.y * f);
                        }
                        *at16 = make_uint4(out[0], out[1], out[2], out[3]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&q_ready);
                }
                if (!failed && !warp_wait(&q_ready, parts & 1)) failed = true;
                mul = q_mul[row];
            }

            float m = -INFINITY, l = 0.f;
            float unit_inv = kv_pow2(-kUnitLow);  // 8-bit: of this row (see kUnitLow)
            const int n = p.tiles;
#pragma unroll 1
            for (int g = 0; g < n; ++g) {
                const int pos = base + g, buf = pos % S::kVBufs;
                const int key0 = (p.first + g) * S::kStep + group * S::kHalf;  // of this group's half
                const uint32_t s_col = lanes + kColS + (pos & 1) * S::kStep + group * S::kHalf, o_col = lanes + kColO + group * DW;
                if (!failed && !warp_wait(&s_full[pos & 1], (pos / 2) & 1)) failed = true;
                if (failed) break;
                tc_fence_after_sync();
                const bool cut = key0 + S::kHalf > p.past;
                float alpha = 1.f;
                const float* sc = reinterpret_cast<const float*>(smem + S::kScaleOff + buf * S::kScaleBytes) + group * S::kHalf;
                // the scales, or the rows of V that are looked through below (complete by now: the scores waited for them)
                if ((kEight || cut) && !warp_wait(kEight ? &k_full[buf] : &v_full[buf], (pos / S::kVBufs) & 1)) { failed = true; break; }
                // 32 scores of this row (8-bit: times the factors' product, each of which may be as far from 1 as the other makes up for); the keys that it
                // sees, as bits (cut)
                auto scores = [&](int c, float (&x)[32]) {
                    uint32_t r[32];
                    tmem_ld_x32(s_col + c, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = __uint_as_float(r[k]);
                    if constexpr (kEight) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 ks = *reinterpret_cast<const float4*>(sc + c + k);
                            x[k] *= ks.x * mul; x[k + 1] *= ks.y * mul; x[k + 2] *= ks.z * mul; x[k + 3] *= ks.w * mul;
                        }
                    }
                };
                auto seen = [&](int c) -> uint32_t {
                    const int d = p.past - key0 - c, have = p.rows - key0 - c;  // the past ends d keys, all rows `have` keys on
                    if (d >= 32) return 0xffffffffu;
                    uint32_t v = d > 0 ? ((1u << d) - 1u) | (uint32_t)(sees << d) : d > -64 ? (uint32_t)(sees >> -d) : 0u;
                    if (have < 32) v &= have > 0 ? (1u << have) - 1u : 0u;
                    return v;
                };
                float kept[S::kHalf / 32][32];
                if (!idle) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int c = 0; c < S::kHalf; c += 32) {
                        float (&x)[32] = kept[c / 32];
                        scores(c, x);
                        if constexpr (!kEight) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] *= mul;
                        }
                        if (cut) {
                            const uint32_t v = seen(c);
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] = v >> k & 1u ? x[k] : -INFINITY;
                        }
#pragma unroll
                        for (int k = 0; k < 32; k += 2) mx = max3(mx, x[k], x[k + 1]);
                    }
                    // the reference is raised only where a score passes it by 2^8 (the first of a row always does)
                    if (mx > m + kRowsAbove) {
                        if constexpr (kEight) mx = ceilf(mx);
                        const float by = m == -INFINITY ? 0.f : m - mx;
                        m = mx;
                        alpha = ex2(by);
                        l *= alpha;
                        if constexpr (kEight) alpha = kv_lower_unit(unit_inv, by);
                    }
                    if constexpr (kEight) {  // p, then p vs
                        const float ref = m == -INFINITY ? 0.f : m - kLift;
                        float most = 0.f;
#pragma unroll
                        for (int c = 0; c < S::kHalf; c += 32) {
                            float (&x)[32] = kept[c / 32];
                            float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                x[k] = ex2(x[k] - ref);
                                add[k & 3] += x[k];
                            }
                            l += (add[0] + add[1]) + (add[2] + add[3]);
#pragma unroll
                            for (int k = 0; k < 32; k += 4) {
                                const float4 vs = *reinterpret_cast<const float4*>(sc + S::kStep + c + k);
                                x[k] *= vs.x; x[k + 1] *= vs.y; x[k + 2] *= vs.z; x[k + 3] *= vs.w;
                            }
                            if (cut) {  // the scale of a row that is not seen may be anything
                                const uint32_t v = seen(c);
#pragma unroll
                                for (int k = 0; k < 32; ++k) x[k] = v >> k & 1u ? x[k] : 0.f;
                            }
#pragma unroll
                            for (int k = 0; k < 32; k += 2) most = max3(most, fabsf(x[k]), fabsf(x[k + 1]));
                        }
                        alpha *= kv_raise_unit(unit_inv, most);
                    }
                }
                if (g > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
                    // O must hold the group's products so far
                    if (!product_done(pos - 1)) { failed = true; break; }
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < DW / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld_x32(o_col + c * 32, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * alpha);
                        tmem_st_x32(o_col + c * 32, r);
                    }
                }
                if (!idle) {
                    const float ref = m == -INFINITY ? 0.f : m - kLift;
#pragma unroll
                    for (int c = 0; c < S::kHalf; c += 32) {
                        float (&x)[32] = kept[c / 32];
                        if constexpr (kEight) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) x[k] *= unit_inv;
                        } else {
                            float add[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int k = 0; k < 32; ++k) {
                                x[k] = ex2(x[k] - ref);
                                add[k & 3] += x[k];
                            }
                            l += (add[0] + add[1]) + (add[2] + add[3]);
                        }
                        // What rounding P to the products' type leaves is multiplied too, from the columns of S that P leaves free, so that outputs are off by
                        // their own rounding alone.  Errors against 64 bits, without and with it: 4 x 32/8 x 64 tokens of bf16 2.3e-3 and 1.66e-3,
                        // 8 x 28/4 x 16 fp16 tokens over int8 rows 2.9e-4 and 2.1e-4; times 29.0 and 30.2 us, 24.2 and 25.1.
                        uint32_t packed[16];
#pragma unroll
                        for (int k = 0; k < 16; ++k) packed[k] = kv_operand<kF16, !kEight>(x[2 * k], x[2 * k + 1]);
                        tmem_st_x16(s_col + c / 2, packed);
#pragma unroll
                        for (int k = 0; k < 16; ++k) packed[k] = kv_rest<kF16, !kEight>(x[2 * k], x[2 * k + 1], packed[k]);
                        tmem_st_x16(s_col + S::kHalf / 2 + c / 2, packed);
                    }
                }
                if constexpr (!kEight) {
                    // What must not reach the product: rows of V past the end, and elements that are not finite numbers in rows that only
                    // some of the tokens see (0 x NaN is NaN); those are remembered and added at the end.
                    if (cut) {
                        constexpr uint32_t kExp = kF16 ? 0x7c00u : 0x7f80u;
                        uint8_t* v = smem + S::kVOff + buf * S::kVEach;
                        // two threads to a key, a half of its elements each
                        const int key = row >> 1, vrow = group * S::kHalf + key;
                        if (key0 + key >= p.past) {
                            const bool out = key0 + key >= p.rows;
                            bool odd = false;
#pragma unroll
                            for (int i = 0; i < DW / 16; ++i) {
                                const int piece = (row & 1) * (DW / 16) + i;
                                uint4* at16 = reinterpret_cast<uint4*>(v + (piece >> 3) * S::kOpChunk + sw128(vrow, piece & 7));
                                uint32_t x[4] = {at16->x, at16->y, at16->z, at16->w};
                                bool put = out;
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    if ((x[k] & kExp) == kExp) { x[k] &= 0xffff0000u; put = odd = true; }
                                    if ((x[k] >> 16 & kExp) == kExp) { x[k] &= 0xffffu; put = odd = true; }
                                    if (out) x[k] = 0;
                                }
                                if (put) *at16 = make_uint4(x[0], x[1], x[2], x[3]);
                            }
                            if (odd && !out) {
                                const int i = atomicAdd(&odd_count[parts & 1], 1);
                                if (i < kMaxOdd) odd_keys[i] = (key0 + key - p.past) * 2 + (row & 1);
                            }
                        }
                        fence_proxy_async_smem();
                    }
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready[pos & 1][group]);
            }
            if (!failed && !product_done(base + n - 1)) failed = true;
            tc_fence_after_sync();
            base += n;
            group_state[group][row] = make_float4(m, l, kv_unit(unit_inv), 0.f);
            rows_sync();  // both groups' products are done, their states and odd_keys complete
            tc_fence_after_sync();

            // ---- the two groups' O together, normalised or not, a half of the columns for each group of threads;
            // int8: column 4 i + 1 holds element 4 i + 2 and the other way round
            const bool whole = p.of == 1;
            uint16_t* orow = out_row(p.b, p.kvh, h, tok);
            const int odds = kEight ? 0 : min(odd_count[parts & 1], kMaxOdd);
            float* mine = slot(idx);  // (of an item with several pieces)
            if (!idle && !failed) {
                const float4 s0 = group_state[0][row], s1 = group_state[1][row];
                const float M = fmaxf(s0.x, s1.x), ref = M == -INFINITY ? 0.f : M;
                const float e0 = ex2(s0.x - ref), e1 = ex2(s1.x - ref), L = fmaf(e0, s0.y, e1 * s1.y);
                const float w0 = kEight ? e0 * s0.z : e0, w1 = kEight ? e1 * s1.z : e1;
#pragma unroll 1
                for (int c = 0; c < kCols / 32; ++c) {
                    const int d = col0 + c * 32;
                    uint32_t r[32];
                    float x[32];
                    tmem_ld_x32(lanes + kColO + d, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = __uint_as_float(r[k]) * w0;
                    tmem_ld_x32(lanes + kColO + DW + d, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = fmaf(__uint_as_float(r[k]), w1, x[k]);
                    if constexpr (kEight && !kE4m3) {
#pragma unroll
                        for (int k = 1; k < 32; k += 4) {
                            const float t = x[k];
                            x[k] = x[k + 1];
                            x[k + 1] = t;
                        }
                    }
                    for (int i = 0; i < odds; ++i) {
                        const int u = odd_keys[i] >> 1;
                        if ((odd_keys[i] & 1) != group || !(sees >> u & 1ull)) continue;
                        const uint16_t* v = static_cast<const uint16_t*>(a.v) + ((int64_t)(p.b * a.Hkv + p.kvh) * a.Smax + p.past + u) * a.D + d;
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            if (d + k >= a.D) continue;
                            const float y = kF16 ? __half2float(__ushort_as_half((unsigned short)v[k])) : __uint_as_float((uint32_t)v[k] << 16);
                            if (!(fabsf(y) <= 3.4028235e38f)) x[k] += y;
                        }
                    }
                    if (whole) {
                        write_out(orow, live, d, x, L == 0.f ? 0.f : 1.f / L);  // no key seen: zeros
                    } else if (live) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            reinterpret_cast<float4*>(mine)[(d / 4 + k) * a.tile_stride + row] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    }
                }
                if (!whole && live && group == 0) reinterpret_cast<float2*>(mine + a.tile_stride * DW)[row] = make_float2(M, L);
            }
            // The next piece's counter, cleared on this side of the barrier, behind which other warps count into it at once: it was last read
            // before the previous piece's.  This piece's is being read.
            if (threadIdx.x == 0) odd_count[(parts + 1) & 1] = 0;
            ++parts;
            tc_fence_before_sync();
            rows_sync();  // the parts are written; odd_keys and O have been read
            if (threadIdx.x == 0 && !whole)
                cuts[idx / ctas] = {p.start, p.of, p.b, p.kvh, p.rt};  // at most two of them: they come first, and are no more than twice the CTAs
        }

        // ---- items that other CTAs have parts of: the CTA that arrives last merges all of them
        rows_sync();
        if (threadIdx.x == 0 || threadIdx.x == 32) {
            const int e = threadIdx.x / 32;
            const Cut cut = cuts[e];
            cut_last[e] = 0;
            if (cut.of > 0) {
                unsigned int before;
                asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.counters + cut.start) : "memory");
                if (before + 1 == (unsigned)cut.of) {
                    a.counters[cut.start] = 0;  // as the next call expects it
                    cut_last[e] = 1;
                }
            }
        }
        rows_sync();
        uint32_t merge_phase = 0;  // a bit for each slot
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            if (!cut_last[e]) continue;
            const Cut cut = cuts[e];
            // The parts come by bulk copies into the rings, which are free by now, a few ahead of the one that is added.
            const int bytes = a.tile_stride * (DW + 2) * 4, slots = min(S::kRing / bytes, kMergeSlots);
            const int at = cut.rt * a.tile_rows + row;
            const bool live = row < a.tile_rows && at < a.rows;
            auto copy = [&](int i, int sl) {  // thread 0
                mbar_expect_tx(&merge_full[sl], bytes);
                bulk_load(smem_u32(smem + S::kKOff + sl * bytes), slot(cut.start + i), bytes, &merge_full[sl]);
            };
            if (threadIdx.x == 0) {
                asm volatile("fence.proxy.async;" ::: "memory");  // what other SMs wrote with plain stores is read by the copy engine
                for (int i = 0; i < min(slots, cut.of); ++i) copy(i, i);
            }
            float M = -INFINITY, L = 0.f, x[kCols / 32][32];
            if (live) {  // the row's reference first, while the copies fly: then a part is one product and sum for each element
#pragma unroll 4
                for (int i = 0; i < cut.of; ++i) M = fmaxf(M, slot(cut.start + i)[a.tile_stride * DW + 2 * row]);
            }
            const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int c = 0; c < kCols / 32; ++c)
#pragma unroll
                for (int k = 0; k < 32; ++k) x[c][k] = 0.f;
#pragma unroll 1
            for (int i = 0, sl = 0; i < cut.of; ++i, sl = sl + 1 == slots ? 0 : sl + 1) {
                if (!failed && !warp_wait(&merge_full[sl], merge_phase >> sl & 1u)) failed = true;
                merge_phase ^= 1u << sl;
                const uint8_t* from = smem + S::kKOff + sl * bytes;
                if (live) {
                    const float2 ml = reinterpret_cast<const float2*>(from + a.tile_stride * DW * 4)[row];
                    const float w = ex2(ml.x - ref);
                    L = fmaf(w, ml.y, L);
#pragma unroll
                    for (int c = 0; c < kCols / 32; ++c)
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float4 y = reinterpret_cast<const float4*>(from)[(col0 / 4 + c * 8 + k) * a.tile_stride + row];
                            x[c][4 * k] = fmaf(w, y.x, x[c][4 * k]);
                            x[c][4 * k + 1] = fmaf(w, y.y, x[c][4 * k + 1]);
                            x[c][4 * k + 2] = fmaf(w, y.z, x[c][4 * k + 2]);
                            x[c][4 * k + 3] = fmaf(w, y.w, x[c][4 * k + 3]);
                        }
                }
                rows_sync();  // read before the next copy lands
                if (threadIdx.x == 0 && i + slots < cut.of && !failed) copy(i + slots, sl);
            }
            const int T = max(a.T, 1), h = at / T;
            const uint16_t* orow = out_row(cut.b, cut.kvh, h, at - h * T);
#pragma unroll
            for (int c = 0; c < kCols / 32; ++c) write_out(orow, live && !failed, col0 + c * 32, x[c], L == 0.f ? 0.f : 1.f / L);
        }
    }

    if (failed) {
        atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and products in flight end before their memory goes away
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, kTmemCols);
}

template <int DW, int FMT>
int launch_attn_kv_rows(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {
    using S = RowsShape<DW, FMT>;
    CUtensorMap tq, tk, tv, tks = {}, tvs = {};
    const uint64_t es = S::kEight ? 1 : 2;
    const uint32_t box[3] = {S::kEight ? (uint32_t)DW : 64u, (uint32_t)S::kStep, 1};
    const uint64_t dims[3] = {(uint64_t)cache.D, (uint64_t)cache.Smax, (uint64_t)cache.B * cache.Hkv};
    const uint64_t strides[2] = {(uint64_t)cache.D * es, (uint64_t)cache.Smax * cache.D * es};
    const auto encode = !S::kEight ? encode_tmap_bf16_sw128 : DW == 128 ? encode_tmap_u8_sw128 : encode_tmap_u8_sw64;
    if (!encode(&tk, cache.k, 3, dims, strides, box) || !encode(&tv, cache.v, 3, dims, strides, box)) return FORGE_ERR_CUDA;
    {
        const int T = a.T > 0 ? a.T : 1;
        const uint64_t qdims[4] = {(uint64_t)cache.D, (uint64_t)T, (uint64_t)a.G * a.Hkv, (uint64_t)a.B};
        const uint64_t qstrides[3] = {(uint64_t)a.qs.s * 2, (uint64_t)a.qs.h * 2, (uint64_t)a.qs.b * 2};
        const uint32_t qbox[4] = {64, (uint32_t)T, (uint32_t)a.tile_heads, 1};
        if (!encode_tmap_bf16_sw128(&tq, a.q, 4, qdims, qstrides, qbox)) return FORGE_ERR_CUDA;
    }
    if (S::kEight) {
        const uint32_t sbox[1] = {(uint32_t)S::kScaleKeys};
        const uint64_t n[1] = {(uint64_t)cache.B * cache.Hkv * cache.Smax};
        if (!encode_tmap_f32_plain(&tks, cache.k_scale, 1, n, nullptr, sbox) || !encode_tmap_f32_plain(&tvs, cache.v_scale, 1, n, nullptr, sbox))
            return FORGE_ERR_CUDA;
    }
    auto kernel = attn_kv_rows_kernel<DW, FMT>;
    FORGE_SET_SMEM_ONCE(kernel, S::kSmem);
    FORGE_CUDA_TRY(launch_pdl(kernel, dim3(ctas), dim3(S::kThreads), S::kSmem, s, tq, tk, tv, tks, tvs, a));
    return finish_launch(1);
}

}  // namespace
}  // namespace forge
