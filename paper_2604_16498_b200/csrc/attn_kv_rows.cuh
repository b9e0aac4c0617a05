// Attention over a KV cache for more than 8 query rows per (sequence, KV head): trees of drafted tokens, and single tokens of large head
// groups.  Included by attn_kv.cuh.
//
// The rows (up to 128: several tokens of several heads that share K and V) are one tile of the tensor cores: per 64 keys
//     S[128 x 64] = Q K^T  and  O[128 x DW] += P V   by tcgen05.mma, S (two buffers), P and O in tensor memory,
// and thread = row does the softmax in between.  The call's 64-key steps are shared evenly by all CTAs, as in the other kernel, and what a CTA
// has of an item that others have parts of too is merged by the one that finishes last.
//   warps 0-3   Q into shared memory, softmax, O out      warp 4  TMA      warp 5  tcgen05.mma
//   warps 6-9   8-bit rows only: codes of K and V to fp16, from the copies' ring into operands
// 8-bit rows stay codes in the products (exact in fp16; int8 elements come in the order 0 2 1 3 of each four, in Q and O too); their scales
// multiply the scores and the probabilities.
#pragma once

namespace forge {
namespace {

constexpr int kRowsStep = 64;
constexpr float kRowsTop = 14.f, kRowsLift = 6.f;  // p reaches 2^14, 2^8 above what the reference stands for

template <int DW, int FMT>
struct RowsShape {
    static constexpr bool kEight = FMT == FORGE_KV_INT8 || FMT == FORGE_KV_E4M3;
    static constexpr int kThreads = (kEight ? 10 : 6) * 32;
    static constexpr int kQChunk = 128 * 128;                        // 128 rows x 64 elements
    static constexpr int kQBytes = DW / 64 * kQChunk;
    static constexpr int kOpChunk = kRowsStep * 128;                 // 64 keys x 64 elements
    static constexpr int kOpBytes = DW / 64 * kOpChunk;              // K, or V
    static constexpr int kRawBytes = kRowsStep * DW;                 // 8-bit: the codes of K, or V
    static constexpr int kScaleBox = 512;                            // 64 scales from the 16-byte boundary at or before the first
    static constexpr int kScaleKeys = kRowsStep + 4;
    static constexpr int kLoadBytes = kEight ? 2 * kRawBytes + 2 * kScaleBox : 2 * kOpBytes;  // a stage of the copies
    static constexpr int kLoads = kEight ? (DW == 128 ? 5 : 6) : (DW == 128 ? 5 : 8);
    static constexpr int kOps = kEight ? 3 : 0;                      // 8-bit: operand buffers, K then V
    static constexpr int kBufs = kEight ? kOps : kLoads;             // of operands, either way
    static constexpr int kOpOff = kQBytes;
    static constexpr int kLoadOff = kOpOff + kOps * 2 * kOpBytes;
    static constexpr int kScaleOff = kLoadOff + kLoads * kLoadBytes; // 8-bit: of each operand buffer, scales of K and V and the largest of V
    static constexpr int kScaleBytes = 2 * kRowsStep * 4 + 16;
    static constexpr int kSmem = 1024 + kScaleOff + kOps * kScaleBytes;
    static_assert(kSmem <= 232448 - 1024, "shared memory");
    static constexpr int kPart = 128 * DW + 256;                     // floats of a CTA's part: [DW / 4][128 rows] of four, then m and l
};

// Where element 8 i of row r of a [rows][64] chunk lies: 16-byte pieces swizzled over 128-byte lines.
__device__ __forceinline__ uint32_t sw128(int r, int piece) { return r * 128 + ((piece ^ (r & 7)) << 4); }

template <int DW, int FMT>
__global__ void __launch_bounds__(RowsShape<DW, FMT>::kThreads, 1)
attn_kv_rows_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                    const __grid_constant__ CUtensorMap tmap_ks, const __grid_constant__ CUtensorMap tmap_vs, const KvAttnArgs a) {
    using S = RowsShape<DW, FMT>;
    using namespace ptx;
    constexpr bool kEight = S::kEight, kE4m3 = FMT == FORGE_KV_E4M3;
    constexpr bool kF16 = FMT != FORGE_KV_BF16;
    constexpr int kColS = 0, kColO = 128, kTmemCols = 256;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t load_full[S::kLoads], load_empty[S::kLoads], op_full[S::kBufs], op_empty[S::kBufs], q_ready, s_full[2], p_ready[2], pv_done[2];
    __shared__ uint32_t tmem_slot;
    __shared__ int last_ctas;
    constexpr int kMaxOdd = 2 * kKvMaxTokens;
    __shared__ int odd_keys[kMaxOdd], odd_count;  // halves of rows of V with elements that are not finite numbers, which some of the tokens see
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    uint8_t* sq = smem;
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kLoads; ++i) {
            mbar_init(&load_full[i], 1);
            mbar_init(&load_empty[i], kEight ? 4 : 1);
        }
        for (int i = 0; i < S::kBufs; ++i) {
            mbar_init(&op_full[i], 4);
            mbar_init(&op_empty[i], 1);
        }
        mbar_init(&q_ready, 4);
        for (int i = 0; i < 2; ++i) { mbar_init(&s_full[i], 1); mbar_init(&p_ready[i], 4); mbar_init(&pv_done[i], 1); }
        fence_mbar_init();
        prefetch_tmap(&tmap_k);
        prefetch_tmap(&tmap_v);
        odd_count = 0;
    }
    if (warp == 5) {
        tmem_alloc(&tmem_slot, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();
    pdl_wait();

    const KvSchedule<kRowsStep> sched(a, a.least, lane);
    const KvShares shares(sched.N, sched.W);
    KvCursor cur;
    cur.u = cur.end = 0;
    if ((int)blockIdx.x < sched.W) {
        cur.u = shares.first(blockIdx.x);
        cur.end = shares.first(blockIdx.x + 1);
        sched.at(a, cur.u, cur, lane);
    }
    bool failed = false;

    if (warp == 4) {
        // ------------------------------------------------------------------ copies
        const uint64_t policy = l2_policy_evict_first();
        int n = 0;
        while (cur.u < cur.end && !failed) {
            const KvPart p = kv_part(a, cur);
            const int bk = p.b * a.Hkv + p.kvh;
            for (int t = 0; t < p.tiles; ++t, ++n) {
                const int st = n % S::kLoads, j0 = (p.first + t) * kRowsStep;
                if (n >= S::kLoads && !warp_wait_relaxed(&load_empty[st], (n / S::kLoads - 1) & 1)) { failed = true; break; }
                if (lane == 0) {
                    uint8_t* dst = smem + S::kLoadOff + st * S::kLoadBytes;
                    if (j0 >= p.rows) {  // a sequence without rows
                        mbar_arrive(&load_full[st]);
                    } else if constexpr (kEight) {
                        const int x = (bk * a.Smax + j0) & ~3;
                        mbar_expect_tx(&load_full[st], 2 * S::kRawBytes + 2 * S::kScaleKeys * 4);
                        tma_load_3d_addr_hint(smem_u32(dst), &tmap_k, &load_full[st], 0, j0, bk, policy);
                        tma_load_1d(smem_u32(dst) + 2 * S::kRawBytes, &tmap_ks, &load_full[st], x);
                        tma_load_3d_addr_hint(smem_u32(dst) + S::kRawBytes, &tmap_v, &load_full[st], 0, j0, bk, policy);
                        tma_load_1d(smem_u32(dst) + 2 * S::kRawBytes + S::kScaleBox, &tmap_vs, &load_full[st], x);
                    } else {
                        mbar_expect_tx(&load_full[st], 2 * S::kOpBytes);
#pragma unroll
                        for (int c = 0; c < DW / 64; ++c) {
                            tma_load_3d_addr_hint(smem_u32(dst) + c * S::kOpChunk, &tmap_k, &load_full[st], c * 64, j0, bk, policy);
                            tma_load_3d_addr_hint(smem_u32(dst) + S::kOpBytes + c * S::kOpChunk, &tmap_v, &load_full[st], c * 64, j0, bk, policy);
                        }
                    }
                }
                __syncwarp();
            }
            kv_advance<kRowsStep>(a, cur, p.tiles);
        }
        if (failed)  // copies in flight land before the ring goes away
            for (int i = n > S::kLoads ? n - S::kLoads : 0; i < n; ++i) warp_wait_relaxed(&load_full[i % S::kLoads], (i / S::kLoads) & 1);
    } else if (warp == 5) {
        // ------------------------------------------------------------------ products
        constexpr uint32_t idesc_s = kF16 ? make_idesc_f16(128, kRowsStep, false, false) : make_idesc_bf16(128, kRowsStep, false, false);
        constexpr uint32_t idesc_o = kF16 ? make_idesc_f16(128, DW, false, true) : make_idesc_bf16(128, DW, false, true);
        const uint64_t qd = make_smem_desc(smem_u32(sq), 16, 1024);
        const uint32_t ops = smem_u32(smem + (kEight ? S::kOpOff : S::kLoadOff));
        uint64_t* ready = kEight ? op_full : load_full;
        uint64_t* empty = kEight ? op_empty : load_empty;
        int base = 0, parts = 0, steps[2] = {0, 0};
        while (cur.u < cur.end && !failed) {
            const KvPart p = kv_part(a, cur);
            const int n = p.tiles;
            auto issue_qk = [&](int g) -> bool {
                const int pos = base + g, buf = pos % S::kBufs;
                if (!warp_wait(&ready[buf], (pos / S::kBufs) & 1)) return false;
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint64_t kd = make_smem_desc(ops + buf * 2 * S::kOpBytes, 16, 1024);
#pragma unroll
                    for (int k = 0; k < DW / 16; ++k)
                        mma_ss(tmem + kColS + (g & 1) * kRowsStep, qd + (((k / 4) * S::kQChunk + (k % 4) * 32) >> 4),
                               kd + (((k / 4) * S::kOpChunk + (k % 4) * 32) >> 4), idesc_s, k != 0);
                    mma_commit(&s_full[g & 1]);
                }
                __syncwarp();
                return true;
            };
            if (!warp_wait(&q_ready, parts & 1) || !issue_qk(0) || (n > 1 && !issue_qk(1))) { failed = true; break; }
            for (int g = 0; g < n; ++g) {
                const int h = g & 1, pos = base + g, buf = pos % S::kBufs;
                if (!warp_wait(&p_ready[h], steps[h] & 1)) { failed = true; break; }
                ++steps[h];
                tc_fence_after_sync();
                if (elect_one()) {
                    const uint64_t vd = make_smem_desc(ops + buf * 2 * S::kOpBytes + S::kOpBytes, S::kOpChunk, 1024);
#pragma unroll
                    for (int k = 0; k < kRowsStep / 16; ++k)
                        mma_ts(tmem + kColO, tmem + kColS + h * kRowsStep + k * 8, vd + k * (2048 >> 4), idesc_o, (g | k) != 0);
                    mma_commit(&pv_done[h]);
                    mma_commit(&empty[buf]);
                }
                __syncwarp();
                if (g + 2 < n && !issue_qk(g + 2)) { failed = true; break; }
            }
            base += n;
            ++parts;
            kv_advance<kRowsStep>(a, cur, n);
        }
    } else if (kEight && warp >= 6) {
        // ------------------------------------------------------------------ codes to fp16
        const int t = threadIdx.x - 6 * 32;  // 0 .. 127
        int n = 0;
        while (cur.u < cur.end && !failed) {
            const KvPart p = kv_part(a, cur);
            for (int i = 0; i < p.tiles; ++i, ++n) {
                const int st = n % S::kLoads, buf = n % (S::kOps ? S::kOps : 1), j0 = (p.first + i) * kRowsStep;
                if (!warp_wait(&load_full[st], (n / S::kLoads) & 1)) { failed = true; break; }
                if (n >= S::kOps && !warp_wait(&op_empty[buf], (n / (S::kOps ? S::kOps : 1) - 1) & 1)) { failed = true; break; }
                const uint32_t raw = smem_u32(smem + S::kLoadOff + st * S::kLoadBytes);
                uint8_t* op = smem + S::kOpOff + buf * 2 * S::kOpBytes;
                // a thread's 16-byte pieces of codes: K's, then V's (16 codes become 32 bytes: two pieces of the operand)
                constexpr int kPieces = 2 * S::kRawBytes / 16 / 128, kPerRow = DW / 16;
#pragma unroll
                for (int x = 0; x < kPieces; ++x) {
                    const int at = x * 128 + t, mat = at / (kRowsStep * kPerRow), row = at / kPerRow % kRowsStep, piece = at % kPerRow;
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
                // scales: those of rows that are not there count as zero; the largest of V's
                float* sc = reinterpret_cast<float*>(smem + S::kScaleOff + buf * S::kScaleBytes);
                const float* from = reinterpret_cast<const float*>(smem + S::kLoadOff + st * S::kLoadBytes + 2 * S::kRawBytes) +
                                    (((p.b * a.Hkv + p.kvh) * a.Smax + j0) & 3);
                if (warp == 6 || warp == 7) {
                    const bool is_v = warp == 7;
                    if (is_v) from += S::kScaleBox / 4;
                    const float x0 = j0 + lane < p.rows ? from[lane] : 0.f, x1 = j0 + 32 + lane < p.rows ? from[32 + lane] : 0.f;
                    sc[is_v * kRowsStep + lane] = x0;
                    sc[is_v * kRowsStep + 32 + lane] = x1;
                    float big = fmaxf(x0, x1);
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
                    if (is_v && lane == 0) sc[2 * kRowsStep] = big;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&op_full[buf]);
                    mbar_arrive(&load_empty[st]);
                }
            }
            kv_advance<kRowsStep>(a, cur, p.tiles);
        }
    } else if (warp < 4) {
        // ------------------------------------------------------------------ Q, softmax, O
        const int row = warp * 32 + lane;
        const uint32_t lanes = tmem + (static_cast<uint32_t>(warp * 32) << 16);
        auto rows_sync = [] { asm volatile("bar.sync 1, 128;" ::: "memory"); };
        int base = 0, steps[2] = {0, 0};
        while (cur.u < cur.end) {
            const KvPart p = kv_part(a, cur);
            const int at = p.rt * a.tile_rows + row;                  // row of the KV head
            const bool live = row < a.tile_rows && at < a.rows;
            const bool idle = warp * 32 >= min(a.tile_rows, a.rows - p.rt * a.tile_rows);  // the whole warp has no row
            const int T = max(a.T, 1), h = at / T, tok = at - h * T;
            const int64_t head = p.kvh * a.G + h;
            unsigned long long sees = 0;
            if (live && a.T > 0) sees = a.tree ? a.tree[(int64_t)p.b * a.tree_stride + tok] : (2ull << tok) - 1ull;
            // ---- Q: the previous item's scores are all done (this thread has read them)
            float mul = a.scale_log2;
            {
                const uint16_t* src = static_cast<const uint16_t*>(a.q) + p.b * a.qs.b + head * a.qs.h + tok * a.qs.s;
                uint32_t big = 0;
                uint4 w[DW / 8];
#pragma unroll
                for (int i = 0; i < DW / 8; ++i) {
                    w[i] = live && i * 8 < a.D ? *reinterpret_cast<const uint4*>(src + i * 8) : make_uint4(0, 0, 0, 0);
                    if (kEight) big = __vmaxu2(__vmaxu2(big, __vmaxu2(w[i].x & 0x7fff7fffu, w[i].y & 0x7fff7fffu)), __vmaxu2(w[i].z & 0x7fff7fffu, w[i].w & 0x7fff7fffu));
                }
                float f = 1.f;
                if constexpr (kEight) {  // a power of two that puts the row's largest into [2^14, 2^15): fp16 keeps bf16's bits
                    big = max(big & 0xffffu, big >> 16);
                    const float top = a.q_f16 ? __half2float(__ushort_as_half((unsigned short)big)) : __uint_as_float(big << 16);
                    const int e = (int)(__float_as_uint(top) >> 23) - 127;
                    const int up = top == 0.f || e == 128 ? 0 : min(max(14 - e, -110), 110);
                    f = __int_as_float((127 + up) << 23);
                    mul *= __int_as_float((127 - up) << 23);
                }
#pragma unroll
                for (int i = 0; i < DW / 8; ++i) {
                    uint4 o = w[i];
                    if constexpr (kEight) {
                        const uint32_t in[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
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
                        o = make_uint4(out[0], out[1], out[2], out[3]);
                    }
                    *reinterpret_cast<uint4*>(sq + (i >> 3) * S::kQChunk + sw128(row, i & 7)) = o;
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_ready);

            float m = -INFINITY, l = 0.f;
            float unit = 1.17549435e-38f, unit_inv = 8.5070592e37f;  // 8-bit: power of two that P is divided by, at least V's largest scale so far
            const int n = p.tiles;
#pragma unroll 1
            for (int g = 0; g < n; ++g) {
                const int hb = g & 1, pos = base + g, buf = pos % S::kBufs;
                const int key0 = (p.first + g) * kRowsStep;
                if (!failed && !warp_wait(&s_full[hb], steps[hb] & 1)) failed = true;
                if (failed) break;
                tc_fence_after_sync();
                const bool cut = key0 + kRowsStep > p.past;
                float s[kRowsStep];
                float alpha = 1.f;
                const float* sc = reinterpret_cast<const float*>(smem + S::kScaleOff + buf * S::kScaleBytes);
                unsigned long long vis = ~0ull;
                // the scales, or the rows of V that are looked through below (complete by now: the scores waited for them)
                if ((kEight || cut) && !warp_wait(kEight ? &op_full[buf] : &load_full[buf], (pos / S::kBufs) & 1)) { failed = true; break; }
                if (!idle) {
#pragma unroll
                    for (int c = 0; c < kRowsStep / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld_x32(lanes + kColS + hb * kRowsStep + c * 32, r);
#pragma unroll
                        for (int k = 0; k < 32; ++k) s[c * 32 + k] = __uint_as_float(r[k]);
                    }
                    tmem_ld_wait();
                    if constexpr (kEight) {
#pragma unroll
                        for (int k = 0; k < kRowsStep; k += 4) {
                            const float4 ks = *reinterpret_cast<const float4*>(sc + k);
                            s[k] *= ks.x; s[k + 1] *= ks.y; s[k + 2] *= ks.z; s[k + 3] *= ks.w;
                        }
                    }
#pragma unroll
                    for (int k = 0; k < kRowsStep; ++k) s[k] *= mul;
                    if (cut) {
                        const int d = p.past - key0, have = p.rows - key0;  // the past ends d keys, all rows `have` keys into the step
                        vis = d > 0 ? ((1ull << d) - 1ull) | sees << d : d > -64 ? sees >> -d : 0ull;
                        if (have < 64) vis &= have > 0 ? (1ull << have) - 1ull : 0ull;
#pragma unroll
                        for (int k = 0; k < kRowsStep; ++k) s[k] = vis >> k & 1ull ? s[k] : -INFINITY;
                    }
                    float mx = s[0];
#pragma unroll
                    for (int k = 1; k < kRowsStep; ++k) mx = fmaxf(mx, s[k]);
                    // the reference is raised only where a score passes it by 2^8 (the first of a row always does)
                    if (mx > m + (kRowsTop - kRowsLift)) {
                        alpha = m == -INFINITY ? 1.f : ex2(m - mx);
                        m = mx;
                        l *= alpha;
                    }
                    if constexpr (kEight) {
                        const float big = sc[2 * kRowsStep];
                        if (big > unit) {  // the same in all threads
                            const uint32_t up = min((__float_as_uint(big) + 0x007fffffu) & 0x7f800000u, 0x7e000000u);
                            unit_inv = __uint_as_float(0x7f000000u - up);
                            alpha *= unit * unit_inv;
                            unit = __uint_as_float(up);
                        }
                    }
                }
                if (g > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
                    // O must hold every product so far and none may be in flight
                    if (!warp_wait(&pv_done[hb ^ 1], (steps[hb ^ 1] - 1) & 1)) { failed = true; break; }
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < DW / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld_x32(lanes + kColO + c * 32, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 32; ++k) r[k] = __float_as_uint(__uint_as_float(r[k]) * alpha);
                        tmem_st_x32(lanes + kColO + c * 32, r);
                    }
                }
                ++steps[hb];
                if (!idle) {
                    const float ref = m == -INFINITY ? 0.f : m - kRowsLift;
                    float add = 0.f;
                    uint32_t packed[kRowsStep / 2];
#pragma unroll
                    for (int k = 0; k < kRowsStep; k += 4) {
                        float pr[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            pr[i] = ex2(s[k + i] - ref);
                            add += pr[i];
                        }
                        if constexpr (kEight) {
                            const float4 vs = *reinterpret_cast<const float4*>(sc + kRowsStep + k);
                            pr[0] *= vs.x * unit_inv; pr[1] *= vs.y * unit_inv; pr[2] *= vs.z * unit_inv; pr[3] *= vs.w * unit_inv;
                            if (cut) {  // the scale of a row that is not seen may be anything
#pragma unroll
                                for (int i = 0; i < 4; ++i) pr[i] = vis >> (k + i) & 1ull ? pr[i] : 0.f;
                            }
                        }
                        packed[k / 2] = pack16<kF16>(pr[0], pr[1]);
                        packed[k / 2 + 1] = pack16<kF16>(pr[2], pr[3]);
                    }
                    tmem_st_x32(lanes + kColS + hb * kRowsStep, packed);
                    l += add;
                }
                if constexpr (!kEight) {
                    // What must not reach the product: rows of V past the end, and elements that are not finite numbers in rows that only
                    // some of the tokens see (0 x NaN is NaN); those are remembered and added at the end.
                    if (cut) {
                        constexpr uint32_t kExp = kF16 ? 0x7c00u : 0x7f80u;
                        uint8_t* v = smem + S::kLoadOff + buf * S::kLoadBytes + S::kOpBytes;
                        const int key = row >> 1;  // two threads to a key, a half of its elements each
                        if (key0 + key >= p.past) {
                            const bool out = key0 + key >= p.rows;
                            bool odd = false;
#pragma unroll
                            for (int i = 0; i < DW / 16; ++i) {
                                const int piece = (row & 1) * (DW / 16) + i;
                                uint4* at16 = reinterpret_cast<uint4*>(v + (piece >> 3) * S::kOpChunk + sw128(key, piece & 7));
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
                                const int i = atomicAdd(&odd_count, 1);
                                if (i < kMaxOdd) odd_keys[i] = (key0 + key) * 2 + (row & 1);
                            }
                        }
                        fence_proxy_async_smem();
                    }
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_ready[hb]);
            }
            for (int i = 0; i < 2; ++i)
                if (!failed && steps[i] > 0 && !warp_wait(&pv_done[i], (steps[i] - 1) & 1)) failed = true;
            tc_fence_after_sync();
            base += n;

            // ---- O out, 32 columns at a time; int8: column 4 i + 1 holds element 4 i + 2 and the other way round
            const bool whole = p.tiles == p.of;
            const bool out_f16 = kEight ? a.q_f16 : kF16;
            uint16_t* orow = static_cast<uint16_t*>(a.out) + p.b * a.os.b + head * a.os.h + tok * a.os.s;
            auto write_out = [&](int d, const float (&x)[32], float scale) {  // elements d .. d + 31
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    auto pair = [&](float y, float z) { return out_f16 ? pack16<true>(y * scale, z * scale) : pack16<false>(y * scale, z * scale); };
                    if (d + i * 8 < a.D)
                        *reinterpret_cast<uint4*>(orow + d + i * 8) = make_uint4(pair(x[i * 8], x[i * 8 + 1]), pair(x[i * 8 + 2], x[i * 8 + 3]),
                                                                                 pair(x[i * 8 + 4], x[i * 8 + 5]), pair(x[i * 8 + 6], x[i * 8 + 7]));
                }
            };
            auto slot = [&](int cta) { return a.parts + (size_t)(cta * 2 + (p.start > shares.first(cta) ? 1 : 0)) * S::kPart; };
            rows_sync();  // odd_keys are complete
            const int odds = kEight ? 0 : min(odd_count, kMaxOdd);
            float* mine = slot(blockIdx.x);
            const float norm = kEight ? unit : 1.f;
            if (!idle && !failed) {
#pragma unroll 1
                for (int c = 0; c < DW / 32; ++c) {
                    uint32_t r[32];
                    tmem_ld_x32(lanes + kColO + c * 32, r);
                    tmem_ld_wait();
                    float x[32];
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        const int e = kEight && !kE4m3 ? (k & ~3) | (k & 1) << 1 | (k >> 1 & 1) : k;
                        x[e] = __uint_as_float(r[k]) * norm;
                    }
                    for (int i = 0; i < odds; ++i) {
                        const int key = odd_keys[i] >> 1;
                        if (!(sees >> (key - p.past) & 1ull)) continue;
                        const uint16_t* v = static_cast<const uint16_t*>(a.v) + ((int64_t)(p.b * a.Hkv + p.kvh) * a.Smax + key) * a.D + c * 32;
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            if (c * 32 + k >= a.D || (odd_keys[i] & 1) != (c * 32 + k >= DW / 2)) continue;
                            const float y = kF16 ? __half2float(__ushort_as_half((unsigned short)v[k])) : __uint_as_float((uint32_t)v[k] << 16);
                            if (!(fabsf(y) <= 3.4028235e38f)) x[k] += y;
                        }
                    }
                    if (whole) {
                        if (live) write_out(c * 32, x, l == 0.f ? 0.f : 1.f / l);  // no key seen: zeros
                    } else if (live) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            reinterpret_cast<float4*>(mine)[(c * 8 + k) * 128 + row] = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
                    }
                }
                if (!whole && live) reinterpret_cast<float2*>(mine + 128 * DW)[row] = make_float2(m, l);
            }
            tc_fence_before_sync();
            rows_sync();  // the parts are written, odd_keys have been read
            if (threadIdx.x == 0) odd_count = 0;
            if (!whole) {
                const int cta0 = shares.of(p.start), ctas = shares.of(p.start + p.of - 1) - cta0 + 1;
                if (threadIdx.x == 0) {
                    unsigned int before;
                    asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(before) : "l"(a.counters + p.item) : "memory");
                    last_ctas = before + 1 == (unsigned)ctas ? ctas : 0;
                    if (last_ctas) a.counters[p.item] = 0;  // as the next call expects it
                }
                rows_sync();
                if (last_ctas && live && !failed) {
                    float M = -INFINITY, L = 0.f;
                    for (int i = 0; i < ctas; ++i) M = fmaxf(M, reinterpret_cast<const float2*>(slot(cta0 + i) + 128 * DW)[row].x);
                    const float ref = M == -INFINITY ? 0.f : M;
                    for (int i = 0; i < ctas; ++i) {
                        const float2 ml = reinterpret_cast<const float2*>(slot(cta0 + i) + 128 * DW)[row];
                        L = fmaf(ex2(ml.x - ref), ml.y, L);
                    }
#pragma unroll 1
                    for (int c = 0; c < DW / 32; ++c) {
                        float x[32];
#pragma unroll
                        for (int k = 0; k < 32; ++k) x[k] = 0.f;
#pragma unroll 2
                        for (int i = 0; i < ctas; ++i) {
                            const float* from = slot(cta0 + i);
                            const float w = ex2(reinterpret_cast<const float2*>(from + 128 * DW)[row].x - ref);
#pragma unroll
                            for (int k = 0; k < 8; ++k) {
                                const float4 y = reinterpret_cast<const float4*>(from)[(c * 8 + k) * 128 + row];
                                x[4 * k] = fmaf(w, y.x, x[4 * k]);
                                x[4 * k + 1] = fmaf(w, y.y, x[4 * k + 1]);
                                x[4 * k + 2] = fmaf(w, y.z, x[4 * k + 2]);
                                x[4 * k + 3] = fmaf(w, y.w, x[4 * k + 3]);
                            }
                        }
                        write_out(c * 32, x, L == 0.f ? 0.f : 1.f / L);
                    }
                }
                rows_sync();  // last_ctas has been read
            }
            kv_advance<kRowsStep>(a, cur, n);
        }
    }

    if (failed) {
        if (lane == 0) atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and products in flight end before their memory goes away
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 5) tmem_dealloc(tmem, kTmemCols);
}

template <int DW, int FMT>
int launch_attn_kv_rows(const forge_kv_cache& cache, const KvAttnArgs& a, int ctas, cudaStream_t s) {
    using S = RowsShape<DW, FMT>;
    CUtensorMap tk, tv, tks = {}, tvs = {};
    const uint64_t es = S::kEight ? 1 : 2;
    const uint32_t box[3] = {S::kEight ? (uint32_t)DW : 64u, (uint32_t)kRowsStep, 1};
    const uint64_t dims[3] = {(uint64_t)cache.D, (uint64_t)cache.Smax, (uint64_t)cache.B * cache.Hkv};
    const uint64_t strides[2] = {(uint64_t)cache.D * es, (uint64_t)cache.Smax * cache.D * es};
    const auto encode = !S::kEight ? encode_tmap_bf16_sw128 : DW == 128 ? encode_tmap_u8_sw128 : encode_tmap_u8_sw64;
    if (!encode(&tk, cache.k, 3, dims, strides, box) || !encode(&tv, cache.v, 3, dims, strides, box)) return FORGE_ERR_CUDA;
    if (S::kEight) {
        const uint32_t sbox[1] = {(uint32_t)S::kScaleKeys};
        const uint64_t n[1] = {(uint64_t)cache.B * cache.Hkv * cache.Smax};
        if (!encode_tmap_f32_plain(&tks, cache.k_scale, 1, n, nullptr, sbox) || !encode_tmap_f32_plain(&tvs, cache.v_scale, 1, n, nullptr, sbox))
            return FORGE_ERR_CUDA;
    }
    auto kernel = attn_kv_rows_kernel<DW, FMT>;
    FORGE_SET_SMEM_ONCE(kernel, S::kSmem);
    FORGE_CUDA_TRY(launch_pdl(kernel, dim3(ctas), dim3(S::kThreads), S::kSmem, s, tk, tv, tks, tvs, a));
    return finish_launch(1);
}

}  // namespace
}  // namespace forge
