// Low-rank adapters of many requests beside a shared projection: out = y + s_i (x A_i^T) B_i^T, with i the adapter of the token.
//
// A cluster of eight CTAs has a tile of tokens.  Each CTA contracts an eighth of K for all of them (u = x A^T), the eighths are summed through the CTAs'
// shared memory, and then each CTA makes every eighth piece of the output's columns: one launch, u never in memory, and no workspace.  Both products
// have the adapter as the matrix instructions' 16-row operand and 8 tokens as their columns,
//     u^T(16 ranks x 8 tokens) += A(16 x 16 of K) x^T,     out^T(16 columns x 8 tokens) += B(16 x 16 ranks) u^T,
// so a token alone costs no rows that do not exist, and A and B go from memory to the instructions' registers in 16- and 8-byte loads: the order of a
// contraction's elements is free, and so are the output columns that a tile's rows stand for (8 side by side for a lane, 16 bytes of out).
// Tokens of a tile with one adapter side by side form groups of up to 8.
//   few tokens (tiles up to 8): the warps share the CTA's part of K, and add up through shared memory
//   many: the warps share the groups, and each goes through the CTA's part of K
// u goes into the second product as two 16-bit numbers, the rounded one and what that left, so that out is off by its own rounding alone.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "attn_math.cuh"
#include "forge_common.cuh"
#include "mma_16816.cuh"
#include "sm100_ptx.cuh"
#include "tmap.cuh"

namespace forge {
namespace {

constexpr int kAdCtas = 8;                 // of a cluster
constexpr int kAdWarps = 8, kAdThreads = kAdWarps * 32;
constexpr int kAdMost = 128;               // tokens of a tile
constexpr int kTileTokens = 512;           // from how many tokens on the tensor cores' tiles of 128 are the faster ones (ranks up to 64)

struct AdapterArgs {
    const void *x, *y, *a, *b;
    void* out;
    const float* scales;
    const int32_t *requests, *adapters;
    int64_t xs, ys, os;                    // elements from a token to the next
    int T, R, n, rank, K, N, tile;
    int* status;
};

// RT: tiles of 16 ranks.
template <int RT>
struct AdapterShape {
    static constexpr int kRanks = RT * 16;
    static constexpr int kHalfRow = RT == 1 ? 16 : kRanks + 16;  // elements from a token's u to the next one's: the lanes' reads meet no bank twice
};

__device__ __forceinline__ uint32_t peer_smem(uint32_t addr, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void store_peer(uint32_t addr, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
__device__ __forceinline__ void store_peer(uint32_t addr, uint32_t v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void ad_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void ad_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

template <bool F16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
    if constexpr (F16) return __half22float2(*reinterpret_cast<const __half2*>(&w));
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ uint4 load16(const void* p, bool there) { return there ? *static_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ uint2 load8(const void* p, bool there) { return there ? *static_cast<const uint2*>(p) : make_uint2(0, 0); }

// Tokens first .. first + n - 1 of the tile (n <= 8), which have the same adapter; -1: none.
struct AdGroup { int16_t first, n; int adapter; };

__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int t) {
    int i = t;
    if (a.requests) i = __ldcg(a.requests + t);
    i = (unsigned)i < (unsigned)a.R ? __ldcg(a.adapters + i) : -1;
    return (unsigned)i < (unsigned)a.n ? i : -1;
}

// One warp: the groups of the tile's tokens.  Returns how many.
__device__ __forceinline__ int make_groups(const int* which, int tokens, AdGroup* groups, int lane) {
    int count = 0, run = 0;  // run: where the current one begins
    for (int s = 0; s < tokens; s += 32) {
        const int t = s + lane, w = t < tokens ? which[t] : -2;
        const bool begins = t < tokens && (t == 0 || which[t - 1] != w);
        const unsigned starts = __ballot_sync(0xffffffffu, begins);
        const unsigned before = starts & (0xffffffffu >> (31 - lane));
        const int from = before ? s + 31 - __clz(before) : run;          // of this token's run
        const bool opens = t < tokens && ((t - from) & 7) == 0;
        const unsigned open = __ballot_sync(0xffffffffu, opens);
        if (opens) {
            int end = t + 1;
            while (end < tokens && end < t + 8 && which[end] == w) ++end;
            groups[count + __popc(open & ((1u << lane) - 1u))] = {(int16_t)t, (int16_t)(end - t), w};
        }
        count += __popc(open);
        if (starts) run = s + 31 - __clz(starts);
    }
    return count;
}

// u^T = A x^T over this CTA's part of K, in blocks of 64, into `mine` ([warp][token][rank] for SMALL, [token][rank]).
template <bool F16, int RT, bool SMALL>
__device__ __forceinline__ void shrink_groups(const AdapterArgs& a, const AdGroup* groups, int n_groups, float* mine, int t0, int cta, int warp, int lane) {
    constexpr int kRanks = AdapterShape<RT>::kRanks;
    const int g = lane >> 2, c = lane & 3;
    const int blocks = (a.K + 63) / 64;
    const uint16_t* const xp = static_cast<const uint16_t*>(a.x) + (int64_t)t0 * a.xs;
    for (int gi = SMALL ? 0 : warp; gi < n_groups; gi += SMALL ? 1 : kAdWarps) {
        const AdGroup gr = groups[gi];
        float u[RT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) u[i][k] = 0.f;
        if (gr.adapter >= 0) {
            const uint16_t* const ap = static_cast<const uint16_t*>(a.a) + (int64_t)gr.adapter * a.rank * a.K;
            const uint16_t* const xrow = xp + (gr.first + min(g, gr.n - 1)) * a.xs;
            const int first = SMALL ? cta * kAdWarps + warp : cta, step = SMALL ? kAdCtas * kAdWarps : kAdCtas;
#pragma unroll 1
            for (int blk = first; blk < blocks; blk += step) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {  // 32 of K: lane c has elements 8 c .. 8 c + 7 of them, four for each of two instructions
                    const int k = blk * 64 + h * 32 + 8 * c;
                    const bool in = k < a.K;
                    const uint4 xv = load16(xrow + k, in && g < gr.n);
#pragma unroll
                    for (int i = 0; i < RT; ++i) {
                        const int row = i * 16 + g;
                        const uint4 lo = load16(ap + (int64_t)row * a.K + k, in && row < a.rank);
                        const uint4 hi = load16(ap + (int64_t)(row + 8) * a.K + k, in && row + 8 < a.rank);
                        const uint32_t f0[4] = {lo.x, hi.x, lo.y, hi.y}, f1[4] = {lo.z, hi.z, lo.w, hi.w};
                        mma_16816<F16>(u[i], f0, xv.x, xv.y);
                        mma_16816<F16>(u[i], f1, xv.z, xv.w);
                    }
                }
            }
        }
        // rows g, g + 8 are ranks, columns 2c, 2c + 1 tokens
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1), r = i * 16 + g + 8 * (k >> 1);
                if (t < gr.n) mine[((SMALL ? warp * a.tile : 0) + gr.first + t) * kRanks + r] = u[i][k];
            }
    }
}

// Each CTA's part of u to where it is summed: to the CTA that has the token's eighth of the tile (`per` tokens).
template <int RT>
__device__ __forceinline__ void send_eighths(const float* mine, uint32_t inbox_addr, int tokens, int per, int cta) {
    constexpr int kRanks = AdapterShape<RT>::kRanks;
    for (int e = threadIdx.x; e < tokens * kRanks; e += kAdThreads) {
        const int t = e / kRanks, p = t / per;
        store_peer(peer_smem(inbox_addr + ((cta * per + t - p * per) * kRanks + e % kRanks) * 4, p), mine[e]);
    }
}

// Tokens sum0 .. sum1 - 1 of the tile: the CTAs' parts ([from][per][rank] in `inbox`) summed, scaled and cut into two; a warp for each token, two ranks to a
// lane.  put(t, r, hi, lo): ranks r, r + 1 as two pairs; put_unit(t, unit): out += unit * u B^T (lane 0).
template <bool F16, int RT, typename Put, typename PutUnit>
__device__ __forceinline__ void sum_parts(const AdapterArgs& a, const int* which, const float* inbox, int per, int sum0, int sum1, int warp, int lane,
                                          Put put, PutUnit put_unit) {
    constexpr int kRanks = AdapterShape<RT>::kRanks, kEach = (kRanks + 63) / 64;
    for (int t = sum0 + warp; t < sum1; t += kAdWarps) {
        float2 v[kEach];
        const int i = which[t];
        const float scale = i >= 0 ? a.scales ? a.scales[i] : 1.f : 0.f;
        uint32_t big = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = j * 64 + 2 * lane;
            v[j] = make_float2(0.f, 0.f);
            if (r < a.rank && i >= 0) {  // (a multiple of 8)
#pragma unroll
                for (int p = 0; p < kAdCtas; ++p) {
                    const float2 w = *reinterpret_cast<const float2*>(inbox + (p * per + t - sum0) * kRanks + r);
                    v[j].x += w.x;
                    v[j].y += w.y;
                }
                v[j].x *= scale;
                v[j].y *= scale;
            }
            const uint32_t x = __float_as_uint(v[j].x) & 0x7fffffffu, y = __float_as_uint(v[j].y) & 0x7fffffffu;
            if (x < 0x7f800000u) big = max(big, x);
            if (y < 0x7f800000u) big = max(big, y);
        }
        // fp16: the token's largest that is finite goes to [2^14, 2^15)
        float up = 1.f;
        if constexpr (F16) {
            big = __reduce_max_sync(0xffffffffu, big);
            const int e = (int)(big >> 23) - 127;
            if (big != 0) up = __int_as_float((127 + min(max(14 - e, -113), 110)) << 23);
        }
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = j * 64 + 2 * lane;
            if (r >= kRanks) continue;
            const float2 x = make_float2(v[j].x * up, v[j].y * up);
            const uint32_t hi = pack16<F16>(x.x, x.y);
            const float2 h = unpack16<F16>(hi), rest = make_float2(x.x - h.x, x.y - h.y);
            put(t, r, hi, pack16<F16>(isfinite(rest.x) ? rest.x : 0.f, isfinite(rest.y) ? rest.y : 0.f));
        }
        if (lane == 0) put_unit(t, __fdiv_rn(1.f, up));  // a power of two
    }
}

// out^T = y^T + unit B u^T, 64 columns at a time: lane (g, c) has columns 8 g .. 8 g + 7 of tokens 2c, 2c + 1.  Row g (+ 8) of tile i of
// the instructions' 16 is column 8 g + 2 i (+ 1).
template <bool F16, int RT>
__device__ __forceinline__ void expand_groups(const AdapterArgs& a, const AdGroup* groups, int n_groups, const uint16_t* u_hi, const uint16_t* u_lo,
                                              const float* unit, int t0, int cta, int warp, int lane) {
    constexpr int kRow = AdapterShape<RT>::kHalfRow;
    const int g = lane >> 2, c = lane & 3;
    const int units = (a.N + 63) / 64;
    for (int un = cta * kAdWarps + warp; un < units; un += kAdCtas * kAdWarps) {
        const int col = un * 64 + 8 * g;
        const bool in = col < a.N;
        uint2 bf[RT][4][2];
        int have = -1;
        for (int gi = 0; gi < n_groups; ++gi) {
            const AdGroup gr = groups[gi];
            const int ta = gr.first + 2 * c, tb = ta + 1;
            const bool has_a = in && 2 * c < gr.n, has_b = in && 2 * c + 1 < gr.n;
            const uint4 ya = load16(static_cast<const uint16_t*>(a.y) + (int64_t)(t0 + ta) * a.ys + col, has_a);
            const uint4 yb = load16(static_cast<const uint16_t*>(a.y) + (int64_t)(t0 + tb) * a.ys + col, has_b);
            uint4 oa = ya, ob = yb;
            if (gr.adapter >= 0) {
                if (gr.adapter != have) {
                    have = gr.adapter;
                    const uint16_t* const bp = static_cast<const uint16_t*>(a.b) + ((int64_t)have * a.N + col) * a.rank;
#pragma unroll
                    for (int s = 0; s < RT; ++s)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) bf[s][i][h] = load8(bp + (2 * i + h) * a.rank + 16 * s + 4 * c, in && 16 * s + 4 * c < a.rank);
                }
                float acc[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
                const int row = (gr.first + min(g, gr.n - 1)) * kRow + 4 * c;
#pragma unroll
                for (int s = 0; s < RT; ++s) {
                    const uint2 hi = *reinterpret_cast<const uint2*>(u_hi + row + 16 * s), lo = *reinterpret_cast<const uint2*>(u_lo + row + 16 * s);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t f[4] = {bf[s][i][0].x, bf[s][i][1].x, bf[s][i][0].y, bf[s][i][1].y};
                        mma_16816<F16>(acc[i], f, hi.x, hi.y);
                        mma_16816<F16>(acc[i], f, lo.x, lo.y);
                    }
                }
                const float ua = has_a ? unit[ta] : 0.f, ub = has_b ? unit[tb] : 0.f;
                const uint32_t wa[4] = {ya.x, ya.y, ya.z, ya.w}, wb[4] = {yb.x, yb.y, yb.z, yb.w};
                uint32_t ra[4], rb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // columns 2 i, 2 i + 1 of the lane's 8
                    const float2 fa = unpack16<F16>(wa[i]), fb = unpack16<F16>(wb[i]);
                    ra[i] = pack16<F16>(fmaf(acc[i][0], ua, fa.x), fmaf(acc[i][2], ua, fa.y));
                    rb[i] = pack16<F16>(fmaf(acc[i][1], ub, fb.x), fmaf(acc[i][3], ub, fb.y));
                }
                oa = make_uint4(ra[0], ra[1], ra[2], ra[3]);
                ob = make_uint4(rb[0], rb[1], rb[2], rb[3]);
            }
            if (has_a) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + (int64_t)(t0 + ta) * a.os + col) = oa;
            if (has_b) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + (int64_t)(t0 + tb) * a.os + col) = ob;
        }
    }
}

template <bool F16, int RT, bool SMALL>
__global__ void __launch_bounds__(kAdThreads) adapters_kernel(const AdapterArgs a) {
    using S = AdapterShape<RT>;
    constexpr int kRanks = S::kRanks, kRow = S::kHalfRow;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ AdGroup groups[kAdMost];
    __shared__ int which[kAdMost];
    __shared__ float unit[kAdMost];  // out += unit * (u in shared memory) B^T
    __shared__ int n_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x % kAdCtas;
    const int t0 = (int)(blockIdx.x / kAdCtas) * a.tile, tokens = min(a.tile, a.T - t0);
    // shared memory: what the warps (SMALL) or the CTA have of u, what the CTAs send, u
    const int own = SMALL ? kAdWarps * a.tile : a.tile, sent = SMALL ? kAdCtas * a.tile : a.tile;  // rows of kRanks floats
    float* mine = reinterpret_cast<float*>(smem);
    float* inbox = mine + own * kRanks;
    uint16_t* u_hi = reinterpret_cast<uint16_t*>(inbox + sent * kRanks);
    uint16_t* u_lo = u_hi + a.tile * kRow;
    ad_arrive();  // waited for before the first store into another CTA's shared memory
    pdl_launch_dependents();
    pdl_wait();
    for (int t = threadIdx.x; t < tokens; t += kAdThreads) which[t] = adapter_of(a, t0 + t);
    __syncthreads();
    if (warp == 0) {
        const int n = make_groups(which, tokens, groups, lane);
        if (lane == 0) n_groups = n;
    }
    __syncthreads();
    shrink_groups<F16, RT, SMALL>(a, groups, n_groups, mine, t0, cta, warp, lane);
    __syncthreads();
    ad_wait();  // all CTAs of the cluster run

    const uint32_t inbox_addr = ptx::smem_u32(inbox), hi_addr = ptx::smem_u32(u_hi), lo_addr = ptx::smem_u32(u_lo), unit_addr = ptx::smem_u32(unit);
    if constexpr (SMALL) {  // every CTA sums all of it
        for (int e = threadIdx.x; e < tokens * kRanks; e += kAdThreads) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kAdWarps; ++w) s += mine[w * a.tile * kRanks + e];
#pragma unroll
            for (int p = 0; p < kAdCtas; ++p) store_peer(peer_smem(inbox_addr + (cta * a.tile * kRanks + e) * 4, p), s);
        }
        ad_arrive();
        ad_wait();
        sum_parts<F16, RT>(a, which, inbox, a.tile, 0, tokens, warp, lane,
                           [&](int t, int r, uint32_t hi, uint32_t lo) {
                               *reinterpret_cast<uint32_t*>(u_hi + t * kRow + r) = hi;
                               *reinterpret_cast<uint32_t*>(u_lo + t * kRow + r) = lo;
                           },
                           [&](int t, float x) { unit[t] = x; });
        __syncthreads();
    } else {  // each its eighth of the tokens
        const int per = a.tile / kAdCtas;
        send_eighths<RT>(mine, inbox_addr, tokens, per, cta);
        ad_arrive();
        ad_wait();
        sum_parts<F16, RT>(a, which, inbox, per, cta * per, min(cta * per + per, tokens), warp, lane,
                           [&](int t, int r, uint32_t hi, uint32_t lo) {
#pragma unroll
                               for (int p = 0; p < kAdCtas; ++p) {
                                   store_peer(peer_smem(hi_addr + (t * kRow + r) * 2, p), hi);
                                   store_peer(peer_smem(lo_addr + (t * kRow + r) * 2, p), lo);
                               }
                           },
                           [&](int t, float x) {
#pragma unroll
                               for (int p = 0; p < kAdCtas; ++p) store_peer(peer_smem(unit_addr + t * 4, p), x);
                           });
        ad_arrive();
        ad_wait();
    }
    expand_groups<F16, RT>(a, groups, n_groups, u_hi, u_lo, unit, t0, cta, warp, lane);
}

// ------------------------------------------------------------------------------------------------- tiles of up to 128 tokens on the tensor cores
// Many tokens: a tile's tokens are the 128 rows of a tcgen05 tile.  Contraction: u[128 x ranks] = x A_i^T for each adapter i that the tile has, x and
// A through a ring filled by TMA; a row takes its own adapter's u.  Output: D[128 x 128 columns] = [u, what rounding left] [B_i, B_i]^T, and the row
// of y, which lies in shared memory, gets its own adapter's D added there and leaves by TMA.  A tile of more than kTileAdapters adapters, each of
// which takes a pass over the tile, goes by groups of 8 tokens like small ones.
constexpr int kTileAdapters = 4;
constexpr int kTileCols = 128;

template <int RT>
struct TileShape {
    static constexpr int kRanks = RT * 16;
    static constexpr int kOp = (2 * kRanks + 63) / 64 * 16384;   // u and its rest: [128 rows x 64] chunks
    static constexpr int kStage = 16384 + kRanks * 128;          // x's and A's 64 of K
    static constexpr int kY = 3, kB = 3;                         // buffers of y (and out), of B
    static constexpr int kYBytes = 2 * 16384, kBBytes = kTileCols * 128;
    static constexpr int kRing = kY * kYBytes + kB * kBBytes;    // the contraction's stages before that
    static constexpr int kStages = kRing / kStage < 8 ? kRing / kStage : 8;
    static constexpr int kInboxOff = kOp, kRingOff = kInboxOff + 128 * kRanks * 4;
    static constexpr int kSmem = 1024 + kRingOff + kRing;
    // by groups: what the CTA has of u, then u, in the ring's place
    static_assert(128 * kRanks * 4 + 128 * AdapterShape<RT>::kHalfRow * 4 <= kRing && kRingOff % 1024 == 0 && kStage % 1024 == 0, "shared memory");
    static_assert(kSmem <= 232448 - 6144, "shared memory");
};

template <bool F16, int RT>
__global__ void __launch_bounds__(kAdThreads, 1)
adapters_tile_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_a, const __grid_constant__ CUtensorMap tmap_y,
                     const __grid_constant__ CUtensorMap tmap_b, const __grid_constant__ CUtensorMap tmap_out, const AdapterArgs a) {
    using S = TileShape<RT>;
    using namespace ptx;
    constexpr int kRanks = S::kRanks, kRow = AdapterShape<RT>::kHalfRow;
    extern __shared__ uint8_t smem_raw[];
    __shared__ AdGroup groups[kAdMost];
    __shared__ int which[kAdMost], several[kTileAdapters];
    __shared__ float unit[kAdMost];
    __shared__ int n_groups, n_several;
    __shared__ uint64_t x_full[S::kStages], x_free[S::kStages], u_done, y_full[S::kY], y_free[S::kY], b_full[S::kB], b_free[S::kB], d_full[2], d_free[2];
    __shared__ uint32_t tmem_slot;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x % kAdCtas;
    const int t0 = (int)(blockIdx.x / kAdCtas) * a.tile, tokens = min(a.tile, a.T - t0), per = a.tile / kAdCtas;
    uint8_t* smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    uint8_t* ring = smem + S::kRingOff;
    float* inbox = reinterpret_cast<float*>(smem + S::kInboxOff);
    ad_arrive();  // waited for before the first store into another CTA's shared memory
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) { mbar_init(&x_full[i], 1); mbar_init(&x_free[i], 1); }
        mbar_init(&u_done, 1);
        for (int i = 0; i < S::kY; ++i) { mbar_init(&y_full[i], 1); mbar_init(&y_free[i], 1); }
        for (int i = 0; i < S::kB; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_free[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_free[i], 4); }
        fence_mbar_init();
        prefetch_tmap(&tmap_x);
        prefetch_tmap(&tmap_a);
        prefetch_tmap(&tmap_y);
        prefetch_tmap(&tmap_b);
        prefetch_tmap(&tmap_out);
        n_several = 0;
    }
    if (warp == 2) {
        tmem_alloc(&tmem_slot, 256);
        tmem_relinquish();
    }
    pdl_launch_dependents();
    pdl_wait();
    for (int t = threadIdx.x; t < tokens; t += kAdThreads) which[t] = adapter_of(a, t0 + t);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    // ---- the adapters that the tile has, in the order of their first tokens
    if (warp == 0) {
        int n = 0;
        for (int s = 0; s < tokens; s += 32) {
            const int t = s + lane, w = t < tokens ? which[t] : -1;
            unsigned starts = __ballot_sync(0xffffffffu, w >= 0 && (t == 0 || which[t - 1] != w));
            for (; starts && n <= kTileAdapters; starts &= starts - 1) {
                const int x = __shfl_sync(0xffffffffu, w, __ffs(starts) - 1);
                bool had = false;
                for (int i = 0; i < n && i < kTileAdapters; ++i) had |= several[i] == x;
                if (had) continue;
                if (lane == 0 && n < kTileAdapters) several[n] = x;
                ++n;
                __syncwarp();
            }
        }
        if (lane == 0) n_several = n;
    } else if (warp == 1) {
        const int n = make_groups(which, tokens, groups, lane);
        if (lane == 0) n_groups = n;
    }
    __syncthreads();
    const int adapters = n_several;
    const bool tiled = adapters > 0 && adapters <= kTileAdapters;
    bool failed = false;
    const uint32_t inbox_addr = smem_u32(inbox), op_addr = smem_u32(smem), unit_addr = smem_u32(unit);
    float* mine = reinterpret_cast<float*>(ring);                                              // (by groups)
    uint16_t* u_hi = reinterpret_cast<uint16_t*>(ring + 128 * kRanks * 4);
    uint16_t* u_lo = u_hi + 128 * kRow;

    // ---- the contraction
    const int blocks = (a.K + 63) / 64, my_blocks = cta < blocks ? (blocks - cta + kAdCtas - 1) / kAdCtas : 0;
    if (!tiled) {
        shrink_groups<F16, RT, false>(a, groups, n_groups, mine, t0, cta, warp, lane);
        __syncthreads();
        ad_wait();
        send_eighths<RT>(mine, inbox_addr, tokens, per, cta);
    } else {
        if (warp == 0 && elect_one()) {
            int n = 0;
            for (int j = 0; j < adapters && !failed; ++j)
                for (int i = 0; i < my_blocks; ++i, ++n) {
                    const int st = n % S::kStages, k = (cta + i * kAdCtas) * 64;
                    if (n >= S::kStages && !mbar_wait(&x_free[st], (n / S::kStages - 1) & 1)) { failed = true; break; }
                    mbar_expect_tx(&x_full[st], a.tile * 128 + kRanks * 128);
                    tma_load_2d(ring + st * S::kStage, &tmap_x, &x_full[st], k, t0);
                    tma_load_2d(ring + st * S::kStage + 16384, &tmap_a, &x_full[st], k, several[j] * a.rank);
                }
        } else if (warp == 1 && elect_one()) {
            constexpr uint32_t idesc = F16 ? make_idesc_f16(128, kRanks, false, false) : make_idesc_bf16(128, kRanks, false, false);
            int n = 0;
            for (int j = 0; j < adapters && !failed; ++j)
                for (int i = 0; i < my_blocks; ++i, ++n) {
                    const int st = n % S::kStages;
                    if (!mbar_wait(&x_full[st], (n / S::kStages) & 1)) { failed = true; break; }
                    tc_fence_after_sync();
                    const uint64_t xd = make_smem_desc(smem_u32(ring + st * S::kStage), 16, 1024), ad = make_smem_desc(smem_u32(ring + st * S::kStage + 16384), 16, 1024);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_ss(tmem + j * kRanks, xd + (k * 32 >> 4), ad + (k * 32 >> 4), idesc, i > 0 || k > 0);
                    mma_commit(&x_free[st]);
                }
            if (my_blocks == 0) mbar_arrive(&u_done);
            else if (!failed) mma_commit(&u_done);
        }
        __syncwarp();
        ad_wait();  // all CTAs of the cluster run
        if (warp >= 4) {  // thread = row: the columns of its own adapter, to the CTA that sums its token
            const int row = threadIdx.x & 127, own = row < tokens ? which[row] : -1;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
            if (!warp_wait(&u_done, 0)) failed = true;
            tc_fence_after_sync();
            const int p = row / per;
            const uint32_t to = own >= 0 ? peer_smem(inbox_addr + (cta * per + row - p * per) * kRanks * 4, p) : 0;
            for (int j = 0; j < adapters && !failed; ++j) {
                const bool hit = own == several[j];
                if (!__any_sync(0xffffffffu, hit)) continue;
#pragma unroll
                for (int r = 0; r < kRanks; r += 16) {
                    uint32_t x[16];
                    __syncwarp();
                    tmem_ld_x16(lanes + j * kRanks + r, x);
                    tmem_ld_wait();
#pragma unroll
                    for (int k = 0; k < 16; k += 4)
                        if (hit) st_cluster_v4(to + (r + k) * 4, my_blocks ? x[k] : 0u, my_blocks ? x[k + 1] : 0u, my_blocks ? x[k + 2] : 0u, my_blocks ? x[k + 3] : 0u);
                }
            }
            tc_fence_before_sync();
        }
        __syncwarp();
    }
    ad_arrive();
    ad_wait();
    tc_fence_after_sync();

    // ---- u, to all CTAs
    sum_parts<F16, RT>(a, which, inbox, per, cta * per, min(cta * per + per, tokens), warp, lane,
                       [&](int t, int r, uint32_t hi, uint32_t lo) {
                           uint32_t to_hi, to_lo;
                           if (tiled) {  // elements r and kRanks + r of row t, in chunks of 64 with 128-byte swizzle
                               auto at = [&](int e) { return op_addr + (e >> 6) * 16384 + t * 128 + ((((e & 63) >> 3) ^ (t & 7)) << 4) + (e & 7) * 2; };
                               to_hi = at(r);
                               to_lo = at(kRanks + r);
                           } else {
                               to_hi = smem_u32(u_hi + t * kRow + r);
                               to_lo = smem_u32(u_lo + t * kRow + r);
                           }
#pragma unroll
                           for (int p = 0; p < kAdCtas; ++p) {
                               store_peer(peer_smem(to_hi, p), hi);
                               store_peer(peer_smem(to_lo, p), lo);
                           }
                       },
                       [&](int t, float x) {
#pragma unroll
                           for (int p = 0; p < kAdCtas; ++p) store_peer(peer_smem(unit_addr + t * 4, p), x);
                       });
    asm volatile("fence.proxy.async;" ::: "memory");  // the tensor cores read what plain stores wrote
    __syncwarp();
    ad_arrive();
    ad_wait();
    asm volatile("fence.proxy.async;" ::: "memory");

    // ---- the output
    if (!tiled) {
        expand_groups<F16, RT>(a, groups, n_groups, u_hi, u_lo, unit, t0, cta, warp, lane);
    } else {
        const int chunks = (a.N + kTileCols - 1) / kTileCols;
        uint8_t* b_ring = ring + S::kY * S::kYBytes;
        if (warp == 0 && elect_one()) {
            int n = 0, m = 0;  // chunks; chunks and adapters
            for (int q = cta; q < chunks && !failed; q += kAdCtas, ++n) {
                const int yb = n % S::kY;
                if (n >= S::kY && !mbar_wait(&y_free[yb], (n / S::kY - 1) & 1)) { failed = true; break; }
                mbar_expect_tx(&y_full[yb], 2 * a.tile * 128);
                tma_load_2d(ring + yb * S::kYBytes, &tmap_y, &y_full[yb], q * kTileCols, t0);
                tma_load_2d(ring + yb * S::kYBytes + 16384, &tmap_y, &y_full[yb], q * kTileCols + 64, t0);
                for (int j = 0; j < adapters; ++j, ++m) {
                    const int bb = m % S::kB;
                    if (m >= S::kB && !mbar_wait(&b_free[bb], (m / S::kB - 1) & 1)) { failed = true; break; }
                    mbar_expect_tx(&b_full[bb], S::kBBytes);
                    tma_load_2d(b_ring + bb * S::kBBytes, &tmap_b, &b_full[bb], 0, several[j] * a.N + q * kTileCols);
                }
            }
        } else if (warp == 1 && elect_one()) {
            constexpr uint32_t idesc = F16 ? make_idesc_f16(128, kTileCols, false, false) : make_idesc_bf16(128, kTileCols, false, false);
            const uint64_t ud = make_smem_desc(op_addr, 16, 1024);
            int m = 0;
            for (int q = cta; q < chunks && !failed; q += kAdCtas)
                for (int j = 0; j < adapters; ++j, ++m) {
                    const int bb = m % S::kB, db = m & 1;
                    if (!mbar_wait(&b_full[bb], (m / S::kB) & 1)) { failed = true; break; }
                    if (m >= 2 && !mbar_wait(&d_free[db], (m / 2 - 1) & 1)) { failed = true; break; }
                    tc_fence_after_sync();
                    const uint64_t bd = make_smem_desc(smem_u32(b_ring + bb * S::kBBytes), 16, 1024);
#pragma unroll
                    for (int e = 0; e < 2 * kRanks; e += 16)  // u's ranks, then what rounding left of them, with the same columns of B
                        mma_ss(tmem + db * kTileCols, ud + (((e >> 6) * 16384 + (e & 63) * 2) >> 4), bd + ((e % kRanks) * 2 >> 4), idesc, e > 0);
                    mma_commit(&b_free[bb]);
                    mma_commit(&d_full[db]);
                }
        } else if (warp >= 4) {
            const int row = threadIdx.x & 127, own = row < tokens ? which[row] : -1;
            const float mul = own >= 0 ? unit[row] : 0.f;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
            int n = 0, m = 0;
            for (int q = cta; q < chunks; q += kAdCtas, ++n) {
                const int yb = n % S::kY;
                uint8_t* y = ring + yb * S::kYBytes + row * 128;
                if (!failed && !warp_wait(&y_full[yb], (n / S::kY) & 1)) failed = true;
                for (int j = 0; j < adapters; ++j, ++m) {
                    const int db = m & 1;
                    if (!failed && !warp_wait(&d_full[db], (m / 2) & 1)) failed = true;
                    const bool hit = own == several[j];
                    if (!failed && __any_sync(0xffffffffu, hit)) {
                        tc_fence_after_sync();
#pragma unroll
                        for (int h = 0; h < kTileCols / 32; ++h) {
                            uint32_t d[32];
                            __syncwarp();
                            tmem_ld_x32(lanes + db * kTileCols + h * 32, d);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                if (!hit) break;
                                uint4* at = reinterpret_cast<uint4*>(y + (h >> 1) * 16384 + ((((h & 1) * 4 + i) ^ (row & 7)) << 4));
                                const uint4 w = *at;
                                const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                                uint32_t out[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const float2 f = unpack16<F16>(in[k]);
                                    out[k] = pack16<F16>(fmaf(__uint_as_float(d[i * 8 + 2 * k]), mul, f.x), fmaf(__uint_as_float(d[i * 8 + 2 * k + 1]), mul, f.y));
                                }
                                *at = make_uint4(out[0], out[1], out[2], out[3]);
                            }
                        }
                        tc_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&d_free[db]);
                }
                fence_proxy_async_smem();
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (threadIdx.x == 128 && !failed) {
                    tma_store_2d(&tmap_out, ring + yb * S::kYBytes, q * kTileCols, t0);
                    if (q * kTileCols + 64 < a.N) tma_store_2d(&tmap_out, ring + yb * S::kYBytes + 16384, q * kTileCols + 64, t0);
                    tma_store_commit();
                    if (n > 0) {
                        tma_store_wait_read<1>();  // all but this one
                        mbar_arrive(&y_free[(n - 1) % S::kY]);
                    }
                }
            }
            if (threadIdx.x == 128) tma_store_wait_all<0>();
        }
        __syncwarp();
    }
    if (failed) {
        atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and products in flight end before their memory goes away
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, 256);
}

// How many clusters of the tile kernel the GPU holds at a time (once per device).
template <typename Kernel>
int resident_clusters(Kernel kernel, int smem) {
    static int known[64] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    if (known[dev] == 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kAdCtas * 32);
        cfg.blockDim = dim3(kAdThreads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kAdCtas;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) {
            cudaGetLastError();
            n = 0;
        }
        known[dev] = n > 0 ? n : sm_count() / kAdCtas;
    }
    return known[dev];
}

template <bool F16, int RT>
int launch_adapters_tiles(AdapterArgs a, cudaStream_t s) {
    using S = TileShape<RT>;
    auto kernel = adapters_tile_kernel<F16, RT>;
    FORGE_SET_SMEM_ONCE(kernel, S::kSmem);
    const int clusters = resident_clusters(kernel, S::kSmem);
    if (clusters <= 0) return FORGE_ERR_CUDA;
    // as many turns of all the clusters that run at a time as tiles of 128 take, in even tiles
    const long long turns = (a.T + 128LL * clusters - 1) / (128LL * clusters);
    const long long want = (a.T + turns * clusters - 1) / (turns * clusters);
    a.tile = (int)((want + 7) / 8 * 8);
    CUtensorMap tx, ta, ty, tb, to;
    auto rows = [&](CUtensorMap* m, const void* p, int64_t width, int64_t n, int64_t stride, int box_rows) {
        const uint64_t dims[2] = {(uint64_t)width, (uint64_t)n}, strides[1] = {(uint64_t)stride * 2};
        const uint32_t box[2] = {64, (uint32_t)box_rows};
        return encode_tmap_bf16_sw128(m, p, 2, dims, strides, box);
    };
    if (!rows(&tx, a.x, a.K, a.T, a.xs, a.tile) || !rows(&ta, a.a, a.K, (int64_t)a.n * a.rank, a.K, S::kRanks) ||
        !rows(&ty, a.y, a.N, a.T, a.ys, a.tile) || !rows(&tb, a.b, a.rank, (int64_t)a.n * a.N, a.rank, kTileCols) ||
        !rows(&to, a.out, a.N, a.T, a.os, a.tile))
        return FORGE_ERR_CUDA;
    const long long tiles = ((long long)a.T + a.tile - 1) / a.tile;
    FORGE_CUDA_TRY(launch_pdl_cluster(kernel, dim3((unsigned)(tiles * kAdCtas)), dim3(kAdThreads), S::kSmem, kAdCtas, s, tx, ta, ty, tb, to, a));
    return finish_launch(1);
}

template <bool F16, int RT, bool SMALL>
int launch_adapters(const AdapterArgs& a, cudaStream_t s) {
    using Sh = AdapterShape<RT>;
    const int own = SMALL ? kAdWarps * a.tile : a.tile, sent = SMALL ? kAdCtas * a.tile : a.tile;
    const size_t smem = (size_t)(own + sent) * Sh::kRanks * 4 + (size_t)a.tile * Sh::kHalfRow * 4;
    auto kernel = adapters_kernel<F16, RT, SMALL>;
    FORGE_SET_SMEM_ONCE(kernel, 200 * 1024);
    const long long tiles = ((long long)a.T + a.tile - 1) / a.tile;
    FORGE_CUDA_TRY(launch_pdl_cluster(kernel, dim3((unsigned)(tiles * kAdCtas)), dim3(kAdThreads), smem, kAdCtas, s, a));
    return finish_launch(1);
}
template <bool F16, int RT>
int launch_adapters(const AdapterArgs& a, cudaStream_t s) {
    if constexpr (RT <= 4)
        if (a.T >= kTileTokens && (long long)a.n * a.N < (1LL << 31)) return launch_adapters_tiles<F16, RT>(a, s);
    return a.tile <= 8 ? launch_adapters<F16, RT, true>(a, s) : launch_adapters<F16, RT, false>(a, s);
}
template <bool F16>
int launch_adapters(const AdapterArgs& a, cudaStream_t s) {
    return a.rank <= 16   ? launch_adapters<F16, 1>(a, s)
           : a.rank <= 32 ? launch_adapters<F16, 2>(a, s)
           : a.rank <= 64 ? launch_adapters<F16, 4>(a, s)
                          : launch_adapters<F16, 8>(a, s);
}

}  // namespace
}  // namespace forge

extern "C" int forge_linear_adapters(const forge_adapters* set, const void* x, const void* y, void* out, int T, int64_t x_stride,
                                     int64_t y_stride, int64_t out_stride, const int32_t* requests, const int32_t* adapters, int R,
                                     void* stream) {
    using namespace forge;
    if (!set || !set->a || !set->b || !x || !y || !out || !adapters || T <= 0 || R <= 0) return FORGE_ERR_INVALID_ARG;
    if (set->n <= 0 || set->rank <= 0 || set->K <= 0 || set->N <= 0 || x_stride < 0 || y_stride < 0 || out_stride < 0) return FORGE_ERR_INVALID_ARG;
    if (!aligned16(set->a) || !aligned16(set->b) || !aligned16(x) || !aligned16(y) || !aligned16(out)) return FORGE_ERR_INVALID_ARG;
    auto odd4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; };
    if (odd4(set->scales) || odd4(requests) || odd4(adapters) || (!requests && R != T)) return FORGE_ERR_INVALID_ARG;
    if (set->dtype != FORGE_DTYPE_BF16 && set->dtype != FORGE_DTYPE_F16) return set->dtype == FORGE_DTYPE_F32 ? FORGE_ERR_UNSUPPORTED : FORGE_ERR_INVALID_ARG;
    AdapterArgs a = {};
    a.xs = x_stride ? x_stride : set->K;
    a.ys = y_stride ? y_stride : set->N;
    a.os = out_stride ? out_stride : set->N;
    if (a.xs < set->K || a.ys < set->N || a.os < set->N) return FORGE_ERR_INVALID_ARG;
    if (y == out && a.ys != a.os) return FORGE_ERR_INVALID_ARG;
    if (set->K % 8 != 0 || set->N % 8 != 0 || set->rank % 8 != 0 || set->rank > 128) return FORGE_ERR_UNSUPPORTED;
    if (a.xs % 8 != 0 || a.ys % 8 != 0 || a.os % 8 != 0) return FORGE_ERR_UNSUPPORTED;
    a.x = x; a.y = y; a.out = out;
    a.a = set->a; a.b = set->b;
    a.scales = set->scales;
    a.requests = requests;
    a.adapters = adapters;
    a.T = T; a.R = R;
    a.n = set->n; a.rank = set->rank; a.K = set->K; a.N = set->N;
    // A tile's tokens: so many that the clusters fill the GPU about twice over; from 16 on the warps share the tokens, by eights.
    const int sms = sm_count();
    a.status = device_status_word();
    if (sms <= 0 || !a.status) return FORGE_ERR_CUDA;
    const int want = (T + sms / 4 - 1) / (sms / 4);
    a.tile = want <= 8 ? want : want <= 16 ? 16 : want <= 32 ? 32 : want <= 64 ? 64 : 128;
    if (a.rank > 64 && a.tile > 64) a.tile = 64;
    if ((long long)T / a.tile >= (1LL << 28)) return FORGE_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return set->dtype == FORGE_DTYPE_F16 ? launch_adapters<true>(a, s) : launch_adapters<false>(a, s);
}
