// Low-rank adapters of many requests beside a shared projection: out = y + s_i (x A_i^T) B_i^T, with i the adapter of the token.
//
// Few tokens: a cluster of eight CTAs has a tile of up to 16 of them.  Each CTA contracts an eighth of K for all of them (u = x A^T), the eighths are summed through the CTAs'
// shared memory, and then each CTA makes every eighth piece of the output's columns: one launch, u never in memory, and no workspace.  Both products
// have the adapter as the matrix instructions' 16-row operand and 8 tokens as their columns,
//     u^T(16 ranks x 8 tokens) += A(16 x 16 of K) x^T,     out^T(16 columns x 8 tokens) += B(16 x 16 ranks) u^T,
// so a token alone costs no rows that do not exist, and A and B go from memory to the instructions' registers in 16- and 8-byte loads: the order of a
// contraction's elements is free, and so are the output columns that a tile's rows stand for (8 side by side for a lane, 16 bytes of out).
// A tile's tokens of one adapter form groups of up to 8.
//   tiles up to 8 tokens: the warps share the CTA's part of K, and add up through shared memory
//   16: the warps share the groups, and each goes through the CTA's part of K
// u goes into the second product as two 16-bit numbers, the rounded one and what that left, so that out is off by its own rounding alone (rounding it
// once would add as much again where the adapter's part is as large as y).
// Bound by a chain of dependent steps (the tokens' adapters, A and B, the exchange, the columns) and by L2, which all read at once: 48 requests of 40
// adapters, 4096 x 4096, 16 ranks (10 MB), 7.1 us in a chain of calls; 13 tokens, 768 x 2304, 8 ranks, 4.6.
//
// Many tokens: see below.
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
constexpr int kAdMost = 16;                // tokens of a tile of the kernel for few of them
// From how many tokens on tiles of 128 on the tensor cores: when more than 32 tiles of 16 are too many to run at a time (which adapters the tokens have is not
// known on the host).  That favours long runs of one adapter and many ranks; short runs of few adapters pay for a pass over the tile for each of them.  Groups and
// tiles, us, 4096 x 4096:
//   16 ranks: one adapter, 512 tokens 10 and 14, 600 19 and 15, 2000 39 and 18; runs of 100 of 8 adapters 11 and 19, 18 and 19, 40 and 25; runs of 16 of 8 adapters
//     10 and 32, 18 and 35, 39 and 47; 8 adapters in turns 21 and 34, 33 and 38, 69 and 50; 40 in turns 29 and 41, 50 and 47, 110 and 68
//   64 ranks: one adapter 15 and 17, 27 and 16, 57 and 21; runs of 16 of 8 adapters 15 and 50, 26 and 55, 57 and 69; 40 in turns 87 and 109, 125 and 111, 281 and 189
//   128 ranks (tiles are the faster ones from 200 tokens on where runs are long): one adapter 48 and 18, 49 and 20, 146 and 28; 40 in turns 224 and 229, 228 and 261, 677 and 439
constexpr int kTileTokens = 513;

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
// Packed zeros while no element of the pairs so far was infinite or no number.
template <bool F16>
__device__ __forceinline__ uint32_t odd_pairs(uint32_t w, uint32_t so_far) {
    uint32_t r;
    if constexpr (F16) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w), "r"(0u), "r"(so_far));
    else asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(w), "r"(0u), "r"(so_far));
    return r;
}
__device__ __forceinline__ bool is_odd(uint32_t pairs) { return (pairs & 0x7fff7fffu) != 0; }
// A pair with what is no number, and what is infinite, taken as 0.
template <bool F16>
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
    constexpr uint32_t kTop = F16 ? 0x7c00u : 0x7f80u;
    return ((w & kTop) == kTop ? 0u : w & 0xffffu) | ((w >> 16 & kTop) == kTop ? 0u : w & 0xffff0000u);
}
__device__ __forceinline__ uint4 load16(const void* p, bool there) { return there ? *static_cast<const uint4*>(p) : make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ uint2 load8(const void* p, bool there) { return there ? *static_cast<const uint2*>(p) : make_uint2(0, 0); }

// n tokens of the tile (up to 8) which have the same adapter (-1: none).
struct AdGroup { uint8_t token[8]; int n, adapter; };

__device__ __forceinline__ int adapter_of(const AdapterArgs& a, int t) {
    int i = t;
    if (a.requests) i = __ldcg(a.requests + t);
    i = (unsigned)i < (unsigned)a.R ? __ldcg(a.adapters + i) : -1;
    return (unsigned)i < (unsigned)a.n ? i : -1;
}

// The CTA's first 128 threads: the groups of the tile's tokens (up to 128), those of one adapter side by side, adapters in the order of their first tokens;
// the same in every CTA.  `base`: room for 128.  Needs a barrier behind it.
__device__ __forceinline__ void make_groups(const int* which, int tokens, AdGroup* groups, int* n_groups, int* base) {
    if (threadIdx.x >= (tokens <= 32 ? 32 : 128)) return;
    const int t = threadIdx.x, lane = t & 31, mine = t < tokens ? which[t] : -2;
    if (tokens <= 32) {  // one warp
        const unsigned same = __match_any_sync(0xffffffffu, mine);
        const int total = __popc(same), before = __popc(same & ((1u << lane) - 1u)), first = __ffs(same) - 1;
        const int n = t < tokens && first == t ? (total + 7) / 8 : 0;
        int sum = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        const int at = __shfl_sync(0xffffffffu, sum - n, first);
        if (lane == 31) *n_groups = sum;
        if (t < tokens) {
            AdGroup& g = groups[at + before / 8];
            g.token[before & 7] = (uint8_t)t;
            if ((before & 7) == 0) {
                g.n = min(8, total - before);
                g.adapter = mine;
            }
        }
        return;
    }
    int total = 0, before = 0, first = t;  // tokens of this one's adapter; those before it; the first of them
    for (int s = tokens - 1; s >= 0; --s) {
        if (which[s] != mine) continue;
        ++total;
        before += s < t;
        first = s;
    }
    // where each adapter's groups begin: a sum over its first token and those before
    int n = t < tokens && first == t ? (total + 7) / 8 : 0, sum = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += v;
    }
    base[t] = sum;
    asm volatile("bar.sync 3, 128;" ::: "memory");
    int at = sum - n, all = 0;
    for (int w = 0; w < 4; ++w) {
        const int part = base[w * 32 + 31];
        if (w < (t >> 5)) at += part;
        all += part;
    }
    asm volatile("bar.sync 3, 128;" ::: "memory");
    base[t] = at;
    if (t == 0) *n_groups = all;
    asm volatile("bar.sync 3, 128;" ::: "memory");
    if (t < tokens) {
        AdGroup& g = groups[base[first] + before / 8];
        g.token[before & 7] = (uint8_t)t;
        if ((before & 7) == 0) {
            g.n = min(8, total - before);
            g.adapter = mine;
        }
    }
}

// A group's 64 elements of K: its tokens' x and its adapter's A, as the instructions take them (32 at a time: lane c has elements 8 c .. 8 c + 7 of
// them, four for each of two instructions).
template <int RT>
struct AdBlock {
    uint4 x[2], lo[RT][2], hi[RT][2];
    __device__ __forceinline__ void load(const AdapterArgs& a, const AdGroup& gr, const uint16_t* xp, int blk, int lane) {
        const int g = lane >> 2, c = lane & 3;
        const uint16_t* const ap = static_cast<const uint16_t*>(a.a) + (int64_t)max(gr.adapter, 0) * a.rank * a.K;
        const uint16_t* const xrow = xp + gr.token[min(g, gr.n - 1)] * a.xs;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = blk * 64 + h * 32 + 8 * c;
            const bool in = k < a.K && gr.adapter >= 0;
            x[h] = load16(xrow + k, in && g < gr.n);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const int row = i * 16 + g;
                lo[i][h] = load16(ap + (int64_t)row * a.K + k, in && row < a.rank);
                hi[i][h] = load16(ap + (int64_t)(row + 8) * a.K + k, in && row + 8 < a.rank);
            }
        }
    }
};

// u^T = A x^T over this CTA's part of K, in blocks of 64, into `mine` ([warp][token][rank] for SMALL, [token][rank]).  Up to 32 ranks the next
// block, which may be the next group's, is on its way while one is worked on, in two sets of registers in turns.
template <bool F16, int RT, bool SMALL, int CTAS>
__device__ __forceinline__ void shrink_groups(const AdapterArgs& a, const AdGroup* groups, int n_groups, float* mine, int t0, int cta, int warp, int lane) {
    constexpr int kRanks = AdapterShape<RT>::kRanks;
    const int g = lane >> 2, c = lane & 3;
    const int blocks = (a.K + 63) / 64;
    const uint16_t* const xp = static_cast<const uint16_t*>(a.x) + (int64_t)t0 * a.xs;
    const int first = SMALL ? cta * kAdWarps + warp : cta, step = SMALL ? CTAS * kAdWarps : CTAS;
    const int g_step = SMALL ? 1 : kAdWarps;
    float u[RT][4];
    auto clear = [&]() {
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) u[i][k] = 0.f;
    };
    auto add = [&](const AdBlock<RT>& b) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const uint32_t f0[4] = {b.lo[i][h].x, b.hi[i][h].x, b.lo[i][h].y, b.hi[i][h].y};
                const uint32_t f1[4] = {b.lo[i][h].z, b.hi[i][h].z, b.lo[i][h].w, b.hi[i][h].w};
                mma_16816<F16>(u[i], f0, b.x[h].x, b.x[h].y);
                mma_16816<F16>(u[i], f1, b.x[h].z, b.x[h].w);
            }
    };
    auto put = [&](const AdGroup& gr) {  // rows g, g + 8 are ranks, columns 2c, 2c + 1 tokens
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = 2 * c + (k & 1), r = i * 16 + g + 8 * (k >> 1);
                if (t < gr.n) mine[((SMALL ? warp * a.tile : 0) + gr.token[t]) * kRanks + r] = u[i][k];
            }
    };
    clear();
    if (first >= blocks) {  // no part of K
        for (int gi = SMALL ? 0 : warp; gi < n_groups; gi += g_step) put(groups[gi]);
        return;
    }
    struct At { int gi, blk; } at = {SMALL ? 0 : warp, first}, next = at;
    auto step_on = [&](At& x) {
        x.blk += step;
        if (x.blk >= blocks) {
            x.blk = first;
            x.gi += g_step;
        }
    };
    if constexpr (RT <= 2) {
        AdBlock<RT> even, odd;
        auto load = [&](AdBlock<RT>& b) {
            if (next.gi < n_groups) b.load(a, groups[next.gi], xp, next.blk, lane);
            step_on(next);
        };
        auto use = [&](const AdBlock<RT>& b) {
            add(b);
            if (at.blk + step >= blocks) {
                put(groups[at.gi]);
                clear();
            }
            step_on(at);
        };
        load(even);
        while (at.gi < n_groups) {
            load(odd);
            use(even);
            if (at.gi >= n_groups) break;
            load(even);
            use(odd);
        }
    } else {
        for (; at.gi < n_groups; step_on(at)) {
            AdBlock<RT> b;
            b.load(a, groups[at.gi], xp, at.blk, lane);
            add(b);
            if (at.blk + step >= blocks) {
                put(groups[at.gi]);
                clear();
            }
        }
    }
}

// Each CTA's part of u to where it is summed: to the CTA that has the token's share of the tile (`per` tokens).
template <int RT>
__device__ __forceinline__ void send_parts(const float* mine, uint32_t inbox_addr, int tokens, int per, int cta) {
    constexpr int kRanks = AdapterShape<RT>::kRanks;
    for (int e = threadIdx.x; e < tokens * kRanks; e += kAdThreads) {
        const int t = e / kRanks, p = t / per;
        store_peer(peer_smem(inbox_addr + ((cta * per + t - p * per) * kRanks + e % kRanks) * 4, p), mine[e]);
    }
}

// Tokens sum0 .. sum1 - 1 of the tile: the CTAs' parts ([from][per][rank] in `inbox`) summed, scaled and cut into two; a warp for each token, two ranks to a
// lane.  put(t, r, hi, lo): ranks r, r + 1 as two pairs; put_unit(t, unit): out += unit * u B^T (lane 0).
template <bool F16, int RT, int CTAS, typename Put, typename PutUnit>
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
                for (int p = 0; p < CTAS; ++p) {
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

// A group's part of the output's 64 columns from `col0` on: B's rows as the instructions take them, and y.  Lane (g, c) has columns 8 g .. 8 g + 7 of the
// group's tokens 2c, 2c + 1; row g (+ 8) of tile i of the instructions' 16 is column 8 g + 2 i (+ 1).
template <int RT>
using AdRows = uint2[RT][4][2];
template <int RT>
__device__ __forceinline__ void load_b(AdRows<RT>& b, const AdapterArgs& a, int adapter, int col0, int lane) {
    const int c = lane & 3, col = col0 + 8 * (lane >> 2);
    const uint16_t* const bp = static_cast<const uint16_t*>(a.b) + ((int64_t)max(adapter, 0) * a.N + col) * a.rank;
#pragma unroll
    for (int s = 0; s < RT; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) b[s][i][h] = load8(bp + (2 * i + h) * a.rank + 16 * s + 4 * c, adapter >= 0 && col < a.N && 16 * s + 4 * c < a.rank);
}
template <int RT>
struct AdColumns {
    AdRows<RT> b;
    uint4 ya, yb;
    __device__ __forceinline__ void load_y(const AdapterArgs& a, const AdGroup& gr, bool there, int t0, int col0, int lane) {
        const int c = lane & 3, col = col0 + 8 * (lane >> 2);
        const uint16_t* const yp = static_cast<const uint16_t*>(a.y) + (int64_t)t0 * a.ys + col;
        there = there && col < a.N;
        ya = load16(yp + gr.token[2 * c] * a.ys, there && 2 * c < gr.n);
        yb = load16(yp + gr.token[2 * c + 1] * a.ys, there && 2 * c + 1 < gr.n);
    }
};

// Which pieces of 64 columns and which groups a warp has: pieces `first` .. end - 1 are shared by kAdWarps * `of` warps, of which this is number `warp`; with
// fewer pieces than warps several have the same one, each some of the groups.
struct AdShare {
    int piece, step, g0, g1;
    __device__ __forceinline__ AdShare(int first, int end, int n_groups, int warp, int of) {
        const int warps = kAdWarps * of, parts = max(warps / max(end - first, 1), 1), part = warp % parts;
        piece = first + warp / parts;
        step = warps / parts;
        g0 = n_groups * part / parts;
        g1 = n_groups * (part + 1) / parts;
    }
};

// The same products anew where what comes out is not all finite (see expand_groups), B from memory once more, where up to 32 ranks leave it in no register.
template <bool F16, int RT>
__device__ __forceinline__ void multiply_finite_rests(float (&acc)[4][4], const AdapterArgs& a, int adapter, int col, const uint16_t* u_hi,
                                                      const uint16_t* u_lo, int c) {
    const uint16_t* const bp = static_cast<const uint16_t*>(a.b) + ((int64_t)adapter * a.N + col) * a.rank;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
#pragma unroll 1
    for (int r = 0; r < RT * 16; r += 16) {
        const uint2 hi = *reinterpret_cast<const uint2*>(u_hi + r), lo = *reinterpret_cast<const uint2*>(u_lo + r);
        const bool there = col < a.N && r + 4 * c < a.rank;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 b0 = load8(bp + 2 * i * a.rank + r + 4 * c, there), b1 = load8(bp + (2 * i + 1) * a.rank + r + 4 * c, there);
            const uint32_t f[4] = {b0.x, b1.x, b0.y, b1.y};
            const uint32_t f_rest[4] = {finite_pair<F16>(f[0]), finite_pair<F16>(f[1]), finite_pair<F16>(f[2]), finite_pair<F16>(f[3])};
            mma_16816<F16>(acc[i], f, hi.x, hi.y);
            mma_16816<F16>(acc[i], f_rest, lo.x, lo.y);
        }
    }
}

// out^T = y^T + unit B u^T.  An infinite element of B is multiplied by the rounded u alone: with what rounding left it would come to an infinity of the
// other sign, or to no number, and so would the sum.  Where the products (up to 32 ranks: the outputs, once they have left) turn out not to be finite, they are made
// anew in that way; looking costs nothing that can be measured here.
// `even`: the first piece's first group, if EARLY.  Up to 32 ranks the next group's y and B are on their way while one is worked
// on, in two sets of registers in turns; more ranks have one set, and B is kept while the adapter stays.
template <bool F16, int RT, bool EARLY>
__device__ __forceinline__ void expand_groups(const AdapterArgs& a, const AdGroup* groups, const uint16_t* u_hi, const uint16_t* u_lo, const float* unit,
                                              int t0, const AdShare& share, int end, AdColumns<RT>& even, int lane) {
    constexpr int kRow = AdapterShape<RT>::kHalfRow;
    const int g = lane >> 2, c = lane & 3;
    uint16_t* const op = static_cast<uint16_t*>(a.out) + (int64_t)t0 * a.os;
    if (share.g0 >= share.g1) return;
    auto use = [&](const AdColumns<RT>& at, const AdGroup& gr, int col0) {
        const int col = col0 + 8 * g, ta = gr.token[2 * c], tb = gr.token[2 * c + 1];
        const bool has_a = col < a.N && 2 * c < gr.n, has_b = col < a.N && 2 * c + 1 < gr.n;
        uint4 oa = at.ya, ob = at.yb;
        auto put = [&]() {
            if (has_a) *reinterpret_cast<uint4*>(op + ta * a.os + col) = oa;
            if (has_b) *reinterpret_cast<uint4*>(op + tb * a.os + col) = ob;
        };
        if (gr.adapter >= 0) {
            float acc[4][4];
            const int row = gr.token[min(g, gr.n - 1)] * kRow + 4 * c;
            auto multiply = [&](auto rest) {  // rest: what a pair of B is for what rounding left of u
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
#pragma unroll
                for (int s = 0; s < RT; ++s) {
                    const uint2 hi = *reinterpret_cast<const uint2*>(u_hi + row + 16 * s), lo = *reinterpret_cast<const uint2*>(u_lo + row + 16 * s);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t f[4] = {at.b[s][i][0].x, at.b[s][i][1].x, at.b[s][i][0].y, at.b[s][i][1].y};
                        const uint32_t f_rest[4] = {rest(f[0]), rest(f[1]), rest(f[2]), rest(f[3])};
                        mma_16816<F16>(acc[i], f, hi.x, hi.y);
                        mma_16816<F16>(acc[i], f_rest, lo.x, lo.y);
                    }
                }
            };
            multiply([](uint32_t w) { return w; });
            const float ua = has_a ? unit[ta] : 0.f, ub = has_b ? unit[tb] : 0.f;
            auto add = [&]() {
                const uint32_t wa[4] = {at.ya.x, at.ya.y, at.ya.z, at.ya.w}, wb[4] = {at.yb.x, at.yb.y, at.yb.z, at.yb.w};
                uint32_t ra[4], rb[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // columns 2 i, 2 i + 1 of the lane's 8
                    const float2 fa = unpack16<F16>(wa[i]), fb = unpack16<F16>(wb[i]);
                    ra[i] = pack16<F16>(fmaf(acc[i][0], ua, fa.x), fmaf(acc[i][2], ua, fa.y));
                    rb[i] = pack16<F16>(fmaf(acc[i][1], ub, fb.x), fmaf(acc[i][3], ub, fb.y));
                }
                oa = make_uint4(ra[0], ra[1], ra[2], ra[3]);
                ob = make_uint4(rb[0], rb[1], rb[2], rb[3]);
            };
            if constexpr (RT > 2) {
                float2 odd[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 none = make_float2(0.f, 0.f);
                    odd[i] = ffma2(make_float2(acc[i][0], acc[i][1]), none, ffma2(make_float2(acc[i][2], acc[i][3]), none, none));
                }
                const float2 any = fadd2(fadd2(odd[0], odd[1]), fadd2(odd[2], odd[3]));
                if (__builtin_expect(__any_sync(0xffffffffu, any.x + any.y != 0.f), 0)) multiply([](uint32_t w) { return finite_pair<F16>(w); });
                add();
                put();
            } else {
                add();
                put();
                const uint32_t odd = odd_pairs<F16>(oa.w, odd_pairs<F16>(oa.z, odd_pairs<F16>(oa.y, odd_pairs<F16>(oa.x, 0u)))) |
                                     odd_pairs<F16>(ob.w, odd_pairs<F16>(ob.z, odd_pairs<F16>(ob.y, odd_pairs<F16>(ob.x, 0u))));
                if (__builtin_expect(__any_sync(0xffffffffu, is_odd(odd)), 0)) {
                    multiply_finite_rests<F16, RT>(acc, a, gr.adapter, col, u_hi + row, u_lo + row, c);
                    add();
                    put();
                }
            }
        } else {
            put();
        }
    };
    struct At { int un, gi; } at = {share.piece, share.g0}, next = at;
    auto step_on = [&](At& x) {
        if (++x.gi >= share.g1) {
            x.gi = share.g0;
            x.un += share.step;
        }
    };
    if constexpr (RT <= 2) {
        AdColumns<RT> odd;
        auto load = [&](AdColumns<RT>& to) {
            if (next.un < end) {
                load_b<RT>(to.b, a, groups[next.gi].adapter, next.un * 64, lane);
                to.load_y(a, groups[next.gi], true, t0, next.un * 64, lane);
            }
            step_on(next);
        };
        if (EARLY) step_on(next);
        else load(even);
        while (at.un < end) {
            load(odd);
            use(even, groups[at.gi], at.un * 64);
            step_on(at);
            if (at.un >= end) break;
            load(even);
            use(odd, groups[at.gi], at.un * 64);
            step_on(at);
        }
    } else {
        int have_un = -1, have = -1;
        for (; at.un < end; step_on(at)) {
            const AdGroup& gr = groups[at.gi];
            even.load_y(a, gr, true, t0, at.un * 64, lane);
            if (at.un != have_un || gr.adapter != have) load_b<RT>(even.b, a, gr.adapter, at.un * 64, lane);
            have_un = at.un;
            have = gr.adapter;
            use(even, gr, at.un * 64);
        }
    }
}

// SMALL: up to 8 tokens to a tile; else 16.
template <bool F16, int RT, bool SMALL>
__global__ void __launch_bounds__(kAdThreads, RT <= 4 ? 2 : 1) adapters_kernel(const AdapterArgs a) {
    using S = AdapterShape<RT>;
    constexpr int kRanks = S::kRanks, kRow = S::kHalfRow;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ AdGroup groups[kAdMost];
    __shared__ int which[kAdMost], base[kAdMost];
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
    make_groups(which, tokens, groups, &n_groups, base);
    __syncthreads();
    // of the output's first columns, B and y are asked for now: they need not wait for u
    constexpr bool kEarly = RT <= 2;
    const int pieces = (a.N + 63) / 64;
    const AdShare share(0, pieces, n_groups, warp * kAdCtas + cta, kAdCtas);
    AdColumns<RT> columns;
    if (kEarly && share.piece < pieces && share.g0 < share.g1) {
        load_b<RT>(columns.b, a, groups[share.g0].adapter, share.piece * 64, lane);
        columns.load_y(a, groups[share.g0], true, t0, share.piece * 64, lane);
    }
    shrink_groups<F16, RT, SMALL, kAdCtas>(a, groups, n_groups, mine, t0, cta, warp, lane);
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
        sum_parts<F16, RT, kAdCtas>(a, which, inbox, a.tile, 0, tokens, warp, lane,
                           [&](int t, int r, uint32_t hi, uint32_t lo) {
                               *reinterpret_cast<uint32_t*>(u_hi + t * kRow + r) = hi;
                               *reinterpret_cast<uint32_t*>(u_lo + t * kRow + r) = lo;
                           },
                           [&](int t, float x) { unit[t] = x; });
        __syncthreads();
    } else {  // each its eighth of the tokens
        const int per = a.tile / kAdCtas;
        send_parts<RT>(mine, inbox_addr, tokens, per, cta);
        ad_arrive();
        ad_wait();
        sum_parts<F16, RT, kAdCtas>(a, which, inbox, per, cta * per, min(cta * per + per, tokens), warp, lane,
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
    expand_groups<F16, RT, kEarly>(a, groups, u_hi, u_lo, unit, t0, share, pieces, columns, lane);
}

// ------------------------------------------------------------------------------------------------- tiles of 128 tokens on the tensor cores
// Many tokens: 128 of them are the rows of a tcgen05 tile, and each product is a kernel of its own with u in the workspace between them, so that the second
// one, which moves most of the bytes, shares them out evenly over all SMs.
//   u[128 x ranks] = x A_i^T for each adapter i that the tile has, a cluster of eight CTAs to a tile; a row takes its own adapter's
//   D[128 x 128 columns] = [u, what rounding left] [B_i, B_i]^T; the rows of y, which lie in shared memory, get their own adapter's D added there and
//     leave by TMA
// What bounds them: the second kernel HBM where tiles have one adapter (4000 tokens, 4096 x 14336, 64 ranks, 229 MB of y and out: 45 us, 5.1 TB/s), else its passes
// and how evenly they are shared out (9 requests of 5 adapters: 49 to 57 us, by where the requests begin); the first one its fixed steps and the copies (33 MB of x: 17 us); both together 62 and 74 to 78 us.
// A tile of more than tile_adapters() adapters, each of which takes a pass over the tile, goes by groups of 8 tokens like small ones.
constexpr int kTileRows = 128, kTileCols = 128;
constexpr int tile_adapters(int ranks) { return ranks <= 32 ? 8 : 4; }  // their u lie side by side in tensor memory, of two CTAs to an SM
constexpr int kListInts = 16;  // of a tile: how many adapters it has (one more than tile_adapters: more than that), and which

inline int padded_ranks(int rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }
// The workspace: adapters and units of the tokens, the tiles' lists, u.
struct TileWorkspace {
    size_t unit, list, u, bytes;
    TileWorkspace(long long T, int ranks) {
        auto up = [](long long n) { return ((size_t)n + 255) / 256 * 256; };
        unit = up(T * 4);
        list = unit + up(T * 4);
        u = list + up((T + kTileRows - 1) / kTileRows * kListInts * 4);
        bytes = u + (size_t)T * ranks * 4;
    }
};
struct TileArgs {
    AdapterArgs a;
    int *which, *list;
    float* unit;
    uint32_t* u;  // [token][ranks], then what rounding left of them, in pairs
};

// DEEP: one CTA to an SM.
template <int RT, bool DEEP>
struct ContractShape {
    static constexpr int kRanks = RT * 16;
    static constexpr int kABytes = kRanks * 128;                 // an adapter's 64 of K
    static constexpr int kX = DEEP ? 7 : RT == 4 ? 3 : 4, kA = RT == 4 && !DEEP ? 3 : 4;  // buffers of x's 64 of K and of A's
    static constexpr int kAOff = kX * 16384, kInboxOff = kAOff + kA * kABytes;
    static constexpr int kSmem = 1024 + kInboxOff + kTileRows * kRanks * 4;
    static constexpr int kAdapters = tile_adapters(kRanks), kTmemCols = kAdapters * kRanks;
    static_assert(kTileRows * kRanks * 4 <= kInboxOff && kInboxOff % 1024 == 0, "by groups: what the CTA has of u, in the rings' place");
    static_assert(kSmem <= 232448 - 4096 && (RT == 8 || DEEP || 2 * (kSmem + 4096) <= 232448), "shared memory");
};

// CTAS: of a cluster, which share K.
template <bool F16, int RT, int CTAS, bool DEEP>
__global__ void __launch_bounds__(kAdThreads, RT == 8 || DEEP ? 1 : 2)
adapters_contract_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_a, const TileArgs ta) {
    using S = ContractShape<RT, DEEP>;
    using namespace ptx;
    constexpr int kRanks = S::kRanks, kPer = kTileRows / CTAS;
    extern __shared__ uint8_t smem_raw[];
    __shared__ AdGroup groups[kTileRows];
    __shared__ int which[kTileRows], base[kTileRows], several[S::kAdapters];
    __shared__ int n_groups, n_several;
    __shared__ uint64_t x_full[S::kX], x_free[S::kX], a_full[S::kA], a_free[S::kA], u_done;
    __shared__ uint32_t tmem_slot;
    const AdapterArgs& a = ta.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x % CTAS, tile = blockIdx.x / CTAS;
    const int t0 = tile * kTileRows, tokens = min(kTileRows, a.T - t0);
    uint8_t* ring = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    float* inbox = reinterpret_cast<float*>(ring + S::kInboxOff);
    ad_arrive();  // waited for before the first store into another CTA's shared memory
    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kX; ++i) { mbar_init(&x_full[i], 1); mbar_init(&x_free[i], 1); }
        for (int i = 0; i < S::kA; ++i) { mbar_init(&a_full[i], 1); mbar_init(&a_free[i], 1); }
        mbar_init(&u_done, 1);
        fence_mbar_init();
        prefetch_tmap(&tmap_x);
        prefetch_tmap(&tmap_a);
    }
    if (warp == 2) {
        tmem_alloc(&tmem_slot, S::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();  // the columns are allocated before another kernel may come to this SM and take some
    tc_fence_after_sync();
    pdl_launch_dependents();
    pdl_wait();
    const int blocks = (a.K + 63) / 64, my_blocks = cta < blocks ? (blocks - cta + CTAS - 1) / CTAS : 0;
    const int early = min(my_blocks, S::kX);
    if (warp == 3 && elect_one()) {  // the first of x, whatever adapters it will meet
        for (int i = 0; i < early; ++i) {
            mbar_expect_tx(&x_full[i], 16384);
            tma_load_2d(ring + i * 16384, &tmap_x, &x_full[i], (cta + i * CTAS) * 64, t0);
        }
    }
    __syncwarp();
    // ---- the adapters that the tile has, in the order of their first tokens
    if (warp == 0) {
        int mine[kTileRows / 32], n = 0;
#pragma unroll
        for (int k = 0; k < kTileRows / 32; ++k) {
            const int t = k * 32 + lane;
            mine[k] = t < tokens ? adapter_of(a, t0 + t) : -1;
        }
#pragma unroll
        for (int k = 0; k < kTileRows / 32; ++k)
            if (k * 32 + lane < tokens) which[k * 32 + lane] = mine[k];
#pragma unroll
        for (int k = 0; k < kTileRows / 32; ++k) {
            for (unsigned left; n <= S::kAdapters && (left = __ballot_sync(0xffffffffu, mine[k] >= 0)) != 0;) {
                const int x = __shfl_sync(0xffffffffu, mine[k], __ffs(left) - 1);
                if (lane == 0 && n < S::kAdapters) several[n] = x;
                ++n;
#pragma unroll
                for (int l = 0; l < kTileRows / 32; ++l)
                    if (mine[l] == x) mine[l] = -1;
            }
        }
        __syncwarp();
        if (lane == 0) n_several = n;
        if (cta == 0) {
            if (lane == 0) ta.list[tile * kListInts] = n;
            if (lane < min(n, S::kAdapters)) ta.list[tile * kListInts + 1 + lane] = several[lane];
        }
    }
    __syncthreads();
    const uint32_t tmem = tmem_slot;
    const int adapters = n_several;
    const bool tiled = adapters <= S::kAdapters;
    bool failed = false;
    const uint32_t inbox_addr = smem_u32(inbox);
    if (!tiled || adapters == 0) {  // what has come of x is not wanted
        if (threadIdx.x == 0)
            for (int i = 0; i < early && !failed; ++i) failed = !mbar_wait(&x_full[i], 0);
        __syncthreads();
    }
    if (!tiled) {
        make_groups(which, tokens, groups, &n_groups, base);
        __syncthreads();
        float* mine = reinterpret_cast<float*>(ring);
        shrink_groups<F16, RT, false, CTAS>(a, groups, n_groups, mine, t0, cta, warp, lane);
        __syncthreads();
        ad_wait();
        send_parts<RT>(mine, inbox_addr, tokens, kPer, cta);
    } else {
        if (warp == 0 && elect_one()) {
            int n = 0;  // A's
            for (int i = 0; i < (adapters > 0 ? my_blocks : 0) && !failed; ++i) {
                const int xb = i % S::kX, k = (cta + i * CTAS) * 64;
                if (i >= early) {
                    if (!mbar_wait(&x_free[xb], (i / S::kX - 1) & 1)) { failed = true; break; }
                    mbar_expect_tx(&x_full[xb], 16384);
                    tma_load_2d(ring + xb * 16384, &tmap_x, &x_full[xb], k, t0);
                }
                for (int j = 0; j < adapters; ++j, ++n) {
                    const int ab = n % S::kA;
                    if (n >= S::kA && !mbar_wait(&a_free[ab], (n / S::kA - 1) & 1)) { failed = true; break; }
                    mbar_expect_tx(&a_full[ab], S::kABytes);
                    tma_load_2d(ring + S::kAOff + ab * S::kABytes, &tmap_a, &a_full[ab], k, several[j] * a.rank);
                }
            }
        } else if (warp == 1 && elect_one()) {
            constexpr uint32_t idesc = F16 ? make_idesc_f16(128, kRanks, false, false) : make_idesc_bf16(128, kRanks, false, false);
            int n = 0;
            for (int i = 0; i < (adapters > 0 ? my_blocks : 0) && !failed; ++i) {
                const int xb = i % S::kX;
                if (!mbar_wait(&x_full[xb], (i / S::kX) & 1)) { failed = true; break; }
                const uint64_t xd = make_smem_desc(smem_u32(ring + xb * 16384), 16, 1024);
                for (int j = 0; j < adapters; ++j, ++n) {
                    const int ab = n % S::kA;
                    if (!mbar_wait(&a_full[ab], (n / S::kA) & 1)) { failed = true; break; }
                    tc_fence_after_sync();
                    const uint64_t ad = make_smem_desc(smem_u32(ring + S::kAOff + ab * S::kABytes), 16, 1024);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma_ss(tmem + j * kRanks, xd + (k * 32 >> 4), ad + (k * 32 >> 4), idesc, i > 0 || k > 0);
                    mma_commit(&a_free[ab]);
                }
                mma_commit(&x_free[xb]);
            }
            if (n == 0) mbar_arrive(&u_done);
            else if (!failed) mma_commit(&u_done);
        }
        __syncwarp();
        ad_wait();  // all CTAs of the cluster run
        if (warp >= 4) {  // thread = row: the columns of its own adapter, to the CTA that sums its token
            const int row = threadIdx.x & 127, own = row < tokens ? which[row] : -1;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
            if (!warp_wait(&u_done, 0)) failed = true;
            tc_fence_after_sync();
            const int p = row / kPer;
            const uint32_t to = peer_smem(inbox_addr + (cta * kPer + row - p * kPer) * kRanks * 4, p);
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

    sum_parts<F16, RT, CTAS>(a, which, inbox, kPer, cta * kPer, min(cta * kPer + kPer, tokens), warp, lane,
                       [&](int t, int r, uint32_t hi, uint32_t lo) {
                           uint32_t* to = ta.u + (int64_t)(t0 + t) * kRanks + r / 2;
                           to[0] = hi;
                           to[kRanks / 2] = lo;
                       },
                       [&](int t, float x) {
                           ta.unit[t0 + t] = x;
                           ta.which[t0 + t] = which[t];
                       });
    if (failed) {
        atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and products in flight end before their memory goes away
    }
    __syncthreads();
    if (warp == 2) tmem_dealloc(tmem, S::kTmemCols);
}

// What a chunk of a tile's columns takes, in quarters of one with one adapter: each further adapter costs a product, its B and a pass of the warps whose rows
// have it; by groups it depends on how many tokens a group has.  Measured with 37 tiles of 14336 columns, all with the same number of adapters in turns, K of 64 (so that the first
// kernel is next to nothing), 16 / 64 ranks: one 66 / 68 us, two 75 / 78, three 93 / 98, four 115 / 121, eight 195 by passes (16 ranks); by groups nine 189 / 247, twelve 232 / 308,
// twenty 206 / 304, forty 355 / 523: 4, 4.5, 5.6, 7 and 11.8 quarters, and 11.5 to 31.
__device__ __forceinline__ int chunk_cost(int adapters, int most) { return adapters > most ? 20 : 3 + max(adapters, 1); }

template <int RT>
struct OutputShape {
    static constexpr int kRanks = RT * 16, kAdapters = tile_adapters(kRanks);
    static constexpr int kOp = (2 * kRanks + 63) / 64 * 16384;   // u and its rest: [128 rows x 64] chunks
    static constexpr int kY = RT == 8 ? 2 : 4, kB = RT == 8 ? 2 : 3;  // buffers of y (and out), of B
    static constexpr int kYBytes = 2 * 16384, kBBytes = (kRanks + 63) / 64 * kTileCols * 128;
    static constexpr int kYOff = kOp, kBOff = kYOff + kY * kYBytes;
    static constexpr int kSmem = 1024 + kBOff + kB * kBBytes;
    static constexpr int kThreads = 10 * 32;  // warps 0-7: out, two groups of 128 threads, each half of the columns; 8: TMA; 9: tcgen05.mma
    static_assert(2 * kTileRows * AdapterShape<RT>::kHalfRow * 2 <= kBOff, "by groups: u, in the tile's and y's place");
    static_assert(kSmem <= 232448 - 4096, "shared memory");
};

// Whether one of the half's 128 threads has it; a barrier for them.
__device__ __forceinline__ bool any_of_half(int half, bool has) {
    uint32_t any;
    __syncwarp();
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %2, 0;\n\tbar.red.or.pred p, %1, 128, q;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(any) : "r"(1 + half), "r"((uint32_t)has) : "memory");
    return any != 0;
}

// 64 columns from `col0` on of the warp's 32 tokens (a lane's from `row` on, in shared memory), of which some are not finite (odd): the ones whose row of B is
// not either are made anew, with the products of what rounding left of u taking B's finite elements alone (see expand_groups).  The lanes share the odd tokens'
// columns.  Out's columns have not left yet, so that y's are there, even if they are the same.  What looking costs where all is finite: 4000 tokens of one
// adapter, 4096 x 14336, 64 ranks, 61.0 -> 62.3 us for both kernels; of nine requests 72.9 .. 75.5 -> 74.3 .. 77.9.
template <bool F16, int RT>
__device__ __forceinline__ void redo_columns(const TileArgs& ta, bool odd, uint8_t* row, int token, int own, float unit, int col0, int lane) {
    const AdapterArgs& a = ta.a;
    constexpr uint32_t kTop = F16 ? 0x7c00u : 0x7f80u;
    for (int r = 0; r < RT * 8 && odd; r += 4) {
        const uint4 w = __ldcg(reinterpret_cast<const uint4*>(ta.u + (int64_t)token * (RT * 16) + r));
        for (uint32_t x : {w.x, w.y, w.z, w.w}) odd = odd && (x & 0x7fffu) <= kTop && (x >> 16 & 0x7fffu) <= kTop;  // else no column is a number, whatever B has
    }
    __syncwarp();
    const unsigned rows = __ballot_sync(0xffffffffu, odd);
    if (rows == 0) return;
    int lanes = 32;  // to a token
    while (lanes * __popc(rows) > 32) lanes /= 2;
    unsigned left = rows;
    for (int k = lane / lanes; k > 0; --k) left &= left - 1;
    const int r0 = left ? __ffs(left) - 1 : lane, adapter = __shfl_sync(0xffffffffu, own, r0);
    const float mul = __shfl_sync(0xffffffffu, unit, r0);
    if (left) {
        token += r0 - lane;
        row += (r0 - lane) * 128;
        const uint32_t* u = ta.u + (int64_t)token * (RT * 16);
#pragma unroll 1
        for (int i = lane % lanes; i < 64 && col0 + i < a.N; i += lanes) {
            uint16_t* at = reinterpret_cast<uint16_t*>(row + (((i >> 3) ^ (r0 & 7)) << 4)) + (i & 7);
            if (!is_odd(odd_pairs<F16>(*at, 0u))) continue;
            const uint16_t* b = static_cast<const uint16_t*>(a.b) + ((int64_t)adapter * a.N + col0 + i) * a.rank;
            float sum = 0.f;
            bool finite = true;
#pragma unroll 4
            for (int r = 0; r < a.rank; r += 2) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(b + r), w_rest = finite_pair<F16>(w);
                const float2 hi = unpack16<F16>(__ldcg(u + r / 2)), lo = unpack16<F16>(__ldcg(u + RT * 8 + r / 2)), f = unpack16<F16>(w), rest = unpack16<F16>(w_rest);
                finite = finite && w == w_rest;
                sum = fmaf(hi.x, f.x, fmaf(hi.y, f.y, fmaf(lo.x, rest.x, fmaf(lo.y, rest.y, sum))));
            }
            const uint16_t* y = static_cast<const uint16_t*>(a.y) + (int64_t)token * a.ys + col0 + i;
            if (!finite) *at = (uint16_t)pack16<F16>(fmaf(sum, mul, unpack16<F16>(*y).x), 0.f);
        }
    }
    __syncwarp();
}

template <bool F16, int RT>
__global__ void __launch_bounds__(OutputShape<RT>::kThreads, 1)
adapters_output_kernel(const __grid_constant__ CUtensorMap tmap_u, const __grid_constant__ CUtensorMap tmap_y, const __grid_constant__ CUtensorMap tmap_b,
                       const __grid_constant__ CUtensorMap tmap_out, const TileArgs ta) {
    using S = OutputShape<RT>;
    using namespace ptx;
    constexpr int kRanks = S::kRanks, kRow = AdapterShape<RT>::kHalfRow;
    extern __shared__ uint8_t smem_raw[];
    __shared__ AdGroup groups[kTileRows];
    __shared__ int which[kTileRows], base[kTileRows];
    __shared__ float unit[kTileRows];
    __shared__ int n_groups;
    __shared__ long long share[2];
    __shared__ uint64_t u_full, y_full[S::kY], y_free[S::kY], b_full[S::kB], b_free[S::kB], d_full[2], d_free[2];
    __shared__ uint32_t tmem_slot;
    const AdapterArgs& a = ta.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* smem = smem_raw + (((smem_u32(smem_raw) + 1023u) & ~1023u) - smem_u32(smem_raw));
    uint8_t *y_ring = smem + S::kYOff, *b_ring = smem + S::kBOff;
    if (threadIdx.x == 0) {
        mbar_init(&u_full, 1);
        for (int i = 0; i < S::kY; ++i) { mbar_init(&y_full[i], 1); mbar_init(&y_free[i], 2); }
        for (int i = 0; i < S::kB; ++i) { mbar_init(&b_full[i], 1); mbar_init(&b_free[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&d_full[i], 1); mbar_init(&d_free[i], 8); }
        fence_mbar_init();
        prefetch_tmap(&tmap_u);
        prefetch_tmap(&tmap_y);
        prefetch_tmap(&tmap_b);
        prefetch_tmap(&tmap_out);
    }
    if (warp == 9) {
        tmem_alloc(&tmem_slot, 2 * kTileCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = tmem_slot;
    pdl_launch_dependents();
    pdl_wait();

    // This CTA's chunks of 128 columns: an even share of what all tiles' chunks take, in quarters of one with one adapter.
    const int chunks = (a.N + kTileCols - 1) / kTileCols, tiles = (a.T + kTileRows - 1) / kTileRows;
    if (warp == 0) {
        auto cost = [&](int t) { return t < tiles ? chunk_cost(__ldcg(ta.list + t * kListInts), S::kAdapters) : 0; };
        const int cost0 = cost(lane);
        long long all = cost0;
        for (int t = 32 + lane; t < tiles; t += 32) all += cost(t);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        all *= chunks;
        const long long lo = all * blockIdx.x / gridDim.x, hi = all * (blockIdx.x + 1) / gridDim.x;
        long long before = 0;
        for (int t1 = 0; t1 < tiles; t1 += 32) {
            const long long mine = (long long)(t1 == 0 ? cost0 : cost(t1 + lane)) * chunks;
            long long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const long long start = before + incl - mine;
            auto mark = [&](long long u, int e) {
                if (mine > 0 && u >= start && u < start + mine) share[e] = (long long)(t1 + lane) * chunks + (u - start) / (mine / chunks);
            };
            mark(lo, 0);
            mark(hi, 1);
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0 && hi == all) share[1] = (long long)tiles * chunks;
    }
    __syncthreads();
    const long long from = share[0], to = share[1];
    bool failed = false;
    int n = 0, m = 0, seg = 0;  // chunks; chunks and adapters; tiles that went through the tensor cores, of this CTA so far
    for (long long at = from; at < to;) {
        const int tile = (int)(at / chunks), q0 = (int)(at - (long long)tile * chunks), q1 = (int)min((long long)chunks, q0 + to - at);
        at += q1 - q0;
        const int t0 = tile * kTileRows, tokens = min(kTileRows, a.T - t0);
        const int* list = ta.list + tile * kListInts;
        const int adapters = __ldcg(list);
        if (adapters == 0 && a.y == a.out) continue;
        if (adapters > S::kAdapters) {
            // ---- by groups of tokens; no copies are in flight, as behind each tile
            uint16_t *u_hi = reinterpret_cast<uint16_t*>(smem), *u_lo = u_hi + kTileRows * kRow;
            for (int t = threadIdx.x; t < tokens; t += S::kThreads) {
                which[t] = __ldcg(ta.which + t0 + t);
                unit[t] = __ldcg(ta.unit + t0 + t);
            }
            for (int e = threadIdx.x; e < tokens * kRanks; e += S::kThreads) {  // pairs
                const int t = e / kRanks, r = e % kRanks * 2;
                const uint32_t w = __ldcg(ta.u + (int64_t)t0 * kRanks + e);
                *reinterpret_cast<uint32_t*>((r < kRanks ? u_hi + r : u_lo + r - kRanks) + t * kRow) = w;
            }
            __syncthreads();
            make_groups(which, tokens, groups, &n_groups, base);
            __syncthreads();
            if (warp < kAdWarps) {
                const int end = min(2 * q1, (a.N + 63) / 64);
                AdColumns<RT> columns;
                expand_groups<F16, RT, false>(a, groups, u_hi, u_lo, unit, t0, AdShare(2 * q0, end, n_groups, warp, 1), end, columns, lane);
            }
            fence_proxy_async_smem();  // the ring is the copy engine's again
            __syncthreads();
            continue;
        }
        if (warp == 8) {
            if (elect_one() && !failed) {
                mbar_expect_tx(&u_full, S::kOp);
#pragma unroll
                for (int c = 0; c < S::kOp / 16384; ++c) tma_load_2d(smem + c * 16384, &tmap_u, &u_full, c * 64, t0);
                int several[S::kAdapters];
#pragma unroll
                for (int j = 0; j < S::kAdapters; ++j) several[j] = j < adapters ? __ldcg(list + 1 + j) : 0;
                int nn = n, mm = m;
                for (int q = q0; q < q1 && !failed; ++q, ++nn) {
                    const int yb = nn % S::kY;
                    if (nn >= S::kY && !mbar_wait(&y_free[yb], (nn / S::kY - 1) & 1)) { failed = true; break; }
                    mbar_expect_tx(&y_full[yb], S::kYBytes);
                    tma_load_2d(y_ring + yb * S::kYBytes, &tmap_y, &y_full[yb], q * kTileCols, t0);
                    tma_load_2d(y_ring + yb * S::kYBytes + 16384, &tmap_y, &y_full[yb], q * kTileCols + 64, t0);
#pragma unroll
                    for (int j = 0; j < S::kAdapters; ++j) {
                        if (j >= adapters) break;
                        const int bb = mm % S::kB;
                        if (mm >= S::kB && !mbar_wait(&b_free[bb], (mm / S::kB - 1) & 1)) { failed = true; break; }
                        mbar_expect_tx(&b_full[bb], S::kBBytes);
#pragma unroll
                        for (int c = 0; c < (kRanks + 63) / 64; ++c)
                            tma_load_2d(b_ring + bb * S::kBBytes + c * (kTileCols * 128), &tmap_b, &b_full[bb], c * 64, several[j] * a.N + q * kTileCols);
                        ++mm;
                    }
                }
            }
            __syncwarp();
        } else if (warp == 9) {
            if (elect_one() && !failed) {
                constexpr uint32_t idesc = F16 ? make_idesc_f16(128, kTileCols, false, false) : make_idesc_bf16(128, kTileCols, false, false);
                const uint64_t ud = make_smem_desc(smem_u32(smem), 16, 1024);
                if (!mbar_wait(&u_full, seg & 1)) failed = true;
                int mm = m;
                for (int q = q0; q < q1 && !failed; ++q)
                    for (int j = 0; j < adapters; ++j, ++mm) {
                        const int bb = mm % S::kB, db = mm & 1;
                        if (!mbar_wait(&b_full[bb], (mm / S::kB) & 1)) { failed = true; break; }
                        if (mm >= 2 && !mbar_wait(&d_free[db], (mm / 2 - 1) & 1)) { failed = true; break; }
                        tc_fence_after_sync();
                        const uint64_t bd = make_smem_desc(smem_u32(b_ring + bb * S::kBBytes), 16, 1024);
#pragma unroll
                        for (int e = 0; e < 2 * kRanks; e += 16) {  // u's ranks, then what rounding left of them, with the same columns of B
                            const int r = e % kRanks;
                            mma_ss(tmem + db * kTileCols, ud + (((e >> 6) * 16384 + (e & 63) * 2) >> 4),
                                   bd + (((r >> 6) * (kTileCols * 128) + (r & 63) * 2) >> 4), idesc, e > 0);
                        }
                        mma_commit(&b_free[bb]);
                        mma_commit(&d_full[db]);
                    }
            }
            __syncwarp();
        } else {
            const int row = threadIdx.x & 127, half = warp >> 2;
            const int own = row < tokens ? __ldcg(ta.which + t0 + row) : -1;
            const float mul = row < tokens ? __ldcg(ta.unit + t0 + row) : 0.f;
            const uint32_t lanes = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + half * 64;
            int several[S::kAdapters];
#pragma unroll
            for (int j = 0; j < S::kAdapters; ++j) several[j] = j < adapters ? __ldcg(list + 1 + j) : -2;
            int nn = n, mm = m;
            for (int q = q0; q < q1; ++q, ++nn) {
                const int yb = nn % S::kY;
                uint8_t* half_ring = y_ring + yb * S::kYBytes + half * 16384;
                uint8_t* y = half_ring + row * 128;
                bool odd = false;
                if (!failed && !warp_wait(&y_full[yb], (nn / S::kY) & 1)) failed = true;
#pragma unroll
                for (int j = 0; j < S::kAdapters; ++j) {
                    if (j >= adapters) break;
                    const int db = mm & 1;
                    if (!failed && !warp_wait(&d_full[db], (mm / 2) & 1)) failed = true;
                    const bool hit = own == several[j];
                    if (!failed && __any_sync(0xffffffffu, hit)) {
                        tc_fence_after_sync();
                        uint32_t d[2][32];
                        __syncwarp();
                        tmem_ld_x32(lanes + db * kTileCols, d[0]);
                        tmem_ld_x32(lanes + db * kTileCols + 32, d[1]);
                        tmem_ld_wait();
                        if (hit) {
                            float2 o[4] = {};  // zeros while D is finite; sums side by side
#pragma unroll
                            for (int i = 0; i < 64; i += 2)
                                o[i / 2 & 3] = ffma2(make_float2(__uint_as_float(d[i >> 5][i & 31]), __uint_as_float(d[i >> 5][(i & 31) + 1])), make_float2(0.f, 0.f), o[i / 2 & 3]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                uint4* at16 = reinterpret_cast<uint4*>(y + ((i ^ (row & 7)) << 4));
                                const uint4 w = *at16;
                                const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                                uint32_t out[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const float2 p = make_float2(__uint_as_float(d[i >> 2][(i & 3) * 8 + 2 * k]), __uint_as_float(d[i >> 2][(i & 3) * 8 + 2 * k + 1]));
                                    const float2 f = ffma2(p, make_float2(mul, mul), unpack16<F16>(in[k]));
                                    out[k] = pack16<F16>(f.x, f.y);
                                }
                                *at16 = make_uint4(out[0], out[1], out[2], out[3]);
                            }
                            const float2 all = fadd2(fadd2(o[0], o[1]), fadd2(o[2], o[3]));
                            odd = all.x + all.y != 0.f;
                        }
                        tc_fence_before_sync();
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&d_free[db]);
                    ++mm;
                }
                fence_proxy_async_smem();
                if (__builtin_expect(any_of_half(half, odd), 0)) {
                    redo_columns<F16, RT>(ta, odd, y, t0 + row, own, mul, q * kTileCols + half * 64, lane);
                    fence_proxy_async_smem();
                    any_of_half(half, false);
                }
                if ((threadIdx.x & 127) == 0 && !failed) {
                    if (q * kTileCols + half * 64 < a.N) tma_store_2d(&tmap_out, half_ring, q * kTileCols + half * 64, t0);
                    tma_store_commit();
                    if (q > q0) {
                        tma_store_wait_read<1>();  // all but this one
                        mbar_arrive(&y_free[(nn - 1) % S::kY]);
                    }
                    if (q == q1 - 1) {
                        tma_store_wait_read<0>();
                        mbar_arrive(&y_free[yb]);
                    }
                }
                __syncwarp();
            }
        }
        ++seg;
        n += q1 - q0;
        m += (q1 - q0) * adapters;
        tc_fence_before_sync();
        __syncthreads();  // all has been read: the next tile's copies may come
        tc_fence_after_sync();
    }
    if ((threadIdx.x & 127) == 0 && warp < 8) tma_store_wait_all<0>();
    if (failed) {
        atomicExch(a.status, 1);
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // let copies and products in flight end before their memory goes away
    }
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 2 * kTileCols);
}

template <bool F16, int RT, int CTAS, bool DEEP>
int launch_contract(const CUtensorMap& tx, const CUtensorMap& ta, const TileArgs& t, long long tiles, cudaStream_t s) {
    auto kernel = adapters_contract_kernel<F16, RT, CTAS, DEEP>;
    constexpr int kSmem = ContractShape<RT, DEEP>::kSmem;
    FORGE_SET_SMEM_ONCE(kernel, kSmem);
    FORGE_CUDA_TRY(launch_pdl_cluster(kernel, dim3((unsigned)(tiles * CTAS)), dim3(kAdThreads), kSmem, CTAS, s, tx, ta, t));
    return FORGE_OK;
}

template <bool F16, int RT>
int launch_adapters_tiles(const AdapterArgs& a, void* workspace, cudaStream_t s) {
    using O = OutputShape<RT>;
    constexpr int kRanks = RT * 16;
    auto output = adapters_output_kernel<F16, RT>;
    FORGE_SET_SMEM_ONCE(output, O::kSmem);
    const TileWorkspace w(a.T, kRanks);
    char* base = static_cast<char*>(workspace);
    TileArgs t = {a, reinterpret_cast<int*>(base), reinterpret_cast<int*>(base + w.list), reinterpret_cast<float*>(base + w.unit), reinterpret_cast<uint32_t*>(base + w.u)};
    CUtensorMap tx, ta, tu, ty, tb, to;
    auto rows = [&](CUtensorMap* m, const void* p, int64_t width, int64_t n, int64_t stride, int box_rows) {
        const uint64_t dims[2] = {(uint64_t)width, (uint64_t)n}, strides[1] = {(uint64_t)stride * 2};
        const uint32_t box[2] = {64, (uint32_t)box_rows};
        return encode_tmap_bf16_sw128(m, p, 2, dims, strides, box);
    };
    if (!rows(&tx, a.x, a.K, a.T, a.xs, kTileRows) || !rows(&ta, a.a, a.K, (int64_t)a.n * a.rank, a.K, kRanks) ||
        !rows(&tu, t.u, 2 * kRanks, a.T, 2 * kRanks, kTileRows) || !rows(&ty, a.y, a.N, a.T, a.ys, kTileRows) ||
        !rows(&tb, a.b, a.rank, (int64_t)a.n * a.N, a.rank, kTileCols) || !rows(&to, a.out, a.N, a.T, a.os, kTileRows))
        return FORGE_ERR_CUDA;
    const long long tiles = ((long long)a.T + kTileRows - 1) / kTileRows, chunks = tiles * ((a.N + kTileCols - 1) / kTileCols);
    const int sms = sm_count();
    // Clusters of four where those of eight would not all run at a time (two CTAs to an SM, and SMs that no cluster fits on), with an SM for each CTA while
    // there are enough, and more buffers (4000 tokens, 14336 x 4096, 64 ranks: 34.7 and 32.4 us; 9 requests, 4096 x 14336, both kernels 75 .. 78 and 73 .. 75).
    constexpr int kHalf = kAdCtas / 2;
    int st;
    if (tiles * kAdCtas * (RT == 8 ? 2 : 1) <= sms * 3 / 2) st = launch_contract<F16, RT, kAdCtas, false>(tx, ta, t, tiles, s);
    else if (RT <= 4 && tiles * kHalf <= sms) st = launch_contract<F16, RT, kHalf, (RT <= 4)>(tx, ta, t, tiles, s);
    else st = launch_contract<F16, RT, kHalf, false>(tx, ta, t, tiles, s);
    if (st != FORGE_OK) return st;
    FORGE_CUDA_TRY(launch_pdl(output, dim3((unsigned)(chunks < sms ? chunks : sms)), dim3(O::kThreads), O::kSmem, s, tu, ty, tb, to, t));
    return finish_launch(2);
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
int launch_adapters(const AdapterArgs& a, void* workspace, cudaStream_t s) {
    if (a.T >= kTileTokens) return launch_adapters_tiles<F16, RT>(a, workspace, s);
    return a.tile <= 8 ? launch_adapters<F16, RT, true>(a, s) : launch_adapters<F16, RT, false>(a, s);
}
template <bool F16>
int launch_adapters(const AdapterArgs& a, void* workspace, cudaStream_t s) {
    return a.rank <= 16   ? launch_adapters<F16, 1>(a, workspace, s)
           : a.rank <= 32 ? launch_adapters<F16, 2>(a, workspace, s)
           : a.rank <= 64 ? launch_adapters<F16, 4>(a, workspace, s)
                          : launch_adapters<F16, 8>(a, workspace, s);
}

}  // namespace
}  // namespace forge

extern "C" size_t forge_linear_adapters_workspace_bytes(int T, int rank) {
    using namespace forge;
    if (T < kTileTokens || rank <= 0 || rank > 128) return 0;
    return TileWorkspace(T, padded_ranks(rank)).bytes;
}

extern "C" int forge_linear_adapters(const forge_adapters* set, const void* x, const void* y, void* out, int T, int64_t x_stride,
                                     int64_t y_stride, int64_t out_stride, const int32_t* requests, const int32_t* adapters, int R,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    using namespace forge;
    if (!set || !set->a || !set->b || !x || !y || !out || !adapters || T <= 0 || R <= 0) return FORGE_ERR_INVALID_ARG;
    if (set->n <= 0 || set->rank <= 0 || set->K <= 0 || set->N <= 0 || x_stride < 0 || y_stride < 0 || out_stride < 0) return FORGE_ERR_INVALID_ARG;
    if (!aligned16(set->a) || !aligned16(set->b) || !aligned16(x) || !aligned16(y) || !aligned16(out) || !aligned16(workspace)) return FORGE_ERR_INVALID_ARG;
    auto odd4 = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; };
    if (odd4(set->scales) || odd4(requests) || odd4(adapters) || (!requests && R != T)) return FORGE_ERR_INVALID_ARG;
    if (set->dtype != FORGE_DTYPE_BF16 && set->dtype != FORGE_DTYPE_F16) return set->dtype == FORGE_DTYPE_F32 ? FORGE_ERR_UNSUPPORTED : FORGE_ERR_INVALID_ARG;
    AdapterArgs a = {};
    a.xs = x_stride ? x_stride : set->K;
    a.ys = y_stride ? y_stride : set->N;
    a.os = out_stride ? out_stride : set->N;
    if (a.xs < set->K || a.ys < set->N || a.os < set->N) return FORGE_ERR_INVALID_ARG;
    if (y == out && a.ys != a.os) return FORGE_ERR_INVALID_ARG;
    if (set->K % 8 != 0 || set->N % 8 != 0 || set->rank % 8 != 0 || set->rank > 128 || T > 1 << 30) return FORGE_ERR_UNSUPPORTED;
    if (a.xs % 8 != 0 || a.ys % 8 != 0 || a.os % 8 != 0) return FORGE_ERR_UNSUPPORTED;
    if ((long long)set->n * set->N >= (1LL << 31) || (long long)set->n * set->rank >= (1LL << 31)) return FORGE_ERR_UNSUPPORTED;  // counted in 32 bits
    const size_t need = forge_linear_adapters_workspace_bytes(T, set->rank);
    if (need > 0 && !workspace) return FORGE_ERR_INVALID_ARG;
    if (workspace_bytes < need) return FORGE_ERR_WORKSPACE;
    a.x = x; a.y = y; a.out = out;
    a.a = set->a; a.b = set->b;
    a.scales = set->scales;
    a.requests = requests;
    a.adapters = adapters;
    a.T = T; a.R = R;
    a.n = set->n; a.rank = set->rank; a.K = set->K; a.N = set->N;
    // A tile's tokens: so many that all clusters run at a time, two CTAs to an SM but for the SMs that no whole cluster fits on (200 tokens of 200 requests of
    // 40 adapters, 4096 x 4096, 16 ranks: 24.6 us in 34 clusters, 21.6 in 29); from 9 on 16, which the warps share.  With more than 64 ranks, one CTA to an SM, that
    // holds up to 256 tokens: more go in two rounds.
    const int sms = sm_count();
    a.status = device_status_word();
    if (sms <= 0 || !a.status) return FORGE_ERR_CUDA;
    const int clusters = (a.rank <= 64 ? 2 : 1) * sms / 9, want = (T + clusters - 1) / clusters;
    a.tile = want <= 8 ? want : 16;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return set->dtype == FORGE_DTYPE_F16 ? launch_adapters<true>(a, workspace, s) : launch_adapters<false>(a, workspace, s);
}
