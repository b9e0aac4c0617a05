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

namespace forge {
namespace {

constexpr int kAdCtas = 8;                 // of a cluster
constexpr int kAdWarps = 8, kAdThreads = kAdWarps * 32;
constexpr int kAdMost = 128;               // tokens of a tile

struct AdapterArgs {
    const void *x, *y, *a, *b;
    void* out;
    const float* scales;
    const int32_t *requests, *adapters;
    int64_t xs, ys, os;                    // elements from a token to the next
    int T, R, n, rank, K, N, tile;
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
__device__ __forceinline__ void store_peer16(uint32_t addr, uint16_t v) { asm volatile("st.shared::cluster.u16 [%0], %1;" ::"r"(addr), "h"(v) : "memory"); }
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

template <bool F16, int RT, bool SMALL>
__global__ void __launch_bounds__(kAdThreads) adapters_kernel(const AdapterArgs a) {
    using S = AdapterShape<RT>;
    constexpr int kRanks = S::kRanks, kRow = S::kHalfRow;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ AdGroup groups[kAdMost];
    __shared__ int which[kAdMost];
    __shared__ float unit[kAdMost];  // out += unit * (u in shared memory) B^T
    __shared__ int n_groups;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
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

    // ---- the tokens' adapters, and their groups
    for (int t = threadIdx.x; t < tokens; t += kAdThreads) {
        int i = t0 + t;
        if (a.requests) i = __ldcg(a.requests + i);
        i = (unsigned)i < (unsigned)a.R ? __ldcg(a.adapters + i) : -1;
        which[t] = (unsigned)i < (unsigned)a.n ? i : -1;
    }
    __syncthreads();
    if (warp == 0) {
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
        if (lane == 0) n_groups = count;
    }
    __syncthreads();

    // ---- u^T = A x^T over this CTA's part of K, in blocks of 64
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
    __syncthreads();
    ad_wait();  // all CTAs of the cluster run

    // ---- the eighths to where they are summed
    const uint32_t inbox_addr = ptx::smem_u32(inbox), hi_addr = ptx::smem_u32(u_hi), lo_addr = ptx::smem_u32(u_lo), unit_addr = ptx::smem_u32(unit);
    const int per = SMALL ? a.tile : a.tile / kAdCtas;  // tokens that a CTA sums up
    if constexpr (SMALL) {  // everyone sums all of it
        for (int e = threadIdx.x; e < tokens * kRanks; e += kAdThreads) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < kAdWarps; ++w) s += mine[w * a.tile * kRanks + e];
#pragma unroll
            for (int p = 0; p < kAdCtas; ++p) store_peer(peer_smem(inbox_addr + (cta * a.tile * kRanks + e) * 4, p), s);
        }
    } else {  // each its eighth of the tokens
        for (int e = threadIdx.x; e < tokens * kRanks; e += kAdThreads) {
            const int t = e / kRanks, p = t / per;
            store_peer(peer_smem(inbox_addr + ((cta * per + t - p * per) * kRanks + e % kRanks) * 4, p), mine[e]);
        }
    }
    ad_arrive();
    ad_wait();

    // ---- summed, scaled and cut into two: a warp for each token
    const int sum0 = SMALL ? 0 : cta * per, sum1 = SMALL ? tokens : min(sum0 + per, tokens);
    for (int t = sum0 + warp; t < sum1; t += kAdWarps) {
        constexpr int kEach = (kRanks + 31) / 32;
        float v[kEach];
        const int i = which[t];
        const float scale = i >= 0 ? a.scales ? a.scales[i] : 1.f : 0.f;
        uint32_t big = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int r = j * 32 + lane;
            v[j] = 0.f;
            if (r < a.rank && i >= 0) {
#pragma unroll
                for (int p = 0; p < kAdCtas; ++p) v[j] += inbox[(p * per + t - sum0) * kRanks + r];
                v[j] *= scale;
            }
            const uint32_t bits = __float_as_uint(v[j]) & 0x7fffffffu;
            if (bits < 0x7f800000u) big = max(big, bits);
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
            const int r = j * 32 + lane;
            if (r >= kRanks) continue;
            const float x = v[j] * up;
            uint16_t hi, lo;
            if constexpr (F16) {
                const __half h = __float2half_rn(x);
                const float rest = x - __half2float(h);
                hi = __half_as_ushort(h);
                lo = __half_as_ushort(__float2half_rn(isfinite(rest) ? rest : 0.f));
            } else {
                const __nv_bfloat16 h = __float2bfloat16_rn(x);
                const float rest = x - __bfloat162float(h);
                hi = __bfloat16_as_ushort(h);
                lo = __bfloat16_as_ushort(__float2bfloat16_rn(isfinite(rest) ? rest : 0.f));
            }
            const int at = t * kRow + r;
            if constexpr (SMALL) {
                u_hi[at] = hi;
                u_lo[at] = lo;
            } else {
#pragma unroll
                for (int p = 0; p < kAdCtas; ++p) {
                    store_peer16(peer_smem(hi_addr + at * 2, p), hi);
                    store_peer16(peer_smem(lo_addr + at * 2, p), lo);
                }
            }
        }
        if (lane == 0) {
            const float inv = __fdiv_rn(1.f, up);  // a power of two
            if constexpr (SMALL) {
                unit[t] = inv;
            } else {
#pragma unroll
                for (int p = 0; p < kAdCtas; ++p) store_peer(peer_smem(unit_addr + t * 4, p), inv);
            }
        }
    }
    if constexpr (SMALL) {
        __syncthreads();
    } else {
        ad_arrive();
        ad_wait();
    }

    // ---- out^T = y^T + unit B u^T, 64 columns at a time: lane (g, c) has columns 8 g .. 8 g + 7 of tokens 2c, 2c + 1.  Row g (+ 8) of tile i of
    // the instructions' 16 is column 8 g + 2 i (+ 1).
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
    if (sms <= 0) return FORGE_ERR_CUDA;
    const int want = (T + sms / 4 - 1) / (sms / 4);
    a.tile = want <= 8 ? want : want <= 16 ? 16 : want <= 32 ? 32 : want <= 64 ? 64 : 128;
    if (a.rank > 64 && a.tile > 64) a.tile = 64;
    if ((long long)T / a.tile >= (1LL << 28)) return FORGE_ERR_UNSUPPORTED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return set->dtype == FORGE_DTYPE_F16 ? launch_adapters<true>(a, s) : launch_adapters<false>(a, s);
}
