// Rotary positions, rows into a KV cache (rotated and quantised on their way), rows back out of it.
//
// Reading back is bound by moving bytes (16 x 8 heads x 4096 e4m3 rows of 128, 254 MB, in 46 us: 5.5 TB/s), rotation and append of many tokens by
// those and the instructions on each element (rotating 3 x 32 heads x 1777 fp16 rows, 87 MB, 18.7 us: 4.7 TB/s; append of 4 x 2048 tokens of 32/8
// heads to e4m3, 185 MB, 39 us: 4.7 TB/s), and all three at a token per sequence by the launch (2.1, 2.7 and 2.5 us in a chain of launches).
//
// Rotation.  A warp works on the heads of one token (or on a share of them), a lane on the same 16 elements of every head, which hold whole
// pairs: so the cosines and sines are made once for all heads (per head they would take longer than the copies), and no
// element leaves its lane.  The angle in turns is position * F mod 2^64 with
// F = inv_freq / 2 pi in 64-bit fixed point: the product wraps around exactly where the circle does, so nothing is lost
// at far positions.
//
// Quantisation.  The row's largest magnitude is a maximum over its lanes (of the bit patterns, where NaN is the largest), then
// each lane rounds its elements and stores them, 8 bytes at a time.  Rows are rounded once, from fp32.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "kv_cache.cuh"

namespace forge {
namespace {

constexpr int kRotWarps = 4;
enum { kNoCache = 0, kCache16 = 1, kCacheInt8 = 2, kCacheE4m3 = 3 };

struct RotArgs {
    const void *q, *k, *v;
    void *q_out, *kc, *vc;
    float *ks, *vs;
    Strides qs, qos, kst, vst;
    const int32_t *positions, *first, *counts, *rows;
    const float* inv_freq;
    float amplitude, sin_sign;
    int half, interleaved;
    int B, Hq, Hkv, S, S_src, Smax, D, parts;
};

template <typename T>
struct Vec8;  // 8 elements as loaded
template <>
struct Vec8<__nv_bfloat16> {
    uint4 r;
    __device__ void load(const void* p) { r = *static_cast<const uint4*>(p); }
    __device__ void unpack(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
    static __device__ void store(void* p, const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec8<__half> {
    uint4 r;
    __device__ void load(const void* p) { r = *static_cast<const uint4*>(p); }
    __device__ void unpack(float (&x)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = t.x;
            x[2 * i + 1] = t.y;
        }
    }
    static __device__ void store(void* p, const float (&x)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __half2 t = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        *static_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Vec8<float> {
    float4 a, b;
    __device__ void load(const void* p) { a = static_cast<const float4*>(p)[0]; b = static_cast<const float4*>(p)[1]; }
    __device__ void unpack(float (&x)[8]) const {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    static __device__ void store(void* p, const float (&x)[8]) {
        static_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        static_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
};

// cos and sin of position * inv_freq.  inv_freq / 2 pi as a 64-bit fraction of a turn is off by 2^-53 of itself (fp64), the
// product by as much times the position; the top 32 bits in fp32 give the angle to 2^-24 of pi.
__device__ __forceinline__ float2 cos_sin(int64_t position, float inv_freq) {
    double turns = (double)inv_freq * 0.15915494309189533577;  // 1 / 2 pi
    turns -= floor(turns);
    const uint64_t f = (uint64_t)(turns * 18446744073709551616.0);
    const int32_t a = (int32_t)(((uint64_t)position * f) >> 32);
    float s, c;
    sincospif((float)a * 4.656612873077392578125e-10f, &s, &c);  // 2^-31: half turns
    return make_float2(c, s);
}

// The row's scale from its largest magnitude (as a bit pattern) and what its elements are multiplied by.
template <int FMT>
__device__ __forceinline__ float row_scale(uint32_t largest, float* mul) {
    constexpr float kTop = FMT == kCacheInt8 ? 127.f : 448.f;
    const float m = __uint_as_float(largest);
    const bool ok = largest < 0x7f800000u && largest >= 0x0d800000u;  // finite, at least 2^-100
    *mul = ok ? __fdiv_rn(kTop, m) : 0.f;
    return ok ? __fdiv_rn(m, kTop) : largest >= 0x7f800000u ? __int_as_float(0x7fc00000) : 0.f;
}
template <int FMT>
__device__ __forceinline__ uint2 encode8(const float (&y)[8], float mul) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (FMT == kCacheInt8) {
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = (uint32_t)__float2int_rn(mul == 0.f ? 0.f : y[4 * i + j] * mul) & 0xffu;
            w[i] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
        } else {
            uint16_t lo, hi;
            float z[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = mul == 0.f ? 0.f : y[4 * i + j] * mul;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(z[1]), "f"(z[0]));
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(z[3]), "f"(z[2]));
            w[i] = (uint32_t)lo | (uint32_t)hi << 16;
        }
    }
    return make_uint2(w[0], w[1]);
}

// LPR lanes of two 8-element pieces to a row (4, 8, 16); FMT: what the k and v rows become (kNoCache: there are q rows only).
// A lane's pieces are chosen so that pairs meet in it: half layout, pieces 8 i and half + 8 i (then the unrotated rest two by two); interleaved,
// pieces 16 i and 16 i + 8.  GENERIC: half layout whose halves are not whole pieces: pairs meet in shared memory.
template <typename T, int LPR, int FMT, bool GENERIC>
__global__ void __launch_bounds__(kRotWarps * 32, 5) rotate_append_kernel(const RotArgs a) {
    constexpr int RPW = 32 / LPR;                            // rows at a time
    constexpr int U = sizeof(T) == 4 || GENERIC ? 1 : 2;     // of those, loads in flight
    constexpr int kAngles = GENERIC ? 16 : 8;
    __shared__ float swap_all[GENERIC ? kRotWarps : 1][GENERIC ? RPW * LPR * 16 : 1];  // rows on the way to their partners
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_launch_dependents();
    const int64_t unit = (int64_t)blockIdx.x * kRotWarps + warp;
    const int64_t token = unit / a.parts;
    const int part = (int)(unit - token * a.parts);
    pdl_wait();
    if (token >= (int64_t)a.B * a.S) return;
    const int b = (int)(token / a.S), s = (int)(token - (int64_t)b * a.S);
    if (a.counts && s >= a.counts[b]) return;
    int src = s;
    if (a.rows) {
        src = a.rows[token];
        if (src < 0 || src >= a.S_src) return;
    }
    int64_t start = a.first ? a.first[b] : 0;
    if (FMT != kNoCache) start = min(max(start, (int64_t)0), (int64_t)a.Smax);
    const int64_t dst = start + s;  // the row of the cache
    const int H = FMT == kNoCache ? a.Hq : a.Hq + 2 * a.Hkv;
    const int sub = lane / LPR, li = lane % LPR;
    const int dims = 2 * a.half;
    const bool together = !GENERIC && !a.interleaved && li < a.half / 8;  // the pieces are halves of the same pairs
    const int d0 = together ? 8 * li : GENERIC || a.interleaved ? 16 * li : dims + 16 * (li - a.half / 8);
    const int d1 = together ? a.half + 8 * li : d0 + 8;
    const bool in0 = d0 < a.D, in1 = d1 < a.D;

    const int iters = (H + RPW - 1) / RPW;
    const int64_t cache_row = FMT == kNoCache ? 0 : ((int64_t)b * a.Hkv) * a.Smax + dst;  // of KV head 0
    const T* const q_row = static_cast<const T*>(a.q) + b * a.qs.b + s * a.qs.s;
    const T* const k_row = FMT == kNoCache ? nullptr : static_cast<const T*>(a.k) + b * a.kst.b + src * a.kst.s;
    const T* const v_row = FMT == kNoCache ? nullptr : static_cast<const T*>(a.v) + b * a.vst.b + src * a.vst.s;
    T* const out_row = static_cast<T*>(a.q_out) + b * a.qos.b + s * a.qos.s;
    // the next rows are on their way while these are worked on; the first ones leave before the cosines are made
    Vec8<T> raw[U][2], then[U][2];
    auto load = [&](int it0, Vec8<T> (&to)[U][2]) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = (it0 + u * a.parts) * RPW + sub;
            if (h >= H) continue;
            const T* p;
            if (FMT == kNoCache || h < a.Hq) p = q_row + h * a.qs.h;
            else if (h < a.Hq + a.Hkv) p = k_row + (h - a.Hq) * a.kst.h;
            else p = v_row + (h - a.Hq - a.Hkv) * a.vst.h;
            if (in0) to[u][0].load(p + d0);
            if (in1) to[u][1].load(p + d1);
        }
    };
    load(part, then);

    // cosines and sines: of this lane's pairs, or (GENERIC) elements
    float cs[kAngles], sn[kAngles];
    if (dims > 0 && (together || ((GENERIC || a.interleaved) && d0 < dims))) {
        const int64_t pos = a.positions ? a.positions[(int64_t)b * a.S_src + src] : start + s;
#pragma unroll
        for (int i = 0; i < kAngles; ++i) {
            int f;
            if constexpr (GENERIC) f = d0 + i < a.half ? d0 + i : d0 + i - a.half;
            else f = together ? d0 + i : d0 / 2 + i;
            const float2 t = cos_sin(pos, a.inv_freq[min(f, a.half - 1)]);
            cs[i] = t.x * a.amplitude;
            sn[i] = t.y * a.amplitude * a.sin_sign;
        }
    }

    for (int it0 = part; it0 < iters; it0 += a.parts * U) {
#pragma unroll
        for (int u = 0; u < U; ++u) { raw[u][0] = then[u][0]; raw[u][1] = then[u][1]; }
        if (it0 + a.parts * U < iters) load(it0 + a.parts * U, then);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if ((it0 + u * a.parts) * RPW >= H) break;  // the whole warp
            const int h = (it0 + u * a.parts) * RPW + sub;
            const bool here = h < H, is_v = FMT != kNoCache && h >= a.Hq + a.Hkv;
            float x[2][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[0][j] = x[1][j] = 0.f;
            if (here && in0) raw[u][0].unpack(x[0]);
            if (here && in1) raw[u][1].unpack(x[1]);
            if constexpr (GENERIC) {
                float* row = swap_all[warp] + sub * LPR * 16;
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 16; ++j) row[d0 + j] = x[j >> 3][j & 7];
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int d = d0 + j;
                    if (is_v || d >= dims) continue;
                    const float other = row[d < a.half ? d + a.half : d - a.half];
                    x[j >> 3][j & 7] = fmaf(other, d < a.half ? -sn[j] : sn[j], x[j >> 3][j & 7] * cs[j]);
                }
            } else if (is_v || dims == 0) {
            } else if (together) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float lo = x[0][j], hi = x[1][j];
                    x[0][j] = fmaf(hi, -sn[j], lo * cs[j]);
                    x[1][j] = fmaf(lo, sn[j], hi * cs[j]);
                }
            } else if (a.interleaved) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (d0 + 2 * i < dims) {
                        float &lo = x[i >> 2][2 * (i & 3)], &hi = x[i >> 2][2 * (i & 3) + 1];
                        const float was = lo;
                        lo = fmaf(hi, -sn[i], was * cs[i]);
                        hi = fmaf(was, sn[i], hi * cs[i]);
                    }
            }
            if (FMT == kNoCache || h < a.Hq) {
                T* p = out_row + h * a.qos.h;
                if (here && in0) Vec8<T>::store(p + d0, x[0]);
                if (here && in1) Vec8<T>::store(p + d1, x[1]);
                if constexpr (FMT == kNoCache || FMT == kCache16) continue;
            }
            if constexpr (FMT != kNoCache) {
                const int64_t row = cache_row + (int64_t)(is_v ? h - a.Hq - a.Hkv : h - a.Hq) * a.Smax;
                if constexpr (FMT == kCache16) {
                    T* p = static_cast<T*>(is_v ? a.vc : a.kc) + row * a.D;
                    if (here && in0 && dst < a.Smax) Vec8<T>::store(p + d0, x[0]);
                    if (here && in1 && dst < a.Smax) Vec8<T>::store(p + d1, x[1]);
                } else {
                    if (!__any_sync(0xffffffffu, h >= a.Hq)) continue;  // q rows only
                    uint32_t m = 0;  // the lanes of a row meet: all lanes take part, those of q rows too
#pragma unroll
                    for (int j = 0; j < 8; ++j) m = max(m, max(__float_as_uint(x[0][j]) & 0x7fffffffu, __float_as_uint(x[1][j]) & 0x7fffffffu));
#pragma unroll
                    for (int o = LPR / 2; o > 0; o >>= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
                    float mul;
                    const float scale = row_scale<FMT>(m, &mul);
                    if (here && h >= a.Hq && dst < a.Smax) {
                        uint8_t* p = static_cast<uint8_t*>(is_v ? a.vc : a.kc) + row * a.D;
                        if (in0) *reinterpret_cast<uint2*>(p + d0) = encode8<FMT>(x[0], mul);
                        if (in1) *reinterpret_cast<uint2*>(p + d1) = encode8<FMT>(x[1], mul);
                        if (li == 0) (is_v ? a.vs : a.ks)[row] = scale;
                    }
                }
            }
        }
    }
}

template <typename T, int LPR, int FMT>
int launch_rotate(RotArgs& a, cudaStream_t s) {
    const int sms = sm_count();
    if (sms <= 0) return FORGE_ERR_CUDA;
    const int H = FMT == kNoCache ? a.Hq : a.Hq + 2 * a.Hkv;
    const int iters = (H + 32 / LPR - 1) / (32 / LPR);
    const long long tokens = (long long)a.B * a.S;
    // A token's heads are shared out while that leaves SMs short of warps (16 of them each): the cosines are made once per share.
    // 16 tokens of 40 heads: 3.8 us in one share, 2.1 in ten; append of 16 tokens of 32/8 heads 7.3 and 2.7.  4 x 2048 tokens: 41.6 in one, 44.0 in
    // two, 49.2 in three.
    const long long want = (16LL * sms + tokens - 1) / tokens;
    a.parts = (int)(want < 1 ? 1 : want > iters ? iters : want);
    const long long ctas = (tokens * a.parts + kRotWarps - 1) / kRotWarps;
    if (ctas > 0x7fffffffLL) return FORGE_ERR_UNSUPPORTED;
    const auto kernel = !a.interleaved && a.half % 8 != 0 ? rotate_append_kernel<T, LPR, FMT, true> : rotate_append_kernel<T, LPR, FMT, false>;
    FORGE_CUDA_TRY(launch_pdl(kernel, dim3((unsigned)ctas), dim3(kRotWarps * 32), 0, s, a));
    return finish_launch(1);
}

template <typename T>
int launch_rotate_only(RotArgs& a, cudaStream_t s) {
    return a.D <= 64 ? launch_rotate<T, 4, kNoCache>(a, s) : a.D <= 128 ? launch_rotate<T, 8, kNoCache>(a, s) : launch_rotate<T, 16, kNoCache>(a, s);
}
template <typename T, int FMT>
int launch_append(RotArgs& a, cudaStream_t s) {
    return a.D <= 64 ? launch_rotate<T, 4, FMT>(a, s) : launch_rotate<T, 8, FMT>(a, s);
}
template <typename T>
int dispatch_append(int format, RotArgs& a, cudaStream_t s) {
    return format == FORGE_KV_INT8   ? launch_append<T, kCacheInt8>(a, s)
           : format == FORGE_KV_E4M3 ? launch_append<T, kCacheE4m3>(a, s)
                                     : launch_append<T, kCache16>(a, s);
}

int check_rotary(const forge_rotary* r, int D) {
    if (!r || !r->inv_freq || (reinterpret_cast<uintptr_t>(r->inv_freq) & 3u)) return FORGE_ERR_INVALID_ARG;
    if (r->dims < 2 || r->dims > D || r->dims % 2 != 0) return FORGE_ERR_INVALID_ARG;
    if (r->layout != FORGE_ROTARY_HALF && r->layout != FORGE_ROTARY_INTERLEAVED) return FORGE_ERR_INVALID_ARG;
    return FORGE_OK;
}
void set_rotary(RotArgs& a, const forge_rotary& r, int inverse) {
    a.inv_freq = r.inv_freq;
    a.amplitude = r.amplitude;
    a.sin_sign = inverse ? -1.f : 1.f;
    a.half = r.dims / 2;
    a.interleaved = r.layout == FORGE_ROTARY_INTERLEAVED;
}
bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

// ------------------------------------------------------------------------------------------------- rows back
constexpr int kReadThreads = 256, kReadUnroll = 4;

struct ReadArgs {
    const void *kc, *vc;
    const float *ks, *vs;
    void *k_out, *v_out;
    Strides kst, vst;
    const int32_t *first, *counts;
    int Hkv, Smax, S, D, blocks, pieces;  // blocks of rows per (batch, head); 16-byte pieces per cached row
};

template <bool F16>
__device__ __forceinline__ uint32_t scaled_pair(uint32_t h2, float scale) {
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h2));
    if constexpr (F16) {
        const __half2 r = __floats2half2_rn(x.x * scale, x.y * scale);
        return *reinterpret_cast<const uint32_t*>(&r);
    } else {
        const __nv_bfloat162 r = __floats2bfloat162_rn(x.x * scale, x.y * scale);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
}

// A CTA takes kReadThreads * kReadUnroll pieces of 16 bytes of one (batch, head), of K (blockIdx.y 0) or V: a piece of 8-bit codes becomes 32 bytes.
template <int FMT, bool F16>
__global__ void __launch_bounds__(kReadThreads) read_rows_kernel(const ReadArgs a) {
    pdl_launch_dependents();
    const bool is_v = blockIdx.y != 0;
    const int bh = blockIdx.x / a.blocks, block = blockIdx.x - bh * a.blocks;
    const int b = bh / a.Hkv, h = bh - b * a.Hkv;
    pdl_wait();
    const int count = a.counts ? min(max(a.counts[b], 0), a.S) : a.S;
    const int64_t first = a.first ? a.first[b] : 0;
    const uint8_t* cache = static_cast<const uint8_t*>(is_v ? a.vc : a.kc);
    const float* scales = is_v ? a.vs : a.ks;
    uint8_t* out = static_cast<uint8_t*>(is_v ? a.v_out : a.k_out);
    const Strides st = is_v ? a.vst : a.kst;
    const int64_t head = (int64_t)b * st.b + (int64_t)h * st.h;
    uint4 raw[kReadUnroll];
    float sc[kReadUnroll];
    int row[kReadUnroll], piece[kReadUnroll];
    bool ok[kReadUnroll];
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        const unsigned at = ((unsigned)block * kReadUnroll + u) * kReadThreads + threadIdx.x;
        row[u] = (int)(at / (unsigned)a.pieces);
        piece[u] = (int)(at - (unsigned)row[u] * (unsigned)a.pieces);
        const int64_t src = first + row[u];
        ok[u] = row[u] < count && src >= 0 && src < a.Smax;
        if (ok[u]) {
            const int64_t r = (int64_t)bh * a.Smax + src;
            raw[u] = *reinterpret_cast<const uint4*>(cache + (r * a.pieces + piece[u]) * 16);
            if constexpr (FMT != kCache16) sc[u] = scales[r];
        }
    }
#pragma unroll
    for (int u = 0; u < kReadUnroll; ++u) {
        if (!ok[u]) continue;
        uint8_t* dst = out + (head + (int64_t)row[u] * st.s) * 2 + piece[u] * (FMT == kCache16 ? 16 : 32);
        if constexpr (FMT == kCache16) {
            *reinterpret_cast<uint4*>(dst) = raw[u];
        } else {
            constexpr bool E = FMT == kCacheE4m3;
            const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t f = flip_codes<E>(w[i]);
                o[2 * i] = scaled_pair<F16>(codes_to_half2<E, false>(f), sc[u]);
                o[2 * i + 1] = scaled_pair<F16>(codes_to_half2<E, true>(f), sc[u]);
            }
            reinterpret_cast<uint4*>(dst)[0] = make_uint4(o[0], o[1], o[2], o[3]);
            reinterpret_cast<uint4*>(dst)[1] = make_uint4(o[4], o[5], o[6], o[7]);
        }
    }
}

template <int FMT, bool F16>
int launch_read(ReadArgs& a, int B, cudaStream_t s) {
    const long long per_head = (long long)a.S * a.pieces;
    const long long blocks = (per_head + kReadThreads * kReadUnroll - 1) / (kReadThreads * kReadUnroll);
    if (per_head >= (1LL << 31)) return FORGE_ERR_UNSUPPORTED;  // counted in 32 bits
    if (blocks * B * a.Hkv > 0x7fffffffLL) return FORGE_ERR_UNSUPPORTED;
    a.blocks = (int)blocks;
    FORGE_CUDA_TRY(launch_pdl(read_rows_kernel<FMT, F16>, dim3((unsigned)(blocks * B * a.Hkv), 2), dim3(kReadThreads), 0, s, a));
    return finish_launch(1);
}

}  // namespace
}  // namespace forge

extern "C" int forge_rotary_frequencies(int dims, double base, const forge_rotary_scaling* scaling, float* inv_freq, float* amplitude) {
    const double kTwoPi = 6.283185307179586476925286766559;
    if (!inv_freq || !amplitude || dims < 2 || dims % 2 != 0 || !(base > 1.0) || !std::isfinite(base)) return FORGE_ERR_INVALID_ARG;
    const int kind = scaling ? scaling->kind : FORGE_ROTARY_SCALE_NONE;
    if (kind < FORGE_ROTARY_SCALE_NONE || kind > FORGE_ROTARY_SCALE_RAMP_WAVELENGTH) return FORGE_ERR_INVALID_ARG;
    double factor = 1.0, lo = 0.0, hi = 0.0;
    if (kind != FORGE_ROTARY_SCALE_NONE) {
        factor = scaling->factor;
        if (!(factor >= 1.0) || !std::isfinite(factor)) return FORGE_ERR_INVALID_ARG;
    }
    if (kind == FORGE_ROTARY_SCALE_BASE) {
        if (dims <= 2) return FORGE_ERR_INVALID_ARG;
        base *= std::pow(factor, (double)dims / (dims - 2));
    }
    const bool ramp = kind == FORGE_ROTARY_SCALE_RAMP_ROTATIONS || kind == FORGE_ROTARY_SCALE_RAMP_WAVELENGTH;
    if (ramp && (!(scaling->slow > 0.0) || !(scaling->fast > scaling->slow) || !std::isfinite(scaling->fast) || scaling->original_len <= 0))
        return FORGE_ERR_INVALID_ARG;
    if (kind == FORGE_ROTARY_SCALE_RAMP_ROTATIONS) {
        // index whose pair makes t turns over the original length: base^(-2i/dims) len / 2 pi = t
        auto index = [&](double t) { return dims * std::log(scaling->original_len / (t * kTwoPi)) / (2.0 * std::log(base)); };
        lo = std::fmax(std::floor(index(scaling->fast)), 0.0);
        hi = std::fmin(std::ceil(index(scaling->slow)), dims - 1.0);
        if (hi <= lo) hi = lo + 0.001;
    }
    for (int i = 0; i < dims / 2; ++i) {
        double f = std::pow(base, -2.0 * i / dims);
        if (kind == FORGE_ROTARY_SCALE_LINEAR) {
            f /= factor;
        } else if (kind == FORGE_ROTARY_SCALE_RAMP_ROTATIONS) {
            const double r = std::fmin(std::fmax((i - lo) / (hi - lo), 0.0), 1.0);
            f = f * (1.0 - r) + f / factor * r;
        } else if (kind == FORGE_ROTARY_SCALE_RAMP_WAVELENGTH) {
            const double t = scaling->original_len * f / kTwoPi;
            if (t < scaling->slow) {
                f /= factor;
            } else if (t <= scaling->fast) {
                const double s = (t - scaling->slow) / (scaling->fast - scaling->slow);
                f *= s + (1.0 - s) / factor;
            }
        }
        inv_freq[i] = (float)f;
    }
    *amplitude = kind == FORGE_ROTARY_SCALE_RAMP_ROTATIONS ? (float)(0.1 * std::log(factor) + 1.0) : 1.f;
    return FORGE_OK;
}

extern "C" int forge_rotary_apply(const void* x, void* y, int dtype, int B, int H, int S, int D, const int64_t* x_strides,
                                  const int64_t* y_strides, const int32_t* positions, const int32_t* first,
                                  const forge_rotary* rotary, int inverse, void* stream) {
    using namespace forge;
    if (!x || !y || !aligned16(x) || !aligned16(y) || B <= 0 || H <= 0 || S <= 0 || D <= 0) return FORGE_ERR_INVALID_ARG;
    if (dtype < FORGE_DTYPE_BF16 || dtype > FORGE_DTYPE_F32 || misaligned4(positions) || misaligned4(first)) return FORGE_ERR_INVALID_ARG;
    RotArgs a = {};
    int st = check_rotary(rotary, D);
    if (st == FORGE_OK) st = check_strides(x_strides, H, S, D, &a.qs);
    if (st == FORGE_OK) st = check_strides(y_strides, H, S, D, &a.qos);
    if (st != FORGE_OK) return st;
    if (D % 8 != 0 || D > 256 || H > 65535) return FORGE_ERR_UNSUPPORTED;
    if (x == y && (a.qs.b != a.qos.b || a.qs.h != a.qos.h || a.qs.s != a.qos.s)) return FORGE_ERR_INVALID_ARG;
    a.q = x;
    a.q_out = y;
    a.positions = positions;
    a.first = first;
    a.B = B;
    a.Hq = H;
    a.S = a.S_src = S;
    a.D = D;
    set_rotary(a, *rotary, inverse);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return dtype == FORGE_DTYPE_F32   ? launch_rotate_only<float>(a, s)
           : dtype == FORGE_DTYPE_F16 ? launch_rotate_only<__half>(a, s)
                                      : launch_rotate_only<__nv_bfloat16>(a, s);
}

extern "C" int forge_kv_append(const forge_kv_cache* cache, const forge_kv_append_desc* desc, void* stream) {
    using namespace forge;
    if (!desc) return FORGE_ERR_INVALID_ARG;
    const forge_kv_append_desc& d = *desc;
    int st = check_cache(cache, d.dtype);
    if (st != FORGE_OK) return st;
    if (!d.k || !d.v || !aligned16(d.k) || !aligned16(d.v) || !d.lens || d.S <= 0) return FORGE_ERR_INVALID_ARG;
    if (misaligned4(d.lens) || misaligned4(d.counts) || misaligned4(d.positions) || misaligned4(d.rows)) return FORGE_ERR_INVALID_ARG;
    const int S_src = d.rows ? d.S_src : d.S;
    if (S_src <= 0) return FORGE_ERR_INVALID_ARG;
    RotArgs a = {};
    if (d.rotary && (st = check_rotary(d.rotary, cache->D)) != FORGE_OK) return st;
    if ((st = check_strides(d.k_strides, cache->Hkv, S_src, cache->D, &a.kst)) != FORGE_OK) return st;
    if ((st = check_strides(d.v_strides, cache->Hkv, S_src, cache->D, &a.vst)) != FORGE_OK) return st;
    if (d.q) {
        if (!d.q_out || !d.rotary || d.rows || d.Hq <= 0 || !aligned16(d.q) || !aligned16(d.q_out)) return FORGE_ERR_INVALID_ARG;
        if (d.Hq > 65535) return FORGE_ERR_UNSUPPORTED;
        if ((st = check_strides(d.q_strides, d.Hq, d.S, cache->D, &a.qs)) != FORGE_OK) return st;
        if ((st = check_strides(d.q_out_strides, d.Hq, d.S, cache->D, &a.qos)) != FORGE_OK) return st;
        if (d.q == d.q_out && (a.qs.b != a.qos.b || a.qs.h != a.qos.h || a.qs.s != a.qos.s)) return FORGE_ERR_INVALID_ARG;
    } else if (d.q_out) {
        return FORGE_ERR_INVALID_ARG;
    }
    a.q = d.q; a.k = d.k; a.v = d.v;
    a.q_out = d.q_out;
    a.kc = cache->k; a.vc = cache->v;
    a.ks = cache->k_scale; a.vs = cache->v_scale;
    a.positions = d.positions;
    a.first = d.lens;
    a.counts = d.counts;
    a.rows = d.rows;
    a.B = cache->B;
    a.Hq = d.q ? d.Hq : 0;
    a.Hkv = cache->Hkv;
    a.S = d.S;
    a.S_src = S_src;
    a.Smax = cache->Smax;
    a.D = cache->D;
    if (d.rotary) set_rotary(a, *d.rotary, 0);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return d.dtype == FORGE_DTYPE_F16 ? dispatch_append<__half>(cache->format, a, s) : dispatch_append<__nv_bfloat16>(cache->format, a, s);
}

extern "C" int forge_kv_read(const forge_kv_cache* cache, void* k_out, void* v_out, int dtype, int S, const int64_t* k_strides,
                             const int64_t* v_strides, const int32_t* first, const int32_t* counts, void* stream) {
    using namespace forge;
    int st = check_cache(cache, dtype);
    if (st != FORGE_OK) return st;
    if (!k_out || !v_out || !aligned16(k_out) || !aligned16(v_out) || S <= 0 || misaligned4(first) || misaligned4(counts)) return FORGE_ERR_INVALID_ARG;
    ReadArgs a = {};
    if ((st = check_strides(k_strides, cache->Hkv, S, cache->D, &a.kst)) != FORGE_OK) return st;
    if ((st = check_strides(v_strides, cache->Hkv, S, cache->D, &a.vst)) != FORGE_OK) return st;
    a.kc = cache->k; a.vc = cache->v;
    a.ks = cache->k_scale; a.vs = cache->v_scale;
    a.k_out = k_out; a.v_out = v_out;
    a.first = first; a.counts = counts;
    a.Hkv = cache->Hkv; a.Smax = cache->Smax; a.S = S; a.D = cache->D;
    a.pieces = eight_bit(cache->format) ? cache->D / 16 : cache->D / 8;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool f16 = dtype == FORGE_DTYPE_F16;
    switch (cache->format) {
        case FORGE_KV_INT8: return f16 ? launch_read<kCacheInt8, true>(a, cache->B, s) : launch_read<kCacheInt8, false>(a, cache->B, s);
        case FORGE_KV_E4M3: return f16 ? launch_read<kCacheE4m3, true>(a, cache->B, s) : launch_read<kCacheE4m3, false>(a, cache->B, s);
        default: return launch_read<kCache16, false>(a, cache->B, s);
    }
}
