// What the operators on a KV cache share (kv_cache.cu, attn_kv.cu): argument checks and the conversions of 8-bit codes.
#pragma once

#include <cuda_fp16.h>
#include <cstdint>

#include "forge_common.cuh"

namespace forge {

inline bool eight_bit(int format) { return format == FORGE_KV_INT8 || format == FORGE_KV_E4M3; }

// A cache and the activations' type that goes with it.
inline int check_cache(const forge_kv_cache* c, int dtype) {
    if (!c || !c->k || !c->v || c->B <= 0 || c->Hkv <= 0 || c->Smax <= 0 || c->D <= 0) return FORGE_ERR_INVALID_ARG;
    if (c->format < FORGE_KV_BF16 || c->format > FORGE_KV_E4M3) return FORGE_ERR_INVALID_ARG;
    if (dtype != FORGE_DTYPE_BF16 && dtype != FORGE_DTYPE_F16) return dtype == FORGE_DTYPE_F32 ? FORGE_ERR_UNSUPPORTED : FORGE_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v)) return FORGE_ERR_INVALID_ARG;
    if (eight_bit(c->format)) {
        if (!c->k_scale || !c->v_scale || !aligned16(c->k_scale) || !aligned16(c->v_scale)) return FORGE_ERR_INVALID_ARG;
        if (c->D % 16 != 0) return FORGE_ERR_UNSUPPORTED;
    } else if (dtype != (c->format == FORGE_KV_F16 ? FORGE_DTYPE_F16 : FORGE_DTYPE_BF16)) {
        return FORGE_ERR_INVALID_ARG;
    }
    if (c->D > 128 || c->D % 8 != 0 || c->B > 65535 || c->Hkv > 65535) return FORGE_ERR_UNSUPPORTED;
    // rows of the whole cache are counted in 32 bits (their elements are not)
    if ((long long)c->B * c->Hkv * (((long long)c->Smax + 127) / 128 * 128) >= (1LL << 31)) return FORGE_ERR_UNSUPPORTED;
    return FORGE_OK;
}

// Element strides {batch, head, token} of a view; the dense ones for NULL.
struct Strides { int64_t b, h, s; };
inline int check_strides(const int64_t* in, int H, int S, int D, Strides* out) {
    *out = {(int64_t)H * S * D, (int64_t)S * D, D};
    if (!in) return FORGE_OK;
    *out = {in[0], in[1], in[2]};
    for (int i = 0; i < 3; ++i)
        if (in[i] <= 0) return FORGE_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (in[i] % 8 != 0) return FORGE_ERR_UNSUPPORTED;
    return FORGE_OK;
}

#ifdef __CUDACC__
// Codes to fp16, two at a time, exactly.  Word w holds four codes.
//   int8: the byte with its top bit flipped is x + 128; put below 0x64 it is the fp16 number 1024 + x + 128.
//   e4m3: a conversion of two codes in the lower half of a register.  NaN codes become NaN; e4m3_finite makes them 448, for operands of
//   products in which they meet zeros that have to stay zeros.
__device__ __forceinline__ uint32_t sub_1152(uint32_t h2) {
    const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&h2), __half2half2(__ushort_as_half((unsigned short)0x6480)));
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t two) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
    return h;
}
__device__ __forceinline__ uint32_t e4m3_finite(uint32_t h2) {
    const __half2 r = __hmin2(*reinterpret_cast<const __half2*>(&h2), __half2half2(__ushort_as_half((unsigned short)0x5f00)));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// the codes in bytes 0, 1 (HI: 2, 3) of a word; int8 words have passed through flip_codes()
template <bool E4M3>
__device__ __forceinline__ uint32_t flip_codes(uint32_t w) { return E4M3 ? w : w ^ 0x80808080u; }
template <bool E4M3, bool HI>
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t w) {
    if constexpr (E4M3) {
        return e4m3_pair(HI ? w >> 16 : w);
    } else {
        return sub_1152(__byte_perm(w, 0x64646464u, HI ? 0x4342 : 0x4140));
    }
}
#endif

}  // namespace forge
