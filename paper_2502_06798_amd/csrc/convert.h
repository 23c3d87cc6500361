// Conversions between float32 and the storage types, shared by the kernels
// that write rows (quantize.hip, norm.hip, kv.hip) and read them back.
#pragma once

#include "apc_internal.h"

namespace apc {

__device__ inline uint32_t enc_f16(float x)
{
    const _Float16 h = (_Float16)x;
    uint16_t b;
    __builtin_memcpy(&b, &h, 2);
    if (x != x) b = (uint16_t)(((__float_as_uint(x) >> 16) & 0x8000u) | 0x7e00u);   // quiet NaN, sign kept
    return b;
}

__device__ inline uint32_t enc_bf16(float x)
{
    const uint32_t u = __float_as_uint(x);
    if (x != x) return ((u >> 16) | 0x0040u) & 0xffffu;          // quiet NaN, sign and top payload kept
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;                 // nearest-even; a carry may reach +-Inf
}

// e4m3fn code of y (|y| <= 448 or NaN), rounded to nearest-even
__device__ inline uint32_t enc_e4m3(float y)
{
    const uint32_t u = __float_as_uint(y);
    const uint32_t sign = (u >> 24) & 0x80u;
    if (y != y) return sign | 0x7fu;
    const uint32_t a = u & 0x7fffffffu;
    uint32_t code;
    if (a < 0x3c800000u) {
        // below 2^-6: the subnormal codes m 2^-9 (m = 8 is the smallest
        // normal); |y| 512 is exact, rint rounds it to nearest-even
        code = (uint32_t)__builtin_rintf(__uint_as_float(a) * 512.0f);
    } else {
        // keep the top 3 of the 23 mantissa bits, nearest-even (a carry moves
        // into the exponent), and rebias the exponent from 127 to 7
        const uint32_t q = a >> 20, rem = a & 0xfffffu;
        const uint32_t up = rem > 0x80000u || (rem == 0x80000u && (q & 1u)) ? 1u : 0u;
        code = q + up - ((127u - 7u) << 3);
    }
    return sign | code;
}

// codes of e4m3fn rows: amax (of |x|; NaN elements reported apart) to the row's scale
__device__ inline float e4m3_scale(float amax, bool nan)
{
    const float s = nan ? 1.0f : amax / 448.0f;
    return s > 0.f ? s : 1.0f;
}

__device__ inline float e4m3_clamp(float y)
{
    return y == y ? __builtin_fminf(__builtin_fmaxf(y, -448.0f), 448.0f) : y;
}

template <int DT> struct Elem;
template <> struct Elem<APC_F32> { using T = float; };
template <> struct Elem<APC_F16> { using T = uint16_t; };
template <> struct Elem<APC_BF16> { using T = uint16_t; };
template <> struct Elem<APC_E4M3> { using T = uint8_t; };

template <int DT> __device__ inline float load_elem(const typename Elem<DT>::T* p)
{
    if constexpr (DT == APC_F32) {
        return *p;
    } else if constexpr (DT == APC_F16) {
        _Float16 h;
        __builtin_memcpy(&h, p, 2);
        return (float)h;
    } else if constexpr (DT == APC_BF16) {
        return __uint_as_float((uint32_t)*p << 16);
    } else {
        return __builtin_amdgcn_cvt_f32_fp8((int)*p, 0);
    }
}

template <int DT> __device__ inline void store_elem(typename Elem<DT>::T* p, float x)
{
    if constexpr (DT == APC_F32) *p = x;
    else if constexpr (DT == APC_F16) *p = (uint16_t)enc_f16(x);
    else if constexpr (DT == APC_BF16) *p = (uint16_t)enc_bf16(x);
    else *p = (uint8_t)enc_e4m3(x);
}

}  // namespace apc
