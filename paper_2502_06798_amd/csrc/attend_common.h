// What the attention kernels share: operand types, conversions of pairs of
// values in 16 bits, and reads of tables that all lanes share.
#pragma once

#include "apc_internal.h"
#include "convert.h"

namespace apc {

// The kernel's parts are lambdas that hold its state in registers, so all of them have to be inlined.
#define INLINE __attribute__((always_inline))

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.0e38f;      // below every score; finite, so that exp2(-inf - m) is 0

using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

template <bool BF> __device__ inline uint32_t pack(float a, float b)
{
    const f32x2 x = {a, b};
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
}

template <bool BF> __device__ inline f32x2 unpack(uint32_t w)
{
    if constexpr (BF) return f32x2{__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)};
    else return __builtin_convertvector(__builtin_bit_cast(f16x2, w), f32x2);
}

// two e4m3 codes (the low or the high half of w) in 16 bits: exact
template <bool BF, bool HIGH> __device__ inline uint32_t from_e4m3(uint32_t w)
{
    if constexpr (BF) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HIGH));
}

// the halves of w that hold infinities or NaN, as a mask
template <bool BF> __device__ inline uint32_t not_finite(uint32_t w)
{
    constexpr uint32_t EXP = BF ? 0x7f80u : 0x7c00u;
    return ((w & EXP) == EXP ? 0xffffu : 0u) | ((w >> 16 & EXP) == EXP ? 0xffff0000u : 0u);
}

// An entry of an input table at an index that all lanes share.  The tables do
// not change while the kernel runs, which the compiler cannot know; as constant
// memory they are read with scalar loads, and what follows from them stays in
// scalar registers.
__device__ inline int32_t table_entry(const int32_t* table, int64_t i)
{
    return ((const __attribute__((address_space(4))) int32_t*)table)[i];
}

}  // namespace apc
