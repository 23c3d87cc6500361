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

template <int DT> struct Elem;
template <> struct Elem<APC_F32> { using T = float; };
template <> struct Elem<APC_F16> { using T = uint16_t; };
template <> struct Elem<APC_BF16> { using T = uint16_t; };
template <> struct Elem<APC_E4M3> { using T = uint8_t; };

using f32x2 = float __attribute__((ext_vector_type(2)));
using f16x2 = _Float16 __attribute__((ext_vector_type(2)));
using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));

// N elements at p as they lie there; p needs only its element's alignment
// (global loads of 16 bytes may start anywhere)
template <int DT, int N> struct Raw {
    static constexpr int BYTES = N * (int)sizeof(typename Elem<DT>::T);
    uint32_t w[(BYTES + 3) / 4];
    __device__ void load(const typename Elem<DT>::T* p) { __builtin_memcpy(w, p, BYTES); }
    __device__ void values(float* v) const
    {
        if constexpr (DT == APC_F32) {
            __builtin_memcpy(v, w, BYTES);
        } else if constexpr (DT == APC_E4M3) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(w[i], true);
                v[4 * i] = lo.x, v[4 * i + 1] = lo.y, v[4 * i + 2] = hi.x, v[4 * i + 3] = hi.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t u = i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu;
                if constexpr (DT == APC_BF16) {
                    v[i] = __uint_as_float(u << 16);
                } else {
                    const uint16_t s = (uint16_t)u;
                    _Float16 h;
                    __builtin_memcpy(&h, &s, 2);
                    v[i] = (float)h;
                }
            }
        }
    }
};

// N dwords to p, wherever it starts.  `past`: marked not to stay in the caches,
// for outputs larger than they are (whole lines only: a part of a line costs
// its line's read and write)
template <int N, typename P> __device__ inline void store_dwords(P* p, const uint32_t* w, bool past)
{
    if constexpr (N == 2 || N == 4) {
        typedef uint32_t V __attribute__((ext_vector_type(N), aligned(1)));
        if (past) {
            V x;
            __builtin_memcpy(&x, w, 4 * N);
            __builtin_nontemporal_store(x, reinterpret_cast<V*>(p));
            return;
        }
    }
    __builtin_memcpy(p, w, 4 * N);
}

// N values rounded to nearest-even into the type at p, wherever it starts
// (f32, f16 and bf16: the hardware's conversions, which equal enc_f16 and
// enc_bf16 on every float32 but for the payload of a half's NaN)
template <int DT, int N> __device__ inline void store_values(typename Elem<DT>::T* p, const float* v, bool past = false)
{
    if constexpr (DT == APC_F32) {
        uint32_t w[N];
        __builtin_memcpy(w, v, 4 * N);
#pragma unroll
        for (int i = 0; i < N; i += 4) store_dwords<(N < 4 ? N : 4)>(p + i, w + i, past);
    } else {
        uint32_t w[(N + 1) / 2];
#pragma unroll
        for (int i = 0; i < (N + 1) / 2; ++i) {
            const f32x2 x = {v[2 * i], 2 * i + 1 < N ? v[2 * i + 1] : 0.f};
            if constexpr (DT == APC_BF16) {
                const bf16x2 b = __builtin_convertvector(x, bf16x2);
                __builtin_memcpy(&w[i], &b, 4);
            } else {
                const f16x2 h = __builtin_convertvector(x, f16x2);
                __builtin_memcpy(&w[i], &h, 4);
            }
        }
        if constexpr (N % 2 == 0) {
#pragma unroll
            for (int i = 0; i < N / 2; i += 4) store_dwords<(N / 2 < 4 ? N / 2 : 4)>(p + 2 * i, w + i, past);
        } else {
            __builtin_memcpy(p, w, 2 * N);
        }
    }
}

// |x| as an integer: orders like the magnitudes, NaN above infinity
__device__ inline uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Sums and largest values over groups of T = 4 .. 64 consecutive lanes, the
// result in each: exchanges within 16 lanes ride on the operation (DPP), the
// others swap rows of 16 lanes or halves of the wave.
template <int CTRL> __device__ inline uint32_t lane_moved(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <int T, typename F> __device__ inline uint32_t over_lanes(uint32_t x, F f)
{
    x = f(x, lane_moved<0xb1>(x));                          // 1 0 3 2
    x = f(x, lane_moved<0x4e>(x));                          // 2 3 0 1
    if constexpr (T >= 8) x = f(x, lane_moved<0x141>(x));   // mirror of 8
    if constexpr (T >= 16) x = f(x, lane_moved<0x140>(x));  // mirror of 16
    if constexpr (T >= 32) {
        const auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = f(y[0], y[1]);
    }
    if constexpr (T >= 64) {
        const auto y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = f(y[0], y[1]);
    }
    return x;
}
template <int T> __device__ inline float sum_over(float x)
{
    return __uint_as_float(over_lanes<T>(__float_as_uint(x), [](uint32_t a, uint32_t b) {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }));
}
template <int T> __device__ inline uint32_t max_over(uint32_t x)
{
    return over_lanes<T>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

// Scale of an e4m3fn row from its largest magnitude, and the codes of x / s.
// top / 448 and r = 1 / s are approximations corrected by their remainders;
// from 2^-80 on they equal the divisions on every float32 (compared over all).
// With r, q = x r corrected by the remainder s q - x (exact in a fused
// multiply-add) is the correctly rounded quotient wherever neither r nor the
// remainder leaves the normal range: s >= 2^-80 leaves it only for quotients
// below 2^-20, code 0 either way.  (Remainder and correction are both negated,
// so that -0 stays -0.)  Such a row's quotients are at most 448 and two units in
// the last place, which the hardware's conversion (nearest-even, equal to
// enc_e4m3 there) takes to 448.  Other rows (NaN, infinite or tiny) divide and
// round by the definition.
struct RowCodes {
    float s, r;
    bool plain;
    __device__ explicit RowCodes(uint32_t top)
    {
        plain = top >= 0x1c000000u && top < 0x7f800000u;    // from 2^-71
        if (plain) {
            constexpr float part = 1.0f / 448.0f;
            const float t = __uint_as_float(top), q = t * part;
            s = __builtin_fmaf(__builtin_fmaf(-448.0f, q, t), part, q);
            const float y = __builtin_amdgcn_rcpf(s);
            r = __builtin_fmaf(__builtin_fmaf(-s, y, 1.0f), y, y);
        } else {
            s = top > 0x7f800000u ? 1.0f : __uint_as_float(top) / 448.0f;
            if (!(s > 0.f)) s = 1.0f;
            r = 1.0f;
            plain = top == 0u;
        }
    }
    __device__ float quotient(float x) const
    {
        const float q = x * r;
        return __builtin_fmaf(-__builtin_fmaf(s, q, -x), r, q);
    }
    __device__ uint32_t code(float x) const
    {
        const float y = x / s;
        return enc_e4m3(y == y ? __builtin_fminf(__builtin_fmaxf(y, -448.0f), 448.0f) : y);
    }
    // ONE_BY_ONE: the divisions of other rows are not put side by side, where N of
    // them would take registers from the plain rows' path (norm of 994,131 x 112 bf16
    // to e4m3: 92 us, 104 without; kv.hip's 77,777 x 20 x 32: 74.5 and 72.7)
    template <int N, bool ONE_BY_ONE = false> __device__ void store(uint8_t* p, const float* v, bool past = false) const
    {
        if constexpr (N == 1) {
            *p = (uint8_t)code(*v);
            return;
        }
        uint32_t w[(N + 3) / 4];
        if (plain) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[4 * i]), quotient(v[4 * i + 1]), 0, false);
                w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(v[4 * i + 2]), quotient(v[4 * i + 3]), w[i], true);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                w[i / 4] = (i % 4 ? w[i / 4] : 0u) | code(v[i]) << i % 4 * 8;
                if constexpr (ONE_BY_ONE) __builtin_amdgcn_sched_barrier(0);
            }
        }
        store_dwords<N / 4>(p, w, past);
    }
};

}  // namespace apc
