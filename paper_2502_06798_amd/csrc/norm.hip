// Root-mean-square norm of rows with the residual's addition before it, to the
// rows' type or to e4m3 codes with a scale per row.
//
// One workgroup of 1024 threads per row; a thread keeps every 1024th element
// of the row in float32 registers, so the row is read once and the sum of
// squares, the largest |y| and the outputs all come from registers.
#include "apc_internal.h"
#include "convert.h"

namespace apc {
namespace {

constexpr int64_t MAX_GRID = 1 << 20;   // more rows than workgroups: a workgroup takes several
constexpr int NT = 1024, PER = APC_MAX_NORM_D / NT;

__device__ inline float block_sum(float v, float* red)
{
    for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < NT / 64; ++i) v += red[i];
    return v;
}

__device__ inline float block_max(float v, float* red)
{
    for (int m = 32; m >= 1; m >>= 1) v = __builtin_fmaxf(v, __shfl_xor(v, m, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < NT / 64; ++i) v = __builtin_fmaxf(v, red[i]);
    return v;
}

template <int DT, int ODT>
__global__ __launch_bounds__(NT) void k_norm_rows(NormArgs a)
{
    using T = typename Elem<DT>::T;
    using O = typename Elem<ODT>::T;
    __shared__ float red[NT / 64];
    for (int64_t r = blockIdx.x; r < a.n; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.ld_x;
        const T* res = a.res ? static_cast<const T*>(a.res) + r * a.ld_res : nullptr;
        const T* w = static_cast<const T*>(a.weight);
        T* sum = a.sum ? static_cast<T*>(a.sum) + r * a.ld_sum : nullptr;
        O* out = static_cast<O*>(a.out) + r * a.ld_out;
        float h[PER], ss = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = i * NT + threadIdx.x;
            h[i] = 0.f;
            if (c < a.d) {
                h[i] = load_elem<DT>(x + c);
                if (res) h[i] += load_elem<DT>(res + c);
                if (sum) store_elem<DT>(sum + c, h[i]);
                ss += h[i] * h[i];
            }
        }
        ss = block_sum(ss, red);
        const float f = 1.0f / __builtin_sqrtf(ss / (float)a.d + a.eps);
        float amax = 0.f, nan = 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = i * NT + threadIdx.x;
            if (c < a.d) {
                h[i] *= f;
                if (w) h[i] *= load_elem<DT>(w + c);
                if (h[i] != h[i]) nan = 1.f;
                amax = __builtin_fmaxf(amax, __builtin_fabsf(h[i]));
            }
        }
        float s = 1.f;
        if constexpr (ODT == APC_E4M3) {
            amax = block_max(amax, red);
            nan = block_max(nan, red);
            s = e4m3_scale(amax, nan != 0.f);
            if (threadIdx.x == 0) a.out_scale[r] = s;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int c = i * NT + threadIdx.x;
            if (c < a.d) store_elem<ODT>(out + c, ODT == APC_E4M3 ? e4m3_clamp(h[i] / s) : h[i]);
        }
    }
}

template <int DT>
hipError_t launch(int out_dt, const NormArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)(a.n < MAX_GRID ? a.n : MAX_GRID)), block(NT);
    if (out_dt == APC_E4M3) k_norm_rows<DT, APC_E4M3><<<grid, block, 0, s>>>(a);
    else k_norm_rows<DT, DT><<<grid, block, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm_rows(int dt, int out_dt, const NormArgs& a, hipStream_t s)
{
    if (a.n <= 0) return hipSuccess;
    switch (dt) {
    case APC_F32: return launch<APC_F32>(out_dt, a, s);
    case APC_F16: return launch<APC_F16>(out_dt, a, s);
    case APC_BF16: return launch<APC_BF16>(out_dt, a, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
