// Attention of one new token per sequence over a paged key-value cache.
//
// One wavefront per (sequence, query head): its lanes share the head's
// elements, and the tokens follow one another under a running maximum m and
// sum l (float32): with m' = max(m, s), l and the output's sums are scaled by
// exp(m - m') before the token's exp(s - m') joins them.
#include "apc_internal.h"
#include "convert.h"

#include <cmath>

namespace apc {
namespace {

constexpr int PER = APC_MAX_HEAD_DIM / 64;

template <int DT> __device__ inline float one(const typename Elem<DT>::T* p)
{
    if constexpr (DT == APC_E4M3) return __builtin_amdgcn_cvt_f32_fp8((int)*p, 0);
    else {
        Raw<DT, 1> r;
        float v;
        r.load(p);
        r.values(&v);
        return v;
    }
}

template <int DT, int CDT>
__global__ __launch_bounds__(64) void k_attend_rows(apc_kv c, AttendArgs a)
{
    using T = typename Elem<DT>::T;
    using C = typename Elem<CDT>::T;
    const int lane = threadIdx.x;
    const int32_t i = blockIdx.x / a.q_heads, qh = blockIdx.x % a.q_heads, h = qh / (a.q_heads / c.heads);
    const T* q = static_cast<const T*>(a.q) + i * a.q_row + qh * a.q_head;
    float qv[PER], o[PER], m = -3.0e38f, l = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        qv[e] = lane + 64 * e < c.d ? one<DT>(q + lane + 64 * e) * a.scale : 0.f;
        o[e] = 0.f;
    }
    const int64_t cap = (int64_t)a.max_pages * c.page;
    int64_t len = a.lengths[i];
    len = len < 0 ? 0 : len > cap ? cap : len;
    const int64_t first = a.window > 0 && len > a.window ? len - a.window : 0;
    for (int64_t j = first; j < len; ++j) {
        const int32_t p = a.pages[i * a.ld_pages + j / c.page];
        if (p < 0 || p >= c.n_pages) continue;
        const int64_t row = ((int64_t)p * c.heads + h) * c.page + j % c.page;
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (lane + 64 * e < c.d) s += qv[e] * one<CDT>(static_cast<const C*>(c.k) + row * c.d + lane + 64 * e);
        for (int x = 32; x >= 1; x >>= 1) s += __shfl_xor(s, x, 64);
        float vs = 1.f;
        if constexpr (CDT == APC_E4M3) {
            s *= c.k_scale[row];
            vs = c.v_scale[row];
        }
        const float to = __builtin_fmaxf(m, s), was = expf(m - to), p1 = expf(s - to);
        m = to;
        l = l * was + p1;
#pragma unroll
        for (int e = 0; e < PER; ++e)
            if (lane + 64 * e < c.d)
                o[e] = o[e] * was + p1 * vs * one<CDT>(static_cast<const C*>(c.v) + row * c.d + lane + 64 * e);
    }
    T* out = static_cast<T*>(a.out) + i * a.out_row + qh * a.out_head;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
            const float v = l == 0.f ? 0.f : o[e] / l;
            if (lane + 64 * e < c.d) store_values<DT, 1>(out + lane + 64 * e, &v);
        }
    if (a.lse && lane == 0) a.lse[(int64_t)i * a.q_heads + qh] = l == 0.f ? -INFINITY : m + logf(l);
}

template <int DT, int CDT>
void launch(const apc_kv& c, const AttendArgs& a, hipStream_t s)
{
    k_attend_rows<DT, CDT><<<dim3((unsigned)a.b * a.q_heads), dim3(64), 0, s>>>(c, a);
}

}  // namespace

size_t attend_workspace(const apc_kv&, int32_t, int32_t, int32_t) { return 256; }

hipError_t launch_attend(int dt, const apc_kv& c, const AttendArgs& a, hipStream_t s)
{
    if (a.b <= 0) return hipSuccess;
    if (c.dt == APC_E4M3) {
        if (dt == APC_F16) launch<APC_F16, APC_E4M3>(c, a, s);
        else launch<APC_BF16, APC_E4M3>(c, a, s);
    } else if (dt == APC_F16) {
        launch<APC_F16, APC_F16>(c, a, s);
    } else {
        launch<APC_BF16, APC_BF16>(c, a, s);
    }
    return hipGetLastError();
}

}  // namespace apc
