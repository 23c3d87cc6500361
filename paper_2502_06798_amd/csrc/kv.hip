// Paged key-value cache: new tokens' keys and values written into their slots,
// rounded or quantised on the way, and slots read back as rows.
//
// One wavefront per (token, head, key or value) row of d elements, a lane
// keeping every 64th.
#include "apc_internal.h"
#include "convert.h"

namespace apc {
namespace {

constexpr int64_t MAX_GRID = 1 << 20;   // more rows: a wavefront takes several
constexpr int PER = APC_MAX_HEAD_DIM / 64;

struct Row {
    int64_t tok;
    int32_t head, which;
};

__device__ inline Row which_row(int64_t r, int32_t heads)
{
    return {r / (2 * heads), (int32_t)(r % (2 * heads)) / 2, (int32_t)(r & 1)};
}

// row number of a slot's head inside k and v, or -1
__device__ inline int64_t slot_row(const apc_kv& c, int32_t slot, int32_t head)
{
    if (slot < 0 || slot >= c.n_pages * c.page) return -1;
    return ((int64_t)(slot / c.page) * c.heads + head) * c.page + slot % c.page;
}

template <int DT, int CDT>
__global__ __launch_bounds__(256) void k_kv_write(apc_kv c, KvRows a)
{
    using T = typename Elem<DT>::T;
    using C = typename Elem<CDT>::T;
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.t * 2 * c.heads; r += (int64_t)gridDim.x * 4) {
    const Row w = which_row(r, c.heads);
    const int64_t row = slot_row(c, a.slots[w.tok], w.head);
    if (row < 0) continue;
    const T* x = static_cast<const T*>(w.which ? a.v : a.k) +
                 (w.which ? w.tok * a.v_tok + w.head * a.v_head : w.tok * a.k_tok + w.head * a.k_head);
    C* out = static_cast<C*>(w.which ? c.v : c.k) + row * c.d;
    float e[PER], amax = 0.f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        e[i] = lane + 64 * i < c.d ? load_elem<DT>(x + lane + 64 * i) : 0.f;
        nan |= e[i] != e[i];
        amax = __builtin_fmaxf(amax, __builtin_fabsf(e[i]));
    }
    float s = 1.f;
    if constexpr (CDT == APC_E4M3) {
        for (int m = 32; m >= 1; m >>= 1) amax = __builtin_fmaxf(amax, __shfl_xor(amax, m, 64));
        s = e4m3_scale(amax, __any(nan));
        if (lane == 0) (w.which ? c.v_scale : c.k_scale)[row] = s;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (lane + 64 * i < c.d)
            store_elem<CDT>(out + lane + 64 * i, CDT == APC_E4M3 ? e4m3_clamp(e[i] / s) : e[i]);
    }
}

template <int DT, int CDT>
__global__ __launch_bounds__(256) void k_kv_read(apc_kv c, KvRows a)
{
    using T = typename Elem<DT>::T;
    using C = typename Elem<CDT>::T;
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.t * 2 * c.heads; r += (int64_t)gridDim.x * 4) {
    const Row w = which_row(r, c.heads);
    const int64_t row = slot_row(c, a.slots[w.tok], w.head);
    T* out = static_cast<T*>(w.which ? a.v : a.k) +
             (w.which ? w.tok * a.v_tok + w.head * a.v_head : w.tok * a.k_tok + w.head * a.k_head);
    float s = 1.f;
    if (CDT == APC_E4M3 && row >= 0) s = (w.which ? c.v_scale : c.k_scale)[row];
    for (int i = lane; i < c.d; i += 64) {
        float x = 0.f;
        if (row >= 0) x = load_elem<CDT>(static_cast<const C*>(w.which ? c.v : c.k) + row * c.d + i) * s;
        store_elem<DT>(out + i, x);
    }
    }
}

template <int DT, int CDT>
void launch(bool write, const apc_kv& c, const KvRows& a, hipStream_t s)
{
    const int64_t groups = (a.t * 2 * c.heads + 3) / 4;
    const dim3 grid((unsigned)(groups < MAX_GRID ? groups : MAX_GRID)), block(256);
    if (write) k_kv_write<DT, CDT><<<grid, block, 0, s>>>(c, a);
    else k_kv_read<DT, CDT><<<grid, block, 0, s>>>(c, a);
}

template <int DT>
hipError_t launch_to(bool write, const apc_kv& c, const KvRows& a, hipStream_t s)
{
    switch (c.dt) {
    case APC_F16: launch<DT, APC_F16>(write, c, a, s); break;
    case APC_BF16: launch<DT, APC_BF16>(write, c, a, s); break;
    case APC_E4M3: launch<DT, APC_E4M3>(write, c, a, s); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_rows(bool write, int dt, const apc_kv& c, const KvRows& a, hipStream_t s)
{
    if (a.t <= 0) return hipSuccess;
    switch (dt) {
    case APC_F32: return launch_to<APC_F32>(write, c, a, s);
    case APC_F16: return launch_to<APC_F16>(write, c, a, s);
    case APC_BF16: return launch_to<APC_BF16>(write, c, a, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
