// Root-mean-square norm of rows with the residual's addition before it, to the
// rows' type or to e4m3 codes with a scale per row.
//
// T threads share a row and keep it in float32 registers, C chunks of 16 bytes
// each, so the row and the residual are read once and everything after the first
// reduction comes from registers.  y = (h f) w with the row's factor f, in this
// order: h w alone can leave float32's range where y does not.  e4m3 rows need
// the largest |y|, a second reduction.  Bound by memory: each row's bytes once.
// 65,536 x 4,096 bf16 with residual to e4m3 311 us, 6.0 TB/s (a large copy
// reaches 4.6); short rows to e4m3 by the arithmetic of a row's scale (994,131 x
// 112: 90 us, 3.7).
//
// A row that does not end on a chunk ends with a chunk moved back to the row's
// end: its first `skip` elements are another thread's too, left out of the sum
// and stored by both with the same bits.  Every load of a row comes before the
// first reduction and every store after it, so that outputs may be the inputs' rows.
#include "apc_internal.h"
#include "convert.h"

namespace apc {
namespace {

// Bytes of output from which it goes past the caches, where nobody would find
// it again (65,536 x 1,024 bf16 with residual: 91 us, 94 without; 100,000 x 768 f16: 50 and 53).
constexpr int64_t PAST_CACHES = 64 << 20;
constexpr int64_t MAX_GRID = 1 << 20;   // more rows than that many workgroups hold: a workgroup takes several

// 1 / sqrt(x) to a unit in the last place; x below the normal range (tiny rows
// with eps = 0) scaled up first, where the instruction would take it for 0
__device__ inline float rsqrt_of(float x)
{
    const bool tiny = x < 0x1p-120f;
    const float y = __builtin_amdgcn_rsqf(tiny ? x * 0x1p60f : x);
    return tiny ? y * 0x1p30f : y;
}

template <int DT, int ODT, int T, int C>
__global__ __launch_bounds__(T > 256 ? T : 256) void k_norm_rows(NormArgs a)
{
    using E = typename Elem<DT>::T;
    using O = typename Elem<ODT>::T;
    constexpr int V = 16 / sizeof(E), ROWS = T > 256 ? 1 : 256 / T, WAVES = T / 64;
    // up to three chunks a thread, the weight is loaded with the row; longer rows
    // have no registers for it until the row is normed, and float32 rows beyond
    // 16,384, with eight chunks, not for all of the residual either: they spill
    // (4,096 x 32,768 with residual to e4m3: 715 us, 2.4 TB/s)
    constexpr bool KEEP_W = C <= 3;
    constexpr int CELLS = WAVES > 1 ? WAVES : 1;
    __shared__ float red_s[2][ROWS][CELLS];
    __shared__ uint32_t red_m[2][ROWS][CELLS];
    const int t = threadIdx.x % T, own = threadIdx.x / T;
    const E* w = static_cast<const E*>(a.weight);
    int turn = 0;
    // every thread of the workgroup goes round as often: threads past the last
    // row read that row once more and store nothing
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.n; r0 += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const bool live = r0 + own < a.n;
        const int64_t r = live ? r0 + own : a.n - 1;
        const E* x = static_cast<const E*>(a.x) + r * a.ld_x;
        const E* res = static_cast<const E*>(a.res) + (a.res ? r * a.ld_res : 0);
        Raw<DT, V> rx[C], rr[C], rw[C];                         // (rw: KEEP_W only)
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * T + t) * V, from = at < a.d - V ? at : a.d - V;
            if (at < a.d) {
                rx[c].load(x + from);
                if (a.res) rr[c].load(res + from);
                if (KEEP_W && a.weight) rw[c].load(w + from);
            }
        }
        float h[C][V], ss = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            float e[V];
            rx[c].values(h[c]);
            if (a.res) {
                rr[c].values(e);
#pragma unroll
                for (int i = 0; i < V; ++i) h[c][i] += e[i];
            }
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * T + t) * V, from = at < a.d - V ? at : a.d - V, skip = at - from;
            if (at < a.d) {
                if (a.d % V == 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) ss = __builtin_fmaf(h[c][i], h[c][i], ss);
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) ss = i < skip ? ss : __builtin_fmaf(h[c][i], h[c][i], ss);
                }
            }
        }
        // two sets of cells in turn: a wave may write the next row's while another
        // still reads this row's
        ss = sum_over<(T < 64 ? T : 64)>(ss);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) red_s[turn][own][t >> 6] = ss;
            __syncthreads();
            ss = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) ss += red_s[turn][own][i];
        }
        const float f = rsqrt_of(__builtin_fmaf(ss, a.inv_d, a.eps));
        E* sum = static_cast<E*>(a.sum) + (a.sum ? r * a.ld_sum : 0);
        O* out = static_cast<O*>(a.out) + r * a.ld_out;
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = (c * T + t) * V, from = at < a.d - V ? at : a.d - V;
            if (at < a.d) {
                if (live && a.sum) store_values<DT, V>(sum + from, h[c], a.past);
                float e[V];
                if (!KEEP_W && a.weight) rw[c].load(w + from);
                if (a.weight) rw[c].values(e);
#pragma unroll
                for (int i = 0; i < V; ++i) h[c][i] = a.weight ? h[c][i] * f * e[i] : h[c][i] * f;
                if constexpr (ODT == APC_E4M3) {
#pragma unroll
                    for (int i = 0; i < V; i += 2) {
                        const uint32_t m0 = magnitude(h[c][i]), m1 = magnitude(h[c][i + 1]), m = m0 > m1 ? m0 : m1;
                        top = m > top ? m : top;
                    }
                } else {
                    if (live) store_values<ODT, V>(out + from, h[c], a.past);
                }
            }
            if constexpr (C >= 4) __builtin_amdgcn_sched_barrier(0);   // chunk by chunk: interleaved, they spill
        }
        if constexpr (ODT == APC_E4M3) {
            top = max_over<(T < 64 ? T : 64)>(top);
            if constexpr (WAVES > 1) {
                if ((threadIdx.x & 63) == 0) red_m[turn][own][t >> 6] = top;
                __syncthreads();
                top = 0;
#pragma unroll
                for (int i = 0; i < WAVES; ++i) top = red_m[turn][own][i] > top ? red_m[turn][own][i] : top;
            }
            const RowCodes codes(top);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = (c * T + t) * V, from = at < a.d - V ? at : a.d - V;
                if (live && at < a.d) codes.store<V, true>(out + from, h[c], a.past);
                if constexpr (C >= 4) __builtin_amdgcn_sched_barrier(0);
            }
            if (live && t == 0) a.out_scale[r] = codes.s;
        }
    }
}

// Rows shorter than a chunk: a thread each.
template <int DT, int ODT>
__global__ __launch_bounds__(256) void k_norm_short_rows(NormArgs a)
{
    using E = typename Elem<DT>::T;
    using O = typename Elem<ODT>::T;
    constexpr int V = 16 / sizeof(E);
    for (int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x; r < a.n; r += (int64_t)gridDim.x * 256) {
        float h[V], w[V], ss = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < a.d) {
                Raw<DT, 1> e;
                e.load(static_cast<const E*>(a.x) + r * a.ld_x + i);
                e.values(&h[i]);
                if (a.res) {
                    float v;
                    e.load(static_cast<const E*>(a.res) + r * a.ld_res + i);
                    e.values(&v);
                    h[i] += v;
                }
                if (a.weight) {
                    e.load(static_cast<const E*>(a.weight) + i);
                    e.values(&w[i]);
                }
                ss = __builtin_fmaf(h[i], h[i], ss);
            }
        const float f = rsqrt_of(__builtin_fmaf(ss, a.inv_d, a.eps));
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < a.d) {
                if (a.sum) store_values<DT, 1>(static_cast<E*>(a.sum) + r * a.ld_sum + i, &h[i]);
                h[i] = a.weight ? h[i] * f * w[i] : h[i] * f;
                top = magnitude(h[i]) > top ? magnitude(h[i]) : top;
            }
        const RowCodes codes(top);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < a.d) {
                if constexpr (ODT == APC_E4M3) codes.store<1>(static_cast<O*>(a.out) + r * a.ld_out + i, &h[i]);
                else store_values<ODT, 1>(static_cast<O*>(a.out) + r * a.ld_out + i, &h[i]);
            }
        if (ODT == APC_E4M3) a.out_scale[r] = codes.s;
    }
}

template <int DT, int ODT, int T, int C>
void launch_t(const NormArgs& a, hipStream_t s)
{
    constexpr int rows = T > 256 ? 1 : 256 / T;
    const int64_t groups = (a.n + rows - 1) / rows;
    k_norm_rows<DT, ODT, T, C><<<dim3((unsigned)(groups < MAX_GRID ? groups : MAX_GRID)), dim3(T > 256 ? T : 256), 0, s>>>(a);
}

// Threads per row from the row's chunks alone, so that a row's bits do not
// depend on the call's other rows: the fewest that leave two or three chunks to
// each, and with them several loads in flight and few threads idle (100,000 x
// 1,536 bf16 to e4m3: 64 threads with three 86 us, 128 with two 99; 65,536 x
// 4,096 bf16 with residual to e4m3: 256 with two 311 us, 128 with four 317).
template <int DT, int ODT>
hipError_t launch(const NormArgs& a, hipStream_t s)
{
    constexpr int V = 16 / sizeof(typename Elem<DT>::T);
    const int chunks = (a.d + V - 1) / V;
    if (a.d < V) {
        const int64_t groups = (a.n + 255) / 256;
        k_norm_short_rows<DT, ODT><<<dim3((unsigned)(groups < MAX_GRID ? groups : MAX_GRID)), dim3(256), 0, s>>>(a);
    } else if (chunks <= 16) launch_t<DT, ODT, 16, 1>(a, s);
    else if (chunks <= 32) launch_t<DT, ODT, 16, 2>(a, s);
    else if (chunks <= 48) launch_t<DT, ODT, 16, 3>(a, s);
    else if (chunks <= 64) launch_t<DT, ODT, 32, 2>(a, s);
    else if (chunks <= 96) launch_t<DT, ODT, 32, 3>(a, s);
    else if (chunks <= 128) launch_t<DT, ODT, 64, 2>(a, s);
    else if (chunks <= 192) launch_t<DT, ODT, 64, 3>(a, s);
    else if (chunks <= 256) launch_t<DT, ODT, 128, 2>(a, s);
    else if (chunks <= 384) launch_t<DT, ODT, 128, 3>(a, s);
    else if (chunks <= 512) launch_t<DT, ODT, 256, 2>(a, s);
    else if (chunks <= 768) launch_t<DT, ODT, 256, 3>(a, s);
    else if (chunks <= 1024) launch_t<DT, ODT, 512, 2>(a, s);
    else if (chunks <= 1536) launch_t<DT, ODT, 512, 3>(a, s);
    else if (chunks <= 2048) launch_t<DT, ODT, 1024, 2>(a, s);
    else if (chunks <= 3072) launch_t<DT, ODT, 1024, 3>(a, s);
    else if (DT != APC_F32 || chunks <= 4096) launch_t<DT, ODT, 1024, 4>(a, s);
    else if constexpr (DT == APC_F32) launch_t<DT, ODT, 1024, 8>(a, s);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_to(int out_dt, const NormArgs& a, hipStream_t s)
{
    return out_dt == APC_E4M3 ? launch<DT, APC_E4M3>(a, s) : launch<DT, DT>(a, s);
}

}  // namespace

hipError_t launch_norm_rows(int dt, int out_dt, const NormArgs& args, hipStream_t s)
{
    if (args.n <= 0) return hipSuccess;
    NormArgs a = args;
    a.past = a.n * a.d * elem_bytes(out_dt) >= PAST_CACHES;
    switch (dt) {
    case APC_F32: return launch_to<APC_F32>(out_dt, a, s);
    case APC_F16: return launch_to<APC_F16>(out_dt, a, s);
    case APC_BF16: return launch_to<APC_BF16>(out_dt, a, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
