// Paged key-value cache: new tokens' keys and values written into their slots,
// rounded or quantised on the way, and slots read back as rows.
//
// L lanes share a row (one head of one token's key or value), eight elements
// each (of float32 rows two fours, so that a wave's 16-byte accesses stand side
// by side), so a row's largest magnitude is a reduction over L lanes and a wave
// carries 64 / L rows.  A lane keeps the same head and goes on to U tokens, all
// of whose loads are in flight before the first is converted.  Bound by memory:
// the rows in and the stored bytes out, once each.  65,536 tokens x 8 x 128
// bf16 to e4m3 76 us, 5.2 TB/s; 100,003 of them back to bf16 112 us, 5.5 TB/s (a
// large copy reaches 4.6).
#include "apc_internal.h"
#include "convert.h"

namespace apc {
namespace {

constexpr int64_t MAX_GRID = 1 << 20;   // more rows than that many workgroups hold: a lane goes on to further tokens

// row of a slot's head inside k and v (page is a power of two), or -1
__device__ inline int64_t slot_row(const apc_kv& c, int32_t slot, int32_t head, int shift, int64_t slots)
{
    if (slot < 0 || slot >= slots) return -1;
    return (((int64_t)(slot >> shift) * c.heads + head) << shift) + (slot & (c.page - 1));
}

template <bool WRITE, int DT, int CDT, int L, int U>
__global__ __launch_bounds__(256) void k_kv_rows(apc_kv c, KvRows a, int shift)
{
    using E = typename Elem<DT>::T;
    using S = typename Elem<CDT>::T;
    constexpr int CH = DT == APC_F32 ? 2 : 1, V = 8 / CH;       // chunks a lane, elements a chunk
    int at[CH];
    bool mine[CH];                              // d is a multiple of 16
#pragma unroll
    for (int k = 0; k < CH; ++k) at[k] = (k * L + threadIdx.x % L) * V, mine[k] = at[k] < c.d;
    const int64_t slots = c.n_pages << shift;
    // Large calls go past the caches, where nobody would find their output again
    // (100,003 tokens x 8 x 128 from e4m3 to bf16: 112 us, 120 without; 65,536
    // bf16 to bf16: 93 and 100), but for pages' rows that are no whole halves of
    // lines (65,536 x 15 x 80 bf16: 137 us, 121 without).
    const bool past = U > 1 && (!WRITE || c.d * (int)sizeof(S) % 64 == 0);
    const int32_t rows = 2 * c.heads;           // of a token: every head's key, then every head's value
    // Workgroups go round the eight L2s: of a large call, each L2 has RUN
    // neighbours, which share the lines of the scales and the pages' rows (65,536
    // x 8 x 128 to e4m3: 75.8 us, 79.7 with one; 100,003 of them read: 111.9 and
    // 115.9).
    constexpr uint32_t RUN = U > 1 ? 32 : 1, SET = 8 * RUN;
    const uint32_t in_sets = gridDim.x / SET * SET, set = blockIdx.x / SET * SET, at_set = blockIdx.x % SET;
    const uint32_t wg = blockIdx.x < in_sets ? set + at_set % 8 * RUN + at_set / 8 : blockIdx.x;
    const int64_t unit0 = (int64_t)wg * (256 / L) + threadIdx.x / L, units = (a.t + U - 1) / U * rows;
    for (int64_t unit = unit0; unit < units; unit += (int64_t)gridDim.x * (256 / L)) {
        // t * heads < 2^31, so there are fewer than 2^32 units
        const uint32_t token = (uint32_t)unit / (uint32_t)rows;
        const int64_t tok0 = (int64_t)token * U;
        const int32_t which = (int32_t)((uint32_t)unit - token * (uint32_t)rows), head = which < c.heads ? which : which - c.heads;
        const bool value = which >= c.heads;
        E* outer = static_cast<E*>(value ? a.v : a.k) + head * (value ? a.v_head : a.k_head);
        const int64_t step = value ? a.v_tok : a.k_tok;
        S* pool = static_cast<S*>(value ? c.v : c.k);
        float* scale = value ? c.v_scale : c.k_scale;
        int32_t slot[U];
#pragma unroll
        for (int u = 0; u < U; ++u) slot[u] = tok0 + u < a.t ? a.slots[tok0 + u] : -1;
        if constexpr (WRITE) {
            Raw<DT, V> x[U][CH];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int k = 0; k < CH; ++k)
                    if (mine[k] && tok0 + u < a.t) x[u][k].load(outer + (tok0 + u) * step + at[k]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = slot_row(c, slot[u], head, shift, slots);
                float v[CH][V];
#pragma unroll
                for (int k = 0; k < CH; ++k) x[u][k].values(v[k]);
                if constexpr (CDT == APC_E4M3) {
                    uint32_t top = 0;
#pragma unroll
                    for (int k = 0; k < CH; ++k)
                        if (mine[k]) {
#pragma unroll
                            for (int i = 0; i < V; ++i) top = magnitude(v[k][i]) > top ? magnitude(v[k][i]) : top;
                        }
                    const RowCodes codes(max_over<L>(top));
#pragma unroll
                    for (int k = 0; k < CH; ++k)
                        if (row >= 0 && mine[k]) codes.template store<V>(pool + row * c.d + at[k], v[k], past);
                    if (row >= 0 && at[0] == 0) scale[row] = codes.s;
                } else {
#pragma unroll
                    for (int k = 0; k < CH; ++k)
                        if (row >= 0 && mine[k]) store_values<CDT, V>(pool + row * c.d + at[k], v[k], past);
                }
            }
        } else {
            Raw<CDT, V> x[U][CH];
            float s[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t row = slot_row(c, slot[u], head, shift, slots);
                s[u] = 1.f;
                if (row >= 0) {
#pragma unroll
                    for (int k = 0; k < CH; ++k)
                        if (mine[k]) x[u][k].load(pool + row * c.d + at[k]);
                    if constexpr (CDT == APC_E4M3) s[u] = scale[row];
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int k = 0; k < CH; ++k) {
                    if (!mine[k] || tok0 + u >= a.t) continue;
                    float v[V] = {};
                    if (slot[u] >= 0 && slot[u] < slots) {
                        x[u][k].values(v);
                        if constexpr (CDT == APC_E4M3) {
#pragma unroll
                            for (int i = 0; i < V; ++i) v[i] *= s[u];
                        }
                    }
                    store_values<DT, V>(outer + (tok0 + u) * step + at[k], v, past);
                }
            }
        }
    }
}

template <bool WRITE, int DT, int CDT, int L>
void launch_l(const apc_kv& c, const KvRows& a, hipStream_t s)
{
    int shift = 0;
    while ((1 << shift) < c.page) ++shift;
    const int64_t rows = a.t * 2 * c.heads;
    // two tokens a lane, or four of wide e4m3 rows, where four would fill the
    // chip's 2,048 lanes a CU all the same (65,536 x 8 x 128 to e4m3: 75.8 us, 77
    // to 85 with two, 80 with eight; 65,536 x 8 x 128 bf16 read: 92 with two, 95
    // with four; 77,777 x 20 x 32 to e4m3: 72 and 79)
    constexpr int MANY = CDT == APC_E4M3 && L >= 16 ? 4 : 2;
    const int u = rows * L >= 4 * 256 * 2048 ? MANY : 1;
    const int64_t groups = ((a.t + u - 1) / u * 2 * c.heads + 256 / L - 1) / (256 / L);
    const dim3 grid((unsigned)(groups < MAX_GRID ? groups : MAX_GRID)), block(256);
    if (u == MANY) k_kv_rows<WRITE, DT, CDT, L, MANY><<<grid, block, 0, s>>>(c, a, shift);
    else k_kv_rows<WRITE, DT, CDT, L, 1><<<grid, block, 0, s>>>(c, a, shift);
}

template <bool WRITE, int DT, int CDT>
void launch(const apc_kv& c, const KvRows& a, hipStream_t s)
{
    if (c.d <= 32) launch_l<WRITE, DT, CDT, 4>(c, a, s);
    else if (c.d <= 64) launch_l<WRITE, DT, CDT, 8>(c, a, s);
    else if (c.d <= 128) launch_l<WRITE, DT, CDT, 16>(c, a, s);
    else launch_l<WRITE, DT, CDT, 32>(c, a, s);
}

template <bool WRITE, int DT>
hipError_t launch_to(const apc_kv& c, const KvRows& a, hipStream_t s)
{
    switch (c.dt) {
    case APC_F16: launch<WRITE, DT, APC_F16>(c, a, s); break;
    case APC_BF16: launch<WRITE, DT, APC_BF16>(c, a, s); break;
    case APC_E4M3: launch<WRITE, DT, APC_E4M3>(c, a, s); break;
    default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv_rows(bool write, int dt, const apc_kv& c, const KvRows& a, hipStream_t s)
{
    if (a.t <= 0) return hipSuccess;
    switch (dt) {
    case APC_F32: return write ? launch_to<true, APC_F32>(c, a, s) : launch_to<false, APC_F32>(c, a, s);
    case APC_F16: return write ? launch_to<true, APC_F16>(c, a, s) : launch_to<false, APC_F16>(c, a, s);
    case APC_BF16: return write ? launch_to<true, APC_BF16>(c, a, s) : launch_to<false, APC_BF16>(c, a, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
