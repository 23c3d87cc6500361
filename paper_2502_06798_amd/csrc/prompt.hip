// Attention of several new tokens of each sequence over a paged key-value
// cache: into which units and parts a call is cut, and the parts' join. The
// kernel is in prompt_kernel.h.
#include "prompt_kernel.h"

#include <algorithm>
#include <limits>

namespace apc {
namespace {

// Row tiles of each 256 sequences
__global__ __launch_bounds__(256) void k_prompt_sums(PromptArgs a, int group, int rows, int32_t* sums)
{
    __shared__ int of[4];
    int first;
    int64_t x = prompt_tiles(prompt_rows(a, blockIdx.x * 256 + threadIdx.x, first), group, rows);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d, 64);
    if (threadIdx.x % 64 == 0) of[threadIdx.x / 64] = x < MOST_TILES ? (int)x : MOST_TILES;
    __syncthreads();
    // (only starts that overlap give as many as that; sums of 64 such stay in 32 bits)
    const int all = of[0] + of[1] + of[2] + of[3];
    if (threadIdx.x == 0) sums[blockIdx.x] = all < MOST_TILES ? all : MOST_TILES;
}

// Joins the parts of units whose keys were cut: a workgroup takes ROWS rows of a
// unit at a time.  The threads of a row first go over its parts' maxima and sums of
// weights, then, as (some of the parts) x (elements), sum the parts' means, each times its
// share of all weights: a mean at no point outside the values' range.  The order of
// the sums follows from the number of parts alone.
template <int DT, int DP, int ROWS>
__global__ __launch_bounds__(256) void k_prompt_join(apc_kv c, PromptArgs a, PromptPlan p, int kt)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = DP / 4, PER = 256 / ROWS, AT_ONCE = PER / LANES, AHEAD = 4, W = PER < 64 ? PER : 64;
    static_assert(AT_ONCE >= 1);
    __shared__ float acc[ROWS][AT_ONCE][DP];
    __shared__ float tops[PER / W], sums[PER / W];              // of waves that share a row
    const int head = blockIdx.x % c.heads, k = blockIdx.x / c.heads, group = a.q_heads / c.heads;
    const PromptUnit u = prompt_unit(a, group, p.rows, k);
    if (u.seq < 0) return;
    const PromptSight sight(a, p.shift, group, u);
    const PromptKeys keys(p, sight, u, p.rows, kt);
    if (keys.parts == 1) return;
    const int left = u.n * group - u.tile * p.rows, rows = left < p.rows ? left : p.rows;
    const int i = threadIdx.x / PER, part0 = threadIdx.x % PER / LANES, d = threadIdx.x % LANES * 4;
    const float* po = static_cast<const float*>(a.ws);
    const float* pm = po + prompt_slots(p, c.heads) * DP;
    for (int r0 = blockIdx.y * ROWS; r0 < rows; r0 += gridDim.y * ROWS) {
        const int r = r0 + i < rows ? r0 + i : r0;              // (a row past the end: the first one's, not stored)
        const int64_t slot = prompt_slot(p, c.heads, k, head, 0) + r;
        f32x4 x[AHEAD];
        float m[AHEAD], l[AHEAD];
        auto load = [&](int q0) INLINE {
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                const int q = q0 + j * AT_ONCE < keys.parts ? q0 + j * AT_ONCE : part0 < keys.parts ? part0 : 0;
                const int64_t at = slot + (int64_t)q * p.rows;
                x[j] = *reinterpret_cast<const f32x4*>(po + at * DP + d);
                m[j] = pm[at * 2];
                l[j] = pm[at * 2 + 1];
            }
        };
        load(part0);
        float top = LOWEST, sum = 0.f;
        auto add = [&](float m, float l) INLINE {
            const float y = __builtin_fmaxf(top, m);
            sum = sum * __builtin_amdgcn_exp2f(top - y) + l * __builtin_amdgcn_exp2f(m - y);
            top = y;
        };
        for (int q = threadIdx.x % PER; q < keys.parts; q += PER) {
            const int64_t at = (slot + (int64_t)q * p.rows) * 2;
            add(pm[at], pm[at + 1]);
        }
#pragma unroll
        for (int x = W / 2; x > 0; x /= 2) {
            const float m = __shfl_xor(top, x, W), l = __shfl_xor(sum, x, W);
            add(m, l);
        }
        top = __shfl(top, 0, W), sum = __shfl(sum, 0, W);       // (the same for all lanes, to the last bit)
        if constexpr (PER > W) {
            if (threadIdx.x % W == 0) tops[threadIdx.x / W] = top, sums[threadIdx.x / W] = sum;
            __syncthreads();
            top = LOWEST, sum = 0.f;
#pragma unroll
            for (int w = 0; w < PER / W; ++w) add(tops[w], sums[w]);
        }
        const float inv = sum == 0.f ? 0.f : 1.0f / sum;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        for (int q0 = part0; q0 < keys.parts; q0 += AT_ONCE * AHEAD) {
            if (q0 != part0) load(q0);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) {
                if (q0 + j * AT_ONCE >= keys.parts) break;
                v += x[j] * (__builtin_amdgcn_exp2f(m[j] - top) * l[j] * inv);
            }
        }
        if constexpr (AT_ONCE > 1) {
            // (waves that share a row have met since the last row's were read)
            if (PER <= W && r0 != (int)blockIdx.y * ROWS) __syncthreads();
            *reinterpret_cast<f32x4*>(&acc[i][part0][d]) = v;
            __syncthreads();
            v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) v += *reinterpret_cast<const f32x4*>(&acc[i][j][d]);
        }
        if (r0 + i < rows && part0 == 0) {
            const float out[4] = {v.x, v.y, v.z, v.w};
            const int row = u.tile * p.rows + r, h = head * group + row % group;
            const int64_t token = u.first + row / group;
            if (d < c.d) store_values<DT, 4>(static_cast<T*>(a.out) + token * a.out_row + h * a.out_head + d, out);
            if (a.lse && d == 0) a.lse[token * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
        }
    }
}

template <int DT, int DP> hipError_t join(const apc_kv& c, const PromptArgs& a, const PromptPlan& p, int kt, hipStream_t s)
{
    // many parts: a workgroup a row; else several rows
    constexpr int SEVERAL = DP > 128 ? 4 : 8;
    const int rows = p.splits > SEVERAL ? 1 : SEVERAL;
    const dim3 grid((unsigned)(p.tiles * c.heads), (unsigned)((p.unit_rows + rows - 1) / rows));
    if (rows == 1) k_prompt_join<DT, DP, 1><<<grid, dim3(256), 0, s>>>(c, a, p, kt);
    else k_prompt_join<DT, DP, SEVERAL><<<grid, dim3(256), 0, s>>>(c, a, p, kt);
    return hipGetLastError();
}

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
int tile_keys(int rows, int dp) { return rows == 32 || dp > 128 ? 32 : 64; }

// Row tiles of 32, whose four waves share the keys out, where sequences have no
// more rows than that on the average, or where tiles of 128, a wave 32 of them,
// would be fewer than the CUs: a call of little work is the latency of its longest
// wave's tiles (7 sequences of 1 to 333 tokens over e4m3, 5 x 2 heads of 80: 19 us,
// 47 in 76 tiles of 128; 256 tokens, 4 x 8 heads of 128: 10.5 and 14; 128 behind 4,000, 8 x
// 4 heads: 33 and 47).  The rule does not see that keys could be cut, and with long keys tiles
// of 128 would be faster far below as many as the CUs: 256 tokens behind 4,000 50 us and 51,
// 512 78 and 69, 992 152 and 110; behind 64,512 128 tokens 403 and 201, 512 1,037 and 599,
// 992 2,043 and 1,159 (1,024 have 256 tiles: 1,190).
constexpr int FEW_ROWS = 32, CUS = 256;
// Keys are cut where units are fewer than the workgroups that the chip holds at
// once (two a CU), into parts whose time is more than the join's.  Row tiles of 32
// are cut further while parts stay long, so that ragged lengths leave less at the
// end (64 single tokens over 16,384 to 32,768 tokens: 625 us, 670 in parts twice as long;
// one over 131,072: 68, 92 in parts of 512 tokens).
constexpr int FULL = 2 * CUS, MANY = 8 * CUS, LONG_KEYS = 4096;
constexpr int min_keys(int rows) { return rows == 32 ? 512 : 1024; }

// Every workgroup looks for its unit among all sequences, 256 a step of some 0.7 us: that is the square of their
// number, and of more than MANY_SEQUENCES a launch of its own sums up their tiles, 256 to a sum.
constexpr int MANY_SEQUENCES = 1024;
size_t sums_bytes(int64_t b) { return b > MANY_SEQUENCES ? ((b + 255) / 256 * sizeof(int32_t) + 255) / 256 * 256 : 0; }

int64_t row_tiles(int64_t t, int64_t b, int group, int rows) { return t * group / rows + (b < t ? b : t); }
int64_t least_tiles(int64_t t, int64_t b, int group, int rows) { return std::max(std::min(b, t), (t * group + rows - 1) / rows); }

}  // namespace

PromptPlan plan_prompt(const apc_kv& c, int64_t t, int32_t b, int32_t q_heads, int32_t max_pages, int32_t window, bool prefix)
{
    PromptPlan p{};
    const int group = q_heads / c.heads;
    while ((1 << p.shift) < c.page) ++p.shift;
    p.dp = padded(c.d);
    const bool few = t * group <= FEW_ROWS * std::min<int64_t>(b, t) || least_tiles(t, b, group, 128) * c.heads < CUS;
    // (a launch has fewer than 2^32 threads)
    p.rows = few && row_tiles(t, b, group, 32) * c.heads < 1 << 23 ? 32 : 128;
    p.tiles = (int32_t)row_tiles(t, b, group, p.rows);
    const int64_t tiles = least_tiles(t, b, group, p.rows), units = tiles * c.heads;
    // keys of a unit, at most
    int64_t keys = (int64_t)max_pages * c.page;
    if (window > 0) keys = std::min(keys, (prefix ? 2 : 1) * (int64_t)window + p.rows / group + 1);
    int64_t splits = FULL / units;
    if (p.rows == 32) splits = std::max(splits, std::min(MANY / units, keys / LONG_KEYS));
    p.splits = (int32_t)std::max<int64_t>(1, std::min(splits, keys / min_keys(p.rows)));
    p.unit_rows = (int32_t)std::min<int64_t>(p.rows, (t * group + tiles - 1) / tiles);
    p.min_tiles = min_keys(p.rows) / tile_keys(p.rows, p.dp);
    return p;
}

size_t prompt_workspace(const apc_kv& c, int64_t t, int32_t b, int32_t q_heads, int32_t max_pages)
{
    // what any call of up to so many tokens, sequences and pages can ask: a plan's tiles
    // are fewer than twice the least there can be, for which its parts are
    if (t == 0 || b == 0) return 0;
    const int group = q_heads / c.heads;
    int64_t slots = 0;
    for (int rows : {32, 128}) {
        if (rows > 32 && t * group <= FEW_ROWS) continue;
        const int64_t most = (int64_t)max_pages * c.page / min_keys(rows), full = 2 * (rows == 32 ? MANY : FULL);
        if (most < 2) continue;
        slots = std::max(slots, std::min(row_tiles(t, b, group, rows) * c.heads * most, full) * rows);
    }
    return sums_bytes(b) + (size_t)slots * (padded(c.d) + 2) * sizeof(float);
}

hipError_t launch_attend_prompt(int dt, const apc_kv& c, const PromptArgs& args, hipStream_t s)
{
    if (args.b <= 0 || args.t <= 0) return hipSuccess;
    PromptArgs a = args;
    PromptPlan p = plan_prompt(c, a.t, a.b, a.q_heads, a.max_pages, a.window, a.prefix != nullptr);
    if (c.n_pages == 0) a.max_pages = 0;                        // no page to read from
    if (const size_t bytes = sums_bytes(a.b)) {
        int32_t* const sums = static_cast<int32_t*>(a.ws);
        k_prompt_sums<<<dim3((unsigned)((a.b + 255) / 256)), dim3(256), 0, s>>>(a, a.q_heads / c.heads, p.rows, sums);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        a.sums = sums;
        a.ws = static_cast<char*>(a.ws) + bytes;
    }
    // (a cap so far away bends nothing; so near, its inverse ends the range)
    if (a.cap > 0x1p100f) a.cap = 0.f;
    if (a.cap > 0.f) p.to_cap = std::min(std::fabs(a.scale) / a.cap, std::numeric_limits<float>::max());
    // (0 times an infinite factor is no score; what passes the range times 4 has an infinite score anyway.  Together with the
    // bias, as a branch of its own in the loop costs 1.5%: 2 x 8,192 tokens, 1,183 us and 1,201.)
    else p.lift = !std::isfinite(a.scale * LOG2E);
    if (p.lift) a.scale *= 0.25f;
    p.bias = a.slopes || p.lift;
    const hipError_t e = c.dt == APC_E4M3 ? launch_prompt_e4m3(dt, c, a, p, s)
                         : c.dt == APC_F16 ? launch_prompt_f16(c, a, p, s) : launch_prompt_bf16(c, a, p, s);
    if (e != hipSuccess || p.splits == 1) return e;
    const int kt = tile_keys(p.rows, p.dp);
    if (dt == APC_F16)
        return p.dp == 64 ? join<APC_F16, 64>(c, a, p, kt, s) : p.dp == 128 ? join<APC_F16, 128>(c, a, p, kt, s) : join<APC_F16, 256>(c, a, p, kt, s);
    return p.dp == 64 ? join<APC_BF16, 64>(c, a, p, kt, s) : p.dp == 128 ? join<APC_BF16, 128>(c, a, p, kt, s) : join<APC_BF16, 256>(c, a, p, kt, s);
}

}  // namespace apc
