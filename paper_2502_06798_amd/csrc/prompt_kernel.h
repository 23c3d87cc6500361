// Attention of several new tokens of each sequence over a paged key-value
// cache: the kernel, built for one cache type by each of prompt_*.hip.
//
// The new tokens of a sequence and the query heads that share a key-value head
// make rows (token by token), cut into tiles of M rows; a row tile of a
// key-value head is a unit, a workgroup's work.  Long units that are few are cut
// along the keys as well, and k_prompt_join (prompt.hip) joins the parts.
//
// Keys and values go through LDS, 16 bits each: from e4m3 exactly, the scales
// beside them.  Per wave of 32 rows and tile of KT keys, in matrix instructions of
// 32 x 32 x 16:
//   S^T = K Q^T    keys are the rows, query rows the columns: a lane holds half
//                  of one query row's scores, the other lane half the rest.
//   P   = exp2(S - m), float32; m is the row's running maximum, raised (and the
//                  sums scaled) only where a score passes it by SLACK, so that a
//                  tile needs no exchange between lanes as a rule.
//   O^T += V^T P^T the lane's weights are the second operand as they stand, given
//                  that the first operand's lanes hold the values of the same
//                  keys, which LDS reads that transpose 4 x 16 elements give.
// Two shapes: SHARED, where R waves have 32 rows each and the same keys (tiles in
// two LDS buffers, the next on its way in registers); else KW waves have the same
// 32 rows and every KW-th tile each, in an LDS buffer of their own.
//
// Bound, for long SHARED units, by the matrix unit and what it waits for: two
// prompts of 8,192 tokens, 4 x 8 heads of 128, bf16, take 1,160 to 1,210 us by box, 0.91 to
// 0.95 PFLOP/s, its unit busy 45% of the time at 1.9 GHz (a large bf16 product reaches 1.44
// among other calls, 1.58 by its own time in a trace, at 93% and 1.72 GHz); loads cost 150
// us of it, the copies to LDS 90.  Tried and not
// kept: 64 rows a wave (half of the LDS reads, but one wave a SIMD: 1,350 us), 8
// waves to a tile (1,150; short calls 5 to 10% more), with loads two tiles ahead
// (no less).  Single tokens are bound by memory: 64 of 16,384 to 32,768, e4m3, 625 us,
// 5.3 TB/s (streaming reads reach 6.2).
#pragma once

#include "attend_common.h"

#include <cmath>
#include <type_traits>

namespace apc {

using f32x16 = float __attribute__((ext_vector_type(16)));
using s16x4 = short __attribute__((ext_vector_type(4)));
using u16x2 = uint16_t __attribute__((ext_vector_type(2)));

// 32 x 32 x 16: D = A B + C; a lane's 8 values of A are row lane % 32, of B
// column lane % 32, both at k = 8 (lane / 32); of D column lane % 32, row
// 8 (r / 4) + 4 (lane / 32) + r % 4
template <bool BF> __device__ inline f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// 16 lanes read 4 rows of 16 elements, lane i the elements 4 (i % 4) on of row
// i / 4, and get columns: lane i element i of the four rows
__device__ inline uint2 read_columns(const uint16_t* lds)
{
    return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(const_cast<uint16_t*>(lds))));
}

// over the two lanes that have a query row
__device__ inline float both_halves_max(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ inline float both_halves_sum(float x)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// the halves of w that hold +inf (kind 0), -inf (1) or NaN (2), each as 1
template <bool BF> __device__ inline uint32_t is_kind(uint32_t w, int kind)
{
    constexpr uint32_t INF = BF ? 0x7f80u : 0x7c00u, ONE = BF ? 0x3f80u : 0x3c00u;
    const uint32_t lo = w & 0xffffu, hi = w >> 16;
    auto is = [&](uint32_t x) { return kind == 0 ? x == INF : kind == 1 ? x == (INF | 0x8000u) : (x & 0x7fffu) > INF; };
    return (is(lo) ? ONE : 0u) | (is(hi) ? ONE << 16 : 0u);
}

// tanh(x) / x for |x| <= NEAR from x^2, within 2^-24 as computed: the polynomial of
// smallest largest relative error (2^-27.7), found by Remez's exchange
constexpr float NEAR = 0.625f;
__device__ inline float tanh_over_x(float z)
{
    float r = __builtin_fmaf(z, -0.0057049873f, 0.020639088f);
    r = __builtin_fmaf(z, r, -0.053739715f);
    r = __builtin_fmaf(z, r, 0.13331442f);
    r = __builtin_fmaf(z, r, -0.3333328f);
    return __builtin_fmaf(z, r, 1.0f);
}

// a row tile of a sequence: the sequence's first row among the new tokens', their number, the tile
struct PromptUnit { int seq, first, n, tile; };

// new tokens of sequence i from its first row on (starts outside the rows are cut, falling ones have none)
__device__ INLINE inline int prompt_rows(const PromptArgs& a, int i, int& first)
{
    const int t = (int)a.t;
    int from = 0, to = 0;
    if (i < a.b) from = a.starts[i], to = a.starts[i + 1];
    first = from < 0 ? 0 : from < t ? from : t;
    to = to < 0 ? 0 : to < t ? to : t;
    return to > first ? to - first : 0;
}
__device__ INLINE inline int prompt_tiles(int n, int group, int rows) { return (int)(((int64_t)n * group + rows - 1) / rows); }

// Of 256 entries, a lane four at a distance of 64, the one with the k-th of what they
// count, k then the place in it; -1 where they have no more than k, which k then is without.
// found(u, l): it is the u-th of lane l.
template <typename F> __device__ INLINE inline int entry_with(const int (&count)[4], int& k, F&& found)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        int upto = count[u];
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d, 64);
            if (lane >= d) upto += o;
        }
        const int total = __builtin_amdgcn_readlane(upto, 63);
        if (k < total) {
            const int l = __builtin_ctzll(__ballot(upto > k));
            k -= __builtin_amdgcn_readlane(upto - count[u], l);
            found(u, l);
            return 64 * u + l;
        }
        k -= total;
    }
    return -1;
}

// The k-th of all sequences' row tiles of `rows` rows, found by every wave for
// itself, 256 sequences a step; of many sequences (a.sums) first 256 times 256, whose tiles
// k_prompt_sums has summed.  The last tiles of a sequence come first: where tokens
// see what stands before them, they have most to do.
constexpr int MOST_TILES = 1 << 24;                             // a call has fewer
__device__ INLINE inline PromptUnit prompt_unit(const PromptArgs& a, int group, int rows, int k)
{
    const int lane = threadIdx.x & 63;
    int seq0 = 0, count[4];
    if (a.sums) {
        const int blocks = (a.b + 255) / 256;
        for (int i = 0;; i += 256) {
            if (i >= blocks) return PromptUnit{-1, 0, 0, 0};
#pragma unroll
            for (int u = 0; u < 4; ++u) count[u] = i + 64 * u + lane < blocks ? a.sums[i + 64 * u + lane] : 0;
            const int x = entry_with(count, k, [](int, int) INLINE {});
            if (x >= 0) {
                seq0 = 256 * (i + x);
                break;
            }
        }
    }
    for (; seq0 < a.b; seq0 += 256) {
        int first[4], n[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            n[u] = prompt_rows(a, seq0 + 64 * u + lane, first[u]);
            count[u] = prompt_tiles(n[u], group, rows);
        }
        PromptUnit unit{0, 0, 0, 0};
        unit.seq = entry_with(count, k, [&](int u, int l) INLINE {
            unit.first = __builtin_amdgcn_readlane(first[u], l), unit.n = __builtin_amdgcn_readlane(n[u], l);
            unit.tile = __builtin_amdgcn_readlane(count[u], l) - 1 - k;
        });
        if (unit.seq >= 0) {
            unit.seq += seq0;
            return unit;
        }
    }
    return PromptUnit{-1, 0, 0, 0};
}

// What the rows of a sequence see: the tokens [first(p), end(p)) of the one at position p.  Both never fall as p rises.
struct PromptSight {
    int len, past, prefix, window, group;
    __device__ INLINE PromptSight(const PromptArgs& a, int shift, int group, const PromptUnit& u) : window(a.window), group(group)
    {
        const int32_t held = table_entry(a.lengths, u.seq), cap = a.max_pages << shift;
        len = held < 0 ? 0 : held < cap ? held : cap;
        past = len - u.n;                                       // position of the first new token
        prefix = a.prefix ? table_entry(a.prefix, u.seq) : 0;
    }
    __device__ INLINE int position(int row) const { return past + row / group; }
    __device__ INLINE int first(int p) const { return window > 0 && p >= window ? p + 1 - window : 0; }
    __device__ INLINE int end(int p) const
    {
        int e = p + 1 > prefix ? p + 1 : prefix;
        if (window > 0 && e > p + window) e = p + window;
        return e < len ? e : len;
    }
};

// A unit's tiles of kt keys, and into how many parts they are cut
struct PromptKeys {
    int tile0, tiles, parts;
    __device__ INLINE PromptKeys(const PromptPlan& p, const PromptSight& s, const PromptUnit& u, int rows, int kt)
    {
        const int r0 = u.tile * rows, all = u.n * s.group, r1 = r0 + rows < all ? r0 + rows : all;
        const int lo = s.first(s.position(r0)), hi = s.end(s.position(r1 - 1));
        tile0 = lo / kt;
        tiles = hi > lo ? (hi + kt - 1) / kt - tile0 : 0;
        const int most = tiles / p.min_tiles;
        parts = most < 1 ? 1 : most < p.splits ? most : p.splits;
    }
};

// partial results in the workspace: means (float32, padded d a row), then each row's maximum and sum of weights.  (Means, as
// sums of values near the end of float32's range would leave it.)
__host__ __device__ inline int64_t prompt_slots(const PromptPlan& p, int heads) { return (int64_t)p.tiles * heads * p.splits * p.rows; }
__device__ inline int64_t prompt_slot(const PromptPlan& p, int heads, int k, int head, int part)
{
    return (((int64_t)k * heads + head) * p.splits + part) * p.rows;
}

// Every lane takes part in all of the loop: where registers are short the compiler
// may move one of the sums to another register inside a branch that only some lanes
// take, and the other lanes' is lost (heads of 256 over f16: wrong values so).
template <int DT, int CDT, int DP, int R, int KW>
__global__ __launch_bounds__(64 * R * KW, DP > 128 ? 1 : 2) void k_attend_prompt(apc_kv c, PromptArgs a, PromptPlan p)
{
    static_assert(R == 1 || KW == 1);
    using T = typename Elem<DT>::T;
    constexpr bool E8 = CDT == APC_E4M3, QBF = DT == APC_BF16, SHARED = R > 1;
    // The weights' type is the values': f16 over f16, else bf16 (e4m3 weights have the
    // value's scale in them, which can leave f16's range).  One part of a weight
    // loses up to half a step of it, 2^-11 or 2^-8, as much as the output's rounding
    // to the same type, and in sums over many values no more.  A second part, the
    // rounded rest, is taken where the waves share the keys out, whose time is the
    // keys' and values' loads, and by f16 queries over e4m3, whose outputs are f16.  (In
    // the others as well: two prompts of 8,192 tokens 1,546 us, 1,194 so; over e4m3, 16 of
    // 300 to 512, 247 and 212.)
    constexpr bool PBF = QBF || E8, TWO = !SHARED || PBF != QBF;
    // f16 weights end at 2^-24 and are whole from 2^-14 on: the row's heaviest stands at
    // 2^OFF to 2^15, so weights from 2^-26 of it are whole and those below 2^-36 are left out.
    // How much more than half a step that costs is bounded on the way (`lack`), and where it
    // could show in f16 the keys are gone over again with what is left of those weights as
    // well.  (The bound costs 5% of long prompts with heads of 128, 15% with heads of 64: two
    // of 8,192, 4 x 8 heads of 128, f16, 1,215 us before and 1,281, with a bias 1,335 and 1,413;
    // the second products in every tile that holds such weights 2,000, as most do.)
    constexpr float SLACK = PBF ? 8.f : 3.f, OFF = PBF ? 0.f : 12.f;
    constexpr int M = 32 * R, ES = E8 ? 1 : 2;
    constexpr int KT = SHARED && DP <= 128 ? 64 : 32;           // keys of a tile
    constexpr int NT = SHARED ? 64 * R : 64;                    // threads that load a tile
    constexpr int CH = DP * ES / 16, RW = 64 / CH;              // 16-byte pieces of a row, rows of a wave's load
    constexpr int ITS = KT * CH / NT, STEP = NT / CH;           // loads of a thread, rows between them
    constexpr int KS = DP + 8, VS = DP + 32;                    // elements between rows in LDS: reads meet every bank once
    constexpr int BUF = KT * (KS + VS) + (E8 ? 4 * KT : 0);     // of a buffer (16 bits each)
    constexpr int BUFS = SHARED ? 2 : KW;
    constexpr int JOIN = SHARED ? 0 : KW * (32 * (DP + 4) + 64) * 2;
    static_assert(RW <= 16 && KT * CH % NT == 0);
    __shared__ __attribute__((aligned(16))) uint16_t lds[BUFS * BUF > JOIN ? BUFS * BUF : JOIN];

    const int lane = threadIdx.x & 63, col = lane & 31, half = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int group = a.q_heads / c.heads;
    // a key-value head's units on one XCD, where the heads are a multiple of 8 (workgroups go round over the XCDs)
    const int head = blockIdx.x % c.heads, k = blockIdx.x / c.heads / p.splits, part = blockIdx.x / c.heads % p.splits;
    const PromptUnit u = prompt_unit(a, group, M, k);
    if (u.seq < 0) return;
    const PromptSight sight(a, p.shift, group, u);
    const PromptKeys keys(p, sight, u, M, KT);
    if (part >= keys.parts) return;
    const int all = u.n * group, len = sight.len;

    // this wave's rows, and this lane's
    const int row0 = u.tile * M + (SHARED ? wave * 32 : 0);
    const bool busy = row0 < all;
    const int rowz = row0 + 31 < all ? row0 + 31 : all - 1;
    const int pa = sight.position(busy ? row0 : rowz), pz = sight.position(rowz);
    const int lo_a = sight.first(pa), lo_z = sight.first(pz), hi_a = sight.end(pa), hi_z = sight.end(pz);
    const int row = row0 + col < all ? row0 + col : all - 1;
    const int token = row / group, qh = head * group + row % group;
    int at = sight.past + token, lo = sight.first(at);
    const int hi = sight.end(at);
    float slope = a.slopes ? a.slopes[qh] : 0.f;
    // (finite where the slope is: no distance times it is 0)
    slope = __builtin_fabsf(slope) > 2.3e38f && __builtin_fabsf(slope) < INFINITY ? __builtin_copysignf(3.4e38f, slope) : slope * LOG2E;

    const int row_bytes = c.d * ES, in_page = c.page - 1;
    u32x4 q[DP / 16];
    {
        const T* from = static_cast<const T*>(a.q) + (u.first + token) * a.q_row + qh * a.q_head + 8 * half;
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u; // scores are multiplied by |scale|
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
            q[s] = u32x4{0, 0, 0, 0};
            if (s * 16 < c.d) __builtin_memcpy(&q[s], from + s * 16, 16);
            q[s] ^= flip;
        }
    }
    const float sc = __builtin_fabsf(a.scale) * LOG2E;

    // keys and values on their way: 16-byte pieces of rows, zeros where there is no row
    const int32_t* table = a.pages + u.seq * a.ld_pages;
    const int last_page = (len - 1) >> p.shift;
    const int r_lane = lane / CH, ch = lane % CH;
    auto row_of = [&](int it) INLINE { return it * STEP + (SHARED ? wave * RW : 0); };
    // A tile's page entries: a lane has the one of key lane % KT.  (By a vector load, which is
    // in order with the others: scalar loads would have the first LDS operand wait for them.)
    auto find = [&](int j0) INLINE {
        const int i = (j0 + lane % KT) >> p.shift;
        return table[i < last_page ? i : last_page];
    };
    auto page_of = [&](int32_t pages, int r) INLINE { return __builtin_amdgcn_readlane(pages, r / 16 * 16); };
    auto there = [&](int32_t id, int j) INLINE { return ((uint32_t)id < (uint64_t)c.n_pages) & (j < len); };
    auto all_there = [&](int32_t pages, int j) INLINE { return __all(there(pages, j)); };
    auto first_row = [&](int32_t id, int j) INLINE { return (((int64_t)id * c.heads + head) << p.shift) + (j & in_page); };
    const bool in_row = ch * 16 < row_bytes;
    struct Tile { u32x4 k[ITS], v[ITS]; float scale; };
    // a lane's place among the sixteen rows that its wave's load is in; past a row's end it reads the row's first piece
    const uint32_t place = (uint32_t)((row_of(0) % 16 + r_lane) * row_bytes + (in_row ? ch * 16 : 0));
    const uint64_t page_bytes = ((uint64_t)c.heads << p.shift) * row_bytes, head_bytes = ((uint64_t)head << p.shift) * row_bytes;
    auto load = [&](Tile& to, int j0, int32_t pages) INLINE {
        // a lane has the first of its key's sixteen rows, which those that load it take from there
        const uint64_t rows = (uint32_t)pages * page_bytes + head_bytes + (uint32_t)((j0 + lane % KT / 16 * 16) & in_page) * row_bytes;
        auto one = [&](int it) INLINE {
            const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)rows, row_of(it) / 16 * 16);
            const uint32_t hi = __builtin_amdgcn_readlane((uint32_t)(rows >> 32), row_of(it) / 16 * 16);
            const uint64_t base = (uint64_t)hi << 32 | lo;
            using Bytes = const __attribute__((address_space(1))) uint8_t;
            using Piece = const __attribute__((address_space(1))) u32x4;
            Bytes *k = (Bytes*)c.k + base, *v = (Bytes*)c.v + base;
            asm("" : "+s"(k), "+s"(v));                         // (the same for all lanes: no 64-bit sums in each)
            const uint32_t off = place + (uint32_t)(it * STEP % 16 * row_bytes);
            to.k[it] = *(Piece*)(k + off);
            to.v[it] = *(Piece*)(v + off);
        };
        if (__builtin_expect(all_there(pages, j0 + lane % KT / 16 * 16), 1)) {
#pragma unroll
            for (int it = 0; it < ITS; ++it) one(it);
        } else {
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                to.k[it] = to.v[it] = u32x4{0, 0, 0, 0};
                if (there(page_of(pages, row_of(it)), j0 + row_of(it) / 16 * 16)) one(it);
            }
        }
        if constexpr (E8) {
            // a scale a lane: of keys in one wave (half), of values in another
            const bool values = SHARED ? wave == 1 : half == 1;
            to.scale = 0.f;
            const int j = j0 + lane % KT;
            if ((!SHARED | (wave < 2)) & there(pages, j)) to.scale = (values ? c.v_scale : c.k_scale)[first_row(pages, j)];
        }
    };
    u16x2 big = {0, 0};                                         // the largest |v| that this thread loads (f16, even and odd ones)
    auto keep = [&](Tile& t, int j0, uint16_t* to) INLINE {
        uint16_t *kk = to, *vv = to + KT * KS;
        if (c.d < DP || j0 + KT > len) {
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const bool out = !in_row | (j0 + row_of(it) + r_lane >= len);
                const u32x4 zero = {0, 0, 0, 0};
                t.k[it] = out ? zero : t.k[it], t.v[it] = out ? zero : t.v[it];
            }
        }
#pragma unroll
        for (int it = 0; it < ITS; ++it) {
            const int r = row_of(it) + r_lane;
            const u32x4 x = t.k[it], y = t.v[it];
            if constexpr (E8) {
                u32x4 w[2], z[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i / 2][i % 2 * 2] = from_e4m3<QBF, false>(x[i]), w[i / 2][i % 2 * 2 + 1] = from_e4m3<QBF, true>(x[i]);
                    z[i / 2][i % 2 * 2] = from_e4m3<PBF, false>(y[i]), z[i / 2][i % 2 * 2 + 1] = from_e4m3<PBF, true>(y[i]);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    *reinterpret_cast<u32x4*>(kk + r * KS + ch * 16 + 8 * i) = w[i];
                    *reinterpret_cast<u32x4*>(vv + r * VS + ch * 16 + 8 * i) = z[i];
                }
            } else {
                *reinterpret_cast<u32x4*>(kk + r * KS + ch * 8) = x;
                *reinterpret_cast<u32x4*>(vv + r * VS + ch * 8) = y;
                if constexpr (!PBF) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        big = __builtin_elementwise_max(big, __builtin_bit_cast(u16x2, y[i] & 0x7fff7fffu));
                    uint32_t z = __builtin_bit_cast(uint32_t, big);
                    asm volatile("" : "+v"(z) :: "memory");     // (before the next tile's loads, which take these registers)
                    big = __builtin_bit_cast(u16x2, z);
                }
            }
        }
        if constexpr (E8) {
            float* scales = reinterpret_cast<float*>(to + KT * (KS + VS));
            if (SHARED) {
                if (wave < 2 && lane < KT) scales[wave * KT + lane] = t.scale;
            } else {
                scales[lane] = t.scale;
            }
        }
    };

    const int many = PBF ? 32 - __builtin_clz(keys.tiles * KT | 1) : 0;             // (f16 values are far from that range's end)
    f32x16 o[DP / 32];
    float m, l;                                                 // the maximum less OFF, the lane's share of the sum
    float lack = 0.f;                                           // f16 weights' errors beyond half a step: 2^-35 of it at most
    auto clear = [&]() INLINE {
        m = LOWEST, l = 0.f;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[b][i] = 0.f;
    };
    // The tile of keys j0 on, at `from` in LDS, into o, m and l.
    // CAREFUL: right for infinite and NaN values, which a weight of 0 makes NaN, and
    // near the end of float32's range, where weights must not pass 1 in all: each is
    // multiplied by 2^-many, a power of two above the number of keys; and for f16
    // weights however light.
    auto add_tile = [&](auto care, int j0, int32_t pages, const uint16_t* from) INLINE {
        constexpr bool CAREFUL = decltype(care)::value;
        const uint16_t *kk = from, *vv = from + KT * KS;
        const float* scales = reinterpret_cast<const float*>(from + KT * (KS + VS));
        if (j0 + KT <= lo_a || j0 >= hi_z) return;              // nothing that these rows see
        float s[KT / 32][16];
        // operands from LDS, so many of them on their way (left to itself the compiler waits for each before its
        // product): what registers hold
        constexpr int NK = KT / 32 * (DP / 16), NV = KT / 16 * (DP / 32);
        constexpr int AHEAD_K = SHARED ? 8 : E8 ? 4 : 3, AHEAD = SHARED || E8 ? 4 : 2;
        int eight = 8 * half;
        if constexpr (CAREFUL) {                                // (else held in a register through the other loop for this one)
            eight = threadIdx.x;
            asm("" : "+v"(eight));
            eight = eight >> 2 & 8;
        }
        auto key_at = [&](int i) INLINE {                       // i: elements 16 (i / (KT / 32)) on of keys 32 (i % (KT / 32)) on
            return *reinterpret_cast<const u32x4*>(kk + (i % (KT / 32) * 32 + col) * KS + i / (KT / 32) * 16 + eight);
        };
        // (of two waves, the one with products to issue goes first: as equals both would wait for the same unit)
        __builtin_amdgcn_s_setprio(1);
        {
            u32x4 key[AHEAD_K];
            f32x16 sum[KT / 32];
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[b][i] = 0.f;
#pragma unroll
            for (int i = 0; i < AHEAD_K; ++i) key[i] = key_at(i);
            __builtin_amdgcn_sched_group_barrier(0x100, AHEAD_K, 0);
#pragma unroll
            for (int i = 0; i < NK; ++i) {
                constexpr int B = KT / 32;
                sum[i % B] = mfma32<QBF>(key[i % AHEAD_K], q[i / B], sum[i % B]);
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (i + AHEAD_K < NK) {
                    key[i % AHEAD_K] = key_at(i + AHEAD_K);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = sum[b][i];
        }
        __builtin_amdgcn_s_setprio(0);
        const bool whole = j0 >= lo_z && j0 + KT <= hi_a && all_there(pages, j0 + lane % KT);
        if constexpr (E8) {
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 y = *reinterpret_cast<const f32x4*>(scales + b * 32 + 2 * i + 4 * half);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[b][i + e] *= y[e];
                }
        }
        int lacks = 0;
        float f = sc;                                           // s times f: scores in units of log2
        if (a.cap > 0.f) {
            float top = 0.f;
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, __builtin_fabsf(s[b][i]));
            // where none of the wave's is far, without the exponentials (and more exactly)
            if (!__any(!(top * p.to_cap <= NEAR))) {
#pragma unroll
                for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float x = s[b][i] * p.to_cap;
                        s[b][i] = x * tanh_over_x(x * x);
                    }
            } else {
#pragma unroll
                for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        // (told apart from the other branch's, or the compiler computes all of the near
                        // ones before the branch, and runs out of registers)
                        float x = s[b][i];
                        asm volatile("" : "+v"(x));
                        x *= p.to_cap;
                        const float z = __builtin_fabsf(x);
                        const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(2.f * LOG2E * z));
                        const float near = x * tanh_over_x(x * x), y = __builtin_copysignf(far, x);
                        s[b][i] = z <= NEAR ? near : y;
                    }
            }
            f = a.cap * LOG2E;
        }
        if (p.bias) {
            if (__builtin_expect(p.lift, 0)) {
#pragma unroll
                for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] *= 4.f;                        // (a.scale is a fourth of the call's)
            }
            float away = (float)(at - j0 - 4 * half);           // of the lane's first key; exact where the product matters
            asm volatile("" : "+v"(away));
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float far = __builtin_fabsf(away - (float)(b * 32 + i / 4 * 8 + i % 4));
                    s[b][i] = __builtin_fmaf(-slope, far, s[b][i] * f);
                }
            f = 1.f;
        }
        if (!whole) {
            // of the lane's keys, `width` from `from` on, without the sixteens whose page is not there
            int from = lo - j0 - 4 * half;
            const int width = hi > lo ? hi - lo : 0;
            asm volatile("" : "+v"(from));                      // (or the loop would keep every key's distance from `lo`)
            const float by = f;
            f = 1.f;                                            // (-inf times a scale of 0 is none)
#pragma unroll
            for (int g = 0; g < KT / 16; ++g) {
                const uint32_t seen = there(page_of(pages, g * 16), j0 + g * 16) ? (uint32_t)width : 0;
#pragma unroll
                for (int i = g % 2 * 8; i < g % 2 * 8 + 8; ++i) {
                    const uint32_t at = (uint32_t)(g / 2 * 32 + i / 4 * 8 + i % 4 - from);
                    s[g / 2][i] = at < seen ? s[g / 2][i] * by : -INFINITY;
                    if constexpr (!PBF && !CAREFUL) lacks -= at < seen ? 0 : 1024;      // (as counted below)
                }
            }
        }
        // the running maximum
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KT / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, s[b][i]);
        top = top * f;
        asm("" : "+v"(top));                                    // (rounded here, as below)
        top -= OFF;
        if (__any(top > m + (CAREFUL ? 0.f : SLACK))) {
            const float y = both_halves_max(__builtin_fmaxf(m, top)), by = __builtin_amdgcn_exp2f(m - y);
            m = y;
            l *= by;
            if constexpr (!PBF && !CAREFUL) lack *= by;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) o[b] *= by;
        }
        // Where a step of float32 at the maximum's size is a good part of 1: the difference of rounded scores, so that the
        // largest is near 0, and no more than weights are meant to reach (the scores are no better known there).
        float less = m;
        if (__builtin_expect(__any((m > LOWEST) & (__builtin_fabsf(m) > 0x1p22f)), 0)) {
            constexpr float TOP = OFF + (CAREFUL ? 0.f : SLACK);
#pragma unroll
            for (int b = 0; b < KT / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float x = s[b][i] * f;
                    asm("" : "+v"(x));
                    x -= m;
                    s[b][i] = x > TOP ? TOP : x;
                }
            f = 1.f, less = 0.f;
        }
        const uint16_t* column = vv + (4 * half + (lane & 15) / 4) * VS + (lane >> 4 & 1) * 16 + lane % 4 * 4;
        auto values_at = [&](int i) INLINE {                    // i: elements 32 (i % (DP / 32)) on of keys 16 (i / (DP / 32)) on
            const uint16_t* from = column + i / (DP / 32) * 16 * VS + i % (DP / 32) * 32;
            const uint2 y = read_columns(from), z = read_columns(from + 8 * VS);
            return u32x4{y.x, y.y, z.x, z.y};
        };
        if constexpr (!PBF && CAREFUL) {
            // What f16 leaves of weights below 2^LIGHT, 2^-25 at most, is taken times 2^39 and added to the sums times 2^39
            // (below 2^-65 nothing is left there either: 2^-77 of the heaviest, which no f16 result shows).
            constexpr float LIGHT = TWO ? 0x1p-9f : 0x1p-14f;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) o[b] *= 0x1p39f;                          // (exactly: sums are below 2^61)
            auto add_part = [&](auto which) INLINE {
                u32x4 w[KT / 16];
#pragma unroll
                for (int x = 0; x < KT / 16; ++x)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float z[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            z[e] = s[x / 2][x % 2 * 8 + 2 * i + e];
                            asm volatile("" : "+v"(z[e]));      // (else the weights below are computed before this)
                            z[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[e], f, -less));
                        }
                        f32x2 rest = {z[0] < LIGHT ? z[0] : 0.f, z[1] < LIGHT ? z[1] : 0.f};
#pragma unroll
                        for (int part = 0; part < (TWO ? 2 : 1); ++part) rest -= unpack<false>(pack<false>(rest.x, rest.y));
                        rest *= 0x1p39f;
                        w[x][i] = pack<false>(rest.x, rest.y);
                        if constexpr (decltype(which)::value) {
                            rest -= unpack<false>(w[x][i]);
                            w[x][i] = pack<false>(rest.x, rest.y);
                        }
                    }
#pragma unroll
                for (int b = 0; b < DP / 32; ++b) {
#pragma unroll
                    for (int x = 0; x < KT / 16; ++x) {
                        u32x4 v = values_at(x * (DP / 32) + b);
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] &= ~not_finite<false>(v[e]);
                        o[b] = mfma32<false>(v, w[x], o[b]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            };
            add_part(std::false_type{});
            if constexpr (TWO) add_part(std::true_type{});
#pragma unroll
            for (int b = 0; b < DP / 32; ++b) o[b] *= 0x1p-39f;
        }
        // weights, of 16 keys at a time, and their values: columns of the keys whose weights the lane has
        u32x4 hi8[KT / 16], lo8[TWO ? KT / 16 : 1], any8[CAREFUL ? KT / 16 : 1];
        float l1 = 0.f;
        const float down = __uint_as_float((uint32_t)(127 - many) << 23);               // 2^-many
        auto weigh = [&](int x, int i) INLINE {                 // keys 2 i and 2 i + 1 of the lane's eight
            const float s0 = s[x / 2][x % 2 * 8 + 2 * i], s1 = s[x / 2][x % 2 * 8 + 2 * i + 1];
            float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s0, f, -less)), w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s1, f, -less));
            if constexpr (CAREFUL && PBF) w0 *= down, w1 *= down;
            l += w0, (SHARED ? l1 : l) += w1;                     // (two sums wait less, where there is a register)
            f32x2 y = {1.f, 1.f};
            if constexpr (E8) y = *reinterpret_cast<const f32x2*>(scales + KT + x * 16 + i / 2 * 8 + i % 2 * 2 + 4 * half);
            if constexpr (CAREFUL) {
                const bool n0 = s0 == -INFINITY, n1 = s1 == -INFINITY;          // (none, told from a weight of 0)
                any8[x][i] = pack<PBF>(n0 ? 0.f : 1.f, n1 ? 0.f : 1.f);
                w0 = n0 ? 0.f : w0 * y.x, w1 = n1 ? 0.f : w1 * y.y;
            } else {
                w0 *= y.x, w1 *= y.y;
            }
            hi8[x][i] = pack<PBF>(w0, w1);
            if constexpr (!PBF && !CAREFUL) {
                // a weight of x 2^-24, x < 1024, is off by at most 2^-25, (1024 - x) 2^-35 more than half a step of it, 2^-35 x
                const u16x2 less = __builtin_elementwise_sub_sat(u16x2{1024, 1024}, __builtin_bit_cast(u16x2, hi8[x][i]));
                lacks = (int)__builtin_amdgcn_udot2(less, u16x2{1, 1}, (uint32_t)lacks, false);
            }
            if constexpr (TWO) {
                const f32x2 z = unpack<PBF>(hi8[x][i]);
                lo8[x][i] = pack<PBF>(w0 - z.x, w1 - z.y);
                if constexpr (CAREFUL) lo8[x][i] &= ~not_finite<PBF>(hi8[x][i]);
            }
        };
        if constexpr (!CAREFUL) {
            // the next sixteen's weights are computed beside this one's products
            constexpr bool BESIDE = SHARED;
            u32x4 v[AHEAD];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int x = 0; x < (BESIDE ? 1 : KT / 16); ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) weigh(x, i);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) v[i] = values_at(i);
            __builtin_amdgcn_sched_group_barrier(0x100, 2 * AHEAD, 0);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                constexpr int B = DP / 32;
                const int x = i / B, b = i % B;
                if constexpr (BESIDE) __builtin_amdgcn_sched_barrier(0);
                o[b] = mfma32<PBF>(v[i % AHEAD], hi8[x], o[b]);
                if constexpr (TWO) o[b] = mfma32<PBF>(v[i % AHEAD], lo8[x], o[b]);
                if constexpr (!BESIDE) __builtin_amdgcn_sched_group_barrier(0x008, TWO ? 2 : 1, 0);
                if (i + AHEAD < NV) {
                    v[i % AHEAD] = values_at(i + AHEAD);
                    if constexpr (!BESIDE) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
                if (BESIDE && x + 1 < KT / 16)
#pragma unroll
                    for (int j = 4 * b / B; j < 4 * (b + 1) / B; ++j) weigh(x + 1, j);
            }
        } else {
#pragma unroll
            for (int x = 0; x < KT / 16; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) weigh(x, i);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                // infinite and NaN values by kind, where a weight is for them; else 0 in their place
                const int x = i / (DP / 32), b = i % (DP / 32);
                u32x4 v = values_at(i), out;
#pragma unroll
                for (int e = 0; e < 4; ++e) out[e] = v[e] & not_finite<PBF>(v[e]), v[e] &= ~not_finite<PBF>(v[e]);
                if (__any(out[0] | out[1] | out[2] | out[3])) {
#pragma unroll 1
                    for (int kind = 0; kind < 3; ++kind) {
                        u32x4 is;
#pragma unroll
                        for (int e = 0; e < 4; ++e) is[e] = is_kind<PBF>(out[e], kind);
                        f32x16 n = {};
                        n = mfma32<PBF>(is, any8[x], n);
                        const float what = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[b][e] += n[e] > 0.f ? what : 0.f;
                    }
                }
                o[b] = mfma32<PBF>(v, hi8[x], o[b]);
                if constexpr (TWO) o[b] = mfma32<PBF>(v, lo8[x], o[b]);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        l += l1;
        // (of so light keys that they lose all they are, no more than that)
        if constexpr (!PBF && !CAREFUL)
            lack += __builtin_fminf((float)lacks, (KT / 2) * __builtin_amdgcn_exp2f(top - m + (OFF + 35.f)));
    };
    auto not_finite_out = [&]() INLINE {
        float z = 0.f;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[b][i], 0.f, z);
        return z != 0.f;
    };
    // Whether light weights can be off by more than 2^-25 of f16's mean, half its smallest step: by 2^-35 lack |v| / l
    auto too_light = [&](float most) INLINE { return both_halves_sum(lack) * most > 1024.f * both_halves_sum(l); };
    auto largest = [&]() INLINE {                               // |v| that the wave has loaded
        int x = big.x > big.y ? big.x : big.y;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int y = __shfl_xor(x, d, 64);
            x = x > y ? x : y;
        }
        return (float)__builtin_bit_cast(_Float16, (uint16_t)(x < 0x7bff ? x : 0x7bff));
    };
    // (else registers hold these through the other loop, for this one alone)
    auto again = [&]() INLINE {
        int x = threadIdx.x;
        asm volatile("" : "+v"(x));
        x = row0 + (x & 31) < all ? row0 + (x & 31) : all - 1;
        at = sight.position(x), lo = sight.first(at);
    };
    // LDS that only this wave writes and reads needs no barrier, but the order kept
    auto settle = [&]() INLINE {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };

    const int t0 = keys.tile0 + (int)((int64_t)keys.tiles * part / keys.parts);
    const int t1 = keys.tile0 + (int)((int64_t)keys.tiles * (part + 1) / keys.parts);
    clear();
    int up = 0;                                                 // what takes 2^-many back, of the sum of weights
    Tile next;
    if constexpr (SHARED) {
        int32_t pg = 0, pn = 0;
        if (t0 < t1) {
            pg = find(t0 * KT);
            load(next, t0 * KT, pg);
            if (t0 + 1 < t1) pn = find((t0 + 1) * KT);
            keep(next, t0 * KT, lds);
        }
        uint16_t *here = lds, *other = lds + BUF;
        for (int t = t0; t < t1; ++t) {
            __syncthreads();
            if (t + 1 < t1) load(next, (t + 1) * KT, pn);
            int32_t pf = 0;
            if (t + 2 < t1) pf = find((t + 2) * KT);
            if (busy) add_tile(std::false_type{}, t * KT, pg, here);
            if (t + 1 < t1) keep(next, (t + 1) * KT, other);
            uint16_t* const x = here;
            here = other, other = x;
            pg = pn, pn = pf;
        }
        bool more = not_finite_out();
        if constexpr (!PBF) {
            float* const of = reinterpret_cast<float*>(lds);
            const float mine = largest();
            __syncthreads();
            if (lane == 0) of[wave] = mine;
            __syncthreads();
            float most = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) most = __builtin_fmaxf(most, of[r]);
            more |= too_light(most);
        }
        if (__builtin_expect(__syncthreads_or(more), 0)) {
            clear();
            up = many;
            again();
            for (int t = t0; t < t1; ++t) {
                pg = find(t * KT);
                load(next, t * KT, pg);
                __syncthreads();
                keep(next, t * KT, lds);
                __syncthreads();
                if (busy) add_tile(std::true_type{}, t * KT, pg, lds);
            }
        }
    } else {
        uint16_t* const mine = lds + wave * BUF;
        int t = t0 + wave;
        int32_t pg = 0, pn = 0;
        if (t < t1) {
            pg = find(t * KT);
            load(next, t * KT, pg);
            if (t + KW < t1) pn = find((t + KW) * KT);
        }
        for (; t < t1; t += KW) {
            settle();
            keep(next, t * KT, mine);
            settle();
            if (t + KW < t1) load(next, (t + KW) * KT, pn);
            int32_t pf = 0;
            if (t + 2 * KW < t1) pf = find((t + 2 * KW) * KT);
            add_tile(std::false_type{}, t * KT, pg, mine);
            pg = pn, pn = pf;
        }
        bool more = not_finite_out();
        if constexpr (!PBF) more |= too_light(largest());
        if (__builtin_expect(__any(more), 0)) {
            clear();
            up = many;
            again();
            for (t = t0 + wave; t < t1; t += KW) {
                pg = find(t * KT);
                load(next, t * KT, pg);
                settle();
                keep(next, t * KT, mine);
                settle();
                add_tile(std::true_type{}, t * KT, pg, mine);
            }
        }
    }

    // results: the rows' own means, or those over a part of their keys
    const int64_t slot = prompt_slot(p, c.heads, k, head, part);
    float* const means = static_cast<float*>(a.ws);
    float* const stats = means + prompt_slots(p, c.heads) * DP;
    l = both_halves_sum(l);
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    l = __builtin_amdgcn_ldexpf(l, up);
    if constexpr (SHARED) {
        const bool store = row0 + col < all;
        if (keys.parts > 1) {
            float* const to = means + (slot + wave * 32 + col) * DP + 4 * half;
#pragma unroll
            for (int b = 0; b < DP / 32; ++b)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    if (store) *reinterpret_cast<f32x4*>(to + b * 32 + 2 * i) = inv * f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
            if (store && half == 0) {
                stats[(slot + wave * 32 + col) * 2] = m;
                stats[(slot + wave * 32 + col) * 2 + 1] = l;
            }
            return;
        }
        T* const to = static_cast<T*>(a.out) + (u.first + token) * a.out_row + qh * a.out_head + 4 * half;
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = o[b][i + e] * inv;
                if (store && b * 32 + 2 * i < c.d) store_values<DT, 4>(to + b * 32 + 2 * i, v);
            }
        if (a.lse && store && half == 0)
            a.lse[(int64_t)(u.first + token) * a.q_heads + qh] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    } else {
        // the waves' results into one
        float* const part_o = reinterpret_cast<float*>(lds);
        float* const part_m = part_o + KW * 32 * (DP + 4);
        __syncthreads();
#pragma unroll
        for (int b = 0; b < DP / 32; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *reinterpret_cast<f32x4*>(part_o + (wave * 32 + col) * (DP + 4) + b * 32 + 2 * i + 4 * half) =
                    inv * f32x4{o[b][i], o[b][i + 1], o[b][i + 2], o[b][i + 3]};
        if (half == 0) part_m[(wave * 32 + col) * 2] = m, part_m[(wave * 32 + col) * 2 + 1] = l;
        __syncthreads();
        constexpr int PER = 64 * KW / 32, OWN = DP / PER;       // threads of a row, elements of a thread
        const int r = threadIdx.x / PER, d0 = threadIdx.x % PER * OWN, mine = u.tile * M + r;
        float top = LOWEST, sum = 0.f, of[KW], v[OWN] = {};
#pragma unroll
        for (int w = 0; w < KW; ++w) top = __builtin_fmaxf(top, part_m[(w * 32 + r) * 2]);
#pragma unroll
        for (int w = 0; w < KW; ++w) {
            of[w] = __builtin_amdgcn_exp2f(part_m[(w * 32 + r) * 2] - top) * part_m[(w * 32 + r) * 2 + 1];
            sum += of[w];
        }
        const float f = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
        for (int w = 0; w < KW; ++w)
#pragma unroll
            for (int i = 0; i < OWN; ++i) v[i] = __builtin_fmaf(of[w] * f, part_o[(w * 32 + r) * (DP + 4) + d0 + i], v[i]);
        if (mine >= all) return;
        if (keys.parts > 1) {
#pragma unroll
            for (int i = 0; i < OWN; i += 4)
                *reinterpret_cast<f32x4*>(means + (slot + r) * DP + d0 + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
            if (d0 == 0) stats[(slot + r) * 2] = top, stats[(slot + r) * 2 + 1] = sum;
            return;
        }
        int by = group;
        asm("" : "+s"(by));                                     // (else its inverse is held in a register through the loop)
        const int tok = mine / by, h = head * group + mine % by;
        T* const to = static_cast<T*>(a.out) + (u.first + tok) * a.out_row + h * a.out_head + d0;
        constexpr int ST = OWN < 16 ? OWN : 16;                 // d is a multiple of 16
#pragma unroll
        for (int i = 0; i < OWN; i += ST)
            if (d0 + i < c.d) store_values<DT, ST>(to + i, v + i);
        if (a.lse && d0 == 0)
            a.lse[(int64_t)(u.first + tok) * a.q_heads + h] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
    }
}

template <int DT, int CDT, int DP>
hipError_t launch_prompt_d(const apc_kv& c, const PromptArgs& a, const PromptPlan& p, hipStream_t s)
{
    const dim3 grid((unsigned)((int64_t)p.tiles * c.heads * p.splits));
    if (p.rows == 32) k_attend_prompt<DT, CDT, DP, 1, 4><<<grid, dim3(256), 0, s>>>(c, a, p);
    else k_attend_prompt<DT, CDT, DP, 4, 1><<<grid, dim3(256), 0, s>>>(c, a, p);
    return hipGetLastError();
}

template <int DT, int CDT>
hipError_t launch_prompt(const apc_kv& c, const PromptArgs& a, const PromptPlan& p, hipStream_t s)
{
    switch (p.dp) {
    case 64: return launch_prompt_d<DT, CDT, 64>(c, a, p, s);
    case 128: return launch_prompt_d<DT, CDT, 128>(c, a, p, s);
    default: return launch_prompt_d<DT, CDT, 256>(c, a, p, s);
    }
}

}  // namespace apc
