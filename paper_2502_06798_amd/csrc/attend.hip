// Attention of one new token per sequence over a paged key-value cache.
//
// A (sequence, key-value head) pair is a unit, its tokens are cut into tiles of
// 32.  Where units can be long, the tiles of all units stand in one row (each
// unit with EXTRA more, for what a unit costs besides its tiles) and every
// workgroup takes an equal stretch of it, so that ragged lengths leave none with
// more than its share; a unit that several workgroups share leaves partial
// results, which k_attend_join joins.  Otherwise a workgroup, of one wave where
// there are many short units, takes a unit at a time.  For each unit it computes up to NQ x 16 of the query heads
// that share the key-value head, wave w of WAVES every WAVES-th tile.
//
// A tile, per wave, in matrix instructions of 16 x 16 x 32:
//   S^T = K Q^T    keys are the rows, query heads the columns: a lane holds one
//                  head's scores of 8 of the 32 keys.  The sum over d runs in
//                  an order that lets a lane load 16 consecutive elements.
//   P   = exp2(S - m), float32; m is the head's running maximum, raised (and
//                  the sums scaled) only where a score passes it by 8, so that
//                  a tile needs no exchange between lanes as a rule.
//   O^T += V^T P^T the lane's 8 weights are the second operand's 8 values as
//                  they stand, given that the first operand's lanes load the
//                  values of the same 8 keys; a lane owns DP / 16 consecutive
//                  elements of those keys' rows, and pairs of keys are put
//                  together in registers.  No value passes through LDS.
// The weights enter as the sum of two bf16 (rounded, and the rounded rest): one
// alone would lose 2^-8 of every weight, two lose 2^-16, of a weight however
// light (two f16 would end at 2^-25 of the heaviest, and many light tokens make
// the output where the heavy one's value is near 0).  f16 values are split into
// two bf16 as well, exactly, so over f16 there are four products (16 sequences
// of 1 to 1,000 tokens, 4 x 8 heads of 128: 16.0 us, 15.0 with f16 weights and
// two products; 64 of 4,096 to 8,192, 12 heads of 64: 199 and 198).  e4m3 keys
// and values are converted exactly to 16 bits; their scales join the scores and
// the weights in float32.
//
// Bound by memory: every key and value is read once, into the registers that
// the matrix instructions take.  A wave's next tile, of the same unit or of the
// workgroup's next one, is on its way while this one is computed, joined with
// the other waves' and stored.  64 sequences of 16,384 to 32,768 tokens, 4 x 8
// heads of 128, e4m3: 525 us, 6.3 TB/s, what streaming reads reach on this
// card; 256 of 100 to 2,048 over bf16: 190 us, 6.0; one of 131,072 over e4m3: 50
// us and 5.5 in the join (its workgroups end from 31 to 49 us: a CU's older
// waves go first).  A call of little work is its latency: some 2 us to launch,
// 2 for its share, 2 to 3 for its first keys, 2 for each further tile of a wave.
#include "attend_common.h"

#include <cmath>
#include <type_traits>

namespace apc {
namespace {

constexpr int TILE = 32;
constexpr int CUS = 256;
constexpr float SLACK = 8.f;            // weights stay below 2^8

// 16 x 16 x 32: D = A B + C; a lane's 8 values of A are row lane % 16, of B
// column lane % 16, both at k = 8 (lane / 16); of D column lane % 16, rows 4 (lane / 16) + r
template <bool BF> __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// two f16 as the sum of two bf16 each: exact, 11 bits are 8 and 3
__device__ inline void split_f16(uint32_t w, uint32_t& hi, uint32_t& lo)
{
    const f32x2 x = unpack<false>(w);
    hi = pack<true>(x.x, x.y);
    const f32x2 y = unpack<true>(hi);
    lo = pack<true>(x.x - y.x, x.y - y.y);
}

// per half of w (bf16 weights): 1 for a weight, 0 for none, NaN for NaN, as f16 or bf16
template <bool BF> __device__ inline uint32_t any_weight(uint32_t w)
{
    constexpr uint32_t ONE = BF ? 0x3f80u : 0x3c00u;
    return ((w & 0xffffu) ? ONE : 0u) | ((w >> 16) ? ONE << 16 : 0u) | (not_finite<true>(w) & 0x7fff7fffu);
}

// N dwords of keys or values.  ONCE: marked not to displace what is in the
// caches (256 sequences of 100 to 2,048 tokens, bf16: 191 us, 213 without; 64 of
// 16,384 to 32,768, e4m3: 538 and 573).  Not so where the next call may find them
// there (16 of 1,024, bf16: 15.9 us, 21.2 marked), and where several workgroups
// have the query heads of one key-value head, the second of which finds what the
// first read (64 sequences, 128 query heads on one of 128, bf16: 160 us, 222 marked).
template <int N, bool ONCE> __device__ inline void stream(uint32_t* to, const uint8_t* from)
{
    if constexpr (N == 1) {
        const auto* p = reinterpret_cast<const uint32_t*>(from);
        *to = ONCE ? __builtin_nontemporal_load(p) : *p;
    } else {
        using V = uint32_t __attribute__((ext_vector_type(N)));
        const auto* p = reinterpret_cast<const V*>(from);
        const V x = ONCE ? __builtin_nontemporal_load(p) : *p;
        __builtin_memcpy(to, &x, 4 * N);
    }
}

// a value that every lane holds alike, in scalar registers
__device__ inline int64_t uniform(int64_t x)
{
    return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)x) | (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// x / y for x, y > 0, in 32 bits where they suffice
__device__ inline int64_t quotient(int64_t x, int64_t y)
{
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// a sequence's visible tokens [first, len), and their tiles
struct Span {
    int first, len, tile0, tiles;
    __device__ Span(const AttendArgs& a, const AttendPlan& p, int32_t held)
    {
        const int32_t cap = a.max_pages << p.shift;
        len = held < 0 ? 0 : held < cap ? held : cap;
        first = a.window > 0 && len > a.window ? len - a.window : 0;
        tile0 = first / TILE;
        tiles = (len + TILE - 1) / TILE - tile0;
    }
};

// what a unit costs, in tiles: a piece of work begins with its queries and ends
// with the waves' results joined, which takes about as long as four tiles
constexpr int EXTRA = 4;
__device__ inline int cost(int tiles) { return tiles > 0 ? tiles + EXTRA : 0; }

// n tiles of a unit, from its tile `off` on; n = 0 with seq < 0: no work
struct Piece {
    int seq, head, off, n;
    Span span;
    __device__ int begin() const { return span.tile0 + off; }
    __device__ int end() const { return span.tile0 + off + n; }
};

// Workspace: the records (int32), then the partial sums (float32, padded d a
// row), then their maxima and sums of weights.  Two records a workgroup, of its
// first cut unit and of its last: the unit, and whether its first tile and its
// last were in the piece.
constexpr int32_t REC_START = 1, REC_END = 2;
__host__ __device__ inline int64_t rec_ints(const AttendPlan& p) { return ((int64_t)p.groups * p.qtiles * 2 + 3) / 4 * 4; }
__device__ inline float* partial_sums(const AttendArgs& a, const AttendPlan& p)
{
    return static_cast<float*>(a.ws) + rec_ints(p);
}
__device__ inline float* partial_stats(const AttendArgs& a, const AttendPlan& p, int rows, int dp)
{
    return partial_sums(a, p) + (int64_t)p.groups * p.qtiles * 2 * rows * dp;
}

// CUT: stretches of the row of all tiles; else whole units.  ONCE: see stream()
template <int DT, int CDT, int DP, int NQ, int WAVES, bool CUT, bool ONCE>
__global__ __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2) void k_attend(apc_kv c, AttendArgs a, AttendPlan p)
{
    using T = typename Elem<DT>::T;
    constexpr bool E8 = CDT == APC_E4M3, QBF = DT == APC_BF16;
    constexpr int ES = E8 ? 1 : 2, EPL = DP / 16;               // values: elements of a row a lane owns
    constexpr int KW = 4 * ES, VW = EPL * ES / 4;               // dwords: 16 elements of a key, EPL of a value
    constexpr int SL = DP < 128 ? DP : 128;                     // elements of a round of the final sums
    __shared__ float part[WAVES][16][SL + 4];
    __shared__ float ml[2][WAVES][NQ * 16][2];

    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // query tiles of one stretch come to one XCD (workgroups go round over 8): they read the same keys
    const int id = blockIdx.x, qt = id / 8 % p.qtiles, wg = id / 8 / p.qtiles * 8 + id % 8;
    if (wg >= p.groups) return;
    const int group = a.q_heads / c.heads, rows = group < NQ * 16 ? group : NQ * 16;
    auto span_of = [&](int seq) INLINE { return Span(a, p, table_entry(a.lengths, seq)); };

    Piece cur{0, 0, 0, 0, Span(a, p, 0)};                       // what is worked on
    int64_t unit_end = (int64_t)a.b * c.heads;                  // CUT: the stretch ends at this unit's tile off_end
    int off_end = 0;
    int32_t* rec = static_cast<int32_t*>(a.ws) + ((int64_t)wg * p.qtiles + qt) * 2;
    if constexpr (CUT) {
        // sequences that hold nothing, shared out among the workgroups: zeros
        for (int seq = wg; seq < a.b; seq += p.groups) {
            if (span_of(seq).tiles > 0) continue;
            const int h0 = qt * NQ * 16, n = group - h0 < NQ * 16 ? group - h0 : NQ * 16;
            for (int i = wave; i < c.heads * n; i += WAVES) {   // a head a wave: all elements pass 32 bits
                const int h = i / n * group + h0 + i % n;
                T* const to = static_cast<T*>(a.out) + seq * a.out_row + h * a.out_head;
                for (int d = lane; d < c.d; d += 64) to[d] = 0;
                if (a.lse && lane == 0) a.lse[(int64_t)seq * a.q_heads + h] = -INFINITY;
            }
        }
        // The stretch, found by every wave for itself: a lane has four of every
        // 256 sequences, their costs (of one head) and the sum up to its last.
        struct Costs { int held[4], cost[4], upto, total; };
        auto costs_of = [&](int seq0) INLINE {
            Costs k;
            int sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int seq = seq0 + lane * 4 + i;
                k.held[i] = seq < a.b ? a.lengths[seq] : 0;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) sum += k.cost[i] = cost(Span(a, p, k.held[i]).tiles);
            k.upto = sum;
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int o = __shfl_up(k.upto, d, 64);
                if (lane >= d) k.upto += o;
            }
            k.total = __builtin_amdgcn_readlane(k.upto, 63);
            return k;
        };
        const Costs all = costs_of(0);                          // of the first 256; the others are read again
        int64_t total = all.total;
        for (int seq0 = 256; seq0 < a.b; seq0 += 256) total += costs_of(seq0).total;
        total *= c.heads;
        // Equal shares of at least min_share.  A CU's second workgroup is its
        // slower one, so a few of them more than there are CUs would only be waited for
        // (one stretch stays one, with more query tiles than CUs too).
        int64_t used = quotient(total, p.min_share);
        used = used < 1 ? 1 : used < p.groups ? used : p.groups;
        if (used > 1 && used * p.qtiles > CUS) used = used * p.qtiles / CUS * CUS / p.qtiles;
        used = uniform(used);
        // A cut inside a unit: of a short one moved to its nearer end, of a
        // longer one to the nearest multiple of four tiles in proportion.
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (wg + i >= used || total == 0) break;
            const int64_t want = uniform(quotient(total * (wg + i), used));
            const int64_t want_seq = uniform(quotient(want, c.heads));      // want < x heads: want_seq < x
            Costs k = all;
            int64_t ahead = 0;                                  // costs (of one head) of the sequences ahead
            int seq = 0;
            while (want_seq >= ahead + k.total) {
                ahead += k.total;
                seq += 256;
                k = costs_of(seq);
            }
            const int l = __builtin_ctzll(__ballot(k.upto > (int)(want_seq - ahead)));
            int sum = 0, held = 0, costs = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_readlane(k.cost[e], l);
            ahead += __builtin_amdgcn_readlane(k.upto, l) - sum;
            seq += l * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                held = __builtin_amdgcn_readlane(k.held[e], l);
                costs = __builtin_amdgcn_readlane(k.cost[e], l);
                if (want_seq < ahead + costs) break;
                ahead += costs;
                ++seq;
            }
            const int64_t inside = want - ahead * c.heads;
            const int head = __builtin_amdgcn_readfirstlane((int)quotient(inside, costs));
            const int at = (int)(inside - (int64_t)head * costs), tiles = costs - EXTRA;
            // in float32: both neighbours do the same operations on the same numbers
            const int near = (int)((float)at * ((float)tiles / (float)costs) / WAVES + 0.5f) * WAVES;
            const int off = __builtin_amdgcn_readfirstlane(tiles <= p.snap ? (2 * at < costs ? 0 : tiles) : near < tiles ? near : tiles);
            if (i == 0) {
                cur = Piece{seq, head, off, 0, Span(a, p, held)};
            } else {
                unit_end = (int64_t)seq * c.heads + head;
                off_end = off;
            }
        }
        if (wg >= used || total == 0) {
            if (threadIdx.x < 2) rec[threadIdx.x] = 0;
            return;
        }
    } else {
        cur.seq = wg / c.heads, cur.head = wg % c.heads;
        cur.span = span_of(cur.seq);
        cur.n = cur.span.tiles;
    }
    // the piece after the unit's first u.off tiles, or of the next unit that the stretch reaches
    auto settle = [&](Piece& u) INLINE {
        int64_t unit = (int64_t)u.seq * c.heads + u.head;
        while (u.off >= u.span.tiles && unit < unit_end) {
            u.off = 0;
            if (u.span.tiles == 0 || ++u.head == c.heads) {
                u.head = 0;
                if (++u.seq < a.b) u.span = span_of(u.seq);
            }
            unit = (int64_t)u.seq * c.heads + u.head;
        }
        u.n = unit < unit_end ? u.span.tiles - u.off : unit == unit_end ? off_end - u.off : 0;
        if (u.n <= 0) u.seq = -1, u.n = 0;
    };
    if constexpr (CUT) {
        settle(cur);
        if (cur.seq < 0) {                                      // the cuts moved past each other's units
            if (threadIdx.x < 2) rec[threadIdx.x] = 0;
            return;
        }
    }
    auto following = [&](Piece u) INLINE {
        Piece v = u;
        if constexpr (CUT) {
            v.off += u.n;
            settle(v);
        } else {
            const int64_t unit = (int64_t)u.seq * c.heads + u.head + p.groups;
            if (unit < (int64_t)a.b * c.heads) {
                v.seq = (int)(unit / c.heads), v.head = (int)(unit % c.heads);
                v.span = span_of(v.seq);
                v.n = v.span.tiles;
            } else {
                v.seq = -1, v.n = 0;
            }
        }
        return v;
    };

    // a lane's places in a row; past a row's end (d < DP) it reads other elements
    // of the row: of keys they meet zeros of q, and are zeroed where they can be
    // infinite; of values they go into columns that are not stored
    const int row_bytes = c.d * ES, in_page = c.page - 1;
    int koff[DP / 64];
    bool in_row[DP / 64];
#pragma unroll
    for (int j = 0; j < DP / 64; ++j) {
        in_row[j] = j < DP / 128 || j * 64 + g * 16 < c.d;      // where DP is 128 or 256, d > DP / 2
        koff[j] = col * row_bytes + (in_row[j] ? j * 64 + g * 16 : 0) * ES;
    }
    const int voff = 4 * g * row_bytes + (col * EPL < c.d ? col * EPL : 0) * ES;

    // Queries: column col of tile n is query head (qt NQ + n) 16 + col of the group,
    // past its last head that one again, whose results nobody stores.  Loads that
    // all lanes do, and zeros past a row's end put in when the loads are there.
    u32x4 q[NQ][DP / 32];
    auto load_q = [&](Piece u) INLINE {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int qh = (qt * NQ + n) * 16 + col, head = qh < group ? qh : group - 1;
            const T* row = static_cast<const T*>(a.q) + u.seq * a.q_row + (int64_t)(u.head * group + head) * a.q_head;
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) __builtin_memcpy(&q[n][j], row + (in_row[j / 2] ? j / 2 * 64 + g * 16 + j % 2 * 8 : 0), 16);
        }
    };
    auto trim_q = [&]() INLINE {
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int j = DP / 128 * 2; j < DP / 32; ++j) q[n][j] = in_row[j / 2] ? q[n][j] : u32x4{0, 0, 0, 0};
    };

    struct Pages { int32_t id[2]; };                            // of a tile's halves
    auto find = [&](Piece u, int t) INLINE {
        const int32_t* table = a.pages + u.seq * a.ld_pages;
        const int last = (u.span.len - 1) >> p.shift;
        Pages pg;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = (t * TILE + 16 * h) >> p.shift;
            pg.id[h] = table_entry(table, at < last ? at : last);
        }
        return pg;
    };
    auto there = [&](int32_t page) INLINE { return (uint32_t)page < (uint64_t)c.n_pages; };
    struct Rows { int64_t at[2]; };                             // first rows of a tile's halves (of page 0 where there is none)
    auto rows_of = [&](int head, int t, Pages pg) INLINE {
        Rows r;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            r.at[h] = (((int64_t)(there(pg.id[h]) ? pg.id[h] : 0) * c.heads + head) << p.shift) + ((t * TILE + 16 * h) & in_page);
        return r;
    };
    struct Keys { uint32_t w[2][DP / 64][KW]; f32x4 scale[2]; };
    struct Values { uint32_t w[8][VW]; f32x4 scale[2]; };
    Keys key;
    Values value;
    auto load_k = [&](Keys& to, Rows r) INLINE {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* base = static_cast<const uint8_t*>(c.k) + r.at[h] * row_bytes;
#pragma unroll
            for (int j = 0; j < DP / 64; ++j)
#pragma unroll
                for (int w = 0; w < KW; w += 4) stream<4, ONCE>(to.w[h][j] + w, base + koff[j] + w * 4);
            if constexpr (E8) to.scale[h] = *reinterpret_cast<const f32x4*>(c.k_scale + r.at[h] + 4 * g);
        }
    };
    auto load_v = [&](Values& to, Rows r) INLINE {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* base = static_cast<const uint8_t*>(c.v) + r.at[h] * row_bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int w = 0; w < VW; w += 4) stream<(VW < 4 ? VW : 4), ONCE>(to.w[4 * h + i] + w, base + voff + i * row_bytes + w * 4);
            if constexpr (E8) to.scale[h] = *reinterpret_cast<const f32x4*>(c.v_scale + r.at[h] + 4 * g);
        }
    };

    // (0 times an infinite factor is no score: then products are taken times 4)
    const bool lift = __builtin_amdgcn_readfirstlane(__builtin_fabsf(a.scale) > 2.3e38f);
    const float to_log2 = (lift ? 0.25f * a.scale : a.scale) * LOG2E;
    constexpr int PER = 4 / ES;                                 // elements of a dword of values
    // the i-th pair of keys' dwords put together, element by element
    auto pairs = [](u32x4* v, int i, uint32_t y, uint32_t z) INLINE {
        if constexpr (E8) {
            const uint32_t a01 = __builtin_amdgcn_perm(z, y, 0x05010400u), a23 = __builtin_amdgcn_perm(z, y, 0x07030602u);
            v[0][i] = from_e4m3<true, false>(a01);
            v[1][i] = from_e4m3<true, true>(a01);
            v[2][i] = from_e4m3<true, false>(a23);
            v[3][i] = from_e4m3<true, true>(a23);
        } else {
            v[0][i] = __builtin_amdgcn_perm(z, y, 0x05040100u);
            v[1][i] = __builtin_amdgcn_perm(z, y, 0x07060302u);
        }
    };
    f32x4 o[NQ][EPL];
    float m[NQ], l[NQ];
    auto clear = [&]() INLINE {
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            m[n] = LOWEST;
            l[n] = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) o[n][e] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    // The loaded tile t, its pages pg, into o, m and l; of what follows, where there
    // is more, keys and values are loaded as soon as their registers are free.
    // CAREFUL: right for infinite values, which a weight's second part (0, or
    // negative) would make NaN, and near the end of float32's range, where weights
    // must not pass 1.
    auto add_tile = [&](auto care, Span span, int t, Pages pg, Keys& key, Values& value, bool more, Rows next) INLINE {
        constexpr bool CAREFUL = decltype(care)::value;
        // scores
        f32x4 s[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                s[n][h] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < DP / 32; ++j) {
                    u32x4 k;
                    if constexpr (E8) {
                        const uint32_t lo = key.w[h][j / 2][j % 2 * 2], hi = key.w[h][j / 2][j % 2 * 2 + 1];
                        k = u32x4{from_e4m3<QBF, false>(lo), from_e4m3<QBF, true>(lo), from_e4m3<QBF, false>(hi),
                                  from_e4m3<QBF, true>(hi)};
                    } else {
                        __builtin_memcpy(&k, &key.w[h][j / 2][j % 2 * 4], 16);
                        if (j / 2 >= DP / 128) k = in_row[j / 2] ? k : u32x4{0, 0, 0, 0};
                    }
                    s[n][h] = mfma<QBF>(k, q[n][j], s[n][h]);
                }
            }
        f32x4 factor[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            factor[h] = f32x4{to_log2, to_log2, to_log2, to_log2};
            if constexpr (E8) factor[h] *= key.scale[h];
        }
        if (more) load_k(key, next);
        if (__builtin_expect(lift, 0))
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) s[n][h] *= 4.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[n][h] *= factor[h];

        // the first and last tiles, and those with pages that are not there: their unseen keys drop out
        const bool whole = t * TILE >= span.first && t * TILE + TILE <= span.len && there(pg.id[0]) && there(pg.id[1]);
        if (!whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int tok = t * TILE + 16 * h + 4 * g + i;
                    const bool seen = tok >= span.first && tok < span.len && there(pg.id[h]);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[n][h][i] = seen ? s[n][h][i] : -INFINITY;
                    if constexpr (E8) value.scale[h][i] = seen ? value.scale[h][i] : 0.f;
#pragma unroll
                    for (int w = 0; w < VW; ++w) value.w[4 * h + i][w] = seen ? value.w[4 * h + i][w] : 0u;
                }
        }

        // the running maximum
        float top[NQ];
        bool over = false;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            top[n] = s[n][0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top[n] = __builtin_fmaxf(top[n], s[n][i / 4][i % 4]);
            over |= top[n] > m[n] + (CAREFUL ? 0.f : SLACK);
        }
        if (__any(over)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float y = __builtin_fmaxf(m[n], top[n]);
                y = __builtin_fmaxf(y, __shfl_xor(y, 16, 64));
                y = __builtin_fmaxf(y, __shfl_xor(y, 32, 64));
                const float f = __builtin_amdgcn_exp2f(m[n] - y);
                m[n] = y;
                l[n] *= f;
#pragma unroll
                for (int e = 0; e < EPL; ++e) o[n][e] *= f;
            }
        }

        // weights, in two parts
        u32x4 hi[NQ], lo[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[i] = __builtin_amdgcn_exp2f(s[n][i / 4][i % 4] - m[n]);
                l[n] += w[i];
                if constexpr (E8) w[i] *= value.scale[i / 4][i % 4];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[n][i] = pack<true>(w[2 * i], w[2 * i + 1]);
                const f32x2 y = unpack<true>(hi[n][i]);
                lo[n][i] = pack<true>(w[2 * i] - y.x, w[2 * i + 1] - y.y);
            }
        }

        // infinite and NaN values, or e4m3 weights: their products alone, and 0 in their place after that
        if constexpr (CAREFUL) {
            u32x4 x[NQ];
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if constexpr (E8) {
                        const uint32_t out = not_finite<true>(hi[n][i]);
                        x[n][i] = hi[n][i] & out;
                        hi[n][i] &= ~out;
                        lo[n][i] &= ~out;
                    } else {
                        x[n][i] = any_weight<QBF>(hi[n][i]);
                    }
                }
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                u32x4 v[PER];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t y = value.w[2 * i][w], z = value.w[2 * i + 1][w];
                    if constexpr (!E8) {
                        y &= not_finite<QBF>(y), z &= not_finite<QBF>(z);
                        value.w[2 * i][w] ^= y, value.w[2 * i + 1][w] ^= z;
                    }
                    pairs(v, i, y, z);
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < PER; ++e) o[n][w * PER + e] = mfma<E8 || QBF>(v[e], x[n], o[n][w * PER + e]);
            }
        }

        // values: element e of every key's row, keys in pairs
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            u32x4 v[PER];
#pragma unroll
            for (int i = 0; i < 4; ++i) pairs(v, i, value.w[2 * i][w], value.w[2 * i + 1][w]);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                u32x4 rest;
                if constexpr (CDT == APC_F16) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t a, b;
                        split_f16(v[e][i], a, b);
                        v[e][i] = a, rest[i] = b;
                    }
                }
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    f32x4& to = o[n][w * PER + e];
                    to = mfma<true>(v[e], hi[n], to);
                    to = mfma<true>(v[e], lo[n], to);
                    if constexpr (CDT == APC_F16) {
                        to = mfma<true>(rest, hi[n], to);
                        to = mfma<true>(rest, lo[n], to);
                    }
                }
            }
        }
        if (more) load_v(value, next);
    };
    int parts = 0;                                              // partial results written
    int turn = 0;
    int t = cur.begin() + wave;                                 // this wave's tile, loaded or on its way
    Pages pc{};                                                 // its pages
    if (t < cur.end()) {
        pc = find(cur, t);
        const Rows r = rows_of(cur.head, t, pc);
        load_k(key, r);
        load_v(value, r);
    }
    load_q(cur);
    while (true) {
        const int end = cur.end();
        const Piece nxt = following(cur);
        const int t_nxt = nxt.begin() + wave;
        const bool more = nxt.n > 0 && t_nxt < nxt.end();       // this wave has a tile of the next piece
        Pages pn{}, pg{};                                       // of the next piece's tile, of the next of this piece
        if (more) pn = find(nxt, t_nxt);
        if (t + WAVES < end) pg = find(cur, t + WAVES);
        if (t >= end && more) {
            const Rows r = rows_of(nxt.head, t_nxt, pn);
            load_k(key, r);
            load_v(value, r);
        }
        trim_q();
        clear();
        while (t < end) {
            const bool inside = t + WAVES < end;
            const Rows r = inside ? rows_of(cur.head, t + WAVES, pg) : rows_of(nxt.head, t_nxt, pn);
            add_tile(std::false_type{}, cur.span, t, pc, key, value, inside || more, r);
            pc = inside ? pg : pn;
            t += WAVES;
            if (t + WAVES < end) pg = find(cur, t + WAVES);
        }
        // Infinities or NaN came out: once more with care, one tile after the other,
        // in registers of its own and the next tile loaded again after it, so that the
        // loop above keeps the registers it has without this (as one loop of both: 64
        // sequences of 4,096 to 8,192, 12 heads of 64, e4m3: 124 us, 118 so).
        float z = 0.f;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < EPL; ++e)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = __builtin_fmaf(o[n][e][i], 0.f, z);
        if (__builtin_expect(__any(z != 0.f), 0)) {
            clear();
            for (int again = cur.begin() + wave; again < end; again += WAVES) {
                const Pages at = find(cur, again);
                const Rows r = rows_of(cur.head, again, at);
                Keys k;
                Values v;
                load_k(k, r);
                load_v(v, r);
                add_tile(std::true_type{}, cur.span, again, at, k, v, false, r);
            }
            // (where no tile follows, the first of the pool, which nobody reads)
            const Rows r = rows_of(more ? nxt.head : 0, more ? t_nxt : 0, pn);
            load_k(key, r);
            load_v(value, r);
        }
        if (nxt.seq >= 0) load_q(nxt);

        // the waves' results into one: m and l first, then the outputs' sums, 128 elements of 16 heads a round
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16, 64);
            l[n] += __shfl_xor(l[n], 32, 64);
            if (g == 0) {
                ml[turn][wave][n * 16 + col][0] = m[n];
                ml[turn][wave][n * 16 + col][1] = l[n];
            }
        }
        const bool whole_unit = cur.n == cur.span.tiles;
        constexpr int TPH = 4 * WAVES, OWN = SL / TPH;          // threads of a head, elements of a thread
        const int hrow = threadIdx.x / TPH, dcol = threadIdx.x % TPH * OWN;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int d0 = 0; d0 < DP; d0 += SL) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = (4 * g + i) * EPL - d0;
                    if (d >= 0 && d < SL) {
#pragma unroll
                        for (int e = 0; e < EPL; e += 4)
                            *reinterpret_cast<f32x4*>(&part[wave][col][d + e]) =
                                f32x4{o[n][e][i], o[n][e + 1][i], o[n][e + 2][i], o[n][e + 3][i]};
                    }
                }
                __syncthreads();
                // every thread sums and only the stores are some threads': copies of the next round's registers,
                // where the compiler makes any here, would be lost in the threads that a branch leaves out
                // (the build looks for such copies)
                const int qh = (qt * NQ + n) * 16 + hrow;
                const bool mine = qh < group && d0 + dcol < c.d;
                float top = LOWEST, sum = 0.f, v[OWN] = {};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = __builtin_fmaxf(top, ml[turn][w][n * 16 + hrow][0]);
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = __builtin_amdgcn_exp2f(ml[turn][w][n * 16 + hrow][0] - top);
                    sum = __builtin_fmaf(f, ml[turn][w][n * 16 + hrow][1], sum);
#pragma unroll
                    for (int i = 0; i < OWN; ++i) v[i] = __builtin_fmaf(f, part[w][hrow][dcol + i], v[i]);
                }
                if (!CUT || whole_unit) {
                    const int64_t qrow = (int64_t)cur.head * group + qh;
                    const float f = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
                    for (int i = 0; i < OWN; ++i) v[i] = sum == 0.f ? 0.f : v[i] * f;
                    T* const to = static_cast<T*>(a.out) + cur.seq * a.out_row + qrow * a.out_head + d0 + dcol;
                    // d is a multiple of 16: a thread's elements, where they are more, can end past it
                    constexpr int ST = OWN < 16 ? OWN : 16;
#pragma unroll
                    for (int i = 0; i < OWN; i += ST)
                        if (mine && d0 + dcol + i < c.d) store_values<DT, ST>(to + i, v + i);
                    if (a.lse && mine && d0 + dcol == 0)
                        a.lse[(int64_t)cur.seq * a.q_heads + qrow] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
                } else if (mine) {
                    const int64_t slot = (((int64_t)wg * p.qtiles + qt) * 2 + parts) * rows + n * 16 + hrow;
                    float* po = partial_sums(a, p) + slot * DP + d0 + dcol;
#pragma unroll
                    for (int i = 0; i < OWN; i += 4) *reinterpret_cast<f32x4*>(po + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
                    if (d0 + dcol == 0) {
                        float* pm = partial_stats(a, p, rows, DP) + slot * 2;
                        pm[0] = top;
                        pm[1] = sum;
                    }
                }
            }
        if (CUT && !whole_unit) {
            if (threadIdx.x == 0)
                rec[parts] = (cur.off == 0 ? REC_START : 0) | (cur.off + cur.n == cur.span.tiles ? REC_END : 0) |
                             (cur.seq * c.heads + cur.head) << 2;
            ++parts;
        }
        if (nxt.seq < 0) break;
        // the next piece; its ml is another one, while this one's is still read
        if (t >= end && !(cur.begin() + wave < end)) pc = pn;   // no tile in this piece: pc is still to be set
        cur = nxt;
        t = t_nxt;
        turn ^= 1;
    }
    if (CUT && (int)threadIdx.x >= parts && threadIdx.x < 2) rec[threadIdx.x] = 0;
}

// Joins the cut units: the workgroups that shared one are neighbours, and each
// one's part is its first but for the one that began the unit.  A workgroup for
// every unit, or for every stretch where there are fewer (a stretch begins at
// most one unit that it does not end), and query head, its threads over (some
// of the parts) x (elements).
template <int DT, int DP, int JOIN>
__global__ __launch_bounds__(JOIN) void k_attend_join(apc_kv c, AttendArgs a, AttendPlan p, int rows, bool by_unit)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = DP / 4, PARTS = JOIN / LANES, AHEAD = 4;
    __shared__ float acc[PARTS][DP];
    __shared__ float sums[PARTS], tops[PARTS];
    __shared__ int from, to;                                    // record that begins the unit, workgroup that ends it
    const int of = blockIdx.x / p.qtiles, qt = blockIdx.x % p.qtiles, h = blockIdx.y, group = a.q_heads / c.heads;
    if (qt * p.nq * 16 + h >= group) return;
    const int32_t* rec = static_cast<const int32_t*>(a.ws);
    auto record = [&](int i) { return rec[((int64_t)(i / 2) * p.qtiles + qt) * 2 + i % 2]; };
    if (threadIdx.x == 0) from = -1, to = -1;
    __syncthreads();
    int unit = of;
    if (by_unit) {
        for (int i = threadIdx.x; i < 2 * p.groups; i += JOIN) {
            const int32_t r = record(i);
            if (r >> 2 == unit && (r & REC_START)) from = i;    // at most one of each
            if (r >> 2 == unit && (r & REC_END)) to = i / 2;
        }
        __syncthreads();
    } else {
        const int32_t r0 = record(2 * of), r1 = record(2 * of + 1);
        const int which = (r0 & 3) == REC_START ? 0 : (r1 & 3) == REC_START ? 1 : -1;
        if (which < 0) return;
        unit = (which ? r1 : r0) >> 2;
        for (int i = of + 1 + threadIdx.x; i < p.groups; i += JOIN) {
            const int32_t r = record(2 * i);
            if (r >> 2 == unit && (r & REC_END)) to = i;
        }
        if (threadIdx.x == 0) from = 2 * of + which;
        __syncthreads();
    }
    if (from < 0 || to < 0) return;                             // not cut
    const int wg0 = from / 2, which = from % 2, n = to - wg0 + 1;
    auto slot = [&](int i) { return (((int64_t)(wg0 + i) * p.qtiles + qt) * 2 + (i == 0 ? which : 0)) * rows + h; };
    const float* po = partial_sums(a, p);
    const float* pm = partial_stats(a, p, rows, DP);
    const int d = threadIdx.x % LANES * 4, part = threadIdx.x / LANES;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    float top = LOWEST, sum = 0.f;
    for (int i0 = part; i0 < n; i0 += PARTS * AHEAD) {
        f32x4 x[AHEAD];
        float m[AHEAD], l[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * PARTS < n ? i0 + k * PARTS : i0;
            x[k] = *reinterpret_cast<const f32x4*>(po + slot(i) * DP + d);
            m[k] = pm[slot(i) * 2];
            l[k] = pm[slot(i) * 2 + 1];
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k * PARTS >= n) break;
            const float y = __builtin_fmaxf(top, m[k]);
            const float was = __builtin_amdgcn_exp2f(top - y), is = __builtin_amdgcn_exp2f(m[k] - y);
            v = v * was + x[k] * is;
            sum = sum * was + l[k] * is;
            top = y;
        }
    }
    *reinterpret_cast<f32x4*>(&acc[part][d]) = v;
    if (threadIdx.x % LANES == 0) sums[part] = sum, tops[part] = top;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int i = 0; i < PARTS; ++i) top = __builtin_fmaxf(top, tops[i]);
    sum = 0.f;
    v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        const float f = __builtin_amdgcn_exp2f(tops[i] - top);
        sum = __builtin_fmaf(f, sums[i], sum);
        v += f * *reinterpret_cast<const f32x4*>(&acc[i][d]);
    }
    const float f = sum == 0.f ? 0.f : 1.0f / sum;
    const float out[4] = {sum == 0.f ? 0.f : v.x * f, sum == 0.f ? 0.f : v.y * f, sum == 0.f ? 0.f : v.z * f,
                          sum == 0.f ? 0.f : v.w * f};
    const int seq = unit / c.heads, qh = unit % c.heads * group + qt * p.nq * 16 + h;
    if (d < c.d) store_values<DT, 4>(static_cast<T*>(a.out) + seq * a.out_row + (int64_t)qh * a.out_head + d, out);
    if (a.lse && d == 0) a.lse[(int64_t)seq * a.q_heads + qh] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
}

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
// query tiles of a wave: two share a key's registers, but wide heads have no registers for them
int query_tiles(int d, int group) { return group > 16 && padded(d) <= 128 ? 2 : 1; }

constexpr int SNAP = 16;                // in a stretch, units of up to so many tiles are not cut
// Up to WIDE_UNITS units, a unit has a workgroup of eight waves, if it has one
// to itself at all.  It has where even the table's longest would be no more
// than WHOLE_UNIT bytes, which spares a second launch (64 x 8 units of 1,024
// tokens, e4m3, heads of 128, 279 KB: 27.4 us, 32.9 in stretches; 4 x 8 of
// 1,024, bf16, 524 KB: 15.5 either way; of 2,048: 24.5 and 17.0), or WHOLE_UNIT_MANY where there is a unit
// for every other CU (32 x 8 of 1,024, bf16: 25.3 us, 31.8 in stretches; 16 x
// 8: 16.0 and 20.5).
constexpr int64_t WIDE_UNITS = 256;
constexpr int64_t WHOLE_UNIT = 288 << 10, WHOLE_UNIT_MANY = 560 << 10;
constexpr int MIN_SHARE = 8;            // tiles of a stretch, at least
// Stretches: the workgroups that the chip holds at once.  Two a CU (64 long
// sequences over e4m3: 538 us; one 627, three 558, four 543); four with rows of
// 64 bytes, whose tiles are small (64 sequences of 8,192 to 16,384 tokens, 12
// heads of 64, e4m3: 228 us, 235 with two); one with wide heads, which leave
// registers for one (32 sequences of 4,096 to 8,192, 4 heads of 256, bf16: 149
// us, 161 with two).
int stretches(const apc_kv& c, int qtiles)
{
    const int groups = padded(c.d) > 128 ? 256 : c.d * elem_bytes(c.dt) <= 64 ? 1024 : 512;
    return groups / qtiles > 0 ? groups / qtiles : 1;
}
// One wave has a unit to itself, and nothing to join, where the unit is a tile,
// or where there are enough short units for every SIMD: of eight tiles at most
// (256 x 8 units of 128 tokens, bf16, heads of 128: 25.5 us, 30.8 with four
// waves; 149 x 11 of one to three, e4m3: 9.1 and 16.9), or of 32 with wide heads,
// whose registers leave a CU a single workgroup of four (256 x 8 of 512, heads of
// 256, e4m3: 102.5 us and 125.7; bf16, 1 MB a unit: 183 us, 209 in stretches).
// Narrower heads have no gain there, and lose where the lengths differ (256 x 12
// of 1 to 500 tokens, heads of 64: 47.2 us and 40.6).
bool one_wave(int d, int64_t units, int64_t seen)
{
    return seen <= 1 || (units >= 1024 && seen <= 8) || (padded(d) > 128 && units >= 2048 && seen <= 32);
}
// Calls that could read as much find little of it again in the 256 MB
// last-level cache, even where a next call reads the same keys and values
// (three caches in turn, 24 x 8 units of 1,024 tokens over bf16, 101 MB: 21.1 us,
// 22.7 marked; 32 x 8, 134 MB: 27.0 and 25.2).
constexpr int64_t ONCE_BYTES = 100 << 20;
constexpr int64_t UNCUT_GROUPS = 1 << 16;
int64_t tiles_of(const apc_kv& c, int64_t max_pages) { return (max_pages * c.page + TILE - 1) / TILE; }
int64_t bytes_of(const apc_kv& c, int64_t tiles) { return tiles * TILE * 2 * c.d * elem_bytes(c.dt); }
// Stretches of units of so many tiles: no fewer for more units or tiles
int32_t cut_groups(const apc_kv& c, int64_t units, int64_t tiles, int qtiles)
{
    const int64_t shares = (units * (tiles + EXTRA) + MIN_SHARE - 1) / MIN_SHARE, most = stretches(c, qtiles);
    return (int32_t)(shares < most ? shares : most);
}
AttendPlan plan(const apc_kv& c, int32_t b, int32_t q_heads, int32_t max_pages, int32_t window)
{
    AttendPlan p{};
    const int group = q_heads / c.heads;
    while ((1 << p.shift) < c.page) ++p.shift;
    p.nq = query_tiles(c.d, group);
    p.qtiles = (group + 16 * p.nq - 1) / (16 * p.nq);
    p.snap = SNAP;
    p.min_share = MIN_SHARE;
    const int64_t units = (int64_t)b * c.heads, tiles = tiles_of(c, max_pages);
    // a window bounds the tiles that are seen, too
    const int64_t seen = window > 0 && window / TILE + 2 < tiles ? window / TILE + 2 : tiles;
    const int64_t unit_bytes = bytes_of(c, seen);
    p.waves = padded(c.d) <= 128 && units * p.qtiles <= WIDE_UNITS && seen > 4 ? 8
              : one_wave(c.d, units * p.qtiles, seen) ? 1 : 4;
    p.cut = p.waves != 1 && unit_bytes > (p.waves == 8 && units >= WIDE_UNITS / 2 ? WHOLE_UNIT_MANY : WHOLE_UNIT);
    p.groups = p.cut ? cut_groups(c, units, seen, p.qtiles) : (int32_t)(units < UNCUT_GROUPS ? units : UNCUT_GROUPS);
    p.once = p.qtiles == 1 && units * unit_bytes >= ONCE_BYTES;
    return p;
}

template <int DT, int CDT, int DP, int NQ, bool ONCE>
hipError_t launch_q(const apc_kv& c, const AttendArgs& a, const AttendPlan& p, hipStream_t s)
{
    const dim3 grid((unsigned)((p.groups + 7) / 8 * 8 * p.qtiles));
    if (!p.cut) {
        if constexpr (DP <= 128) {
            if (p.waves == 8) k_attend<DT, CDT, DP, NQ, 8, false, ONCE><<<grid, dim3(512), 0, s>>>(c, a, p);
        }
        if (p.waves == 1) k_attend<DT, CDT, DP, NQ, 1, false, ONCE><<<grid, dim3(64), 0, s>>>(c, a, p);
        if (p.waves == 4) k_attend<DT, CDT, DP, NQ, 4, false, ONCE><<<grid, dim3(256), 0, s>>>(c, a, p);
        return hipGetLastError();
    }
    k_attend<DT, CDT, DP, NQ, 4, true, ONCE><<<grid, dim3(256), 0, s>>>(c, a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int group = a.q_heads / c.heads, rows = group < NQ * 16 ? group : NQ * 16;
    const int64_t units = (int64_t)a.b * c.heads;
    const bool by_unit = units <= p.groups;
    const dim3 joins((unsigned)((by_unit ? (int)units : p.groups) * p.qtiles), (unsigned)rows);
    // few units are cut into many parts: more threads to read them (256 parts
    // of 64 heads: 9.6 us, 14.7 with 256; 2,048 workgroups: 7.9 us, 5.9 with 256)
    if (joins.x * joins.y <= 512) k_attend_join<DT, DP, 512><<<joins, dim3(512), 0, s>>>(c, a, p, rows, by_unit);
    else k_attend_join<DT, DP, 256><<<joins, dim3(256), 0, s>>>(c, a, p, rows, by_unit);
    return hipGetLastError();
}

template <int DT, int CDT, int DP>
hipError_t launch_d(const apc_kv& c, const AttendArgs& a, const AttendPlan& p, hipStream_t s)
{
    if constexpr (DP <= 128) {
        if (p.nq == 2) return p.once ? launch_q<DT, CDT, DP, 2, true>(c, a, p, s) : launch_q<DT, CDT, DP, 2, false>(c, a, p, s);
    }
    return p.once ? launch_q<DT, CDT, DP, 1, true>(c, a, p, s) : launch_q<DT, CDT, DP, 1, false>(c, a, p, s);
}

template <int DT, int CDT>
hipError_t launch(const apc_kv& c, const AttendArgs& a, const AttendPlan& p, hipStream_t s)
{
    switch (padded(c.d)) {
    case 64: return launch_d<DT, CDT, 64>(c, a, p, s);
    case 128: return launch_d<DT, CDT, 128>(c, a, p, s);
    default: return launch_d<DT, CDT, 256>(c, a, p, s);
    }
}

}  // namespace

size_t attend_workspace(const apc_kv& c, int32_t b, int32_t q_heads, int32_t max_pages)
{
    // what the call would ask if its units were cut, where the units of a smaller
    // batch over the same table, or with a window, could be
    AttendPlan p = plan(c, b, q_heads, max_pages, 0);
    const int64_t tiles = tiles_of(c, max_pages);
    if (bytes_of(c, tiles) <= WHOLE_UNIT) return 0;
    p.groups = cut_groups(c, (int64_t)b * c.heads, tiles, p.qtiles);
    const int group = q_heads / c.heads, rows = group < p.nq * 16 ? group : p.nq * 16;
    return (size_t)(rec_ints(p) + (int64_t)p.groups * p.qtiles * 2 * rows * (padded(c.d) + 2)) * sizeof(float);
}

hipError_t launch_attend(int dt, const apc_kv& c, const AttendArgs& args, hipStream_t s)
{
    if (args.b <= 0) return hipSuccess;
    AttendArgs a = args;
    if (c.n_pages == 0) a.max_pages = 0;                        // no page to read from
    const AttendPlan p = plan(c, a.b, a.q_heads, a.max_pages, a.window);
    if (c.dt == APC_E4M3) return dt == APC_F16 ? launch<APC_F16, APC_E4M3>(c, a, p, s) : launch<APC_BF16, APC_E4M3>(c, a, p, s);
    return dt == APC_F16 ? launch<APC_F16, APC_F16>(c, a, p, s) : launch<APC_BF16, APC_BF16>(c, a, p, s);
}

}  // namespace apc
