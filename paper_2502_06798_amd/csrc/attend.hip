// Attention of one new token per sequence over a paged key-value cache.
//
// A workgroup of four waves has one sequence, one key-value head, up to NQ x 16
// of the query heads that share it, and a range of the sequence's 32-token
// tiles; wave w takes every fourth tile.  Long sequences are cut into several
// ranges whose partial results k_attend_join joins.
//
// A tile, per wave, in matrix instructions of 16 x 16 x 32:
//   S^T = K Q^T    keys are the rows, query heads the columns: a lane holds one
//                  head's scores of 8 of the 32 keys.  The sum over d runs in
//                  an order that lets a lane load 16 consecutive elements.
//   P   = exp2(S - m), float32; m is the head's running maximum, raised (and
//                  the sums scaled) only where a score passes it by 2^8, so
//                  that a tile needs no exchange between lanes as a rule.
//   O^T += V^T P^T the lane's 8 weights are the second operand's 8 values as
//                  they stand, given that the first operand's lanes load the
//                  values of the same 8 keys; a lane owns DP / 16 consecutive
//                  elements of those keys' rows, and pairs of keys are put
//                  together in registers.  No value passes through LDS.
// The weights enter as the sum of two 16-bit numbers (rounded, and the rounded
// rest): one alone would lose 2^-9 (bf16) of every weight, two lose 2^-17, and
// the matrix cores have time to spare.  e4m3 keys and values are converted
// exactly to 16 bits; their scales join the scores and the weights in float32.
//
// Bound by memory: every key and value is read once, into the registers that
// the matrix instructions take, the next tile's while this one is computed.
#include "apc_internal.h"
#include "convert.h"

#include <cmath>

namespace apc {
namespace {

constexpr int WAVES = 4, TILE = 32;
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr float LOWEST = -3.0e38f;      // below every score; finite, so that exp2(-inf - m) is 0
constexpr float SLACK = 8.f;            // weights stay below 2^8

using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

// 16 x 16 x 32: D = A B + C; a lane's 8 values of A are row lane % 16, of B
// column lane % 16, both at k = 8 (lane / 16); of D column lane % 16, rows 4 (lane / 16) + r
template <bool BF> __device__ inline f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (BF)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

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

template <int DT, int CDT, int DP, int NQ>
__global__ __launch_bounds__(64 * WAVES, DP > 128 ? 1 : 2) void k_attend(apc_kv c, AttendArgs a, AttendPlan p)
{
    using T = typename Elem<DT>::T;
    constexpr bool E8 = CDT == APC_E4M3, QBF = DT == APC_BF16, PBF = E8 || QBF;
    constexpr int ES = E8 ? 1 : 2, EPL = DP / 16;               // values: elements of a row a lane owns
    constexpr int KW = 4 * ES, VW = EPL * ES / 4;               // dwords: 16 elements of a key, EPL of a value
    constexpr int SL = DP < 128 ? DP : 128;                     // elements of a round of the final sums
    __shared__ float part[WAVES][16][SL + 4];
    __shared__ float ml[WAVES][NQ * 16][2];

    const int lane = threadIdx.x & 63, col = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // query tiles of one range come to one XCD (workgroups go round over 8): they read the same keys
    const int id = blockIdx.x, qt = id / 8 % p.qtiles;
    const int64_t range = (int64_t)(id / 8 / p.qtiles) * 8 + id % 8;
    if (range >= (int64_t)a.b * c.heads * p.splits) return;
    const int unit = (int)(range % ((int64_t)a.b * c.heads)), split = (int)(range / ((int64_t)a.b * c.heads));
    const int seq = unit / c.heads, head = unit % c.heads, group = a.q_heads / c.heads;

    const int32_t held = a.lengths[seq], cap = a.max_pages << p.shift;
    const int len = held < 0 ? 0 : held < cap ? held : cap;
    const int first = a.window > 0 && len > a.window ? len - a.window : 0;
    const Ranges r(first, len, p);
    if (split > 0 && split >= r.used) return;                   // split 0 of an empty sequence writes its zeros
    const int begin = r.tile0 + split * r.per, last = r.tile0 + r.tiles;
    const int end = begin + r.per < last ? begin + r.per : last;

    // queries: column col of tile n is query head (qt NQ + n) 16 + col of the group
    u32x4 q[NQ][DP / 32];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        const int qh = (qt * NQ + n) * 16 + col;
        const T* row = static_cast<const T*>(a.q) + seq * a.q_row + (int64_t)(head * group + qh) * a.q_head;
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
            const int d = j / 2 * 64 + g * 16 + j % 2 * 8;
            q[n][j] = u32x4{0, 0, 0, 0};
            if (qh < group && d < c.d) __builtin_memcpy(&q[n][j], row + d, 16);
        }
    }

    f32x4 o[NQ][EPL];
    float m[NQ], l[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        m[n] = LOWEST;
        l[n] = 0.f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) o[n][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // a lane's places in a row; past a row's end (d < DP) it reads another
    // lane's elements: they meet zeros of q, or columns that are not stored
    const int row_bytes = c.d * ES;
    int koff[DP / 64];
#pragma unroll
    for (int j = 0; j < DP / 64; ++j) koff[j] = col * row_bytes + (j * 64 + g * 16 < c.d ? j * 64 + g * 16 : 0) * ES;
    const int voff = 4 * g * row_bytes + (col * EPL < c.d ? col * EPL : 0) * ES;
    const int32_t* table = a.pages + seq * a.ld_pages;
    const int last_page = len > 0 ? (len - 1) >> p.shift : 0, in_page = c.page - 1;

    int32_t pg[2];                                              // of the next tile's halves; -1: none
    uint32_t kr[2][DP / 64][KW], vr[8][VW];
    f32x4 ks[2], vs[2];
    auto find = [&](int t) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = (t * TILE + 16 * h) >> p.shift;
            pg[h] = table[at < last_page ? at : last_page];
        }
    };
    auto row_of = [&](int t, int h, int32_t pgh) {              // first row of a half tile (page 0 where there is none)
        const uint32_t page = (uint32_t)pgh < (uint64_t)c.n_pages ? (uint32_t)pgh : 0u;
        return (((int64_t)page * c.heads + head) << p.shift) + ((t * TILE + 16 * h) & in_page);
    };
    auto load_k = [&](int t, const int64_t* row) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* base = static_cast<const uint8_t*>(c.k) + row[h] * row_bytes;
#pragma unroll
            for (int j = 0; j < DP / 64; ++j) __builtin_memcpy(kr[h][j], __builtin_assume_aligned(base + koff[j], 16), 16 * ES);
            if constexpr (E8) ks[h] = *reinterpret_cast<const f32x4*>(c.k_scale + row[h] + 4 * g);
        }
    };
    auto load_v = [&](int t, const int64_t* row) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* base = static_cast<const uint8_t*>(c.v) + row[h] * row_bytes;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_memcpy(vr[4 * h + i], __builtin_assume_aligned(base + voff + i * row_bytes, EPL * ES < 16 ? EPL * ES : 16), EPL * ES);
            if constexpr (E8) vs[h] = *reinterpret_cast<const f32x4*>(c.v_scale + row[h] + 4 * g);
        }
    };

    const float to_log2 = a.scale * LOG2E;
    int t = begin + wave;
    int64_t row[2];
    int32_t pc[2];                                              // this tile's pages
    if (t < end) {
        find(t);
        pc[0] = pg[0], pc[1] = pg[1];
        row[0] = row_of(t, 0, pc[0]), row[1] = row_of(t, 1, pc[1]);
        load_k(t, row);
        load_v(t, row);
        if (t + WAVES < end) find(t + WAVES);
    }
    while (t < end) {
        const int next = t + WAVES;
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
                        const uint32_t lo = kr[h][j / 2][j % 2 * 2], hi = kr[h][j / 2][j % 2 * 2 + 1];
                        k = u32x4{from_e4m3<QBF, false>(lo), from_e4m3<QBF, true>(lo), from_e4m3<QBF, false>(hi),
                                  from_e4m3<QBF, true>(hi)};
                    } else {
                        __builtin_memcpy(&k, &kr[h][j / 2][j % 2 * 4], 16);
                    }
                    s[n][h] = mfma<QBF>(k, q[n][j], s[n][h]);
                }
            }
        f32x4 factor[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            factor[h] = f32x4{to_log2, to_log2, to_log2, to_log2};
            if constexpr (E8) factor[h] *= ks[h];
        }
        int64_t row_next[2] = {0, 0};
        int32_t pn[2] = {-1, -1};
        if (next < end) {
            pn[0] = pg[0], pn[1] = pg[1];
            row_next[0] = row_of(next, 0, pn[0]), row_next[1] = row_of(next, 1, pn[1]);
            load_k(next, row_next);
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) s[n][h] *= factor[h];

        // the first and last tiles, and those with pages that are not there: their unseen keys drop out
        const bool whole = t * TILE >= first && t * TILE + TILE <= len && (uint32_t)pc[0] < (uint64_t)c.n_pages &&
                           (uint32_t)pc[1] < (uint64_t)c.n_pages;
        if (!whole) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int tok = t * TILE + 16 * h + 4 * g + i;
                    const bool seen = tok >= first && tok < len && (uint32_t)pc[h] < (uint64_t)c.n_pages;
#pragma unroll
                    for (int n = 0; n < NQ; ++n) s[n][h][i] = seen ? s[n][h][i] : -INFINITY;
                    if constexpr (E8) vs[h][i] = seen ? vs[h][i] : 0.f;
#pragma unroll
                    for (int w = 0; w < VW; ++w) vr[4 * h + i][w] = seen ? vr[4 * h + i][w] : 0u;
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
            over |= top[n] > m[n] + SLACK;
        }
        if (__any(over)) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float x = __builtin_fmaxf(m[n], top[n]);
                x = __builtin_fmaxf(x, __shfl_xor(x, 16, 64));
                x = __builtin_fmaxf(x, __shfl_xor(x, 32, 64));
                const float f = __builtin_amdgcn_exp2f(m[n] - x);
                m[n] = x;
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
                if constexpr (E8) w[i] *= vs[i / 4][i % 4];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hi[n][i] = pack<PBF>(w[2 * i], w[2 * i + 1]);
                const f32x2 r = unpack<PBF>(hi[n][i]);
                lo[n][i] = pack<PBF>(w[2 * i] - r.x, w[2 * i + 1] - r.y);
            }
        }

        // values: element e of every key's row, keys in pairs
#pragma unroll
        for (int w = 0; w < VW; ++w) {
            constexpr int PER = 4 / ES;
            u32x4 v[PER];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = vr[2 * i][w], y = vr[2 * i + 1][w];
                if constexpr (E8) {
                    const uint32_t a01 = __builtin_amdgcn_perm(y, x, 0x05010400u), a23 = __builtin_amdgcn_perm(y, x, 0x07030602u);
                    v[0][i] = from_e4m3<PBF, false>(a01);
                    v[1][i] = from_e4m3<PBF, true>(a01);
                    v[2][i] = from_e4m3<PBF, false>(a23);
                    v[3][i] = from_e4m3<PBF, true>(a23);
                } else {
                    v[0][i] = __builtin_amdgcn_perm(y, x, 0x05040100u);
                    v[1][i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                }
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int e = 0; e < PER; ++e) {
                    o[n][w * PER + e] = mfma<PBF>(v[e], hi[n], o[n][w * PER + e]);
                    o[n][w * PER + e] = mfma<PBF>(v[e], lo[n], o[n][w * PER + e]);
                }
        }
        if (next < end) {
            load_v(next, row_next);
            if (next + WAVES < end) find(next + WAVES);
        }
        pc[0] = pn[0], pc[1] = pn[1];
        t = next;
    }

    // the waves' results into one: m and l first, then the outputs' sums, 128 elements of 16 heads a round
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
        if (g == 0) {
            ml[wave][n * 16 + col][0] = m[n];
            ml[wave][n * 16 + col][1] = l[n];
        }
    }
    const int hrow = threadIdx.x >> 4, dcol = (threadIdx.x & 15) * (SL / 16);
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
            const int qh = (qt * NQ + n) * 16 + hrow;
            if (qh < group && d0 + dcol < c.d) {
                float top = LOWEST, sum = 0.f, v[SL / 16] = {};
#pragma unroll
                for (int w = 0; w < WAVES; ++w) top = __builtin_fmaxf(top, ml[w][n * 16 + hrow][0]);
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float f = __builtin_amdgcn_exp2f(ml[w][n * 16 + hrow][0] - top);
                    sum = __builtin_fmaf(f, ml[w][n * 16 + hrow][1], sum);
#pragma unroll
                    for (int i = 0; i < SL / 16; ++i) v[i] = __builtin_fmaf(f, part[w][hrow][dcol + i], v[i]);
                }
                if (r.used <= 1) {
                    const int64_t qrow = (int64_t)head * group + qh;
                    const float f = sum == 0.f ? 0.f : 1.0f / sum;
#pragma unroll
                    for (int i = 0; i < SL / 16; ++i) v[i] = sum == 0.f ? 0.f : v[i] * f;
                    store_values<DT, SL / 16>(static_cast<T*>(a.out) + seq * a.out_row + qrow * a.out_head + d0 + dcol, v);
                    if (a.lse && d0 + dcol == 0)
                        a.lse[(int64_t)seq * a.q_heads + qrow] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
                } else {
                    const int64_t slot = ((int64_t)unit * p.splits + split) * group + qh;
                    float* po = static_cast<float*>(a.ws) + slot * DP + d0 + dcol;
#pragma unroll
                    for (int i = 0; i < SL / 16; i += 4) *reinterpret_cast<f32x4*>(po + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
                    if (d0 + dcol == 0) {
                        float* pm = static_cast<float*>(a.ws) + (int64_t)a.b * p.splits * a.q_heads * DP + slot * 2;
                        pm[0] = top;
                        pm[1] = sum;
                    }
                }
            }
        }
}

// Joins a sequence's ranges: one workgroup per query head, its threads over
// (part of the ranges) x (elements).
template <int DT, int DP>
__global__ __launch_bounds__(256) void k_attend_join(apc_kv c, AttendArgs a, AttendPlan p)
{
    using T = typename Elem<DT>::T;
    constexpr int LANES = DP / 4, PARTS = 256 / LANES;
    __shared__ float acc[PARTS][DP];
    __shared__ float sums[PARTS];
    const int seq = blockIdx.x / a.q_heads, qh = blockIdx.x % a.q_heads, group = a.q_heads / c.heads;
    const int head = qh / group;
    const int32_t held = a.lengths[seq], cap = a.max_pages << p.shift;
    const int len = held < 0 ? 0 : held < cap ? held : cap;
    const Ranges r(a.window > 0 && len > a.window ? len - a.window : 0, len, p);
    if (r.used <= 1) return;                                    // written by its only range
    const int64_t slot0 = ((int64_t)seq * c.heads + head) * p.splits * group + qh % group;
    const float* po = static_cast<const float*>(a.ws);
    const float* pm = po + (int64_t)a.b * p.splits * a.q_heads * DP;
    const int d = threadIdx.x % LANES * 4, part = threadIdx.x / LANES;
    float top = LOWEST;
    for (int i = threadIdx.x & 63; i < r.used; i += 64) top = __builtin_fmaxf(top, pm[(slot0 + (int64_t)i * group) * 2]);
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, m, 64));
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
    for (int i = part; i < r.used; i += PARTS) {
        const int64_t slot = slot0 + (int64_t)i * group;
        const float f = __builtin_amdgcn_exp2f(pm[slot * 2] - top);
        sum = __builtin_fmaf(f, pm[slot * 2 + 1], sum);
        v += f * *reinterpret_cast<const f32x4*>(po + slot * DP + d);
    }
    *reinterpret_cast<f32x4*>(&acc[part][d]) = v;
    if (threadIdx.x % LANES == 0) sums[part] = sum;
    __syncthreads();
    if (part > 0) return;
    sum = 0.f;
    v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PARTS; ++i) {
        sum += sums[i];
        v += *reinterpret_cast<const f32x4*>(&acc[i][d]);
    }
    const float f = sum == 0.f ? 0.f : 1.0f / sum;
    const float out[4] = {sum == 0.f ? 0.f : v.x * f, sum == 0.f ? 0.f : v.y * f, sum == 0.f ? 0.f : v.z * f,
                          sum == 0.f ? 0.f : v.w * f};
    if (d < c.d) store_values<DT, 4>(static_cast<T*>(a.out) + seq * a.out_row + qh * a.out_head + d, out);
    if (a.lse && d == 0) a.lse[(int64_t)seq * a.q_heads + qh] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
}

int padded(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
// query tiles of a wave: two share a key's registers, but wide heads have no registers for them
int query_tiles(int d, int group) { return group > 16 && padded(d) <= 128 ? 2 : 1; }

// Ranges per sequence: enough workgroups to fill the chip, none shorter than
// MIN_TILES where the table could hold the tiles; sequences are cut evenly by
// their own length in the kernel.
constexpr int MIN_TILES = 8;
constexpr int64_t TARGET = 2048;        // workgroups
AttendPlan plan(const apc_kv& c, int32_t b, int32_t q_heads, int32_t max_pages)
{
    AttendPlan p{};
    const int group = q_heads / c.heads;
    while ((1 << p.shift) < c.page) ++p.shift;
    p.nq = query_tiles(c.d, group);
    p.qtiles = (group + 16 * p.nq - 1) / (16 * p.nq);
    const int64_t units = (int64_t)b * c.heads * p.qtiles, tiles = (((int64_t)max_pages << p.shift) + TILE - 1) / TILE + 1;
    const int64_t most = (tiles + MIN_TILES - 1) / MIN_TILES, want = units > 0 ? (TARGET + units - 1) / units : 1;
    p.splits = (int32_t)(want < most ? want : most);
    p.min_tiles = MIN_TILES;
    return p;
}

template <int DT, int CDT, int DP>
hipError_t launch_d(const apc_kv& c, const AttendArgs& a, const AttendPlan& p, hipStream_t s)
{
    const int64_t ranges = ((int64_t)a.b * c.heads * p.splits + 7) / 8 * 8;
    const dim3 grid((unsigned)(ranges * p.qtiles)), block(64 * WAVES);
    if constexpr (DP <= 128) {
        if (p.nq == 2) k_attend<DT, CDT, DP, 2><<<grid, block, 0, s>>>(c, a, p);
    }
    if (p.nq == 1) k_attend<DT, CDT, DP, 1><<<grid, block, 0, s>>>(c, a, p);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits <= 1) return e;
    k_attend_join<DT, DP><<<dim3((unsigned)(a.b * a.q_heads)), dim3(256), 0, s>>>(c, a, p);
    return hipGetLastError();
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
    // the ranges' sums and statistics; the bound of all smaller batches and tables too
    const int group = q_heads / c.heads, nq = query_tiles(c.d, group), qtiles = (group + 16 * nq - 1) / (16 * nq);
    const int64_t rows = (int64_t)b * c.heads, tiles = ((int64_t)max_pages * c.page + TILE - 1) / TILE + 1;
    const int64_t most = (tiles + MIN_TILES - 1) / MIN_TILES;
    // splits > 1 only below TARGET units, and then units x splits < TARGET + units
    const int64_t limit = (TARGET + qtiles - 1) / qtiles, r = rows < limit ? rows : limit;
    const int64_t ranges = most <= 1 ? 0 : r * most < 2 * limit ? r * most : 2 * limit;
    return (size_t)ranges * group * (padded(c.d) + 2) * sizeof(float);
}

hipError_t launch_attend(int dt, const apc_kv& c, const AttendArgs& args, hipStream_t s)
{
    if (args.b <= 0) return hipSuccess;
    AttendArgs a = args;
    if (c.n_pages == 0) a.max_pages = 0;                        // no page to read from
    const AttendPlan p = plan(c, a.b, a.q_heads, a.max_pages);
    if (c.dt == APC_E4M3) return dt == APC_F16 ? launch<APC_F16, APC_E4M3>(c, a, p, s) : launch<APC_BF16, APC_E4M3>(c, a, p, s);
    return dt == APC_F16 ? launch<APC_F16, APC_F16>(c, a, p, s) : launch<APC_BF16, APC_BF16>(c, a, p, s);
}

}  // namespace apc
