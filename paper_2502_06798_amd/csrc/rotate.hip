// Rotary positions: pairs of elements of heads' rows turned by an angle that
// grows with the token's position.
//
// The angle position x freq is taken in float64 and in turns, of which only the
// fraction matters: at position 2^31 that leaves 2^-21 of a turn, where float32
// would leave nothing.  Sine and cosine of the fraction, and the products with
// the elements, are float32.
//
// Bound by memory: every element is read and written once.  A thread has V pairs
// of one token, whose sines and cosines it computes once for all of the heads
// it takes.
#include "apc_internal.h"
#include "convert.h"

namespace apc {
namespace {

constexpr int64_t MAX_GRID = 1 << 20;
constexpr double TURNS = 0.15915494309189533577;                // 1 / (2 pi)

// x / y for x < 2^63, y > 0, in 32 bits where they suffice
__device__ inline int64_t quotient(int64_t x, int64_t y)
{
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

template <int DT> __device__ inline float one(const typename Elem<DT>::T* p)
{
    Raw<DT, 1> r;
    float v;
    r.load(p);
    r.values(&v);
    return v;
}

// chunks: of V pairs in the rotated part of a row; copies: of 2 V elements in
// the rest, where that is to be copied; groups: threads that share a token's heads
template <int DT, bool PAIRS, int V>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a, int chunks, int copies, int groups)
{
    using T = typename Elem<DT>::T;
    const int half = a.rot / 2, per_head = chunks + copies;
    const int64_t per_token = (int64_t)per_head * groups, total = a.t * per_token;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
        const int64_t token = quotient(id, per_token);
        const int in = (int)(id - token * per_token), chunk = in % per_head, head0 = in / per_head;
        const int position = a.positions[token];
        if (position < 0) continue;
        const T* x = static_cast<const T*>(a.x) + token * a.x_tok;
        T* out = static_cast<T*>(a.out) + token * a.out_tok;
        if (chunk >= chunks) {
            const int d0 = a.rot + (chunk - chunks) * 2 * V, n = a.d - d0 < 2 * V ? a.d - d0 : 2 * V;
            for (int h = head0; h < a.heads; h += groups) {
                const T* from = x + h * a.x_head + d0;
                T* to = out + h * a.out_head + d0;
                if (n == 2 * V) {
                    uint32_t w[V * sizeof(T) / 2];
                    __builtin_memcpy(w, from, 2 * V * sizeof(T));
                    store_dwords<4>(to, w, a.past);
                    store_dwords<4>(to + V, w + 4, a.past);
                } else {
                    for (int i = 0; i < n; ++i) to[i] = from[i];
                }
            }
            continue;
        }
        const int p0 = chunk * V, n = half - p0 < V ? half - p0 : V;
        const bool whole = n == V;
        float c[V], s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const double turns = (double)position * (a.freq[i < n ? p0 + i : p0] * TURNS);
            const float f = (float)(turns - __builtin_rint(turns));
            sincospif(2.f * f, &s[i], &c[i]);
            s[i] *= a.mag, c[i] *= a.mag;
        }
        const int d0 = PAIRS ? 2 * p0 : p0, d1 = PAIRS ? 2 * p0 + V : p0 + half;
        for (int h = head0; h < a.heads; h += groups) {
            const T* from = x + h * a.x_head;
            T* to = out + h * a.out_head;
            if (whole) {
                Raw<DT, V> r0, r1;
                float u[V], w[V];
                r0.load(from + d0);
                r1.load(from + d1);
                r0.values(u);
                r1.values(w);
                if constexpr (PAIRS) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float* e = i < V / 2 ? u + 2 * i : w + 2 * i - V;
                        const float y = e[0], z = e[1];
                        e[0] = __builtin_fmaf(y, c[i], -(z * s[i]));
                        e[1] = __builtin_fmaf(z, c[i], y * s[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float y = u[i], z = w[i];
                        u[i] = __builtin_fmaf(y, c[i], -(z * s[i]));
                        w[i] = __builtin_fmaf(z, c[i], y * s[i]);
                    }
                }
                store_values<DT, V>(to + d0, u, a.past);
                store_values<DT, V>(to + d1, w, a.past);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (i >= n) break;
                    const int e0 = PAIRS ? d0 + 2 * i : d0 + i, e1 = PAIRS ? e0 + 1 : d1 + i;
                    const float y = one<DT>(from + e0), z = one<DT>(from + e1);
                    const float u = __builtin_fmaf(y, c[i], -(z * s[i])), w = __builtin_fmaf(z, c[i], y * s[i]);
                    store_values<DT, 1>(to + e0, &u);
                    store_values<DT, 1>(to + e1, &w);
                }
            }
        }
    }
}

// Outputs that the caches could not hold for whoever reads them go past them.
constexpr int64_t PAST_CACHES = 64 << 20;

template <int DT, int V> hipError_t launch(const RotateArgs& a, hipStream_t s)
{
    const bool in_place = a.x == a.out && a.x_tok == a.out_tok && a.x_head == a.out_head;
    const int chunks = (a.rot / 2 + V - 1) / V, copies = in_place ? 0 : (a.d - a.rot + 2 * V - 1) / (2 * V);
    // one head a thread until the chip is full, then up to four, which share the sines
    const int64_t threads = a.t * a.heads * (chunks + copies);
    const int heads_each = threads >= 4 << 19 ? 4 : threads >= 2 << 19 ? 2 : 1;
    const int groups = (a.heads + heads_each - 1) / heads_each;
    const int64_t blocks = (a.t * groups * (chunks + copies) + 255) / 256;
    const dim3 grid((unsigned)(blocks < MAX_GRID ? blocks : MAX_GRID));
    if (a.interleaved) k_rotate<DT, true, V><<<grid, dim3(256), 0, s>>>(a, chunks, copies, groups);
    else k_rotate<DT, false, V><<<grid, dim3(256), 0, s>>>(a, chunks, copies, groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(int dt, const RotateArgs& args, hipStream_t s)
{
    if (args.t <= 0) return hipSuccess;
    RotateArgs a = args;
    a.past = a.t * a.heads * a.d * elem_bytes(dt) >= PAST_CACHES;
    switch (dt) {
    case APC_F32: return launch<APC_F32, 4>(a, s);
    case APC_F16: return launch<APC_F16, 8>(a, s);
    case APC_BF16: return launch<APC_BF16, 8>(a, s);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
