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

#include <type_traits>

namespace apc {
namespace {

constexpr int64_t MAX_GRID = 1 << 20;
constexpr double TURNS = 0.15915494309189533577;                // 1 / (2 pi)

// x / y for x < 2^63, y > 0, in 32 bits where they suffice
__device__ inline int64_t quotient(int64_t x, int64_t y)
{
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// Pieces of V elements, 16 bytes or what divides the row's parts.  chunks: of V pairs in
// the turned part of a row, V / 2 where pairs are neighbours; copies: pieces of the
// rest, where that is to be copied; groups: threads that share a token's heads.
// Neighbouring threads' pieces are neighbours in every layout: with 32 bytes of
// neighbours' pairs a thread, lines reached memory in halves (65,536 x 40 heads of 128,
// bf16: 226 us, 597 so).
template <int DT, bool PAIRS, int V>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a, int chunks, int copies, int groups)
{
    using T = typename Elem<DT>::T;
    constexpr int P = PAIRS ? V / 2 : V;                        // pairs of a thread
    const int half = a.rot / 2, per_head = chunks + copies;
    const int64_t per_token = (int64_t)per_head * groups, total = a.t * per_token;
    for (int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x; id < total; id += (int64_t)gridDim.x * 256) {
        const int64_t token = quotient(id, per_token);
        const int64_t in = id - token * per_token, head0 = quotient(in, per_head);     // (heads may be 2^31 - 1)
        const int chunk = (int)(in - head0 * per_head);
        const int position = a.positions[token];
        if (position < 0) continue;
        const T* x = static_cast<const T*>(a.x) + token * a.x_tok;
        T* out = static_cast<T*>(a.out) + token * a.out_tok;
        if (chunk >= chunks) {
            const int d0 = a.rot + (chunk - chunks) * V, n = a.d - d0 < V ? a.d - d0 : V;
            for (int64_t h = head0; h < a.heads; h += groups) {
                const T* from = x + h * a.x_head + d0;
                T* to = out + h * a.out_head + d0;
                if (n == V) {
                    uint32_t w[(V * sizeof(T) + 3) / 4];
                    __builtin_memcpy(w, from, V * sizeof(T));
                    if constexpr (V * sizeof(T) >= 4) store_dwords<V * sizeof(T) / 4>(to, w, a.past);
                    else __builtin_memcpy(to, w, V * sizeof(T));
                } else {
                    for (int i = 0; i < n; ++i) to[i] = from[i];
                }
            }
            continue;
        }
        const int p0 = chunk * P;
        float c[P], s[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            const double turns = (double)position * (a.freq[p0 + i] * TURNS);
            const float f = (float)(turns - __builtin_rint(turns));
            sincospif(2.f * f, &s[i], &c[i]);
            s[i] *= a.mag, c[i] *= a.mag;
        }
        const int d0 = PAIRS ? 2 * p0 : p0, d1 = p0 + half;
        for (int64_t h = head0; h < a.heads; h += groups) {
            const T* from = x + h * a.x_head;
            T* to = out + h * a.out_head;
            if constexpr (PAIRS) {
                Raw<DT, V> r;
                float v[V];
                r.load(from + d0);
                r.values(v);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float y = v[2 * i], z = v[2 * i + 1];
                    v[2 * i] = __builtin_fmaf(y, c[i], -(z * s[i]));
                    v[2 * i + 1] = __builtin_fmaf(z, c[i], y * s[i]);
                }
                store_values<DT, V>(to + d0, v, a.past);
            } else {
                Raw<DT, V> r0, r1;
                float u[V], w[V];
                r0.load(from + d0);
                r1.load(from + d1);
                r0.values(u);
                r1.values(w);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float y = u[i], z = w[i];
                    u[i] = __builtin_fmaf(y, c[i], -(z * s[i]));
                    w[i] = __builtin_fmaf(z, c[i], y * s[i]);
                }
                store_values<DT, V>(to + d0, u, a.past);
                store_values<DT, V>(to + d1, w, a.past);
            }
        }
    }
}

// Outputs that the caches could not hold for whoever reads them go past them.
constexpr int64_t PAST_CACHES = 64 << 20;

template <int DT, int V> hipError_t launch(const RotateArgs& a, hipStream_t s)
{
    const int pairs = a.interleaved ? V / 2 : V, chunks = a.rot / 2 / pairs;
    const int copies = a.in_place ? 0 : (a.d - a.rot + V - 1) / V;
    // one head a thread until the chip is full, then up to four, which share the sines
    const int64_t threads = a.t * a.heads * (chunks + copies);
    const int heads_each = threads >= 4 << 19 ? 4 : threads >= 2 << 19 ? 2 : 1;
    const int groups = (int)(((int64_t)a.heads + heads_each - 1) / heads_each);
    const int64_t blocks = (a.t * groups * (chunks + copies) + 255) / 256;
    const dim3 grid((unsigned)(blocks < MAX_GRID ? blocks : MAX_GRID));
    if (!a.interleaved) k_rotate<DT, false, V><<<grid, dim3(256), 0, s>>>(a, chunks, copies, groups);
    else if constexpr (V > 1) k_rotate<DT, true, V><<<grid, dim3(256), 0, s>>>(a, chunks, copies, groups);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(int dt, const RotateArgs& args, hipStream_t s)
{
    if (args.t <= 0) return hipSuccess;
    RotateArgs a = args;
    a.in_place = a.x == a.out && a.x_tok == a.out_tok && a.x_head == a.out_head;
    const int e = elem_bytes(dt), part = a.interleaved ? a.rot : a.rot / 2, rest = a.in_place ? 0 : a.d - a.rot;
    // A piece never ends inside a part: threads of a wave that took an end element by element would have all of it wait
    // (6,739 x 61 heads of 128, 30 elements turned, float32: 113 us, 144 so).
    int v = 16 / e;
    while (v > (a.interleaved ? 2 : 1) && (part % v || rest % v)) v /= 2;
    a.past = a.t * a.heads * a.d * e >= PAST_CACHES && v * e == 16;
    auto go = [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if constexpr (DT != APC_F32)
            if (v == 8) return launch<DT, 8>(a, s);
        return v == 4 ? launch<DT, 4>(a, s) : v == 2 ? launch<DT, 2>(a, s) : launch<DT, 1>(a, s);
    };
    switch (dt) {
    case APC_F32: return go(std::integral_constant<int, APC_F32>{});
    case APC_F16: return go(std::integral_constant<int, APC_F16>{});
    case APC_BF16: return go(std::integral_constant<int, APC_BF16>{});
    default: return hipErrorInvalidValue;
    }
}

}  // namespace apc
