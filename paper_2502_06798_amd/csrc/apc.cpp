// C ABI of the matching library: argument checks, handle lifetime,
// workspace sizing and kernel launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdarg>
#include <climits>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <new>
#include <string>

#include "apc_internal.h"
#include "route_plan.h"

struct apc_cache {
    apc_dtype dt;
    int64_t n;
    int32_t d;
    const void* emb;
    const float* row_scale;
    const void* latents;
    int64_t n_slots;
    int64_t latent_bytes;
    const int32_t* slot_of_entry;
    float* fe;          // owned: row factors and group bounds (layout in apc_internal.h)
    int device;
};

// Workspace of apc_match_batch_static: one copy per device, held until the
// process ends.  In host code `scratch` only names the symbol; its device
// address (per device) comes from hipGetSymbolAddress.
static __device__ __align__(256) uint8_t scratch[APC_STATIC_WS_BYTES];

namespace {

constexpr int MAX_DEVICES = 64;
std::atomic<void*> g_scratch_ptr[MAX_DEVICES];   // device address of `scratch` per device (null: not looked up yet)

thread_local std::string g_err;
thread_local hipEvent_t g_ev_start = nullptr, g_ev_stop = nullptr;

apc_status fail(apc_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
apc_status fail(apc_status s, const char* fmt, ...)
{
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    g_err = buf;
    return s;
}

apc_status ok()
{
    g_err.clear();
    return APC_OK;
}

apc_status hip_fail(hipError_t e, const char* what)
{
    return fail(APC_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool valid_dtype(int dt) { return dt >= APC_F32 && dt <= APC_E4M3; }

apc_status check_rows(apc_dtype dt, int64_t n, int32_t d, const void* rows, const char* what)
{
    if (!valid_dtype(dt)) return fail(APC_E_DTYPE, "unknown dtype %d", (int)dt);
    if (n < 0 || d < 1) return fail(APC_E_ARG, "%s: need n >= 0 and d >= 1 (n=%lld d=%d)", what, (long long)n, d);
    if (((int64_t)d * apc::elem_bytes(dt)) % 16 != 0)
        return fail(APC_E_ARG, "%s: row of %d elements is not a multiple of 16 bytes", what, d);
    if (n > 0 && (!rows || !aligned16(rows)))
        return fail(APC_E_ARG, "%s: rows must be a non-NULL 16-byte aligned device pointer", what);
    return APC_OK;
}

// Calls that take a handle run on the handle's device: its row factors and
// the caller's borrowed buffers live there.
apc_status check_device(const char* who, const apc_cache* c)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(APC_E_HIP, "%s: hipGetDevice: %s", who, hipGetErrorString(e));
    if (dev != c->device)
        return fail(APC_E_ARG, "%s: the cache was built on device %d but device %d is current", who, c->device, dev);
    return APC_OK;
}

bool aligned_to(const void* p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }

bool float_dtype(int dt) { return dt == APC_F32 || dt == APC_F16 || dt == APC_BF16; }

// The description of a key-value cache.
apc_status check_kv(const char* who, const apc_kv* c)
{
    if (!c) return fail(APC_E_ARG, "%s: NULL cache", who);
    if (c->dt != APC_F16 && c->dt != APC_BF16 && c->dt != APC_E4M3)
        return fail(APC_E_DTYPE, "%s: a key-value cache is f16, bf16 or e4m3 (got %d)", who, (int)c->dt);
    // (the kernels count a token's rows, two a head, in 32 bits)
    if (c->heads < 1 || c->heads > APC_MAX_ATTEND_ROWS || c->d < 16 || c->d > APC_MAX_HEAD_DIM || c->d % 16 != 0)
        return fail(APC_E_ARG, "%s: need 1 <= heads <= %d and d a multiple of 16 up to %d (heads=%d d=%d)", who,
                    APC_MAX_ATTEND_ROWS, APC_MAX_HEAD_DIM, c->heads, c->d);
    if (c->page < 16 || c->page > APC_MAX_PAGE || (c->page & (c->page - 1)) != 0)
        return fail(APC_E_ARG, "%s: page must be a power of two from 16 to %d (page=%d)", who, APC_MAX_PAGE, c->page);
    if (c->n_pages < 0 || c->n_pages > INT32_MAX / c->page)
        return fail(APC_E_ARG, "%s: need 0 <= n_pages * page < 2^31 (n_pages=%lld)", who, (long long)c->n_pages);
    if (c->n_pages > 0) {
        if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v))
            return fail(APC_E_ARG, "%s: k and v must be non-NULL 16-byte aligned device pointers", who);
        const bool scaled = c->dt == APC_E4M3;
        if (scaled != (c->k_scale != nullptr) || scaled != (c->v_scale != nullptr))
            return fail(APC_E_ARG, "%s: k_scale and v_scale are required for e4m3 and only for e4m3", who);
        if (scaled && (!aligned16(c->k_scale) || !aligned16(c->v_scale)))
            return fail(APC_E_ARG, "%s: k_scale and v_scale must be 16-byte aligned", who);
    }
    return APC_OK;
}

apc_status kv_rows(const char* who, bool write, const apc_kv* c, apc_dtype dt, int64_t t, const void* k, int64_t k_tok,
                   int64_t k_head, const void* v, int64_t v_tok, int64_t v_head, const int32_t* slots, void* stream)
{
    if (apc_status st = check_kv(who, c)) return st;
    if (!float_dtype(dt)) return fail(APC_E_DTYPE, "%s: rows are f32, f16 or bf16 (got %d)", who, (int)dt);
    // one workgroup holds at least four rows, and a grid has fewer than 2^31 workgroups
    if (t < 0 || t > (int64_t)INT32_MAX / c->heads)
        return fail(APC_E_ARG, "%s: need 0 <= t * heads < 2^31 (t=%lld)", who, (long long)t);
    if (k_tok < 0 || k_head < 0 || v_tok < 0 || v_head < 0) return fail(APC_E_ARG, "%s: negative stride", who);
    if (t == 0) return ok();
    const int e = apc::elem_bytes(dt);
    if (!k || !v || !slots || !aligned_to(k, e) || !aligned_to(v, e) || !aligned_to(slots, 4))
        return fail(APC_E_ARG, "%s: k, v and slots must be device pointers aligned to their elements", who);
    const apc::KvRows a{const_cast<void*>(k), const_cast<void*>(v), slots, t, k_tok, k_head, v_tok, v_head};
    hipError_t err = apc::launch_kv_rows(write, dt, *c, a, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return hip_fail(err, who);
    return ok();
}

}  // namespace

extern "C" {

const char* apc_status_str(apc_status s)
{
    switch (s) {
    case APC_OK: return "ok";
    case APC_E_ARG: return "invalid argument";
    case APC_E_DTYPE: return "unknown dtype";
    case APC_E_TABLE: return "invalid threshold or instance table";
    case APC_E_NONFINITE: return "non-finite value";
    case APC_E_ZERO_NORM: return "zero-norm row";
    case APC_E_WORKSPACE: return "workspace too small";
    case APC_E_NOMEM: return "out of memory";
    case APC_E_HIP: return "HIP error";
    default: break;
    }
    return "unknown status";
}

const char* apc_last_error(void) { return g_err.c_str(); }

apc_status apc_set_kernel_events(void* start, void* stop)
{
    if ((start == nullptr) != (stop == nullptr))
        return fail(APC_E_ARG, "apc_set_kernel_events: give both events or neither");
    g_ev_start = static_cast<hipEvent_t>(start);
    g_ev_stop = static_cast<hipEvent_t>(stop);
    return ok();
}

apc_status apc_row_factors(apc_dtype dt, int64_t n, int32_t d, const void* rows, float* out, void* stream)
{
    apc_status st = check_rows(dt, n, d, rows, "apc_row_factors");
    if (st != APC_OK) return st;
    if (n > 0 && !out) return fail(APC_E_ARG, "apc_row_factors: out is NULL");
    if (n == 0) return ok();
    hipError_t e = apc::launch_row_factors(dt, n, d, rows, nullptr, nullptr, 0, out, nullptr,
                                           static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "row factor launch");
    return ok();
}

apc_status apc_quantize_rows(apc_dtype dt, int64_t n, int32_t d, const float* x, void* out, float* row_scale,
                             void* stream)
{
    if (valid_dtype(dt) && dt == APC_F32)
        return fail(APC_E_DTYPE, "apc_quantize_rows: the target must be f16, bf16 or e4m3");
    apc_status st = check_rows(dt, n, d, out, "apc_quantize_rows");
    if (st != APC_OK) return st;
    if (n > 0 && (!x || !aligned16(x)))
        return fail(APC_E_ARG, "apc_quantize_rows: x must be a non-NULL 16-byte aligned device pointer");
    if (n > 0 && (dt == APC_E4M3) != (row_scale != nullptr))
        return fail(APC_E_ARG, "apc_quantize_rows: row_scale is required for e4m3 and only for e4m3");
    if (n == 0) return ok();
    hipError_t e = apc::launch_quantize_rows(dt, n, d, x, out, row_scale, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    return ok();
}

apc_status apc_validate_rows(apc_dtype dt, int64_t n, int32_t d, const void* rows, const float* row_scale,
                             uint8_t* bad, int64_t* n_bad, int64_t* first_bad, void* stream)
{
    if (!n_bad) return fail(APC_E_ARG, "apc_validate_rows: n_bad is NULL");
    *n_bad = 0;
    if (first_bad) *first_bad = -1;
    apc_status st = check_rows(dt, n, d, rows, "apc_validate_rows");
    if (st != APC_OK) return st;
    if (n > 0 && (dt == APC_E4M3) != (row_scale != nullptr))
        return fail(APC_E_ARG, "apc_validate_rows: row_scale is required for e4m3 and only for e4m3");
    if (n == 0) return ok();
    hipStream_t s = static_cast<hipStream_t>(stream);
    apc::BuildStatus* dst = nullptr;
    apc::BuildStatus hst{};
    hst.first_bad = ~0ull;
    hipError_t e = hipMalloc(&dst, sizeof(apc::BuildStatus));
    if (e != hipSuccess) return fail(APC_E_NOMEM, "apc_validate_rows: hipMalloc: %s", hipGetErrorString(e));
    if ((e = hipMemcpyAsync(dst, &hst, sizeof hst, hipMemcpyHostToDevice, s)) != hipSuccess ||
        (e = apc::launch_row_factors(dt, n, d, rows, row_scale, nullptr, 0, nullptr, dst, s, bad)) != hipSuccess ||
        (e = hipMemcpyAsync(&hst, dst, sizeof hst, hipMemcpyDeviceToHost, s)) != hipSuccess ||
        (e = hipStreamSynchronize(s)) != hipSuccess) {
        (void)hipFree(dst);
        return hip_fail(e, "apc_validate_rows");
    }
    (void)hipFree(dst);
    *n_bad = (int64_t)hst.n_bad;
    if (first_bad) *first_bad = hst.n_bad ? (int64_t)hst.first_bad : -1;
    return ok();
}

apc_status apc_build_cache(apc_dtype dt, int64_t n, int32_t d, const void* emb, const float* row_scale,
                           const void* latents, int64_t n_slots, int64_t latent_bytes,
                           const int32_t* slot_of_entry, void* stream, apc_cache** out)
{
    if (!out) return fail(APC_E_ARG, "apc_build_cache: out is NULL");
    *out = nullptr;
    apc_status st = check_rows(dt, n, d, emb, "apc_build_cache");
    if (st != APC_OK) return st;
    if (n < 1 || n >= INT32_MAX)
        return fail(APC_E_ARG, "apc_build_cache: need 1 <= n < 2^31 - 1 entries (n=%lld)", (long long)n);
    if ((dt == APC_E4M3) != (row_scale != nullptr))
        return fail(APC_E_ARG, "apc_build_cache: row_scale is required for e4m3 and only for e4m3");
    if (n_slots < 0 || latent_bytes < 0)
        return fail(APC_E_ARG, "apc_build_cache: negative n_slots or latent_bytes");
    if (n_slots > 0) {
        if (!latents || !aligned16(latents))
            return fail(APC_E_ARG, "apc_build_cache: latents must be a 16-byte aligned device pointer");
        if (latent_bytes <= 0 || latent_bytes % 16 != 0)
            return fail(APC_E_ARG, "apc_build_cache: latent_bytes must be a positive multiple of 16");
        if (!slot_of_entry && n_slots < n)
            return fail(APC_E_ARG, "apc_build_cache: identity slot map needs n_slots >= n");
    } else if (latents || slot_of_entry) {
        return fail(APC_E_ARG, "apc_build_cache: latents/slot_of_entry given with n_slots = 0");
    }

    hipStream_t s = static_cast<hipStream_t>(stream);
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");

    apc_cache* c = new (std::nothrow) apc_cache{};
    if (!c) return fail(APC_E_NOMEM, "apc_build_cache: host allocation failed");
    const int64_t n_pad = apc::factor_pad(n);
    apc::BuildStatus* dst = nullptr;
    apc::BuildStatus hst{};
    if ((e = hipMalloc(&c->fe, sizeof(float) * n_pad)) != hipSuccess) {
        delete c;
        return fail(APC_E_NOMEM, "apc_build_cache: hipMalloc of %lld row factors: %s", (long long)n,
                    hipGetErrorString(e));
    }
    auto cleanup = [&]() {
        if (dst) (void)hipFree(dst);
        (void)hipFree(c->fe);
        delete c;
    };
    if ((e = hipMalloc(&dst, sizeof(apc::BuildStatus))) != hipSuccess) {
        cleanup();
        return fail(APC_E_NOMEM, "apc_build_cache: hipMalloc: %s", hipGetErrorString(e));
    }
    hst.first_bad = ~0ull;
    if ((e = hipMemsetAsync(c->fe + n, 0, sizeof(float) * (n_pad - n), s)) != hipSuccess ||
        (e = hipMemcpyAsync(dst, &hst, sizeof hst, hipMemcpyHostToDevice, s)) != hipSuccess ||
        (e = apc::launch_row_factors(dt, n, d, emb, row_scale, slot_of_entry, n_slots, c->fe, dst, s)) != hipSuccess ||
        (e = hipMemcpyAsync(&hst, dst, sizeof hst, hipMemcpyDeviceToHost, s)) != hipSuccess ||
        (e = hipStreamSynchronize(s)) != hipSuccess) {
        cleanup();
        return hip_fail(e, "apc_build_cache");
    }
    if (hst.flags) {
        const unsigned long long r = hst.first_bad;
        cleanup();
        if (hst.flags & apc::ST_NONFINITE)
            return fail(APC_E_NONFINITE, "apc_build_cache: non-finite values (first bad row %llu)", r);
        if (hst.flags & apc::ST_SCALE)
            return fail(APC_E_NONFINITE, "apc_build_cache: row scale not finite and > 0 (first bad row %llu)", r);
        if (hst.flags & apc::ST_ZERO)
            return fail(APC_E_ZERO_NORM, "apc_build_cache: zero-norm row (first bad row %llu)", r);
        return fail(APC_E_ARG, "apc_build_cache: slot_of_entry out of range (first bad entry %llu)", r);
    }
    (void)hipFree(dst);
    c->dt = dt;
    c->n = n;
    c->d = d;
    c->emb = emb;
    c->row_scale = row_scale;
    c->latents = latents;
    c->n_slots = n_slots;
    c->latent_bytes = latent_bytes;
    c->slot_of_entry = slot_of_entry;
    c->device = dev;
    *out = c;
    return ok();
}

void apc_destroy_cache(apc_cache* c)
{
    if (!c) return;
    (void)hipFree(c->fe);
    delete c;
}

apc_status apc_cache_row_factors(const apc_cache* c, float* out, void* stream)
{
    if (!c || !out) return fail(APC_E_ARG, "apc_cache_row_factors: NULL argument");
    if (apc_status st = check_device("apc_cache_row_factors", c)) return st;
    hipError_t e = hipMemcpyAsync(out, c->fe, sizeof(float) * c->n, hipMemcpyDeviceToDevice,
                                  static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_cache_row_factors");
    return ok();
}

apc_status apc_match_workspace(const apc_cache* c, int32_t b, int32_t k, size_t* bytes)
{
    if (!c || !bytes) return fail(APC_E_ARG, "apc_match_workspace: NULL argument");
    if (b < 0) return fail(APC_E_ARG, "apc_match_workspace: b < 0");
    if (k < 1 || k > APC_MAX_K || k > c->n)
        return fail(APC_E_ARG, "apc_match_workspace: need 1 <= k <= min(n, %d) (k=%d)", APC_MAX_K, k);
    *bytes = b == 0 ? 0 : apc::match_workspace(c->dt, c->n, c->d, b, k);
    return ok();
}

apc_status apc_match_batch(const apc_cache* c, const void* q, const float* q_scale, int32_t b, int32_t k,
                           float* top_score, int32_t* top_idx, void* ws, size_t ws_bytes, void* stream)
{
    if (!c) return fail(APC_E_ARG, "apc_match_batch: NULL cache");
    if (b < 0) return fail(APC_E_ARG, "apc_match_batch: b < 0");
    if (k < 1 || k > APC_MAX_K || k > c->n)
        return fail(APC_E_ARG, "apc_match_batch: need 1 <= k <= min(n, %d) (k=%d)", APC_MAX_K, k);
    if (b == 0) return ok();
    apc_status st = check_rows(c->dt, b, c->d, q, "apc_match_batch queries");
    if (st != APC_OK) return st;
    if ((st = check_device("apc_match_batch", c)) != APC_OK) return st;
    if ((c->dt == APC_E4M3) != (q_scale != nullptr))
        return fail(APC_E_ARG, "apc_match_batch: q_scale is required for e4m3 and only for e4m3");
    if (!top_score || !top_idx || !aligned16(top_score) || !aligned16(top_idx))
        return fail(APC_E_ARG, "apc_match_batch: outputs must be 16-byte aligned device pointers");
    const apc::MatchPlan p = apc::plan_match(c->dt, c->n, c->d, b, k);
    const size_t need = apc::match_workspace(c->dt, c->n, c->d, b, k);
    if (!ws || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u))
        return fail(APC_E_WORKSPACE, "apc_match_batch: workspace needs %zu bytes, 256-byte aligned (got %zu)",
                    need, ws_bytes);
    hipEvent_t ev0 = g_ev_start, ev1 = g_ev_stop;
    g_ev_start = g_ev_stop = nullptr;
    hipError_t e = apc::launch_match(p, c->dt, c->n, c->d, c->emb, c->fe, q, q_scale, b, k, top_score,
                                     top_idx, ws, static_cast<hipStream_t>(stream), ev0, ev1);
    if (e != hipSuccess) return hip_fail(e, "apc_match_batch launch");
    return ok();
}

apc_status apc_match_batch_static(const apc_cache* c, const void* q, const float* q_scale, int32_t b, int32_t k,
                                  float* top_score, int32_t* top_idx, void* stream)
{
    if (!c) return fail(APC_E_ARG, "apc_match_batch_static: NULL cache");
    if (b < 0) return fail(APC_E_ARG, "apc_match_batch_static: b < 0");
    if (k < 1 || k > APC_MAX_K || k > c->n)
        return fail(APC_E_ARG, "apc_match_batch_static: need 1 <= k <= min(n, %d) (k=%d)", APC_MAX_K, k);
    if (b == 0) return ok();
    apc_status st = check_rows(c->dt, b, c->d, q, "apc_match_batch_static queries");
    if (st != APC_OK) return st;
    if ((st = check_device("apc_match_batch_static", c)) != APC_OK) return st;
    if ((c->dt == APC_E4M3) != (q_scale != nullptr))
        return fail(APC_E_ARG, "apc_match_batch_static: q_scale is required for e4m3 and only for e4m3");
    if (!top_score || !top_idx || !aligned16(top_score) || !aligned16(top_idx))
        return fail(APC_E_ARG, "apc_match_batch_static: outputs must be 16-byte aligned device pointers");
    const apc::MatchPlan p = apc::plan_match(c->dt, c->n, c->d, b, k);
    if (p.bytes > (size_t)APC_STATIC_WS_BYTES)
        return fail(APC_E_WORKSPACE,
                    "apc_match_batch_static: b = %d, k = %d needs %zu workspace bytes, more than the %u of the "
                    "static workspace (use apc_match_batch with a workspace of apc_match_workspace() bytes)",
                    b, k, p.bytes, (unsigned)APC_STATIC_WS_BYTES);
    if (c->device < 0 || c->device >= MAX_DEVICES)
        return fail(APC_E_ARG, "apc_match_batch_static: device %d beyond the %d this library tracks", c->device,
                    MAX_DEVICES);
    void* ws = g_scratch_ptr[c->device].load(std::memory_order_acquire);
    if (!ws) {
        // first call on this device (the handle's device is current): the
        // device's own copy of the array
        hipError_t e = hipGetSymbolAddress(&ws, HIP_SYMBOL(scratch));
        if (e != hipSuccess || !ws) return hip_fail(e, "apc_match_batch_static: hipGetSymbolAddress");
        g_scratch_ptr[c->device].store(ws, std::memory_order_release);
    }
    hipEvent_t ev0 = g_ev_start, ev1 = g_ev_stop;
    g_ev_start = g_ev_stop = nullptr;
    hipError_t e = apc::launch_match(p, c->dt, c->n, c->d, c->emb, c->fe, q, q_scale, b, k, top_score, top_idx, ws,
                                     static_cast<hipStream_t>(stream), ev0, ev1);
    if (e != hipSuccess) return hip_fail(e, "apc_match_batch_static launch");
    return ok();
}

namespace {

// Checks the level and instance tables shared by the assignment entry points
// and builds the device table (levels, instances ordered by (level, queue
// desc, index asc), places per level).
// With inst_rand (uniform routing at batch size 1), instances are ordered by
// (level, inst_rand asc, index asc) and each takes at most one query.
apc_status build_assign_table(const char* who, const float* top_score, int32_t ld, int32_t b, int32_t L,
                              const float* theta, const int32_t* K, int32_t n_inst, const int32_t* inst_level,
                              const int32_t* inst_cap, const int32_t* inst_queue, const int32_t* opt_level,
                              const int32_t* out_level, const int32_t* out_inst, const int32_t* out_slot,
                              const int32_t* inst_fill, apc::AssignTable& t, const uint32_t* inst_rand = nullptr)
{
    if (b < 0 || ld < 1) return fail(APC_E_ARG, "%s: need b >= 0 and ld >= 1", who);
    if (L < 0 || L > APC_MAX_LEVELS) return fail(APC_E_TABLE, "%s: need 0 <= L <= %d", who, APC_MAX_LEVELS);
    if (L > 0 && (!theta || !K)) return fail(APC_E_TABLE, "%s: theta/K are NULL", who);
    for (int l = 0; l < L; ++l) {
        if (!std::isfinite(theta[l])) return fail(APC_E_TABLE, "%s: theta[%d] is not finite", who, l);
        if (K[l] <= 0) return fail(APC_E_TABLE, "%s: K[%d] must be > 0", who, l);
        if (l > 0 && !(theta[l] > theta[l - 1]))
            return fail(APC_E_TABLE, "%s: thresholds must be strictly increasing", who);
        if (l > 0 && !(K[l] > K[l - 1])) return fail(APC_E_TABLE, "%s: K must be strictly increasing", who);
    }
    if (n_inst < 0 || n_inst > APC_MAX_INST)
        return fail(APC_E_TABLE, "%s: need 0 <= n_inst <= %d", who, APC_MAX_INST);
    if (n_inst > 0 && (!inst_level || !inst_cap)) return fail(APC_E_TABLE, "%s: instance table is NULL", who);
    int64_t total = 0;
    for (int i = 0; i < n_inst; ++i) {
        if (inst_level[i] < 0 || inst_level[i] > L)
            return fail(APC_E_TABLE, "%s: inst_level[%d] = %d not in 0..%d", who, i, inst_level[i], L);
        if (inst_cap[i] < 0) return fail(APC_E_TABLE, "%s: inst_cap[%d] < 0", who, i);
        total += inst_cap[i];
    }
    if (total > INT32_MAX) return fail(APC_E_TABLE, "%s: total capacity exceeds 2^31 - 1", who);
    if (b > 0 && (!top_score || !opt_level || !out_level || !out_inst || !out_slot))
        return fail(APC_E_ARG, "%s: NULL device buffer", who);
    if (n_inst > 0 && !inst_fill) return fail(APC_E_ARG, "%s: inst_fill is NULL", who);

    t = apc::AssignTable{};
    t.L = L;
    t.n_inst = n_inst;
    for (int l = 0; l < L; ++l) {
        t.theta[l] = theta[l];
        t.K[l + 1] = K[l];
    }
    int order[APC_MAX_INST];
    for (int i = 0; i < n_inst; ++i) order[i] = i;
    std::stable_sort(order, order + n_inst, [&](int a, int c) {
        if (inst_level[a] != inst_level[c]) return inst_level[a] < inst_level[c];
        if (inst_rand) {
            if (inst_rand[a] != inst_rand[c]) return inst_rand[a] < inst_rand[c];
            return a < c;
        }
        const int qa = inst_queue ? inst_queue[a] : 0, qc = inst_queue ? inst_queue[c] : 0;
        if (qa != qc) return qa > qc;
        return a < c;
    });
    auto cap_of = [&](int i) { return inst_rand ? std::min(inst_cap[i], 1) : inst_cap[i]; };
    int j = 0;
    for (int p = 0; p <= L; ++p) {
        t.level_first[p] = j;
        int64_t cum = 0;
        while (j < n_inst && inst_level[order[j]] == p) {
            t.ord_inst[j] = (int16_t)order[j];
            t.ord_cap[j] = cap_of(order[j]);
            t.ord_cum[j] = (int32_t)cum;
            cum += cap_of(order[j]);
            ++j;
        }
        t.level_cap[p] = (int32_t)cum;
    }
    t.level_first[L + 1] = j;
    return APC_OK;
}

}  // namespace

apc_status apc_assign(const float* top_score, int32_t ld, int32_t b, int32_t L, const float* theta,
                      const int32_t* K, int32_t n_inst, const int32_t* inst_level, const int32_t* inst_cap,
                      const int32_t* inst_queue, int32_t* opt_level, int32_t* out_level, int32_t* out_inst,
                      int32_t* out_slot, int32_t* inst_fill, void* stream)
{
    apc::AssignTable t;
    apc_status st = build_assign_table("apc_assign", top_score, ld, b, L, theta, K, n_inst, inst_level, inst_cap,
                                       inst_queue, opt_level, out_level, out_inst, out_slot, inst_fill, t);
    if (st != APC_OK) return st;
    if (b == 0 && n_inst == 0) return ok();
    hipError_t e = apc::launch_assign(t, top_score, ld, b, opt_level, out_level, out_inst, out_slot,
                                      inst_fill, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_assign launch");
    return ok();
}

apc_status apc_assign_load_aware(const float* top_score, int32_t ld, int32_t b, int32_t L, const float* theta,
                                 const int32_t* K, int32_t n_inst, const int32_t* inst_level,
                                 const int32_t* inst_cap, const int32_t* inst_queue, const uint32_t* inst_rand,
                                 int64_t load, int64_t load_threshold, int32_t* routing, int32_t* opt_level,
                                 int32_t* out_level, int32_t* out_inst, int32_t* out_slot, int32_t* inst_fill,
                                 void* stream)
{
    if (!routing) return fail(APC_E_ARG, "apc_assign_load_aware: routing is NULL");
    const bool greedy = load >= load_threshold;
    if (!greedy && n_inst > 0 && !inst_rand)
        return fail(APC_E_ARG, "apc_assign_load_aware: uniform routing needs inst_rand");
    apc::AssignTable t;
    apc_status st = build_assign_table("apc_assign_load_aware", top_score, ld, b, L, theta, K, n_inst, inst_level,
                                       inst_cap, inst_queue, opt_level, out_level, out_inst, out_slot, inst_fill, t,
                                       greedy ? nullptr : inst_rand);
    if (st != APC_OK) return st;
    *routing = greedy ? 1 : 0;
    if (b == 0 && n_inst == 0) return ok();
    hipError_t e = apc::launch_assign(t, top_score, ld, b, opt_level, out_level, out_inst, out_slot, inst_fill,
                                      static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_assign_load_aware launch");
    return ok();
}

apc_status apc_route_plan(int32_t L, const int32_t* K, const int32_t* H, const int32_t* F, int32_t* X,
                          int64_t* degradation)
{
    if (L < 0 || L > APC_MAX_LEVELS) return fail(APC_E_TABLE, "apc_route_plan: need 0 <= L <= %d", APC_MAX_LEVELS);
    if ((L > 0 && !K) || !H || !F || !X) return fail(APC_E_ARG, "apc_route_plan: NULL argument");
    for (int l = 0; l < L; ++l) {
        if (K[l] <= 0) return fail(APC_E_TABLE, "apc_route_plan: K[%d] must be > 0", l);
        if (l > 0 && !(K[l] > K[l - 1])) return fail(APC_E_TABLE, "apc_route_plan: K must be strictly increasing");
    }
    int64_t sh = 0, sf = 0;
    for (int i = 0; i <= L; ++i) {
        if (H[i] < 0 || F[i] < 0) return fail(APC_E_ARG, "apc_route_plan: H[%d] or F[%d] < 0", i, i);
        sh += H[i];
        sf += F[i];
    }
    if (sh > INT32_MAX || sf > INT32_MAX) return fail(APC_E_ARG, "apc_route_plan: sums exceed 2^31 - 1");
    apc::plan_route_host(L, H, F, X);
    if (degradation) {
        int64_t d = 0;
        for (int i = 0; i <= L; ++i)
            for (int j = i + 1; j <= L; ++j)
                d += (int64_t)X[i * (L + 1) + j] * ((int64_t)K[j - 1] - (i > 0 ? K[i - 1] : 0));
        *degradation = d;
    }
    return ok();
}

static apc_status assign_with_plan(const char* who, bool planned, const float* top_score, int32_t ld, int32_t b,
                                   int32_t L, const float* theta, const int32_t* K, int32_t n_inst,
                                   const int32_t* inst_level, const int32_t* inst_cap, const int32_t* inst_queue,
                                   int32_t* plan, int32_t* opt_level, int32_t* out_level, int32_t* out_inst,
                                   int32_t* out_slot, int32_t* inst_fill, void* stream)
{
    apc::AssignTable t;
    apc_status st = build_assign_table(who, top_score, ld, b, L, theta, K, n_inst, inst_level, inst_cap,
                                       inst_queue, opt_level, out_level, out_inst, out_slot, inst_fill, t);
    if (st != APC_OK) return st;
    if (b > APC_MAX_ROUTED_BATCH) return fail(APC_E_ARG, "%s: b = %d exceeds %d", who, b, APC_MAX_ROUTED_BATCH);
    if (!plan) return fail(APC_E_ARG, "%s: plan is NULL", who);
    hipError_t e = apc::launch_assign_plan(t, planned, top_score, ld, b, plan, opt_level, out_level, out_inst,
                                           out_slot, inst_fill, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, who);
    return ok();
}

apc_status apc_assign_routed(const float* top_score, int32_t ld, int32_t b, int32_t L, const float* theta,
                             const int32_t* K, int32_t n_inst, const int32_t* inst_level, const int32_t* inst_cap,
                             const int32_t* inst_queue, const int32_t* plan, int32_t* opt_level,
                             int32_t* out_level, int32_t* out_inst, int32_t* out_slot, int32_t* inst_fill,
                             void* stream)
{
    return assign_with_plan("apc_assign_routed", false, top_score, ld, b, L, theta, K, n_inst, inst_level,
                            inst_cap, inst_queue, const_cast<int32_t*>(plan), opt_level, out_level, out_inst,
                            out_slot, inst_fill, stream);
}

apc_status apc_assign_planned(const float* top_score, int32_t ld, int32_t b, int32_t L, const float* theta,
                              const int32_t* K, int32_t n_inst, const int32_t* inst_level, const int32_t* inst_cap,
                              const int32_t* inst_queue, int32_t* plan, int32_t* opt_level, int32_t* out_level,
                              int32_t* out_inst, int32_t* out_slot, int32_t* inst_fill, void* stream)
{
    return assign_with_plan("apc_assign_planned", true, top_score, ld, b, L, theta, K, n_inst, inst_level,
                            inst_cap, inst_queue, plan, opt_level, out_level, out_inst, out_slot, inst_fill,
                            stream);
}

apc_status apc_resident_best(const apc_cache* c, const float* top_score, const int32_t* top_idx, int32_t ld,
                             int32_t k, int32_t b, float* out_score, int32_t* out_idx, void* stream)
{
    if (!c) return fail(APC_E_ARG, "apc_resident_best: NULL cache");
    if (c->n_slots == 0) return fail(APC_E_ARG, "apc_resident_best: the cache has no latents");
    if (b < 0 || k < 1 || k > APC_MAX_K || ld < k)
        return fail(APC_E_ARG, "apc_resident_best: need b >= 0 and 1 <= k <= min(ld, %d)", APC_MAX_K);
    if (b == 0) return ok();
    if (!top_score || !top_idx || !out_score || !out_idx)
        return fail(APC_E_ARG, "apc_resident_best: NULL device buffer");
    if (apc_status st = check_device("apc_resident_best", c)) return st;
    hipError_t e = apc::launch_resident_best(c->slot_of_entry, c->n, c->n_slots, top_score, top_idx, ld, k, b,
                                             out_score, out_idx, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_resident_best launch");
    return ok();
}

apc_status apc_level_histogram(const int32_t* level, int32_t b, int32_t L, int32_t* hist, void* stream)
{
    if (b < 0 || L < 0 || L > APC_MAX_LEVELS)
        return fail(APC_E_ARG, "apc_level_histogram: need b >= 0 and 0 <= L <= %d", APC_MAX_LEVELS);
    if ((b > 0 && !level) || !hist) return fail(APC_E_ARG, "apc_level_histogram: NULL device buffer");
    hipError_t e = apc::launch_level_histogram(level, b, L, hist, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_level_histogram launch");
    return ok();
}

apc_status apc_merge_shards(const float* scores, const int32_t* idx, int32_t g, int32_t b, int32_t k_in,
                            const int32_t* offsets, int32_t k, float* out_score, int32_t* out_idx, void* stream)
{
    if (g < 1 || g > APC_MAX_SHARDS || b < 0 || k < 1 || k > APC_MAX_K || k_in < 1 || k_in > APC_MAX_K)
        return fail(APC_E_ARG, "apc_merge_shards: need 1 <= g <= %d, b >= 0, 1 <= k, k_in <= %d", APC_MAX_SHARDS,
                    APC_MAX_K);
    if (!offsets) return fail(APC_E_ARG, "apc_merge_shards: offsets is NULL");
    apc::ShardOffsets off{};
    for (int s = 0; s < g; ++s) {
        if (offsets[s] < 0) return fail(APC_E_ARG, "apc_merge_shards: offsets[%d] < 0", s);
        off.v[s] = offsets[s];
    }
    if (b == 0) return ok();
    if (!scores || !idx || !out_score || !out_idx) return fail(APC_E_ARG, "apc_merge_shards: NULL device buffer");
    hipError_t e = apc::launch_merge_shards(scores, idx, g, b, k_in, off, k, out_score, out_idx,
                                            static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, "apc_merge_shards launch");
    return ok();
}

static apc_status gather_impl(const char* who, const apc_cache* c, const int32_t* top_idx, int32_t ld, int32_t b,
                              const int32_t* out_level, const int32_t* out_inst, const int32_t* out_slot,
                              int32_t n_inst, int32_t slots_per_inst, int32_t lps, void* batch_latents,
                              int32_t* hit, void* stream)
{
    if (!c) return fail(APC_E_ARG, "%s: NULL cache", who);
    if (c->n_slots == 0) return fail(APC_E_ARG, "%s: the cache has no latents", who);
    if (b < 0 || ld < 1 || n_inst < 0 || slots_per_inst < 0)
        return fail(APC_E_ARG, "%s: need b >= 0, ld >= 1, n_inst >= 0, slots_per_inst >= 0", who);
    if (lps < 1 || lps > APC_MAX_LEVELS || c->n_slots % lps != 0)
        return fail(APC_E_ARG, "%s: levels_per_slot must be in 1..%d and divide the cache's %lld latents", who,
                    APC_MAX_LEVELS, (long long)c->n_slots);
    if (b == 0) return ok();
    if (!top_idx || !out_level || !out_inst || !out_slot || !hit)
        return fail(APC_E_ARG, "%s: NULL device buffer", who);
    if ((int64_t)n_inst * slots_per_inst > 0 && (!batch_latents || !aligned16(batch_latents)))
        return fail(APC_E_ARG, "%s: batch_latents must be 16-byte aligned", who);
    if (apc_status st = check_device(who, c)) return st;
    hipError_t e = apc::launch_gather(c->latents, c->n, c->n_slots, c->latent_bytes, c->slot_of_entry,
                                      top_idx, ld, b, out_level, out_inst, out_slot, n_inst, slots_per_inst, lps,
                                      batch_latents, hit, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return hip_fail(e, who);
    return ok();
}

apc_status apc_gather_latents(const apc_cache* c, const int32_t* top_idx, int32_t ld, int32_t b,
                              const int32_t* out_level, const int32_t* out_inst, const int32_t* out_slot,
                              int32_t n_inst, int32_t slots_per_inst, void* batch_latents, int32_t* hit,
                              void* stream)
{
    return gather_impl("apc_gather_latents", c, top_idx, ld, b, out_level, out_inst, out_slot, n_inst,
                       slots_per_inst, 1, batch_latents, hit, stream);
}

apc_status apc_gather_latents_at_level(const apc_cache* c, const int32_t* top_idx, int32_t ld, int32_t b,
                                       const int32_t* out_level, const int32_t* out_inst, const int32_t* out_slot,
                                       int32_t n_inst, int32_t slots_per_inst, int32_t levels_per_slot,
                                       void* batch_latents, int32_t* hit, void* stream)
{
    return gather_impl("apc_gather_latents_at_level", c, top_idx, ld, b, out_level, out_inst, out_slot, n_inst,
                       slots_per_inst, levels_per_slot, batch_latents, hit, stream);
}

apc_status apc_norm_rows(apc_dtype dt, apc_dtype out_dt, int64_t n, int32_t d, const void* x, int64_t ld_x,
                         const void* res, int64_t ld_res, const void* weight, float eps, void* sum, int64_t ld_sum,
                         void* out, int64_t ld_out, float* out_scale, void* stream)
{
    if (!float_dtype(dt)) return fail(APC_E_DTYPE, "apc_norm_rows: rows are f32, f16 or bf16 (got %d)", (int)dt);
    if (out_dt != dt && out_dt != APC_E4M3)
        return fail(APC_E_DTYPE, "apc_norm_rows: the output is of the rows' type or e4m3 (got %d)", (int)out_dt);
    if (n < 0 || n > INT32_MAX || d < 1 || d > APC_MAX_NORM_D)
        return fail(APC_E_ARG, "apc_norm_rows: need 0 <= n < 2^31 and 1 <= d <= %d (n=%lld d=%d)", APC_MAX_NORM_D,
                    (long long)n, d);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(APC_E_ARG, "apc_norm_rows: eps must be finite and >= 0");
    if (n == 0) return ok();
    const int e = apc::elem_bytes(dt);
    if (!x || !out || !aligned_to(x, e) || !aligned_to(out, apc::elem_bytes(out_dt)) || !aligned_to(res, e) ||
        !aligned_to(weight, e) || !aligned_to(sum, e) || !aligned_to(out_scale, 4))
        return fail(APC_E_ARG, "apc_norm_rows: x and out are required, every pointer aligned to its elements");
    if (sum && !res) return fail(APC_E_ARG, "apc_norm_rows: sum is the sum with a residual: res is NULL");
    if (ld_x < d || ld_out < d || (res && ld_res < d) || (sum && ld_sum < d))
        return fail(APC_E_ARG, "apc_norm_rows: a row stride is smaller than d = %d", d);
    if ((out_dt == APC_E4M3) != (out_scale != nullptr))
        return fail(APC_E_ARG, "apc_norm_rows: out_scale is required for e4m3 and only for e4m3");
    const apc::NormArgs a{x, res, weight, sum, out, out_scale, n, ld_x, ld_res, ld_sum, ld_out, d, eps, 1.0f / (float)d, false};
    hipError_t err = apc::launch_norm_rows(dt, out_dt, a, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return hip_fail(err, "apc_norm_rows launch");
    return ok();
}

apc_status apc_kv_write(const apc_kv* c, apc_dtype dt, int64_t t, const void* k, int64_t k_tok, int64_t k_head,
                        const void* v, int64_t v_tok, int64_t v_head, const int32_t* slots, void* stream)
{
    return kv_rows("apc_kv_write", true, c, dt, t, k, k_tok, k_head, v, v_tok, v_head, slots, stream);
}

apc_status apc_kv_read(const apc_kv* c, apc_dtype dt, int64_t t, const int32_t* slots, void* k, int64_t k_tok,
                       int64_t k_head, void* v, int64_t v_tok, int64_t v_head, void* stream)
{
    return kv_rows("apc_kv_read", false, c, dt, t, k, k_tok, k_head, v, v_tok, v_head, slots, stream);
}

static apc_status check_attend(const char* who, const apc_kv* c, int32_t b, int32_t q_heads, int32_t max_pages)
{
    if (apc_status st = check_kv(who, c)) return st;
    // a workgroup per query head in the join, and fewer than 2^32 threads in a launch
    if (b < 0 || q_heads < 1 || q_heads % c->heads != 0 || (int64_t)b * q_heads > APC_MAX_ATTEND_ROWS)
        return fail(APC_E_ARG, "%s: need b >= 0, q_heads a multiple of the cache's %d heads and b * q_heads <= %d "
                    "(b=%d q_heads=%d)", who, c->heads, APC_MAX_ATTEND_ROWS, b, q_heads);
    if (max_pages < 0 || max_pages > APC_MAX_TOKENS / c->page)
        return fail(APC_E_ARG, "%s: need 0 <= max_pages * page <= %d (max_pages=%d)", who, APC_MAX_TOKENS, max_pages);
    // the kernel counts all sequences' tiles of 32 tokens, and a few more each, in 32 bits
    if ((int64_t)b * ((int64_t)max_pages * c->page + 256) > APC_MAX_TABLE_TOKENS)
        return fail(APC_E_ARG, "%s: b page tables of max_pages * page tokens hold more than 2^35", who);
    return APC_OK;
}

apc_status apc_attend_workspace(const apc_kv* c, int32_t b, int32_t q_heads, int32_t max_pages, size_t* bytes)
{
    if (!bytes) return fail(APC_E_ARG, "apc_attend_workspace: bytes is NULL");
    if (apc_status st = check_attend("apc_attend_workspace", c, b, q_heads, max_pages)) return st;
    *bytes = apc::attend_workspace(*c, b, q_heads, max_pages);
    return ok();
}

apc_status apc_attend(const apc_kv* c, apc_dtype dt, const void* q, int64_t q_row, int64_t q_head, int32_t b,
                      int32_t q_heads, const int32_t* pages, int32_t max_pages, int64_t ld_pages,
                      const int32_t* lengths, int32_t window, float scale, void* out, int64_t out_row,
                      int64_t out_head, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    if (apc_status st = check_attend("apc_attend", c, b, q_heads, max_pages)) return st;
    if ((dt != APC_F16 && dt != APC_BF16) || (c->dt != APC_E4M3 && dt != c->dt))
        return fail(APC_E_DTYPE, "apc_attend: queries are of the cache's type, or f16 or bf16 over e4m3 (got %d)",
                    (int)dt);
    if (window < 0) return fail(APC_E_ARG, "apc_attend: window < 0");
    if (!std::isfinite(scale)) return fail(APC_E_ARG, "apc_attend: scale is not finite");
    if (q_row < 0 || q_head < 0 || out_row < 0 || out_head < 0 || ld_pages < max_pages)
        return fail(APC_E_ARG, "apc_attend: negative stride, or ld_pages < max_pages");
    if (b == 0) return ok();
    if (!q || !out || !lengths || (max_pages > 0 && !pages) || !aligned_to(q, 2) || !aligned_to(out, 2) ||
        !aligned_to(pages, 4) || !aligned_to(lengths, 4) || !aligned_to(lse, 4))
        return fail(APC_E_ARG, "apc_attend: q, out, lengths and pages must be device pointers aligned to their elements");
    const size_t need = apc::attend_workspace(*c, b, q_heads, max_pages);
    if (need > 0 && (!ws || !aligned16(ws)))
        return fail(APC_E_ARG, "apc_attend: workspace must be a non-NULL 16-byte aligned device pointer");
    if (ws_bytes < need)
        return fail(APC_E_WORKSPACE, "apc_attend: workspace of %zu bytes, %zu needed", ws_bytes, need);
    const apc::AttendArgs a{q, out, pages, lengths, lse, ws, q_row, q_head, out_row, out_head, ld_pages,
                            b, q_heads, max_pages, window, scale};
    hipError_t err = apc::launch_attend(dt, *c, a, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return hip_fail(err, "apc_attend launch");
    return ok();
}

apc_status apc_rotary_freqs(int32_t rot, double base, double factor, double original, double low, double high,
                            double* freq)
{
    if (rot < 2 || rot > APC_MAX_HEAD_DIM || rot % 2 != 0)
        return fail(APC_E_ARG, "apc_rotary_freqs: rot must be even, from 2 to %d (rot=%d)", APC_MAX_HEAD_DIM, rot);
    auto good = [](double x) { return std::isfinite(x) && x > 0.0; };
    if (!good(base) || !good(factor) || !std::isfinite(original) || original < 0.0)
        return fail(APC_E_ARG, "apc_rotary_freqs: base and factor must be finite and > 0, original finite and >= 0");
    if (original > 0.0 && (!std::isfinite(low) || !std::isfinite(high) || !(high > low)))
        return fail(APC_E_ARG, "apc_rotary_freqs: low and high must be finite and high > low");
    if (!freq) return fail(APC_E_ARG, "apc_rotary_freqs: freq is NULL");
    const double two_pi = 6.283185307179586476925;
    for (int i = 0; i < rot / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot);
        double g = 0.0;
        if (original > 0.0) {
            g = (original * f / two_pi - low) / (high - low);
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        }
        freq[i] = g * f + (1.0 - g) * f / factor;
    }
    return ok();
}

apc_status apc_rotate(const apc_rotary* r, apc_dtype dt, int64_t t, int32_t heads, int32_t d, const void* x, int64_t x_tok,
                      int64_t x_head, const int32_t* positions, void* out, int64_t out_tok, int64_t out_head, void* stream)
{
    if (!r) return fail(APC_E_ARG, "apc_rotate: NULL description");
    if (!float_dtype(dt)) return fail(APC_E_DTYPE, "apc_rotate: rows are f32, f16 or bf16 (got %d)", (int)dt);
    if (d < 1 || d > APC_MAX_HEAD_DIM || r->rot < 2 || r->rot > d || r->rot % 2 != 0)
        return fail(APC_E_ARG, "apc_rotate: need d <= %d and an even rot from 2 to d (d=%d rot=%d)", APC_MAX_HEAD_DIM, d,
                    r->rot);
    if (r->interleaved != 0 && r->interleaved != 1) return fail(APC_E_ARG, "apc_rotate: interleaved must be 0 or 1");
    if (!std::isfinite(r->mag)) return fail(APC_E_ARG, "apc_rotate: mag is not finite");
    if (heads < 1 || t < 0 || t > (int64_t)INT32_MAX / heads)
        return fail(APC_E_ARG, "apc_rotate: need heads >= 1 and 0 <= t * heads < 2^31 (t=%lld heads=%d)", (long long)t, heads);
    if (x_tok < 0 || x_head < 0 || out_tok < 0 || out_head < 0) return fail(APC_E_ARG, "apc_rotate: negative stride");
    if (t == 0) return ok();
    const int e = apc::elem_bytes(dt);
    if (!x || !out || !positions || !r->freq || !aligned_to(x, e) || !aligned_to(out, e) || !aligned_to(positions, 4) ||
        !aligned_to(r->freq, 8))
        return fail(APC_E_ARG, "apc_rotate: x, out, positions and freq must be device pointers aligned to their elements");
    // rows of out that share elements would be written by several threads
    if ((heads > 1 && out_head < d) || (t > 1 && out_tok < d) || (heads > 1 && t > 1 && out_head == out_tok))
        return fail(APC_E_ARG, "apc_rotate: rows of out overlap");
    const apc::RotateArgs a{x, out, positions, r->freq, t, x_tok, x_head, out_tok, out_head, heads, d, r->rot, r->mag,
                            r->interleaved != 0, false, false};
    hipError_t err = apc::launch_rotate(dt, a, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return hip_fail(err, "apc_rotate launch");
    return ok();
}

static apc_status check_attend_prompt(const char* who, const apc_kv* c, int64_t t, int32_t b, int32_t q_heads,
                                      int32_t max_pages)
{
    if (apc_status st = check_kv(who, c)) return st;
    // (the kernel counts a sequence's rows in 32 bits, and a launch has fewer than 2^32 threads)
    if (b < 0 || q_heads < 1 || q_heads % c->heads != 0 || (int64_t)b * q_heads > APC_MAX_ATTEND_ROWS)
        return fail(APC_E_ARG, "%s: need b >= 0, q_heads a multiple of the cache's %d heads and b * q_heads <= %d "
                    "(b=%d q_heads=%d)", who, c->heads, APC_MAX_ATTEND_ROWS, b, q_heads);
    if (t < 0 || t > APC_MAX_TOKENS || t * q_heads > APC_MAX_PROMPT_ROWS)
        return fail(APC_E_ARG, "%s: need 0 <= t <= %d and t * q_heads <= %d (t=%lld q_heads=%d)", who, APC_MAX_TOKENS,
                    APC_MAX_PROMPT_ROWS, (long long)t, q_heads);
    if (max_pages < 0 || max_pages > APC_MAX_TOKENS / c->page)
        return fail(APC_E_ARG, "%s: need 0 <= max_pages * page <= %d (max_pages=%d)", who, APC_MAX_TOKENS, max_pages);
    return APC_OK;
}

apc_status apc_attend_prompt_workspace(const apc_kv* c, int64_t t, int32_t b, int32_t q_heads, int32_t max_pages,
                                       size_t* bytes)
{
    if (!bytes) return fail(APC_E_ARG, "apc_attend_prompt_workspace: bytes is NULL");
    if (apc_status st = check_attend_prompt("apc_attend_prompt_workspace", c, t, b, q_heads, max_pages)) return st;
    *bytes = apc::prompt_workspace(*c, t, b, q_heads, max_pages);
    return ok();
}

apc_status apc_attend_prompt(const apc_kv* c, apc_dtype dt, int64_t t, const void* q, int64_t q_row, int64_t q_head,
                             int32_t b, const int32_t* starts, int32_t q_heads, const int32_t* pages, int32_t max_pages,
                             int64_t ld_pages, const int32_t* lengths, const int32_t* prefix, const float* slopes,
                             int32_t window, float cap, float scale, void* out, int64_t out_row, int64_t out_head,
                             float* lse, void* ws, size_t ws_bytes, void* stream)
{
    if (apc_status st = check_attend_prompt("apc_attend_prompt", c, t, b, q_heads, max_pages)) return st;
    if ((dt != APC_F16 && dt != APC_BF16) || (c->dt != APC_E4M3 && dt != c->dt))
        return fail(APC_E_DTYPE, "apc_attend_prompt: queries are of the cache's type, or f16 or bf16 over e4m3 (got %d)",
                    (int)dt);
    if (window < 0) return fail(APC_E_ARG, "apc_attend_prompt: window < 0");
    if (!std::isfinite(scale)) return fail(APC_E_ARG, "apc_attend_prompt: scale is not finite");
    if (!(cap >= 0.f) || !std::isfinite(cap)) return fail(APC_E_ARG, "apc_attend_prompt: cap must be finite and >= 0");
    if (q_row < 0 || q_head < 0 || out_row < 0 || out_head < 0 || ld_pages < max_pages)
        return fail(APC_E_ARG, "apc_attend_prompt: negative stride, or ld_pages < max_pages");
    if (b == 0 || t == 0) return ok();
    if (!q || !out || !starts || !lengths || (max_pages > 0 && !pages) || !aligned_to(q, 2) || !aligned_to(out, 2) ||
        !aligned_to(starts, 4) || !aligned_to(pages, 4) || !aligned_to(lengths, 4) || !aligned_to(prefix, 4) ||
        !aligned_to(slopes, 4) || !aligned_to(lse, 4))
        return fail(APC_E_ARG, "apc_attend_prompt: q, out, starts, lengths and pages must be device pointers, all aligned to "
                    "their elements");
    const size_t need = apc::prompt_workspace(*c, t, b, q_heads, max_pages);
    if (need > 0 && (!ws || !aligned16(ws)))
        return fail(APC_E_ARG, "apc_attend_prompt: workspace must be a non-NULL 16-byte aligned device pointer");
    if (ws_bytes < need)
        return fail(APC_E_WORKSPACE, "apc_attend_prompt: workspace of %zu bytes, %zu needed", ws_bytes, need);
    // (positions are below 2^30, and no window beyond all of them differs from none)
    const int32_t within = window < APC_MAX_TOKENS ? window : 0;
    const apc::PromptArgs a{q, out, starts, pages, lengths, prefix, slopes, lse, ws, t, q_row, q_head, out_row, out_head,
                            ld_pages, b, q_heads, max_pages, within, scale, cap, nullptr};
    hipError_t err = apc::launch_attend_prompt(dt, *c, a, static_cast<hipStream_t>(stream));
    if (err != hipSuccess) return hip_fail(err, "apc_attend_prompt launch");
    return ok();
}

}  // extern "C"
