// C ABI: argument validation and dispatch.  Nothing here touches device data;
// every check is on the host-visible arguments, and a rejected call launches
// nothing.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <vector>
#include "launch.h"

namespace zipvl {

static thread_local char g_err[512] = "";

int set_error(int code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

int check_launch(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return set_error(ZIPVL_EHIP, "%s: launch failed: %s", what, hipGetErrorString(e));
    return ZIPVL_OK;
}

// ---- optional kernel timing -------------------------------------------------
namespace {
constexpr int kMaxTimed = 8192;
struct TimedLaunch { int id; hipEvent_t start, stop; };
std::mutex g_tmu;
bool g_timing = false;
std::vector<TimedLaunch> g_timed;
std::vector<hipEvent_t> g_pool;       // created once, reused
int g_pool_used = 0;
}  // namespace

KernelTimer::KernelTimer(int kernel_id, hipStream_t s) : slot(-1), st(s) {
    if (!g_timing) return;
    std::lock_guard<std::mutex> lk(g_tmu);
    if ((int)g_timed.size() >= kMaxTimed) return;
    while ((int)g_pool.size() < g_pool_used + 2) {
        hipEvent_t e;
        if (hipEventCreate(&e) != hipSuccess) return;
        g_pool.push_back(e);
    }
    TimedLaunch t{kernel_id, g_pool[g_pool_used], g_pool[g_pool_used + 1]};
    g_pool_used += 2;
    if (hipEventRecord(t.start, st) != hipSuccess) return;
    slot = (int)g_timed.size();
    g_timed.push_back(t);
}

KernelTimer::~KernelTimer() {
    if (slot < 0) return;
    std::lock_guard<std::mutex> lk(g_tmu);
    (void)hipEventRecord(g_timed[slot].stop, st);
}

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

static int check_dims(const char* fn, const zipvl_dims* d, bool need_q, bool need_k, bool need_v) {
    if (!d) return set_error(ZIPVL_EINVAL, "%s: dims is NULL", fn);
    if (d->dtype != ZIPVL_F32 && d->dtype != ZIPVL_BF16)
        return set_error(ZIPVL_EUNSUPPORTED, "%s: dtype %d (0 = fp32, 1 = bf16)", fn, d->dtype);
    if (d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->n < 1)
        return set_error(ZIPVL_EINVAL, "%s: B, Hq, Hkv, n must be positive (got %d %d %d %d)", fn, d->B, d->Hq, d->Hkv, d->n);
    if (d->Hq % d->Hkv != 0) return set_error(ZIPVL_ESHAPE, "%s: Hq=%d is not a multiple of Hkv=%d", fn, d->Hq, d->Hkv);
    if (d->d != 64 && d->d != 128) return set_error(ZIPVL_ESHAPE, "%s: head dim %d (supported: 64, 128)", fn, d->d);
    if ((int64_t)d->B * d->Hq > 65535) return set_error(ZIPVL_ESHAPE, "%s: B*Hq = %lld exceeds 65535", fn, (long long)d->B * d->Hq);
    if (d->n > (1 << 24)) return set_error(ZIPVL_ESHAPE, "%s: n = %d exceeds 2^24", fn, d->n);
    const int per16 = d->dtype == ZIPVL_BF16 ? 8 : 4;
    const int64_t* s[3] = {d->q_strides, d->k_strides, d->v_strides};
    const bool need[3] = {need_q, need_k, need_v};
    const char* nm[3] = {"q", "k", "v"};
    for (int t = 0; t < 3; ++t) {
        if (!need[t]) continue;
        for (int a = 0; a < 3; ++a) {
            if (s[t][a] < 0) return set_error(ZIPVL_EINVAL, "%s: %s_strides[%d] is negative", fn, nm[t], a);
            if (s[t][a] % per16) return set_error(ZIPVL_EALIGN, "%s: %s_strides[%d]=%lld is not a multiple of 16 bytes", fn, nm[t], a, (long long)s[t][a]);
        }
        if (s[t][2] < d->d) return set_error(ZIPVL_EINVAL, "%s: %s token stride %lld is smaller than d", fn, nm[t], (long long)s[t][2]);
    }
    return ZIPVL_OK;
}

#define ZIPVL_REQUIRE_PTR(fn, p)                                                         \
    do {                                                                                 \
        if (!(p)) return set_error(ZIPVL_EINVAL, "%s: %s is NULL", fn, #p);              \
        if (!aligned16(p)) return set_error(ZIPVL_EALIGN, "%s: %s is not 16-byte aligned", fn, #p); \
    } while (0)

}  // namespace zipvl

using namespace zipvl;

extern "C" {

int zipvl_version(void) { return 100; }

const char* zipvl_last_error(void) { return g_err; }

size_t zipvl_workspace_bytes(int op, const zipvl_dims* dims, int m) {
    if (check_dims("zipvl_workspace_bytes", dims, false, false, false)) return 0;
    switch (op) {
        case ZIPVL_OP_SCORE: return score_workspace_bytes(*dims, m);
        case ZIPVL_OP_SELECT: return select_workspace_bytes(dims->B * dims->Hkv);
        case ZIPVL_OP_SPARSE_PREFILL: return prefill_workspace_bytes(*dims);
        case ZIPVL_OP_DECODE: return decode_workspace_bytes(*dims, dims->n);
        case ZIPVL_OP_QUANTIZE_KV: return quantize_workspace_bytes(*dims);
        case ZIPVL_OP_DECODE_Q: return decode_workspace_bytes(*dims, dims->n);
        case ZIPVL_OP_SCORE_ALL_ROWS: return allrows_workspace_bytes(*dims);
        case ZIPVL_OP_DECODE_STEP: return decode_step_workspace_bytes(*dims, dims->n);
        case ZIPVL_OP_DECODE_PAGED:
            if (m < 0) { set_error(ZIPVL_EINVAL, "zipvl_workspace_bytes: m = %d is negative", m); return 0; }
            return decode_paged_workspace_bytes(*dims, dims->n, m);
        case ZIPVL_OP_CHUNK_PAGED:
        case ZIPVL_OP_PAGED_EVICT:
            if (m < 0) { set_error(ZIPVL_EINVAL, "zipvl_workspace_bytes: m = %d is negative", m); return 0; }
            return op == ZIPVL_OP_CHUNK_PAGED ? chunk_attn_workspace_bytes(*dims, m) : paged_evict_workspace_bytes((int64_t)dims->B * dims->Hkv, dims->n, m);
        default: set_error(ZIPVL_EUNSUPPORTED, "zipvl_workspace_bytes: unknown op %d", op); return 0;
    }
}

int zipvl_score(const void* Q, const void* K, const zipvl_dims* dims, const int32_t* probe_pos, int m,
                float softmax_scale, int flags, float* mass, float* rank, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_score";
    int rc = check_dims(fn, dims, true, true, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, Q);
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, mass);
    if (rank && !aligned16(rank)) return set_error(ZIPVL_EALIGN, "%s: rank is not 16-byte aligned", fn);
    if (!probe_pos) return set_error(ZIPVL_EINVAL, "%s: probe_pos is NULL", fn);
    if (m < 1) return set_error(ZIPVL_EINVAL, "%s: m = %d must be positive", fn, m);
    if (m > ZIPVL_MAX_PROBES) return set_error(ZIPVL_ESHAPE, "%s: m = %d exceeds %d probe rows", fn, m, ZIPVL_MAX_PROBES);
    for (int t = 0; t < m; ++t) {
        if (probe_pos[t] < 0 || probe_pos[t] >= dims->n)
            return set_error(ZIPVL_EINVAL, "%s: probe_pos[%d] = %d is outside [0, %d)", fn, t, probe_pos[t], dims->n);
        if (t && probe_pos[t] <= probe_pos[t - 1])
            return set_error(ZIPVL_EINVAL, "%s: probe_pos must be strictly ascending (entry %d)", fn, t);
    }
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    if (flags & ~ZIPVL_SCORE_PER_QHEAD) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    const size_t need = score_workspace_bytes(*dims, m);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_score(Q, K, *dims, probe_pos, m, softmax_scale, flags, mass, rank, ws, (hipStream_t)stream);
}

int zipvl_score_all_rows(const void* Q, const void* K, const zipvl_dims* dims, float softmax_scale,
                         float* mass, float* rank, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_score_all_rows";
    int rc = check_dims(fn, dims, true, true, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, Q);
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, mass);
    if (rank && !aligned16(rank)) return set_error(ZIPVL_EALIGN, "%s: rank is not 16-byte aligned", fn);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = allrows_workspace_bytes(*dims);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_score_all_rows(Q, K, *dims, softmax_scale, mass, rank, ws, (hipStream_t)stream);
}

int zipvl_select(const float* mass, const float* rank, int units, int n, double tau,
                 int32_t* idx, int32_t* k, int32_t* status, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_select";
    if (!mass || !idx || !k) return set_error(ZIPVL_EINVAL, "%s: mass, idx and k must not be NULL", fn);
    if (units < 1 || n < 1) return set_error(ZIPVL_EINVAL, "%s: units and n must be positive (got %d, %d)", fn, units, n);
    if (n >= (1 << 23)) return set_error(ZIPVL_ESHAPE, "%s: n = %d must be below 2^23", fn, n);
    if (!(tau > 0.0) || !(tau <= 1.0)) return set_error(ZIPVL_EINVAL, "%s: tau = %g is outside (0, 1]", fn, tau);
    if ((reinterpret_cast<uintptr_t>(mass) | reinterpret_cast<uintptr_t>(rank) |
         reinterpret_cast<uintptr_t>(idx) | reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(status)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: pointers must be 4-byte aligned", fn);
    if (ws && (reinterpret_cast<uintptr_t>(ws) & 15u)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    if (ws && ws_bytes < select_workspace_bytes(units))
        return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given (or pass NULL)", fn, select_workspace_bytes(units), ws_bytes);
    return launch_select(mass, rank, units, n, tau, idx, k, status, ws, ws_bytes, (hipStream_t)stream);
}

int zipvl_share_scores(const float* mass, const float* rank, int B, int Hkv, int n,
                       float* mass_b, float* rank_b, void* stream)
{
    const char* fn = "zipvl_share_scores";
    if (!mass || !mass_b) return set_error(ZIPVL_EINVAL, "%s: mass and mass_b must not be NULL", fn);
    if ((rank == nullptr) != (rank_b == nullptr)) return set_error(ZIPVL_EINVAL, "%s: rank and rank_b must both be given or both be NULL", fn);
    if (B < 1 || Hkv < 1 || n < 1) return set_error(ZIPVL_EINVAL, "%s: B, Hkv and n must be positive (got %d, %d, %d)", fn, B, Hkv, n);
    if ((reinterpret_cast<uintptr_t>(mass) | reinterpret_cast<uintptr_t>(rank) |
         reinterpret_cast<uintptr_t>(mass_b) | reinterpret_cast<uintptr_t>(rank_b)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: pointers must be 4-byte aligned", fn);
    return launch_share_scores(mass, rank, B, Hkv, n, mass_b, rank_b, (hipStream_t)stream);
}

int zipvl_sparse_prefill(const void* Q, const void* K, const void* V, const zipvl_dims* dims,
                         const int32_t* idx, const int32_t* k, float softmax_scale, int flags,
                         void* O, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_sparse_prefill";
    int rc = check_dims(fn, dims, true, true, true);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, Q);
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, V);
    ZIPVL_REQUIRE_PTR(fn, O);
    if ((idx == nullptr) != (k == nullptr)) return set_error(ZIPVL_EINVAL, "%s: idx and k must both be given or both be NULL", fn);
    if (flags & ~(ZIPVL_OUT_COMPACT | ZIPVL_KV_ALREADY_COMPACT | ZIPVL_T_PER_BATCH)) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = prefill_workspace_bytes(*dims);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return set_error(ZIPVL_EALIGN, "%s: ws is not 256-byte aligned", fn);
    return launch_sparse_prefill(Q, K, V, *dims, idx, k, softmax_scale, flags, O, ws, (hipStream_t)stream);
}

int zipvl_compact_kv(const void* K, const void* V, const zipvl_dims* dims, const int32_t* idx,
                     const int32_t* k, void* Kc, void* Vc, int32_t cap, int32_t* len, int flags, void* stream)
{
    const char* fn = "zipvl_compact_kv";
    int rc = check_dims(fn, dims, false, true, true);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, V);
    ZIPVL_REQUIRE_PTR(fn, Kc);
    ZIPVL_REQUIRE_PTR(fn, Vc);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if ((idx == nullptr) != (k == nullptr)) return set_error(ZIPVL_EINVAL, "%s: idx and k must both be given or both be NULL", fn);
    if (cap < 1) return set_error(ZIPVL_EINVAL, "%s: cap = %d must be positive", fn, cap);
    if (flags & ~ZIPVL_T_PER_BATCH) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    return launch_compact_kv(K, V, *dims, idx, k, Kc, Vc, cap, len, flags, (hipStream_t)stream);
}

int zipvl_kv_append(void* Kc, void* Vc, int32_t* len, int32_t cap, const void* k_new,
                    const void* v_new, const zipvl_dims* dims, void* stream)
{
    const char* fn = "zipvl_kv_append";
    int rc = check_dims(fn, dims, false, false, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, Kc);
    ZIPVL_REQUIRE_PTR(fn, Vc);
    ZIPVL_REQUIRE_PTR(fn, k_new);
    ZIPVL_REQUIRE_PTR(fn, v_new);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if (cap < 1) return set_error(ZIPVL_EINVAL, "%s: cap = %d must be positive", fn, cap);
    return launch_kv_append(Kc, Vc, len, cap, k_new, v_new, *dims, (hipStream_t)stream);
}

int zipvl_decode_attn(const void* q, const void* Kc, const void* Vc, const int32_t* len, int32_t cap,
                      const zipvl_dims* dims, float softmax_scale, void* o, void* ws, size_t ws_bytes,
                      void* stream)
{
    const char* fn = "zipvl_decode_attn";
    int rc = check_dims(fn, dims, false, false, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, q);
    ZIPVL_REQUIRE_PTR(fn, Kc);
    ZIPVL_REQUIRE_PTR(fn, Vc);
    ZIPVL_REQUIRE_PTR(fn, o);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if (cap < 1) return set_error(ZIPVL_EINVAL, "%s: cap = %d must be positive", fn, cap);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = decode_workspace_least(*dims, cap);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_decode_attn(q, Kc, Vc, len, cap, *dims, softmax_scale, o, ws, ws_bytes, (hipStream_t)stream);
}

int zipvl_decode_attn_static(const void* q, const void* Kc, const void* Vc, const int32_t* len, int32_t cap,
                             const zipvl_dims* dims, float softmax_scale, void* o, void* stream)
{
    const char* fn = "zipvl_decode_attn_static";
    int rc = check_dims(fn, dims, false, false, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, q);
    ZIPVL_REQUIRE_PTR(fn, Kc);
    ZIPVL_REQUIRE_PTR(fn, Vc);
    ZIPVL_REQUIRE_PTR(fn, o);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if (cap < 1) return set_error(ZIPVL_EINVAL, "%s: cap = %d must be positive", fn, cap);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    return launch_decode_attn_static(q, Kc, Vc, len, cap, *dims, softmax_scale, o, (hipStream_t)stream);
}

int zipvl_decode_step(const void* q, void* Kc, void* Vc, int32_t* len, int32_t cap, const void* k_new,
                      const void* v_new, const zipvl_dims* dims, float softmax_scale, void* o,
                      void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_decode_step";
    int rc = check_dims(fn, dims, false, false, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, q);
    ZIPVL_REQUIRE_PTR(fn, Kc);
    ZIPVL_REQUIRE_PTR(fn, Vc);
    ZIPVL_REQUIRE_PTR(fn, k_new);
    ZIPVL_REQUIRE_PTR(fn, v_new);
    ZIPVL_REQUIRE_PTR(fn, o);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if (cap < 1) return set_error(ZIPVL_EINVAL, "%s: cap = %d must be positive", fn, cap);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = decode_step_workspace_least(*dims, cap);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_decode_step(q, Kc, Vc, len, cap, k_new, v_new, *dims, softmax_scale, o, ws, ws_bytes, (hipStream_t)stream);
}

static int check_qtensor(const char* fn, const char* what, const zipvl_qtensor* t) {
    if (!t) return set_error(ZIPVL_EINVAL, "%s: %s is NULL", fn, what);
    const void* ptrs[4] = {t->hi_codes, t->hi_params, t->lo_codes, t->lo_params};
    for (const void* p : ptrs) {
        if (!p) return set_error(ZIPVL_EINVAL, "%s: an array of %s is NULL", fn, what);
        if (!aligned16(p)) return set_error(ZIPVL_EALIGN, "%s: an array of %s is not 16-byte aligned", fn, what);
    }
    return ZIPVL_OK;
}

int zipvl_quantize_kv(const void* K, const void* V, const zipvl_dims* dims, const int32_t* idx, const int32_t* k,
                      const zipvl_qtensor* Kq, const zipvl_qtensor* Vq, int32_t cap_hi, int32_t cap_lo,
                      int32_t* len_hi, int32_t* len_lo, int flags, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_quantize_kv";
    int rc = check_dims(fn, dims, false, true, true);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, V);
    if ((rc = check_qtensor(fn, "Kq", Kq)) || (rc = check_qtensor(fn, "Vq", Vq))) return rc;
    if (!len_hi || !len_lo) return set_error(ZIPVL_EINVAL, "%s: len_hi / len_lo is NULL", fn);
    if ((idx == nullptr) != (k == nullptr)) return set_error(ZIPVL_EINVAL, "%s: idx and k must both be given or both be NULL", fn);
    if (cap_hi < 1 || cap_lo < 1) return set_error(ZIPVL_EINVAL, "%s: cap_hi = %d and cap_lo = %d must be positive", fn, cap_hi, cap_lo);
    if (flags & ~ZIPVL_T_PER_BATCH) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    const size_t need = quantize_workspace_bytes(*dims);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (reinterpret_cast<uintptr_t>(ws) & 3u) return set_error(ZIPVL_EALIGN, "%s: ws is not 4-byte aligned", fn);
    return launch_quantize_kv(K, V, *dims, idx, k, *Kq, *Vq, cap_hi, cap_lo, len_hi, len_lo, flags, ws, (hipStream_t)stream);
}

int zipvl_decode_attn_q(const void* q, const zipvl_qtensor* Kq, const zipvl_qtensor* Vq,
                        const int32_t* len_hi, const int32_t* len_lo, int32_t cap_hi, int32_t cap_lo,
                        const void* K_tail, const void* V_tail, const int32_t* len_tail, int32_t cap_tail,
                        const zipvl_dims* dims, float softmax_scale, void* o, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_decode_attn_q";
    int rc = check_dims(fn, dims, false, false, false);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, q);
    ZIPVL_REQUIRE_PTR(fn, o);
    if ((rc = check_qtensor(fn, "Kq", Kq)) || (rc = check_qtensor(fn, "Vq", Vq))) return rc;
    if (!len_hi || !len_lo) return set_error(ZIPVL_EINVAL, "%s: len_hi / len_lo is NULL", fn);
    if (cap_hi < 1 || cap_lo < 1) return set_error(ZIPVL_EINVAL, "%s: cap_hi = %d and cap_lo = %d must be positive", fn, cap_hi, cap_lo);
    const bool tail = K_tail || V_tail || len_tail;
    if (tail) {
        if (!K_tail || !V_tail || !len_tail) return set_error(ZIPVL_EINVAL, "%s: K_tail, V_tail and len_tail must all be given or all be NULL", fn);
        if (!aligned16(K_tail) || !aligned16(V_tail)) return set_error(ZIPVL_EALIGN, "%s: K_tail / V_tail is not 16-byte aligned", fn);
        if (cap_tail < 1) return set_error(ZIPVL_EINVAL, "%s: cap_tail = %d must be positive", fn, cap_tail);
    } else {
        cap_tail = 0;
    }
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = decode_workspace_least(*dims, cap_hi + cap_lo + cap_tail);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_decode_attn_q(q, *Kq, *Vq, len_hi, len_lo, cap_hi, cap_lo, K_tail, V_tail, len_tail, cap_tail,
                                *dims, softmax_scale, o, ws, ws_bytes, (hipStream_t)stream);
}

static int check_rope(const char* fn, const zipvl_rope* r, int d) {
    if (!r) return set_error(ZIPVL_EINVAL, "%s: rope is NULL", fn);
    if (r->axes < 1 || r->axes > ZIPVL_MAX_AXES) return set_error(ZIPVL_EINVAL, "%s: rope has %d axes (1 to %d)", fn, r->axes, ZIPVL_MAX_AXES);
    if (r->pairs < 8 || r->pairs % 8 || 2 * r->pairs > d) return set_error(ZIPVL_ESHAPE, "%s: rope has %d pairs (a multiple of 8 up to d / 2 = %d)", fn, r->pairs, d / 2);
    if (r->layout != ZIPVL_ROPE_HALVES && r->layout != ZIPVL_ROPE_NEIGHBOURS) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown layout %d of rope", fn, r->layout);
    if (r->reserved) return set_error(ZIPVL_EUNSUPPORTED, "%s: reserved field of rope is %d", fn, r->reserved);
    for (int i = 0; i < r->pairs; ++i) {
        if (!(std::fabs(r->freq[i]) <= 6.283185307179587)) return set_error(ZIPVL_EINVAL, "%s: freq[%d] = %g is not within 2 pi of zero", fn, i, r->freq[i]);
        if (r->axis[i] < 0 || r->axis[i] >= r->axes) return set_error(ZIPVL_EINVAL, "%s: axis[%d] = %d is outside [0, %d)", fn, i, r->axis[i], r->axes);
    }
    return ZIPVL_OK;
}

// An output of `sizes` rows of d elements: no element twice (every stride goes past all that the smaller ones cover).
static int check_apart(const char* fn, const char* what, const int64_t* strides, const int (&sizes)[3], int d) {
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return strides[a] < strides[b]; });
    int64_t covered = d;
    for (int a : order) {
        if (sizes[a] == 1) continue;
        if (strides[a] < covered) return set_error(ZIPVL_EINVAL, "%s: rows of %s overlap (stride %lld)", fn, what, (long long)strides[a]);
        covered = strides[a] * (sizes[a] - 1) + covered;
    }
    return ZIPVL_OK;
}

static int check_tokens(const char* fn, const zipvl_dims& d) {
    if ((int64_t)d.B * d.n >= (1 << 30)) return set_error(ZIPVL_ESHAPE, "%s: B*n = %lld is not below 2^30", fn, (long long)d.B * d.n);
    return ZIPVL_OK;
}

int zipvl_rotate(const void* Q, const void* K, const zipvl_dims* dims, const int32_t* pos, const zipvl_rope* rope, int flags,
                 void* Qo, void* Ko, const zipvl_dims* out, void* stream)
{
    const char* fn = "zipvl_rotate";
    int rc = check_dims(fn, dims, Q != nullptr, K != nullptr, false);
    if (rc || (rc = check_tokens(fn, *dims)) || (rc = check_rope(fn, rope, dims->d))) return rc;
    if (!Q && !K) return set_error(ZIPVL_EINVAL, "%s: Q and K are NULL", fn);
    if ((Q == nullptr) != (Qo == nullptr) || (K == nullptr) != (Ko == nullptr))
        return set_error(ZIPVL_EINVAL, "%s: Q and Qo, K and Ko must both be given or both be NULL", fn);
    for (const void* p : {Q, K, (const void*)Qo, (const void*)Ko})
        if (!aligned16(p)) return set_error(ZIPVL_EALIGN, "%s: Q, K, Qo or Ko is not 16-byte aligned", fn);
    if (!pos) return set_error(ZIPVL_EINVAL, "%s: pos is NULL", fn);
    if (reinterpret_cast<uintptr_t>(pos) & 3u) return set_error(ZIPVL_EALIGN, "%s: pos is not 4-byte aligned", fn);
    if (flags & ~ZIPVL_ROTATE_INVERSE) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    zipvl_dims o = *dims;
    if (out) {
        std::copy(out->q_strides, out->q_strides + 3, o.q_strides);
        std::copy(out->k_strides, out->k_strides + 3, o.k_strides);
        if ((rc = check_dims(fn, &o, Q != nullptr, K != nullptr, false))) return rc;
    }
    if (Q && (rc = check_apart(fn, "Qo", o.q_strides, {o.B, o.Hq, o.n}, o.d))) return rc;
    if (K && (rc = check_apart(fn, "Ko", o.k_strides, {o.B, o.Hkv, o.n}, o.d))) return rc;
    auto same = [](const int64_t* a, const int64_t* b) { return std::equal(a, a + 3, b); };
    if ((Q && Qo == Q && !same(o.q_strides, dims->q_strides)) || (K && Ko == K && !same(o.k_strides, dims->k_strides)))
        return set_error(ZIPVL_EINVAL, "%s: an output in the place of its input must have its strides", fn);
    return launch_rotate(Q, K, *dims, pos, *rope, flags, Qo, Ko, o, (hipStream_t)stream);
}

static int check_pages(const char* fn, const zipvl_pages* p) {
    if (!p) return set_error(ZIPVL_EINVAL, "%s: pages is NULL", fn);
    if (!p->K || !p->V) return set_error(ZIPVL_EINVAL, "%s: an array of pages is NULL", fn);
    if (!aligned16(p->K) || !aligned16(p->V)) return set_error(ZIPVL_EALIGN, "%s: an array of pages is not 16-byte aligned", fn);
    if (p->num_pages < 1) return set_error(ZIPVL_EINVAL, "%s: num_pages = %d must be positive", fn, p->num_pages);
    if (p->page < 16 || p->page > 256 || (p->page & (p->page - 1))) return set_error(ZIPVL_ESHAPE, "%s: pages of %d rows (16, 32, 64, 128 or 256)", fn, p->page);
    return ZIPVL_OK;
}

static int check_table(const char* fn, const char* what, const int32_t* table, int32_t width, int page) {
    if (!table) return set_error(ZIPVL_EINVAL, "%s: %s is NULL", fn, what);
    if (reinterpret_cast<uintptr_t>(table) & 3u) return set_error(ZIPVL_EALIGN, "%s: %s is not 4-byte aligned", fn, what);
    if (width < 1) return set_error(ZIPVL_EINVAL, "%s: %s of %d pages a unit", fn, what, width);
    if ((int64_t)width * page > (1 << 24)) return set_error(ZIPVL_ESHAPE, "%s: %s holds %lld rows a unit, more than 2^24", fn, what, (long long)width * page);
    return ZIPVL_OK;
}

int zipvl_paged_append(const void* K, const void* V, const zipvl_dims* dims, const int32_t* idx, const int32_t* k, const int32_t* pos,
                       const zipvl_rope* rope, const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const int32_t* start,
                       int32_t* len, const void* Q, void* Qo, int flags, void* stream)
{
    const char* fn = "zipvl_paged_append";
    int rc = check_dims(fn, dims, Q != nullptr, true, true);
    if (rc || (rc = check_tokens(fn, *dims)) || (rc = check_pages(fn, pages)) || (rc = check_table(fn, "table", table, table_pages, pages->page))) return rc;
    ZIPVL_REQUIRE_PTR(fn, K);
    ZIPVL_REQUIRE_PTR(fn, V);
    if (!start || !len) return set_error(ZIPVL_EINVAL, "%s: start / len is NULL", fn);
    if (rope && (rc = check_rope(fn, rope, dims->d))) return rc;
    if (rope && !pos) return set_error(ZIPVL_EINVAL, "%s: pos is NULL", fn);
    if (idx && !k) return set_error(ZIPVL_EINVAL, "%s: idx is given without k", fn);
    if ((Q == nullptr) != (Qo == nullptr)) return set_error(ZIPVL_EINVAL, "%s: Q and Qo must both be given or both be NULL", fn);
    if (!aligned16(Q) || !aligned16(Qo)) return set_error(ZIPVL_EALIGN, "%s: Q or Qo is not 16-byte aligned", fn);
    if (Q && idx) return set_error(ZIPVL_EUNSUPPORTED, "%s: Q together with idx", fn);
    if (Q && !rope) return set_error(ZIPVL_EINVAL, "%s: Q is given without rope", fn);
    if (Q && Qo == Q) {
        const int64_t dense[3] = {(int64_t)dims->Hq * dims->n * dims->d, (int64_t)dims->n * dims->d, dims->d};
        const int sizes[3] = {dims->B, dims->Hq, dims->n};
        for (int a = 0; a < 3; ++a)
            if (sizes[a] > 1 && dims->q_strides[a] != dense[a]) return set_error(ZIPVL_EINVAL, "%s: Qo in the place of a Q that is not contiguous", fn);
    }
    if (flags & ~ZIPVL_T_PER_BATCH) return set_error(ZIPVL_EUNSUPPORTED, "%s: unknown flags 0x%x", fn, flags);
    if ((reinterpret_cast<uintptr_t>(idx) | reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(rope ? pos : nullptr) |
         reinterpret_cast<uintptr_t>(start) | reinterpret_cast<uintptr_t>(len)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: idx, k, pos, start or len is not 4-byte aligned", fn);
    // len is written while other workgroups read the rest
    const int64_t units = (int64_t)dims->B * dims->Hkv, sets = flags & ZIPVL_T_PER_BATCH ? dims->B : units, tokens = (int64_t)dims->B * dims->n;
    auto meets = [&](const int32_t* a, int64_t n) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(len);
        return a && x < y + 4 * units && y < x + 4 * n;
    };
    if ((start != len && meets(start, units)) || meets(k, sets) || meets(idx, sets * dims->n) || meets(table, units * table_pages) ||
        meets(rope ? pos : nullptr, rope ? rope->axes * tokens : 0))
        return set_error(ZIPVL_EINVAL, "%s: len overlaps start, k, idx, pos or table (it may be start itself)", fn);
    return launch_paged_append(K, V, *dims, idx, k, pos, rope, *pages, table, table_pages, start, len, Q, Qo, flags, (hipStream_t)stream);
}

int zipvl_decode_attn_paged(const void* q, const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const int32_t* len,
                            const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin,
                            int32_t groups, const zipvl_dims* dims, float softmax_scale, void* o, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_decode_attn_paged";
    zipvl_dims d = dims ? *dims : zipvl_dims{};
    d.n = 1;                                                 // not looked at
    int rc = check_dims(fn, dims ? &d : nullptr, false, false, false);
    if (rc || (rc = check_pages(fn, pages)) || (rc = check_table(fn, "table", table, table_pages, pages->page))) return rc;
    if (d.Hq / d.Hkv > 32) return set_error(ZIPVL_ESHAPE, "%s: %d query heads per KV head (up to 32)", fn, d.Hq / d.Hkv);
    ZIPVL_REQUIRE_PTR(fn, q);
    ZIPVL_REQUIRE_PTR(fn, o);
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if (groups < 0 || groups > d.B) return set_error(ZIPVL_EINVAL, "%s: %d groups of %d batch elements", fn, groups, d.B);
    if (groups) {
        if ((rc = check_table(fn, "prefix_table", prefix_table, prefix_pages, pages->page))) return rc;
        if (!prefix_len || !group_begin) return set_error(ZIPVL_EINVAL, "%s: prefix_len / group_begin is NULL", fn);
    } else {
        prefix_table = prefix_len = group_begin = nullptr;
        prefix_pages = 0;
    }
    if ((reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(prefix_len) | reinterpret_cast<uintptr_t>(group_begin)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: len, prefix_len or group_begin is not 4-byte aligned", fn);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    const size_t need = decode_paged_workspace_bytes(d, table_pages * pages->page, prefix_pages * pages->page);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_decode_attn_paged(q, *pages, table, table_pages, len, prefix_table, prefix_pages, prefix_len, group_begin, groups, d,
                                    softmax_scale, o, ws, (hipStream_t)stream);
}

// Two arrays of `a` and `b` bytes: apart, or NULL.
static bool apart(const void* x, int64_t a, const void* y, int64_t b) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
    return !x || !y || p + a <= q || q + b <= p;
}

static int check_chunk(const char* fn, const zipvl_dims* dims, const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                       float softmax_scale) {
    int rc = check_dims(fn, dims, true, false, false);
    if (rc || (rc = check_tokens(fn, *dims)) || (rc = check_pages(fn, pages)) || (rc = check_table(fn, "table", table, table_pages, pages->page))) return rc;
    if ((int64_t)dims->n * (dims->Hq / dims->Hkv) >= (1 << 30)) return set_error(ZIPVL_ESHAPE, "%s: n * Hq / Hkv = %lld is not below 2^30", fn, (long long)dims->n * (dims->Hq / dims->Hkv));
    if (!len) return set_error(ZIPVL_EINVAL, "%s: len is NULL", fn);
    if ((reinterpret_cast<uintptr_t>(len) | reinterpret_cast<uintptr_t>(k)) & 3u) return set_error(ZIPVL_EALIGN, "%s: len or k is not 4-byte aligned", fn);
    if (!(softmax_scale > 0.f) || !(softmax_scale < 1e30f)) return set_error(ZIPVL_EINVAL, "%s: softmax_scale must be positive and finite", fn);
    return ZIPVL_OK;
}

int zipvl_chunk_attn_paged(const void* Q, const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                           const int32_t* prefix_table, int32_t prefix_pages, const int32_t* prefix_len, const int32_t* group_begin, int32_t groups,
                           const zipvl_dims* dims, float softmax_scale, void* O, const zipvl_dims* out, float* lse, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_chunk_attn_paged";
    int rc = check_chunk(fn, dims, pages, table, table_pages, len, k, softmax_scale);
    if (rc) return rc;
    const zipvl_dims& d = *dims;
    ZIPVL_REQUIRE_PTR(fn, Q);
    ZIPVL_REQUIRE_PTR(fn, O);
    if (groups < 0 || groups > d.B) return set_error(ZIPVL_EINVAL, "%s: %d groups of %d batch elements", fn, groups, d.B);
    if (groups) {
        if ((rc = check_table(fn, "prefix_table", prefix_table, prefix_pages, pages->page))) return rc;
        if (!prefix_len || !group_begin) return set_error(ZIPVL_EINVAL, "%s: prefix_len / group_begin is NULL", fn);
    } else {
        prefix_table = prefix_len = group_begin = nullptr;
        prefix_pages = 0;
    }
    if ((reinterpret_cast<uintptr_t>(prefix_len) | reinterpret_cast<uintptr_t>(group_begin) | reinterpret_cast<uintptr_t>(lse)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: prefix_len, group_begin or lse is not 4-byte aligned", fn);
    zipvl_dims o = d;
    const int64_t dense[3] = {(int64_t)d.Hq * d.n * d.d, (int64_t)d.n * d.d, d.d};
    std::copy(out ? out->q_strides : dense, (out ? out->q_strides : dense) + 3, o.q_strides);
    if ((rc = check_dims(fn, &o, true, false, false)) || (rc = check_apart(fn, "O", o.q_strides, {d.B, d.Hq, d.n}, d.d))) return rc;
    if (O == Q) return set_error(ZIPVL_EINVAL, "%s: O in the place of Q", fn);
    const size_t need = chunk_attn_workspace_bytes(d, ((int64_t)table_pages + prefix_pages) * pages->page);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_chunk_attn_paged(Q, *pages, table, table_pages, len, k, prefix_table, prefix_pages, prefix_len, group_begin, groups, d, softmax_scale,
                                   O, o.q_strides, lse, ws, (hipStream_t)stream);
}

int zipvl_paged_weigh(const void* Q, const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const int32_t* len, const int32_t* k,
                      const float* lse, int64_t lse_pitch, const zipvl_dims* dims, float softmax_scale, const float* before, float* weight, void* stream)
{
    const char* fn = "zipvl_paged_weigh";
    const int rc = check_chunk(fn, dims, pages, table, table_pages, len, k, softmax_scale);
    if (rc) return rc;
    ZIPVL_REQUIRE_PTR(fn, Q);
    if (!lse || !weight) return set_error(ZIPVL_EINVAL, "%s: lse / weight is NULL", fn);
    if (lse_pitch < dims->n) return set_error(ZIPVL_EINVAL, "%s: lse_pitch = %lld is smaller than n = %d", fn, (long long)lse_pitch, dims->n);
    if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(before) | reinterpret_cast<uintptr_t>(weight)) & 3u)
        return set_error(ZIPVL_EALIGN, "%s: lse, before or weight is not 4-byte aligned", fn);
    const int64_t units = (int64_t)dims->B * dims->Hkv, bytes = units * table_pages * pages->page * 4, queries = ((int64_t)dims->B * dims->Hq - 1) * lse_pitch + dims->n;
    if ((before != weight && !apart(before, bytes, weight, bytes)) || !apart(len, units * 4, weight, bytes) || !apart(k, units * 4, weight, bytes) ||
        !apart(lse, queries * 4, weight, bytes) || !apart(table, units * table_pages * 4, weight, bytes))
        return set_error(ZIPVL_EINVAL, "%s: weight overlaps before, len, k, lse or table (it may be before itself)", fn);
    return launch_paged_weigh(Q, *pages, table, table_pages, len, k, lse, lse_pitch, *dims, softmax_scale, before, weight, (hipStream_t)stream);
}

int zipvl_paged_evict(const zipvl_pages* pages, const int32_t* table, int32_t table_pages, const zipvl_dims* dims, const int32_t* len, const int32_t* k,
                      const float* weight, const int32_t* tokens, int32_t budget, int32_t sinks, int32_t recent,
                      int32_t* len_out, float* weight_out, int32_t* tokens_out, void* ws, size_t ws_bytes, void* stream)
{
    const char* fn = "zipvl_paged_evict";
    zipvl_dims d = dims ? *dims : zipvl_dims{};
    d.n = 1;                                                 // not looked at
    d.Hq = d.Hkv;
    int rc = check_dims(fn, dims ? &d : nullptr, false, false, false);
    if (rc || (rc = check_pages(fn, pages)) || (rc = check_table(fn, "table", table, table_pages, pages->page))) return rc;
    if (!len || !weight || !len_out || !weight_out) return set_error(ZIPVL_EINVAL, "%s: len, weight, len_out or weight_out is NULL", fn);
    if ((tokens == nullptr) != (tokens_out == nullptr)) return set_error(ZIPVL_EINVAL, "%s: tokens and tokens_out must both be given or both be NULL", fn);
    if (budget < 0 || sinks < 0 || recent < 0) return set_error(ZIPVL_EINVAL, "%s: budget, sinks and recent must not be negative (got %d %d %d)", fn, budget, sinks, recent);
    for (const void* p : {(const void*)len, (const void*)k, (const void*)weight, (const void*)tokens, (const void*)len_out, (const void*)weight_out, (const void*)tokens_out})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return set_error(ZIPVL_EALIGN, "%s: an array is not 4-byte aligned", fn);
    for (const void* p : {(const void*)weight, (const void*)tokens, (const void*)weight_out, (const void*)tokens_out})
        if (!aligned16(p)) return set_error(ZIPVL_EALIGN, "%s: weight, tokens, weight_out or tokens_out is not 16-byte aligned", fn);
    const int64_t units = (int64_t)d.B * d.Hkv, room = (int64_t)table_pages * pages->page;
    struct Span { const void* p; int64_t bytes; };
    const Span ins[5] = {{len, units * 4}, {weight, units * room * 4}, {tokens, units * room * 4}, {k, units * 4}, {table, units * table_pages * 4}};
    const Span outs[3] = {{len_out, units * 4}, {weight_out, units * room * 4}, {tokens_out, units * room * 4}};
    for (int y = 0; y < 3; ++y) {
        for (int x = 0; x < 5; ++x)
            if (!(x == y && ins[x].p == outs[y].p) && !apart(ins[x].p, ins[x].bytes, outs[y].p, outs[y].bytes))
                return set_error(ZIPVL_EINVAL, "%s: an output overlaps another array (len_out may be len, weight_out weight, tokens_out tokens)", fn);
        for (int x = 0; x < y; ++x)
            if (!apart(outs[x].p, outs[x].bytes, outs[y].p, outs[y].bytes)) return set_error(ZIPVL_EINVAL, "%s: two outputs overlap", fn);
    }
    const size_t need = paged_evict_workspace_bytes(units, room, budget);
    if (!ws || ws_bytes < need) return set_error(ZIPVL_EWORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (!aligned16(ws)) return set_error(ZIPVL_EALIGN, "%s: ws is not 16-byte aligned", fn);
    return launch_paged_evict(*pages, table, table_pages, d, len, k, weight, tokens, budget, sinks, recent, len_out, weight_out, tokens_out, ws, (hipStream_t)stream);
}

int zipvl_probe_mfma(int iters, int workgroups, float* out, void* stream)
{
    if (iters < 1 || workgroups < 1 || !out) return set_error(ZIPVL_EINVAL, "zipvl_probe_mfma: iters, workgroups must be positive and out given");
    return launch_probe_mfma(iters, workgroups, out, (hipStream_t)stream);
}

int zipvl_probe_stream_read(const void* src, size_t bytes, int workgroups, uint32_t* out, void* stream)
{
    if (!src || !out || workgroups < 1 || bytes < 16 || (bytes & 15)) return set_error(ZIPVL_EINVAL, "zipvl_probe_stream_read: src, out, workgroups >= 1 and bytes a positive multiple of 16 are required");
    if (!aligned16(src)) return set_error(ZIPVL_EALIGN, "zipvl_probe_stream_read: src is not 16-byte aligned");
    return launch_probe_read(src, bytes, workgroups, out, (hipStream_t)stream);
}

int zipvl_timing_enable(int on) {
    std::lock_guard<std::mutex> lk(g_tmu);
    g_timed.clear();
    g_pool_used = 0;
    g_timing = on != 0;
    return ZIPVL_OK;
}

int zipvl_timing_read(int kernel_id, double* total_ms, int* launches) {
    if (!total_ms || !launches) return set_error(ZIPVL_EINVAL, "zipvl_timing_read: NULL output");
    if (kernel_id < 0 || kernel_id >= ZIPVL_K_COUNT) return set_error(ZIPVL_EINVAL, "zipvl_timing_read: kernel id %d", kernel_id);
    std::lock_guard<std::mutex> lk(g_tmu);
    double sum = 0.0;
    int cnt = 0;
    for (const TimedLaunch& t : g_timed) {
        if (t.id != kernel_id) continue;
        if (hipEventSynchronize(t.stop) != hipSuccess) return set_error(ZIPVL_EHIP, "zipvl_timing_read: event wait failed");
        float ms = 0.f;
        if (hipEventElapsedTime(&ms, t.start, t.stop) != hipSuccess) return set_error(ZIPVL_EHIP, "zipvl_timing_read: elapsed time failed");
        sum += ms;
        ++cnt;
    }
    *total_ms = sum;
    *launches = cnt;
    return ZIPVL_OK;
}

}  // extern "C"
