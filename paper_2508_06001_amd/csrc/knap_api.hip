// C-ABI entry points of libknapattn: argument checks, workspace carving and
// launches.  Nothing here allocates, frees or synchronises.
#include "knapattn.h"
#include "knapattn_bench.h"
#include "knap_kernels.h"

#include <hip/hip_runtime.h>

#include <atomic>
#include <mutex>

// Scratch of knap_varlen_attn_bwd_noalloc: the per-row dot products of dout and out and the base-2
// log-sum-exp (fp32, (H, T) each) and, in the last 256 bytes, the work-queue counters.  Part of the library's device image:
// every GPU the library runs on holds its own copy until the process ends.  Host code never uses this
// name as an address; it uses the pointer hipGetSymbolAddress returned on that device (DeviceInfo::scratch).
static __device__ __align__(256) unsigned char scratch[2 * KNAP_NOALLOC_MAX_ROWS * sizeof(float) + 256];

namespace {

thread_local int g_last_hip_error = 0;
thread_local hipEvent_t g_prof_start = nullptr;
thread_local hipEvent_t g_prof_stop = nullptr;

struct DeviceInfo {
  int cus = 0;
  int fwd_wg[2] = {0, 0};   // workgroups per CU, index 0: d = 64, 1: d = 128
  int dq_wg[2] = {0, 0};
  unsigned* queues = nullptr;      // this device's copy of the forward's work-queue counters (a backward has its own in its workspace)
  std::atomic<uint64_t> fwd_calls{0}, fwd_captured{0};      // eager and captured forward calls so far, which take the sets in turn
  unsigned char* scratch = nullptr;   // this device's copy of `scratch`
};

constexpr int kMaxDevices = 64;

void fill_device_info(DeviceInfo& di, int dev) {
  int cus = 0;
  if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) {
    (void)hipGetLastError();
    return;
  }
  di.fwd_wg[0] = knap::fwd_workgroups_per_cu(64);
  di.fwd_wg[1] = knap::fwd_workgroups_per_cu(128);
  di.dq_wg[0] = knap::bwd_dq_workgroups_per_cu(64);
  di.dq_wg[1] = knap::bwd_dq_workgroups_per_cu(128);
  di.queues = knap::queue_base();
  if (!di.queues) return;
  void* p = nullptr;
  if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) {
    (void)hipGetLastError();
    return;
  }
  di.scratch = static_cast<unsigned char*>(p);
  di.cus = cus;     // last: marks the entry as complete
}

// per-device launch geometry and device-image addresses, looked up once per device with that
// device current (occupancy and symbol queries do not allocate); nullptr if the lookup failed
DeviceInfo* device_info() {
  static DeviceInfo info[kMaxDevices];
  static std::once_flag once[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) { (void)hipGetLastError(); return nullptr; }
  std::call_once(once[dev], fill_device_info, std::ref(info[dev]), dev);
  return info[dev].cus > 0 ? &info[dev] : nullptr;
}

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int check_common(const void* q, const void* k, const void* v, const int32_t* cu, int n_seq, int H, int d,
                 float scale) {
  if (n_seq < 0 || H <= 0 || (d != 64 && d != 128)) return KNAP_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !(scale < 3.0e38f)) return KNAP_ERR_INVALID_ARG;   // positive and finite
  if (n_seq > KNAP_MAX_SEQS) return KNAP_ERR_TOO_MANY_SEQS;
  if (n_seq == 0) return KNAP_OK;
  if (!q || !k || !v || !cu) return KNAP_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(cu, 4)) return KNAP_ERR_INVALID_ARG;
  return KNAP_OK;
}

bool capturing(void* stream) {
  hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(static_cast<hipStream_t>(stream), &capture) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return capture != hipStreamCaptureStatusNone;
}

// the counters that a forward launch draws from: the next set in turn
hipError_t next_counters(DeviceInfo* di, void* stream, unsigned** counters) {
  if (capturing(stream)) {
    *counters = di->queues + 8 * knap::captured_set(di->fwd_captured.fetch_add(1));
    return hipSuccess;
  }
  const knap::EagerSet s = knap::eager_set(di->fwd_calls.fetch_add(1));
  *counters = di->queues + 8 * s.set;
  return s.clear >= 0 ? knap::clear_queue_sets(di->queues + 8 * s.clear, knap::kSetsPerThird, static_cast<hipStream_t>(stream)) : hipSuccess;
}

int fwd_impl(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq,
             int H, int d, float scale, bool causal, void* out, float* lse, void* stream) {
  const int rc = check_common(q, k, v, cu_seqlens, n_seq, H, d, scale);
  if (rc != KNAP_OK) return rc;
  if (n_seq == 0) return KNAP_OK;
  if (!out || !lse || !aligned(out, 16) || !aligned(lse, 4)) return KNAP_ERR_INVALID_ARG;
  if (out == q || out == k || out == v) return KNAP_ERR_INVALID_ARG;
  DeviceInfo* di = device_info();
  if (!di) return KNAP_ERR_LAUNCH_FAILED;
  const int grid = di->cus * di->fwd_wg[d == 128];
  unsigned* counters;
  hipError_t e = next_counters(di, stream, &counters);
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  e = (causal ? knap::launch_fwd_causal : knap::launch_fwd_full)(q, k, v, cu_seqlens, n_seq, H, d, scale, out, lse, counters, grid,
                                                                 static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

int bwd_impl(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq,
             int H, int d, float scale, bool causal,
             const void* out, const float* lse, const void* dout, void* dq, void* dk, void* dv,
             int64_t total_tokens, void* workspace, size_t workspace_bytes, bool own_scratch, void* stream);

}  // namespace

int knap::device_cus() {
  DeviceInfo* di = device_info();
  return di ? di->cus : 0;
}

int knap::launch_status(hipError_t e) {
  if (e == hipSuccess) return KNAP_OK;
  g_last_hip_error = static_cast<int>(e);
  return KNAP_ERR_LAUNCH_FAILED;
}

extern "C" {

int knap_varlen_attn_fwd(const void* q, const void* k, const void* v,
                         const int32_t* cu_seqlens, int n_seq,
                         int H, int d, float scale,
                         void* out, float* lse, void* stream) {
  return fwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, false, out, lse, stream);
}

int knap_varlen_attn_causal_fwd(const void* q, const void* k, const void* v,
                                const int32_t* cu_seqlens, int n_seq,
                                int H, int d, float scale,
                                void* out, float* lse, void* stream) {
  return fwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, true, out, lse, stream);
}

size_t knap_varlen_attn_bwd_workspace_bytes(int64_t total_tokens, int n_seq, int H, int d) {
  (void)n_seq;
  if (total_tokens <= 0 || H <= 0 || d <= 0) return 0;
  // -delta and the base-2 log-sum-exp, fp32 (H, T) each, then 256 bytes of work-queue counters
  return 2 * round_up(static_cast<size_t>(total_tokens) * H * sizeof(float), 256) + 256;
}

int knap_varlen_attn_bwd(const void* q, const void* k, const void* v,
                         const int32_t* cu_seqlens, int n_seq,
                         int H, int d, float scale,
                         const void* out, const float* lse, const void* dout,
                         void* dq, void* dk, void* dv,
                         int64_t total_tokens,
                         void* workspace, size_t workspace_bytes, void* stream) {
  return bwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, false, out, lse, dout, dq, dk, dv, total_tokens,
                  workspace, workspace_bytes, false, stream);
}

int knap_varlen_attn_bwd_noalloc(const void* q, const void* k, const void* v,
                                 const int32_t* cu_seqlens, int n_seq,
                                 int H, int d, float scale,
                                 const void* out, const float* lse, const void* dout,
                                 void* dq, void* dk, void* dv,
                                 int64_t total_tokens, void* stream) {
  return bwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, false, out, lse, dout, dq, dk, dv, total_tokens,
                  nullptr, 0, true, stream);
}

int knap_varlen_attn_causal_bwd(const void* q, const void* k, const void* v,
                                const int32_t* cu_seqlens, int n_seq,
                                int H, int d, float scale,
                                const void* out, const float* lse, const void* dout,
                                void* dq, void* dk, void* dv,
                                int64_t total_tokens,
                                void* workspace, size_t workspace_bytes, void* stream) {
  return bwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, true, out, lse, dout, dq, dk, dv, total_tokens,
                  workspace, workspace_bytes, false, stream);
}

}  // extern "C"

namespace {

int bwd_impl(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq,
             int H, int d, float scale, bool causal,
             const void* out, const float* lse, const void* dout, void* dq, void* dk, void* dv,
             int64_t total_tokens, void* workspace, size_t workspace_bytes, bool own_scratch, void* stream) {
  const int rc = check_common(q, k, v, cu_seqlens, n_seq, H, d, scale);
  if (rc != KNAP_OK) return rc;
  if (total_tokens < 0 || total_tokens > INT32_MAX) return KNAP_ERR_INVALID_ARG;
  // the library's own scratch holds one float per (row, head): larger bags are refused, whatever else is wrong
  if (own_scratch && total_tokens * (int64_t)H > (int64_t)KNAP_NOALLOC_MAX_ROWS) return KNAP_ERR_SCRATCH_TOO_SMALL;
  if (n_seq == 0 || total_tokens == 0) return KNAP_OK;
  if (!out || !lse || !dout || !dq || !dk || !dv) return KNAP_ERR_INVALID_ARG;
  if (!aligned(out, 16) || !aligned(dout, 16) || !aligned(dq, 16) || !aligned(dk, 16) || !aligned(dv, 16) ||
      !aligned(lse, 4))
    return KNAP_ERR_INVALID_ARG;
  if (dq == dk || dq == dv || dk == dv || dq == q || dk == k || dv == v) return KNAP_ERR_INVALID_ARG;
  const size_t need = knap_varlen_attn_bwd_workspace_bytes(total_tokens, n_seq, H, d);
  if (!own_scratch) {
    if (!workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
    if (workspace_bytes < need) return KNAP_ERR_WORKSPACE_TOO_SMALL;
  }
  DeviceInfo* di = device_info();
  if (!di) return KNAP_ERR_LAUNCH_FAILED;
  if (own_scratch) workspace = di->scratch;     // carved exactly as a caller's workspace; need <= sizeof(scratch)

  float* delta = static_cast<float*>(workspace);
  float* lse2 = reinterpret_cast<float*>(static_cast<char*>(workspace) + (need - 256) / 2);
  unsigned* counters = reinterpret_cast<unsigned*>(static_cast<char*>(workspace) + need - 256);
  const int dq_wg = di->dq_wg[d == 128];
  const knap::BwdArgs args = {q, k, v, out, dout, lse, cu_seqlens, n_seq, H, scale, dq, dk, dv, delta, lse2, counters};
  if (knap::bwd_joint(total_tokens, n_seq, H, d, causal, di->cus)) {
    const hipError_t e = knap::launch_joint(args, d, causal, knap::bwd_small(total_tokens, n_seq, H, d, causal, di->cus), (int)total_tokens, di->cus, static_cast<hipStream_t>(stream), g_prof_start,
                                            g_prof_stop);
    if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
    return KNAP_OK;
  }
  const int pairs = knap::dkdv_pairs(total_tokens, n_seq, H, d, causal, di->cus);
  const hipError_t e = knap::launch_bwd(args, d, causal, pairs, di->cus, dq_wg, static_cast<hipStream_t>(stream),
                                        g_prof_start, g_prof_stop);
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------
// Ulysses layout switch: local data movement
// ---------------------------------------------------------------------------

namespace {

// 16-byte units per row of `heads` heads of d two-byte elements; 0 if the row is not a whole number of units
uint64_t row_units(int heads, int d) {
  const uint64_t bytes = (uint64_t)heads * (uint64_t)d * 2u;
  return bytes % 16u ? 0u : bytes / 16u;
}

int ulysses_heads(const void* src, void* dst, int64_t local_tokens, int H, int d, int g, bool pack, void* stream) {
  if (local_tokens < 0 || H <= 0 || d <= 0 || g <= 0 || H % g != 0) return KNAP_ERR_INVALID_ARG;
  const uint64_t U = row_units(H / g, d);
  if (U == 0) return KNAP_ERR_INVALID_ARG;
  if (local_tokens == 0) return KNAP_OK;
  if ((uint64_t)local_tokens * g * U > (1ull << 31)) return KNAP_ERR_INVALID_ARG;
  if (!src || !dst || src == dst || !aligned(src, 16) || !aligned(dst, 16)) return KNAP_ERR_INVALID_ARG;
  if (!device_info()) return KNAP_ERR_LAUNCH_FAILED;
  const hipError_t e = knap::launch_ulysses_heads(src, dst, (uint32_t)local_tokens, (uint32_t)U, (uint32_t)g, pack,
                                                  static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

int ulysses_rows(const void* src, void* dst, const int32_t* row_map, int64_t total_tokens, int heads_local, int d,
                 bool gather, void* stream) {
  if (total_tokens < 0 || heads_local <= 0 || d <= 0) return KNAP_ERR_INVALID_ARG;
  const uint64_t U = row_units(heads_local, d);
  if (U == 0) return KNAP_ERR_INVALID_ARG;
  if (total_tokens == 0) return KNAP_OK;
  if ((uint64_t)total_tokens * U > (1ull << 31)) return KNAP_ERR_INVALID_ARG;
  if (!src || !dst || !row_map || src == dst || !aligned(src, 16) || !aligned(dst, 16) || !aligned(row_map, 4))
    return KNAP_ERR_INVALID_ARG;
  if (!device_info()) return KNAP_ERR_LAUNCH_FAILED;
  const hipError_t e = knap::launch_ulysses_rows(src, dst, row_map, (uint32_t)total_tokens, (uint32_t)U, gather,
                                                 static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

}  // namespace

int knap_ulysses_pack_heads(const void* x, int64_t local_tokens, int H, int d, int g, void* y, void* stream) {
  return ulysses_heads(x, y, local_tokens, H, d, g, true, stream);
}

int knap_ulysses_unpack_heads(const void* y, int64_t local_tokens, int H, int d, int g, void* x, void* stream) {
  return ulysses_heads(y, x, local_tokens, H, d, g, false, stream);
}

size_t knap_ulysses_plan_workspace_bytes(int n_seq, int g) {
  if (n_seq < 0 || g <= 0) return 0;
  return round_up((static_cast<size_t>(n_seq) + 1) * static_cast<size_t>(g) * sizeof(int32_t), 256);
}

int knap_ulysses_plan(const int32_t* cu_seqlens, int n_seq, int64_t total_tokens, int g,
                      int32_t* row_map, void* workspace, size_t workspace_bytes, void* stream) {
  if (n_seq < 0 || g <= 0 || g > KNAP_ULYSSES_MAX_GPUS || total_tokens < 0 || total_tokens > INT32_MAX)
    return KNAP_ERR_INVALID_ARG;
  if (n_seq > KNAP_MAX_SEQS) return KNAP_ERR_TOO_MANY_SEQS;
  if (n_seq == 0 || total_tokens == 0) return KNAP_OK;
  if (!cu_seqlens || !row_map || !workspace || !aligned(cu_seqlens, 4) || !aligned(row_map, 4) ||
      !aligned(workspace, 4))
    return KNAP_ERR_INVALID_ARG;
  if (workspace_bytes < knap_ulysses_plan_workspace_bytes(n_seq, g)) return KNAP_ERR_WORKSPACE_TOO_SMALL;
  const hipError_t e = knap::launch_ulysses_plan(cu_seqlens, n_seq, g, (int)total_tokens, row_map,
                                                 static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

int knap_ulysses_gather_chunks(const void* recv, const int32_t* row_map, int64_t total_tokens,
                               int heads_local, int d, void* z, void* stream) {
  return ulysses_rows(recv, z, row_map, total_tokens, heads_local, d, true, stream);
}

int knap_ulysses_scatter_chunks(const void* z, const int32_t* row_map, int64_t total_tokens,
                                int heads_local, int d, void* send, void* stream) {
  return ulysses_rows(z, send, row_map, total_tokens, heads_local, d, false, stream);
}

// ---------------------------------------------------------------------------
// Differential attention
// ---------------------------------------------------------------------------

namespace {

int diff_fwd_impl(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                  const float* lambda, bool causal, void* out, void* out2, float* lse, void* stream) {
  const int rc = check_common(q, k, v, cu_seqlens, n_seq, H, d, scale);
  if (rc != KNAP_OK || n_seq == 0) return rc;
  if (!lambda || !out || !lse || !aligned(lambda, 4) || !aligned(out, 16) || !aligned(out2, 16) || !aligned(lse, 4)) return KNAP_ERR_INVALID_ARG;
  if (out == q || out == k || out == v || out == out2 || (out2 && (out2 == q || out2 == k || out2 == v))) return KNAP_ERR_INVALID_ARG;
  DeviceInfo* di = device_info();
  if (!di) return KNAP_ERR_LAUNCH_FAILED;
  knap::DiffFwdArgs a = {static_cast<const __bf16*>(q), static_cast<const __bf16*>(k), static_cast<const __bf16*>(v), cu_seqlens, n_seq, H, scale,
                         lambda, static_cast<__bf16*>(out), static_cast<__bf16*>(out2), lse, nullptr};
  hipError_t e = next_counters(di, stream, &a.counters);
  if (e == hipSuccess) e = knap::launch_diff_fwd(a, d, causal, di->cus, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

int diff_bwd_impl(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                  const float* lambda, bool causal, const void* out, const void* out2, const float* lse, const void* dout, void* dq, void* dk,
                  void* dv, float* dlambda, int64_t total_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_common(q, k, v, cu_seqlens, n_seq, H, d, scale);
  if (rc != KNAP_OK) return rc;
  if (total_tokens < 0 || total_tokens > INT32_MAX) return KNAP_ERR_INVALID_ARG;
  if (n_seq == 0) return KNAP_OK;
  if (!dlambda || !aligned(dlambda, 4) || dlambda == lambda) return KNAP_ERR_INVALID_ARG;
  hipError_t e;
  if (total_tokens == 0) {
    e = knap::launch_layer_norm_zero(dlambda, nullptr, H, static_cast<hipStream_t>(stream));
  } else {
    if (!lambda || !out || !out2 || !lse || !dout || !dq || !dk || !dv) return KNAP_ERR_INVALID_ARG;
    if (!aligned(lambda, 4) || !aligned(out, 16) || !aligned(out2, 16) || !aligned(lse, 4) || !aligned(dout, 16) || !aligned(dq, 16) ||
        !aligned(dk, 16) || !aligned(dv, 16))
      return KNAP_ERR_INVALID_ARG;
    if (dq == dk || dq == dv || dk == dv || dq == q || dk == k || dv == v) return KNAP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
    if (workspace_bytes < knap_varlen_diff_attn_bwd_workspace_bytes(total_tokens, n_seq, H, d)) return KNAP_ERR_WORKSPACE_TOO_SMALL;
    DeviceInfo* di = device_info();
    if (!di) return KNAP_ERR_LAUNCH_FAILED;
    const size_t part = round_up(static_cast<size_t>(total_tokens) * H * sizeof(float), 256);
    char* ws = static_cast<char*>(workspace);
    auto at = [&](int i) { return reinterpret_cast<float*>(ws + i * part); };
    knap::DiffBwdArgs a = {static_cast<const __bf16*>(q), static_cast<const __bf16*>(k), static_cast<const __bf16*>(v),
                                 static_cast<const __bf16*>(out), static_cast<const __bf16*>(out2), static_cast<const __bf16*>(dout), cu_seqlens,
                                 n_seq, H, scale, lambda, lse, static_cast<__bf16*>(dq), static_cast<__bf16*>(dk), static_cast<__bf16*>(dv),
                                 dlambda, at(0), at(1), at(2), at(3), at(4), reinterpret_cast<unsigned*>(ws + 5 * part), nullptr};
    e = next_counters(di, stream, &a.dq_counters);
    if (e == hipSuccess) e = knap::launch_diff_bwd(a, d, causal, (int)total_tokens, di->cus, static_cast<hipStream_t>(stream));
  }
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

}  // namespace

int knap_varlen_diff_attn_fwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                              const float* lambda, void* out, void* out2, float* lse, void* stream) {
  return diff_fwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, lambda, false, out, out2, lse, stream);
}

int knap_varlen_diff_attn_causal_fwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                                     const float* lambda, void* out, void* out2, float* lse, void* stream) {
  return diff_fwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, lambda, true, out, out2, lse, stream);
}

size_t knap_varlen_diff_attn_bwd_workspace_bytes(int64_t total_tokens, int n_seq, int H, int d) {
  (void)n_seq;
  if (total_tokens <= 0 || H <= 0 || d <= 0) return 0;
  // five values of each (row, head), then 256 bytes of work-queue counters
  return 5 * round_up(static_cast<size_t>(total_tokens) * H * sizeof(float), 256) + 256;
}

int knap_varlen_diff_attn_bwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                              const float* lambda, const void* out, const void* out2, const float* lse, const void* dout, void* dq, void* dk,
                              void* dv, float* dlambda, int64_t total_tokens, void* workspace, size_t workspace_bytes, void* stream) {
  return diff_bwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, lambda, false, out, out2, lse, dout, dq, dk, dv, dlambda, total_tokens, workspace,
                       workspace_bytes, stream);
}

int knap_varlen_diff_attn_causal_bwd(const void* q, const void* k, const void* v, const int32_t* cu_seqlens, int n_seq, int H, int d, float scale,
                                     const float* lambda, const void* out, const void* out2, const float* lse, const void* dout, void* dq,
                                     void* dk, void* dv, float* dlambda, int64_t total_tokens, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  return diff_bwd_impl(q, k, v, cu_seqlens, n_seq, H, d, scale, lambda, true, out, out2, lse, dout, dq, dk, dv, dlambda, total_tokens, workspace,
                       workspace_bytes, stream);
}

// ---------------------------------------------------------------------------
// Rotary positions
// ---------------------------------------------------------------------------

namespace {

// rows of an output must not overlap: the heads of a token lie between two tokens, or the tokens of a head between two heads
bool rows_apart(int64_t tokens, int heads, int d, int64_t token, int64_t head) {
  if (token < 0 || head < 0) return false;
  if ((heads == 1 || head >= d) && (tokens == 1 || (token >= d && token - d >= (heads - 1) * head))) return true;
  return (tokens == 1 || token >= d) && (heads == 1 || (head >= d && (head - d) / token >= tokens - 1));
}

int rope_impl(const void* q, const void* k, int64_t tokens, int H, int H_k, int d, const int64_t* strides, int rot, int layout,
              const int32_t* positions, int n_axes, const int* axis_pairs, const int32_t* cu_seqlens, int n_seq,
              const double* freq, float factor, void* q_out, void* k_out, bool backward, void* stream) {
  if (tokens < 0 || tokens > INT32_MAX || H < 1 || H_k < 0 || d < 2 || d > KNAP_ROPE_MAX_DIM || rot < 2 || rot > d || rot % 2)
    return KNAP_ERR_INVALID_ARG;
  if (((int64_t)H + H_k) * d > (1 << 24) || (layout != KNAP_ROPE_HALF && layout != KNAP_ROPE_INTERLEAVED)) return KNAP_ERR_INVALID_ARG;
  if (!(factor > -3.0e38f && factor < 3.0e38f)) return KNAP_ERR_INVALID_ARG;
  knap::RopeArgs a{};
  if (positions) {
    if (n_axes < 1 || n_axes > KNAP_ROPE_MAX_AXES || (n_axes > 1 && !axis_pairs)) return KNAP_ERR_INVALID_ARG;
    int64_t end = 0;
    for (int x = 0; x < KNAP_ROPE_MAX_AXES; ++x) {
      if (x < n_axes && axis_pairs) {
        if (axis_pairs[x] < 0) return KNAP_ERR_INVALID_ARG;
        end += axis_pairs[x];
      } else if (x == 0) {
        end = rot / 2;
      }
      if (end > rot / 2) return KNAP_ERR_INVALID_ARG;
      a.axis_end[x] = (int)end;
    }
    if (end != rot / 2) return KNAP_ERR_INVALID_ARG;
  } else {
    if (n_seq < 0) return KNAP_ERR_INVALID_ARG;
    if (n_seq > KNAP_MAX_SEQS) return KNAP_ERR_TOO_MANY_SEQS;
    if (n_seq == 0) return KNAP_OK;
  }
  if (tokens == 0) return KNAP_OK;
  if (!q || !q_out || !freq || (H_k > 0 && (!k || !k_out)) || (!positions && !cu_seqlens)) return KNAP_ERR_INVALID_ARG;
  if (!aligned(q, 2) || !aligned(q_out, 2) || !aligned(freq, 8) || !aligned(positions, 4) || !aligned(cu_seqlens, 4)) return KNAP_ERR_INVALID_ARG;
  if (H_k > 0 && (!aligned(k, 2) || !aligned(k_out, 2) || q_out == k_out || q_out == k || k_out == q)) return KNAP_ERR_INVALID_ARG;
  const int64_t row_q = (int64_t)H * d, row_k = (int64_t)H_k * d;
  const int64_t packed[8] = {row_q, d, row_k, d, row_q, d, row_k, d};
  const int64_t* s = strides ? strides : packed;
  constexpr int64_t kMostStride = (int64_t)1 << 40;         // (row, stride) products stay far from 64 bits
  for (int i = 0; i < 8; ++i)
    if ((H_k > 0 || (i & 2) == 0) && (s[i] < 0 || s[i] > kMostStride)) return KNAP_ERR_INVALID_ARG;
  if (!rows_apart(tokens, H, d, s[4], s[5]) || (H_k > 0 && !rows_apart(tokens, H_k, d, s[6], s[7]))) return KNAP_ERR_INVALID_ARG;
  const bool in_place_q = q_out == q, in_place_k = H_k > 0 && k_out == k;
  if ((in_place_q && (s[0] != s[4] || s[1] != s[5])) || (in_place_k && (s[2] != s[6] || s[3] != s[7]))) return KNAP_ERR_INVALID_ARG;
  a.q = static_cast<const __bf16*>(q);
  a.q_out = static_cast<__bf16*>(q_out);
  a.q_token = s[0]; a.q_head = s[1]; a.qo_token = s[4]; a.qo_head = s[5];
  const bool half = layout == KNAP_ROPE_HALF;
  bool on16 = d % 8 == 0 && aligned(q, 16) && aligned(q_out, 16) && (s[0] | s[1] | s[4] | s[5]) % 8 == 0;
  if (H_k > 0) {
    a.k = static_cast<const __bf16*>(k);
    a.k_out = static_cast<__bf16*>(k_out);
    a.k_token = s[2]; a.k_head = s[3]; a.ko_token = s[6]; a.ko_head = s[7];
    on16 = on16 && aligned(k, 16) && aligned(k_out, 16) && (s[2] | s[3] | s[6] | s[7]) % 8 == 0;
  }
  a.T = (int)tokens; a.H = H; a.Hk = H_k; a.d = d; a.rot = rot;
  a.positions = positions; a.n_axes = n_axes;
  a.cu = cu_seqlens; a.n_seq = n_seq;
  a.freq = freq;
  a.factor = factor;
  a.sign = backward ? -1.f : 1.f;
  a.copies = rot < d && !(in_place_q && (in_place_k || H_k == 0));
  DeviceInfo* di = device_info();
  if (!di) return KNAP_ERR_LAUNCH_FAILED;
  const hipError_t e = knap::launch_rope(a, half, on16, di->cus, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

// type codes, strides and pointers of one tensor of rows
bool rows_ok(const void* p, int type, int64_t stride, int width) {
  return p && aligned(p, type == KNAP_BF16 ? 2 : 4) && stride >= width && stride <= ((int64_t)1 << 30);
}
// whether 16-byte accesses reach every row; rows further apart than 2^22 columns take the other form, whose offsets count one row alone
bool rows_wide(const void* p, int64_t stride, int64_t rows) { return aligned(p, 16) && (rows == 1 || (stride % 8 == 0 && stride <= (1 << 22))); }
bool type_ok(int type) { return type == KNAP_BF16 || type == KNAP_F32; }

}  // namespace

int knap_rope_fwd(const void* q, const void* k, int64_t tokens, int H, int H_k, int d, const int64_t* strides, int rot, int layout,
                  const int32_t* positions, int n_axes, const int* axis_pairs, const int32_t* cu_seqlens, int n_seq,
                  const double* freq, float factor, void* q_out, void* k_out, void* stream) {
  return rope_impl(q, k, tokens, H, H_k, d, strides, rot, layout, positions, n_axes, axis_pairs, cu_seqlens, n_seq, freq, factor, q_out,
                   k_out, false, stream);
}

int knap_rope_bwd(const void* dq_out, const void* dk_out, int64_t tokens, int H, int H_k, int d, const int64_t* strides, int rot,
                  int layout, const int32_t* positions, int n_axes, const int* axis_pairs, const int32_t* cu_seqlens, int n_seq,
                  const double* freq, float factor, void* dq, void* dk, void* stream) {
  return rope_impl(dq_out, dk_out, tokens, H, H_k, d, strides, rot, layout, positions, n_axes, axis_pairs, cu_seqlens, n_seq, freq, factor,
                   dq, dk, true, stream);
}

// ---------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------

int knap_layer_norm_fwd(const void* x, int x_type, int64_t x_stride, int64_t rows, int width, const void* weight, const void* bias,
                        int w_type, float eps, void* y, int y_type, int64_t y_stride, float* mean, float* rstd, void* stream) {
  if (!type_ok(x_type) || !type_ok(y_type) || !type_ok(w_type) || (x_type == KNAP_BF16 && y_type == KNAP_F32)) return KNAP_ERR_INVALID_ARG;
  if (rows < 0 || rows > INT32_MAX || width < 1 || width > KNAP_LAYER_NORM_MAX_WIDTH || !(eps >= 0.f) || !(eps < 3.0e38f)) return KNAP_ERR_INVALID_ARG;
  if (rows == 0) return KNAP_OK;
  if (rows == 1) x_stride = y_stride = width;
  if (!rows_ok(x, x_type, x_stride, width) || !rows_ok(y, y_type, y_stride, width) || x == y) return KNAP_ERR_INVALID_ARG;
  const size_t w_align = w_type == KNAP_BF16 ? 2 : 4;
  if (!aligned(weight, w_align) || !aligned(bias, w_align) || !aligned(mean, 4) || !aligned(rstd, 4)) return KNAP_ERR_INVALID_ARG;
  knap::NormArgs a{};
  a.x = x; a.weight = weight; a.bias = bias; a.y = y;
  a.mean = mean; a.rstd = rstd;
  a.x_stride = x_stride; a.y_stride = y_stride; a.rows = rows;
  a.width = width; a.eps = eps; a.w_bf16 = w_type == KNAP_BF16;
  DeviceInfo* di = device_info();
  if (!di) return KNAP_ERR_LAUNCH_FAILED;
  const bool wide = width % 8 == 0 && rows_wide(x, x_stride, rows) && rows_wide(y, y_stride, rows);
  const hipError_t e = knap::launch_layer_norm_fwd(a, x_type == KNAP_BF16, y_type == KNAP_BF16, wide, di->cus, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

size_t knap_layer_norm_bwd_workspace_bytes(int64_t rows, int width) {
  if (rows <= 0 || width <= 0) return 0;
  const size_t groups = rows < knap::kNormMaxGroups ? (size_t)rows : (size_t)knap::kNormMaxGroups;
  return round_up(groups * 2 * (size_t)width * sizeof(float), 256);
}

int knap_layer_norm_bwd(const void* x, int x_type, int64_t x_stride, int64_t rows, int width, const void* weight, int w_type,
                        const float* mean, const float* rstd, const void* dy, int y_type, int64_t dy_stride, void* dx, int64_t dx_stride,
                        float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!type_ok(x_type) || !type_ok(y_type) || !type_ok(w_type) || (x_type == KNAP_BF16 && y_type == KNAP_F32)) return KNAP_ERR_INVALID_ARG;
  if (rows < 0 || rows > INT32_MAX || width < 1 || width > KNAP_LAYER_NORM_MAX_WIDTH) return KNAP_ERR_INVALID_ARG;
  if (!aligned(dweight, 4) || !aligned(dbias, 4) || (dweight && dweight == dbias)) return KNAP_ERR_INVALID_ARG;
  const bool sums = dweight || dbias;
  hipError_t e;
  if (rows == 0) {
    if (!sums) return KNAP_OK;
    e = knap::launch_layer_norm_zero(dweight, dbias, width, static_cast<hipStream_t>(stream));
  } else {
    if (rows == 1) x_stride = dy_stride = dx_stride = width;
    if (!rows_ok(x, x_type, x_stride, width) || !rows_ok(dy, y_type, dy_stride, width) ||
        !rows_ok(dx, x_type, dx_stride, width) || dx == x || dx == dy)
      return KNAP_ERR_INVALID_ARG;
    if (!mean || !rstd || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(weight, w_type == KNAP_BF16 ? 2 : 4)) return KNAP_ERR_INVALID_ARG;
    if (sums) {
      if (!workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
      if (workspace_bytes < knap_layer_norm_bwd_workspace_bytes(rows, width)) return KNAP_ERR_WORKSPACE_TOO_SMALL;
    }
    knap::NormArgs a{};
    a.x = x; a.weight = weight; a.dy = dy; a.dx = dx;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.partial = sums ? static_cast<float*>(workspace) : nullptr;
    a.x_stride = x_stride; a.y_stride = dy_stride; a.dx_stride = dx_stride; a.rows = rows;
    a.width = width; a.w_bf16 = w_type == KNAP_BF16;
    DeviceInfo* di = device_info();
    if (!di) return KNAP_ERR_LAUNCH_FAILED;
    const bool wide = width % 8 == 0 && rows_wide(x, x_stride, rows) && rows_wide(dy, dy_stride, rows) && rows_wide(dx, dx_stride, rows);
    e = knap::launch_layer_norm_bwd(a, dweight, dbias, x_type == KNAP_BF16, y_type == KNAP_BF16, wide, di->cus, static_cast<hipStream_t>(stream));
  }
  if (e != hipSuccess) { g_last_hip_error = static_cast<int>(e); return KNAP_ERR_LAUNCH_FAILED; }
  return KNAP_OK;
}

const char* knap_strerror(int code) {
  switch (code) {
    case KNAP_OK: return "success";
    case KNAP_ERR_INVALID_ARG: return "invalid argument";
    case KNAP_ERR_WORKSPACE_TOO_SMALL: return "workspace too small";
    case KNAP_ERR_LAUNCH_FAILED: return "kernel launch failed";
    case KNAP_ERR_TOO_MANY_SEQS: return "too many sequences in one bag";
    case KNAP_ERR_CAPACITY: return "output array too small";
    case KNAP_ERR_PARSE: return "malformed topology string";
    case KNAP_ERR_SCRATCH_TOO_SMALL: return "bag exceeds the library's own scratch (KNAP_NOALLOC_MAX_ROWS)";
    default: return "unknown error";
  }
}

int knap_last_hip_error(void) { return g_last_hip_error; }

void knap_bwd_profile_events(void* start, void* stop) {
  g_prof_start = static_cast<hipEvent_t>(start);
  g_prof_stop = static_cast<hipEvent_t>(stop);
}

int knap_launch_workgroups(int which) {
  DeviceInfo* di = device_info();
  if (!di) return -1;
  switch (which) {
    case 0: return di->cus * di->fwd_wg[1];
    case 1: return di->cus * knap::dkdv_workgroups_per_cu(128, 4);
    case 3: return di->cus * di->fwd_wg[0];
    case 4: return di->cus * knap::dkdv_workgroups_per_cu(64, 2);
    case 5: return di->cus * di->dq_wg[0];
    default: return di->cus * di->dq_wg[1];
  }
}

unsigned* knap_fwd_queue_counters(int* count) {
  DeviceInfo* di = device_info();
  if (!di) return nullptr;
  *count = 8 * knap::kQueueSets;
  return di->queues;
}

}  // extern "C"
