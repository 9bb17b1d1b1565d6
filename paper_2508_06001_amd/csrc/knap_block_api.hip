// C-ABI entry points of the operators between the attention calls of a block and behind its backward: argument checks and launches.
// Nothing here allocates device memory, frees or synchronises.
#include "knapattn.h"
#include "knap_kernels.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdlib>

namespace {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline size_t size_of(int type) { return type == KNAP_BF16 ? 2 : 4; }
inline bool type_ok(int type) { return type == KNAP_BF16 || type == KNAP_F32; }
inline bool finite_f(float x) { return x > -3.0e38f && x < 3.0e38f; }

// a tensor of rows that is given, and whether 16-byte accesses reach every row of it (rows further apart than 2^22 columns take the other
// form, whose offsets count one row alone)
struct Rows {
  bool ok = true, wide = true;
  int64_t rows;
  int width;
  void add(const void* p, int type, int64_t stride) {
    if (!p) return;
    if (rows == 1) stride = width;
    ok = ok && aligned(p, size_of(type)) && stride >= width && stride <= ((int64_t)1 << 30);
    wide = wide && aligned(p, 16) && (rows == 1 || (stride % 8 == 0 && stride <= (1 << 22)));
  }
};

// what both directions of the residual norm check alike
int check_residual(const void* x, int x_type, int64_t rows, int width, const void* f, int branch_type, const int32_t* cu, int n_seq,
                   const void* gate, int64_t gate_stride, const void* scale, const void* shift, int64_t mod_stride, int mod_type,
                   const void* post_weight, const void* weight, int w_type, int post_norm, int norm, float alpha) {
  if (!type_ok(x_type) || !type_ok(branch_type) || !type_ok(mod_type) || !type_ok(w_type) || (x_type == KNAP_BF16 && branch_type == KNAP_F32)) return KNAP_ERR_INVALID_ARG;
  if (rows < 0 || rows > INT32_MAX || width < 1 || width > KNAP_LAYER_NORM_MAX_WIDTH || n_seq < 0) return KNAP_ERR_INVALID_ARG;
  if (n_seq > KNAP_MAX_SEQS) return KNAP_ERR_TOO_MANY_SEQS;
  if (!cu && n_seq != 1) return KNAP_ERR_INVALID_ARG;
  if (post_norm < KNAP_NORM_NONE || post_norm > KNAP_NORM_LAYER || norm < KNAP_NORM_NONE || norm > KNAP_NORM_LAYER || !finite_f(alpha)) return KNAP_ERR_INVALID_ARG;
  const bool branch = f || rows == 0;      // no rows: no tensors either
  if (!branch && (gate || post_weight || post_norm != KNAP_NORM_NONE || norm == KNAP_NORM_NONE)) return KNAP_ERR_INVALID_ARG;
  if (norm == KNAP_NORM_NONE && (weight || scale || shift)) return KNAP_ERR_INVALID_ARG;
  if (n_seq > 1 && ((gate && (gate_stride < 0 || gate_stride > ((int64_t)1 << 40))) || ((scale || shift) && (mod_stride < 0 || mod_stride > ((int64_t)1 << 40)))))
    return KNAP_ERR_INVALID_ARG;
  if (!aligned(cu, 4) || !aligned(gate, size_of(mod_type)) || !aligned(scale, size_of(mod_type)) || !aligned(shift, size_of(mod_type)) ||
      !aligned(weight, size_of(w_type)) || !aligned(post_weight, size_of(w_type)))
    return KNAP_ERR_INVALID_ARG;
  if (rows > 0 && !x) return KNAP_ERR_INVALID_ARG;
  return KNAP_OK;
}

}  // namespace

extern "C" {

// ---------------------------------------------------------------------------
// Residual norm
// ---------------------------------------------------------------------------

int knap_residual_norm_fwd(const void* x, int x_type, int64_t x_stride, int64_t rows, int width, const void* f, int branch_type, int64_t f_stride,
                           const int32_t* cu_seqlens, int n_seq, const void* gate, int64_t gate_stride, const void* scale, const void* shift,
                           int64_t mod_stride, int mod_type, const void* post_weight, const void* weight, int w_type, int post_norm, int norm,
                           float alpha, float eps, void* x_out, int64_t x_out_stride, void* y, int64_t y_stride, float* stats, void* stream) {
  const int rc = check_residual(x, x_type, rows, width, f, branch_type, cu_seqlens, n_seq, gate, gate_stride, scale, shift, mod_stride, mod_type,
                                post_weight, weight, w_type, post_norm, norm, alpha);
  if (rc != KNAP_OK) return rc;
  if (!(eps >= 0.f) || !finite_f(eps)) return KNAP_ERR_INVALID_ARG;
  if (rows == 0 || n_seq == 0) return KNAP_OK;
  if (!!f != !!x_out || (norm != KNAP_NORM_NONE) != !!y || !aligned(stats, 4)) return KNAP_ERR_INVALID_ARG;
  Rows t;
  t.rows = rows; t.width = width;
  t.add(x, x_type, x_stride);
  t.add(f, branch_type, f_stride);
  t.add(x_out, x_type, x_out_stride);
  t.add(y, branch_type, y_stride);
  if (!t.ok || x == y || f == x || (f && (f == x_out || f == y)) || (y && y == x_out)) return KNAP_ERR_INVALID_ARG;
  if (x == x_out && rows > 1 && x_stride != x_out_stride) return KNAP_ERR_INVALID_ARG;
  knap::ResidualArgs a{};
  a.x = x; a.f = f; a.gate = gate; a.scale = scale; a.shift = shift; a.weight = weight; a.post_weight = post_weight;
  a.cu = cu_seqlens; a.n_seq = n_seq;
  a.x_out = x_out; a.y = y; a.stats = stats;
  a.x_stride = rows == 1 ? width : x_stride; a.f_stride = rows == 1 ? width : f_stride;
  a.x_out_stride = rows == 1 ? width : x_out_stride; a.y_stride = rows == 1 ? width : y_stride;
  a.gate_stride = n_seq == 1 ? 0 : gate_stride; a.mod_stride = n_seq == 1 ? 0 : mod_stride;
  a.rows = rows; a.width = width; a.alpha = alpha; a.eps = eps; a.norm = norm; a.post_norm = post_norm;
  a.w_bf16 = w_type == KNAP_BF16; a.mod_bf16 = mod_type == KNAP_BF16;
  const int cus = knap::device_cus();
  if (!cus) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_residual_norm_fwd(a, x_type == KNAP_BF16, branch_type == KNAP_BF16, width % 8 == 0 && t.wide, cus,
                                                            static_cast<hipStream_t>(stream)));
}

size_t knap_residual_norm_bwd_workspace_bytes(int64_t rows, int width, int n_seq) {
  if (rows <= 0 || width <= 0 || n_seq <= 0) return 0;
  const size_t groups = (size_t)std::min<int64_t>(rows, knap::kResidualMaxGroups);
  return round_up(((groups + n_seq) * 3 + groups * 2) * (size_t)width * sizeof(float), 256);
}

int knap_residual_norm_bwd(const void* x, int x_type, int64_t x_stride, int64_t rows, int width, const void* f, int branch_type, int64_t f_stride,
                           const int32_t* cu_seqlens, int n_seq, const void* gate, int64_t gate_stride, const void* scale, int64_t mod_stride,
                           int mod_type, const void* post_weight, const void* weight, int w_type, int post_norm, int norm, float alpha,
                           const float* stats, const void* dx_out, int64_t dx_out_stride, const void* dy, int64_t dy_stride, void* dx,
                           int64_t dx_stride, void* df, int64_t df_stride, float* dgate, int64_t dgate_stride, float* dscale, float* dshift,
                           int64_t dmod_stride, float* dweight, float* dpost_weight, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_residual(x, x_type, rows, width, f, branch_type, cu_seqlens, n_seq, gate, gate_stride, scale, nullptr, mod_stride, mod_type,
                                post_weight, weight, w_type, post_norm, norm, alpha);
  if (rc != KNAP_OK) return rc;
  const bool none = rows == 0 || n_seq == 0;
  const bool sums = dgate || dscale || dshift || dweight || dpost_weight;
  float* const outs[5] = {dgate, dscale, dshift, dweight, dpost_weight};
  for (int i = 0; i < 5; ++i) {
    if (!aligned(outs[i], 4)) return KNAP_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return KNAP_ERR_INVALID_ARG;
  }
  if (n_seq > 1 && ((dgate && dgate_stride < width) || ((dscale || dshift) && dmod_stride < width))) return KNAP_ERR_INVALID_ARG;
  knap::ResidualArgs a{};
  a.cu = cu_seqlens; a.n_seq = n_seq;
  a.rows = none ? 0 : rows; a.width = width; a.alpha = alpha; a.norm = norm; a.post_norm = post_norm;
  a.w_bf16 = w_type == KNAP_BF16; a.mod_bf16 = mod_type == KNAP_BF16;
  a.gate = gate; a.scale = scale; a.weight = weight; a.post_weight = post_weight;
  a.gate_stride = n_seq == 1 ? 0 : gate_stride; a.mod_stride = n_seq == 1 ? 0 : mod_stride;
  a.dgate = dgate; a.dscale = dscale; a.dshift = dshift; a.dweight = dweight; a.dpost_weight = dpost_weight;
  a.dgate_stride = n_seq == 1 ? 0 : dgate_stride; a.dmod_stride = n_seq == 1 ? 0 : dmod_stride;
  Rows t;
  t.rows = rows; t.width = width;
  if (!none) {
    const bool normed = norm != KNAP_NORM_NONE;
    if (normed != !!dy || (df && !f) || (!f && (dgate || dpost_weight)) || (!normed && (dscale || dshift || dweight))) return KNAP_ERR_INVALID_ARG;
    if ((normed || post_norm != KNAP_NORM_NONE) && (!stats || !aligned(stats, 4))) return KNAP_ERR_INVALID_ARG;
    t.add(x, x_type, x_stride);
    t.add(f, branch_type, f_stride);
    t.add(dx_out, x_type, dx_out_stride);
    t.add(dy, branch_type, dy_stride);
    t.add(dx, x_type, dx_stride);
    t.add(df, branch_type, df_stride);
    if (!t.ok || f == x) return KNAP_ERR_INVALID_ARG;
    if (dx && (dx == x || dx == f || dx == dy || dx == df || (dx == dx_out && rows > 1 && dx_stride != dx_out_stride))) return KNAP_ERR_INVALID_ARG;
    if (df && (df == x || df == f || df == dy || df == dx_out)) return KNAP_ERR_INVALID_ARG;
    if (sums) {
      if (!workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
      if (workspace_bytes < knap_residual_norm_bwd_workspace_bytes(rows, width, n_seq)) return KNAP_ERR_WORKSPACE_TOO_SMALL;
      const size_t groups = (size_t)std::min<int64_t>(rows, knap::kResidualMaxGroups);
      a.partial = static_cast<float*>(workspace);
      a.totals = dweight || dpost_weight ? a.partial + (groups + n_seq) * 3 * (size_t)width : nullptr;
    }
    a.x = x; a.f = f; a.dx_out = dx_out; a.dy = dy; a.dx = dx; a.df = df;
    a.stats = const_cast<float*>(stats);
    a.x_stride = rows == 1 ? width : x_stride; a.f_stride = rows == 1 ? width : f_stride;
    a.dx_out_stride = rows == 1 ? width : dx_out_stride; a.dy_stride = rows == 1 ? width : dy_stride;
    a.dx_stride = rows == 1 ? width : dx_stride; a.df_stride = rows == 1 ? width : df_stride;
  }
  if (none && !sums) return KNAP_OK;
  const int cus = knap::device_cus();
  if (!cus) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_residual_norm_bwd(a, x_type == KNAP_BF16, branch_type == KNAP_BF16, width % 8 == 0 && t.wide, cus,
                                                            static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// Gated feed-forward
// ---------------------------------------------------------------------------

}  // extern "C"

namespace {

constexpr int64_t kFfnMostTokens = (int64_t)1 << 26;
constexpr int64_t kFfnMostElements = (int64_t)1 << 37;      // of x or h: what a launch's workgroups cover (launch_gemm)

bool ffn_sizes(int64_t tokens, int width, int hidden) {
  return tokens <= kFfnMostTokens && width <= KNAP_FFN_MAX_WIDTH && hidden <= KNAP_FFN_MAX_WIDTH && tokens * std::max(width, hidden) <= kFfnMostElements;
}
int check_ffn(int64_t tokens, int width, int hidden, const void* w_gate, const void* w_up, const void* w_down, int act) {
  if (tokens < 0 || width < 8 || width % 8 || hidden < 8 || hidden % 8 || !ffn_sizes(tokens, width, hidden)) return KNAP_ERR_INVALID_ARG;
  if (act != KNAP_SILU && act != KNAP_GELU_TANH) return KNAP_ERR_INVALID_ARG;
  if (tokens > 0 && (!w_gate || !w_up || !w_down || !aligned(w_gate, 16) || !aligned(w_up, 16) || !aligned(w_down, 16))) return KNAP_ERR_INVALID_ARG;
  return KNAP_OK;
}
bool ffn_rows(const void* p, int64_t stride, int64_t rows, int width) {
  return p && aligned(p, 16) && (rows == 1 || (stride >= width && stride % 8 == 0 && stride <= (1 << 20)));
}
size_t ffn_hidden_bytes(int64_t tokens, int hidden) { return round_up((size_t)tokens * hidden * 2, 256); }

}  // namespace

extern "C" {

size_t knap_gated_ffn_fwd_workspace_bytes(int64_t tokens, int width, int hidden) {
  if (tokens <= 0 || width <= 0 || hidden <= 0 || !ffn_sizes(tokens, width, hidden)) return 0;
  return round_up(knap::ffn_partial_bytes(tokens, width, hidden, false), 256);
}

size_t knap_gated_ffn_bwd_workspace_bytes(int64_t tokens, int width, int hidden) {
  if (tokens <= 0 || width <= 0 || hidden <= 0 || !ffn_sizes(tokens, width, hidden)) return 0;
  return 2 * ffn_hidden_bytes(tokens, hidden) + round_up(knap::ffn_partial_bytes(tokens, width, hidden, true), 256);
}

int knap_gated_ffn_fwd(const void* x, int64_t x_stride, int64_t tokens, int width, int hidden, const void* w_gate, const void* w_up, const void* w_down,
                       int act, void* gate, void* up, void* h, void* y, int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_ffn(tokens, width, hidden, w_gate, w_up, w_down, act);
  if (rc != KNAP_OK) return rc;
  if (tokens == 0) return KNAP_OK;
  if (!ffn_rows(x, x_stride, tokens, width) || !ffn_rows(y, y_stride, tokens, width) || !h || !aligned(h, 16) || !gate != !up || !aligned(gate, 16) ||
      !aligned(up, 16))
    return KNAP_ERR_INVALID_ARG;
  if (x == y || x == h || y == h || (gate && (gate == up || gate == h || up == h || gate == x || up == x || gate == y || up == y))) return KNAP_ERR_INVALID_ARG;
  const size_t need = knap_gated_ffn_fwd_workspace_bytes(tokens, width, hidden);
  if ((need && !workspace) || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
  if (workspace_bytes < need) return KNAP_ERR_WORKSPACE_TOO_SMALL;
  knap::FfnArgs a{};
  a.x = static_cast<const __bf16*>(x);
  a.w_gate = static_cast<const __bf16*>(w_gate); a.w_up = static_cast<const __bf16*>(w_up); a.w_down = static_cast<const __bf16*>(w_down);
  a.x_stride = tokens == 1 ? width : x_stride; a.y_stride = tokens == 1 ? width : y_stride;
  a.tokens = (int)tokens; a.width = width; a.hidden = hidden; a.gelu = act == KNAP_GELU_TANH;
  a.gate = static_cast<__bf16*>(gate); a.up = static_cast<__bf16*>(up); a.h = static_cast<__bf16*>(h); a.y = static_cast<__bf16*>(y);
  a.partial = static_cast<float*>(workspace);
  if (!knap::device_cus()) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_ffn_fwd(a, static_cast<hipStream_t>(stream)));
}

int knap_gated_ffn_bwd(const void* x, int64_t x_stride, int64_t tokens, int width, int hidden, const void* w_gate, const void* w_up, const void* w_down,
                       int act, const void* gate, const void* up, const void* h, const void* dy, int64_t dy_stride, void* dx, int64_t dx_stride,
                       void* dw_gate, void* dw_up, void* dw_down, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = check_ffn(tokens, width, hidden, w_gate, w_up, w_down, act);
  if (rc != KNAP_OK) return rc;
  void* const outs[4] = {dx, dw_gate, dw_up, dw_down};
  const void* const ins[6] = {x, gate, up, h, dy, workspace};
  for (int i = 0; i < 4; ++i) {
    if (!aligned(outs[i], 16)) return KNAP_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (outs[i] && outs[i] == outs[j]) return KNAP_ERR_INVALID_ARG;
    for (const void* in : ins)
      if (outs[i] && tokens > 0 && outs[i] == in) return KNAP_ERR_INVALID_ARG;
    if (outs[i] && tokens > 0 && (outs[i] == w_gate || outs[i] == w_up || outs[i] == w_down)) return KNAP_ERR_INVALID_ARG;
  }
  if (tokens > 0) {
    if (!ffn_rows(x, x_stride, tokens, width) || !ffn_rows(dy, dy_stride, tokens, width) || (dx && !ffn_rows(dx, dx_stride, tokens, width)))
      return KNAP_ERR_INVALID_ARG;
    if (!gate || !up || !h || !aligned(gate, 16) || !aligned(up, 16) || !aligned(h, 16)) return KNAP_ERR_INVALID_ARG;
    if (!workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
    if (workspace_bytes < knap_gated_ffn_bwd_workspace_bytes(tokens, width, hidden)) return KNAP_ERR_WORKSPACE_TOO_SMALL;
  } else if (!dw_gate && !dw_up && !dw_down) {
    return KNAP_OK;
  }
  knap::FfnArgs a{};
  a.x = static_cast<const __bf16*>(x); a.dy = static_cast<const __bf16*>(dy);
  a.w_gate = static_cast<const __bf16*>(w_gate); a.w_up = static_cast<const __bf16*>(w_up); a.w_down = static_cast<const __bf16*>(w_down);
  a.x_stride = tokens == 1 ? width : x_stride; a.dy_stride = tokens == 1 ? width : dy_stride; a.dx_stride = tokens == 1 ? width : dx_stride;
  a.tokens = (int)tokens; a.width = width; a.hidden = hidden; a.gelu = act == KNAP_GELU_TANH;
  a.gate = const_cast<__bf16*>(static_cast<const __bf16*>(gate)); a.up = const_cast<__bf16*>(static_cast<const __bf16*>(up));
  a.h = const_cast<__bf16*>(static_cast<const __bf16*>(h));
  a.dx = static_cast<__bf16*>(dx);
  a.dw_gate = static_cast<__bf16*>(dw_gate); a.dw_up = static_cast<__bf16*>(dw_up); a.dw_down = static_cast<__bf16*>(dw_down);
  if (tokens > 0) {
    char* ws = static_cast<char*>(workspace);
    const size_t each = ffn_hidden_bytes(tokens, hidden);
    a.dgate = reinterpret_cast<__bf16*>(ws);
    a.dup = reinterpret_cast<__bf16*>(ws + each);
    a.partial = reinterpret_cast<float*>(ws + 2 * each);
  }
  if (!knap::device_cus()) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_ffn_bwd(a, static_cast<hipStream_t>(stream)));
}

// ---------------------------------------------------------------------------
// Gradient norm and clipping
// ---------------------------------------------------------------------------

}  // extern "C"

namespace {

constexpr int64_t kGradMost = (int64_t)1 << 40;      // elements of a tensor

// Whether every part of `out` is apart from the others and from all gradients but its own.  In ascending order, as tensors of one
// allocation mostly are, one walk does; else an array of their order is sorted.
int grads_apart(const void* const* grads, void* const* out, const int64_t* numel, const int* types, int n) {
  struct Span { uintptr_t from, to; int i; };
  constexpr int kOnStack = 512;
  Span some[kOnStack], *spans = some;
  if (n > kOnStack) {
    spans = static_cast<Span*>(malloc((size_t)n * sizeof(Span)));
    if (!spans) return KNAP_ERR_CAPACITY;
  }
  int m = 0;
  bool in_place = true, sorted = true;
  for (int i = 0; i < n; ++i) {
    if (numel[i] == 0) continue;
    const uintptr_t at = reinterpret_cast<uintptr_t>(out[i]);
    spans[m] = {at, at + (size_t)numel[i] * size_of(types[i]), i};
    sorted = sorted && (m == 0 || spans[m - 1].from <= at);
    in_place = in_place && grads[i] == out[i];
    ++m;
  }
  if (!sorted) std::sort(spans, spans + m, [](const Span& a, const Span& b) { return a.from < b.from; });
  bool ok = true;
  for (int k = 1; k < m && ok; ++k) ok = spans[k - 1].to <= spans[k].from;
  if (ok && !in_place)
    for (int i = 0; i < n && ok; ++i) {
      if (numel[i] == 0) continue;
      const uintptr_t from = reinterpret_cast<uintptr_t>(grads[i]), to = from + (size_t)numel[i] * size_of(types[i]);
      // the parts of `out` do not overlap, so that their ends ascend too: the first that ends behind `from`
      const Span* s = std::upper_bound(spans, spans + m, from, [](uintptr_t v, const Span& x) { return v < x.to; });
      for (; s < spans + m && s->from < to && ok; ++s) ok = s->i == i && s->from == from;
    }
  if (spans != some) free(spans);
  return ok ? KNAP_OK : KNAP_ERR_INVALID_ARG;
}

}  // namespace

extern "C" {

size_t knap_grad_plan_bytes(const int64_t* numel, int n) {
  size_t chunks = 0;
  for (int i = 0; numel && i < n; ++i)
    if (numel[i] > 0 && numel[i] < kGradMost) chunks += (size_t)((numel[i] + KNAP_GRAD_CHUNK - 1) / KNAP_GRAD_CHUNK);
  return chunks * sizeof(knap::GradChunk);
}

int knap_grad_plan(const void* const* grads, void* const* out, const int64_t* numel, const int* types, int n, void* plan, size_t plan_bytes) {
  if (n < 0 || (n > 0 && (!grads || !out || !numel || !types))) return KNAP_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i) {
    if (!type_ok(types[i]) || numel[i] < 0 || numel[i] >= kGradMost) return KNAP_ERR_INVALID_ARG;
    if (numel[i] > 0 && (!grads[i] || !out[i] || !aligned(grads[i], size_of(types[i])) || !aligned(out[i], size_of(types[i])))) return KNAP_ERR_INVALID_ARG;
  }
  const int apart = grads_apart(grads, out, numel, types, n);
  if (apart != KNAP_OK) return apart;
  const size_t need = knap_grad_plan_bytes(numel, n);
  if (need == 0) return KNAP_OK;
  if (!plan || !aligned(plan, 8)) return KNAP_ERR_INVALID_ARG;
  if (plan_bytes < need) return KNAP_ERR_CAPACITY;
  knap::GradChunk* to = static_cast<knap::GradChunk*>(plan);
  for (int i = 0; i < n; ++i)
    for (int64_t at = 0; at < numel[i]; at += KNAP_GRAD_CHUNK) {
      const size_t bytes = (size_t)at * size_of(types[i]);
      *to++ = knap::GradChunk{static_cast<const char*>(grads[i]) + bytes, static_cast<char*>(out[i]) + bytes,
                              (int32_t)std::min<int64_t>(KNAP_GRAD_CHUNK, numel[i] - at), types[i] == KNAP_BF16};
    }
  return KNAP_OK;
}

static bool plan_ok(const void* plan, size_t plan_bytes) {
  return plan_bytes % sizeof(knap::GradChunk) == 0 && (plan_bytes == 0 || (plan && aligned(plan, 8)));
}

int knap_grad_sum_squares(const void* plan, size_t plan_bytes, double* sum_sq, void* workspace, size_t workspace_bytes, void* stream) {
  if (!plan_ok(plan, plan_bytes) || !sum_sq || !aligned(sum_sq, 8) || !workspace || !aligned(workspace, 256)) return KNAP_ERR_INVALID_ARG;
  if (workspace_bytes < KNAP_GRAD_WORKSPACE_BYTES) return KNAP_ERR_WORKSPACE_TOO_SMALL;
  const int cus = knap::device_cus();
  if (!cus) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_grad_squares(static_cast<const knap::GradChunk*>(plan), (int64_t)(plan_bytes / sizeof(knap::GradChunk)),
                                                       static_cast<double*>(workspace), sum_sq, cus, static_cast<hipStream_t>(stream)));
}

int knap_grad_clip(const void* plan, size_t plan_bytes, const double* sum_sq, float max_norm, float eps, float* norm, void* stream) {
  if (!plan_ok(plan, plan_bytes) || !sum_sq || !aligned(sum_sq, 8) || !aligned(norm, 4) || !(max_norm > 0.f) || !(eps >= 0.f) || !finite_f(eps))
    return KNAP_ERR_INVALID_ARG;
  if (plan_bytes == 0 && !norm) return KNAP_OK;
  const int cus = knap::device_cus();
  if (!cus) return KNAP_ERR_LAUNCH_FAILED;
  return knap::launch_status(knap::launch_grad_clip(static_cast<const knap::GradChunk*>(plan), (int64_t)(plan_bytes / sizeof(knap::GradChunk)), sum_sq,
                                                    max_norm, eps, norm, cus, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
