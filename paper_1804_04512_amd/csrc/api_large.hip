// C ABI of the large-model operators: argument checks, workspace sizes, the launch sequences' arguments.
#include "../../include/dll_conv.h"
#include "large_ops.h"

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <new>

using namespace dllk;

namespace {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
// labels, losses and norms: 32-bit values at any place of theirs
inline bool off_element(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }
inline dll_status dev(hipError_t e) { return e == hipSuccess ? DLL_OK : DLL_ERR_DEVICE; }

dll_status check_ws(const void *ws, size_t have, size_t need) {
  if (!ws || (reinterpret_cast<uintptr_t>(ws) & (kAlign - 1))) return DLL_ERR_WORKSPACE;
  return have >= need ? DLL_OK : DLL_ERR_WORKSPACE;
}

// Whether any of the outputs is one of the inputs or another output (exact equality; NULLs apart)
bool aliased(const void *const *in, int n_in, const void *const *out, int n_out) {
  for (int o = 0; o < n_out; ++o) {
    if (!out[o]) continue;
    for (int i = 0; i < n_in; ++i)
      if (out[o] == in[i]) return true;
    for (int i = 0; i < o; ++i)
      if (out[o] == out[i]) return true;
  }
  return false;
}

constexpr int kMaxTokens = 1 << 24, kMaxFeatures = 1 << 20;
constexpr size_t kMaxElements = (size_t)1 << 31;

dll_status check_sizes(int tokens, int width, int rows, int dtype) {
  if (tokens <= 0 || width <= 0 || rows <= 0) return DLL_ERR_SHAPE;
  if (dtype != DLL_FP32 && dtype != DLL_BF16) return DLL_ERR_UNSUPPORTED;
  if (tokens > kMaxTokens || width > kMaxFeatures || rows > kMaxFeatures) return DLL_ERR_UNSUPPORTED;
  if ((size_t)tokens * width >= kMaxElements || (size_t)rows * width >= kMaxElements) return DLL_ERR_UNSUPPORTED;
  return DLL_OK;
}

dll_status check_gated(const dll_gated_desc *d) {
  if (!d) return DLL_ERR_NULL;
  const dll_status st = check_sizes(d->tokens, d->width, d->hidden, d->dtype);
  if (st != DLL_OK) return st;
  if (d->gate < DLL_GATE_IDENTITY || d->gate > DLL_GATE_GELU) return DLL_ERR_UNSUPPORTED;
  return (size_t)d->tokens * d->hidden >= kMaxElements ? DLL_ERR_UNSUPPORTED : DLL_OK;
}

dll_status check_vocab(const dll_vocab_desc *d) {
  if (!d) return DLL_ERR_NULL;
  return check_sizes(d->tokens, d->width, d->classes, d->dtype);
}

// counts and types, the gradients behind them
dll_status check_list(const dll_tensor_list *l, const void *const *grads, bool with_grads) {
  if (!l || !l->counts || !l->dtypes) return DLL_ERR_NULL;
  if (l->n <= 0) return DLL_ERR_SHAPE;
  if (with_grads && !grads) return DLL_ERR_NULL;
  for (int i = 0; i < l->n; ++i) {
    if (l->dtypes[i] != DLL_FP32 && l->dtypes[i] != DLL_BF16) return DLL_ERR_UNSUPPORTED;
    if (l->counts[i] >= ((size_t)1 << 40)) return DLL_ERR_UNSUPPORTED;
    if (!with_grads || l->counts[i] == 0) continue;
    if (!grads[i]) return DLL_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(grads[i]) % type_bytes(l->dtypes[i])) return DLL_ERR_SHAPE;
  }
  return DLL_OK;
}

// One address of a list: of tensor `tensor`, or of the norm or the workspace (-1)
struct Place {
  uintptr_t at;
  int tensor, output;
};
// Whether the norm is no place of a 32-bit value, or an output of a list of tensors, the norm or the workspace is another of these or any tensor's gradient; with in_place an
// output may be its own.  The kernels
// take all tensors at once, so a tensor listed twice would be stepped by two workgroups that race.
dll_status check_places(const dll_tensor_list *l, const void *const *grads, const void *const *const *outs, int n_outs, const float *norm, const void *ws,
                        bool in_place) {
  if (off_element(norm)) return DLL_ERR_SHAPE;
  constexpr int kHere = 256;
  Place here[kHere];
  const size_t most = (size_t)l->n * (n_outs + 1) + 2;
  Place *const p = most <= kHere ? here : new (std::nothrow) Place[most];
  if (!p) return DLL_ERR_DEVICE;
  size_t n = 0;
  p[n++] = Place{reinterpret_cast<uintptr_t>(norm), -1, 1};
  p[n++] = Place{reinterpret_cast<uintptr_t>(ws), -1, 1};
  for (int i = 0; i < l->n; ++i) {
    if (l->counts[i] == 0) continue;
    p[n++] = Place{reinterpret_cast<uintptr_t>(grads[i]), i, 0};
    for (int k = 0; k < n_outs; ++k)
      if (outs[k] && outs[k][i]) p[n++] = Place{reinterpret_cast<uintptr_t>(outs[k][i]), i, 1};
  }
  std::sort(p, p + n, [](const Place &a, const Place &b) { return a.at < b.at; });
  bool clash = false;
  for (size_t i = 0, j; i < n && !clash; i = j) {
    int outputs = 0;
    for (j = i; j < n && p[j].at == p[i].at; ++j) outputs += p[j].output;
    const bool own = in_place && j - i == 2 && outputs == 1 && p[i].tensor == p[i + 1].tensor;
    clash = j - i > 1 && outputs > 0 && !own;
  }
  if (p != here) delete[] p;
  return clash ? DLL_ERR_SHAPE : DLL_OK;
}

GradList list_of(const dll_tensor_list *l) {
  GradList g;
  g.n = l->n;
  g.counts = l->counts;
  g.dtypes = l->dtypes;
  return g;
}

GatedArgs gated_args(const dll_gated_desc *d, const void *x, const void *w_gate, const void *w_up, const void *w_down) {
  GatedArgs a;
  a.T = d->tokens; a.D = d->width; a.H = d->hidden; a.gate = d->gate; a.dtype = d->dtype;
  a.x = x; a.w_gate = w_gate; a.w_up = w_up; a.w_down = w_down;
  return a;
}

}  // namespace

extern "C" {

size_t dll_gated_fwd_workspace_bytes(const dll_gated_desc *d) {
  return check_gated(d) == DLL_OK ? align_up(gated_fwd_scratch(d->tokens, d->width, d->hidden, d->dtype)) : 0;
}

dll_status dll_gated_fwd(const dll_gated_desc *d, const void *x, const void *w_gate, const void *w_up, const void *w_down, void *y, void *gate_pre,
                         void *up_pre, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_gated(d);
  if (st != DLL_OK) return st;
  if (!x || !w_gate || !w_up || !w_down || !y || !gate_pre != !up_pre) return DLL_ERR_NULL;
  const void *in[] = {x, w_gate, w_up, w_down}, *out[] = {y, gate_pre, up_pre, ws};
  if (aliased(in, 4, out, 4)) return DLL_ERR_SHAPE;
  for (const void *p : in)
    if (misaligned(p)) return DLL_ERR_SHAPE;
  for (int i = 0; i < 3; ++i)
    if (misaligned(out[i])) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_gated_fwd_workspace_bytes(d))) != DLL_OK) return st;
  GatedArgs a = gated_args(d, x, w_gate, w_up, w_down);
  a.y = y; a.gate_pre = gate_pre; a.up_pre = up_pre;
  return dev(launch_gated_fwd(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

size_t dll_gated_bwd_workspace_bytes(const dll_gated_desc *d) {
  return check_gated(d) == DLL_OK ? align_up(gated_bwd_scratch(d->tokens, d->width, d->hidden, d->dtype)) : 0;
}

dll_status dll_gated_bwd(const dll_gated_desc *d, const void *x, const void *w_gate, const void *w_up, const void *w_down, const void *gate_pre,
                         const void *up_pre, const void *dy, void *dx, void *dw_gate, void *dw_up, void *dw_down, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_gated(d);
  if (st != DLL_OK) return st;
  if (!x || !w_gate || !w_up || !w_down || !gate_pre || !up_pre || !dy || (!dx && !dw_gate && !dw_up && !dw_down)) return DLL_ERR_NULL;
  const void *in[] = {x, w_gate, w_up, w_down, gate_pre, up_pre, dy}, *out[] = {dx, dw_gate, dw_up, dw_down, ws};
  if (aliased(in, 7, out, 5)) return DLL_ERR_SHAPE;
  for (const void *p : in)
    if (misaligned(p)) return DLL_ERR_SHAPE;
  for (int i = 0; i < 4; ++i)
    if (misaligned(out[i])) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_gated_bwd_workspace_bytes(d))) != DLL_OK) return st;
  GatedArgs a = gated_args(d, x, w_gate, w_up, w_down);
  a.gate_pre = const_cast<void *>(gate_pre); a.up_pre = const_cast<void *>(up_pre); a.dy = dy;
  a.dx = dx; a.dw_gate = dw_gate; a.dw_up = dw_up; a.dw_down = dw_down;
  return dev(launch_gated_bwd(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

size_t dll_vocab_loss_fwd_workspace_bytes(const dll_vocab_desc *d) {
  return check_vocab(d) == DLL_OK ? align_up(vocab_fwd_scratch(d->tokens, d->width, d->classes, d->dtype)) : 0;
}

dll_status dll_vocab_loss_fwd(const dll_vocab_desc *d, const void *x, const void *w, const void *bias, const int *labels, float *row_loss, float *row_lse,
                              float *loss, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_vocab(d);
  if (st != DLL_OK) return st;
  if (!x || !w || !labels || !loss) return DLL_ERR_NULL;
  const void *in[] = {x, w, bias, labels}, *out[] = {row_loss, row_lse, loss, ws};
  if (aliased(in, 4, out, 4) || misaligned(x) || misaligned(w) || misaligned(bias)) return DLL_ERR_SHAPE;
  if (off_element(labels) || off_element(row_loss) || off_element(row_lse) || off_element(loss)) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_vocab_loss_fwd_workspace_bytes(d))) != DLL_OK) return st;
  VocabArgs a;
  a.T = d->tokens; a.D = d->width; a.V = d->classes; a.dtype = d->dtype;
  a.x = x; a.w = w; a.bias = bias; a.labels = labels;
  a.row_loss = row_loss; a.row_lse = row_lse; a.loss = loss;
  return dev(launch_vocab_fwd(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

size_t dll_vocab_loss_grad_workspace_bytes(const dll_vocab_desc *d) {
  return check_vocab(d) == DLL_OK ? align_up(vocab_grad_scratch(d->tokens, d->width, d->classes, d->dtype)) : 0;
}

dll_status dll_vocab_loss_grad(const dll_vocab_desc *d, const void *x, const void *w, const void *bias, const int *labels, float scale, float *row_loss,
                               float *row_lse, float *loss, void *dx, void *dw, void *dbias, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_vocab(d);
  if (st != DLL_OK) return st;
  if (!x || !w || !labels || !loss || (!dx && !dw && !dbias) || (dbias && !bias)) return DLL_ERR_NULL;
  const void *in[] = {x, w, bias, labels}, *out[] = {row_loss, row_lse, loss, dx, dw, dbias, ws};
  if (aliased(in, 4, out, 7) || misaligned(x) || misaligned(w) || misaligned(bias) || misaligned(dx) || misaligned(dw) || misaligned(dbias))
    return DLL_ERR_SHAPE;
  if (off_element(labels) || off_element(row_loss) || off_element(row_lse) || off_element(loss)) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_vocab_loss_grad_workspace_bytes(d))) != DLL_OK) return st;
  VocabArgs a;
  a.T = d->tokens; a.D = d->width; a.V = d->classes; a.dtype = d->dtype;
  a.x = x; a.w = w; a.bias = bias; a.labels = labels; a.scale = scale;
  a.row_loss = row_loss; a.row_lse = row_lse; a.loss = loss;
  a.dx = dx; a.dw = dw; a.dbias = dbias;
  return dev(launch_vocab_grad(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

size_t dll_grad_norm_workspace_bytes(const dll_tensor_list *list) {
  return check_list(list, nullptr, false) == DLL_OK ? align_up(grad_norm_scratch(list_of(list))) : 0;
}

dll_status dll_grad_norm(const dll_tensor_list *list, const void *const *grads, float *norm, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_list(list, grads, true);
  if (st != DLL_OK) return st;
  if (!norm) return DLL_ERR_NULL;
  if ((st = check_places(list, grads, nullptr, 0, norm, ws, false)) != DLL_OK) return st;
  if ((st = check_ws(ws, ws_bytes, dll_grad_norm_workspace_bytes(list))) != DLL_OK) return st;
  return dev(launch_grad_norm(list_of(list), grads, norm, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

dll_status dll_grad_clip(const dll_tensor_list *list, const void *const *grads, void *const *out, float max_norm, float *norm, void *ws, size_t ws_bytes,
                         void *stream) {
  dll_status st = check_list(list, grads, true);
  if (st != DLL_OK) return st;
  if (!out || !norm) return DLL_ERR_NULL;
  if (!(max_norm > 0.0f)) return DLL_ERR_SHAPE;
  for (int i = 0; i < list->n; ++i) {
    if (list->counts[i] == 0) continue;
    if (!out[i]) return DLL_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(out[i]) % type_bytes(list->dtypes[i])) return DLL_ERR_SHAPE;
  }
  const void *const *outs[] = {out};
  if ((st = check_places(list, grads, outs, 1, norm, ws, true)) != DLL_OK) return st;
  if ((st = check_ws(ws, ws_bytes, dll_grad_norm_workspace_bytes(list))) != DLL_OK) return st;
  return dev(launch_grad_clip(list_of(list), grads, out, max_norm, norm, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

dll_status dll_momentum_update_clipped(const dll_tensor_list *list, float *const *params, float *const *velocity, const void *const *grads, float lr,
                                       float momentum, const float *weight_decay, float max_norm, float *norm, void *const *copies, void *ws,
                                       size_t ws_bytes, void *stream) {
  dll_status st = check_list(list, grads, true);
  if (st != DLL_OK) return st;
  if (!params || !velocity || !norm) return DLL_ERR_NULL;
  if (!(max_norm > 0.0f)) return DLL_ERR_SHAPE;
  for (int i = 0; i < list->n; ++i) {
    if (list->counts[i] == 0) continue;
    if (!params[i] || !velocity[i]) return DLL_ERR_NULL;
    const void *copy = copies ? copies[i] : nullptr;
    if ((reinterpret_cast<uintptr_t>(params[i]) | reinterpret_cast<uintptr_t>(velocity[i])) % 4 || reinterpret_cast<uintptr_t>(copy) % 2) return DLL_ERR_SHAPE;
  }
  const void *const *outs[] = {reinterpret_cast<const void *const *>(params), reinterpret_cast<const void *const *>(velocity), copies};
  if ((st = check_places(list, grads, outs, 3, norm, ws, false)) != DLL_OK) return st;
  if ((st = check_ws(ws, ws_bytes, dll_grad_norm_workspace_bytes(list))) != DLL_OK) return st;
  return dev(launch_momentum_clipped(list_of(list), params, velocity, grads, weight_decay, lr, momentum, max_norm, norm, copies, static_cast<char *>(ws),
                                     static_cast<hipStream_t>(stream)));
}

}  // extern "C"
