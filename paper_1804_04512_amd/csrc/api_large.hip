// C ABI of the large-model operators: argument checks, workspace sizes, the launch sequences' arguments.
#include "../../include/dll_conv.h"
#include "large_ops.h"

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
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

// rows of `heads` heads: contiguous where `row` is 0
inline long row_of(int row, int heads, int dim) { return row ? row : (long)heads * dim; }
constexpr int kMaxHeads = 1 << 12, kMaxDim = 256;

dll_status check_heads(int heads, int kv_heads, int dim, int dtype) {
  if (heads <= 0 || kv_heads <= 0 || dim <= 0 || heads % kv_heads) return DLL_ERR_SHAPE;
  if (dtype != DLL_FP32 && dtype != DLL_BF16) return DLL_ERR_UNSUPPORTED;
  return heads > kMaxHeads || dim > kMaxDim ? DLL_ERR_UNSUPPORTED : DLL_OK;
}

dll_status check_attention(const dll_attention_desc *d) {
  if (!d) return DLL_ERR_NULL;
  if (d->q_tokens <= 0 || d->kv_tokens <= 0 || d->sequences <= 0) return DLL_ERR_SHAPE;
  const dll_status st = check_heads(d->heads, d->kv_heads, d->head_dim, d->dtype);
  if (st != DLL_OK) return st;
  if (d->causal != 0 && d->causal != 1) return DLL_ERR_UNSUPPORTED;
  const long q_least = (long)d->heads * d->head_dim, kv_least = (long)d->kv_heads * d->head_dim;
  const long q_row = row_of(d->q_row, d->heads, d->head_dim), kv_row = row_of(d->kv_row, d->kv_heads, d->head_dim);
  if (q_row < q_least || kv_row < kv_least) return DLL_ERR_SHAPE;
  if (d->q_tokens > kMaxTokens || d->kv_tokens > kMaxTokens || d->sequences > kMaxFeatures || q_row > kMaxFeatures || kv_row > kMaxFeatures)
    return DLL_ERR_UNSUPPORTED;
  if ((size_t)d->q_tokens * q_row >= kMaxElements || (size_t)d->kv_tokens * kv_row >= kMaxElements) return DLL_ERR_UNSUPPORTED;
  return attention_fits(d->q_tokens, d->kv_tokens, d->sequences, d->heads) ? DLL_OK : DLL_ERR_UNSUPPORTED;
}

AttentionArgs attention_args(const dll_attention_desc *d) {
  AttentionArgs a;
  a.Tq = d->q_tokens; a.Tk = d->kv_tokens; a.S = d->sequences; a.H = d->heads; a.KV = d->kv_heads; a.D = d->head_dim;
  a.causal = d->causal; a.dtype = d->dtype;
  a.q_row = row_of(d->q_row, d->heads, d->head_dim);
  a.kv_row = row_of(d->kv_row, d->kv_heads, d->head_dim);
  return a;
}

dll_status check_cache(const dll_cache_desc *d) {
  if (!d) return DLL_ERR_NULL;
  if (d->requests <= 0 || d->pages <= 0 || d->page_tokens <= 0 || d->table_pages <= 0) return DLL_ERR_SHAPE;
  const dll_status st = check_heads(d->heads, d->kv_heads, d->head_dim, d->dtype);
  if (st != DLL_OK) return st;
  if (d->requests > 1 << 16 || (long)d->requests * d->heads > kMaxGrid || (size_t)d->requests * d->table_pages >= kMaxElements) return DLL_ERR_UNSUPPORTED;
  if ((size_t)d->pages * d->page_tokens >= kMaxElements || (size_t)d->table_pages * d->page_tokens > (size_t)1 << 30) return DLL_ERR_UNSUPPORTED;
  return DLL_OK;
}

CacheArgs cache_args(const dll_cache_desc *d) {
  CacheArgs a;
  a.R = d->requests; a.H = d->heads; a.KV = d->kv_heads; a.D = d->head_dim;
  a.pages = d->pages; a.page = d->page_tokens; a.columns = d->table_pages; a.dtype = d->dtype;
  return a;
}

// Scores are scale * log2 e times a product: that factor has to be a number
bool off_scale(float scale) { return !(std::fabs(scale) <= 0x1p127f); }

// q, k, v and their gradients stand at any multiple of their elements; o and its gradient at 16 bytes
bool off_type(const void *p, int dtype) { return reinterpret_cast<uintptr_t>(p) % type_bytes(dtype) != 0; }

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

size_t dll_attention_fwd_workspace_bytes(const dll_attention_desc *d) {
  return check_attention(d) == DLL_OK ? align_up(attention_fwd_scratch(attention_args(d))) : 0;
}

dll_status dll_attention_fwd(const dll_attention_desc *d, const void *q, const void *k, const void *v, const int *q_starts, const int *kv_starts, float scale,
                             void *o, float *lse, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_attention(d);
  if (st != DLL_OK) return st;
  if (!q || !k || !v || !q_starts || !kv_starts || !o) return DLL_ERR_NULL;
  const void *in[] = {q, k, v, q_starts, kv_starts}, *out[] = {o, lse, ws};
  if (aliased(in, 5, out, 3) || misaligned(o) || off_element(lse) || off_element(q_starts) || off_element(kv_starts)) return DLL_ERR_SHAPE;
  if (off_type(q, d->dtype) || off_type(k, d->dtype) || off_type(v, d->dtype) || off_scale(scale)) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_attention_fwd_workspace_bytes(d))) != DLL_OK) return st;
  AttentionArgs a = attention_args(d);
  a.q = q; a.k = k; a.v = v; a.q_starts = q_starts; a.kv_starts = kv_starts; a.scale = scale; a.o = o; a.lse = lse;
  return dev(launch_attention_fwd(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

size_t dll_attention_bwd_workspace_bytes(const dll_attention_desc *d) {
  return check_attention(d) == DLL_OK ? align_up(attention_bwd_scratch(attention_args(d))) : 0;
}

dll_status dll_attention_bwd(const dll_attention_desc *d, const void *q, const void *k, const void *v, const int *q_starts, const int *kv_starts, float scale,
                             const void *o, const float *lse, const void *d_o, void *dq, void *dk, void *dv, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_attention(d);
  if (st != DLL_OK) return st;
  if (!q || !k || !v || !q_starts || !kv_starts || !o || !lse || !d_o || (!dq && !dk && !dv)) return DLL_ERR_NULL;
  const void *in[] = {q, k, v, q_starts, kv_starts, o, lse, d_o}, *out[] = {dq, dk, dv, ws};
  if (aliased(in, 8, out, 4) || misaligned(o) || misaligned(d_o) || off_element(lse) || off_element(q_starts) || off_element(kv_starts)) return DLL_ERR_SHAPE;
  for (const void *p : {q, k, v, (const void *)dq, (const void *)dk, (const void *)dv})
    if (off_type(p, d->dtype)) return DLL_ERR_SHAPE;
  if (off_scale(scale)) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_attention_bwd_workspace_bytes(d))) != DLL_OK) return st;
  AttentionArgs a = attention_args(d);
  a.q = q; a.k = k; a.v = v; a.q_starts = q_starts; a.kv_starts = kv_starts; a.scale = scale;
  a.o = const_cast<void *>(o); a.lse = const_cast<float *>(lse); a.d_o = d_o; a.dq = dq; a.dk = dk; a.dv = dv;
  return dev(launch_attention_bwd(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
}

dll_status dll_cache_plan(const dll_cache_desc *d, const int *lengths, const int *added, const int *free_pages, int n_free, const int *free_at, int *table,
                          int *starts, int *slots, int tokens, int *state, void *stream) {
  const dll_status st = check_cache(d);
  if (st != DLL_OK) return st;
  if (!lengths || !added || (!free_pages && n_free > 0) || !table || !starts || !slots || !state) return DLL_ERR_NULL;
  if (n_free < 0 || tokens <= 0) return DLL_ERR_SHAPE;
  if (tokens > kMaxTokens) return DLL_ERR_UNSUPPORTED;
  const void *in[] = {lengths, added, free_pages, free_at}, *out[] = {table, starts, slots, state};
  if (aliased(in, 4, out, 4)) return DLL_ERR_SHAPE;
  for (int i = 0; i < 4; ++i)
    if (off_element(in[i]) || off_element(out[i])) return DLL_ERR_SHAPE;
  CacheArgs a = cache_args(d);
  a.lengths = lengths; a.added = added; a.free_pages = free_pages; a.n_free = n_free; a.free_at = free_at;
  a.table = table; a.starts = starts; a.slots = slots; a.tokens = tokens; a.state = state;
  return dev(launch_cache_plan(a, static_cast<hipStream_t>(stream)));
}

dll_status dll_cache_write(const dll_cache_desc *d, int tokens, int row, const void *k, const void *v, const int *slots, void *k_cache, void *v_cache,
                           void *stream) {
  const dll_status st = check_cache(d);
  if (st != DLL_OK) return st;
  if (!k || !v || !slots || !k_cache || !v_cache) return DLL_ERR_NULL;
  const long least = (long)d->kv_heads * d->head_dim, between = row_of(row, d->kv_heads, d->head_dim);
  if (tokens <= 0 || between < least) return DLL_ERR_SHAPE;
  if (tokens > kMaxTokens || between > kMaxFeatures || (size_t)tokens * between >= kMaxElements) return DLL_ERR_UNSUPPORTED;
  const void *in[] = {k, v, slots}, *out[] = {k_cache, v_cache};
  if (aliased(in, 3, out, 2) || misaligned(k_cache) || misaligned(v_cache) || off_type(k, d->dtype) || off_type(v, d->dtype) || off_element(slots))
    return DLL_ERR_SHAPE;
  CacheArgs a = cache_args(d);
  a.tokens = tokens; a.row = between; a.k = k; a.v = v; a.slots = const_cast<int *>(slots); a.k_cache = k_cache; a.v_cache = v_cache;
  return dev(launch_cache_write(a, static_cast<hipStream_t>(stream)));
}

size_t dll_paged_attention_workspace_bytes(const dll_cache_desc *d) {
  return check_cache(d) == DLL_OK ? align_up(paged_attention_scratch(cache_args(d))) : 0;
}

dll_status dll_paged_attention(const dll_cache_desc *d, const void *q, const void *k_cache, const void *v_cache, const int *table, const int *lengths,
                               float scale, void *o, float *lse, void *ws, size_t ws_bytes, void *stream) {
  dll_status st = check_cache(d);
  if (st != DLL_OK) return st;
  if (!q || !k_cache || !v_cache || !table || !lengths || !o) return DLL_ERR_NULL;
  const void *in[] = {q, k_cache, v_cache, table, lengths}, *out[] = {o, lse, ws};
  if (aliased(in, 5, out, 3) || misaligned(q) || misaligned(k_cache) || misaligned(v_cache) || misaligned(o)) return DLL_ERR_SHAPE;
  if (off_element(table) || off_element(lengths) || off_element(lse) || off_scale(scale)) return DLL_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, dll_paged_attention_workspace_bytes(d))) != DLL_OK) return st;
  CacheArgs a = cache_args(d);
  a.q = q; a.k_cache = const_cast<void *>(k_cache); a.v_cache = const_cast<void *>(v_cache); a.table = const_cast<int *>(table); a.lengths = lengths;
  a.scale = scale; a.o = o; a.lse = lse;
  return dev(launch_paged_attention(a, static_cast<char *>(ws), static_cast<hipStream_t>(stream)));
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
