// Internal launch interfaces of the large-model operators: gated feed-forward block, vocabulary loss, attention, gradient clipping.
// Every pointer is a device pointer unless it says host.
#pragma once

#include "dll_internal.h"

namespace dllk {

enum { TYPE_F32 = 0, TYPE_BF16 = 1 };
enum { GATE_IDENTITY = 0, GATE_SIGMOID = 1, GATE_RELU = 2, GATE_SILU = 3, GATE_GELU = 4 };

inline size_t type_bytes(int dtype) { return dtype == TYPE_BF16 ? 2 : 4; }
// Elements of a row that is kept in the workspace: whole 128-byte lines (of either type), so that no slab's row takes two.
inline long padded(long n) { return (n + 63) & ~63L; }
// Rows of n elements that a product can load as they are (they start at multiples of four bytes); others are copied into padded rows
// first.
inline bool loadable(long n, int dtype) { return n * (long)type_bytes(dtype) % 4 == 0; }

// n / d for n from 0 to 2^31 - 1: n * (floor(2^(31 + shift) / d) + 1) / 2^(31 + shift), off by less than 1 / d where 2^shift >= d
struct Divisor {
  unsigned factor, shift;
  explicit Divisor(int d) : shift(0) {
    while (1L << shift < d) ++shift;
    factor = (unsigned)((1L << (31 + shift)) / d + 1);
  }
  __device__ __forceinline__ int of(int n) const { return (int)(__umulhi((unsigned)n << 1, factor) >> shift); }
};

// ---- gated feed-forward block -------------------------------------------------------------------------------------
struct GatedArgs {
  int T = 0, D = 0, H = 0, gate = 0, dtype = 0;
  const void *x = nullptr, *w_gate = nullptr, *w_up = nullptr, *w_down = nullptr;
  void *y = nullptr;
  void *gate_pre = nullptr, *up_pre = nullptr;   // forward: nullable outputs; backward: inputs
  const void *dy = nullptr;
  void *dx = nullptr, *dw_gate = nullptr, *dw_up = nullptr, *dw_down = nullptr;   // each nullable
};
size_t gated_fwd_scratch(int T, int D, int H, int dtype);
size_t gated_bwd_scratch(int T, int D, int H, int dtype);
hipError_t launch_gated_fwd(const GatedArgs &a, char *scratch, hipStream_t stream);
hipError_t launch_gated_bwd(const GatedArgs &a, char *scratch, hipStream_t stream);

// ---- softmax cross entropy over a vocabulary ------------------------------------------------------------------------
struct VocabArgs {
  int T = 0, D = 0, V = 0, dtype = 0;
  const void *x = nullptr, *w = nullptr, *bias = nullptr;   // bias nullable
  const int *labels = nullptr;
  float scale = 1.0f;
  float *row_loss = nullptr, *row_lse = nullptr, *loss = nullptr;   // row_*: nullable
  void *dx = nullptr, *dw = nullptr, *dbias = nullptr;              // gradient call: each nullable
};
size_t vocab_fwd_scratch(int T, int D, int V, int dtype);
size_t vocab_grad_scratch(int T, int D, int V, int dtype);
hipError_t launch_vocab_fwd(const VocabArgs &a, char *scratch, hipStream_t stream);
hipError_t launch_vocab_grad(const VocabArgs &a, char *scratch, hipStream_t stream);

// ---- global gradient norm, clipping, momentum step --------------------------------------------------------------------
struct GradList {              // host arrays of n entries
  int n = 0;
  const size_t *counts = nullptr;
  const int *dtypes = nullptr;
};
size_t grad_norm_scratch(const GradList &l);
// *norm = the 2-norm over all tensors
hipError_t launch_grad_norm(const GradList &l, const void *const *grads, float *norm, char *scratch, hipStream_t stream);
// out = grad * min(1, max_norm / norm)
hipError_t launch_grad_clip(const GradList &l, const void *const *grads, void *const *out, float max_norm, float *norm, char *scratch, hipStream_t stream);
hipError_t launch_momentum_clipped(const GradList &l, float *const *params, float *const *velocity, const void *const *grads, const float *decay,
                                   float lr, float mu, float max_norm, float *norm, void *const *copies, char *scratch, hipStream_t stream);

// ---- attention over packed sequences ------------------------------------------------------------------------------------
struct AttentionArgs {
  int Tq = 0, Tk = 0, S = 0, H = 0, KV = 0, D = 0, causal = 0, dtype = 0;
  long q_row = 0, kv_row = 0;      // elements between tokens of q and dq; of k, v, dk and dv
  float scale = 1.0f;
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  const int *q_starts = nullptr, *kv_starts = nullptr;
  void *o = nullptr;               // forward: output; backward: input.  [Tq][H][D]
  float *lse = nullptr;            // [H][Tq]; forward: nullable output; backward: input
  const void *d_o = nullptr;       // [Tq][H][D]
  void *dq = nullptr, *dk = nullptr, *dv = nullptr;   // each nullable
};
// whether the launches' grids hold so many tiles
bool attention_fits(int q_tokens, int kv_tokens, int sequences, int heads);
size_t attention_fwd_scratch(const AttentionArgs &a);
size_t attention_bwd_scratch(const AttentionArgs &a);
hipError_t launch_attention_fwd(const AttentionArgs &a, char *scratch, hipStream_t stream);
hipError_t launch_attention_bwd(const AttentionArgs &a, char *scratch, hipStream_t stream);

// ---- paged cache of keys and values ---------------------------------------------------------------------------------------
struct CacheArgs {
  int R = 0, H = 0, KV = 0, D = 0, pages = 0, page = 0, columns = 0, dtype = 0;
  const int *lengths = nullptr;
  // plan
  const int *added = nullptr, *free_pages = nullptr, *free_at = nullptr;   // free_at: nullable
  int n_free = 0;
  int *table = nullptr, *starts = nullptr, *state = nullptr;
  int *slots = nullptr;            // plan: output; store: input
  int tokens = 0;                  // of slots
  // store
  const void *k = nullptr, *v = nullptr;
  long row = 0;                    // elements between tokens of k and v
  void *k_cache = nullptr, *v_cache = nullptr;   // [pages][KV][page][D]
  // attention
  const void *q = nullptr;
  float scale = 1.0f;
  void *o = nullptr;
  float *lse = nullptr;            // nullable, [R][H]
};
hipError_t launch_cache_plan(const CacheArgs &a, hipStream_t stream);
hipError_t launch_cache_write(const CacheArgs &a, hipStream_t stream);
size_t paged_attention_scratch(const CacheArgs &a);
hipError_t launch_paged_attention(const CacheArgs &a, char *scratch, hipStream_t stream);

// ---- shared: rows copied into padded rows -------------------------------------------------------------------------------
// dst [rows][padded(cols)] = src [rows][cols], zeros behind; bfloat16, as single precision's rows are loadable whatever their length
hipError_t launch_pad_rows(const void *src, void *dst, long rows, long cols, hipStream_t stream);

}  // namespace dllk
