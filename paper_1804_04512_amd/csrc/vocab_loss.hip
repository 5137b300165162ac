// Softmax cross entropy over a large vocabulary, with its gradients, without the logits ever being stored:
//   z = x W^T + bias, lse_t = ln sum_v exp z_tv, loss_t = lse_t - z_t[label_t], loss = mean over the counted rows
//   dz = scale / count * (softmax(z) - onehot), dx = dz W, dW = dz^T x, dbias = sum_t dz
// Rows whose label lies outside [0, V) do not count; the others are gathered to the front first, so that rows left out cost
// no products and what they hold (also infinities and NaN) reaches nothing.
//
// The product's epilogue takes each row's maximum m_g and sum of exp(z - m_g) over groups of 64 columns; one kernel joins
// the groups to lse.  For the gradients the epilogue also leaves e = exp(z - m_g) in the operands' type, and a second pass
// turns it in place into dz = e * exp(m_g - lse) * scale / count (minus the label's share): exponentials in (0, 1] relative
// to their own group keep all the type's digits, which rounded logits would not (bfloat16 logits of size 10 are 2 % off
// after exp).  This takes three products of T D V; forming the logits again for the gradients would take four.
// The exponentials are kept for a piece of the tokens at a time, 1 GiB at most.
#include "large_ops.h"
#include "tile_product.h"

namespace dllk {

using namespace tile;

namespace {

constexpr int kGroup = 64;                       // columns of a row that share a maximum
constexpr size_t kPieceBytes = (size_t)1 << 30;  // of exponentials kept at a time
constexpr size_t kStatBytes = (size_t)1 << 28;   // of group statistics kept at a time (forward pass alone)

// exp(x) for x <= 0 through the hardware's 2^x: off by |x| * 2^-24 relative, and what is small weighs little in the sums
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// Row statistics (and exponentials) of 32 x 64 logits.
template <class T, bool KEEP>
struct LogitEpi {
  const T *bias;         // nullable
  const int *labels;     // of the gathered rows
  const int *count;
  int first;
  float2 *stats;         // [row][groups]: maximum, sum
  int groups;
  float *hit;            // [row]: the label's logit
  T *e;                  // KEEP: [row][ld], zeros behind column V
  long ld;
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int V, int, int) const {
    const int lane = threadIdx.x & 63, col = 8 * (lane & 7);
    if (n >= V) return;
    float b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (bias) load8<T>(bias + n + col, b, false, V - n - col);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      const int row = m + 8 * p + (lane >> 3);
      float z[8];
      stage8(stage, 8 * p + (lane >> 3), col, z);
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[j] = n + col + j < V ? z[j] + b[j] : -INFINITY;
        top = fmaxf(top, z[j]);
      }
#pragma unroll
      for (int s = 1; s < 8; s <<= 1) top = fmaxf(top, __shfl_xor(top, s));
      const float from = top == -INFINITY ? 0.0f : top;   // a group that the bias masks out altogether: all terms are 0
      float e8[8], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e8[j] = exp_below(z[j] - from);
        sum += e8[j];
      }
#pragma unroll
      for (int s = 1; s < 8; s <<= 1) sum += __shfl_xor(sum, s);
      if (row >= M) continue;
      if ((lane & 7) == 0) stats[(long)row * groups + n / kGroup] = make_float2(top, sum);
      const int at = labels[row] - (n + col);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (at == j) hit[row] = z[j];
      if (KEEP && n + col < ld) store8<T>(e + (long)row * ld + n + col, e8, true, 8);
    }
  }
};

// One workgroup: the rows that count, in their order, with their labels; the others' outputs are zeros.
__global__ __launch_bounds__(1024) void gather_list_kernel(const int *labels, int T, int V, int *rows, int *row_labels, int *count, float *row_loss,
                                                            float *row_lse) {
  __shared__ int wave_sum[16];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int before = 0;
  for (int base = 0; base < T; base += 1024) {
    const int i = base + t, label = i < T ? labels[i] : -1;
    const bool in = label >= 0 && label < V;
    const unsigned long long mask = __ballot(in);
    if (lane == 0) wave_sum[wave] = __popcll(mask);
    __syncthreads();
    int at = before, all = 0;
    for (int w = 0; w < 16; ++w) {
      if (w < wave) at += wave_sum[w];
      all += wave_sum[w];
    }
    if (in) {
      at += __popcll(mask & ((1ull << lane) - 1));
      rows[at] = i;
      row_labels[at] = label;
    } else if (i < T) {
      if (row_loss) row_loss[i] = 0.0f;
      if (row_lse) row_lse[i] = 0.0f;
    }
    before += all;
    __syncthreads();
  }
  if (t == 0) *count = before;
}

// xc = the counted rows of x in padded rows, zeros up to the next whole slab of rows; rows of dx that do not count become zeros.
template <class T>
__global__ __launch_bounds__(256) void gather_rows_kernel(const T *x, T *xc, long ld, int T_, int D, const int *rows, const int *count, const int *labels, int V,
                                                           T *dx, int vec_x, int vec_dx) {
  const int n = *count, groups = (int)(ld / 8), whole = (n + 63) & ~63;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < (long)(T_ + 63) * groups; i += (long)gridDim.x * 256) {
    const int r = (int)(i / groups), c = (int)(i % groups) * 8, left = D - c;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r < n) load8<T>(x + (long)rows[r] * D + c, v, vec_x && left >= 8, left);
    if (r < whole) store8<T>(xc + (long)r * ld + c, v, true, 8);
    if (dx && r < T_ && (labels[r] < 0 || labels[r] >= V)) {
      const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      store8<T>(dx + (long)r * D + c, zero, vec_dx && left >= 8, left);
    }
  }
}

// A wavefront per row joins its groups: lse = M + ln sum_g s_g exp(m_g - M).
__global__ __launch_bounds__(256) void join_groups_kernel(const float2 *stats, int groups, const float *hit, int M, const int *count, int first, const int *rows,
                                                           float *lse, float *piece_loss, float *row_loss, float *row_lse) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows_left(count, first, M)) return;
  const float2 *s = stats + (long)row * groups;
  float top = -INFINITY, sum = 0.0f;
  for (int g = lane; g < groups; g += 64) {
    const float2 v = s[g];
    if (v.x > top) {
      sum = sum * exp_below(top - v.x) + v.y;   // the first finite group: 0 * exp(-inf) + s
      top = v.x;
    } else {
      sum += v.x == -INFINITY ? v.y : v.y * exp_below(v.x - top);
    }
  }
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const float t2 = __shfl_xor(top, k), s2 = __shfl_xor(sum, k), m = fmaxf(top, t2);
    const float a = top == -INFINITY ? sum : sum * exp_below(top - m), b = t2 == -INFINITY ? s2 : s2 * exp_below(t2 - m);
    sum = lane & k ? b + a : a + b;   // the same order in both lanes
    top = m;
  }
  if (lane == 0) {
    const float l = top + logf(sum), loss = l - hit[row];
    if (lse) lse[row] = l;
    piece_loss[row] = loss;
    if (row_loss) row_loss[rows[row]] = loss;
    if (row_lse) row_lse[rows[row]] = l;
  }
}

// dz from the exponentials, in place; a workgroup takes 64 rows x 512 columns and leaves the column sums of its rows
template <class T>
__global__ __launch_bounds__(256) void exp_to_gradient_kernel(T *e, long ld, int V, int M, const int *count, int first, const float2 *stats, int groups,
                                                               const float *lse, const int *labels, float scale, float *sums) {
  __shared__ float part[3][512];
  const int n = rows_left(count, first, M), t = threadIdx.x, r0 = blockIdx.y * 64, sub = t >> 6;
  if (r0 >= n) return;
  const float share = scale / (float)*count;
  const int col = blockIdx.x * 512 + (t & 63) * 8;
  float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (col < ld) {
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int row = r0 + 4 * i + sub;
      T *p = e + (long)row * ld + col;
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (row < n) {
        load8<T>(p, v, true, 8);
        const float m = stats[(long)row * groups + col / kGroup].x;
        const float f = m == -INFINITY ? 0.0f * lse[row] : exp_below(m - lse[row]) * share;   // 0 unless the row's sum is not finite
        const int at = labels[row] - col;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] *= f;
          if (j == at) v[j] -= share;
          total[j] += v[j];
        }
      }
      store8<T>(p, v, true, 8);
    }
  }
  if (!sums) return;
  if (sub > 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) part[sub - 1][(t & 63) * 8 + j] = total[j];
  __syncthreads();
  if (sub == 0 && col < ld) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int w = 0; w < 3; ++w) total[j] += part[w][(t & 63) * 8 + j];
    store8<float>(sums + (long)blockIdx.y * ld + col, total, true, 8);
  }
}

// acc (fp32, between pieces) or dbias (at the last piece) = what was there + the pieces' column sums in order
template <class T>
__global__ __launch_bounds__(256) void sum_columns_kernel(const float *sums, long ld, int V, int M, const int *count, int first, float *acc, T *dbias, int begin,
                                                           int end) {
  const int v = blockIdx.x * 256 + threadIdx.x;
  if (v >= V) return;
  const int strips = (rows_left(count, first, M) + 63) / 64;
  float s = begin ? 0.0f : acc[v];
#pragma unroll 8
  for (int i = 0; i < strips; ++i) s += sums[(long)i * ld + v];
  if (end) dbias[v] = (T)s;
  else acc[v] = s;
}

// One workgroup: the mean of the counted rows' losses; no rows: 0.  Sums in 64 bits.
__global__ __launch_bounds__(1024) void mean_loss_kernel(const float *row, const int *count, float *loss) {
  __shared__ double part[16];
  const int n = *count, t = threadIdx.x;
  double s = 0.0;
  for (int i = t; i < n; i += 1024) s += (double)row[i];
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) s += __shfl_down(s, k);
  if ((t & 63) == 0) part[t >> 6] = s;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < 16; ++w) s += part[w];
    *loss = n > 0 ? (float)(s / n) : 0.0f;
  }
}

template <class T>
__global__ __launch_bounds__(256) void convert_kernel(const float *src, T *dst, long n) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) dst[i] = (T)src[i];
}

struct Plan {
  long ldd, lde;
  int groups, piece, pieces;
  ProductPlan z, dx, dw;
  int *count, *rows, *labels;
  void *x, *w, *e;
  float2 *stats;
  float *hit, *lse, *loss, *sums, *bias_sum, *dw_sum, *part;
  size_t bytes;
  Plan(int T, int D, int V, int dtype, bool grad, char *base) {
    Take take{base};
    const size_t b = type_bytes(dtype);
    ldd = padded(D);
    lde = padded(V);
    groups = (V + kGroup - 1) / kGroup;
    size_t most = grad ? kPieceBytes / ((size_t)lde * b) : kStatBytes / ((size_t)groups * sizeof(float2));
    most = most / 256 * 256;
    if (most < 256) most = 256;
    if (most > (1u << 20)) most = 1u << 20;   // 64 rows a workgroup along the grid's second axis
    piece = (size_t)T < most ? T : (int)most;
    pieces = (T + piece - 1) / piece;
    const size_t slab_rows = (size_t)(piece + 63) / 64 * 64;
    count = (int *)take(sizeof(int));
    rows = (int *)take((size_t)T * sizeof(int));
    labels = (int *)take((size_t)T * sizeof(int));
    x = take((size_t)(T + 63) * ldd * b);
    w = whole_groups(D, dtype) ? nullptr : take((size_t)V * ldd * b);
    stats = (float2 *)take((size_t)piece * groups * sizeof(float2));
    hit = (float *)take((size_t)piece * sizeof(float));
    loss = (float *)take((size_t)T * sizeof(float));
    lse = nullptr, e = nullptr, sums = bias_sum = dw_sum = part = nullptr;
    z = plan_product(dtype, piece, V, slabs_of(D, dtype), 1, false, false);
    if (grad) {
      lse = (float *)take((size_t)piece * sizeof(float));
      e = take(slab_rows * lde * b);
      sums = (float *)take(slab_rows / 64 * lde * sizeof(float));
      bias_sum = (float *)take((size_t)V * sizeof(float));
      if (pieces > 1 && dtype == TYPE_BF16) dw_sum = (float *)take((size_t)V * D * sizeof(float));
      dx = plan_product(dtype, piece, D, slabs_of(V, dtype), 1, false, true);
      dw = plan_product(dtype, V, D, slabs_of(piece, dtype), 1, false, false);
      if (dx.splits > 1) part = (float *)take((size_t)dx.splits * piece * ldd * sizeof(float));
    }
    bytes = take.used;
  }
};

// The counted rows in front, w in rows that a product can load
template <class T>
hipError_t begin(const VocabArgs &a, const Plan &p, const void **w, long *ldw, hipStream_t stream) {
  gather_list_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a.labels, a.T, a.V, p.rows, p.labels, p.count, a.row_loss, a.row_lse);
  DLL_TRY(hipGetLastError());
  const long blocks = ((long)(a.T + 63) * (p.ldd / 8) + 255) / 256;
  gather_rows_kernel<T><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream>>>(
      (const T *)a.x, (T *)p.x, p.ldd, a.T, a.D, p.rows, p.count, a.labels, a.V, (T *)a.dx, rows16<T>(a.x, a.D), rows16<T>(a.dx, a.D));
  DLL_TRY(hipGetLastError());
  *w = a.w;
  *ldw = a.D;
  if (p.w) {
    DLL_TRY(launch_pad_rows(a.w, p.w, a.V, a.D, a.dtype, stream));
    *w = p.w;
    *ldw = p.ldd;
  }
  return hipSuccess;
}

// logits of one piece: statistics, and the exponentials where they are kept
template <class T, bool KEEP>
hipError_t logits(const VocabArgs &a, const Plan &p, int first, const void *w, long ldw, hipStream_t stream) {
  ProductArgs g;
  g.M = a.T - first < p.piece ? a.T - first : p.piece;
  g.N = a.V;
  g.A[0] = {(const T *)p.x + (long)first * p.ldd, p.ldd};
  g.B[0] = {w, ldw};
  g.K[0] = a.D;
  g.m_rows = p.count;
  g.first = first;
  const LogitEpi<T, KEEP> epi{(const T *)a.bias, p.labels + first, p.count, first, p.stats, p.groups, p.hit, (T *)p.e, p.lde};
  DLL_TRY((launch_product<T, true, true, false>(g, epi, p.z.tiling, stream)));
  join_groups_kernel<<<dim3((unsigned)((g.M + 3) / 4)), dim3(256), 0, stream>>>(p.stats, p.groups, p.hit, g.M, p.count, first, p.rows + first, p.lse,
                                                                                   p.loss + first, a.row_loss, a.row_lse);
  return hipGetLastError();
}

template <class T>
hipError_t vocab_fwd(const VocabArgs &a, char *scratch, hipStream_t stream) {
  const Plan p(a.T, a.D, a.V, a.dtype, false, scratch);
  const void *w;
  long ldw;
  DLL_TRY(begin<T>(a, p, &w, &ldw, stream));
  for (int first = 0; first < a.T; first += p.piece) DLL_TRY((logits<T, false>(a, p, first, w, ldw, stream)));
  mean_loss_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p.loss, p.count, a.loss);
  return hipGetLastError();
}

template <class T>
hipError_t vocab_grad(const VocabArgs &a, char *scratch, hipStream_t stream) {
  const Plan p(a.T, a.D, a.V, a.dtype, true, scratch);
  const void *w;
  long ldw;
  DLL_TRY(begin<T>(a, p, &w, &ldw, stream));
  for (int first = 0; first < a.T; first += p.piece) {
    const int M = a.T - first < p.piece ? a.T - first : p.piece;
    const bool last = first + p.piece >= a.T;
    DLL_TRY((logits<T, true>(a, p, first, w, ldw, stream)));
    float *sums = a.dbias ? p.sums : nullptr;
    exp_to_gradient_kernel<T><<<dim3((unsigned)((p.lde + 511) / 512), (unsigned)((M + 63) / 64)), dim3(256), 0, stream>>>(
        (T *)p.e, p.lde, a.V, M, p.count, first, p.stats, p.groups, p.lse, p.labels + first, a.scale, sums);
    DLL_TRY(hipGetLastError());
    if (a.dbias) {
      sum_columns_kernel<T><<<dim3((unsigned)((a.V + 255) / 256)), dim3(256), 0, stream>>>(p.sums, p.lde, a.V, M, p.count, first, p.bias_sum, (T *)a.dbias,
                                                                                             first == 0, last);
      DLL_TRY(hipGetLastError());
    }
    if (a.dx) {
      ProductArgs g;
      g.M = M;
      g.N = a.D;
      g.A[0] = {p.e, p.lde};
      g.B[0] = {w, ldw};
      g.K[0] = a.V;
      g.m_rows = p.count;
      g.first = first;
      const StoreEpi<T> out{{(T *)a.dx, nullptr}, a.D, rows16<T>(a.dx, a.D), p.rows + first, 0};
      DLL_TRY((product_to<T, true, false>(g, out, p.dx, p.part, stream)));
    }
    if (a.dw) {
      ProductArgs g;
      g.M = a.V;
      g.N = a.D;
      g.A[0] = {p.e, p.lde};
      g.B[0] = {(const T *)p.x + (long)first * p.ldd, p.ldd};
      g.K[0] = M;
      g.k_rows = p.count;
      g.first = first;
      if (p.dw_sum) {   // pieces of bfloat16 products add up in 32 bits
        const StoreEpi<float> out{{p.dw_sum, nullptr}, a.D, rows16<float>(p.dw_sum, a.D), nullptr, first > 0};
        DLL_TRY((launch_product<T, false, false, false>(g, out, p.dw.tiling, stream)));
        if (last) {
          const long n = (long)a.V * a.D, blocks = (n + 255) / 256;
          convert_kernel<T><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, stream>>>(p.dw_sum, (T *)a.dw, n);
          DLL_TRY(hipGetLastError());
        }
      } else {
        const StoreEpi<T> out{{(T *)a.dw, nullptr}, a.D, rows16<T>(a.dw, a.D), nullptr, first > 0};
        DLL_TRY((launch_product<T, false, false, false>(g, out, p.dw.tiling, stream)));
      }
    }
  }
  mean_loss_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p.loss, p.count, a.loss);
  return hipGetLastError();
}

}  // namespace

size_t vocab_fwd_scratch(int T, int D, int V, int dtype) { return Plan(T, D, V, dtype, false, nullptr).bytes; }
size_t vocab_grad_scratch(int T, int D, int V, int dtype) { return Plan(T, D, V, dtype, true, nullptr).bytes; }

hipError_t launch_vocab_fwd(const VocabArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? vocab_fwd<bf16>(a, scratch, stream) : vocab_fwd<float>(a, scratch, stream);
}
hipError_t launch_vocab_grad(const VocabArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? vocab_grad<bf16>(a, scratch, stream) : vocab_grad<float>(a, scratch, stream);
}

}  // namespace dllk
