// Softmax cross entropy over a large vocabulary, with its gradients, without the logits ever being stored:
//   z = x W^T + bias, lse_t = ln sum_v exp z_tv, loss_t = lse_t - z_t[label_t], loss = mean over the counted rows
//   dz = scale / count * (softmax(z) - onehot), dx = dz W, dW = dz^T x, dbias = sum_t dz
// Rows whose label lies outside [0, V) do not count; the others are gathered to the front first, so that rows left out cost
// no products and what they hold (also infinities and NaN) reaches nothing.
//
// The product's epilogue takes each row's maximum m_g and sum of exp(z - m_g) over groups of 64 or 32 columns; one kernel joins
// the groups to lse.  For the gradients the epilogue also leaves e = exp(z - m_g) in the operands' type, and a second pass
// turns it in place into p - onehot, p = e * exp((M - lse) + (m_g - M)) with the row's maximum M (whose distance to lse is kept, as the
// difference of the two afterwards would have lost it).  Exponentials in (0, 1] relative to their own group keep all the type's digits,
// which rounded logits would not (bfloat16 logits of size 10 are 2 % off after exp); e and p - onehot are rounded to the type once
// each.  scale / count multiplies the products' sums: inside dz its rounding to bfloat16, up to 0.4 %, would be the same for all
// gradients.  This takes three products of T D V; forming the logits again for the gradients would take four.
// The exponentials are kept for a piece of the tokens at a time, 1 GiB at most.
//
// With gradients the matrix pipe bounds it: 4096 x 2048 x 50257 bf16, 3690 rows counted, 2.39 ms = 950 TFLOP/s (logits 868 us, both
// gradients 1371, the pass over the exponentials 140 = 5.3 TB/s).  Without them a few tokens are bound by the weights' bytes:
// 16 x 1024 x 32000 bf16 20.3 us, 14.7 of which read 66 MB at 4.5 TB/s; the rest joins the groups.  A small layer is a chain of short
// launches: 128 x 2048 x 1000 in single precision 51 us in seven.
#include "large_ops.h"
#include "skinny_product.h"

namespace dllk {

using namespace tile;

namespace {

constexpr size_t kPieceBytes = (size_t)1 << 30;  // of exponentials kept at a time
constexpr int kGatherRows = 2;                   // of a workgroup then: copies of more rows would be a chain of round trips
constexpr int kOneGather = 4096;                 // labels that every workgroup counts by itself
constexpr int kFewRows = 32;                     // rows of a forward pass that are not gathered and that one workgroup joins
constexpr size_t kStatBytes = (size_t)1 << 28;   // of group statistics kept at a time (forward pass alone)

// exp(x) for x <= 0 through the hardware's 2^x: off by |x| * 2^-24 relative, and what is small weighs little in the sums
__device__ __forceinline__ float exp_below(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

// Among N = 4 or 8 neighbouring lanes, without LDS: each lane's neighbour, its pair's neighbour, the other four.
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kMirror8 = 0x141;   // quad_perm 1 0 3 2, quad_perm 2 3 0 1, row_half_mirror
template <int N>
__device__ __forceinline__ float max_of(float v) {
  v = fmaxf(v, lane_swap<kSwap1>(v));
  v = fmaxf(v, lane_swap<kSwap2>(v));
  return N == 8 ? fmaxf(v, lane_swap<kMirror8>(v)) : v;
}
template <int N>
__device__ __forceinline__ float sum_of(float v) {
  v += lane_swap<kSwap1>(v);
  v += lane_swap<kSwap2>(v);
  return N == 8 ? v + lane_swap<kMirror8>(v) : v;
}

// Row statistics (and exponentials) of 32 x WC logits; a group is WC columns.
template <class T, bool KEEP>
struct LogitEpi {
  const T *bias;         // nullable
  const int *labels;     // of the product's rows
  float2 *stats;         // [group][rows_ld]: maximum, sum
  long rows_ld;
  float *hit;            // [row]: the label's logit
  T *e;                  // KEEP: [row][ld], zeros behind column V
  long ld;
  // the labels of up to 128 rows, one or two a lane
  struct Ahead { int label[2]; };
  __device__ __forceinline__ Ahead ahead(int m, int M, int lane) const {
    return Ahead{{labels[min(m + lane, M - 1)], labels[min(m + 64 + lane, M - 1)]}};
  }
  // rows that were not gathered may hold anything where their label is none
  __device__ __forceinline__ bool counts(Ahead of, int q, int lane, int V) const {
    return (unsigned)__shfl(q & 2 ? of.label[1] : of.label[0], (q & 1) * 32 + (lane & 31)) < (unsigned)V;
  }
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int V, int, int, int q, Ahead of) const {
    const Lanes<WC> l;
    const int col = l.col;
    if (n >= V) return;
    float b[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (bias) load8<T>(bias + n + col, b, V - n - col);
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int at_row = l.kRows * p + l.row, row = m + at_row;
      const int at = (int)((unsigned)__shfl(q & 2 ? of.label[1] : of.label[0], (q & 1) * 32 + at_row) - (unsigned)(n + col));   // any label
      float z[8];
      stage8(stage, at_row, col, z);
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        z[j] = n + col + j < V ? z[j] + b[j] : -INFINITY;
        top = fmaxf(top, z[j]);
      }
      top = max_of<l.kARow>(top);
      const float from = top == -INFINITY ? 0.0f : top;   // a group that the bias masks out altogether: all terms are 0
      float e8[8], sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e8[j] = exp_below(z[j] - from);
        sum += e8[j];
      }
      sum = sum_of<l.kARow>(sum);
      if (row >= M) continue;
      if (col == 0) stats[(long)(n / WC) * rows_ld + row] = make_float2(top, sum);
      if ((unsigned)at < 8u) {
        float z_at = z[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) z_at = at == j ? z[j] : z_at;
        hit[row] = z_at;
      }
      if (KEEP && n + col < ld) store8<T>(e + (long)row * ld + n + col, e8, 8);
    }
  }
};

// The statistics alone for a few tokens: groups of 32 columns, four neighbours a lane and 16 columns an accumulator.
template <class T>
struct SkinnyLogits {
  const T *bias;
  const int *labels;
  float2 *stats;
  long rows_ld;
  float *hit;
  template <int R>
  __device__ __forceinline__ void tile(const floatx4 (&v)[R], int m, int n, int M, int V) const {
    static_assert(R == 2, "groups of 32 columns");
    float z[R][4], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int at = n + kSkinnyColumns * r + j;
        z[r][j] = at < V ? v[r][j] + (bias ? to_float(bias[at]) : 0.0f) : -INFINITY;
        top = fmaxf(top, z[r][j]);
      }
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum += exp_below(z[r][j] - from);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (m >= M) return;
    if ((threadIdx.x & 63) < 16) stats[(long)(n / (R * kSkinnyColumns)) * rows_ld + m] = make_float2(top, sum);
    const int label = labels[m];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (label == n + kSkinnyColumns * r + j && label < V) hit[m] = z[r][j];
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

// The same and the copies in one launch, where T is at most kOneGather: every workgroup counts the labels before its rows
// by itself.
template <class T>
__global__ __launch_bounds__(256) void gather_kernel(const int *labels, int T_, int V, const T *x, int D, T *xc, long ld, int *rows, int *row_labels, int *count,
                                                      float *row_loss, float *row_lse, T *dx) {
  __shared__ int before_[4], all_[4], to[kGatherRows];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, r0 = blockIdx.x * kGatherRows;
  int before = 0, all = 0;
#pragma unroll 4
  for (int i = t; i < T_; i += 256) {
    const int in = labels[i] >= 0 && labels[i] < V;
    all += in;
    before += i < r0 ? in : 0;
  }
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) {
    before += __shfl_down(before, k);
    all += __shfl_down(all, k);
  }
  if (lane == 0) before_[wave] = before, all_[wave] = all;
  __syncthreads();
  before = before_[0] + before_[1] + before_[2] + before_[3];
  all = all_[0] + all_[1] + all_[2] + all_[3];
  if (wave == 0) {
    const int r = r0 + lane, label = lane < kGatherRows && r < T_ ? labels[r] : -1;
    const bool in = label >= 0 && label < V;
    const int at = before + __popcll(__ballot(in) & ((1ull << lane) - 1));
    if (in) {
      rows[at] = r;
      row_labels[at] = label;
    } else if (lane < kGatherRows && r < T_) {
      if (row_loss) row_loss[r] = 0.0f;
      if (row_lse) row_lse[r] = 0.0f;
    }
    if (lane < kGatherRows) to[lane] = in ? at : -1;
    if (blockIdx.x == 0 && lane == 0) *count = all;
  }
  __syncthreads();
  const int groups = (int)(ld / 8), whole = (all + 63) & ~63;
  const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 2
  for (int i = t; i < kGatherRows * groups; i += 256) {
    const int k = i / groups, c = (i - k * groups) * 8, left = D - c, r = r0 + k;
    if (r >= T_) break;
    if (to[k] >= 0) {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (left > 0) load8<T>(x + (long)r * D + c, v, left);
      store8<T>(xc + (long)to[k] * ld + c, v, 8);
    } else if (dx && left > 0) {
      store8<T>(dx + (long)r * D + c, zero, left);
    }
  }
  for (int r = all + (int)blockIdx.x; r < whole; r += (int)gridDim.x)
    for (int c = t; c < groups; c += 256) store8<T>(xc + (long)r * ld + 8 * c, zero, 8);
}

// xc = the counted rows of x in padded rows, zeros up to the next whole slab of rows; rows of dx that do not count become zeros.
template <class T>
__global__ __launch_bounds__(256) void gather_rows_kernel(const T *x, T *xc, long ld, int T_, int D, const int *rows, const int *count, const int *labels, int V,
                                                           T *dx) {
  const int n = *count, groups = (int)(ld / 8), whole = (n + 63) & ~63;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < (long)(T_ + 63) * groups; i += (long)gridDim.x * 256) {
    const int r = (int)(i / groups), c = (int)(i % groups) * 8, left = D - c;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r < n && left > 0) load8<T>(x + (long)rows[r] * D + c, v, left);
    if (r < whole) store8<T>(xc + (long)r * ld + c, v, 8);
    if (dx && left > 0 && r < T_ && (labels[r] < 0 || labels[r] >= V)) {
      const float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      store8<T>(dx + (long)r * D + c, zero, left);
    }
  }
}

// lse = M + ln sum_g s_g exp(m_g - M), loss = (M - z_label) + the same logarithm.  A workgroup takes 16 rows at a time, 64 threads
// each.  Rows that were not gathered (all_labels given) are taken by one workgroup, which passes over those that do not count and
// leaves the mean as well.
__global__ __launch_bounds__(1024) void join_groups_kernel(const float2 *stats, int groups, long rows_ld, const float *hit, int M, const int *count, int first,
                                                            const int *rows, float2 *lse, float *piece_loss, float *row_loss, float *row_lse, const int *all_labels, int V, float *loss) {
  __shared__ float2 part[16][17];
  __shared__ double mean[16];
  __shared__ int counts[16];
  const int t = threadIdx.x, r = t & 15, sub = t >> 4, lane = t & 63, n = rows_left(count, first, M);
  double total = 0.0;
  int counted = 0;
  for (int r0 = blockIdx.x * 16; r0 < n; r0 += gridDim.x * 16) {
    const int row = r0 + r;
    float top = -INFINITY, sum = 0.0f;
    if (row < n) {
#pragma unroll 4
      for (int g = sub; g < groups; g += 64) {
        const float2 v = stats[(long)g * rows_ld + row];
        const float m = fmaxf(top, v.x);
        // -infinity: nothing finite in it, and its sum is 0 (or NaN, which is to stay)
        sum = (top == -INFINITY ? sum : sum * exp_below(top - m)) + (v.x == -INFINITY ? v.y : v.y * exp_below(v.x - m));
        top = m;
      }
    }
    const auto join = [&](float t2, float s2) {
      const float m = fmaxf(top, t2);
      sum = (top == -INFINITY ? sum : sum * exp_below(top - m)) + (t2 == -INFINITY ? s2 : s2 * exp_below(t2 - m));
      top = m;
    };
    // four subs of a wavefront, then the sixteen wavefronts
#pragma unroll
    for (int k = 16; k < 64; k <<= 1) {
      const float t2 = __shfl_down(top, k), s2 = __shfl_down(sum, k);
      join(t2, s2);
    }
    __syncthreads();   // the former rows' parts have been read
    if (lane < 16) part[t >> 6][r] = make_float2(top, sum);
    __syncthreads();
    if (t < 16 && row < n) {
      top = -INFINITY, sum = 0.0f;
#pragma unroll
      for (int w = 0; w < 16; ++w) join(part[w][r].x, part[w][r].y);
      const bool in = !all_labels || (all_labels[row] >= 0 && all_labels[row] < V);
      // The loss from the two logits' difference: where the label has nearly all the probability it is the small logarithm alone, which
      // top + logf(sum) would round to a last digit of top.
      const float tail = logf(sum), l = in ? top + tail : 0.0f, each = in ? (top - hit[row]) + tail : 0.0f;
      const int to = all_labels ? row : rows[row];
      if (lse) lse[row] = make_float2(top, tail);
      if (piece_loss) piece_loss[row] = each;
      if (row_loss) row_loss[to] = each;
      if (row_lse) row_lse[to] = l;
      total += (double)each;
      counted += in;
    }
  }
  if (!all_labels) return;
  if (t < 16) mean[t] = total, counts[t] = counted;
  __syncthreads();
  if (t == 0) {
    double s = 0.0;
    int k = 0;
    for (int i = 0; i < 16; ++i) s += mean[i], k += counts[i];
    *loss = k > 0 ? (float)(s / k) : 0.0f;
  }
}

// the mean of the counted rows' losses by one workgroup of 256 or more; no rows: 0.  Sums in 64 bits.
__device__ __forceinline__ void mean_loss(const float *row, const int *count, float *loss) {
  __shared__ double part[16];
  const int n = *count, t = threadIdx.x, threads = blockDim.x;
  double s = 0.0;
#pragma unroll 4
  for (int i = t; i < n; i += threads) s += (double)row[i];
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) s += __shfl_down(s, k);
  if ((t & 63) == 0) part[t >> 6] = s;
  __syncthreads();
  if (t == 0) {
    for (int w = 1; w < threads / 64; ++w) s += part[w];
    *loss = n > 0 ? (float)(s / n) : 0.0f;
  }
}
__global__ __launch_bounds__(1024) void mean_loss_kernel(const float *row, const int *count, float *loss) { mean_loss(row, count, loss); }

// p - onehot from the exponentials, in place; a workgroup takes 64 rows x 128 columns and leaves its rows' column sums of dz.  With the
// last piece one workgroup more (the last column's) leaves the mean loss.
template <class T>
__global__ __launch_bounds__(256) void exp_to_gradient_kernel(T *e, long ld, int V, int M, const int *count, int first, const float2 *stats, long rows_ld,
                                                               const float2 *lse, const int *labels, int group, float scale, float *sums, const float *row_loss, float *loss) {
  __shared__ float part[16][128 + 4];
  const int n = rows_left(count, first, M), t = threadIdx.x, r0 = blockIdx.y * 64, sub = t >> 4, col = blockIdx.x * 128 + (t & 15) * 8;
  if (loss && blockIdx.x == gridDim.x - 1) {
    if (blockIdx.y == 0) mean_loss(row_loss, count, loss);
    return;
  }
  if (r0 >= n) return;
  float total[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (col < V) {
    float v[4][8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = r0 + 16 * i + sub;
      if (row < n) load8<T>(e + (long)row * ld + col, v[i], 8);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = r0 + 16 * i + sub;
      if (row < n) {
        const float m = stats[(long)(col / group) * rows_ld + row].x;
        const float2 l = lse[row];   // lse = l.x + l.y
        const float f = m == -INFINITY ? 0.0f * (l.x + l.y) : exp_below((m - l.x) - l.y);   // 0 unless the row's sum is not finite
        const int at = labels[row] - col;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[i][j] *= f;
          if (j == at) v[i][j] -= 1.0f;
          total[j] += v[i][j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;   // up to the next whole slab of rows
      }
      store8<T>(e + (long)row * ld + col, v[i], 8);
    }
  }
  if (!sums) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) part[sub][(t & 15) * 8 + j] = total[j];
  __syncthreads();
  if (t < 128 && blockIdx.x * 128 + t < V) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += part[w][t];
    sums[(long)blockIdx.y * ld + blockIdx.x * 128 + t] = s * (scale / (float)*count);
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

__global__ __launch_bounds__(256) void convert_kernel(const float *src, bf16 *dst, long n) {
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) dst[i] = (bf16)src[i];
}

// A few tokens straight from memory, where a workgroup reads every token for its 32 classes: up to 16, or 32 where the tiles would have
// rows of odd bfloat16 length copied first, as long as the tokens' rows are not too long.  Odd rows are read twice as slowly, and
// with few classes their copies cost little.  The constants leave least time over 1057 measured calls of 1 to 32 tokens, widths of 64 to
// 16001 and 500 to 100000 classes with weights from memory: against the faster way 2.1 % on average, 31 % at most, with odd rows 3.0 %
// (32 x 255 x 100000 is 74 % off).  Microseconds, straight / tiles:
//   1 x 1024 x 5000 9.8 / 11.6, x 100000 49.6 / 59.3; fp32 12.8 / 16.4, 83.5 / 112.8; 16 x 1024 x 32000 21.0 / 22.3; fp32 36.1 / 42.1
//   16 x 4098 x 32000 78.6 / 75.0; fp32 149.6 / 118.4; 1 x 8192 x 100000 354.8 / 289.2; 4 x 2048 x 12000 19.2 / 18.6
//   odd: 16 x 1001 x 32000 34.5 / 49.9; 32 x 513 x 8000 18.4 / 26.5; 16 x 16001 x 500 151.7 / 50.7; 32 x 4095 x 32000 217 / 163
bool skinny(int T, int D, int V, int dtype) {
  const bool odd = !loadable(D, dtype);
  if (D < kSkinnyLeastK || T > (odd ? kSkinnyRows : 16)) return false;
  const long classes = !odd || V > 8192 ? 8192 : V < 1024 ? 1024 : V;
  return (4 + T) * (long)D * (long)type_bytes(dtype) <= 24 * classes;
}

struct Plan {
  long ldd, lde;
  int group, groups, piece, pieces;   // group: columns of a row that share a maximum
  ProductPlan z, gradients;
  int *count, *rows, *labels;
  void *x, *w, *e;
  float2 *stats;
  float2 *lse;    // the row's maximum, and the logarithm of its sum
  float *hit, *loss, *sums, *bias_sum, *dw_sum, *part;
  size_t bytes;
  Plan(int T, int D, int V, int dtype, bool grad, char *base) {
    Take take{base};
    const size_t b = type_bytes(dtype);
    ldd = padded(D);
    lde = padded(V);
    size_t most = grad ? kPieceBytes / ((size_t)lde * b) : kStatBytes / ((size_t)(V / 64 + 1) * sizeof(float2));
    most = most / 256 * 256;
    if (most < 256) most = 256;
    if (most > (1u << 20)) most = 1u << 20;   // 64 rows a workgroup along the grid's second axis
    piece = (size_t)T < most ? T : (int)most;
    pieces = (T + piece - 1) / piece;
    z = plan_product(dtype, piece, V, slabs_of(D, dtype), false, false);
    group = !grad && skinny(T, D, V, dtype) ? 2 * kSkinnyColumns : piece_columns(z.tiling);
    groups = (V + group - 1) / group;
    const size_t slab_rows = (size_t)(piece + 63) / 64 * 64;
    count = (int *)take(sizeof(int));
    rows = (int *)take((size_t)T * sizeof(int));
    labels = (int *)take((size_t)T * sizeof(int));
    x = take((size_t)(T + 63) * ldd * b);
    w = loadable(D, dtype) ? nullptr : take((size_t)V * ldd * b);
    stats = (float2 *)take((size_t)piece * groups * sizeof(float2));
    hit = (float *)take((size_t)piece * sizeof(float));
    loss = (float *)take((size_t)T * sizeof(float));
    lse = nullptr, e = nullptr, sums = bias_sum = dw_sum = part = nullptr;
    if (grad) {
      lse = (float2 *)take((size_t)piece * sizeof(float2));
      e = take(slab_rows * lde * b);
      sums = (float *)take(slab_rows / 64 * lde * sizeof(float));
      bias_sum = (float *)take((size_t)V * sizeof(float));
      if (pieces > 1 && dtype == TYPE_BF16) dw_sum = (float *)take((size_t)V * D * sizeof(float));
      const GradientShape shape[2] = {{piece, D, slabs_of(V, dtype), 1, true}, {V, D, slabs_of(piece, dtype), 1, false}};
      gradients = plan_gradients(dtype, shape, 2);
      part = (float *)take(partial_bytes(gradients.splits, piece, D));
    }
    bytes = take.used;
  }
};

// The counted rows in front, w in rows that a product can load
template <class T>
hipError_t begin(const VocabArgs &a, const Plan &p, const void **w, long *ldw, hipStream_t stream) {
  *w = a.w;
  *ldw = a.D;
  if (p.w) {
    DLL_TRY(launch_pad_rows(a.w, p.w, a.V, a.D, stream));
    *w = p.w;
    *ldw = p.ldd;
  }
  if (a.T <= kOneGather) {
    gather_kernel<T><<<dim3((unsigned)((a.T + kGatherRows - 1) / kGatherRows)), dim3(256), 0, stream>>>(a.labels, a.T, a.V, (const T *)a.x, a.D, (T *)p.x, p.ldd, p.rows, p.labels,
                                                                                      p.count, a.row_loss, a.row_lse, (T *)a.dx);
    return hipGetLastError();
  }
  gather_list_kernel<<<dim3(1), dim3(1024), 0, stream>>>(a.labels, a.T, a.V, p.rows, p.labels, p.count, a.row_loss, a.row_lse);
  DLL_TRY(hipGetLastError());
  const long blocks = ((long)(a.T + 63) * (p.ldd / 8) + 255) / 256;
  gather_rows_kernel<T><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream>>>(
      (const T *)a.x, (T *)p.x, p.ldd, a.T, a.D, p.rows, p.count, a.labels, a.V, (T *)a.dx);
  return hipGetLastError();
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
  const LogitEpi<T, KEEP> epi{(const T *)a.bias, p.labels + first, p.stats, p.piece, p.hit, (T *)p.e, p.lde};
  DLL_TRY((launch_product<T, true, true, false>(g, epi, p.z.tiling, stream)));
  join_groups_kernel<<<dim3((unsigned)((g.M + 15) / 16)), dim3(1024), 0, stream>>>(p.stats, p.groups, p.piece, p.hit, g.M, p.count, first, p.rows + first,
                                                                                       p.lse, p.loss + first, a.row_loss, a.row_lse, nullptr, a.V, nullptr);
  return hipGetLastError();
}

// Few rows: gathering them would cost two launches and save no work, as they are one tile high; rows that do not count come to
// nothing in their own statistics.
template <class T>
hipError_t few_rows_fwd(const VocabArgs &a, const Plan &p, hipStream_t stream) {
  const void *x = a.x, *w = a.w;
  if (skinny(a.T, a.D, a.V, a.dtype)) {
    SkinnyArgs s;
    s.M = a.T;
    s.N = a.V;
    s.K = a.D;
    s.x = x;
    s.w[0] = w;
    DLL_TRY((launch_skinny<T, 2, false, sizeof(T) == 4 ? 16 : kSkinnyRows>(s, SkinnyLogits<T>{(const T *)a.bias, a.labels, p.stats, p.piece, p.hit}, stream)));
    join_groups_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p.stats, p.groups, p.piece, p.hit, a.T, nullptr, 0, nullptr, nullptr, nullptr, a.row_loss, a.row_lse,
                                                               a.labels, a.V, a.loss);
    return hipGetLastError();
  }
  if (p.w) {
    DLL_TRY(launch_pad_rows(a.x, p.x, a.T, a.D, stream));
    DLL_TRY(launch_pad_rows(a.w, p.w, a.V, a.D, stream));
    x = p.x;
    w = p.w;
  }
  ProductArgs g;
  g.M = a.T;
  g.N = a.V;
  g.A[0] = {x, p.w ? p.ldd : a.D};
  g.B[0] = {w, p.w ? p.ldd : a.D};
  g.K[0] = a.D;
  const LogitEpi<T, false> epi{(const T *)a.bias, a.labels, p.stats, p.piece, p.hit, nullptr, 0};
  DLL_TRY((launch_product<T, true, true, false>(g, epi, p.z.tiling, stream)));
  join_groups_kernel<<<dim3(1), dim3(1024), 0, stream>>>(p.stats, p.groups, p.piece, p.hit, a.T, nullptr, 0, nullptr, nullptr, nullptr, a.row_loss, a.row_lse,
                                                             a.labels, a.V, a.loss);
  return hipGetLastError();
}

template <class T>
hipError_t vocab_fwd(const VocabArgs &a, char *scratch, hipStream_t stream) {
  const Plan p(a.T, a.D, a.V, a.dtype, false, scratch);
  if (a.T <= kFewRows) return few_rows_fwd<T>(a, p, stream);
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
    exp_to_gradient_kernel<T><<<dim3((unsigned)((a.V + 127) / 128 + (last ? 1 : 0)), (unsigned)((M + 63) / 64)), dim3(256), 0, stream>>>(
        (T *)p.e, p.lde, a.V, M, p.count, first, p.stats, p.piece, p.lse, p.labels + first, p.group, a.scale, sums, p.loss, last ? a.loss : nullptr);
    DLL_TRY(hipGetLastError());
    if (a.dbias) {
      sum_columns_kernel<T><<<dim3((unsigned)((a.V + 255) / 256)), dim3(256), 0, stream>>>(p.sums, p.lde, a.V, M, p.count, first, p.bias_sum, (T *)a.dbias,
                                                                                             first == 0, last);
      DLL_TRY(hipGetLastError());
    }
    GradientJobs<T> jobs;
    jobs.plan = p.gradients;
    jobs.partial = p.part;
    if (a.dx) {
      ProductArgs g;
      g.M = M;
      g.N = a.D;
      g.A[0] = {p.e, p.lde};
      g.B[0] = {w, ldw};
      g.K[0] = a.V;
      g.m_rows = p.count;
      g.first = first;
      jobs.add(g, StoreEpi<T>((T *)a.dx, nullptr, a.D, p.rows + first, 0, p.count, a.scale), true);
    }
    ProductArgs g;
    g.M = a.V;
    g.N = a.D;
    g.A[0] = {p.e, p.lde};
    g.B[0] = {(const T *)p.x + (long)first * p.ldd, p.ldd};
    g.K[0] = M;
    g.k_rows = p.count;
    g.first = first;
    if (a.dw && !p.dw_sum) jobs.add(g, StoreEpi<T>((T *)a.dw, nullptr, a.D, nullptr, first > 0, p.count, a.scale), false);
    DLL_TRY(launch_gradients<T>(jobs, stream));
    if constexpr (sizeof(T) == 2) {   // pieces of bfloat16 products add up in 32 bits; single precision's in dw itself
      if (a.dw && p.dw_sum) {
        const StoreEpi<float> out(p.dw_sum, nullptr, a.D, nullptr, first > 0, p.count, a.scale);
        DLL_TRY((launch_product<T, false, false, false>(g, out, p.gradients.tiling, stream)));
        if (last) {
          const long n = (long)a.V * a.D, blocks = (n + 255) / 256;
          convert_kernel<<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, stream>>>(p.dw_sum, (bf16 *)a.dw, n);
          DLL_TRY(hipGetLastError());
        }
      }
    }
  }
  return hipSuccess;
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
