// Global gradient norm over many tensors, clipping by it, and the momentum step with clipping folded in:
//   norm = sqrt(sum over all tensors of g^2), c = min(1, max_norm / norm)
//   clip:   out = c g
//   update: v <- mu v - lr (c g + decay theta), theta <- theta + v
// The tensors' addresses travel in the kernel arguments (kTable of them a launch), so a call copies nothing and can be
// captured.  Squares are added in 64 bits: no gradient overflows or vanishes in the sum, whose order is fixed.  What bounds
// both kernels is memory: the norm reads the gradients once; the second kernel adds the few partial sums again in
// every workgroup, which saves a launch between the two.
#include "large_ops.h"
#include "tile_product.h"

namespace dllk {

using namespace tile;

namespace {

constexpr int kTable = 64;          // tensors of a launch
constexpr int kChunk = 8192;        // elements a workgroup takes at a time
constexpr int kPartials = 1024;     // workgroups of the norm, over all its launches

struct NormTable {
  int n, chunks;
  const void *g[kTable];
  long count[kTable];
  int first[kTable + 1];            // chunk at which each tensor starts
  unsigned char type[kTable], vec[kTable];
};
struct ClipTable {
  NormTable t;
  void *out[kTable];
};
struct StepTable {
  NormTable t;
  float *p[kTable], *v[kTable];
  bf16 *copy[kTable];
  float decay[kTable];
};
static_assert(sizeof(StepTable) <= 4000, "kernel arguments");

__device__ __forceinline__ int tensor_of(const NormTable &t, int chunk) {
  int low = 0, high = t.n - 1;   // the last tensor that starts at or before the chunk
  while (low < high) {
    const int mid = (low + high + 1) >> 1;
    if (t.first[mid] <= chunk) low = mid;
    else high = mid - 1;
  }
  return low;
}

// the sum of a workgroup of 256, in every thread
__device__ __forceinline__ double group_sum(double s) {
  __shared__ double part[4];
#pragma unroll
  for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <class T>
__device__ __forceinline__ double squares(const T *g, long begin, long end, bool vec) {
  double s = 0.0;
  if (vec) {
#pragma unroll 4
    for (long i = begin + 8 * threadIdx.x; i < end; i += 8 * 256) {
      float v[8];
      const long left = end - i;
      load8<T>(g + i, v, left >= 8, (int)(left < 8 ? left : 8));
#pragma unroll
      for (int j = 0; j < 8; ++j) s += (double)v[j] * (double)v[j];
    }
  } else {
#pragma unroll 8
    for (long i = begin + threadIdx.x; i < end; i += 256) {
      const double v = (double)to_float(g[i]);
      s += v * v;
    }
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(const NormTable t, double *partial) {
  double s = 0.0;
  for (int c = blockIdx.x; c < t.chunks; c += gridDim.x) {
    const int i = tensor_of(t, c);
    const long begin = (long)(c - t.first[i]) * kChunk, end = min(t.count[i], begin + kChunk);
    s += t.type[i] == TYPE_BF16 ? squares<bf16>((const bf16 *)t.g[i], begin, end, t.vec[i]) : squares<float>((const float *)t.g[i], begin, end, t.vec[i]);
  }
  s = group_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// the norm from the partial sums, the same in every workgroup
__device__ __forceinline__ double norm_of(const double *partial, int n) {
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 256) s += partial[i];
  return sqrt(group_sum(s));
}

__global__ __launch_bounds__(256) void norm_kernel(const double *partial, int n, float *norm) {
  const double x = norm_of(partial, n);
  if (threadIdx.x == 0) *norm = (float)x;
}

template <class T>
__device__ __forceinline__ void scale_chunk(const T *g, T *out, long begin, long end, bool vec, float c) {
  if (vec) {
#pragma unroll 4
    for (long i = begin + 8 * threadIdx.x; i < end; i += 8 * 256) {
      float v[8];
      const int left = (int)(end - i < 8 ? end - i : 8);
      load8<T>(g + i, v, left == 8, left);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= c;
      store8<T>(out + i, v, left == 8, left);
    }
  } else {
#pragma unroll 8
    for (long i = begin + threadIdx.x; i < end; i += 256) out[i] = (T)(to_float(g[i]) * c);
  }
}

__global__ __launch_bounds__(256) void grad_scale_kernel(const ClipTable a, const double *partial, int n, float max_norm, float *norm) {
  const double x = norm_of(partial, n);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
  const float c = x > (double)max_norm && isfinite(x) ? (float)((double)max_norm / x) : 1.0f;
  const NormTable &t = a.t;
  for (int k = blockIdx.x; k < t.chunks; k += gridDim.x) {
    const int i = tensor_of(t, k);
    if (c == 1.0f && a.out[i] == t.g[i]) continue;   // in place, and nothing to scale
    const long begin = (long)(k - t.first[i]) * kChunk, end = min(t.count[i], begin + kChunk);
    if (t.type[i] == TYPE_BF16) scale_chunk<bf16>((const bf16 *)t.g[i], (bf16 *)a.out[i], begin, end, t.vec[i], c);
    else scale_chunk<float>((const float *)t.g[i], (float *)a.out[i], begin, end, t.vec[i], c);
  }
}

template <class T>
__device__ __forceinline__ void step_chunk(const T *g, float *p, float *v, bf16 *copy, long begin, long end, bool vec, float c, float step, float mu, float decay) {
  if (vec) {
#pragma unroll 2
    for (long i = begin + 8 * threadIdx.x; i < end; i += 8 * 256) {
      float vg[8], vp[8], vv[8];
      const int left = (int)(end - i < 8 ? end - i : 8);
      load8<T>(g + i, vg, left == 8, left);
      load8<float>(p + i, vp, left == 8, left);
      load8<float>(v + i, vv, left == 8, left);
#pragma unroll
      for (int j = 0; j < 8; ++j) update_param(&vp[j], &vv[j], vg[j] * c, step, mu, decay);
      store8<float>(p + i, vp, left == 8, left);
      store8<float>(v + i, vv, left == 8, left);
      if (copy) store8<bf16>(copy + i, vp, left == 8, left);
    }
  } else {
#pragma unroll 4
    for (long i = begin + threadIdx.x; i < end; i += 256) {
      float q = p[i], w = v[i];
      update_param(&q, &w, to_float(g[i]) * c, step, mu, decay);
      p[i] = q;
      v[i] = w;
      if (copy) copy[i] = (bf16)q;
    }
  }
}

__global__ __launch_bounds__(256) void momentum_step_kernel(const StepTable a, const double *partial, int n, float max_norm, float step, float mu, float *norm) {
  const double x = norm_of(partial, n);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
  if (!isfinite(x)) return;   // a gradient that overflowed: no step
  const float c = x > (double)max_norm ? (float)((double)max_norm / x) : 1.0f;
  const NormTable &t = a.t;
  for (int k = blockIdx.x; k < t.chunks; k += gridDim.x) {
    const int i = tensor_of(t, k);
    const long begin = (long)(k - t.first[i]) * kChunk, end = min(t.count[i], begin + kChunk);
    if (t.type[i] == TYPE_BF16) step_chunk<bf16>((const bf16 *)t.g[i], a.p[i], a.v[i], a.copy[i], begin, end, t.vec[i], c, step, mu, a.decay[i]);
    else step_chunk<float>((const float *)t.g[i], a.p[i], a.v[i], a.copy[i], begin, end, t.vec[i], c, step, mu, a.decay[i]);
  }
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

// Tensors [at, at + kTable) of the list that hold anything; returns where the next table starts
int fill(NormTable &t, const GradList &l, const void *const *grads, int at, int *which) {
  t.n = t.chunks = 0;
  for (; at < l.n && t.n < kTable; ++at) {
    if (l.counts[at] == 0) continue;
    const long chunks = ((long)l.counts[at] + kChunk - 1) / kChunk;
    if (t.chunks + chunks > 0x40000000L) break;   // of one launch; a tensor has 2^31 elements at most
    which[t.n] = at;
    t.g[t.n] = grads[at];
    t.count[t.n] = (long)l.counts[at];
    t.type[t.n] = (unsigned char)l.dtypes[at];
    t.vec[t.n] = aligned16(grads[at]);
    t.first[t.n] = t.chunks;
    t.chunks += (int)chunks;
    ++t.n;
  }
  t.first[t.n] = t.chunks;
  return at;
}

hipError_t launch_squares(const GradList &l, const void *const *grads, double *partial, int *used, hipStream_t stream) {
  long total = 0;
  for (int i = 0; i < l.n; ++i) total += ((long)l.counts[i] + kChunk - 1) / kChunk;
  *used = 0;
  int which[kTable];
  for (int at = 0; at < l.n;) {
    NormTable t;
    at = fill(t, l, grads, at, which);
    if (t.n == 0) break;
    // workgroups in proportion to the work, all launches together at most kPartials (and one each)
    long blocks = total <= kPartials / 2 ? t.chunks : (long)((double)t.chunks / total * (kPartials / 2));
    if (blocks < 1) blocks = 1;
    grad_squares_kernel<<<dim3((unsigned)blocks), dim3(256), 0, stream>>>(t, partial + *used);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    *used += (int)blocks;
  }
  return hipSuccess;
}

unsigned apply_blocks(int chunks) { return (unsigned)(chunks < 8 * chip().cus ? chunks : 8 * chip().cus); }

}  // namespace

size_t grad_norm_scratch(const GradList &l) { return ((size_t)kPartials + l.n / kTable + 1) * sizeof(double); }

hipError_t launch_grad_norm(const GradList &l, const void *const *grads, float *norm, char *scratch, hipStream_t stream) {
  double *partial = (double *)scratch;
  int used = 0;
  DLL_TRY(launch_squares(l, grads, partial, &used, stream));
  norm_kernel<<<dim3(1), dim3(256), 0, stream>>>(partial, used, norm);
  return hipGetLastError();
}

hipError_t launch_grad_clip(const GradList &l, const void *const *grads, void *const *out, float max_norm, float *norm, char *scratch, hipStream_t stream) {
  double *partial = (double *)scratch;
  int used = 0, which[kTable], at = 0;
  DLL_TRY(launch_squares(l, grads, partial, &used, stream));
  do {
    ClipTable a;
    at = fill(a.t, l, grads, at, which);
    for (int i = 0; i < a.t.n; ++i) {
      a.out[i] = out[which[i]];
      a.t.vec[i] = a.t.vec[i] && aligned16(a.out[i]);
    }
    grad_scale_kernel<<<dim3(a.t.n ? apply_blocks(a.t.chunks) : 1), dim3(256), 0, stream>>>(a, partial, used, max_norm, norm);
    DLL_TRY(hipGetLastError());
  } while (at < l.n);
  return hipSuccess;
}

hipError_t launch_momentum_clipped(const GradList &l, float *const *params, float *const *velocity, const void *const *grads, const float *decay, float lr, float mu,
                                   float max_norm, float *norm, void *const *copies, char *scratch, hipStream_t stream) {
  double *partial = (double *)scratch;
  int used = 0, which[kTable], at = 0;
  DLL_TRY(launch_squares(l, grads, partial, &used, stream));
  do {
    StepTable a;
    at = fill(a.t, l, grads, at, which);
    for (int i = 0; i < a.t.n; ++i) {
      const int k = which[i];
      a.p[i] = params[k];
      a.v[i] = velocity[k];
      a.copy[i] = copies ? (bf16 *)copies[k] : nullptr;
      a.decay[i] = decay ? decay[k] : 0.0f;
      a.t.vec[i] = a.t.vec[i] && aligned16(a.p[i]) && aligned16(a.v[i]) && aligned16(a.copy[i]);
    }
    momentum_step_kernel<<<dim3(a.t.n ? apply_blocks(a.t.chunks) : 1), dim3(256), 0, stream>>>(a, partial, used, max_norm, -lr, mu, norm);
    DLL_TRY(hipGetLastError());
  } while (at < l.n);
  return hipSuccess;
}

}  // namespace dllk
