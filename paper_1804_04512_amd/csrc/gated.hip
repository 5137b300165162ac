// Gated feed-forward block, forward and backward:
//   a = x Wg^T, b = x Wu^T, h = act(a) * b, y = h Wd^T
//   dh = dy Wd, da = dh * b * act'(a), db = dh * act(a)
//   dWd = dy^T h, dWg = da^T x, dWu = db^T x, dx = da Wg + db Wu
// Sums in 32 bits.  With bfloat16 operands h, da and db are rounded to bfloat16 on the way to the next product, as its
// matrix instructions take nothing wider; a and b are kept for the backward pass in the operands' type.  Gradients are then off by
// 3.5e-3 relative, where a and b in 32 bits and one rounding at the end would give 1.7e-3; they would take twice the memory.
//
// Forward: a and b in one product, whose wavefronts hold both factors of a hidden unit, so that h leaves from its epilogue; then y.
// Backward: dh, whose epilogue leaves da, db and h; then every gradient in one launch.  A few tokens are bound by the weights' bytes:
// 2048 x 8192 bf16, one token, 25.8 us for 101 MB = 3.9 TB/s.  Many are bound by the matrix pipe: 4096 tokens, training pass 1.19 ms,
// 1040 TFLOP/s of 18 T D H (a and b 279 us, y 147, dh 183, a third of it what its epilogue reads and writes, gradients 586).
// In between workgroups are few and short: 777 x 1000 x 2730 bf16 41 us, 310 TFLOP/s, 301 tiles of 16 slabs; 1000 x 500 x 1337 in single
// precision 145 us with its backward pass.
#include "large_ops.h"
#include "skinny_product.h"

namespace dllk {

using namespace tile;

namespace {

// 1 / (1 + exp(-a)) through the hardware's 2^x and reciprocal: off by 1.5 |a| 2^-24 and two last digits, relative
__device__ __forceinline__ float sigmoid(float a) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * a)); }

// The normal distribution's cumulative function, by the complement, which keeps its digits where 1 + erf has lost them (below -5.5 all).
// Where its product is rounded to bfloat16, erf by the formula 7.1.26 of Abramowitz and Stegun's handbook, a third of the library
// function's instructions: 40 of these an element were a quarter of the forward kernel at 777 x 1000 x 2730.  Its absolute error is
// 1.5e-7; in the left tail that is half a bfloat16 step at -6 (relative 3.6e-3, of a value of 1e-9) and 1 % at -8.
template <class T>
__device__ __forceinline__ float normal_cdf(float a) {
  if (sizeof(T) == 4) return 0.5f * erfcf(a * -0.70710678118654752f);
  const float x = fabsf(a) * 0.70710678118654752f, t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * x);
  const float poly = t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
  const float half = 0.5f * poly * __builtin_amdgcn_exp2f(-1.44269504088896341f * x * x);   // (1 - erf(x)) / 2
  return a < 0.0f ? half : 1.0f - half;
}

// act(a) and act'(a)
template <class T>
__device__ __forceinline__ void gate_both(int gate, float a, float *f, float *d) {
  switch (gate) {
    case GATE_SIGMOID: {
      const float s = sigmoid(a);
      *f = s;
      *d = s * (1.0f - s);
      return;
    }
    case GATE_RELU:
      *f = a > 0.0f ? a : 0.0f;
      *d = a > 0.0f ? 1.0f : 0.0f;
      return;
    case GATE_SILU: {
      const float s = sigmoid(a);
      *f = a * s;
      *d = s * (1.0f + a * (1.0f - s));
      return;
    }
    case GATE_GELU: {
      const float c = normal_cdf<T>(a);
      *f = a * c;
      *d = c + a * __builtin_amdgcn_exp2f(-0.72134752044448170f * a * a) * 0.39894228040143268f;
      return;
    }
    default:
      *f = a;
      *d = 1.0f;
  }
}
template <class T>
__device__ __forceinline__ float gate_value(int gate, float a) {
  float f, d;
  gate_both<T>(gate, a, &f, &d);
  return f;
}

// h = act(a) * b from a piece whose first half's columns are a and whose second half's are b of the same hidden units; h in
// padded rows
template <class T>
struct GateEpi : NothingAhead {
  GateEpi(int gate_, T *h_, long ldh_, T *a_, T *b_) : gate(gate_), h(h_), ldh(ldh_), kept_a(a_), kept_b(b_) {}
  int gate;
  T *h;
  long ldh;
  T *kept_a, *kept_b;   // nullable, [T][H]
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int H, int, int, int, Nothing) const {
    const Lanes<WC / 2> l;
    const int col = l.col;
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int row = l.kRows * p + l.row;
      if (m + row >= M || n + col >= H) continue;
      float va[8], vb[8], vh[8];
      stage8(stage, row, col, va);
      stage8(stage, row, WC / 2 + col, vb);
      const int left = H - n - col;
#pragma unroll
      for (int j = 0; j < 8; ++j) vh[j] = j < left ? gate_value<T>(gate, va[j]) * vb[j] : 0.0f;
      store8<T>(h + (long)(m + row) * ldh + n + col, vh, 8);
      if (kept_a) {
        const long o = (long)(m + row) * H + n + col;
        store8<T>(kept_a + o, va, left);
        store8<T>(kept_b + o, vb, left);
      }
    }
  }
};

// The same for a few tokens; h in rows of H
template <class T>
struct SkinnyGate {
  int gate;
  T *h, *kept_a, *kept_b;   // kept_*: nullable
  template <int R>
  __device__ __forceinline__ void tile(const floatx4 (&v)[R], int m, int n, int M, int H) const {
    static_assert(R == 2, "a and b");
    if (m >= M || n >= H) return;
    float a[4], b[4], o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[j] = v[0][j];
      b[j] = v[1][j];
      o[j] = gate_value<T>(gate, a[j]) * b[j];
    }
    const long at = (long)m * H + n;
    store4<T>(h + at, o, H - n);
    if (kept_a) {
      store4<T>(kept_a + at, a, H - n);
      store4<T>(kept_b + at, b, H - n);
    }
  }
};

// da, db and h from dh and the kept a and b, all three in padded rows
template <class T>
struct GateBackEpi : NothingAhead {
  GateBackEpi(int gate_, const T *a_, const T *b_, T *da_, T *db_, T *h_, long ld_)
      : gate(gate_), a(a_), b(b_), da(da_), db(db_), h(h_), ld(ld_) {}
  int gate;
  const T *a, *b;
  T *da, *db, *h;
  long ld;
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int H, int, int, int, Nothing) const {
    const Lanes<WC> l;
    const int col = l.col, left = H - n - col;
    if (left <= 0) return;
    Eight<T> va[l.kPasses], vb[l.kPasses];   // all loads of the piece go out together
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int row = min(m + l.kRows * p + l.row, M - 1);
      va[p].load(a + (long)row * H + n + col, left);
      vb[p].load(b + (long)row * H + n + col, left);
    }
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int row = l.kRows * p + l.row;
      if (m + row >= M) continue;
      float g[8], oa[8], ob[8], oh[8];
      stage8(stage, row, col, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float va_ = (float)va[p].v[j], vb_ = (float)vb[p].v[j];
        float f, d;
        gate_both<T>(gate, va_, &f, &d);
        oa[j] = j < left ? g[j] * vb_ * d : 0.0f;
        ob[j] = j < left ? g[j] * f : 0.0f;
        oh[j] = j < left ? f * vb_ : 0.0f;
      }
      const long o = (long)(m + row) * ld + n + col;
      store8<T>(da + o, oa, 8);
      store8<T>(db + o, ob, 8);
      store8<T>(h + o, oh, 8);
    }
  }
};

__global__ __launch_bounds__(256) void pad_rows_kernel(const bf16 *src, bf16 *dst, int rows, int cols, long ld) {
  const int c0 = blockIdx.x * 512 + (threadIdx.x & 63);
  for (long r = blockIdx.y * 4 + (threadIdx.x >> 6); r < rows; r += gridDim.y * 4) {
    bf16 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = src[r * cols + min(c0 + 64 * j, cols - 1)];   // all on their way before the first is stored
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (c0 + 64 * j < ld) dst[r * ld + c0 + 64 * j] = c0 + 64 * j < cols ? v[j] : (bf16)0.0f;
  }
}

// A few tokens: the weights straight from memory, or tiles with k in parts.  Straight from memory y has a workgroup for 16 of its D
// columns, which reads 16 rows of Wd and every token's h: with long rows of H and few columns some compute units read much and
// the others nothing, and each token adds a row (of h in single precision two rows' time).  With many columns all units read.  The
// constants leave least time over 1386 measured calls of 1 to 32 tokens, widths of 63 to 8192 and 256 to 22016 hidden units with weights
// from memory, odd sizes too (rows of odd bfloat16 length are copied before the tiles): against the faster of both 1.1 % on
// average in bfloat16 and 1.3 % in single precision, 29 % at most.  Microseconds, straight / tiles:
//   1 x 2048 x 8192 27.4 / 30.1, x 11008 37.3 / 39.8, x 14336 45.3 / 44.1; fp32 51.0 / 53.8, 69.6 / 84.7, 86.4 / 88.3
//   4 x 2048 x 8192 28.5 / 30.0, x 11008 39.1 / 40.0, x 14336 47.9 / 44.3; fp32 53.2 / 54.4, 73.2 / 85.0, 90.7 / 88.7
//   16 x 2048 x 8192 33.3 / 30.7, x 4096 18.9 / 23.7; fp32 64.0 / 54.9, 34.8 / 36.9; 16 x 4096 x 8192 47.4 / 48.2; fp32 93.3 / 95.4
//   16 x 63 x 22015 146 / 37; 1 x 512 x 14336 26.5 / 22.4; 32 x 2048 x 8192 37.2 / 32.7; 24 x 1000 x 2730 14.5 / 21.8
bool skinny(int T, int D, int H, int dtype) {
  if (T > kSkinnyRows || D < kSkinnyLeastK || H < kSkinnyLeastK) return false;
  const long row = (long)H * (long)type_bytes(dtype), columns = D < 4096 ? D : 4096;
  return dtype == TYPE_BF16 ? (16 + T) * row <= 192 * (columns > 1536 ? columns : 1536) : (8 + T) * row <= 288 * (columns > 640 ? columns : 640);
}

// The workspace's parts, the same walk for the query and the call
struct FwdPlan {
  long ldh, ldd;
  void *h, *x, *wg, *wu, *wd;
  float *part;
  ProductPlan up, down;
  size_t bytes;
  FwdPlan(int T, int D, int H, int dtype, char *base) {
    Take take{base};
    const size_t e = type_bytes(dtype);
    ldh = padded(H);
    ldd = padded(D);
    h = take((size_t)T * ldh * e);
    x = wg = wu = wd = nullptr;
    part = nullptr;
    if (skinny(T, D, H, dtype)) {   // nothing else
      bytes = take.used;
      return;
    }
    if (!loadable(D, dtype)) x = take((size_t)T * ldd * e), wg = take((size_t)H * ldd * e), wu = take((size_t)H * ldd * e);
    if (!loadable(H, dtype)) wd = take((size_t)D * ldh * e);
    up = plan_product(dtype, T, H, slabs_of(D, dtype), true, false);
    down = plan_product(dtype, T, D, slabs_of(H, dtype), false, true);
    part = (float *)take(partial_bytes(down.splits, T, D));
    bytes = take.used;
  }
};

struct BwdPlan {
  long ldh, ldd;
  void *da, *db, *h, *x, *wg, *wu, *wd, *dy;
  float *part;
  ProductPlan dh, gradients;
  size_t bytes;
  BwdPlan(int T, int D, int H, int dtype, char *base) {
    Take take{base};
    const size_t e = type_bytes(dtype);
    ldh = padded(H);
    ldd = padded(D);
    da = take((size_t)T * ldh * e);
    db = take((size_t)T * ldh * e);
    h = take((size_t)T * ldh * e);
    x = wg = wu = wd = dy = nullptr;
    if (!loadable(D, dtype)) x = take((size_t)T * ldd * e), dy = take((size_t)T * ldd * e), wg = take((size_t)H * ldd * e), wu = take((size_t)H * ldd * e);
    if (!loadable(H, dtype)) wd = take((size_t)D * ldh * e);
    dh = plan_product(dtype, T, H, slabs_of(D, dtype), false, false);
    const long tokens = slabs_of(T, dtype);
    const GradientShape shape[3] = {{T, D, 2 * slabs_of(H, dtype), 1, true}, {H, D, tokens, 2, false}, {D, H, tokens, 1, false}};
    gradients = plan_gradients(dtype, shape, 3);
    part = (float *)take(partial_bytes(gradients.splits, T, D));
    bytes = take.used;
  }
};

template <class T>
hipError_t gated_fwd(const GatedArgs &a, char *scratch, hipStream_t stream) {
  const FwdPlan p(a.T, a.D, a.H, a.dtype, scratch);
  if (skinny(a.T, a.D, a.H, a.dtype)) {
    SkinnyArgs s;
    s.M = a.T;
    s.N = a.H;
    s.K = a.D;
    s.x = a.x;
    s.w[0] = a.w_gate;
    s.w[1] = a.w_up;
    DLL_TRY((launch_skinny<T, 2, true, kSkinnyRows>(s, SkinnyGate<T>{a.gate, (T *)p.h, (T *)a.gate_pre, (T *)a.up_pre}, stream)));
    s.N = a.D;
    s.K = a.H;
    s.x = p.h;
    s.w[0] = a.w_down;
    return launch_skinny<T, 1, false, kSkinnyRows>(s, SkinnyStore<T>{(T *)a.y}, stream);
  }
  const void *x = a.x, *wg = a.w_gate, *wu = a.w_up, *wd = a.w_down;
  if (p.x) {
    DLL_TRY(launch_pad_rows(x, p.x, a.T, a.D, stream));
    DLL_TRY(launch_pad_rows(wg, p.wg, a.H, a.D, stream));
    DLL_TRY(launch_pad_rows(wu, p.wu, a.H, a.D, stream));
    x = p.x, wg = p.wg, wu = p.wu;
  }
  if (p.wd) {
    DLL_TRY(launch_pad_rows(wd, p.wd, a.D, a.H, stream));
    wd = p.wd;
  }
  const long ldx = p.x ? p.ldd : a.D, ldd = p.wd ? p.ldh : a.H;
  ProductArgs g;
  g.M = a.T;
  g.N = a.H;
  g.A[0] = {x, ldx};
  g.B[0] = {wg, ldx};
  g.B[1] = {wu, ldx};
  g.K[0] = a.D;
  const GateEpi<T> ge(a.gate, (T *)p.h, p.ldh, (T *)a.gate_pre, (T *)a.up_pre);
  DLL_TRY((launch_product<T, true, true, true>(g, ge, p.up.tiling, stream)));
  ProductArgs y;
  y.M = a.T;
  y.N = a.D;
  y.A[0] = {p.h, p.ldh};
  y.B[0] = {wd, ldd};
  y.K[0] = a.H;
  StoreEpi<T> out((T *)a.y, nullptr, a.D, nullptr, 0);
  return product_to<T, true, true>(y, out, p.down, p.part, stream);
}

template <class T>
hipError_t gated_bwd(const GatedArgs &a, char *scratch, hipStream_t stream) {
  const BwdPlan p(a.T, a.D, a.H, a.dtype, scratch);
  const void *x = a.x, *wg = a.w_gate, *wu = a.w_up, *wd = a.w_down, *dy = a.dy;
  if (p.x) {
    DLL_TRY(launch_pad_rows(dy, p.dy, a.T, a.D, stream));
    dy = p.dy;
    if (a.dw_gate || a.dw_up) DLL_TRY(launch_pad_rows(x, p.x, a.T, a.D, stream));
    x = p.x;
    if (a.dx) {
      DLL_TRY(launch_pad_rows(wg, p.wg, a.H, a.D, stream));
      DLL_TRY(launch_pad_rows(wu, p.wu, a.H, a.D, stream));
      wg = p.wg, wu = p.wu;
    }
  }
  if (p.wd) {
    DLL_TRY(launch_pad_rows(wd, p.wd, a.D, a.H, stream));
    wd = p.wd;
  }
  const long ldx = p.x ? p.ldd : a.D, ldd = p.wd ? p.ldh : a.H;
  // dh = dy Wd, leaving as da, db and h
  ProductArgs g;
  g.M = a.T;
  g.N = a.H;
  g.A[0] = {dy, ldx};
  g.B[0] = {wd, ldd};
  g.K[0] = a.D;   // Wd lies across k
  const GateBackEpi<T> ge(a.gate, (const T *)a.gate_pre, (const T *)a.up_pre,
                    (T *)p.da, (T *)p.db, (T *)p.h, p.ldh);
  DLL_TRY((launch_product<T, true, false, false>(g, ge, p.dh.tiling, stream)));
  GradientJobs<T> jobs;
  jobs.plan = p.gradients;
  jobs.partial = p.part;
  if (a.dx) {
    ProductArgs w;
    w.M = a.T;
    w.N = a.D;
    w.A[0] = {p.da, p.ldh};
    w.A[1] = {p.db, p.ldh};
    w.B[0] = {wg, ldx};
    w.B[1] = {wu, ldx};
    w.K[0] = w.K[1] = a.H;
    jobs.add(w, StoreEpi<T>((T *)a.dx, nullptr, a.D, nullptr, 0), true);
  }
  if (a.dw_gate || a.dw_up) {
    ProductArgs w;
    w.M = a.H;
    w.N = a.D;
    w.problems = a.dw_gate && a.dw_up ? 2 : 1;
    const int first = a.dw_gate ? 0 : 1;
    const void *d[2] = {p.da, p.db};
    T *o[2] = {(T *)a.dw_gate, (T *)a.dw_up};
    w.A[0] = {d[first], p.ldh};
    w.A[1] = {d[1], p.ldh};
    w.B[0] = w.B[1] = {x, ldx};
    w.K[0] = a.T;
    jobs.add(w, StoreEpi<T>(o[first], o[1], a.D, nullptr, 0), false);
  }
  if (a.dw_down) {
    ProductArgs w;
    w.M = a.D;
    w.N = a.H;
    w.A[0] = {dy, ldx};
    w.B[0] = {p.h, p.ldh};
    w.K[0] = a.T;
    jobs.add(w, StoreEpi<T>((T *)a.dw_down, nullptr, a.H, nullptr, 0), false);
  }
  return launch_gradients<T>(jobs, stream);
}

}  // namespace

hipError_t launch_pad_rows(const void *src, void *dst, long rows, long cols, hipStream_t stream) {
  const long ld = padded(cols), fours = (rows + 3) / 4;
  const dim3 grid((unsigned)((ld + 511) / 512), (unsigned)(fours < 32768 ? fours : 32768));
  pad_rows_kernel<<<grid, dim3(256), 0, stream>>>((const bf16 *)src, (bf16 *)dst, (int)rows, (int)cols, ld);
  return hipGetLastError();
}

size_t gated_fwd_scratch(int T, int D, int H, int dtype) { return FwdPlan(T, D, H, dtype, nullptr).bytes; }
size_t gated_bwd_scratch(int T, int D, int H, int dtype) { return BwdPlan(T, D, H, dtype, nullptr).bytes; }

hipError_t launch_gated_fwd(const GatedArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? gated_fwd<bf16>(a, scratch, stream) : gated_fwd<float>(a, scratch, stream);
}
hipError_t launch_gated_bwd(const GatedArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? gated_bwd<bf16>(a, scratch, stream) : gated_bwd<float>(a, scratch, stream);
}

}  // namespace dllk
