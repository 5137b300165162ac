// Products of a few tokens with a large weight matrix, gfx950: C(m, n) = sum_k X(m, k) * W(n, k) for at most 32 rows m.
//
// Every weight is used 32 times at most, so reading them bounds the product and they go straight from memory into registers:
// 16 rows of W are the first operand of 16x16 matrix instructions, the tokens the second.  A
// workgroup owns 16 R columns of C; its wavefronts take 128 bytes of each row in turn, two sets of loads in flight each, and
// add their sums in LDS in wavefront order.  Rows may start at any element: the loads ask for no alignment, so weights of odd
// sizes are not copied first (which would read and write them once more).
#pragma once

#include "tile_product.h"

namespace dllk {
namespace tile {

constexpr int kSkinnyRows = 32;    // tokens at most, sixteen a matrix instruction
constexpr int kSkinnyColumns = 16; // of C for each of a workgroup's R accumulators

template <class T> struct Step;
template <> struct Step<bf16> {
  static constexpr int kK = 32, kGroup = 8;   // k of a step, of a lane's 16 bytes
  static __device__ __forceinline__ floatx4 mfma(bf16x8 w, bf16x8 x, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, c, 0, 0, 0); }
};
template <> struct Step<float> {
  static constexpr int kK = 16, kGroup = 4;
  static __device__ __forceinline__ floatx4 mfma(floatx4 w, floatx4 x, floatx4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j], x[j], c, 0, 0, 0);
    return c;
  }
};

struct SkinnyArgs {
  int M = 0, N = 0, K = 0;
  const void *x = nullptr, *w[2] = {nullptr, nullptr};   // w[1]: the second accumulator's matrix (pair), else columns 16 .. 31 of w[0]
};

// 16 bytes of a row from any element
template <class T>
__device__ __forceinline__ typename Elem<T>::Frag row16(const T *row, int k) {
  typedef typename Elem<T>::Frag Frag;
  typedef Frag Any __attribute__((aligned(sizeof(T))));
  return *reinterpret_cast<const Any *>(row + k);
}
// The row's last 16 bytes where k + 16 bytes would pass its end, with zeros for what lies before k: each k once, no access outside
// (the row has 16 bytes at least).
template <class T>
__device__ __forceinline__ typename Elem<T>::Frag row16_cut(const T *row, int k, int K) {
  constexpr int n = Step<T>::kGroup;
  const int at = min(k, K - n);
  typename Elem<T>::Frag v = row16<T>(row, at);
#pragma unroll
  for (int j = 0; j < n; ++j) v[j] = at + j >= k ? v[j] : (T)0.0f;
  return v;
}
constexpr int kSkinnyLeastK = 8;   // 16 bytes of either type

// TOKENS: tiles of 16 rows of x.
// Epi: `tile<R>(c, m, n, M, N)`: lane's four neighbouring sums c[r][0..3] of row m, columns n + 16 r (or of both projections).
template <class T, int TOKENS, int R, bool PAIR, int WAVES, class Epi>
__global__ __launch_bounds__(64 * WAVES, 2) void skinny_kernel(const SkinnyArgs a, const Epi epi) {
  constexpr int kK = Step<T>::kK, kAhead = 4;
  typedef typename Elem<T>::Frag Frag;
  __shared__ __attribute__((aligned(16))) floatx4 part[WAVES][TOKENS * R][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), i16 = lane & 15, kq = (lane >> 4) * Step<T>::kGroup;
  const int n0 = blockIdx.x * (PAIR ? kSkinnyColumns : R * kSkinnyColumns);
  const int m0 = 16 * TOKENS * blockIdx.y;
  const T *x[TOKENS], *w[R];  // rows of x and W that do not exist stand in as the last one: their sums are not stored
#pragma unroll
  for (int t = 0; t < TOKENS; ++t) x[t] = (const T *)a.x + (long)min(m0 + 16 * t + i16, a.M - 1) * a.K;
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = (const T *)a.w[PAIR ? r : 0] + (long)min(n0 + i16 + (PAIR ? 0 : kSkinnyColumns * r), a.N - 1) * a.K;
  // A wavefront takes 128 bytes of each row at a time, 32 of them a lane in two loads (the order of k is the same for both
  // operands), and two sets of kAhead loads in turn: the next set goes out before this one is multiplied.
  constexpr int kPair = 2 * kK, kSet = kAhead / 2 * WAVES;
  const int pairs = (a.K + kPair - 1) / kPair;
  floatx4 c[TOKENS][R];
#pragma unroll
  for (int t = 0; t < TOKENS; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) c[t][r] = floatx4{0.f, 0.f, 0.f, 0.f};
  Frag fx[2][kAhead][TOKENS], fw[2][kAhead][R];
  const auto load = [&](int set, int p0) {
    // whole sets without a test a load; what lies behind K only in a last one
    if ((p0 + (kAhead / 2 - 1) * WAVES + 1) * kPair <= a.K) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = (p0 + (u >> 1) * WAVES) * kPair + 2 * kq + (u & 1) * Step<T>::kGroup;
#pragma unroll
        for (int r = 0; r < R; ++r) fw[set][u][r] = row16<T>(w[r], k);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) fx[set][u][t] = row16<T>(x[t], k);
      }
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int k = (p0 + (u >> 1) * WAVES) * kPair + 2 * kq + (u & 1) * Step<T>::kGroup;
#pragma unroll
        for (int r = 0; r < R; ++r) fw[set][u][r] = row16_cut<T>(w[r], k, a.K);
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) fx[set][u][t] = row16_cut<T>(x[t], k, a.K);
      }
    }
  };
  const auto multiply = [&](int set) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int t = 0; t < TOKENS; ++t)
#pragma unroll
        for (int r = 0; r < R; ++r) c[t][r] = Step<T>::mfma(fw[set][u][r], fx[set][u][t], c[t][r]);
  };
  int p = wave;
  if (p < pairs) load(0, p);
  while (p < pairs) {
    if (p + kSet >= pairs) {
      multiply(0);
      break;
    }
    load(1, p + kSet);
    multiply(0);
    p += 2 * kSet;
    if (p >= pairs) {
      multiply(1);
      break;
    }
    load(0, p);
    multiply(1);
  }
#pragma unroll
  for (int t = 0; t < TOKENS; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) part[wave][t * R + r][lane] = c[t][r];
  __syncthreads();
  if (wave >= TOKENS) return;   // a wavefront for each tile of tokens
  floatx4 sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] = part[0][wave * R + r][lane];
#pragma unroll
    for (int v = 1; v < WAVES; ++v) sum[r] += part[v][wave * R + r][lane];
  }
  epi.template tile<R>(sum, m0 + 16 * wave + i16, n0 + 4 * (lane >> 4), a.M, a.N);
}

template <class T, int TOKENS, int R, bool PAIR, class Epi>
hipError_t launch_skinny_tokens(const SkinnyArgs &a, const Epi &epi, unsigned blocks, hipStream_t stream) {
  const unsigned tiles = (unsigned)((a.M + 16 * TOKENS - 1) / (16 * TOKENS));
  // few workgroups: sixteen wavefronts share a workgroup's k (eight with two tiles of tokens, whose registers allow no more);
  // short rows: four, so that each has a set and one ahead
  constexpr int kMost = TOKENS == 1 ? 16 : 8;
  if ((long)a.K * (int)sizeof(T) <= 2048) skinny_kernel<T, TOKENS, R, PAIR, 4, Epi><<<dim3(blocks, tiles), dim3(256), 0, stream>>>(a, epi);
  else if ((int)(blocks * tiles) < chip().cus) skinny_kernel<T, TOKENS, R, PAIR, kMost, Epi><<<dim3(blocks, tiles), dim3(64 * kMost), 0, stream>>>(a, epi);
  else skinny_kernel<T, TOKENS, R, PAIR, 8, Epi><<<dim3(blocks, tiles), dim3(512), 0, stream>>>(a, epi);
  return hipGetLastError();
}
// MOST: rows at most that the caller sends here
template <class T, int R, bool PAIR, int MOST, class Epi>
hipError_t launch_skinny(const SkinnyArgs &a, const Epi &epi, hipStream_t stream) {
  // The second sixteen tokens share their weights' loads, or take workgroups of their own where the columns leave half the compute
  // units empty (24 x 784 x 500 in single precision: 15.3 us shared, 11.6 apart; 24 x 1000 x 2730 bf16: 11.7 against 13.2).
  constexpr int kEach = PAIR ? kSkinnyColumns : R * kSkinnyColumns;
  const unsigned blocks = (unsigned)((a.N + kEach - 1) / kEach);
  if constexpr (MOST > 16) {
    if (a.M > 16 && 2 * (int)blocks > chip().cus) return launch_skinny_tokens<T, 2, R, PAIR>(a, epi, blocks, stream);
  }
  return launch_skinny_tokens<T, 1, R, PAIR>(a, epi, blocks, stream);
}

// four neighbours of a row
template <class T>
__device__ __forceinline__ void store4(T *p, const float (&v)[4], int n) {
  typedef T V __attribute__((ext_vector_type(4)));
  typedef V Any __attribute__((aligned(sizeof(T))));
  if (n >= 4) {
    *reinterpret_cast<Any *>(p) = V{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = (T)v[j];
  }
}

template <class T>
struct SkinnyStore {
  T *c;
  template <int R>
  __device__ __forceinline__ void tile(const floatx4 (&v)[R], int m, int n, int M, int N) const {
    if (m >= M) return;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int at = n + kSkinnyColumns * r;
      const float o[4] = {v[r][0], v[r][1], v[r][2], v[r][3]};
      if (at < N) store4<T>(c + (long)m * N + at, o, N - at);
    }
  }
};

}  // namespace tile
}  // namespace dllk
