// What the attention kernels share: tiles of tokens' rows in LDS, fragments for the matrix instructions, and which sequence a
// workgroup's tile belongs to.
//
// Every product is one of two kinds.  Scores (q k, do v) contract over a head's elements: a lane of the 32 x 32 x 16 product holds
// eight neighbouring elements of its token's row, for both operands.  The others (p v, ds k, and their transposes) contract over
// tokens: one operand is the scores' own result.  A result's register r of lane half h is token 8 (r / 4) + 4 h + r % 4 of its 32, so
// registers 8 s to 8 s + 7 are a fragment of sixteen tokens in the order (h, j) -> 16 s + 8 (j / 4) + 4 h + j % 4.  The sum over
// tokens may be taken in any order, so the other operand is read from LDS in that same order (two transposing reads) and the scores
// never leave their registers.
//
// LDS: rows of a power of two of elements, each 16-byte group at place group ^ flip(row), chosen so that sixteen rows' same group
// (scores) and four rows' same 64 bytes (the transposing read) lie in different banks.
#pragma once

#include "tile_product.h"

namespace dllk {
namespace attn {

using namespace tile;

typedef float floatx8 __attribute__((ext_vector_type(8)));
template <class T> struct FragOf;
template <> struct FragOf<bf16> { typedef bf16x8 Type; };
template <> struct FragOf<float> { typedef floatx8 Type; };
template <class T> using Frag = typename FragOf<T>::Type;

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// c += a b over sixteen: a's 32 rows become c's registers, b's its lanes
__device__ __forceinline__ floatx16 mma(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx16 mma(floatx8 a, floatx8 b, floatx16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

// Registers 8 s to 8 s + 7 of a 32 x 32 result as a fragment; bfloat16 is rounded to nearest
template <class T>
__device__ __forceinline__ Frag<T> frag_of(const floatx16 &c, int s) {
  Frag<T> f;
#pragma unroll
  for (int j = 0; j < 8; ++j) f[j] = (T)c[8 * s + j];
  return f;
}
// the token of a 32 x 32 result's register, without the lane half's 4
__device__ __forceinline__ constexpr int token_of(int r) { return 8 * (r >> 2) + (r & 3); }

template <class T, int DP>
struct Tile {
  static constexpr int kPitch = DP <= 64 ? 64 : DP <= 128 ? 128 : 256;   // elements of a row
  static constexpr int kRowBytes = kPitch * (int)sizeof(T), kGroups = kRowBytes / 16;
  static constexpr int kSteps = DP / 16, kBlocks = DP / 32;
  static_assert(DP % 32 == 0 && kRowBytes >= 128, "");
  static __device__ __forceinline__ int flip(int row) {
    return kGroups == 8 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

// NR tokens' rows from memory into LDS
template <class T, int DP, int NR, int THREADS>
struct Stager {
  typedef Tile<T, DP> G;
  static constexpr int kBytes = NR * G::kRowBytes, kIts = kBytes / (16 * THREADS), kLoads = kIts;
  static_assert(kBytes % (16 * THREADS) == 0, "whole steps");
  const char *base;
  long ld;          // bytes from row to row
  int dim_bytes;
  bool whole;       // rows come in 16-byte groups from multiples of four bytes
  unsigned off[kIts];

  __device__ __forceinline__ void init(const void *p, long ld_, int dim, int t) {
    base = (const char *)p;
    ld = ld_ * (long)sizeof(T);
    dim_bytes = dim * (int)sizeof(T);
    whole = ((ld | (long)(uintptr_t)p) & 3) == 0 && dim_bytes % 16 == 0;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int at = it * THREADS + t, row = at / G::kGroups, group = (at % G::kGroups) ^ G::flip(row);
      off[it] = group * 16 < dim_bytes ? (unsigned)(row * ld) + 16u * group : kOutOfRange;
    }
  }
  // rows row0 to row0 + NR of `rows`; what lies behind them, and behind a row's dim elements, is zeros
  __device__ __forceinline__ void load(char *lds, int wave, int row0, int rows) const {
    const int left = max(0, min(rows - row0, NR));
    const char *p = base + (long)row0 * ld;
    if (whole) {
      const uintx4 rs = buffer_of(p, left > 0 ? (unsigned)((left - 1) * ld) + dim_bytes : 0u);
      const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
#pragma unroll
      for (int it = 0; it < kIts; ++it) load_to_lds(rs, off[it], at + (it * THREADS + wave * 64) * 16);
      return;
    }
    constexpr int kE = 16 / (int)sizeof(T);
    const int t = (int)(threadIdx.x % THREADS), dim = dim_bytes / (int)sizeof(T);
#pragma unroll 1
    for (int it = 0; it < kIts; ++it) {
      const int at = it * THREADS + t, row = at / G::kGroups, col = ((at % G::kGroups) ^ G::flip(row)) * kE;
      const T *src = reinterpret_cast<const T *>(p + row * ld);
      T *dst = reinterpret_cast<T *>(lds + at * 16);
#pragma unroll
      for (int j = 0; j < kE; ++j) dst[j] = row < left && col + j < dim ? src[col + j] : (T)0.0f;
    }
  }
};

// Fragments of a tile in LDS for lane l: of scores, elements 16 s + 8 (l / 32) on of row x0 + l % 32; of sums over tokens, element
// d0 + l % 32 of the sixteen tokens from x0 on, in the order of a result's registers.  x0 is a multiple of 32 and of 16.
template <class T, int DP>
struct Reader {
  typedef Tile<T, DP> G;
  int row, half, low;     // scores
  int trow, tgroup, tlow, tbyte;   // sums over tokens
  __device__ __forceinline__ explicit Reader(int lane) {
    row = (lane & 31) * G::kRowBytes;
    half = lane >> 5;
    low = G::flip(lane & 31);
    const int i = lane & 15;
    if (sizeof(T) == 2) {
      trow = (4 * half + (i >> 2)) * G::kRowBytes;
      tgroup = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      tlow = G::flip(4 * half + (i >> 2));
      tbyte = 8 * (i & 1);
    } else {
      trow = 4 * half * G::kRowBytes;
      tgroup = (lane & 31) >> 2;
      tlow = 0;
      tbyte = 4 * (lane & 3);
    }
  }
  __device__ __forceinline__ Frag<T> along(const char *lds, int x0, int s) const {
    const char *p = lds + x0 * G::kRowBytes + row;
    if constexpr (sizeof(T) == 2) {
      return *reinterpret_cast<const bf16x8 *>(p + (((2 * s + half) ^ low) << 4));
    } else {
      const int g = (4 * s + 2 * half) ^ low;
      const floatx4 a = *reinterpret_cast<const floatx4 *>(p + (g << 4)), b = *reinterpret_cast<const floatx4 *>(p + ((g ^ 1) << 4));
      return floatx8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
  }
  __device__ __forceinline__ Frag<T> across(const char *lds, int x0, int d0) const {
    const char *p = lds + x0 * G::kRowBytes + trow;
    if constexpr (sizeof(T) == 2) {
      typedef __attribute__((address_space(3))) shortx4 *Lp;
      const int g = d0 / 8 + tgroup;
      // eight rows on, flip differs in its second bit, whatever the row
      const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p + ((g ^ tlow) << 4) + tbyte));
      const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p + 8 * G::kRowBytes + ((g ^ tlow ^ 2) << 4) + tbyte));
      const shortx8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
      return __builtin_bit_cast(bf16x8, v);
    } else {
      floatx8 v;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int r = 8 * (j >> 2) + (j & 3);   // of sixteen, and 4 * half more
        v[j] = *reinterpret_cast<const float *>(p + r * G::kRowBytes + (((d0 / 4 + tgroup) ^ G::flip(r + 4 * half)) << 4) + tbyte);
      }
      return v;
    }
  }
};

// A token's row straight from memory: the fragments of lane half `half`, zeros behind dim elements
template <class T, int DP>
__device__ __forceinline__ void load_row(Frag<T> (&f)[DP / 16], const T *p, int dim, int half) {
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    Eight<T> e;
    const int at = 16 * s + 8 * half;
    e.load(p + at, dim - at);
    f[s] = e.v;
  }
}

// A lane's part of a result's row (32 x 32 results over elements d0 = 0, 32, ..): element 32 i + 8 q + 4 half + j from register 4 q + j
template <class T, int N>
__device__ __forceinline__ void store_row(T *p, const floatx16 (&c)[N], float factor, int dim, int half) {
  typedef T V __attribute__((ext_vector_type(4)));
  typedef V Any __attribute__((aligned(sizeof(T))));
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = 32 * i + 8 * q + 4 * half;
      V v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (T)(c[i][4 * q + j] * factor);
      if (at + 4 <= dim) {
        *reinterpret_cast<Any *>(p + at) = v;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + j < dim) p[at + j] = v[j];
      }
    }
}

// What the other half of the wavefront's lanes holds for the same column
__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// Packed sequences in tiles of B tokens: sequence s has its tiles from starts[s] / B + s on, which leaves room for the last, part-filled one
// of each, so no table of tiles is needed.  The last s with starts[s] / B + s <= t is found by sixty-four probes at a time.
struct Place {
  int sequence, first;   // of the packed tokens
  int count, at;         // tokens of the sequence; the tile's first among them.  at >= count: no tile
};
__device__ __forceinline__ int start_of(const int *starts, int s, int tokens) { return max(0, min(starts[s], tokens)); }
__device__ __forceinline__ Place place_of(const int *starts, int sequences, int tokens, int tile, int B) {
  const int lane = threadIdx.x & 63;
  int low = 0, n = sequences;   // the answer lies in [low, low + n)
  while (n > 1) {
    const int step = (n + 63) / 64, s = low + lane * step;
    const bool before = lane * step < n && start_of(starts, s, tokens) / B + s <= tile;
    const int hits = __popcll(__ballot(before));
    const int take = max(hits - 1, 0) * step;
    n = min(step, n - take);
    low += take;
  }
  low = __builtin_amdgcn_readfirstlane(low);
  Place p;
  p.sequence = low;
  p.first = __builtin_amdgcn_readfirstlane(start_of(starts, low, tokens));
  p.count = __builtin_amdgcn_readfirstlane(start_of(starts, low + 1, tokens)) - p.first;
  p.at = (tile - p.first / B - low) * B;
  if (p.at < 0) p.at = p.count;   // starts that do not grow
  return p;
}
inline long tiles_of(int tokens, int sequences, int B) { return (long)tokens / B + sequences; }

}  // namespace attn
}  // namespace dllk
