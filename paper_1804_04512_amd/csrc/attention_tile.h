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
// LDS: rows of a power of two of bfloat16 elements (single precision: three planes of them), each 16-byte group at place group ^ flip(row), chosen so that sixteen rows' same group
// (scores) and four rows' same 64 bytes (the transposing read) lie in different banks.
#pragma once

#include "tile_product.h"

namespace dllk {
namespace attn {

using namespace tile;

typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef float floatx8 __attribute__((ext_vector_type(8)));
// Eight elements as the 32 x 32 x 16 products take them.  Single precision is three bfloat16 parts of each number (split3): six products on
// a pipe of sixteen times the rate.
template <class T> struct FragOf;
template <> struct FragOf<bf16> { typedef bf16x8 Type; };
template <> struct FragOf<float> { typedef Split Type; };
template <class T> using Frag = typename FragOf<T>::Type;
template <class T> constexpr int planes() { return sizeof(T) == 2 ? 1 : 3; }

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;

// What makes exponents to the base 2 of scores.  A masked score of -infinity stays one where the scale is 0: the smallest number takes its place, with
// which no score passes 2^-21.
__device__ __forceinline__ float factor_of(float scale) { return fmaxf(fabsf(scale) * kLog2e, 0x1p-149f); }

// c += a b over sixteen: a's 32 rows become c's registers, b's its lanes
__device__ __forceinline__ floatx16 mma(bf16x8 a, bf16x8 b, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx16 mma(const Split &a, const Split &b, floatx16 c) { return mfma6(a, b, c); }

__device__ __forceinline__ Split split_of(const floatx8 &v) { return split3(floatx4{v[0], v[1], v[2], v[3]}, floatx4{v[4], v[5], v[6], v[7]}); }

// Registers 8 s to 8 s + 7 of a 32 x 32 result as a fragment; bfloat16 is rounded to nearest
template <class T>
__device__ __forceinline__ Frag<T> frag_of(const floatx16 &c, int s) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (bf16)c[8 * s + j];
    return f;
  } else {
    floatx8 f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = c[8 * s + j];
    return split_of(f);
  }
}
// the token of a 32 x 32 result's register, without the lane half's 4
__device__ __forceinline__ constexpr int token_of(int r) { return 8 * (r >> 2) + (r & 3); }

// Rows of bfloat16 in LDS, of numbers or of one of their parts
template <int DP>
struct Tile {
  static constexpr int kPitch = DP <= 64 ? 64 : DP <= 128 ? 128 : 256;   // elements of a row
  static constexpr int kRowBytes = kPitch * 2, kGroups = kRowBytes / 16;
  static_assert(DP % 32 == 0, "");
  static __device__ __forceinline__ int flip(int row) {
    return kGroups == 8 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

// NR tokens' rows from memory into LDS, for a loop over tiles of them: `start` sends the first tile on its way; `turn`, called by everyone behind a
// barrier at which the former tile is done with and, `landed`, this one has come, sends the next one on its way and says where this one lies.  What
// lies behind the last row, and behind a row's dim elements, is zeros.
//
// bfloat16 goes straight into LDS, the tiles into the halves of the area in turn.  Single precision comes through registers, where it is split once for
// all wavefronts, and has one area, which `turn` writes: `written` has to follow.
template <class T, int DP, int NR, int THREADS>
struct Stager;

template <int DP, int NR, int THREADS>
struct Stager<bf16, DP, NR, THREADS> {
  typedef Tile<DP> G;
  static constexpr int kTile = NR * G::kRowBytes, kBytes = 2 * kTile, kIts = kTile / (16 * THREADS);
  static_assert(kTile % (16 * THREADS) == 0, "whole steps");
  char *area;
  long ld;          // bytes from row to row
  int dim_bytes;
  bool whole;       // rows come in 16-byte groups from multiples of four bytes
  unsigned off[kIts];

  __device__ __forceinline__ void init(char *area_, const void *p, long ld_, int dim) {
    area = area_;
    ld = ld_ * 2;
    dim_bytes = dim * 2;
    whole = ((ld | (long)(uintptr_t)p) & 3) == 0 && dim_bytes % 16 == 0;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int at = it * THREADS + (int)threadIdx.x, row = at / G::kGroups, group = (at % G::kGroups) ^ G::flip(row);
      off[it] = group * 16 < dim_bytes ? (unsigned)(row * ld) + 16u * group : kOutOfRange;
    }
  }
  __device__ __forceinline__ void load(char *lds, int wave, const bf16 *base, int row0, int rows) const {
    const int left = max(0, min(rows - row0, NR));
    const char *p = (const char *)base + (long)row0 * ld;
    if (whole) {
      const uintx4 rs = buffer_of(p, left > 0 ? (unsigned)((left - 1) * ld) + dim_bytes : 0u);
      const unsigned at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
#pragma unroll
      for (int it = 0; it < kIts; ++it) load_to_lds(rs, off[it], at + (it * THREADS + wave * 64) * 16);
      return;
    }
    const int dim = dim_bytes / 2;
#pragma unroll 1
    for (int it = 0; it < kIts; ++it) {
      const int at = it * THREADS + (int)threadIdx.x, row = at / G::kGroups, col = ((at % G::kGroups) ^ G::flip(row)) * 8;
      const bf16 *src = reinterpret_cast<const bf16 *>(p + row * ld);
      bf16 *dst = reinterpret_cast<bf16 *>(lds + at * 16);
#pragma unroll
      for (int j = 0; j < 8; ++j) dst[j] = row < left && col + j < dim ? src[col + j] : (bf16)0.0f;
    }
  }
  __device__ __forceinline__ void start(int wave, const bf16 *base, int row0, int rows) { load(area, wave, base, row0, rows); }
  // tiles alternate between the halves: `odd` is the next one's
  __device__ __forceinline__ const char *turn(int wave, int odd, const bf16 *base, int next_row0, int rows) {
    load(area + odd * kTile, wave, base, next_row0, rows);
    return area + (odd ^ 1) * kTile;
  }
};

template <int DP, int NR, int THREADS>
struct Stager<float, DP, NR, THREADS> {
  typedef Tile<DP> G;
  static constexpr int kTile = NR * G::kRowBytes, kBytes = 3 * kTile, kIts = kTile / (16 * THREADS);
  static_assert(kTile % (16 * THREADS) == 0, "whole steps");
  char *area;
  long ld;
  int dim;
  floatx8 held[kIts];

  __device__ __forceinline__ void init(char *area_, const void *, long ld_, int dim_) {
    area = area_;
    ld = ld_;
    dim = dim_;
  }
  static __device__ __forceinline__ int row_of(int it) { return (it * THREADS + (int)threadIdx.x) / G::kGroups; }
  static __device__ __forceinline__ int col_of(int it) { return ((it * THREADS + (int)threadIdx.x) % G::kGroups ^ G::flip(row_of(it))) * 8; }
  __device__ __forceinline__ void start(int, const float *base, int row0, int rows) {
    const int left = rows - row0;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      Eight<float> e;
      const int row = row_of(it), n = row < left ? dim - col_of(it) : 0;
      e.load(base + (long)(row0 + row) * ld + col_of(it), n);
      held[it] = e.v;
    }
  }
  __device__ __forceinline__ const char *turn(int wave, int, const float *base, int next_row0, int rows) {
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const Split s = split_of(held[it]);
#pragma unroll
      for (int k = 0; k < 3; ++k) *reinterpret_cast<bf16x8 *>(area + k * kTile + (it * THREADS + (int)threadIdx.x) * 16) = s.p[k];
    }
    start(wave, base, next_row0, rows);
    return area;
  }
};

// All that this wavefront has on its way into LDS has arrived: the loads that go there, and the stores of rows that do not come whole.  It stands in front
// of every barrier behind which others may write or read those places, and behind a loop over tiles, whose last `turn` still sends a tile of zeros.
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
// The barrier in front of `turn`
template <class T>
__device__ __forceinline__ void landed() {
  if constexpr (sizeof(T) == 2) arrived();
  barrier();
}
// The one behind it
template <class T>
__device__ __forceinline__ void written() {
  if constexpr (sizeof(T) == 4) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  }
}

// A product's 0 for a token that a mask leaves out stays 0 only while the other operand is finite.  Where sums turn out not to be finite under a mask (outputs:
// not small, and without a mask too, as sums of large values may overflow on their way to a mean that does not), a
// workgroup takes its tiles again (or another launch's does): in those that the mask cuts, rows with such numbers lose them, and the lanes that see one of these rows are
// told, whose results are NaN.  All of this is off the usual path but for one look at the sums and the registers that a second copy of the loop
// takes.  With it / without, microseconds: forward 16384 tokens in five sequences, 16 heads of 128 on 4, 310 / 305; 4096, 16 heads, 91.3 / 89.1, all keys seen 139 / 138; 777, 10.6 /
// 10.4; 1024 in single precision, 8 heads of 64 on 2, 25.1 / 24.8; the gradients of a training pass over 4096, 16 heads of 128, 373 / 373; 1024 in single precision 91.0 / 89.3.
constexpr int kCareful = 256;   // bytes of LDS for it
template <int N>
__device__ __forceinline__ bool all_finite(const floatx16 (&c)[N]) {
  float zero[4] = {};   // a finite number leaves it 0, any other makes it NaN
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) zero[r % 4] = __builtin_fmaf(c[i][r], 0.0f, zero[r % 4]);
  return (zero[0] + zero[1]) + (zero[2] + zero[3]) == 0.0f;
}
// Whether all sums are below 2^120, so that a few wavefronts' may be added up; what is not finite is not
template <int N>
__device__ __forceinline__ bool all_small(const floatx16 (&c)[N]) {
  float x[4] = {};   // finite as long as every sum's 2^8 fold is
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r % 4] = __builtin_fmaf(c[i][r], 256.0f, x[r % 4]);
#pragma unroll
  for (float &f : x) f -= f;   // 0 or NaN
  return (x[0] + x[1]) + (x[2] + x[3]) == 0.0f;
}
// An exponential follows the running maximum at up to 2^8 above it.  The power of two that brings the sum of that many of them below 1: products with it
// lose no digits, and sums of values that it has made weights of cannot pass the largest of them.
__device__ __forceinline__ int fold_of(int keys) { return 8 + 32 - __builtin_clz((unsigned)keys | 1u); }
__device__ __forceinline__ float power(int e) { return __builtin_bit_cast(float, (127 + e) << 23); }   // 2^e, -126 <= e <= 127
// Whether any of a workgroup's four wavefronts says so, once all of them are done with the tiles; its flags lie behind clear_rows's, so that no one
// needs to wait until all have read them
__device__ __forceinline__ bool anyone(bool here, char *lds, int wave) {
  unsigned *flags = reinterpret_cast<unsigned *>(lds + kCareful / 2);
  const unsigned any = __any(here) ? 1u : 0u;
  if ((threadIdx.x & 63) == 0) flags[wave] = any;
  __syncthreads();
  const unsigned all = flags[0] | flags[1] | flags[2] | flags[3];
  return __builtin_amdgcn_readfirstlane((int)all) != 0;
}
// Clears what is not finite in a tile of NR rows, by everyone; the first and the last row that had any, NR and -1 where none had
struct Cleared { int first, last; };
template <class T, int DP, int NR>
__device__ __forceinline__ Cleared clear_rows(char *tile, char *lds) {
  int *rows = reinterpret_cast<int *>(lds);
  if (threadIdx.x == 0) rows[0] = NR, rows[1] = -1;
  __syncthreads();
  for (int at = threadIdx.x; at < NR * Tile<DP>::kGroups; at += 256) {
    uintx4 keep = {~0u, ~0u, ~0u, ~0u};   // of all parts of a number, where all are numbers
#pragma unroll
    for (int k = 0; k < planes<T>(); ++k) {
      const uintx4 v = *reinterpret_cast<const uintx4 *>(tile + k * NR * Tile<DP>::kRowBytes + at * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) keep[j] &= ((v[j] & 0x7F80u) == 0x7F80u ? 0u : 0xFFFFu) | ((v[j] & 0x7F800000u) == 0x7F800000u ? 0u : 0xFFFF0000u);
    }
    if ((keep[0] & keep[1] & keep[2] & keep[3]) == ~0u) continue;
    const int row = at / Tile<DP>::kGroups;
    atomicMin(&rows[0], row);
    atomicMax(&rows[1], row);
#pragma unroll
    for (int k = 0; k < planes<T>(); ++k) *reinterpret_cast<uintx4 *>(tile + k * NR * Tile<DP>::kRowBytes + at * 16) &= keep;
  }
  __syncthreads();
  const Cleared c{rows[0], rows[1]};
  __syncthreads();
  return c;
}

// Fragments of a tile of NR rows in LDS for lane l: of scores, elements 16 s + 8 (l / 32) on of row x0 + l % 32; of sums over tokens, element
// d0 + l % 32 of the sixteen tokens from x0 on, in the order of a result's registers.  x0 is a multiple of 32 and of 16.
template <class T, int DP, int NR>
struct Reader {
  typedef Tile<DP> G;
  int row, half, low;     // scores
  int trow, tgroup, tlow, tbyte;   // sums over tokens
  __device__ __forceinline__ explicit Reader(int lane) {
    row = (lane & 31) * G::kRowBytes;
    half = lane >> 5;
    low = G::flip(lane & 31);
    const int i = lane & 15;
    trow = (4 * half + (i >> 2)) * G::kRowBytes;
    tgroup = 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    tlow = G::flip(4 * half + (i >> 2));
    tbyte = 8 * (i & 1);
  }
  __device__ __forceinline__ bf16x8 along_plane(const char *p, int s) const { return *reinterpret_cast<const bf16x8 *>(p + (((2 * s + half) ^ low) << 4)); }
  __device__ __forceinline__ bf16x8 across_plane(const char *p, int d0) const {
    typedef __attribute__((address_space(3))) shortx4 *Lp;
    const int g = d0 / 8 + tgroup;
    // eight rows on, flip differs in its second bit, whatever the row
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p + ((g ^ tlow) << 4) + tbyte));
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p + 8 * G::kRowBytes + ((g ^ tlow ^ 2) << 4) + tbyte));
    const shortx8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
  }
  __device__ __forceinline__ Frag<T> along(const char *lds, int x0, int s) const {
    const char *p = lds + x0 * G::kRowBytes + row;
    if constexpr (sizeof(T) == 2) {
      return along_plane(p, s);
    } else {
      Split f;
#pragma unroll
      for (int k = 0; k < 3; ++k) f.p[k] = along_plane(p + k * NR * G::kRowBytes, s);
      return f;
    }
  }
  __device__ __forceinline__ Frag<T> across(const char *lds, int x0, int d0) const {
    const char *p = lds + x0 * G::kRowBytes + trow;
    if constexpr (sizeof(T) == 2) {
      return across_plane(p, d0);
    } else {
      Split f;
#pragma unroll
      for (int k = 0; k < 3; ++k) f.p[k] = across_plane(p + k * NR * G::kRowBytes, d0);
      return f;
    }
  }
};

// A token's row straight from memory, kept as fragments of lane half `half`, zeros behind dim elements.  Single precision of more than 128
// elements is split where it is used, as its parts would not fit the registers.
template <class T, int DP>
struct RowFrags {
  static constexpr bool kLate = sizeof(T) == 4 && DP > 128;
  typedef typename std::conditional<kLate, floatx8, Frag<T>>::type Kept;
  Kept f[DP / 16];
  __device__ __forceinline__ void load(const T *p, int dim, int half, bool negate = false) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      Eight<T> e;
      const int at = 16 * s + 8 * half;
      e.load(p + at, dim - at);
      if (negate) e.v = -e.v;
      if constexpr (sizeof(T) == 2 || kLate) f[s] = e.v;
      else f[s] = split_of(e.v);
    }
  }
  __device__ __forceinline__ Frag<T> operator[](int s) const {
    if constexpr (kLate) return split_of(f[s]);
    else return f[s];
  }
};

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

// The same unrounded, into a row of sums whose length is a multiple of four
template <int N>
__device__ __forceinline__ void store_sums(float *p, const floatx16 (&c)[N], int ld, int half, float factor = 1.0f) {
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (32 * i + 8 * q + 4 * half < ld)
        *reinterpret_cast<floatx4 *>(p + 32 * i + 8 * q + 4 * half) = floatx4{c[i][4 * q], c[i][4 * q + 1], c[i][4 * q + 2], c[i][4 * q + 3]} * factor;
}

// Here is where a fragment's value is made: it is not moved behind what follows
__device__ __forceinline__ void made(bf16x8 &f) {
  uintx4 v = __builtin_bit_cast(uintx4, f);
  asm volatile("" : "+v"(v));
  f = __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ void made(Split &f) {
#pragma unroll
  for (int k = 0; k < 3; ++k) made(f.p[k]);
}

// Over both halves of the wavefront's lanes.  The swap of the one's upper with the other's lower half leaves both halves' values in two registers.
struct Halves { float a, b; };
__device__ __forceinline__ Halves halves(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const unsigned a = r[0], b = r[1];
  return Halves{__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)};
}
__device__ __forceinline__ float most_of_halves(float v) { const Halves h = halves(v); return fmaxf(h.a, h.b); }
__device__ __forceinline__ float sum_of_halves(float v) { const Halves h = halves(v); return h.a + h.b; }

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

// Work split along the axis that a workgroup goes over: part k of n of a workgroup's `turns`, its sums left in 32 bits for a launch that adds them
// up in order.  Taken where there are too few workgroups for the chip.
constexpr int kMostParts = 16;
struct Parts {
  int n = 1;
  float *sums[2] = {nullptr, nullptr};   // [n][tokens][heads][ld]: the parts' own outputs; or a gradient's sums, or both gradients'
  float *ml = nullptr;                   // [n][heads][tokens][2]: maximum in the exponent's base, sum
  int ld = 0;                            // head_dim in whole fours
};
__device__ __forceinline__ int turn_from(int part, int parts, int turns) { return (int)((long)part * turns / parts); }
// The n that fills the chip's `slots` places for workgroups, with `least` turns a part left on average; grid: workgroups of one part's launch,
// empty ones too.  Forced n, microseconds of a training pass: 2001 ragged tokens, six heads of 80 in single precision, n = 1 / 2 / 3 / 4 / 6: 460 / 266 / 230 / 202 / 205;
// 1024 tokens, 8 heads of 64 on 2, n = 1 / 4 / 6 / 12: 121 / 69 / 55 / 49; 6000 tokens, 8 heads of 128, n = 1 / 2 / 4: 503 / 452 / 528.
inline int parts_of(long workgroups, long grid, long slots, long turns, long least) {
  long n = (slots + workgroups - 1) / workgroups;
  for (const long most : {turns / least, kMaxGrid / grid, (long)kMostParts}) n = n < most ? n : most;
  return (int)(n > 1 ? n : 1);
}

// What `call` makes of the smallest instance that holds a head
template <class F>
auto instance(int dim, const F &call) {
  if (dim <= 32) return call(std::integral_constant<int, 32>{});
  if (dim <= 64) return call(std::integral_constant<int, 64>{});
  if (dim <= 96) return call(std::integral_constant<int, 96>{});
  if (dim <= 128) return call(std::integral_constant<int, 128>{});
  return call(std::integral_constant<int, 256>{});
}

}  // namespace attn
}  // namespace dllk
