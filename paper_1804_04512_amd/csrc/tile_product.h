// Matrix products of the large-model operators on MFMA, gfx950: operands in bfloat16 or single precision, sums in 32 bits.
//
//   C(m, n) = sum_k A(m, k) * B(n, k)
//
// Each operand lies either along k ("KC": element (x, k) at p[x * ld + k]) or across it ("KS": p[k * ld + x]), so the three
// forms of a layer's products (forward KC KC, data gradient KC KS, weight gradient KS KS) need no transposed copies.
//
// A workgroup owns a BM x BN tile of C and walks k in slabs of 128 bytes a row (64 bf16, 32 fp32).  Slabs go from global
// memory straight into LDS (16 bytes a lane from any multiple of four, no registers in between), the next ones on their way while
// the current one is multiplied.  Every access is range checked by the buffer descriptor: rows behind the end read as zeros,
// columns behind K are sent out of range where the last slab is not whole, and where K ends inside a 16-byte group what follows
// it is cleared in LDS, so no operand needs padding.
//
// LDS layouts.  The hardware writes a wavefront's 64 x 16 bytes in lane order, so a swizzle is made by permuting which
// global bytes a lane fetches.  KC: rows of 128 bytes, 16-byte group c of row r at place c ^ ((r >> 1) & 7), so that the
// sixteen lanes that read at a time (16 rows, one group each) touch all 64 banks once (c ^ (r & 7), made for 32 banks, had two
// lanes on each: half of all LDS cycles).  KS bf16: rows of X columns, 64-byte block b of
// row k at place b ^ g(k) with g from bits 0, 1 and 3 of k; the transposing read ds_read_b64_tr_b16 turns four rows of
// sixteen columns into four k's a lane.  KS fp32: four 4-byte reads a fragment, 128-byte block b of row k at b ^ bit 2 of k.
//
// MFMA: 32x32x16 bf16; for fp32 the same on numbers split into three bf16 parts, or 32x32x2 with the four floats of a 16-byte group
// as four steps (the order of k within a slab is the same permutation for both operands).  B rides on the first operand, so a lane holds one row m of C and runs
// of four neighbouring n.  The epilogue passes 32 x 64 pieces of C through LDS, one wavefront at a time, so that outputs
// leave as whole rows of 64 columns.
#pragma once

#include "large_ops.h"

#include <type_traits>

namespace dllk {
namespace tile {

typedef __bf16 bf16;
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef short shortx8 __attribute__((ext_vector_type(8)));

constexpr int kSlabBytes = 128;              // of one row along k
constexpr unsigned kOutOfRange = 0xFFFFFFF0u;
constexpr int kStageLd = 68;                 // floats: row stride of an epilogue piece (64 or 32 columns)

template <class T> struct Elem;
template <> struct Elem<bf16> { static constexpr int kSlab = 64; typedef bf16x8 Frag; };
template <> struct Elem<float> { static constexpr int kSlab = 32; typedef floatx4 Frag; };

struct Operand {
  const void *p = nullptr;
  long ld = 0;   // elements; rows start at multiples of 4 bytes
};

struct ProductArgs {
  int M = 0, N = 0;
  // segment 0 and, where K[1] > 0, a second pair of operands whose products are added to the first's;
  // or two products of one shape side by side (problems == 2), each with its own operands and outputs
  Operand A[2], B[2];
  int K[2] = {0, 0};
  int problems = 1;
  // Rows that exist as the device counts them: M (m_rows) and K[0] (k_rows) become what *p leaves behind `first`.
  const int *m_rows = nullptr, *k_rows = nullptr;
  int first = 0;
  int slabs_per_split = 1 << 30;
  int tiles_m = 0, tiles_n = 0, splits = 1;
};

__device__ __forceinline__ int rows_left(const int *rows, int first, int most) {
  return rows ? max(0, min(most, *rows - first)) : most;
}

// Workgroups are dealt to the 8 XCDs in turn; each XCD gets a contiguous run of tiles (of one part of k or problem after the
// other), eight tile rows high, so that the 32 tiles it works on at a time share their operands in its L2.
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int units, int *tm, int *tn, int *unit) {
  const int tiles = tiles_m * tiles_n, n = tiles * units, q = n >> 3, r = n & 7, xcd = id & 7, i = id >> 3;
  int t = xcd * q + min(xcd, r) + i;
  *unit = t / tiles;
  t -= *unit * tiles;
  constexpr int kRows = 8;
  const int group = t / (kRows * tiles_n), first = group * kRows, rows = min(kRows, tiles_m - first), at = t - group * kRows * tiles_n;
  *tm = first + at % rows;
  *tn = at / rows;
}

// ------------------------------------------------------------------------------------------------ loading
// A raw buffer's descriptor: 48-bit address, extent in bytes; what lies outside reads as zeros.
__device__ __forceinline__ uintx4 buffer_of(const char *p, unsigned bytes) {
  const uint64_t at = (uint64_t)p;
  return uintx4{(unsigned)__builtin_amdgcn_readfirstlane((int)at), (unsigned)__builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xFFFF),
                (unsigned)__builtin_amdgcn_readfirstlane((int)bytes), 0x00020000u};
}
// 16 bytes a lane from the buffer to 1024 bytes of LDS in lane order.  Written out because the compiler, which sees that the
// builtin writes LDS, waits for it before any transposing LDS read, of the other slab too.  It has no output register, and
// the caller waits for it (vmcnt) before the barrier behind which the slab is read.
__device__ __forceinline__ void load_to_lds(const uintx4 &rs, unsigned off, unsigned lds) {
  const unsigned at = (unsigned)__builtin_amdgcn_readfirstlane((int)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(rs) : "memory");   // m0 is never the compiler's to keep
}
// the swizzle of a KS bf16 row of X columns: which of its 64-byte blocks change places
template <int X>
__device__ __forceinline__ int mix(int k) { return X >= 256 ? (k & 3) | ((k >> 1) & 4) : X >= 128 ? k & 3 : X >= 64 ? (k >> 1) & 1 : 0; }

// One operand's slab of X rows (KC) or X columns (KS).
template <class T, int X, bool KC, int THREADS>
struct Slab {
  static constexpr int kK = Elem<T>::kSlab;
  static constexpr int kBytes = X * kSlabBytes;
  static constexpr int kIts = kBytes / (16 * THREADS);
  static constexpr int kRowGroups = KC ? 8 : X * (int)sizeof(T) / 16;   // 16-byte groups of a row in LDS
  static_assert(kBytes % (16 * THREADS) == 0 && (THREADS / kRowGroups) * kRowGroups == THREADS, "whole rows a step");
  static constexpr int kStep = THREADS / kRowGroups;                     // rows between a thread's loads

  unsigned off[kIts];   // bytes from the slab's first element

  static __device__ __forceinline__ int group_of(int row, int place) {
    if (KC) return place ^ ((row >> 1) & 7);
    if (sizeof(T) == 2) return (((place >> 2) ^ mix<X>(row)) << 2) | (place & 3);
    return X >= 64 ? place ^ (((row >> 2) & 1) << 3) : place;
  }
  __device__ __forceinline__ void init(long ld, int t) {   // t: the thread among the THREADS that load this slab
    const int place = t % kRowGroups, row0 = t / kRowGroups;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int row = row0 + it * kStep;
      off[it] = (unsigned)((long)row * ld * (int)sizeof(T)) + 16u * group_of(row, place);
    }
  }
  // x0: the tile's first row (KC) or column (KS); k0: the slab's first k; X_, K: extents of the operand
  // and [from, to) the loads of kIts that are made (constants)
  __device__ __forceinline__ void load(unsigned lds, int wave, const Operand &o, int x0, int X_, int k0, int K, int from, int to) const {
    if (from >= to) return;
    const long first = KC ? (long)x0 * o.ld + k0 : (long)k0 * o.ld + x0;
    const long end = KC ? (long)X_ * o.ld : (long)K * o.ld;
    long bytes = (end - first) * (long)sizeof(T);
    bytes = bytes < 0 ? 0 : (bytes > 0xFFFFFF00L ? 0xFFFFFF00L : bytes);
    const uintx4 rs = buffer_of((const char *)o.p + first * (long)sizeof(T), (unsigned)bytes);
    if (KC && k0 + kK > K) {   // uniform: only a last slab
      const int t = (int)(threadIdx.x % THREADS), place = t % kRowGroups, row0 = t / kRowGroups;
#pragma unroll
      for (int it = 0; it < kIts; ++it) {
        if (it < from || it >= to) continue;
        const bool out = k0 + group_of(row0 + it * kStep, place) * (16 / (int)sizeof(T)) >= K;
        load_to_lds(rs, out ? kOutOfRange : off[it], lds + (it * THREADS + wave * 64) * 16);
      }
      return;
    }
#pragma unroll
    for (int it = 0; it < kIts; ++it)
      if (it >= from && it < to) load_to_lds(rs, off[it], lds + (it * THREADS + wave * 64) * 16);
  }
};

// A gate's and an up projection's rows side by side: of each wavefront's WC columns the first half are gate rows and the
// second half the same rows of the up projection, so that a wavefront holds both factors of WC / 2 hidden units.
template <class T, int X, int WC, int THREADS>
struct PairSlab {
  typedef Slab<T, X, true, THREADS> Base;
  static constexpr int kBytes = Base::kBytes, kIts = Base::kIts;
  static_assert(WC % 16 == 0, "the eight rows of a wavefront's load lie in one projection");
  unsigned off[kIts];
  __device__ __forceinline__ void init(long ld, int t) {
    const int place = t & 7, row0 = t >> 3;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      const int row = row0 + it * Base::kStep;
      off[it] = (unsigned)((long)((row / WC) * (WC / 2) + row % (WC / 2)) * ld * (int)sizeof(T)) + 16u * Base::group_of(row, place);
    }
  }
  // x0: the tile's first hidden unit; H: hidden units
  __device__ __forceinline__ void load(unsigned lds, int wave, const Operand &gate, const Operand &up, int x0, int H, int k0, int K, int from, int to) const {
    if (from >= to) return;
    const long first = (long)x0 * gate.ld + k0;
    long bytes = ((long)H * gate.ld - first) * (long)sizeof(T);
    bytes = bytes < 0 ? 0 : (bytes > 0xFFFFFF00L ? 0xFFFFFF00L : bytes);
    const bool cut = k0 + Base::kK > K;   // uniform
    const int t = (int)(threadIdx.x % THREADS), place = t & 7, row0 = t >> 3;
#pragma unroll
    for (int it = 0; it < kIts; ++it) {
      if (it < from || it >= to) continue;
      const bool second = (wave * 8 + it * Base::kStep) % WC >= WC / 2;
      const uintx4 rs = buffer_of((const char *)(second ? up.p : gate.p) + first * (long)sizeof(T), (unsigned)bytes);
      const bool out = cut && k0 + Base::group_of(row0 + it * Base::kStep, place) * (16 / (int)sizeof(T)) >= K;
      load_to_lds(rs, out ? kOutOfRange : off[it], lds + (it * THREADS + wave * 64) * 16);
    }
  }
};

// A workgroup barrier that waits for nothing by itself (the callers count their loads) and that no LDS access moves across
__device__ __forceinline__ void barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ------------------------------------------------------------------------------------------------ fragments
// Lane l's part of a 32-row fragment at step s (of 4 a slab): row x0 + l % 32, 16-byte group 2 s + l / 32 along k.
template <class T, int X, bool KC>
struct FragReader;
template <class T, int X>
struct FragReader<T, X, true> {
  int row, half, low;
  __device__ __forceinline__ explicit FragReader(int lane) : row((lane & 31) * kSlabBytes), half(lane >> 5), low((lane >> 1) & 7) {}
  __device__ __forceinline__ typename Elem<T>::Frag operator()(const char *lds, int x0, int s) const {
    return *reinterpret_cast<const typename Elem<T>::Frag *>(lds + x0 * kSlabBytes + row + (((2 * s + half) ^ low) << 4));
  }
};
template <int X>
struct FragReader<bf16, X, false> {
  int base, g;
  __device__ __forceinline__ explicit FragReader(int lane) {
    const int i = lane & 15, k = 8 * (lane >> 5) + (i >> 2);
    base = k * X * 2 + (((lane >> 4) & 1) * 16 + 4 * (i & 3)) * 2;
    g = mix<X>(k);
  }
  __device__ __forceinline__ bf16x8 operator()(const char *lds, int x0, int s) const {
    typedef __attribute__((address_space(3))) shortx4 *Lp;
    const char *p = lds + base + s * 16 * X * 2 + (((x0 >> 5) ^ g) << 6);
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p)), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(p + 4 * X * 2));
    const shortx8 v = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return __builtin_bit_cast(bf16x8, v);
  }
};
template <int X>
struct FragReader<float, X, false> {
  int base, flip;
  __device__ __forceinline__ explicit FragReader(int lane) : base((4 * (lane >> 5) * X + (lane & 31)) * 4), flip(X >= 64 ? lane & 32 : 0) {}
  __device__ __forceinline__ floatx4 operator()(const char *lds, int x0, int s) const {
    const float *p = reinterpret_cast<const float *>(lds + base) + s * 8 * X + (x0 ^ flip);
    return floatx4{p[0], p[X], p[2 * X], p[3 * X]};
  }
};

__device__ __forceinline__ floatx16 mfma(bf16x8 b, bf16x8 a, floatx16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b, a, c, 0, 0, 0); }
__device__ __forceinline__ floatx16 mfma(floatx4 b, floatx4 a, floatx16 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(b[j], a[j], c, 0, 0, 0);
  return c;
}

// Single precision on the bfloat16 matrix pipe, which has 16 times the rate: x = hi + mid + lo up to 2^-24 |x|, each the rest so far
// rounded to nearest (the rests are exact), and of the nine products of two such sums the six that reach 2^-24 of the whole.
// dot2 takes a number off its rounded pair without unpacking it.
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
struct Split { bf16x8 p[3]; };
__device__ __forceinline__ Split split3(floatx4 x, floatx4 y) {
  unsigned lo_ = 0xBF80u, hi_ = 0xBF800000u;   // (-1, 0) and (0, -1), in registers: as inline constants they are single precision's
  asm("" : "+s"(lo_), "+s"(hi_));
  const bf16x2 first = __builtin_bit_cast(bf16x2, lo_), second = __builtin_bit_cast(bf16x2, hi_);
  Split s;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float a = j < 2 ? x[2 * j] : y[2 * j - 4], b = j < 2 ? x[2 * j + 1] : y[2 * j - 3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      bf16x2 h;
      h[0] = (bf16)a;
      h[1] = (bf16)b;
      s.p[k][2 * j] = h[0];
      s.p[k][2 * j + 1] = h[1];
      if (k < 2) {
        a = __builtin_amdgcn_fdot2_f32_bf16(h, first, a, false);
        b = __builtin_amdgcn_fdot2_f32_bf16(h, second, b, false);
      }
    }
  }
  return s;
}
__device__ __forceinline__ floatx16 mfma6(const Split &b, const Split &a, floatx16 c) {   // the small products first
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[0], a.p[2], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[2], a.p[0], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[1], a.p[1], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[0], a.p[1], c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[1], a.p[0], c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.p[0], a.p[0], c, 0, 0, 0);
}

// ------------------------------------------------------------------------------------------------ kernel
// WK groups of WM x WN wavefronts of (BM / WM) x (BN / WN) each; the groups take the slabs in turn and their sums are added in LDS in
// group order (products with too few tiles to fill the chip: the chain of slabs is WK times shorter).
// Epi: `piece<WC>(stage, m, n, M, N, problem, split, q, ahead)` takes 32 x WC sums (WC = 64 or 32) from the wavefront's LDS area
// (row stride kStageLd floats), first element C(m, n), the wavefront's q-th piece along m; `ahead(m, M, lane)` is called before the products;
// `counts(ahead, q, lane, N)`, called by whole wavefronts, says whether row lane % 32 of the q-th piece is used.
// PAIR: B[0] and B[1] are the gate and up projections (KC), N counts hidden units, a tile covers BN / 2 of them.
template <class T, int BM, int BN, int WM, int WN, int WK, int STAGES, bool AKC, bool BKC, bool PAIR, class Epi>
__device__ __forceinline__ void product_tile(const ProductArgs &a, const Epi &epi, int id, char *smem) {
  constexpr int kThreads = 64 * WM * WN, TM = BM / WM / 32, WC = BN / WN, TN = WC / 32, kK = Elem<T>::kSlab;
  static_assert((WC == 64 || WC == 32) && BM % (32 * WM) == 0, "wavefront tiles are 64 or 32 columns wide");
  typedef Slab<T, BM, AKC, kThreads> SA;
  typedef Slab<T, BN, BKC, kThreads> SB;
  constexpr int kA = SA::kBytes, kStage = SA::kBytes + SB::kBytes, kLoads = SA::kIts + SB::kIts;
  const int lane = threadIdx.x & 63, all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = all % (WM * WN), group = all / (WM * WN);
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * WC;
  int tm, tn, unit;
  tile_of(id, a.tiles_m, a.tiles_n, a.splits * a.problems, &tm, &tn, &unit);
  const int problem = unit / a.splits, split = unit % a.splits;
  const int M = rows_left(a.m_rows, a.first, a.M);
  const int K0 = rows_left(a.k_rows, a.first, a.K[0]);
  const int m0 = tm * BM, n0 = tn * (PAIR ? BN / 2 : BN);
  if (m0 >= M) return;
  const int slabs0 = (K0 + kK - 1) / kK, slabs = slabs0 + (a.K[1] + kK - 1) / kK;
  const int t0 = min(slabs, split * a.slabs_per_split), t1 = min(slabs, t0 + a.slabs_per_split);
  const int turns = (t1 - t0 + WK - 1) / WK;   // a group's slabs: t0 + group, then every WK-th

  SA sa;
  SB sb;
  PairSlab<T, BN, WC, kThreads> sp;
  sa.init(a.A[0].ld, threadIdx.x % kThreads);
  if (PAIR) sp.init(a.B[0].ld, threadIdx.x % kThreads);
  else sb.init(a.B[0].ld, threadIdx.x % kThreads);
  char *mine = smem + group * STAGES * kStage;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)mine;
  // A slab behind the last is loaded as zeros, out of range of everything: the number of loads on their way stays the same, and a
  // group without a slab in the last turn adds nothing.
  const auto load = [&](int turn, int stage, int from, int to) {   // loads [from, to) of the kLoads of both operands
    const int t = t0 + turn * WK + group;
    const unsigned lds = lds0 + stage * kStage;
    const bool second = t >= slabs0;
    const int k0 = (second ? t - slabs0 : t) * kK, K = t >= t1 ? 0 : second ? a.K[1] : K0, which = second && a.K[1] > 0 ? 1 : problem;
    constexpr int kFirst = SA::kIts;
    sa.load(lds, wave, a.A[which], m0, M, k0, K, from, min(to, kFirst));
    if (PAIR) sp.load(lds + kA, wave, a.B[0], a.B[1], n0, a.N, k0, K, max(from - kFirst, 0), to - kFirst);
    else sb.load(lds + kA, wave, a.B[which], n0, a.N, k0, K, max(from - kFirst, 0), to - kFirst);
  };

  floatx16 acc[TM][TN];
  const typename Epi::Ahead ahead = epi.ahead(m0 + wm, M, lane);   // what the epilogue wants on its way during the products
  const FragReader<T, BM, AKC> ra(lane);
  const FragReader<T, BN, BKC> rb(lane);
  // Fragments are read ahead of the products that take them: of one of a slab's four steps, or of half a slab where single
  // precision is split.  The one barrier of a slab stands before its last products: by then every wavefront holds its last
  // fragments of this slab, so its place can take the slab STAGES turns on, and has seen its part of the next slab land, whose
  // first fragments are read behind the barrier while the last products run.
  constexpr bool kSplits = sizeof(T) == 4 && TM * TN > 1;
  typename Elem<T>::Frag fa[kSplits ? 4 : 2][TM], fb[kSplits ? 4 : 2][TN];
  const auto read = [&](int set, const char *lds, int s) {
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[set][j] = rb(lds + kA, wn + 32 * j, s);
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[set][i] = ra(lds, wm + 32 * i, s);
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto multiply = [&](int set) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = mfma(fb[set][j], fa[set][i], acc[i][j]);
    __builtin_amdgcn_sched_barrier(0);
  };
  const auto multiply_split = [&](int set) {
    if constexpr (sizeof(T) == 4) {
      Split b[TN];
#pragma unroll
      for (int j = 0; j < TN; ++j) b[j] = split3(fb[set][j], fb[set + 1][j]);
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const Split x = split3(fa[set][i], fa[set + 1][i]);
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = mfma6(b[j], x, acc[i][j]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A slab in which K ends inside a 16-byte group holds what lies behind the row's end there: cleared before anyone reads it.
  // Called behind the barrier that the turn's slabs have landed at, by everyone.
  constexpr int kG = 16 / (int)sizeof(T);
  const int ragged0 = AKC || BKC ? K0 % kG : 0, ragged1 = AKC || BKC ? a.K[1] % kG : 0;
  const auto clear_tail = [&](int turn, int stage) {
    if (ragged0 == 0 && ragged1 == 0) return;
    const int from = t0 + turn * WK, mine_t = from + group;
    const auto ends_in = [&](int t) {   // the k's of slab t's cut group that exist, 0: it is whole or has none
      return t >= t1 ? 0 : t == slabs0 - 1 ? ragged0 : t == slabs - 1 ? ragged1 : 0;
    };
    int any = 0;
#pragma unroll
    for (int g = 0; g < WK; ++g) any |= ends_in(from + g);
    if (any == 0) return;
    const int keep = ends_in(mine_t);
    if (keep) {
      const int K = mine_t == slabs0 - 1 ? K0 : a.K[1], cut = K % kK / kG;
      char *slab = mine + stage * kStage;
      for (int row = threadIdx.x % kThreads; row < (AKC ? BM : 0) + (BKC ? BN : 0); row += kThreads) {
        const int r = AKC && row < BM ? row : row - (AKC ? BM : 0);
        T *p = reinterpret_cast<T *>(slab + (AKC && row < BM ? 0 : kA) + r * kSlabBytes + ((cut ^ ((r >> 1) & 7)) << 4));
        for (int k = keep; k < kG; ++k) p[k] = (T)0.0f;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  };
  // Where a step has eight matrix instructions or more a wavefront, the loads go out between a slab's last ones: 4096 x 2048 x 8192
  // both ways in bfloat16 1.5 % faster (with four a step, in tiles of 128 x 128, 4096 x 2048 x 8192 took 170 us against 147).
  constexpr bool kSpread = TM * TN >= 8;
  const auto products = [&](auto split) {
    constexpr bool kSplit = decltype(split)::value;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j) acc[i][j] = floatx16{};
    if (turns == 0) return;
#pragma unroll
    for (int p = 0; p < STAGES; ++p) load(p, p, 0, kLoads);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads * (STAGES - 1)) : "memory");
    barrier();
    clear_tail(0, 0);
    read(0, mine, 0);
    if (kSplit) read(1, mine, 1);
    int stage = 0;
    for (int turn = 0; turn < turns; ++turn) {
      const int next = STAGES == 2 ? stage ^ 1 : stage + 1 == STAGES ? 0 : stage + 1;
      const char *now = mine + stage * kStage;
      if constexpr (kSplit) {
        read(2, now, 2);
        read(3, now, 3);
        multiply_split(0);
      } else {
        read(1, now, 1);
        multiply(0);
        read(0, now, 2);
        multiply(1);
        read(1, now, 3);
        multiply(0);
      }
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads * (STAGES - 2)) : "memory");
      barrier();
      if constexpr (!kSpread) load(turn + STAGES, stage, 0, kLoads);
      clear_tail(turn + 1, next);
      read(0, mine + next * kStage, 0);
      if constexpr (kSplit) {
        read(1, mine + next * kStage, 1);
        multiply_split(2);
      } else if constexpr (!kSpread) {
        multiply(1);
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) {
            const int part = i * TN + j;
            acc[i][j] = mfma(fb[1][j], fa[1][i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            load(turn + STAGES, stage, part * kLoads / (TM * TN), (part + 1) * kLoads / (TM * TN));
            __builtin_amdgcn_sched_barrier(0);
          }
      }
      stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // of the slabs of zeros too
  };
  // Single precision is split where a fragment is used twice at least (4096 x 8192 x 1024 in tiles of 128 x 128: 187 TFLOP/s against
  // 123 as it is, and an error of 3.4e-7 against 4.1e-7).  A number beyond bfloat16's range, an infinity or a NaN leaves sums that
  // are not finite: such a tile is taken again as it is.  Numbers below 2^-110 lose digits, as their parts fall below 2^-126.
  if constexpr (kSplits) {
    products(std::true_type{});
    bool finite = true;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) finite = finite && fabsf(acc[i][j][r]) < INFINITY;
    // Only sums that exist and whose rows count for the epilogue do: an operand across k may hold anything behind its last row or
    // column (a workspace's rows are written up to their last whole group of eight), and what a former call left there must change
    // neither digits nor time.  Looked at only where there is something: for every tile it would cost 2.5 % of 1000 x 500 x 1337 both ways.
    if (__any(!finite)) {
      const int left = PAIR ? WC : a.N - n0 - wn - 4 * (lane >> 5);   // a pair's rows behind the last one are zeros
      finite = true;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const bool counts = epi.counts(ahead, i, lane, a.N), row = m0 + wm + 32 * i + (lane & 31) < M && counts;
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) finite = finite && (fabsf(acc[i][j][r]) < INFINITY || !row || 32 * j + 8 * (r >> 2) + (r & 3) >= left);
      }
    }
    unsigned *flag = reinterpret_cast<unsigned *>(smem);   // one a wavefront, in the slabs' place
    __syncthreads();
    if (lane == 0) flag[all] = 0u;
    if (!finite) flag[all] = 1u;
    __syncthreads();
    unsigned again = 0u;
#pragma unroll
    for (int w = 0; w < WM * WN * WK; ++w) again |= flag[w];
    if (__builtin_amdgcn_readfirstlane((int)again)) {
      __syncthreads();   // everyone has read the flags
      products(std::false_type{});
    }
  } else {
    products(std::false_type{});
  }
  __syncthreads();   // the slabs' place becomes the epilogue's
  constexpr int kPiece = 32 * kStageLd;
  float *stage = reinterpret_cast<float *>(smem) + all * kPiece;
  const auto to_stage = [&](const floatx16 (&c)[TN]) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<floatx4 *>(stage + (lane & 31) * kStageLd + 32 * j + 8 * r + 4 * (lane >> 5)) =
            floatx4{c[j][4 * r], c[j][4 * r + 1], c[j][4 * r + 2], c[j][4 * r + 3]};
  };
  if constexpr (WK > 1) {
    static_assert(TM == 1, "one piece a wavefront");
    to_stage(acc[0]);
    __syncthreads();
    if (group > 0 || m0 + wm >= M) return;
#pragma unroll
    for (int e = 0; e < 32; e += 256 / WC) {   // 16 bytes a lane
      float *p = stage + (e + lane / (WC / 4)) * kStageLd + 4 * (lane % (WC / 4));
      floatx4 v = *reinterpret_cast<floatx4 *>(p);
#pragma unroll
      for (int g = 1; g < WK; ++g) v += *reinterpret_cast<floatx4 *>(p + g * WM * WN * kPiece);
      *reinterpret_cast<floatx4 *>(p) = v;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    epi.template piece<WC>(stage, m0 + wm, PAIR ? n0 + wn / 2 : n0 + wn, M, a.N, problem, split, 0, ahead);
  } else {
#pragma unroll 1   // one copy of the epilogue; the sums' registers are chosen by uniform branches
    for (int q = 0; q < TM; ++q) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
      for (int i = 0; i < TM; ++i)
        if (i == q) to_stage(acc[i]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      if (m0 + wm + 32 * q < M) epi.template piece<WC>(stage, m0 + wm + 32 * q, PAIR ? n0 + wn / 2 : n0 + wn, M, a.N, problem, split, q, ahead);
    }
  }
}

template <class T, int BM, int BN, int WM, int WN, int WK, int STAGES, bool AKC, bool BKC, bool PAIR, class Epi>
__global__ __launch_bounds__(64 * WM *WN *WK, 2) void product_kernel(const ProductArgs a, const Epi epi) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  product_tile<T, BM, BN, WM, WN, WK, STAGES, AKC, BKC, PAIR, Epi>(a, epi, blockIdx.x, smem);
}

// ------------------------------------------------------------------------------------------------ outputs
__device__ __forceinline__ float to_float(bf16 v) { return (float)v; }
__device__ __forceinline__ float to_float(float v) { return v; }

// Eight neighbours of a row from any element on: accesses of 16 bytes ask for no more than an element's alignment (a column a
// lane instead made the backward epilogue of 1000 x 1337 rows 14 us slower than that of 1000 x 1336).
template <class T> struct Eight {
  typedef T V __attribute__((ext_vector_type(8)));
  typedef V Any __attribute__((aligned(sizeof(T))));
  V v;
  __device__ __forceinline__ void load(const T *p, int n) {   // the first n exist
    if (n >= 8) {
      v = *reinterpret_cast<const Any *>(p);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : (T)0.0f;
    }
  }
  __device__ __forceinline__ void store(T *p, int n) const {
    if (n >= 8) {
      *reinterpret_cast<Any *>(p) = v;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) p[j] = v[j];
    }
  }
};
template <class T> __device__ __forceinline__ void store8(T *p, const float (&v)[8], int n) {
  Eight<T> e;
#pragma unroll
  for (int j = 0; j < 8; ++j) e.v[j] = (T)v[j];   // to nearest, ties to even
  e.store(p, n);
}
template <class T> __device__ __forceinline__ void load8(const T *p, float (&v)[8], int n) {
  Eight<T> e;
  e.load(p, n);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)e.v[j];
}
__device__ __forceinline__ void stage8(const float *stage, int row, int col, float (&v)[8]) {
  const floatx4 a = *reinterpret_cast<const floatx4 *>(stage + row * kStageLd + col), b = *reinterpret_cast<const floatx4 *>(stage + row * kStageLd + col + 4);
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
}

// How a wavefront's lanes take a piece of 32 rows x WC columns: eight columns a lane, whole rows side by side, so that outputs leave
// as full lines (runs of eight straight from the products' registers, 32 rows at a time, made the epilogues' stores 1.5 to 3
// times as slow)
template <int WC> struct Lanes {
  static constexpr int kARow = WC / 8, kRows = 64 / kARow, kPasses = 32 / kRows;
  int row, col;
  __device__ __forceinline__ Lanes() : row((int)(threadIdx.x & 63) / kARow), col(8 * ((int)(threadIdx.x & 63) % kARow)) {}
};
struct Nothing {};
struct NothingAhead {
  typedef Nothing Ahead;
  __device__ __forceinline__ Nothing ahead(int, int, int) const { return Nothing{}; }
  __device__ __forceinline__ bool counts(Nothing, int, int, int) const { return true; }
};

// C[problem][m][n] in T, rows optionally through a map, times scale / *count; or += to what a former piece left (fp32 sums)
template <class T>
struct StoreEpi : NothingAhead {
  StoreEpi(T *c0, T *c1, long ld_, const int *rows_, int add_, const int *count_ = nullptr, float scale_ = 1.0f)
      : c{c0, c1}, ld(ld_), rows(rows_), add(add_), count(count_), scale(scale_) {}
  T *c[2];
  long ld;
  const int *rows;         // nullable: row m of the product goes to row rows[m]
  int add;                 // T = float only: add to what is there
  const int *count;        // nullable: no factor
  float scale;
  __device__ __forceinline__ float factor() const {   // of no rows: the sums are zeros
    const int n = *count;
    return n > 0 ? scale / (float)n : 0.0f;
  }
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int N, int problem, int, int, Nothing) const {
    const Lanes<WC> l;
    const int col = l.col;
    const float f = count ? factor() : 1.0f;
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int row = l.kRows * p + l.row;
      if (m + row >= M || n + col >= N) continue;
      float v[8];
      stage8(stage, row, col, v);
      if (count)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= f;
      T *d = c[problem] + (long)(rows ? rows[m + row] : m + row) * ld + n + col;
      const int left = N - n - col;
      if (sizeof(T) == 4 && add) {
        float o[8];
        load8<T>(d, o, left);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += o[j];
      }
      store8<T>(d, v, left);
    }
  }
};

// Sums of one split of k in fp32, [split][M][N8], N8 = N rounded up to 8
struct PartialEpi : NothingAhead {
  PartialEpi(float *part_, long rows_) : part(part_), rows(rows_) {}
  float *part;
  long rows;   // of a split (the M of the launch)
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int N, int, int split, int, Nothing) const {
    const Lanes<WC> l;
    const int col = l.col;
    const long n8 = (N + 7) & ~7;
#pragma unroll
    for (int p = 0; p < l.kPasses; ++p) {
      const int row = l.kRows * p + l.row;
      if (m + row >= M || n + col >= N) continue;
      float v[8];
      stage8(stage, row, col, v);
      store8<float>(part + ((long)split * rows + m + row) * n8 + n + col, v, 8);
    }
  }
};

// The splits added up in order, as a StoreEpi of one problem would have stored them (products that add to a former piece's have no
// split k)
template <class T>
__global__ __launch_bounds__(256) void sum_splits_kernel(const float *part, int splits, int M, int N, const int *m_rows, int first, StoreEpi<T> out) {
  const long n8 = (N + 7) & ~7;
  const int rows = rows_left(m_rows, first, M), g = (int)(n8 >> 3);
  const float f = out.count ? out.factor() : 1.0f;
  for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < (long)rows * g; i += (long)gridDim.x * 256) {
    const int m = (int)(i / g), n = (int)(i % g) * 8;
    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      float o[8];
      load8<float>(part + ((long)s * M + m) * n8 + n, o, 8);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += o[j];
    }
    if (out.count)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= f;
    store8<T>(out.c[0] + (long)(out.rows ? out.rows[m] : m) * out.ld + n, v, N - n);
  }
}

// ------------------------------------------------------------------------------------------------ host
// The tilings of a product: tile edges, groups of wavefronts that take the slabs in turn, slabs on their way.  256 x 256 keeps two
// slabs (128 KB of LDS, a workgroup a compute unit); 128 x 128 and 64 x 64 two with two workgroups a unit, or four with one, as
// operands that come from memory rather than L2 take longer to arrive than a slab to multiply (on cold weights 2048 x 2048 x
// 2048 takes 28 us with four slabs of 128 x 128 and 34 with two, but 777 x 5472 x 1000, with two tiles for some units, 32 against 23).
enum Tiling { TILE_256 = 0, TILE_128, TILE_128_DEEP, TILE_64_K2, TILE_64_K2_DEEP, TILE_32_K4, TILE_32_K8, TILINGS };
struct ProductPlan { int tiling = TILE_128, splits = 1; };

// What a tiling costs, in microseconds, as measured on products of 32 to 8192 rows and columns: a workgroup's share of a
// compute unit for one turn (a slab for each group) with the unit full, the least time of a turn's chain of load, barrier and
// products, what a workgroup takes besides its turns, and how many a unit holds.
struct TilingCost { int bm, bn, groups, resident; double share[2], chain[2], besides[2]; };   // [fp32, bf16]
constexpr TilingCost kTilings[TILINGS] = {
    {256, 256, 1, 1, {0, 1.62}, {0, 1.5}, {0, 8.0}},   // bfloat16 alone: a split's fragments would not fit beside 128 sums
    {128, 128, 1, 2, {1.4, 0.55}, {1.45, 1.0}, {4.0, 4.0}},
    {128, 128, 1, 1, {1.6, 0.78}, {1.48, 0.78}, {3.5, 3.0}},
    {64, 64, 2, 2, {0.9, 0.45}, {1.08, 0.88}, {3.0, 2.5}},
    {64, 64, 2, 1, {1.12, 0.62}, {1.12, 0.62}, {3.0, 2.5}},
    {32, 64, 4, 1, {1.35, 0.9}, {1.35, 0.9}, {3.5, 2.5}},
    {32, 32, 8, 1, {1.35, 0.9}, {1.35, 0.9}, {3.5, 3.0}},   // 32 columns a wavefront
};

// The tiling and the number of parts of k with the least estimated time.  Parts of k cost their sums' way to memory and back and
// a second launch.
inline ProductPlan plan_product(int dtype, int M, int N, long slabs, bool pair, bool may_split) {
  ProductPlan best;
  double least = 1e30;
  const int type = dtype == TYPE_BF16 ? 1 : 0, cus = chip().cus;
  for (int i = type ? TILE_256 : TILE_128; i < TILINGS; ++i) {
    if (i == TILE_64_K2_DEEP && !type) continue;   // as long as with two slabs for a lone workgroup, longer with two a unit
    const TilingCost &c = kTilings[i];
    const long nn = pair ? 2L * N : N, tiles = (long)((M + c.bm - 1) / c.bm) * ((nn + c.bn - 1) / c.bn);
    for (int s = 1; s <= (may_split ? 32 : 1); s *= 2) {
      if (s > 1 && (slabs < 4L * s || tiles * s > 4L * cus * c.resident)) break;
      const long each = ((slabs + s - 1) / s + c.groups - 1) / c.groups, n = (tiles * s + cus - 1) / cus, full = n / c.resident, rest = n % c.resident;
      const double whole = c.resident * c.share[type] > c.chain[type] ? c.resident * c.share[type] : c.chain[type];
      const double part = rest * c.share[type] > c.chain[type] ? rest * c.share[type] : c.chain[type];
      double t = full * (each * whole + c.besides[type]) + (rest ? each * part + c.besides[type] : 0.0);
      if (s > 1) t += 5.0 + (double)s * M * N * 8.0 / 4.0e6;
      if (t < least) {
        least = t;
        best.tiling = i;
        best.splits = s;
      }
    }
  }
  return best;
}
// columns of a wavefront's pieces
inline int piece_columns(int tiling) { return tiling == TILE_32_K8 ? 32 : 64; }
inline long slabs_of(long k, int dtype) { return (k * (long)type_bytes(dtype) + kSlabBytes - 1) / kSlabBytes; }

// LDS of a workgroup: its slabs, or in their place a piece of sums for each wavefront
template <int BM, int BN, int WM, int WN, int WK, int STAGES>
constexpr size_t product_lds() {
  constexpr size_t slabs = (size_t)STAGES * WK * (BM + BN) * kSlabBytes, stage = (size_t)WM * WN * WK * 32 * kStageLd * sizeof(float);
  static_assert(slabs <= 160 * 1024 && stage <= 160 * 1024, "a compute unit's LDS");
  return slabs > stage ? slabs : stage;
}

template <class T, int BM, int BN, int WM, int WN, int WK, int STAGES, bool AKC, bool BKC, bool PAIR, class Epi>
hipError_t launch_tiling(ProductArgs a, const Epi &epi, hipStream_t stream) {
  constexpr int kThreads = 64 * WM * WN * WK;
  constexpr size_t lds = product_lds<BM, BN, WM, WN, WK, STAGES>();
  const auto kernel = product_kernel<T, BM, BN, WM, WN, WK, STAGES, AKC, BKC, PAIR, Epi>;
  hipError_t e = allow_large_lds(reinterpret_cast<const void *>(kernel), lds);
  if (e != hipSuccess) return e;
  a.tiles_m = (a.M + BM - 1) / BM;
  a.tiles_n = (a.N + (PAIR ? BN / 2 : BN) - 1) / (PAIR ? BN / 2 : BN);
  const long tiles = (long)a.tiles_m * a.tiles_n * a.splits * a.problems;
  if (tiles * kThreads >= (1L << 31)) return hipErrorInvalidValue;
  kernel<<<dim3((unsigned)tiles), dim3(kThreads), lds, stream>>>(a, epi);
  return hipGetLastError();
}

template <class T, bool AKC, bool BKC, bool PAIR, class Epi>
hipError_t launch_product(const ProductArgs &a, const Epi &epi, int tiling, hipStream_t stream) {
  switch (tiling) {
    case TILE_256:
      if constexpr (sizeof(T) == 2) return launch_tiling<T, 256, 256, 2, 4, 1, 2, AKC, BKC, PAIR, Epi>(a, epi, stream);
      [[fallthrough]];   // not planned for single precision
    case TILE_128: return launch_tiling<T, 128, 128, 2, 2, 1, 2, AKC, BKC, PAIR, Epi>(a, epi, stream);
    case TILE_128_DEEP: return launch_tiling<T, 128, 128, 2, 2, 1, 4, AKC, BKC, PAIR, Epi>(a, epi, stream);
    case TILE_64_K2: return launch_tiling<T, 64, 64, 2, 1, 2, 2, AKC, BKC, PAIR, Epi>(a, epi, stream);
    case TILE_64_K2_DEEP:
      if constexpr (sizeof(T) == 2) return launch_tiling<T, 64, 64, 2, 1, 2, 4, AKC, BKC, PAIR, Epi>(a, epi, stream);
      [[fallthrough]];   // nor this one
    case TILE_32_K4: return launch_tiling<T, 32, 64, 1, 1, 4, 3, AKC, BKC, PAIR, Epi>(a, epi, stream);
    default: return launch_tiling<T, 32, 32, 1, 1, 8, 2, AKC, BKC, PAIR, Epi>(a, epi, stream);
  }
}

struct Take {
  char *base;
  size_t used = 0;
  void *operator()(size_t bytes) {
    void *p = base ? base + used : nullptr;
    used += (bytes + 255) / 256 * 256;
    return p;
  }
};

template <class T>
hipError_t launch_sum_splits(const ProductArgs &p, const StoreEpi<T> &out, int splits, const float *part, hipStream_t stream) {
  const long groups = (long)p.M * ((p.N + 7) / 8), blocks = (groups + 255) / 256;
  sum_splits_kernel<T><<<dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, stream>>>(part, splits, p.M, p.N, p.m_rows, p.first, out);
  return hipGetLastError();
}
inline size_t partial_bytes(int splits, int M, int N) { return splits > 1 ? (size_t)splits * M * ((N + 7) & ~7) * sizeof(float) : 0; }

// a product whose k may be split, its sums stored as T
template <class T, bool AKC, bool BKC>
hipError_t product_to(ProductArgs p, StoreEpi<T> out, const ProductPlan &plan, float *part, hipStream_t stream) {
  if (plan.splits <= 1) return launch_product<T, AKC, BKC, false>(p, out, plan.tiling, stream);
  const int slabs = (p.K[0] + Elem<T>::kSlab - 1) / Elem<T>::kSlab;   // one segment
  p.slabs_per_split = (slabs + plan.splits - 1) / plan.splits;
  p.splits = plan.splits;
  hipError_t e = launch_product<T, AKC, BKC, false>(p, PartialEpi(part, p.M), plan.tiling, stream);
  if (e != hipSuccess) return e;
  return launch_sum_splits<T>(p, out, plan.splits, part, stream);
}

// The products of a backward pass that do not wait for each other, in one launch: a data gradient (A along k, B across it), whose k
// may be split, and up to two kinds of weight gradients (both across k).  Those with the longest chains of slabs come first, the
// others fill the compute units that these leave.
template <class T>
struct GradientEpi : NothingAhead {
  GradientEpi() : store(nullptr, nullptr, 0, nullptr, 0), part(nullptr, 0), partial(0) {}
  StoreEpi<T> store;
  PartialEpi part;
  int partial;
  template <int WC>
  __device__ __forceinline__ void piece(const float *stage, int m, int n, int M, int N, int problem, int split, int q, Nothing a) const {
    if (partial) part.template piece<WC>(stage, m, n, M, N, problem, split, q, a);
    else store.template piece<WC>(stage, m, n, M, N, problem, split, q, a);
  }
};
template <class T>
struct GradientJobs {
  int n = 0;
  struct Job { ProductArgs a; GradientEpi<T> epi; int data = 0, begin = 0; } job[3];
  ProductPlan plan;
  float *partial = nullptr;
  void add(const ProductArgs &a, const StoreEpi<T> &out, bool data) {
    Job &j = job[n++];
    j.a = a;
    j.epi.store = out;
    j.data = data;
  }
};

template <class T, int BM, int BN, int WM, int WN, int WK, int STAGES>
__global__ __launch_bounds__(64 * WM *WN *WK, 2) void gradient_kernel(const GradientJobs<T> g) {
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int id = blockIdx.x, k = g.n > 2 && id >= g.job[2].begin ? 2 : g.n > 1 && id >= g.job[1].begin ? 1 : 0;
  const typename GradientJobs<T>::Job &j = g.job[k];
  if (j.data) product_tile<T, BM, BN, WM, WN, WK, STAGES, true, false, false, GradientEpi<T>>(j.a, j.epi, id - j.begin, smem);
  else product_tile<T, BM, BN, WM, WN, WK, STAGES, false, false, false, GradientEpi<T>>(j.a, j.epi, id - j.begin, smem);
}

struct GradientShape { int M, N; long slabs; int problems; bool data; };

// When `n` kinds (at most three) of units, count[k] of time[k] each, the longest first, are all done on `slots` places, each unit taken by the place
// that is free first.  Places that are free at the same time are counted together; what would be more than a few rounds is taken as
// spread evenly with half a unit's tail.
inline double makespan(const double *count, const double *time, int n, int slots) {
  double all = 0, units = 0;
  for (int k = 0; k < n; ++k) all += count[k] * time[k], units += count[k];
  if (units > 4.0 * slots) return all / slots + 0.5 * time[n - 1];
  struct Level { double at; int places; } level[4];   // each kind leaves one more at most
  int levels = 1;
  level[0] = Level{0.0, slots};
  double end = 0;
  for (int k = 0; k < n; ++k)
    for (int left = (int)count[k]; left > 0;) {
      int low = 0;
      for (int i = 1; i < levels; ++i)
        if (level[i].at < level[low].at) low = i;
      const int take = left < level[low].places ? left : level[low].places;
      const double at = level[low].at + time[k];
      left -= take;
      end = at > end ? at : end;
      if (take == level[low].places) {
        level[low].at = at;
      } else {
        level[low].places -= take;
        level[levels++] = Level{at, take};
      }
    }
  return end;
}

// As plan_product, for the launch as a whole.  Counting units and not their work alone: 1000 x 500 x 1337 in single precision had 260
// of them on 256 compute units, 77 us.
inline ProductPlan plan_gradients(int dtype, const GradientShape *shape, int n) {
  ProductPlan best;
  double least = 1e30;
  const int type = dtype == TYPE_BF16 ? 1 : 0, cus = chip().cus;
  constexpr int kParts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32};
  for (int i = type ? TILE_256 : TILE_128; i < TILINGS; ++i) {
    const TilingCost &c = kTilings[i];
    for (const int s : kParts) {
      double count[3], time[3], units = 0, work = 0, extra = 0;
      bool ok = true;
      for (int k = 0; k < n; ++k) {
        const GradientShape &g = shape[k];
        const int parts = g.data ? s : 1;
        if (parts > 1 && g.slabs < 4L * parts) ok = false;
        const long each = ((g.slabs + parts - 1) / parts + c.groups - 1) / c.groups;
        count[k] = (double)((g.M + c.bm - 1) / c.bm) * ((g.N + c.bn - 1) / c.bn) * g.problems * parts;
        time[k] = (double)each;
        units += count[k];
        if (parts > 1) extra = 5.0 + (double)parts * g.M * g.N * 8.0 / 4.0e6;
      }
      if (!ok) break;
      const int resident = units > cus ? c.resident : 1;   // of a compute unit, by then
      const double turn = resident * c.share[type] > c.chain[type] ? resident * c.share[type] : c.chain[type];
      double longest = 0;
      for (int k = 0; k < n; ++k) {
        time[k] = time[k] * turn + c.besides[type];
        work += count[k] * time[k];
        longest = time[k] > longest ? time[k] : longest;
      }
      const double most = work / (cus * resident);
      if ((most > longest ? most : longest) + extra >= least) continue;
      for (int a = 0; a < n; ++a)   // the longest first
        for (int b = a + 1; b < n; ++b)
          if (time[b] > time[a]) {
            double t = time[a];
            time[a] = time[b], time[b] = t;
            t = count[a], count[a] = count[b], count[b] = t;
          }
      const double t = makespan(count, time, n, cus * resident) + extra;
      if (t < least) {
        least = t;
        best.tiling = i;
        best.splits = s;
      }
    }
  }
  return best;
}

template <class T, int BM, int BN, int WM, int WN, int WK, int STAGES>
hipError_t launch_gradients_as(GradientJobs<T> g, hipStream_t stream) {
  constexpr size_t lds = product_lds<BM, BN, WM, WN, WK, STAGES>();
  const auto kernel = gradient_kernel<T, BM, BN, WM, WN, WK, STAGES>;
  hipError_t e = allow_large_lds(reinterpret_cast<const void *>(kernel), lds);
  if (e != hipSuccess) return e;
  long chain[3], begin = 0;
  for (int k = 0; k < g.n; ++k) {
    ProductArgs &a = g.job[k].a;
    a.tiles_m = (a.M + BM - 1) / BM;
    a.tiles_n = (a.N + BN - 1) / BN;
    const int slab = Elem<T>::kSlab, all = (a.K[0] + slab - 1) / slab + (a.K[1] + slab - 1) / slab;
    chain[k] = all;
    if (g.job[k].data && g.plan.splits > 1) {
      a.splits = g.plan.splits;
      a.slabs_per_split = (all + a.splits - 1) / a.splits;
      g.job[k].epi.part = PartialEpi(g.partial, a.M);
      g.job[k].epi.partial = 1;
      chain[k] = a.slabs_per_split;
    }
  }
  for (int i = 0; i < g.n; ++i)   // the longest first
    for (int k = i + 1; k < g.n; ++k)
      if (chain[k] > chain[i]) {
        const typename GradientJobs<T>::Job j = g.job[i];
        g.job[i] = g.job[k];
        g.job[k] = j;
        const long c = chain[i];
        chain[i] = chain[k];
        chain[k] = c;
      }
  for (int k = 0; k < g.n; ++k) {
    g.job[k].begin = (int)begin;
    begin += (long)g.job[k].a.tiles_m * g.job[k].a.tiles_n * g.job[k].a.splits * g.job[k].a.problems;
    if (begin * 64 * WM * WN * WK >= (1L << 31)) return hipErrorInvalidValue;
  }
  kernel<<<dim3((unsigned)begin), dim3(64 * WM * WN * WK), lds, stream>>>(g);
  e = hipGetLastError();
  for (int k = 0; k < g.n && e == hipSuccess; ++k)
    if (g.job[k].epi.partial) e = launch_sum_splits<T>(g.job[k].a, g.job[k].epi.store, g.plan.splits, g.partial, stream);
  return e;
}

template <class T>
hipError_t launch_gradients(const GradientJobs<T> &g, hipStream_t stream) {
  if (g.n == 0) return hipSuccess;
  switch (g.plan.tiling) {
    case TILE_256:
      if constexpr (sizeof(T) == 2) return launch_gradients_as<T, 256, 256, 2, 4, 1, 2>(g, stream);
      [[fallthrough]];   // not planned for single precision
    case TILE_128: return launch_gradients_as<T, 128, 128, 2, 2, 1, 2>(g, stream);
    case TILE_128_DEEP: return launch_gradients_as<T, 128, 128, 2, 2, 1, 4>(g, stream);
    case TILE_64_K2: return launch_gradients_as<T, 64, 64, 2, 1, 2, 2>(g, stream);
    case TILE_64_K2_DEEP: return launch_gradients_as<T, 64, 64, 2, 1, 2, 4>(g, stream);
    case TILE_32_K4: return launch_gradients_as<T, 32, 64, 1, 1, 4, 3>(g, stream);
    default: return launch_gradients_as<T, 32, 32, 1, 1, 8, 2>(g, stream);
  }
}

#define DLL_TRY(call) do { const hipError_t e_ = (call); if (e_ != hipSuccess) return e_; } while (0)

}  // namespace tile
}  // namespace dllk
