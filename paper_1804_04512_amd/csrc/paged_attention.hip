// Attention of one new token a request over a paged cache: o = softmax(scale q k^T) v over the request's keys, which the block table finds.
//
// Bound by memory: each request's keys and values are read once, for all heads that share them.  Those are the columns of 16 x 16 x 32
// products (scores transposed: keys are registers, the head is the lane), up to sixteen at a time.
//
// The work is units of kUnit keys of one request and key head, dealt to the workgroups in equal runs whatever the lengths are: each
// workgroup finds its run by adding the lengths up.  Where a run holds all of a request's head the result is written; where it
// begins or ends inside one, its outputs with their maximum and sum go to the workspace (two places a workgroup) and a second
// launch makes their mean, in the order of the keys.
//
// Inside a workgroup the wavefronts take tiles of 32 keys in turn, each with its own running maximum and sums.  A lane holds eight elements of
// two keys a step, straight from memory into the operand's registers; values have the same addresses, and go through the
// wavefront's own LDS to be read across keys, in the order in which the scores' registers hold them: register r of quarter c is key 4 c + r of
// its sixteen, so eight registers of two results are keys 4 c + j and 16 + 4 c + j.
//
// 64 requests of up to 8192 keys, 32 heads of 128 on 8, bfloat16: 196 us for 1.04 GB = 5.3 TB/s, above what a copy reaches (4.8); three of up to 60000, eight heads of
// 96 in single precision, 163 us = 5.4.  One request of 1000 keys 13.5 us: two launches, each a chain of loads.  What it took: pages asked for before the
// rows of the tile in between, as loads come back in order (312 to 193 us), and no branch between loads.
#include "attention_tile.h"

namespace dllk {

using namespace attn;

namespace {

constexpr int kThreads = 256, kWaves = 4, kTile = 32, kUnit = kWaves * kTile, kHeads = 16;
constexpr int kMaxGroups = 1024;   // workgroups of a launch

// workgroups that a compute unit holds, by their registers
template <class T, int DP> constexpr int residents() { return (sizeof(T) == 2 ? DP <= 128 : DP <= 96) ? 2 : 1; }

// Eight numbers of an operand: single precision is multiplied as it is, as what bounds these kernels is memory
template <class T> struct EightOf;
template <> struct EightOf<bf16> { typedef bf16x8 Type; };
template <> struct EightOf<float> { typedef floatx8 Type; };
template <class T> using Numbers = typename EightOf<T>::Type;
// Rows in LDS, places as in Tile
template <class T, int DP>
struct Rows {
  static constexpr int kRowBytes = Tile<DP>::kPitch * (int)sizeof(T), kGroups = kRowBytes / 16;
  static __device__ __forceinline__ int flip(int row) {
    return kGroups == 8 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3);
  }
};

__device__ __forceinline__ floatx4 mma16(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 mma16(floatx8 a, floatx8 b, floatx4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
// over the four quarters of the lanes
__device__ __forceinline__ float most4(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ __forceinline__ float sum4(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// keys of a request: what its table has room for at most
__device__ __forceinline__ int keys_of(const CacheArgs &a, int r) { return (int)max(0L, min((long)a.lengths[r], (long)a.columns * a.page)); }
__device__ __forceinline__ int units_of(int keys) { return (keys + kUnit - 1) / kUnit; }

struct Runs {
  float *o;    // [2 groups][kHeads][ld]
  float *ml;   // [2 groups][kHeads][2]: maximum in the exponent's base, sum
  int ld;      // head_dim in whole fours
  int blocks;  // of at most kHeads heads that share a key head
};

// Units before request r and in all, by the whole workgroup
__device__ __forceinline__ void add_units(const CacheArgs &a, int r, long *before, long *all, long *scratch) {
  long b = 0, s = 0;
  for (int i = threadIdx.x; i < a.R; i += kThreads) {
    const int u = units_of(keys_of(a, i));
    s += u;
    if (i < r) b += u;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) b += __shfl_xor(b, d), s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = b, scratch[kWaves + (threadIdx.x >> 6)] = s;
  __syncthreads();
  b = s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) b += scratch[w], s += scratch[kWaves + w];
  *before = b;
  *all = s;
}
// runs of units: workgroup w of n has those from w * all / n on, and where there are fewer units than workgroups one each
__device__ __forceinline__ int working(long all, int n) { return (int)min((long)n, all); }
__device__ __forceinline__ long run_of(long w, long all, int n) { return w * all / n; }
__device__ __forceinline__ int owner_of(long unit, long all, int n) { return (int)(((unit + 1) * n - 1) / all); }

// behind the wavefronts' areas in LDS
struct Shared {
  long scratch[kWaves + 1];
  int found, keys, empty[kWaves];
  float ml[kWaves][kHeads][2];
};

// WHOLE: a head's rows are whole runs of eight elements, so every load is 16 bytes or more from a place that exists and no branch stands
// between the loads; what a lane has no run for it takes from its row's last one, and is cleared before it meets the zeros of q: 0 times an
// infinity would make a score of -infinity NaN.
template <class T, int DP, bool WHOLE>
__global__ __launch_bounds__(kThreads, (residents<T, DP>())) void paged_attention_kernel(const CacheArgs a, const Runs parts, const Divisor page) {
  typedef Rows<T, DP> G;
  constexpr int kSteps = DP / 32, kArea = kTile * G::kRowBytes;   // LDS of a wavefront: its values, or at the end its sums [16][DP] fp32
  constexpr int kLeast = DP == 256 ? 136 : DP - 24;               // the shortest WHOLE row that comes here
  static_assert(kArea >= kHeads * DP * 4, "");
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  Shared &shared = *reinterpret_cast<Shared *>(smem + kWaves * kArea);
  long (&scratch)[kWaves + 1] = shared.scratch;
  auto &ml = shared.ml;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, col = lane & 15;
  char *area = smem + wave * kArea;
  const int group = a.H / a.KV, blocks = parts.blocks, VH = a.KV * blocks;
  const float c = factor_of(a.scale);

  // this workgroup's units, and the request that the first of them belongs to
  const int each = (a.R + kThreads - 1) / kThreads, r0 = min((int)threadIdx.x * each, a.R), r1 = min(r0 + each, a.R);
  long mine = 0;
  int empty = 0, keys = 0;   // some request has no keys; the last one's
  for (int r = r0; r < r1; ++r) {
    keys = keys_of(a, r);
    mine += units_of(keys);
    empty |= keys == 0;
  }
  long up = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long o = __shfl_up(up, d);
    if (lane >= d) up += o;
  }
  const int some = __any(empty);
  if (lane == 63) scratch[wave] = up, shared.empty[wave] = some;
  __syncthreads();
  if (shared.empty[0] | shared.empty[1] | shared.empty[2] | shared.empty[3]) {   // their outputs, by all workgroups in turn
    for (int r = blockIdx.x; r < a.R; r += gridDim.x)
      if (keys_of(a, r) == 0)
        for (int i = threadIdx.x; i < a.H * a.D; i += kThreads) {
          ((T *)a.o)[(long)r * a.H * a.D + i] = (T)0.0f;
          if (a.lse && i < a.H) a.lse[(long)r * a.H + i] = -INFINITY;
        }
  }
  long before = up - mine, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += scratch[w];
    all += scratch[w];
  }
  all *= VH;
  const int n = working(all, gridDim.x);
  if ((int)blockIdx.x >= n) return;
  const long first = run_of(blockIdx.x, all, n), end = run_of(blockIdx.x + 1, all, n);
  if (before * VH <= first && first < (before + mine) * VH) {
    long base = before * VH;
    for (int r = r0; r < r1; ++r) {
      if (each > 1) keys = keys_of(a, r);
      const long n = (long)units_of(keys) * VH;
      if (first < base + n) {
        shared.found = r;
        shared.keys = keys;
        scratch[kWaves] = base;
        break;
      }
      base += n;
    }
  }
  __syncthreads();
  int r = __builtin_amdgcn_readfirstlane(shared.found);
  long base = scratch[kWaves];
  keys = __builtin_amdgcn_readfirstlane(shared.keys);

  int off[kSteps];   // a lane's run of each step in its row, in bytes
#pragma unroll
  for (int s = 0; s < kSteps; ++s) off[s] = min(32 * s + 8 * quarter, a.D - 8) * (int)sizeof(T);
  const long row_bytes = (long)a.D * (int)sizeof(T), head_bytes = a.page * row_bytes, page_bytes = a.KV * head_bytes;

  for (long u = first; u < end;) {
    const int per = units_of(keys);
    const long rel = u - base;
    const int vh = (int)(rel / per), unit0 = (int)(rel % per), units = (int)min((long)(per - unit0), end - u);
    const int kv = vh / blocks, block = vh % blocks, heads = min(kHeads, group - block * kHeads), head0 = kv * group + block * kHeads;
    const int key_begin = unit0 * kUnit, key_end = min(keys, (unit0 + units) * kUnit);
    const int *table = a.table + (long)r * a.columns;
    const char *k_head = (const char *)a.k_cache + kv * head_bytes, *v_head = (const char *)a.v_cache + kv * head_bytes;

    Numbers<T> q[kSteps];
    {
      const T *row = (const T *)a.q + ((long)r * a.H + head0 + min(col, heads - 1)) * a.D;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        Eight<T> e;
        const int at = 32 * s + 8 * quarter;
        e.load(row + at, a.D - at);
        q[s] = a.scale < 0.0f ? -e.v : e.v;
      }
    }
    // A lane's two keys of a tile: their pages (-1: none), and where their rows lie.  A key without a page gets a row of page 0, which
    // exists.
    const auto pages = [&](int key0, int (&id)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = key0 + 16 * h + col;
        id[h] = table[page.of(min(key, key_end - 1))];
        if (key >= key_end) id[h] = -1;
      }
    };
    const auto places = [&](int key0, const int (&id)[2], long (&at)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int key = key0 + 16 * h + col;
        at[h] = (unsigned)id[h] < (unsigned)a.pages ? id[h] * page_bytes + (key - page.of(key) * a.page) * row_bytes : -1;
      }
    };
    const auto load = [&](Numbers<T> (&f)[2][kSteps], const char *head, const long (&at)[2]) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const char *row = head + max(at[h], 0L);
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          Eight<T> e;
          if (WHOLE) {
            e.load(reinterpret_cast<const T *>(row + off[s]), 8);
          } else {
            const int d = 32 * s + 8 * quarter;
            e.load(reinterpret_cast<const T *>(row) + d, a.D - d);
          }
          f[h][s] = e.v;
        }
      }
    };

    floatx4 o[DP / 16];
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) o[i] = floatx4{};
    float m = -INFINITY, l = 0.0f;
    // p times a power of two that brings all of a request's below 1, as sums of large values would overflow on their way to a mean that does not.  (Of
    // 60000 keys, those with weights below 2^-102 of the largest lose digits.)
    const float weight = power(-fold_of(keys));
    // On their way while a tile is worked on: the next one's values and keys, and the pages of the one behind it, which are asked
    // for first: loads come back in order, and the next rows' addresses must not wait for rows.
    int key0 = key_begin + wave * kTile, id[2], id_next[2];
    long at[2], next[2];
    Numbers<T> k[2][kSteps], v[2][kSteps];
    constexpr int kNext = kWaves * kTile;
    pages(key0, id);
    pages(key0 + kNext, id_next);
    places(key0, id, at);
    load(v, v_head, at);
    __builtin_amdgcn_sched_barrier(0);
    load(k, k_head, at);
    __builtin_amdgcn_sched_barrier(0);
    for (; key0 < key_end; key0 += kNext) {
      places(key0 + kNext, id_next, next);
      pages(key0 + 2 * kNext, id_next);
      __builtin_amdgcn_sched_barrier(0);
      const unsigned long seen0 = __ballot(at[0] >= 0), seen1 = __ballot(at[1] >= 0);   // bits of the first quarter: keys
      if ((seen0 & seen1) != ~0ul)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int s = 0; s < kSteps; ++s)
            if (at[h] < 0) v[h][s] = Numbers<T>{};
      // values into LDS, row by row; the rows' same groups of sixteen lanes land in different banks
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
          const int row = 16 * h + col;
          char *p = area + row * G::kRowBytes;
          if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<bf16x8 *>(p + (((4 * s + quarter) ^ G::flip(row)) << 4)) = v[h][s];
          } else {
            const int g = (8 * s + 2 * quarter) ^ G::flip(row);
            *reinterpret_cast<floatx4 *>(p + (g << 4)) = floatx4{v[h][s][0], v[h][s][1], v[h][s][2], v[h][s][3]};
            *reinterpret_cast<floatx4 *>(p + ((g ^ 1) << 4)) = floatx4{v[h][s][4], v[h][s][5], v[h][s][6], v[h][s][7]};
          }
        }
      __builtin_amdgcn_sched_barrier(0);
      load(v, v_head, next);
      __builtin_amdgcn_sched_barrier(0);
      floatx4 z[2] = {};
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        if (WHOLE && 32 * (s + 1) > kLeast && 32 * (s + 1) > a.D && 32 * s + 8 * quarter >= a.D)
#pragma unroll
          for (int h = 0; h < 2; ++h) k[h][s] = Numbers<T>{};
#pragma unroll
        for (int h = 0; h < 2; ++h) z[h] = mma16(k[h][s], q[s], z[h]);
      }
      __builtin_amdgcn_sched_barrier(0);
      load(k, k_head, next);
      __builtin_amdgcn_sched_barrier(0);
      at[0] = next[0];
      at[1] = next[1];
      if ((seen0 & seen1) != ~0ul)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!(seen0 >> (4 * quarter + j) & 1)) z[0][j] = -INFINITY;
          if (!(seen1 >> (4 * quarter + j) & 1)) z[1][j] = -INFINITY;
        }
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = fmaxf(top, fmaxf(z[0][j], z[1][j]));
      top = most4(top) * c;
      if (__any(top > m + 8.0f)) {
        const float grown = fmaxf(m, top), shrink = grown == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - grown);
        m = grown;
        l *= shrink;
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) o[i] *= shrink;
      }
      const float from = m == -INFINITY ? 0.0f : m;
      Numbers<T> p, rest;   // bfloat16: in two parts, as the second's products cost nothing beside memory
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = weight * __builtin_amdgcn_exp2f(__builtin_fmaf(z[j >> 2][j & 3], c, -from));
        l += e;
        p[j] = (T)e;
        rest[j] = (T)(e - (float)p[j]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      constexpr int kAhead = DP * (int)sizeof(T) <= 256 ? DP / 16 : DP % 64 ? 3 : 4;   // fragments read at a time
      static_assert(DP / 16 % kAhead == 0, "");
      Numbers<T> w[kAhead];
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        if constexpr (sizeof(T) == 2) {
          typedef __attribute__((address_space(3))) shortx4 *Lp;
          const int row = 4 * quarter + (col >> 2);
          const char *at0 = area + row * G::kRowBytes + (((2 * i + ((col & 3) >> 1)) ^ G::flip(row)) << 4) + 8 * (col & 1);
          const shortx4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)at0), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lp)(at0 + 16 * G::kRowBytes));
          const shortx8 b = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
          w[i % kAhead] = __builtin_bit_cast(bf16x8, b);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int row = 16 * (j >> 2) + 4 * quarter + (j & 3);
            w[i % kAhead][j] = *reinterpret_cast<const float *>(area + row * G::kRowBytes + (((4 * i + (col >> 2)) ^ G::flip(row)) << 4) + 4 * (col & 3));
          }
        }
        if (i % kAhead < kAhead - 1) continue;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int b = 0; b < kAhead; ++b) o[i - kAhead + 1 + b] = mma16(w[b], p, o[i - kAhead + 1 + b]);
        if constexpr (sizeof(T) == 2)
#pragma unroll
          for (int b = 0; b < kAhead; ++b) o[i - kAhead + 1 + b] = mma16(w[b], rest, o[i - kAhead + 1 + b]);
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    const float lift = power(fold_of(keys));
    l = sum4(l) * lift;

    // the wavefronts' outputs joined
    if (quarter == 0) ml[wave][col][0] = m, ml[wave][col][1] = l;
    const float by = l == 0.0f ? 0.0f : lift / l;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) *reinterpret_cast<floatx4 *>(area + (col * DP + 16 * i + 4 * quarter) * 4) = o[i] * by;
    __syncthreads();
    const bool full = units == per;
    const int slot = 2 * (int)blockIdx.x + (u == first ? 0 : 1);
    for (int i = threadIdx.x; i < heads * DP; i += kThreads) {
      const int h = i / DP, d = i % DP;
      float top = -INFINITY, sum = 0.0f, out = 0.0f, f[kWaves];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][h][0]);
      const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += f[w] = __builtin_amdgcn_exp2f(ml[w][h][0] - from) * ml[w][h][1];
      const float share = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) out += f[w] * share * *reinterpret_cast<const float *>(smem + w * kArea + i * 4);
      if (d >= a.D) continue;
      if (full) {
        const long to = (long)r * a.H + head0 + h;
        ((T *)a.o)[to * a.D + d] = (T)out;
        if (a.lse && d == 0) a.lse[to] = sum == 0.0f ? -INFINITY : top * kLn2 + logf(sum);
      } else {
        parts.o[((long)slot * kHeads + h) * parts.ld + d] = out;
        if (d == 0) parts.ml[(slot * kHeads + h) * 2] = top, parts.ml[(slot * kHeads + h) * 2 + 1] = sum;
      }
    }
    __syncthreads();
    u += units;
    if (rel + units == (long)per * VH) {
      base += (long)per * VH;
      if (u < end)   // some later request has the next unit
        do keys = __builtin_amdgcn_readfirstlane(keys_of(a, ++r));
        while (keys == 0);
    }
  }
}

// One request's heads that share a key head, or one of them, where more than one workgroup had a part of them: each head's factors by sixteen
// threads or a wavefront, then the outputs, four elements a thread and as many parts side by side as there are threads
template <class T>
__global__ __launch_bounds__(kThreads) void paged_join_kernel(const CacheArgs a, const Runs parts, int groups, const int single) {
  __shared__ long scratch[2 * kWaves];
  __shared__ float from[kHeads], total[kHeads], shift[kHeads];
  __shared__ floatx4 sums[kThreads];
  const int group = a.H / a.KV, VH = a.KV * parts.blocks, t = threadIdx.x;
  const int wide_group = min(kHeads, group), id = single ? blockIdx.x / wide_group : blockIdx.x, r = id / VH, vh = id % VH;
  const int per = units_of(keys_of(a, r));
  if (per <= 1) return;
  long before, all;
  add_units(a, r, &before, &all, scratch);
  all *= VH;
  groups = working(all, groups);
  const long unit = before * VH + (long)vh * per;
  const int w0 = owner_of(unit, all, groups), n = owner_of(unit + per - 1, all, groups) - w0 + 1;
  if (n == 1) return;
  const int slot0 = 2 * w0 + (unit == run_of(w0, all, groups) ? 0 : 1);
  const int block = vh % parts.blocks, all_heads = min(kHeads, group - block * kHeads),
            skip = single ? blockIdx.x % wide_group : 0, heads = single ? 1 : all_heads, head0 = vh / parts.blocks * group + block * kHeads + skip;
  if (skip >= all_heads) return;
  const auto row_of = [&](int i, int h) { return (long)(i == 0 ? slot0 : 2 * (w0 + i)) * kHeads + skip + h; };
  {
    const int lanes = single ? 64 : 16, h = single ? 0 : t / 16;
    float top = -INFINITY, sum = 0.0f;
    if (h < heads)
      for (int i = t % lanes; i < n; i += lanes) top = fmaxf(top, parts.ml[row_of(i, h) * 2]);
    for (int d = 1; d < lanes; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float base = top == -INFINITY ? 0.0f : top;
    if (h < heads)
      for (int i = t % lanes; i < n; i += lanes) sum += __builtin_amdgcn_exp2f(parts.ml[row_of(i, h) * 2] - base) * parts.ml[row_of(i, h) * 2 + 1];
    for (int d = 1; d < lanes; d *= 2) sum += __shfl_xor(sum, d);
    if (t % lanes == 0 && (!single || t == 0)) from[h] = base, total[h] = sum, shift[h] = top;
  }
  __syncthreads();
  const int wide = parts.ld / 4, items = heads * wide, side = max(1, kThreads / items);   // wide: 1 to 64
  for (int first = 0; first < items; first += kThreads) {   // more than one turn with more items than threads
    const int item = first + t % (side > 1 ? items : kThreads), p = side > 1 ? t / items : 0, h = min(item / wide, heads - 1), c = item % wide;
    const float share = total[h] == 0.0f ? 0.0f : 1.0f / total[h];
    floatx4 out = {};
    if (item < items && p < side)
#pragma unroll 4
      for (int i = p; i < n; i += side) {
        const long row = row_of(i, h);
        out += __builtin_amdgcn_exp2f(parts.ml[row * 2] - from[h]) * parts.ml[row * 2 + 1] * share * *reinterpret_cast<const floatx4 *>(parts.o + row * parts.ld + 4 * c);
      }
    if (side > 1) {
      sums[t] = out;
      __syncthreads();
      if (p > 0) return;
      for (int i = 1; i < side; ++i) out += sums[i * items + item];
    }
    if (item >= items) return;
    const long to = (long)r * a.H + head0 + h;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * c + j < a.D) ((T *)a.o)[to * a.D + 4 * c + j] = (T)out[j];
    if (a.lse && c == 0) a.lse[to] = total[h] == 0.0f ? -INFINITY : shift[h] * kLn2 + logf(total[h]);
  }
}

int blocks_of(const CacheArgs &a) { return (a.H / a.KV + kHeads - 1) / kHeads; }
// Workgroups: as many as the chip holds, and no more than units that there may be
int groups_of(const CacheArgs &a, int resident) {
  const long room = (long)a.columns * a.page, units = ((room + kUnit - 1) / kUnit) * a.R * a.KV * blocks_of(a), most = (long)resident * chip().cus;
  return (int)(units < most ? units : most < kMaxGroups ? most : kMaxGroups);
}

// The workspace's parts, the same walk for the query and the call
struct PagedParts {
  Runs parts;
  size_t bytes;
  PagedParts(const CacheArgs &a, char *base) {
    Take take{base};
    const size_t rows = (size_t)2 * groups_of(a, 2) * kHeads;
    parts.blocks = blocks_of(a);
    parts.ld = (a.D + 3) & ~3;
    parts.o = (float *)take(rows * parts.ld * sizeof(float));
    parts.ml = (float *)take(rows * 2 * sizeof(float));
    bytes = take.used;
  }
};

template <class T, int DP, bool WHOLE>
hipError_t paged_as(const CacheArgs &a, const Runs &parts, hipStream_t stream) {
  constexpr size_t lds = kWaves * kTile * Rows<T, DP>::kRowBytes + sizeof(Shared);
  const auto kernel = paged_attention_kernel<T, DP, WHOLE>;
  DLL_TRY(allow_large_lds(reinterpret_cast<const void *>(kernel), lds));
  const int groups = groups_of(a, residents<T, DP>());
  kernel<<<dim3((unsigned)groups), dim3(kThreads), lds, stream>>>(a, parts, Divisor(a.page));
  DLL_TRY(hipGetLastError());
  if ((long)a.columns * a.page <= kUnit) return hipSuccess;   // one unit a request and head
  // a workgroup a head while that makes no more than the chip takes at a time: 8 requests with 32 heads on 2 key heads 15.9 us, by key heads 20.0;
  // 64 requests with 32 on 8, 199.4 and 195.7
  const int single = (long)a.R * a.H <= 4L * chip().cus;
  const int wide_group = a.H / a.KV < kHeads ? a.H / a.KV : kHeads;
  paged_join_kernel<T><<<dim3((unsigned)(a.R * a.KV * parts.blocks * (single ? wide_group : 1))), dim3(kThreads), 0, stream>>>(a, parts, groups, single);
  return hipGetLastError();
}

template <class T>
hipError_t paged(const CacheArgs &a, const Runs &parts, hipStream_t stream) {
  if (a.D % 8) return a.D <= 64 ? paged_as<T, 64, false>(a, parts, stream) : a.D <= 128 ? paged_as<T, 128, false>(a, parts, stream) : paged_as<T, 256, false>(a, parts, stream);
  if (a.D <= 32) return paged_as<T, 32, true>(a, parts, stream);
  if (a.D <= 64) return paged_as<T, 64, true>(a, parts, stream);
  if (a.D <= 96) return paged_as<T, 96, true>(a, parts, stream);
  if (a.D <= 128) return paged_as<T, 128, true>(a, parts, stream);
  return paged_as<T, 256, true>(a, parts, stream);
}

}  // namespace

size_t paged_attention_scratch(const CacheArgs &a) { return PagedParts(a, nullptr).bytes; }

hipError_t launch_paged_attention(const CacheArgs &a, char *scratch, hipStream_t stream) {
  const PagedParts p(a, scratch);
  return a.dtype == TYPE_BF16 ? paged<bf16>(a, p.parts, stream) : paged<float>(a, p.parts, stream);
}

}  // namespace dllk
