// Attention over packed sequences, forward: o_i = sum_j softmax_j(scale q_i k_j) v_j over the keys that query i may see.
//
// One pass over the keys with a running maximum m and sum l for each query: p = exp2(s - m), l += sum p, o += p v, and where m grows,
// o and l shrink by exp2(old m - m).  The scale and log2 e are one factor.  m follows the true maximum only where that has grown by
// more than 2^8: until then p is at most 256, which its rounding does not mind, and o is left alone.  Sums that get near the largest number on their way
// are taken again with p times a power of two that brings all of a row's below 1 (the careful pass, with the same digits).
//
// A workgroup has 128 queries of one head, 32 a wavefront, which hold their rows of q as fragments.  Tiles of keys and values come
// straight into LDS, the next one while one is worked on.  Scores are taken transposed (keys are registers, the query is the lane), so
// maximum and sum are a lane's own but for the two halves, and p goes into the second product as it lies.  Where workgroups are few their
// wavefronts share 64 or 32 queries and take a tile's keys between them, joined in LDS at the end; where they are few still, the keys are
// cut into parts that a second launch joins.
//
// Bound by the matrix pipe beside the exponentials: a tile of 64 keys is 1024 cycles of products and 980 of vector instructions for a wavefront, and
// two wavefronts a SIMD overlap them only in part.  In bfloat16 p is rounded on its way into the second product: its rest in a second part would be half as many
// products again.  Heads of 128: 4096 tokens, all keys seen, 16 heads, 134 to 144 us = 950 to 1030 TFLOP/s; causal
// 88 to 94 us = 730 to 780 (its longest row of 64 tiles decides); 16384 tokens in five sequences 305 to 317 us = 900 to 940.  777 tokens, 16 heads of 64,
// 9.7 us (latency).  Tried and slower: exponentials of one block of keys beside the products of the next and the former (134 to 162 us), wavefront
// priorities around the products (the same), the second products beside the other half's exponentials (the same).
#include "attention_tile.h"

namespace dllk {

using namespace attn;

namespace {

constexpr int kThreads = 256, kMostRows = 4;

// A workgroup's four wavefronts are ROWS groups of 32 queries times 4 / ROWS groups that share a tile's keys.
template <class T, int DP, int ROWS>
struct Shape {
  // keys of a tile: 32 or 64 a wavefront, and 128 KB of LDS at most for the keys' and the values' two tiles (single precision: three planes)
  static constexpr int kKeyGroups = 4 / ROWS, kPer = ROWS < 4 || DP > 128 || (sizeof(T) == 4 && DP > 64) ? 32 : 64, kKeys = kPer * kKeyGroups;
  static constexpr int kQueries = 32 * ROWS;
  typedef Stager<T, DP, kKeys, kThreads> Rows;
  static constexpr int kLeft = DP * 128 + 512;   // bytes that a wavefront leaves for another one: its outputs, maxima and sums
  static constexpr int kTiles = 2 * Rows::kBytes > (kKeyGroups - 1) * ROWS * kLeft ? 2 * Rows::kBytes : (kKeyGroups - 1) * ROWS * kLeft, kLds = kTiles + kCareful;
  static constexpr bool kExists = ROWS == 4 || (sizeof(T) == 2 && kTiles <= 128 * 1024);
  // workgroups that a compute unit holds
  static constexpr int kResident = (sizeof(T) == 2 ? DP <= 128 : DP <= 96) && kLds <= 80 * 1024 ? 2 : 1;
};

template <class T, int DP, int ROWS>
__global__ __launch_bounds__(kThreads, (Shape<T, DP, ROWS>::kResident)) void attention_fwd_kernel(const AttentionArgs a, const Parts parts, const int tiles) {
  typedef Shape<T, DP, ROWS> Sh;
  typedef typename Sh::Rows S;
  constexpr int BN = Sh::kKeys, kPer = Sh::kPer, kQueries = Sh::kQueries;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int mine = wave / ROWS * kPer;   // this wavefront's keys of a tile
  // heads of one key head side by side, on as few XCDs as may be; the last tiles, which see most keys, first
  const int part = blockIdx.x % parts.n, id = blockIdx.x / parts.n, kv = id % a.KV, rest = id / a.KV, group = a.H / a.KV, head = kv * group + rest % group,
            tile = tiles - 1 - rest / group;
  const Place pq = place_of(a.q_starts, a.S, a.Tq, tile, kQueries);
  if (pq.at >= pq.count) return;
  const int kv_first = start_of(a.kv_starts, pq.sequence, a.Tk), keys = max(0, start_of(a.kv_starts, pq.sequence + 1, a.Tk) - kv_first);
  const int row0 = pq.at + 32 * (wave % ROWS), row = row0 + (lane & 31), shift = keys - pq.count;
  const int seen = a.causal ? max(0, min(keys, row + shift + 1)) : keys;                                    // by this lane's query
  const int seen_first = a.causal ? max(0, min(keys, row0 + shift + 1)) : keys;                             // by the wavefront's first
  const int seen_last = row0 >= pq.count ? 0 : a.causal ? max(0, min(keys, min(row0 + 32, pq.count) + shift)) : keys;   // by its last
  const int seen_all = a.causal ? max(0, min(keys, min(pq.at + kQueries, pq.count) + shift)) : keys;        // by the workgroup's last

  const T *k = (const T *)a.k + (long)kv_first * a.kv_row + kv * a.D, *v = (const T *)a.v + (long)kv_first * a.kv_row + kv * a.D;
  S sk, sv;
  sk.init(smem, k, a.kv_row, a.D);
  sv.init(smem + S::kBytes, v, a.kv_row, a.D);
  const int turns = (seen_all + BN - 1) / BN, begin = turn_from(part, parts.n, turns) * BN, end = min(seen_all, turn_from(part + 1, parts.n, turns) * BN);
  RowFrags<T, DP> q;   // with a scale below 0 the maximum of the scores is that of -q k
  q.load((const T *)a.q + (long)(pq.first + min(row, pq.count - 1)) * a.q_row + head * a.D, a.D, half, a.scale < 0.0f);
  const float c = factor_of(a.scale);

  floatx16 o[DP / 32];
  float m, l;
  const Reader<T, DP, BN> reader(lane);
  bool reached = false;   // by a value that is not finite, in a careful pass
  float lift = 1.0f;      // what o has to be multiplied with behind it
  const auto pass = [&](auto careful) {
    const float weight = power(-fold_of(keys));
    if (decltype(careful)::value) lift = power(fold_of(keys));
    sk.start(wave, k, begin, keys);
    sv.start(wave, v, begin, keys);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = floatx16{};
    m = -INFINITY, l = 0.0f;
    int odd = 1;
    for (int key0 = begin; key0 < end; key0 += BN, odd ^= 1) {
      landed<T>();
      const char *lk = sk.turn(wave, odd, k, key0 + BN, keys), *lv = sv.turn(wave, odd, v, key0 + BN, keys);
      written<T>();
      if (decltype(careful)::value && a.causal && key0 + BN > pq.at + shift + 1) {   // more keys than the workgroup's first query sees
        const Cleared c = clear_rows<T, DP, BN>(const_cast<char *>(lv), smem + Sh::kTiles);
        reached = reached || (c.first < BN && key0 + c.first < seen);
      }
      if (key0 + mine < seen_last) {
        floatx16 z[kPer / 32];
#pragma unroll
        for (int b = 0; b < kPer / 32; ++b) z[b] = floatx16{};
        // keys are read a step ahead of the products that take them
        Frag<T> kf[2][kPer / 32];
        const auto read = [&](int s) {
#pragma unroll
          for (int b = 0; b < kPer / 32; ++b) kf[s & 1][b] = reader.along(lk, mine + 32 * b, s);
        };
        read(0);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          if (s + 1 < DP / 16) read(s + 1);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int b = 0; b < kPer / 32; ++b) z[b] = mma(kf[s & 1][b], q[s], z[b]);
          __builtin_amdgcn_sched_barrier(0);
        }
        if (key0 + mine + kPer > seen_first)
#pragma unroll
          for (int b = 0; b < kPer / 32; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (key0 + mine + 32 * b + token_of(r) + 4 * half >= seen) z[b][r] = -INFINITY;
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < kPer / 32; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, z[b][r]);
        top = most_of_halves(top) * c;
        if (__any(top > m + 8.0f)) {
          const float grown = fmaxf(m, top), shrink = grown == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - grown);
          m = grown;
          l *= shrink;
#pragma unroll
          for (int i = 0; i < DP / 32; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= shrink;
        }
        const float from = m == -INFINITY ? 0.0f : m;
#pragma unroll
        for (int b = 0; b < kPer / 32; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            z[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][r], c, -from));
            l += z[b][r];
            if (decltype(careful)::value) z[b][r] *= weight;
          }
#pragma unroll
        for (int s = 0; s < kPer / 16; ++s) {
          const Frag<T> p = frag_of<T>(z[s / 2], s % 2);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) o[i] = mma(reader.across(lv, mine + 16 * s, 32 * i), p, o[i]);
        }
      }
    }
    arrived();
  };
  pass(std::false_type{});
  if (anyone(!all_small(o), smem + Sh::kTiles, wave)) pass(std::true_type{});
  if (reached)
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] += NAN;
  l = sum_of_halves(l);
  if constexpr (ROWS < 4) {   // the groups' outputs together, in the tiles' place, in the groups' order
    constexpr int kLeft = Sh::kLeft;
    barrier();
    if (wave >= ROWS) {
      char *to = smem + (wave - ROWS) * kLeft;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<floatx4 *>(to + ((i * 4 + r) * 64 + lane) * 16) = floatx4{o[i][4 * r], o[i][4 * r + 1], o[i][4 * r + 2], o[i][4 * r + 3]};
      float *ml = reinterpret_cast<float *>(to + DP * 128);
      ml[lane] = m;
      ml[64 + lane] = l;
    }
    __syncthreads();
    if (wave >= ROWS) return;
    float top = m;
#pragma unroll
    for (int g = 1; g < 4 / ROWS; ++g) top = fmaxf(top, reinterpret_cast<const float *>(smem + (wave + (g - 1) * ROWS) * kLeft + DP * 128)[lane]);
    const float from = top == -INFINITY ? 0.0f : top, own = __builtin_amdgcn_exp2f(m - from);
    l *= own;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] *= own;
#pragma unroll
    for (int g = 1; g < 4 / ROWS; ++g) {
      const char *other = smem + (wave + (g - 1) * ROWS) * kLeft;
      const float *ml = reinterpret_cast<const float *>(other + DP * 128), f = __builtin_amdgcn_exp2f(ml[lane] - from);
      l += f * ml[64 + lane];
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const floatx4 v = *reinterpret_cast<const floatx4 *>(other + ((i * 4 + r) * 64 + lane) * 16);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[i][4 * r + j] += f * v[j];
        }
    }
    m = top;
  }
  if (row >= pq.count) return;
  const long at = pq.first + row;
  const float by = l == 0.0f ? 0.0f : lift * (1.0f / l);
  if (parts.n > 1) {
    const long to = (long)part * a.Tq + at;
    store_sums(parts.sums[0] + (to * a.H + head) * parts.ld, o, parts.ld, half, by);
    if (half == 0) {
      float *ml = parts.ml + (((long)part * a.H + head) * a.Tq + at) * 2;
      ml[0] = m;
      ml[1] = l;
    }
    return;
  }
  store_row<T>((T *)a.o + at * a.H * a.D + head * a.D, o, by, a.D, half);
  if (a.lse && half == 0) a.lse[(long)head * a.Tq + at] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
}

// A row's parts, each with its own maximum and sum: a mean of their outputs.  Four elements a thread
template <class T>
__global__ __launch_bounds__(kThreads) void attention_join_kernel(const AttentionArgs a, const Parts parts, const long units) {
  const int wide = parts.ld / 4, first = start_of(a.q_starts, 0, a.Tq), end = start_of(a.q_starts, a.S, a.Tq);
  for (long u = (long)blockIdx.x * kThreads + threadIdx.x; u < units; u += (long)gridDim.x * kThreads) {
    const int d = (int)(u % wide) * 4;
    const long row = u / wide, head = row % a.H, at = row / a.H;
    if (at < first || at >= end) continue;   // nobody's
    floatx2 ml[kMostParts];   // all on their way at once
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) ml[p] = p < parts.n ? *reinterpret_cast<const floatx2 *>(parts.ml + ((p * (long)a.H + head) * a.Tq + at) * 2) : floatx2{-INFINITY, 0.0f};
    float top = -INFINITY, l = 0.0f;
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) top = fmaxf(top, ml[p][0]);
    const float from = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int p = 0; p < kMostParts; ++p) {
      ml[p][1] *= __builtin_amdgcn_exp2f(ml[p][0] - from);
      l += ml[p][1];
    }
    const float by = l == 0.0f ? 0.0f : 1.0f / l;
    floatx4 o = {};
#pragma unroll
    for (int p = 0; p < kMostParts; ++p)
      if (p < parts.n) o += ml[p][1] * by * *reinterpret_cast<const floatx4 *>(parts.sums[0] + ((p * (long)a.Tq + at) * a.H + head) * parts.ld + d);
    T *to = (T *)a.o + row * a.D + d;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (d + j < a.D) to[j] = (T)o[j];
    if (a.lse && d == 0) a.lse[head * a.Tq + at] = l == 0.0f ? -INFINITY : top * kLn2 + logf(l);
  }
}

// The workspace's parts, the same walk for the query and the call
struct FwdPlan {
  int rows = kMostRows;
  Parts parts;
  size_t bytes;
};
template <class T, int DP, int ROWS>
FwdPlan plan_as(const AttentionArgs &a, char *base) {
  typedef Shape<T, DP, ROWS> S;
  FwdPlan p;
  Take take{base};
  p.rows = ROWS;
  // four turns a part at least.  Microseconds with 2 / 4 / 8 / 16: 777 tokens, 4 heads of 64, 12.3 / 9.6 / 9.6 / 9.6; 1500, 4 of 128 on one, 24.4 / 24.4 / 21.2 / 21.2, in two 23.5 / 18.2 / 18.2 / 18.2;
  // 600, 8 of 256, 33.8 / 26.3 / 25.1 / 25.1; in single precision 500, 8 of 64, 20.6 / 28.4 / 28.4 / 28.4, 1000, 8 of 128, 43.5 / 43.4 / 49.7 / 96.1, 2001 ragged, six of 80, 51.2 / 48.8 / 54.0 / 82.5
  p.parts.n = parts_of((a.Tq + S::kQueries - 1) / S::kQueries * (long)a.H, tiles_of(a.Tq, a.S, S::kQueries) * a.H, (long)(ROWS == 4 ? S::kResident : 1) * chip().cus,
                       a.Tk / a.S / S::kKeys, 4);
  p.parts.ld = (a.D + 3) & ~3;
  if (p.parts.n > 1) {
    p.parts.sums[0] = (float *)take((size_t)p.parts.n * a.Tq * a.H * p.parts.ld * sizeof(float));
    p.parts.ml = (float *)take((size_t)p.parts.n * a.Tq * a.H * 2 * sizeof(float));
  }
  p.bytes = take.used;
  return p;
}
template <class T, int DP>
FwdPlan plan(const AttentionArgs &a, char *base) {
  // as many workgroups of 128 queries as there are at least.  Microseconds with 128 / 64 / 32 queries a workgroup: 777 tokens, 16 heads of 64 18 / 17 / 11; 1000, 8 of 128
  // 24 / 22 / 18; 300, 8 of 128 11.6 / 10.2 / 11.1; 2048, 8 of 128 33 / 33 / 34; 3000, 16 of 64 44 / 39 / 48; 4096 in 50 sequences, 16 of 64 14 / 15 / 28.  Single
  // precision gains nothing from fewer (1000, 8 of 128: 42 / 43 / 43) as its rows are split by four wavefronts for four.
  const long all = (a.Tq + 127) / 128 > a.S ? (a.Tq + 127) / 128 : a.S, workgroups = all * a.H;
  if constexpr (Shape<T, DP, 2>::kExists) {
    if constexpr (Shape<T, DP, 1>::kExists)
      if (2 * workgroups < chip().cus && a.Tk / a.S >= 512) return plan_as<T, DP, 1>(a, base);
    if (workgroups < 2 * chip().cus) return plan_as<T, DP, 2>(a, base);
  }
  return plan_as<T, DP, 4>(a, base);
}

template <class T, int DP, int ROWS>
hipError_t fwd_as(const AttentionArgs &a, const FwdPlan &p, hipStream_t stream) {
  typedef Shape<T, DP, ROWS> S;
  if constexpr (S::kExists) {
    const auto kernel = attention_fwd_kernel<T, DP, ROWS>;
    DLL_TRY(allow_large_lds(reinterpret_cast<const void *>(kernel), S::kLds));
    const long tiles = tiles_of(a.Tq, a.S, S::kQueries);
    kernel<<<dim3((unsigned)(tiles * a.H * p.parts.n)), dim3(kThreads), S::kLds, stream>>>(a, p.parts, (int)tiles);
    DLL_TRY(hipGetLastError());
    if (p.parts.n == 1) return hipSuccess;
    const long units = (long)a.Tq * a.H * (p.parts.ld / 4), blocks = (units + kThreads - 1) / kThreads;
    attention_join_kernel<T><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kThreads), 0, stream>>>(a, p.parts, units);
    return hipGetLastError();
  }
  return hipErrorInvalidValue;   // not planned
}

template <class T>
hipError_t fwd(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  return instance(a.D, [&](auto dp) {
    constexpr int DP = decltype(dp)::value;
    const FwdPlan p = plan<T, DP>(a, scratch);
    return p.rows == 4 ? fwd_as<T, DP, 4>(a, p, stream) : p.rows == 2 ? fwd_as<T, DP, 2>(a, p, stream) : fwd_as<T, DP, 1>(a, p, stream);
  });
}
template <class T>
size_t fwd_bytes(const AttentionArgs &a) {
  return instance(a.D, [&](auto dp) { return plan<T, decltype(dp)::value>(a, nullptr).bytes; });
}

}  // namespace

bool attention_fits(int q_tokens, int kv_tokens, int sequences, int heads) {
  return tiles_of(q_tokens > kv_tokens ? q_tokens : kv_tokens, sequences, 32) * heads <= kMaxGrid;
}

size_t attention_fwd_scratch(const AttentionArgs &a) { return (a.dtype == TYPE_BF16 ? fwd_bytes<bf16>(a) : fwd_bytes<float>(a)) + 1; }   // never nothing

hipError_t launch_attention_fwd(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? fwd<bf16>(a, scratch, stream) : fwd<float>(a, scratch, stream);
}

}  // namespace dllk
