// Attention over packed sequences, forward: o_i = sum_j softmax_j(scale q_i k_j) v_j over the keys that query i may see.
//
// One pass over the keys with a running maximum m and sum l for each query: p = exp2(s - m), l += sum p, o += p v, and where m grows,
// o and l shrink by exp2(old m - m).  The scale and log2 e are one factor.  m follows the true maximum only where that has grown by
// more than 2^8: until then p is at most 256, which neither its rounding nor the sums mind, and o is left alone.
//
// A workgroup has 128 queries of one head, 32 a wavefront, which hold their rows of q as fragments.  Tiles of keys and values come
// straight into LDS, the next one while one is worked on.  Scores are taken transposed (keys are registers, the query is the lane), so
// maximum and sum are a lane's own but for the two halves, and p goes into the second product as it lies.
#include "attention_tile.h"

namespace dllk {

using namespace attn;

namespace {

constexpr int kQueries = 128, kThreads = 256;

template <class T, int DP> constexpr int keys_of() { return Tile<T, DP>::kRowBytes >= 512 ? 32 : 64; }

template <class T, int DP, int BN>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 ? DP <= 128 : DP <= 96) ? 2 : 1) void attention_fwd_kernel(const AttentionArgs a, const int tiles) {
  typedef Stager<T, DP, BN, kThreads> S;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  // heads of one key head side by side, on as few XCDs as may be; the last tiles, which see most keys, first
  const int kv = blockIdx.x % a.KV, rest = blockIdx.x / a.KV, group = a.H / a.KV, head = kv * group + rest % group, tile = tiles - 1 - rest / group;
  const Place pq = place_of(a.q_starts, a.S, a.Tq, tile, kQueries);
  if (pq.at >= pq.count) return;
  const int kv_first = start_of(a.kv_starts, pq.sequence, a.Tk), keys = max(0, start_of(a.kv_starts, pq.sequence + 1, a.Tk) - kv_first);
  const int row0 = pq.at + 32 * wave, row = row0 + (lane & 31), shift = keys - pq.count;
  const int seen = a.causal ? max(0, min(keys, row + shift + 1)) : keys;                                    // by this lane's query
  const int seen_first = a.causal ? max(0, min(keys, row0 + shift + 1)) : keys;                             // by the wavefront's first
  const int seen_last = row0 >= pq.count ? 0 : a.causal ? max(0, min(keys, min(row0 + 32, pq.count) + shift)) : keys;   // by its last
  const int seen_all = a.causal ? max(0, min(keys, min(pq.at + kQueries, pq.count) + shift)) : keys;        // by the workgroup's last

  S sk, sv;
  sk.init((const T *)a.k + (long)kv_first * a.kv_row + kv * a.D, a.kv_row, a.D, threadIdx.x);
  sv.init((const T *)a.v + (long)kv_first * a.kv_row + kv * a.D, a.kv_row, a.D, threadIdx.x);
  const auto load = [&](int stage, int key0) {   // behind the last key: zeros
    char *at = smem + stage * 2 * S::kBytes;
    sk.load(at, wave, key0, keys);
    sv.load(at + S::kBytes, wave, key0, keys);
  };
  load(0, 0);
  Frag<T> q[DP / 16];
  load_row<T, DP>(q, (const T *)a.q + (long)(pq.first + min(row, pq.count - 1)) * a.q_row + head * a.D, a.D, half);
  if (a.scale < 0.0f)   // the maximum of the scores is then that of -q k
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) q[s] = -q[s];
  const float c = fmaxf(fabsf(a.scale) * kLog2e, 0x1p-126f);   // a masked score of -infinity stays one where the scale is 0

  floatx16 o[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = floatx16{};
  float m = -INFINITY, l = 0.0f;
  const Reader<T, DP> reader(lane);
  int stage = 0;
  for (int key0 = 0; key0 < seen_all; key0 += BN, stage ^= 1) {
    load(stage ^ 1, key0 + BN);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * S::kLoads) : "memory");
    barrier();
    if (key0 < seen_last) {
      const char *lk = smem + stage * 2 * S::kBytes, *lv = lk + S::kBytes;
      floatx16 z[BN / 32];
#pragma unroll
      for (int b = 0; b < BN / 32; ++b) z[b] = floatx16{};
#pragma unroll
      for (int s = 0; s < DP / 16; ++s)
#pragma unroll
        for (int b = 0; b < BN / 32; ++b) z[b] = mma(reader.along(lk, 32 * b, s), q[s], z[b]);
      if (key0 + BN > seen_first)
#pragma unroll
        for (int b = 0; b < BN / 32; ++b)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (key0 + 32 * b + token_of(r) + 4 * half >= seen) z[b][r] = -INFINITY;
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < BN / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, z[b][r]);
      top = fmaxf(top, other_half(top)) * c;
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
      for (int b = 0; b < BN / 32; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          z[b][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[b][r], c, -from));
          l += z[b][r];
        }
#pragma unroll
      for (int s = 0; s < BN / 16; ++s) {
        const Frag<T> p = frag_of<T>(z[s / 2], s % 2);
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) o[i] = mma(reader.across(lv, 16 * s, 32 * i), p, o[i]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // of the tile of zeros too
  if (row >= pq.count) return;
  l += other_half(l);
  const long at = pq.first + row;
  store_row<T>((T *)a.o + at * a.H * a.D + head * a.D, o, l == 0.0f ? 0.0f : 1.0f / l, a.D, half);
  if (a.lse && half == 0) a.lse[(long)head * a.Tq + at] = l == 0.0f ? -INFINITY : m * kLn2 + logf(l);
}

template <class T, int DP>
hipError_t fwd_as(const AttentionArgs &a, hipStream_t stream) {
  constexpr int BN = keys_of<T, DP>();
  constexpr size_t lds = 4 * Stager<T, DP, BN, kThreads>::kBytes;
  const auto kernel = attention_fwd_kernel<T, DP, BN>;
  const hipError_t e = allow_large_lds(reinterpret_cast<const void *>(kernel), lds);
  if (e != hipSuccess) return e;
  const long tiles = tiles_of(a.Tq, a.S, kQueries), grid = tiles * a.H;
  kernel<<<dim3((unsigned)grid), dim3(kThreads), lds, stream>>>(a, (int)tiles);
  return hipGetLastError();
}

template <class T>
hipError_t fwd(const AttentionArgs &a, hipStream_t stream) {
  if (a.D <= 32) return fwd_as<T, 32>(a, stream);
  if (a.D <= 64) return fwd_as<T, 64>(a, stream);
  if (a.D <= 96) return fwd_as<T, 96>(a, stream);
  if (a.D <= 128) return fwd_as<T, 128>(a, stream);
  return fwd_as<T, 256>(a, stream);
}

}  // namespace

bool attention_fits(int q_tokens, int kv_tokens, int sequences, int heads) {
  return tiles_of(q_tokens > kv_tokens ? q_tokens : kv_tokens, sequences, kQueries) * heads <= kMaxGrid;
}

size_t attention_fwd_scratch(const AttentionArgs &) { return 256; }

hipError_t launch_attention_fwd(const AttentionArgs &a, char *, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? fwd<bf16>(a, stream) : fwd<float>(a, stream);
}

}  // namespace dllk
