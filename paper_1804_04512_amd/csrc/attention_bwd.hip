// Attention over packed sequences, backward, from q, k, v, the outputs o, their gradients do and lse_i = ln sum_j exp s_ij:
//   p_ij = exp(s_ij - lse_i), delta_i = do_i . o_i, ds_ij = p_ij (do_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij do_i
//
// Two kernels, so that every sum has one owner and a fixed order: one has 128 queries of a head and goes over the keys (dq), the
// other 128 keys of a key head and goes over the queries of its heads (dk, dv).  Both take scores and do.v again, seven products for
// the five of one kernel that would have to add its dq up in memory.  32 rows a wavefront stay in registers as fragments; the others come
// through LDS tile by tile, read along a head's elements for the scores and across tokens for the sums.  p and ds go from one
// product's result to the next one's operand in registers, rounded to the operands' type there.
#include "attention_tile.h"

namespace dllk {

using namespace attn;

namespace {

constexpr int kRows = 128, kThreads = 256;

template <class T, int DP> constexpr int tile_rows() { return Tile<T, DP>::kRowBytes >= 512 ? 32 : 64; }

// Four bytes a lane from the buffer to 256 bytes of LDS, as load_to_lds
__device__ __forceinline__ void load_words_to_lds(const uintx4 &rs, unsigned off, unsigned lds) {
  const unsigned at = (unsigned)__builtin_amdgcn_readfirstlane((int)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(rs) : "memory");
}

// Per query, [H][Tq]: lse in the exponent's base, and -delta, which the products with v start from
struct Rows {
  float *lse2, *minus_delta;
};

template <class T, int DP>
__device__ __forceinline__ float row_delta(const Frag<T> (&g)[DP / 16], const T *o, int dim, int half) {
  float sum = 0.0f;
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    Eight<T> e;
    const int at = 16 * s + 8 * half;
    e.load(o + at, dim - at);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += to_float(g[s][j]) * to_float(e.v[j]);
  }
  return sum + other_half(sum);
}

// ------------------------------------------------------------------------------------------------ dq
// dq may be NULL: then the rows' figures are all that is wanted
template <class T, int DP, int BN>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 ? DP <= 96 : DP <= 64) ? 2 : 1) void attention_dq_kernel(const AttentionArgs a, const Rows rows, const int tiles) {
  typedef Stager<T, DP, BN, kThreads> S;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int kv = blockIdx.x % a.KV, rest = blockIdx.x / a.KV, group = a.H / a.KV, head = kv * group + rest % group, tile = tiles - 1 - rest / group;
  const Place pq = place_of(a.q_starts, a.S, a.Tq, tile, kRows);
  if (pq.at >= pq.count) return;
  const int kv_first = start_of(a.kv_starts, pq.sequence, a.Tk), keys = max(0, start_of(a.kv_starts, pq.sequence + 1, a.Tk) - kv_first);
  const int row0 = pq.at + 32 * wave, row = row0 + (lane & 31), shift = keys - pq.count;
  const int seen = a.causal ? max(0, min(keys, row + shift + 1)) : keys;
  const int seen_first = a.causal ? max(0, min(keys, row0 + shift + 1)) : keys;
  const int seen_last = row0 >= pq.count ? 0 : a.causal ? max(0, min(keys, min(row0 + 32, pq.count) + shift)) : keys;
  const int seen_all = a.causal ? max(0, min(keys, min(pq.at + kRows, pq.count) + shift)) : keys;

  Frag<T> g[DP / 16];
  const long at = pq.first + min(row, pq.count - 1);
  load_row<T, DP>(g, (const T *)a.d_o + at * a.H * a.D + head * a.D, a.D, half);
  const float minus_delta = -row_delta<T, DP>(g, (const T *)a.o + at * a.H * a.D + head * a.D, a.D, half);
  const float lse2 = a.lse[(long)head * a.Tq + at] * kLog2e;
  if (half == 0 && row < pq.count) {
    rows.lse2[(long)head * a.Tq + at] = lse2;
    rows.minus_delta[(long)head * a.Tq + at] = minus_delta;
  }
  if (!a.dq) return;

  S sk, sv;
  sk.init((const T *)a.k + (long)kv_first * a.kv_row + kv * a.D, a.kv_row, a.D, threadIdx.x);
  sv.init((const T *)a.v + (long)kv_first * a.kv_row + kv * a.D, a.kv_row, a.D, threadIdx.x);
  const auto load = [&](int stage, int key0) {
    char *to = smem + stage * 2 * S::kBytes;
    sk.load(to, wave, key0, keys);
    sv.load(to + S::kBytes, wave, key0, keys);
  };
  load(0, 0);
  Frag<T> q[DP / 16];
  load_row<T, DP>(q, (const T *)a.q + at * a.q_row + head * a.D, a.D, half);
  const float c = a.scale * kLog2e;

  floatx16 dq[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) dq[i] = floatx16{};
  const Reader<T, DP> reader(lane);
  int stage = 0;
  for (int key0 = 0; key0 < seen_all; key0 += BN, stage ^= 1) {
    load(stage ^ 1, key0 + BN);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * S::kLoads) : "memory");
    barrier();
    const char *lk = smem + stage * 2 * S::kBytes, *lv = lk + S::kBytes;
#pragma unroll 1
    for (int b = 0; b < BN && key0 + b < seen_last; b += 32) {
      floatx16 z = {}, d;
#pragma unroll
      for (int r = 0; r < 16; ++r) d[r] = minus_delta;
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        z = mma(reader.along(lk, b, s), q[s], z);
        d = mma(reader.along(lv, b, s), g[s], d);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[r], c, -lse2));
      if (key0 + b + 32 > seen_first)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key0 + b + token_of(r) + 4 * half >= seen) z[r] = 0.0f, d[r] = 0.0f;
#pragma unroll
      for (int r = 0; r < 16; ++r) d[r] *= z[r];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const Frag<T> ds = frag_of<T>(d, s);
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) dq[i] = mma(reader.across(lk, b + 16 * s, 32 * i), ds, dq[i]);
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (row >= pq.count) return;
  store_row<T>((T *)a.dq + at * a.q_row + head * a.D, dq, a.scale, a.D, half);
}

// ------------------------------------------------------------------------------------------------ dk, dv
// DK, DV: which of the two this instance takes (single precision with more than 128 elements a head takes them one after the other, as their
// sums and both rows would not fit the registers)
template <class T, int DP, int BN, bool DK, bool DV>
__global__ __launch_bounds__(kThreads, (sizeof(T) == 2 ? DP <= 64 : DP <= 32) ? 2 : 1) void attention_dkv_kernel(const AttentionArgs a, const Rows rows) {
  typedef Stager<T, DP, BN, kThreads> S;
  constexpr int kStage = 2 * S::kBytes + 2 * 256, kWait = 2 * S::kLoads + 1;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int kv = blockIdx.x % a.KV, tile = blockIdx.x / a.KV, group = a.H / a.KV;
  const Place pk = place_of(a.kv_starts, a.S, a.Tk, tile, kRows);
  if (pk.at >= pk.count) return;
  const int q_first = start_of(a.q_starts, pk.sequence, a.Tq), queries = max(0, start_of(a.q_starts, pk.sequence + 1, a.Tq) - q_first);
  const int key0 = pk.at + 32 * wave, key = key0 + (lane & 31), shift = pk.count - queries;
  const int from = a.causal ? max(0, pk.at - shift) : 0;         // the first query that sees any of the workgroup's keys
  const int sees = key - shift;                                  // the first that sees this lane's key, where causal
  const int sees_first = key0 - shift, sees_all = key0 + 31 - shift;

  const long at = pk.first + min(key, pk.count - 1);
  Frag<T> k[DP / 16], v[DK ? DP / 16 : 1];
  load_row<T, DP>(k, (const T *)a.k + at * a.kv_row + kv * a.D, a.D, half);
  if constexpr (DK) load_row<T, DP>(v, (const T *)a.v + at * a.kv_row + kv * a.D, a.D, half);
  const float c = a.scale * kLog2e;
  floatx16 dk[DK ? DP / 32 : 1], dv[DV ? DP / 32 : 1];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) {
    if (DK) dk[i] = floatx16{};
    if (DV) dv[i] = floatx16{};
  }
  const Reader<T, DP> reader(lane);
  S sq, sg;
  sq.init(a.q, a.q_row, a.D, threadIdx.x);
  sg.init(a.d_o, (long)a.H * a.D, a.D, threadIdx.x);
  // turns: the group's heads, each over the tiles of queries
  const int tiles = queries > from ? (queries - from + BN - 1) / BN : 0, turns = tiles * group;
  const auto load = [&](int stage, int turn) {   // behind the last turn: zeros
    const int h = kv * group + min(turn / max(tiles, 1), group - 1), i0 = turn < turns ? from + (turn % max(tiles, 1)) * BN : queries;
    char *to = smem + stage * kStage;
    sq.base = (const char *)((const T *)a.q + (long)q_first * a.q_row + h * a.D);
    sg.base = (const char *)((const T *)a.d_o + ((long)q_first * a.H + h) * a.D);
    sq.load(to, wave, i0, queries);
    sg.load(to + S::kBytes, wave, i0, queries);
    // two wavefronts bring the one, two the other: as many loads on their way in each
    const float *figures = (wave & 1 ? rows.minus_delta : rows.lse2) + (long)h * a.Tq + q_first + i0;
    const uintx4 rs = buffer_of((const char *)figures, (unsigned)max(0, min(queries - i0, BN)) * 4u);
    load_words_to_lds(rs, lane * 4, (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)(to + 2 * S::kBytes + (wave & 1) * 256));
  };
  if (turns > 0) load(0, 0);
  int stage = 0;
  for (int turn = 0; turn < turns; ++turn, stage ^= 1) {
    load(stage ^ 1, turn + 1);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kWait) : "memory");
    barrier();
    const char *lq = smem + stage * kStage, *lg = lq + S::kBytes;
    const float *lse2 = reinterpret_cast<const float *>(lg + S::kBytes), *minus_delta = lse2 + 64;
    const int i0 = from + (turn % tiles) * BN;
#pragma unroll 1
    for (int b = 0; b < BN && i0 + b < queries; b += 32) {
      if (a.causal && i0 + b + 31 < sees_first) continue;
      floatx16 z = {}, d;
      if constexpr (DK)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const floatx4 w = *reinterpret_cast<const floatx4 *>(minus_delta + b + 8 * r + 4 * half);
#pragma unroll
          for (int j = 0; j < 4; ++j) d[4 * r + j] = w[j];
        }
#pragma unroll
      for (int s = 0; s < DP / 16; ++s) {
        z = mma(reader.along(lq, b, s), k[s], z);
        if constexpr (DK) d = mma(reader.along(lg, b, s), v[s], d);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const floatx4 w = *reinterpret_cast<const floatx4 *>(lse2 + b + 8 * r + 4 * half);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[4 * r + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[4 * r + j], c, -w[j]));
      }
      if (a.causal && i0 + b < sees_all)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (i0 + b + token_of(r) + 4 * half < sees) {
            z[r] = 0.0f;
            if constexpr (DK) d[r] = 0.0f;
          }
      if constexpr (DK)
#pragma unroll
        for (int r = 0; r < 16; ++r) d[r] *= z[r];
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if constexpr (DV) {
          const Frag<T> p = frag_of<T>(z, s);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) dv[i] = mma(reader.across(lg, b + 16 * s, 32 * i), p, dv[i]);
        }
        if constexpr (DK) {
          const Frag<T> ds = frag_of<T>(d, s);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) dk[i] = mma(reader.across(lq, b + 16 * s, 32 * i), ds, dk[i]);
        }
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (key >= pk.count) return;
  if (DK && a.dk) store_row<T>((T *)a.dk + at * a.kv_row + kv * a.D, dk, a.scale, a.D, half);
  if (DV && a.dv) store_row<T>((T *)a.dv + at * a.kv_row + kv * a.D, dv, 1.0f, a.D, half);
}

// ------------------------------------------------------------------------------------------------ host
template <class T, int DP>
hipError_t dq_as(const AttentionArgs &a, const Rows &rows, hipStream_t stream) {
  constexpr int BN = tile_rows<T, DP>();
  constexpr size_t lds = 4 * Stager<T, DP, BN, kThreads>::kBytes;
  const auto kernel = attention_dq_kernel<T, DP, BN>;
  DLL_TRY(allow_large_lds(reinterpret_cast<const void *>(kernel), lds));
  const long tiles = tiles_of(a.Tq, a.S, kRows), grid = tiles * a.H;
  kernel<<<dim3((unsigned)grid), dim3(kThreads), lds, stream>>>(a, rows, (int)tiles);
  return hipGetLastError();
}

template <class T, int DP, bool DK, bool DV>
hipError_t dkv_as(const AttentionArgs &a, const Rows &rows, hipStream_t stream) {
  constexpr int BN = tile_rows<T, DP>();
  constexpr size_t lds = 2 * (2 * Stager<T, DP, BN, kThreads>::kBytes + 2 * 256);
  const auto kernel = attention_dkv_kernel<T, DP, BN, DK, DV>;
  DLL_TRY(allow_large_lds(reinterpret_cast<const void *>(kernel), lds));
  const long grid = tiles_of(a.Tk, a.S, kRows) * a.KV;
  kernel<<<dim3((unsigned)grid), dim3(kThreads), lds, stream>>>(a, rows);
  return hipGetLastError();
}

template <class T, int DP>
hipError_t bwd_as(const AttentionArgs &a, const Rows &rows, hipStream_t stream) {
  DLL_TRY((dq_as<T, DP>(a, rows, stream)));
  if (!a.dk && !a.dv) return hipSuccess;
  if constexpr (sizeof(T) == 4 && DP > 128) {
    if (a.dv) DLL_TRY((dkv_as<T, DP, false, true>(a, rows, stream)));
    return a.dk ? dkv_as<T, DP, true, false>(a, rows, stream) : hipSuccess;
  } else {
    return dkv_as<T, DP, true, true>(a, rows, stream);
  }
}

template <class T>
hipError_t bwd(const AttentionArgs &a, const Rows &rows, hipStream_t stream) {
  if (a.D <= 32) return bwd_as<T, 32>(a, rows, stream);
  if (a.D <= 64) return bwd_as<T, 64>(a, rows, stream);
  if (a.D <= 96) return bwd_as<T, 96>(a, rows, stream);
  if (a.D <= 128) return bwd_as<T, 128>(a, rows, stream);
  return bwd_as<T, 256>(a, rows, stream);
}

// The workspace's parts, the same walk for the query and the call
struct BwdParts {
  Rows rows;
  size_t bytes;
  BwdParts(const AttentionArgs &a, char *base) {
    Take take{base};
    rows.lse2 = (float *)take((size_t)a.H * a.Tq * sizeof(float));
    rows.minus_delta = (float *)take((size_t)a.H * a.Tq * sizeof(float));
    bytes = take.used;
  }
};

}  // namespace

size_t attention_bwd_scratch(const AttentionArgs &a) { return BwdParts(a, nullptr).bytes; }

hipError_t launch_attention_bwd(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  const BwdParts p(a, scratch);
  return a.dtype == TYPE_BF16 ? bwd<bf16>(a, p.rows, stream) : bwd<float>(a, p.rows, stream);
}

}  // namespace dllk
