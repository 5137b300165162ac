// Attention over packed sequences, backward, from q, k, v, the outputs o, their gradients do and lse_i = ln sum_j exp s_ij:
//   p_ij = exp(s_ij - lse_i), delta_i = do_i . o_i, ds_ij = p_ij (do_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j, dk_j = scale sum_i ds_ij q_i, dv_j = sum_i p_ij do_i
//
// Two kernels, so that every sum has one owner and a fixed order: one has 128 queries of a head and goes over the keys (dq), the
// other 128 keys of a key head and goes over the queries of its heads (dk, dv).  Both take scores and do.v again, seven products for
// the five of one kernel that would have to add its dq up in memory.  32 rows a wavefront stay in registers as fragments; the others come
// through LDS tile by tile, read along a head's elements for the scores and across tokens for the sums.  p and ds go from one
// product's result to the next one's operand in registers, rounded to the operands' type there (in bfloat16 a second part of each would be two products
// more, of nine).
//
// Bound by the matrix pipe and by what stands between its products (exponentials, waits for fragments).  4096 tokens, causal, 16 heads of 128 in
// bfloat16: dq 126 us, dk and dv 183 us, 172 GFLOP of five products at 555 TFLOP/s, and of the seven that are done at 780.
// 2001 tokens in three sequences, six heads of 80 on three in single precision: dq 68, dk and dv 73 and their parts' sums 12 us.
// Tried and slower: two blocks of scores a turn with one's exponentials between the other's products (twice the registers, sums moved
// between the register files at each product: 390 to 840 us for the pass), fragments three steps ahead instead of one (the same), all
// fragments of the second products ahead of the exponentials (3 % slower).
#include "attention_tile.h"

namespace dllk {

using namespace attn;

namespace {

constexpr int kRows = 128, kThreads = 256;

template <class T, int DP> constexpr int tile_rows() { return DP > 128 || (sizeof(T) == 4 && DP > 64) ? 32 : 64; }

// Four bytes a lane from the buffer to 256 bytes of LDS, as load_to_lds
__device__ __forceinline__ void load_words_to_lds(const uintx4 &rs, unsigned off, unsigned lds) {
  const unsigned at = (unsigned)__builtin_amdgcn_readfirstlane((int)lds);
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(at), "v"(off), "s"(rs) : "memory");
}

// Per query, [H][Tq]: lse in the exponent's base, and -delta, which the products with v start from
struct Rows {
  float *lse2, *minus_delta;
  unsigned *again = nullptr;   // per workgroup, where the careful pass is a launch of its own: whether it is to be taken
};

// Where a kernel's careful pass is.  NONE: without a mask there is none; HERE: a second copy of the loop; a launch of its own, after that of
// the workgroups that leave word where it is needed (LEAVE), by those that find it (TAKE).  As compiled, the copy makes no kernel spill but dq's of 97 to 128 elements in
// bfloat16 with 128 queries (36 bytes a lane, outside the loop: 4224 tokens, 16 heads, 310 us, as a launch 319).  Where sums and rows fill the registers anyway it makes the usual
// pass slower: 2048 tokens in two sequences, causal, 4 heads on 2, of 128 in single precision, microseconds without it / HERE / as a launch: 171 / 235 / 176; of 256, 725 / 839 / 749; in
// bfloat16 332 / 408 / 341; 2001 ragged ones, six heads of 80 in single precision 146 / 162 / 153.  Without a mask the latter take 200 with NONE, 214 with HERE.
// Scratch of the usual pass, bytes a lane: single precision, dk and dv of 97 to 128 elements 240, of 129 to 256 dq 1250 to 1270, dk 510, dv 1210 to 1230; bfloat16, dk and dv
// of 129 to 256 870.
enum Careful { NONE, HERE, LEAVE, TAKE };
template <class T, int DP> constexpr bool dq_apart() { return DP > 128; }
template <class T, int DP> constexpr bool dkv_apart() { return DP > (sizeof(T) == 2 ? 128 : 64); }

// The sum of two rows' products, over both lane halves
template <class T, int DP>
__device__ __forceinline__ float row_product(const T *x, const T *y, int dim, int half) {
  float sum = 0.0f;
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    Eight<T> e, f;
    const int at = 16 * s + 8 * half;
    e.load(x + at, dim - at);
    f.load(y + at, dim - at);
#pragma unroll
    for (int j = 0; j < 8; ++j) sum += to_float(e.v[j]) * to_float(f.v[j]);
  }
  return sum_of_halves(sum);
}

// ------------------------------------------------------------------------------------------------ dq
// workgroups that a compute unit holds, by their registers.  Single precision of 33 to 64 elements spills 75 of them with two; backward pass, microseconds with two / one:
// 1024 tokens, 8 heads of 64 on 2, 74.1 / 66.3, all keys seen 79.3 / 71.4; 2048 in two, 4 on 2, 77.4 / 66.3; 600 in 24, 8 heads, 22.5 / 20.0; 8192 in four, 16 heads, 749 / 685,
// all keys seen 1240 / 1231; 4096, 8 heads, 529 / 565 (as many workgroups as units, so not cut into parts).  Two with the careful pass as a launch of its own
// spill 33 and take 72.9, 76.4, 76.4, 22.7, 718, 1213 and 512.
template <class T, int DP> constexpr int dq_residents() { return (sizeof(T) == 2 ? DP <= 128 : DP <= 32) ? 2 : 1; }

// dq may be NULL: then the rows' figures are all that is wanted
// ROWS groups of 32 queries; with two, the wavefronts share a tile's keys two by two
template <class T, int DP, int BN, int ROWS, Careful CARE>
__global__ __launch_bounds__(kThreads, (dq_residents<T, DP>())) void attention_dq_kernel(const AttentionArgs a, const Rows rows, const Parts parts, const int tiles) {
  constexpr int kQueries = 32 * ROWS, kPer = BN * ROWS / 4;   // keys of a tile that a wavefront takes
  typedef Stager<T, DP, BN, kThreads> S;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int part = blockIdx.x % parts.n, id = blockIdx.x / parts.n, kv = id % a.KV, rest = id / a.KV, group = a.H / a.KV, head = kv * group + rest % group,
            tile = tiles - 1 - rest / group;
  const Place pq = place_of(a.q_starts, a.S, a.Tq, tile, kQueries);
  if (pq.at >= pq.count || (CARE == TAKE && !rows.again[blockIdx.x])) return;
  const int kv_first = start_of(a.kv_starts, pq.sequence, a.Tk), keys = max(0, start_of(a.kv_starts, pq.sequence + 1, a.Tk) - kv_first);
  const int mine = wave / ROWS * kPer, row0 = pq.at + 32 * (wave % ROWS), row = row0 + (lane & 31), shift = keys - pq.count;
  const int seen = a.causal ? max(0, min(keys, row + shift + 1)) : keys;
  const int seen_first = a.causal ? max(0, min(keys, row0 + shift + 1)) : keys;
  const int seen_last = row0 >= pq.count ? 0 : a.causal ? max(0, min(keys, min(row0 + 32, pq.count) + shift)) : keys;
  const int seen_all = a.causal ? max(0, min(keys, min(pq.at + kQueries, pq.count) + shift)) : keys;

  const long at = pq.first + min(row, pq.count - 1);
  const T *g_row = (const T *)a.d_o + at * a.H * a.D + head * a.D;
  float minus_delta = -row_product<T, DP>(g_row, (const T *)a.o + at * a.H * a.D + head * a.D, a.D, half);
  const float lse2 = a.lse[(long)head * a.Tq + at] * kLog2e;
  const auto leave_figures = [&] {
    if (part > 0 || wave >= ROWS || half > 0 || row >= pq.count) return;
    rows.lse2[(long)head * a.Tq + at] = lse2;
    rows.minus_delta[(long)head * a.Tq + at] = minus_delta;
  };
  // Rows that see few keys take delta as sum_j p_ij (do_i . v_j) instead, in a pass of its own: o was rounded, and where a few keys have most of p,
  // ds is small beside that error (of a row with one key it is 0).  600 tokens in 24 sequences in bfloat16: dq and dk off by
  // 2.8e-3, with it by 2.4e-3, for 1.2 us of 21.
  const int turns = (seen_all + BN - 1) / BN;
  const bool measures = sizeof(T) == 2 && turns > 0 && seen_all <= 128;
  if (!measures) {
    leave_figures();
    if (!a.dq) return;
  }

  const T *k = (const T *)a.k + (long)kv_first * a.kv_row + kv * a.D, *v = (const T *)a.v + (long)kv_first * a.kv_row + kv * a.D;
  S sk, sv;
  sk.init(smem, k, a.kv_row, a.D);
  sv.init(smem + S::kBytes, v, a.kv_row, a.D);
  RowFrags<T, DP> q, g;
  q.load((const T *)a.q + at * a.q_row + head * a.D, a.D, half);
  g.load(g_row, a.D, half);
  const float c = a.scale * kLog2e;

  const Reader<T, DP, BN> reader(lane);
  // p (dp + from) of the 32 keys from b on in a tile
  const auto ds_of = [&](const char *lk, const char *lv, int key0, int b, float from) {
    floatx16 z = {}, d;
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = from;
    Frag<T> kf[2], vf[2];   // read a step ahead of the products that take them
    kf[0] = reader.along(lk, b, 0);
    vf[0] = reader.along(lv, b, 0);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      if (s + 1 < DP / 16) {
        kf[(s + 1) & 1] = reader.along(lk, b, s + 1);
        vf[(s + 1) & 1] = reader.along(lv, b, s + 1);
      }
      __builtin_amdgcn_sched_barrier(0);
      z = mma(kf[s & 1], q[s], z);
      d = mma(vf[s & 1], g[s], d);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[r], c, -lse2));
    if (key0 + b + 32 > seen_first)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (key0 + b + token_of(r) + 4 * half >= seen) z[r] = 0.0f, d[r] = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] *= z[r];
    return d;
  };
  if constexpr (sizeof(T) == 2)
    if (measures) {
      sk.start(wave, k, 0, keys);
      sv.start(wave, v, 0, keys);
      float delta = 0.0f;
      for (int key0 = 0, odd = 1; key0 < seen_all; key0 += BN, odd ^= 1) {
        landed<T>();
        const char *lk = sk.turn(wave, odd, k, key0 + BN, keys), *lv = sv.turn(wave, odd, v, key0 + BN, keys);
        for (int b = mine; b < mine + kPer && key0 + b < seen_last; b += 32) {
          const floatx16 d = ds_of(lk, lv, key0, b, 0.0f);
#pragma unroll
          for (int r = 0; r < 16; ++r) delta += d[r];
        }
      }
      arrived();
      barrier();   // everyone is done with the tiles
      delta = sum_of_halves(delta);
      if constexpr (ROWS == 2) {   // of both pairs' keys
        float *shared = reinterpret_cast<float *>(smem);
        shared[wave * 64 + lane] = delta;
        __syncthreads();
        delta = shared[wave % 2 * 64 + lane] + shared[(wave % 2 + 2) * 64 + lane];
        __syncthreads();
      }
      minus_delta = -delta;
      leave_figures();
      if (!a.dq) return;
    }
  const int begin = turn_from(part, parts.n, turns) * BN, end = min(seen_all, turn_from(part + 1, parts.n, turns) * BN);
  floatx16 dq[DP / 32];
  bool reached = false;   // by a key that is not finite, in a careful pass
  const auto pass = [&](auto careful) {
    sk.start(wave, k, begin, keys);
    sv.start(wave, v, begin, keys);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) dq[i] = floatx16{};
    int odd = 1;
    for (int key0 = begin; key0 < end; key0 += BN, odd ^= 1) {
      landed<T>();
      const char *lk = sk.turn(wave, odd, k, key0 + BN, keys), *lv = sv.turn(wave, odd, v, key0 + BN, keys);
      written<T>();
      if (decltype(careful)::value && key0 + BN > pq.at + shift + 1) {
        const Cleared c = clear_rows<T, DP, BN>(const_cast<char *>(lk), smem + 2 * S::kBytes);
        reached = reached || (c.first < BN && key0 + c.first < seen);
      }
#pragma unroll 1
      for (int b = mine; b < mine + kPer && key0 + b < seen_last; b += 32) {
        const floatx16 d = ds_of(lk, lv, key0, b, minus_delta);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          const Frag<T> ds = frag_of<T>(d, s);
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) dq[i] = mma(reader.across(lk, b + 16 * s, 32 * i), ds, dq[i]);
        }
      }
    }
    arrived();
  };
  if constexpr (CARE == TAKE) {
    pass(std::true_type{});
  } else {
    pass(std::false_type{});
    if (CARE != NONE && a.causal) {
      const bool again = anyone(!all_finite(dq), smem + 2 * S::kBytes, wave);
      if constexpr (CARE == LEAVE) {
        if (threadIdx.x == 0) rows.again[blockIdx.x] = again;
      } else if (again) {
        pass(std::true_type{});
      }
    }
  }
  if (reached)
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) dq[i] += NAN;
  if constexpr (ROWS == 2) {   // the second pair's sums to the first, in the tiles' place
    constexpr int kLeft = DP * 128;
    static_assert(2 * kLeft <= 2 * S::kBytes, "");
    barrier();
    if (wave >= ROWS)
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<floatx4 *>(smem + (wave - ROWS) * kLeft + ((i * 4 + r) * 64 + lane) * 16) =
              floatx4{dq[i][4 * r], dq[i][4 * r + 1], dq[i][4 * r + 2], dq[i][4 * r + 3]};
    __syncthreads();
    if (wave >= ROWS) return;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const floatx4 v = *reinterpret_cast<const floatx4 *>(smem + wave * kLeft + ((i * 4 + r) * 64 + lane) * 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) dq[i][4 * r + j] += v[j];
      }
  }
  if (row >= pq.count) return;
  if (parts.n > 1) return store_sums(parts.sums[0] + (((long)part * a.Tq + at) * a.H + head) * parts.ld, dq, parts.ld, half);
  store_row<T>((T *)a.dq + at * a.q_row + head * a.D, dq, a.scale, a.D, half);
}

// ------------------------------------------------------------------------------------------------ dk, dv
// The kernel's forms.  BOTH: both gradients.  HELD_LESS: both, the values' rows in LDS instead of registers, so that two workgroups fit a compute unit.
// KEYS, VALUES: one of the two gradients (single precision with more than 128 elements a head takes them one after the other, as their
// sums and both rows would not fit the registers).
enum Form { BOTH, HELD_LESS, KEYS, VALUES };
template <class T, int DP, Form F>
struct DkvShape {
  static constexpr bool kDK = F != VALUES, kDV = F != KEYS, kInLds = F == HELD_LESS;
  static constexpr int kQueries = kInLds ? 32 : tile_rows<T, DP>();   // of a tile
  static constexpr int kFigures = 256;                                // bytes of one kind of figures of a tile
  typedef Stager<T, DP, kQueries, kThreads> Rows;
  typedef Stager<T, DP, kRows, kThreads> Values;
  static constexpr int kTiles = 2 * Rows::kBytes + 4 * kFigures + (kInLds ? Values::kTile : 0), kLds = kTiles + kCareful;
  static constexpr int kResident = kInLds || (sizeof(T) == 2 ? DP <= 64 : DP <= 32) ? 2 : 1;
};

template <class T, int DP, Form F, Careful CARE>
__global__ __launch_bounds__(kThreads, (DkvShape<T, DP, F>::kResident)) void attention_dkv_kernel(const AttentionArgs a, const Rows rows, const Parts parts, int) {
  typedef DkvShape<T, DP, F> Sh;
  typedef typename Sh::Rows S;
  constexpr bool DK = Sh::kDK, DV = Sh::kDV;
  constexpr int BN = Sh::kQueries, kFigures = Sh::kFigures;
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
  const int part = blockIdx.x % parts.n, id = blockIdx.x / parts.n, kv = id % a.KV, tile = id / a.KV, group = a.H / a.KV;
  const Place pk = place_of(a.kv_starts, a.S, a.Tk, tile, kRows);
  if (pk.at >= pk.count || (CARE == TAKE && !rows.again[blockIdx.x])) return;
  const int q_first = start_of(a.q_starts, pk.sequence, a.Tq), queries = max(0, start_of(a.q_starts, pk.sequence + 1, a.Tq) - q_first);
  const int key0 = pk.at + 32 * wave, key = key0 + (lane & 31), shift = pk.count - queries;
  const int from = a.causal ? max(0, pk.at - shift) : 0;         // the first query that sees any of the workgroup's keys
  const int sees = key - shift;                                  // the first that sees this lane's key, where causal
  const int sees_first = key0 - shift, sees_all = key0 + 31 - shift;

  const long at = pk.first + min(key, pk.count - 1);
  RowFrags<T, DP> k, v;
  k.load((const T *)a.k + at * a.kv_row + kv * a.D, a.D, half);
  char *const values = smem + 2 * S::kBytes + 4 * kFigures;
  if constexpr (Sh::kInLds) {   // landed, as the first tile is
    typename Sh::Values sv;
    const T *p = (const T *)a.v + (long)pk.first * a.kv_row + kv * a.D;
    sv.init(values, p, a.kv_row, a.D);
    sv.start(wave, p, pk.at, pk.count);
  } else if (DK) {
    v.load((const T *)a.v + at * a.kv_row + kv * a.D, a.D, half);
  }
  const Reader<T, DP, kRows> values_reader(lane);
  const auto value = [&](int s) {
    if constexpr (Sh::kInLds) return values_reader.along(values, 32 * wave, s);
    else return v[s];
  };
  const float c = a.scale * kLog2e;
  floatx16 dk[DK ? DP / 32 : 1], dv[DV ? DP / 32 : 1];
  const Reader<T, DP, BN> reader(lane);
  S sq, sg;
  sq.init(smem, a.q, a.q_row, a.D);
  sg.init(smem + S::kBytes, a.d_o, (long)a.H * a.D, a.D);
  char *const figures = smem + 2 * S::kBytes;   // lse2 and minus_delta of a tile; twice
  // turns: the group's heads, each over the tiles of queries
  const int tiles = queries > from ? (queries - from + BN - 1) / BN : 0, turns = tiles * group;
  const int begin = turn_from(part, parts.n, turns), end = turn_from(part + 1, parts.n, turns);
  struct Turn { const T *q, *g; const float *figures; int i0; };
  const auto turn_of = [&](int turn) {   // behind the last one: no queries
    const int h = kv * group + min(turn / max(tiles, 1), group - 1), i0 = turn < end ? from + (turn % max(tiles, 1)) * BN : queries;
    return Turn{(const T *)a.q + (long)q_first * a.q_row + h * a.D, (const T *)a.d_o + ((long)q_first * a.H + h) * a.D,
                (wave & 1 ? rows.minus_delta : rows.lse2) + (long)h * a.Tq + q_first + i0, i0};
  };
  // two wavefronts bring the one kind of figures, two the other: as many loads on their way in each.  Like the rows, they go straight
  // into LDS or come through a register.
  float held = 0.0f;
  const auto load_figures = [&](const Turn &t, int odd) {
    if constexpr (sizeof(T) == 4) {
      held = lane < min(queries - t.i0, BN) ? t.figures[lane] : 0.0f;
      return;
    }
    const uintx4 rs = buffer_of((const char *)t.figures, (unsigned)max(0, min(queries - t.i0, BN)) * 4u);
    load_words_to_lds(rs, lane * 4, (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)(figures + (2 * odd + (wave & 1)) * kFigures));
  };
  bool reached = false;   // by a query, or its outputs' gradients, that is not finite, in a careful pass
  const auto pass = [&](auto careful) {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
      if (DK) dk[i] = floatx16{};
      if (DV) dv[i] = floatx16{};
    }
    if (begin < end) {
      const Turn t = turn_of(begin);
      sq.start(wave, t.q, t.i0, queries);
      sg.start(wave, t.g, t.i0, queries);
      load_figures(t, 0);
    }
    int odd = 1;
    for (int turn = begin; turn < end; ++turn, odd ^= 1) {
      const Turn next = turn_of(turn + 1);
      landed<T>();
      const char *lq = sq.turn(wave, odd, next.q, next.i0, queries), *lg = sg.turn(wave, odd, next.g, next.i0, queries);
      if constexpr (sizeof(T) == 4) reinterpret_cast<float *>(figures)[(2 * (odd ^ 1) + (wave & 1)) * (kFigures / 4) + lane] = held;
      load_figures(next, odd);
      written<T>();
      const float *lse2 = reinterpret_cast<const float *>(figures + 2 * (odd ^ 1) * kFigures), *minus_delta = lse2 + kFigures / 4;
      const int i0 = from + (turn % tiles) * BN;
      if (decltype(careful)::value && i0 < pk.at + kRows - 1 - shift) {   // a query that does not see all of the workgroup's keys
        const Cleared of_q = clear_rows<T, DP, BN>(const_cast<char *>(lq), smem + Sh::kTiles), of_g = clear_rows<T, DP, BN>(const_cast<char *>(lg), smem + Sh::kTiles);
        const int last = max(of_q.last, of_g.last);
        reached = reached || (last >= 0 && i0 + last >= sees);
      }
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
        Frag<T> qf[2], gf[2];
        qf[0] = reader.along(lq, b, 0);
        if constexpr (DK) gf[0] = reader.along(lg, b, 0);
#pragma unroll
        for (int s = 0; s < DP / 16; ++s) {
          if (s + 1 < DP / 16) {
            qf[(s + 1) & 1] = reader.along(lq, b, s + 1);
            if constexpr (DK) gf[(s + 1) & 1] = reader.along(lg, b, s + 1);
          }
          __builtin_amdgcn_sched_barrier(0);
          z = mma(qf[s & 1], k[s], z);
          if constexpr (DK) d = mma(gf[s & 1], value(s), d);
          __builtin_amdgcn_sched_barrier(0);
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
    }
    arrived();
  };
  if constexpr (CARE == TAKE) {
    pass(std::true_type{});
  } else {
    pass(std::false_type{});
    if constexpr (CARE != NONE) {
      bool finite = true;
      if (DK) finite = all_finite(dk);
      if (DV) finite = finite && all_finite(dv);
      const bool again = anyone(!finite, smem + Sh::kTiles, wave);
      if constexpr (CARE == LEAVE) {
        if (threadIdx.x == 0) rows.again[blockIdx.x] = again;
      } else if (again) {
        pass(std::true_type{});
      }
    }
  }
  if (reached)
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) {
      if (DK) dk[i] += NAN;
      if (DV) dv[i] += NAN;
    }
  if (key >= pk.count) return;
  if (parts.n > 1) {
    const long to = (((long)part * a.Tk + at) * a.KV + kv) * parts.ld;
    if (DK && a.dk) store_sums(parts.sums[0] + to, dk, parts.ld, half);
    if (DV && a.dv) store_sums(parts.sums[1] + to, dv, parts.ld, half);
    return;
  }
  if (DK && a.dk) store_row<T>((T *)a.dk + at * a.kv_row + kv * a.D, dk, a.scale, a.D, half);
  if (DV && a.dv) store_row<T>((T *)a.dv + at * a.kv_row + kv * a.D, dv, 1.0f, a.D, half);
}

// ------------------------------------------------------------------------------------------------ parts
// One or two gradients' rows from their parts, four elements a thread
struct Sums {
  Parts parts;
  const int *starts;
  int sequences, tokens, heads, dim;
  long row;
  void *out[2];
  float factor[2];
};
template <class T>
__global__ __launch_bounds__(kThreads) void attention_sums_kernel(const Sums s, const long units) {
  const int wide = s.parts.ld / 4, first = start_of(s.starts, 0, s.tokens), end = start_of(s.starts, s.sequences, s.tokens);
  const long part = (long)s.tokens * s.heads * s.parts.ld;
  for (long u = (long)blockIdx.x * kThreads + threadIdx.x; u < units; u += (long)gridDim.x * kThreads) {
    const int d = (int)(u % wide) * 4;
    const long row = u / wide, head = row % s.heads, at = row / s.heads;
    if (at < first || at >= end) continue;   // nobody's
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (!s.out[k]) continue;
      floatx4 v = {};
#pragma unroll 4
      for (int p = 0; p < s.parts.n; ++p) v += *reinterpret_cast<const floatx4 *>(s.parts.sums[k] + p * part + row * s.parts.ld + d);
      T *to = (T *)s.out[k] + at * s.row + head * s.dim + d;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (d + j < s.dim) to[j] = (T)(v[j] * s.factor[k]);
    }
  }
}
template <class T>
hipError_t launch_sums(const Sums &s, hipStream_t stream) {
  const long units = (long)s.tokens * s.heads * (s.parts.ld / 4), blocks = (units + kThreads - 1) / kThreads;
  attention_sums_kernel<T><<<dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kThreads), 0, stream>>>(s, units);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------------ host
// The workspace's parts, the same walk for the query and the call
struct BwdPlan {
  int rows = 4;          // groups of 32 queries of a workgroup that takes dq
  bool less = false;     // HELD_LESS
  Rows figures;
  Parts dq, dkv;
  size_t bytes;
};
template <class T, int DP>
BwdPlan plan(const AttentionArgs &a, char *base) {
  constexpr int BN = tile_rows<T, DP>();
  constexpr bool kTwo = sizeof(T) == 2 && BN == 64, kLess = sizeof(T) == 2 && DP > 64 && DP <= 128;
  const long cus = chip().cus, all_q = (a.Tq + kRows - 1) / kRows, all_k = (a.Tk + kRows - 1) / kRows;
  const long q_work = (all_q > a.S ? all_q : a.S) * a.H, k_work = (all_k > a.S ? all_k : a.S) * a.KV;
  BwdPlan p;
  Take take{base};
  p.figures.lse2 = (float *)take((size_t)a.H * a.Tq * sizeof(float));
  p.figures.minus_delta = (float *)take((size_t)a.H * a.Tq * sizeof(float));
  const auto dq_parts = [&](int rows) {
    const int queries = 32 * rows;
    return parts_of((a.Tq + queries - 1) / queries * (long)a.H, tiles_of(a.Tq, a.S, queries) * a.H, dq_residents<T, DP>() * cus, a.Tk / a.S / BN, 2);
  };
  const auto dkv_parts = [&](int resident) {
    return parts_of(all_k * a.KV, tiles_of(a.Tk, a.S, kRows) * a.KV, resident * cus, (long)a.Tq / a.S * (a.H / a.KV) / BN, 2);
  };
  // Both rules below come from 207 causal and open calls taken either way: 500 to 20480 tokens in one to forty sequences, 4 to 128 heads, groups of 1, 2, 4 and 8.  They
  // lose 0.4 and 0.3 % to the better way on average and 11 and 8 % at most.
  // Sequences so long that, under a causal mask, their first keys' and last queries' workgroups last: 1365 and 1536 tokens 9 and 4 % faster the other way, 2000 and 2048
  // 8 and 4 % slower (dk and dv).
  const bool chain = a.causal && a.Tk / a.S >= 1792;
  // 64 queries a workgroup where 128 have their keys cut into parts, whose sums cost a pass; where they leave most of the chip idle; and where a causal
  // mask's longest workgroups decide, as all of them run at once (heads up to 64: nearly so).  Microseconds of a backward pass with 128 / 64, causal: 40 heads of 128, 1024 tokens
  // 111 / 85; 16, 3328 tokens 233 / 207, 4096 in one 291 / 282, in two 182 / 168, in four 126 / 128, 4480 348 / 347, 4992 422 / 430; 16 of 64, 4096 188 / 172, 5120 244 / 229, 6400
  // 324 / 323, 8192 522 / 521, 4096 in twenty 46 / 48; all keys seen, 16 of 64, 2560 161 / 143, 4096 256 / 270.
  p.dq.n = dq_parts(4);
  if (kTwo && (p.dq.n > 1 || 2 * q_work <= cus || (chain && q_work <= (DP <= 64 ? 3 : 2) * cus))) {
    p.rows = 2;
    p.dq.n = dq_parts(2);
  }
  // values in LDS, so that a unit has two workgroups: where there are two for it, but for causal calls with so few that all run at once and nothing evens out their long
  // and short ones; and where that takes more parts than values in registers do, only if the parts are long enough for their sums.  Values in registers / in LDS: 16 heads
  // of 128, causal, 3328 tokens 233 / 245, 3968 296 / 315, 4096 291 / 327, 4480 348 / 367, 5120 438 / 439, 5632 509 / 493, 8192 991 / 927; in two 537 / 488; 8 heads, 3500 tokens 165 / 167,
  // 4500 249 / 232, 8192 540 / 620, 10000 792 / 811; 16 on 4, 2048 141 / 133, 4096 406 / 348, 16384 3911 / 5065; 32 on 8, 9216 2526 / 2825, 10240 3172 / 3340; 3000 in thirty, 16 heads, 67 / 60;
  // all keys seen, 16 heads, 2048 160 / 166, 2560 315 / 285, 4096 507 / 449
  const int apart = dkv_parts(DkvShape<T, DP, BOTH>::kResident), beside = kLess ? dkv_parts(DkvShape<T, DP, kLess ? HELD_LESS : BOTH>::kResident) : apart;
  const bool at_once = chain && k_work >= 2 * cus && 2 * k_work < 5 * cus;
  const long part_work = (long)a.Tq / a.S * (a.H / a.KV) * (a.causal ? 1 : 2);
  p.less = kLess && !at_once && (beside == apart ? k_work * beside > cus : part_work >= 4096);
  p.dkv.n = p.less ? beside : apart;
  p.dq.ld = p.dkv.ld = (a.D + 3) & ~3;
  if (p.dq.n > 1) p.dq.sums[0] = (float *)take((size_t)p.dq.n * a.Tq * a.H * p.dq.ld * sizeof(float));
  if (p.dkv.n > 1)
    for (float *&s : p.dkv.sums) s = (float *)take((size_t)p.dkv.n * a.Tk * a.KV * p.dkv.ld * sizeof(float));
  const int queries = 32 * p.rows;
  if (a.causal && dkv_apart<T, DP>()) {   // of one launch at a time
    const long q_grid = tiles_of(a.Tq, a.S, queries) * a.H * p.dq.n, k_grid = tiles_of(a.Tk, a.S, kRows) * a.KV * p.dkv.n;
    p.figures.again = (unsigned *)take((size_t)(q_grid > k_grid ? q_grid : k_grid) * sizeof(unsigned));
  }
  p.bytes = take.used;
  return p;
}

template <class K>
hipError_t launch(K kernel, long grid, size_t lds, const AttentionArgs &a, const BwdPlan &p, const Parts &parts, int tiles, hipStream_t stream) {
  DLL_TRY(allow_large_lds(reinterpret_cast<const void *>(kernel), lds));
  kernel<<<dim3((unsigned)grid), dim3(kThreads), lds, stream>>>(a, p.figures, parts, tiles);
  return hipGetLastError();
}

template <class T, int DP, int ROWS>
hipError_t launch_dq(const AttentionArgs &a, const BwdPlan &p, hipStream_t stream) {
  constexpr int BN = tile_rows<T, DP>();
  constexpr size_t lds = 2 * Stager<T, DP, BN, kThreads>::kBytes + kCareful;
  const long tiles = tiles_of(a.Tq, a.S, 32 * ROWS);
  const Parts one, &dq = a.dq ? p.dq : one;
  const auto run = [&](auto kernel) { return launch(kernel, tiles * a.H * dq.n, lds, a, p, dq, (int)tiles, stream); };
  if constexpr (dq_apart<T, DP>()) {
    DLL_TRY(run(a.causal ? attention_dq_kernel<T, DP, BN, ROWS, LEAVE> : attention_dq_kernel<T, DP, BN, ROWS, NONE>));
    if (a.causal && a.dq) DLL_TRY(run(attention_dq_kernel<T, DP, BN, ROWS, TAKE>));
  } else {
    DLL_TRY(run(attention_dq_kernel<T, DP, BN, ROWS, HERE>));   // without a mask the copy costs less than 1 % (instances without it: 14 calls in 0.993 to 1.007 of the time)
  }
  return dq.n > 1 ? launch_sums<T>(Sums{dq, a.q_starts, a.S, a.Tq, a.H, a.D, a.q_row, {a.dq, nullptr}, {a.scale, 0.0f}}, stream) : hipSuccess;
}

template <class T, int DP, Form F>
hipError_t launch_dkv(const AttentionArgs &a, const BwdPlan &p, hipStream_t stream) {
  const auto run = [&](auto kernel) { return launch(kernel, tiles_of(a.Tk, a.S, kRows) * a.KV * p.dkv.n, DkvShape<T, DP, F>::kLds, a, p, p.dkv, 0, stream); };
  if (!a.causal) return run(attention_dkv_kernel<T, DP, F, NONE>);
  if constexpr (dkv_apart<T, DP>()) {
    DLL_TRY(run(attention_dkv_kernel<T, DP, F, LEAVE>));
    return run(attention_dkv_kernel<T, DP, F, TAKE>);
  } else {
    return run(attention_dkv_kernel<T, DP, F, HERE>);
  }
}

template <class T, int DP>
hipError_t bwd_as(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  const BwdPlan p = plan<T, DP>(a, scratch);
  if constexpr (sizeof(T) == 2 && tile_rows<T, DP>() == 64)
    DLL_TRY((p.rows == 2 ? launch_dq<T, DP, 2>(a, p, stream) : launch_dq<T, DP, 4>(a, p, stream)));
  else
    DLL_TRY((launch_dq<T, DP, 4>(a, p, stream)));
  if (!a.dk && !a.dv) return hipSuccess;
  if constexpr (sizeof(T) == 4 && DP > 128) {
    if (a.dv) DLL_TRY((launch_dkv<T, DP, VALUES>(a, p, stream)));
    if (a.dk) DLL_TRY((launch_dkv<T, DP, KEYS>(a, p, stream)));
  } else if constexpr (sizeof(T) == 2 && DP > 64 && DP <= 128) {
    DLL_TRY((p.less ? launch_dkv<T, DP, HELD_LESS>(a, p, stream) : launch_dkv<T, DP, BOTH>(a, p, stream)));
  } else {
    DLL_TRY((launch_dkv<T, DP, BOTH>(a, p, stream)));
  }
  if (p.dkv.n == 1) return hipSuccess;
  return launch_sums<T>(Sums{p.dkv, a.kv_starts, a.S, a.Tk, a.KV, a.D, a.kv_row, {a.dk, a.dv}, {a.scale, 1.0f}}, stream);
}

template <class T>
hipError_t bwd(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  return instance(a.D, [&](auto dp) { return bwd_as<T, decltype(dp)::value>(a, scratch, stream); });
}
template <class T>
size_t bwd_bytes(const AttentionArgs &a) {
  return instance(a.D, [&](auto dp) { return plan<T, decltype(dp)::value>(a, nullptr).bytes; });
}

}  // namespace

size_t attention_bwd_scratch(const AttentionArgs &a) { return a.dtype == TYPE_BF16 ? bwd_bytes<bf16>(a) : bwd_bytes<float>(a); }

hipError_t launch_attention_bwd(const AttentionArgs &a, char *scratch, hipStream_t stream) {
  return a.dtype == TYPE_BF16 ? bwd<bf16>(a, scratch, stream) : bwd<float>(a, scratch, stream);
}

}  // namespace dllk
