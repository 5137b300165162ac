// A paged cache of keys and values: pages and slots for new tokens from the requests' lengths, and the store of their rows.
//
// Plan.  A request with `length` tokens, `added` of them new, has pages for the others and takes one from the free list for each of its
// new tokens that stands first in a page; the requests take theirs in turn.  One launch: a workgroup has 1024 neighbouring new
// tokens, one a thread.  It sums up added tokens and taken pages over all requests, notes at each of its own tokens that is a
// request's first one that request's figures, and the last note before a token is its request (a running maximum).  So nothing goes from
// one workgroup to another and a few bytes a request are read again by each.
//
// Store.  Rows go from [token][head] to [page][head][place in page], so that a head's keys of a page lie together for the
// attention that streams them; both sides move 16 bytes or more a lane.
#include "large_ops.h"
#include "tile_product.h"

namespace dllk {

using namespace tile;

namespace {

constexpr int kPlanThreads = 1024;

struct Sums {
  long added, fresh, missing;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) { return Sums{a.added + b.added, a.fresh + b.fresh, a.missing + b.missing}; }

// What a request asks for: its figures with lengths below 0 taken as 0 and no more new tokens than there are tokens
struct Asked {
  int before, added, have, fresh;   // tokens and pages before the step, new tokens, new pages
  int missing;                      // pages that the table has no column for
  __device__ __forceinline__ Asked(const CacheArgs &a, int r) {
    const int length = max(0, a.lengths[r]);
    added = max(0, min(a.added[r], length));
    before = length - added;
    const unsigned page = a.page;
    have = (int)((before + page - 1) / page);
    const int need = (int)((length + page - 1) / page);
    fresh = max(0, min(need, a.columns) - have);
    missing = need - have - fresh;
  }
};

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const CacheArgs a) {
  struct Note { int request, first, before, have; long page; };
  __shared__ Note note[kPlanThreads];
  __shared__ Sums wave_sum[kPlanThreads / 64];
  __shared__ int wave_top[kPlanThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const long lo = (long)blockIdx.x * kPlanThreads;
  // sums over this thread's requests, then over the threads before it
  const int each = (a.R + kPlanThreads - 1) / kPlanThreads, r0 = min(t * each, a.R), r1 = min(r0 + each, a.R);
  Sums mine{0, 0, 0};
  for (int r = r0; r < r1; ++r) {
    const Asked q(a, r);
    mine = mine + Sums{q.added, q.fresh, q.missing};
  }
  Sums up = mine;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const Sums o{__shfl_up(up.added, d), __shfl_up(up.fresh, d), __shfl_up(up.missing, d)};
    if (lane >= d) up = up + o;
  }
  note[t].request = -1;
  if (lane == 63) wave_sum[wave] = up;
  __syncthreads();
  Sums base{0, 0, 0}, all{0, 0, 0};
#pragma unroll 4
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) base = base + wave_sum[w];
    all = all + wave_sum[w];
  }
  long start = base.added + up.added - mine.added, page = base.fresh + up.fresh - mine.fresh;
  const int at = a.free_at ? max(0, min(*a.free_at, a.n_free)) : 0;
  for (int r = r0; r < r1; ++r) {
    const Asked q(a, r);
    if (blockIdx.x == 0) a.starts[r] = (int)min(start, 0x7FFFFFFFL);
    if (q.added > 0 && start < lo + kPlanThreads && start + q.added > lo)   // at its first token here
      note[max(start - lo, 0L)] = Note{r, (int)(start - lo), q.before, q.have, page - q.have};
    start += q.added;
    page += q.fresh;
  }
  if (blockIdx.x == 0 && t == 0) {
    a.starts[a.R] = (int)min(all.added, 0x7FFFFFFFL);
    const long taken = min(all.fresh, (long)(a.n_free - at));
    a.state[0] = at + (int)taken;
    a.state[1] = (int)min(all.fresh - taken + all.missing, 0x7FFFFFFFL);
  }
  __syncthreads();
  int top = note[t].request >= 0 ? t : -1;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(top, d);
    if (lane >= d) top = max(top, o);
  }
  if (lane == 63) wave_top[wave] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w)
    if (w < wave) top = max(top, wave_top[w]);
  const long token = lo + t;
  if (token >= a.tokens || token >= all.added || top < 0) return;
  const Note n = note[top];
  const int p = n.before + (t - n.first);   // the token's place in its request
  const int column = p / a.page, place = p - column * a.page;
  int id = -1;
  if (column < a.columns) {
    int *entry = a.table + (long)n.request * a.columns + column;
    if (column >= n.have) {
      const long i = at + n.page + column;
      id = i < a.n_free ? a.free_pages[i] : -1;
      if (place == 0) *entry = id;
    } else {
      id = *entry;
    }
  }
  a.slots[token] = id >= 0 && id < a.pages ? id * a.page + place : -1;
}

// units: runs of eight elements of a head's row
template <class T>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArgs a, const int runs, const unsigned units) {
  const unsigned per = (unsigned)a.KV * runs;
  for (unsigned u = blockIdx.x * 256 + threadIdx.x; u < units; u += gridDim.x * 256) {
    const unsigned token = u / per, rest = u - token * per, head = rest / runs, d = (rest - head * runs) * 8;
    const int slot = a.slots[token], n = a.D - (int)d;
    if (slot < 0 || slot >= a.pages * a.page) continue;
    Eight<T> k, v;
    const long from = (long)token * a.row + head * a.D + d;
    k.load((const T *)a.k + from, n);
    v.load((const T *)a.v + from, n);
    const int id = slot / a.page, place = slot - id * a.page;
    const long to = (((long)id * a.KV + head) * a.page + place) * a.D + d;
    k.store((T *)a.k_cache + to, n);
    v.store((T *)a.v_cache + to, n);
  }
}

}  // namespace

hipError_t launch_cache_plan(const CacheArgs &a, hipStream_t stream) {
  cache_plan_kernel<<<dim3((unsigned)((a.tokens + kPlanThreads - 1) / kPlanThreads)), dim3(kPlanThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheArgs &a, hipStream_t stream) {
  const int runs = (a.D + 7) / 8;
  const long units = (long)a.tokens * a.KV * runs, blocks = (units + 255) / 256, most = 16L * chip().cus;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  if (a.dtype == TYPE_BF16) cache_write_kernel<bf16><<<grid, dim3(256), 0, stream>>>(a, runs, (unsigned)units);
  else cache_write_kernel<float><<<grid, dim3(256), 0, stream>>>(a, runs, (unsigned)units);
  return hipGetLastError();
}

}  // namespace dllk
