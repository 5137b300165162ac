// A paged cache of keys and values: pages and slots for new tokens from the requests' lengths, and the store of their rows.
//
// Plan.  A request with `length` tokens, `added` of them new, has pages for the others and takes one from the free list for each of its
// new tokens that stands first in a page; the requests take theirs in turn.  One launch: a workgroup has 1024 neighbouring new
// tokens, four a thread.  It sums up added tokens and taken pages over all requests, notes at each of its own tokens that is a
// request's first one that request's figures, and the last note before a token is its request (a running maximum).  So nothing goes from
// one workgroup to another and a few bytes a request are read again by each.
//
// Store.  Rows go from [token][head] to [page][head][place in page], so that a head's keys of a page lie together for the
// attention that streams them; both sides move 16 bytes or more a lane.
//
// The plan is bound by latency: 64 requests with a new token each 4.3 us on the GPU, 2000 prompts with 272 000 tokens 7.3 (as much for an empty
// kernel: 2.7).  The store is bound by memory: 15 000 tokens of 8 heads of 128 in single precision, 236 MB, 41 us = 5.8 TB/s.
#include "large_ops.h"
#include "tile_product.h"

namespace dllk {

using namespace tile;

namespace {

constexpr int kPlanThreads = 256, kEach = 4, kTokens = kPlanThreads * kEach;   // of a workgroup
constexpr int kRequests = 8;
constexpr int kMost = 1 << 30;   // sums stop there, above any token that has a slot

// of two up to kMost, whose sum may pass 31 bits
__device__ __forceinline__ int add(int a, int b) { return (int)min((unsigned)a + (unsigned)b, (unsigned)kMost); }

// What a request asks for: its figures with lengths below 0 taken as 0 and no more new tokens than there are tokens
struct Asked {
  int before, added, have, fresh;   // tokens and pages before the step, new tokens, new pages
  int missing;                      // pages that the table has no column for
  __device__ __forceinline__ Asked(const Divisor &page, int columns, int length, int new_tokens) {
    length = max(0, length);
    added = max(0, min(new_tokens, length));
    before = length - added;
    have = before ? page.of(before - 1) + 1 : 0;
    const int need = length ? page.of(length - 1) + 1 : 0;
    fresh = max(0, min(need, columns) - have);
    missing = need - have - fresh;
  }
};

__global__ __launch_bounds__(kPlanThreads) void cache_plan_kernel(const CacheArgs a, const Divisor by) {
  struct Note { int request, first, before, have, page; };
  __shared__ Note note[kTokens];
  __shared__ int sums[3][kPlanThreads / 64], tops[kPlanThreads / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int lo = (int)blockIdx.x * kTokens;
  const int at = a.free_at ? max(0, min(*a.free_at, a.n_free)) : 0;
  // sums over this thread's requests, then over the threads before it
  const int each = (a.R + kPlanThreads - 1) / kPlanThreads, r0 = min(t * each, a.R), r1 = min(r0 + each, a.R);
  // eight requests at a time, all on their way before the first is looked at; none behind the last asks for anything
  int length[kRequests], new_tokens[kRequests];
  const auto load = [&](int r) {
    typedef int Run __attribute__((ext_vector_type(kRequests)));
    typedef Run Any __attribute__((aligned(4)));
    if (r + kRequests <= r1) {
      const Run x = *reinterpret_cast<const Any *>(a.lengths + r), y = *reinterpret_cast<const Any *>(a.added + r);
#pragma unroll
      for (int k = 0; k < kRequests; ++k) length[k] = x[k], new_tokens[k] = y[k];
      return;
    }
#pragma unroll
    for (int k = 0; k < kRequests; ++k) {
      length[k] = r + k < r1 ? a.lengths[r + k] : 0;
      new_tokens[k] = r + k < r1 ? a.added[r + k] : 0;
    }
  };
  int added = 0, fresh = 0, missing = 0;
  for (int r = r0; r < r1; r += kRequests) {
    load(r);
#pragma unroll
    for (int k = 0; k < kRequests; ++k) {
      const Asked q(by, a.columns, length[k], new_tokens[k]);
      added = add(added, min(q.added, kMost));
      fresh = add(fresh, min(q.fresh, kMost));
      missing = add(missing, min(q.missing, kMost));
    }
  }
  int added_up = added, fresh_up = fresh;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int x = __shfl_up(added_up, d), y = __shfl_up(fresh_up, d);
    missing = add(missing, __shfl_xor(missing, d));
    if (lane >= d) added_up = add(added_up, x), fresh_up = add(fresh_up, y);
  }
#pragma unroll
  for (int k = 0; k < kEach; ++k) note[t * kEach + k].request = -1;
  if (lane == 63) sums[0][wave] = added_up, sums[1][wave] = fresh_up, sums[2][wave] = missing;
  // of the lanes before this one: the sum of one lane less (its own cannot be taken off a sum that has stopped)
  int start = __shfl_up(added_up, 1), page = __shfl_up(fresh_up, 1);
  if (lane == 0) start = page = 0;
  __syncthreads();
  int all_added = 0, all_fresh = 0, all_missing = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) start = add(start, sums[0][w]), page = add(page, sums[1][w]);
    all_added = add(all_added, sums[0][w]);
    all_fresh = add(all_fresh, sums[1][w]);
    all_missing = add(all_missing, sums[2][w]);
  }
  for (int r = r0; r < r1; r += kRequests) {
    if (each > kRequests) load(r);   // otherwise they are still there
#pragma unroll
    for (int k = 0; k < kRequests; ++k) {
      if (r + k >= r1) continue;
      const Asked q(by, a.columns, length[k], new_tokens[k]);
      if (blockIdx.x == 0) a.starts[r + k] = start;
      const int end = add(start, min(q.added, kMost));
      if (start < lo + kTokens && end > max(start, lo))   // at its first token here
        note[max(start - lo, 0)] = Note{r + k, start - lo, q.before, q.have, page - q.have};
      start = end;
      page = add(page, min(q.fresh, kMost));
    }
  }
  if (blockIdx.x == 0 && t == 0) {
    a.starts[a.R] = all_added;
    const int taken = min(all_fresh, a.n_free - at);
    a.state[0] = at + taken;
    a.state[1] = add(all_fresh - taken, all_missing);
  }
  __syncthreads();
  // each token's request: the last note up to it
  int top = -1;
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    if (note[t * kEach + k].request >= 0) top = t * kEach + k;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(top, d);
    if (lane >= d) top = max(top, o);
  }
  if (lane == 63) tops[wave] = top;
  top = __shfl_up(top, 1);
  if (lane == 0) top = -1;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w)
    if (w < wave) top = max(top, tops[w]);
  // where each token's page stands, all loads before the first store: in the table, or where it is new in the free list; -1 where nowhere
  const int count = min(min(a.tokens, all_added) - lo - t * kEach, kEach);   // of this thread's tokens that there are
  int id[kEach], place[kEach];
  int *entry[kEach];   // that is to be written
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    const int i = t * kEach + k;
    if (note[i].request >= 0) top = i;
    const Note n = note[max(top, 0)];
    const int p = n.before + (i - n.first);   // the token's place in its request
    const int column = by.of(p);
    place[k] = p - column * a.page;
    const bool there = k < count && column < a.columns, fresh_page = column >= n.have;
    int *const at_table = a.table + (long)n.request * a.columns + column;
    const long at_free = (long)at + n.page + column;
    const bool some = there && (!fresh_page || at_free < a.n_free);
    const int *const from = !some ? a.lengths : fresh_page ? a.free_pages + at_free : at_table;
    id[k] = *from;
    if (!some) id[k] = -1;
    entry[k] = there && fresh_page && place[k] == 0 ? at_table : nullptr;
  }
  int *to = a.slots + lo + t * kEach;
#pragma unroll
  for (int k = 0; k < kEach; ++k) {
    if (entry[k]) *entry[k] = id[k];
    if (k < count) to[k] = id[k] >= 0 && id[k] < a.pages ? id[k] * a.page + place[k] : -1;
  }
}

// units: runs of eight elements of a head's row
template <class T>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArgs a, const Divisor by, const int runs, const unsigned units) {
  const unsigned per = (unsigned)a.KV * runs;
  for (unsigned u = blockIdx.x * 256 + threadIdx.x; u < units; u += gridDim.x * 256) {
    const unsigned token = u / per, rest = u - token * per, head = rest / runs, d = (rest - head * runs) * 8;
    const int slot = a.slots[token], n = a.D - (int)d;
    if (slot < 0 || slot >= a.pages * a.page) continue;
    Eight<T> k, v;
    const long from = (long)token * a.row + head * a.D + d;
    k.load((const T *)a.k + from, n);
    v.load((const T *)a.v + from, n);
    const int id = by.of(slot), place = slot - id * a.page;
    const long to = (((long)id * a.KV + head) * a.page + place) * a.D + d;
    k.store((T *)a.k_cache + to, n);
    v.store((T *)a.v_cache + to, n);
  }
}

}  // namespace

hipError_t launch_cache_plan(const CacheArgs &a, hipStream_t stream) {
  cache_plan_kernel<<<dim3((unsigned)((a.tokens + kTokens - 1) / kTokens)), dim3(kPlanThreads), 0, stream>>>(a, Divisor(a.page));
  return hipGetLastError();
}

hipError_t launch_cache_write(const CacheArgs &a, hipStream_t stream) {
  const int runs = (a.D + 7) / 8;
  const long units = (long)a.tokens * a.KV * runs, blocks = (units + 255) / 256, most = 16L * chip().cus;
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  if (a.dtype == TYPE_BF16) cache_write_kernel<bf16><<<grid, dim3(256), 0, stream>>>(a, Divisor(a.page), runs, (unsigned)units);
  else cache_write_kernel<float><<<grid, dim3(256), 0, stream>>>(a, Divisor(a.page), runs, (unsigned)units);
  return hipGetLastError();
}

}  // namespace dllk
