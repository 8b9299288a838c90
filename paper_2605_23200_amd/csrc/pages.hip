// Pages of a pool from sequence lengths (ams_assign_pages): block tables, slots of new tokens, the ring of free pages; one launch.
//
// With had = ceil(from / 16), want = ceil(to / 16): a sequence asks for max(want - had, 0) pages and gives back max(had - want, 0).
// Where its pages begin in the ring, and where its tokens begin among those of the call, are sums over the sequences before it, which every
// workgroup forms for itself (batch * 8 bytes out of the cache; a second launch that waited for the first's sums would cost more
// than they do).  Pages are taken from the front of the free stretch as it was before the call and put behind its end, so that no
// workgroup reads what another writes: the stretches cannot meet, since a page is free or with a sequence.
// What bounds it: latency (launch, lengths, sums over a workgroup: 3.6 of 4.2 us for 64 sequences with a token each), then the
// instructions that a stretch of a table and a slot take: 768 sequences of up to 32768 positions and 750000 slots, 19 MB, in 11.3 us, of
// which 4.5 are the sums.  (A wave that writes the slots of its stretch of a table from the pages that it has found, without a search:
// 13 us, since the tokens of a prompt are with few waves; 256 slots a wave at a time: 12.5.)
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kHeld = 2048;    // sequences whose lengths lie in LDS
constexpr int kStretch = 128;  // entries of a table that a wave takes at a time
constexpr int kSlots = 64;     // slots, likewise

struct Lens {
  int from, to;
  __device__ __forceinline__ int had() const { return (from + kBlockRows - 1) / kBlockRows; }
  __device__ __forceinline__ int want() const { return (to + kBlockRows - 1) / kBlockRows; }
  __device__ __forceinline__ int asked() const { return max(want() - had(), 0); }
  __device__ __forceinline__ int freed() const { return max(had() - want(), 0); }
  __device__ __forceinline__ int fresh() const { return max(to - from, 0); }
};

// Sums over the threads before this one; the total of all.
__device__ __forceinline__ int sum_before(int x, int* scratch, int& total) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 63) scratch[wave] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? scratch[w] : 0;
    total += scratch[w];
  }
  return before + sum - x;
}

__global__ __launch_bounds__(kThreads) void pages_kernel(PagesArgs a) {
  __shared__ int from_held[kHeld], to_held[kHeld];
  __shared__ int asked_before[kThreads], freed_before[kThreads], start[kThreads];
  __shared__ int scratch[3][kWaves], used_by[kWaves];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const bool held = a.batch <= kHeld;
  auto read = [&](int b) __attribute__((always_inline)) {
    return Lens{min(max(a.from[b], 0), a.t_max), min(max(a.to[b], 0), a.t_max)};
  };
  auto lens = [&](int b) __attribute__((always_inline)) { return held ? Lens{from_held[b], to_held[b]} : read(b); };
  const int count = min(max(a.state[1], 0), a.n_pages), given_head = a.state[0];
  const int head = given_head < 0 || given_head >= a.n_pages ? 0 : given_head;
  if (held) {
    Lens x[kHeld / kThreads];  // (all loads at once)
#pragma unroll
    for (int i = 0; i < kHeld / kThreads; ++i)
      if (i * kThreads < a.batch) x[i] = read(min(i * kThreads + (int)threadIdx.x, a.batch - 1));
#pragma unroll
    for (int i = 0; i < kHeld / kThreads; ++i)
      if (i * kThreads < a.batch) from_held[i * kThreads + threadIdx.x] = x[i].from, to_held[i * kThreads + threadIdx.x] = x[i].to;
    __syncthreads();
  }
  // a thread's stretch of sequences
  const int per = (a.batch + kThreads - 1) / kThreads, b0 = min((int)threadIdx.x * per, a.batch), b1 = min(b0 + per, a.batch);
  int asked = 0, freed = 0, fresh = 0;
  for (int b = b0; b < b1; ++b) {
    const Lens x = lens(b);
    asked += x.asked(), freed += x.freed(), fresh += x.fresh();
  }
  int all_asked, all_freed, all_fresh;
  asked_before[threadIdx.x] = sum_before(asked, scratch[0], all_asked);
  freed_before[threadIdx.x] = sum_before(freed, scratch[1], all_freed);
  start[threadIdx.x] = sum_before(fresh, scratch[2], all_fresh);
  __syncthreads();
  if (blockIdx.x == 0) {  // what there is one of per sequence, and per call
    int before = asked_before[threadIdx.x], at = start[threadIdx.x], used = 0;
    for (int b = b0; b < b1; ++b) {
      const Lens x = lens(b);
      const bool served = x.asked() == 0 || before + x.asked() <= count;
      if (a.lens_out) a.lens_out[b] = served ? x.to : x.from;
      if (a.starts) a.starts[b] = at;
      before += x.asked(), at += x.fresh();
      if (before <= count) used = before;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) used = max(used, __shfl_xor(used, o));
    if (lane == 0) used_by[wave] = used;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) used = max(used, used_by[w]);
      if (a.starts) a.starts[a.batch] = all_fresh;
      a.state_out[0] = (int)(((int64_t)head + used) % a.n_pages);
      a.state_out[1] = (int)min((int64_t)count - used + all_freed, (int64_t)a.n_pages);
    }
  }
  auto taken = [&](int64_t i) __attribute__((always_inline)) {  // i < count
    const int64_t at = head + i;
    return a.ring[at >= a.n_pages ? at - a.n_pages : at];
  };
  const uint32_t pieces = (a.max_blocks + kStretch - 1) / kStretch, tables = pieces * a.batch, tasks = tables + (uint32_t)((a.n_slots + kSlots - 1) / kSlots);
  for (uint32_t task = blockIdx.x * kWaves + wave; task < tasks; task += gridDim.x * kWaves) {
    if (task < tables) {  // a stretch of one sequence's row
      const int b = (int)(task / pieces), first = (int)(task % pieces) * kStretch;
      int asked_at = asked_before[b / per], freed_at = freed_before[b / per];
      for (int c = b / per * per; c < b; ++c) {
        const Lens x = lens(c);
        asked_at += x.asked(), freed_at += x.freed();
      }
      const Lens x = lens(b);
      const bool served = x.asked() == 0 || asked_at + x.asked() <= count;
      const int had = x.had(), want = served ? x.want() : had, stay = min(had, want), behind = max(had, want);
      const int32_t* row = a.table + (int64_t)b * a.max_blocks;
      int32_t* to = a.table_out + (int64_t)b * a.max_blocks;
      if (first + kStretch <= stay) {  // pages that stay
        if (to == row) continue;
        int page[kStretch / 64];
#pragma unroll
        for (int k = 0; k < kStretch / 64; ++k) page[k] = row[first + 64 * k + lane];
#pragma unroll
        for (int k = 0; k < kStretch / 64; ++k) to[first + 64 * k + lane] = page[k];
        continue;
      }
      const int last = min(first + kStretch, a.max_blocks);
      if (first >= behind) {  // none
        for (int j = first + lane; j < last; j += 64) to[j] = -1;
        continue;
      }
#pragma unroll
      for (int k = 0; k < kStretch; k += 64) {
        const int j = first + k + lane;
        if (j >= last) continue;
        int page = -1;
        if (j < had) page = row[j];
        if (j >= want && j < had) {
          a.ring[((int64_t)head + count + freed_at + j - want) % a.n_pages] = page;
          page = -1;
        }
        if (j >= had && j < want) page = taken((int64_t)asked_at + j - had);
        if (j >= stay || to != row) to[j] = page;
      }
      continue;
    }
    const int64_t first = (int64_t)(task - tables) * kSlots;
    if (first >= all_fresh) {  // behind the last token
      for (int64_t i = first + lane; i < min(first + kSlots, a.n_slots); i += 64) a.slots[i] = -1;
      continue;
    }
#pragma unroll
    for (int k = 0; k < kSlots; k += 64) {
      const int64_t i = first + k + lane;
      if (i >= a.n_slots) continue;
      int64_t slot = -1;
      if (i < all_fresh) {
        int t = 0;  // the last stretch of sequences that begins at i or before
#pragma unroll
        for (int o = kThreads / 2; o > 0; o >>= 1)
          if (start[t + o] <= i) t += o;
        int b = t * per, at = start[t], asked_at = asked_before[t];
        Lens x = lens(b);
        while (i >= at + x.fresh() && b + 1 < a.batch) {
          at += x.fresh(), asked_at += x.asked();
          x = lens(++b);
        }
        if (x.asked() == 0 || asked_at + x.asked() <= count) {
          const int pos = x.from + (int)(i - at), blk = pos / kBlockRows, had = x.had();
          const int64_t page = blk < had ? a.table[(int64_t)b * a.max_blocks + blk] : taken((int64_t)asked_at + blk - had);
          slot = page * kBlockRows + pos % kBlockRows;
        }
      }
      a.slots[i] = slot;
    }
  }
}

}  // namespace

hipError_t launch_pages(const PagesArgs& a, hipStream_t s) {
  const int64_t tasks = (int64_t)div_up(a.max_blocks, kStretch) * a.batch + (a.n_slots + kSlots - 1) / kSlots;
  if (tasks > INT32_MAX) return hipErrorNotSupported;
  // Six workgroups on a CU: more of them form the sums more often than their waves gain (768 sequences: 12.2 us with three, 11.7 with four,
  // 11.3 with six, 12.8 with eight); where the lengths of a long batch are read anew by each, one.
  const int64_t most = a.batch <= kHeld ? 1536 : 256;
  prof_mark("pages", s);
  hipLaunchKernelGGL(pages_kernel, dim3((unsigned)min((tasks + kWaves - 1) / kWaves, most)), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ams
