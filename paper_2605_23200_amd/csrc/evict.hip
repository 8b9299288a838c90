// Which positions stay by accumulated attention weight (ams_evict): the first and last ones of the rules, and of the others
// the `need` of largest weight, equal ones by lower position.  One workgroup per unit finds the need-th largest weight by its
// digits (8 bits at a time from the top, counts in LDS; three of the four passes over the row come out of L2), then every wave
// walks a stretch of the row and writes its kept positions behind those of the stretches before it.
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 16, kThreads = 64 * kWaves;

// Larger weight, larger key; no number: 0, below every number (-inf: 0x007FFFFF); -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__global__ __launch_bounds__(kThreads) void evict_pick_kernel(EvictArgs a) {
  __shared__ int bins[256];
  __shared__ int sums[kWaves], ties[kWaves];
  __shared__ uint32_t found[2];  // digit, keys above it
  const int unit = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int T = seq_len(a.d, a.seq_lens, b);
  const int kept = min(a.budget, T), sinks = min(a.n_sink, kept), last = min(a.n_last, kept - sinks);
  const int from = sinks, to = T - last;  // candidates
  const float* w = a.weights + (int64_t)unit * a.d.t_stride;
  float* out = a.weights_out + (int64_t)unit * a.d.t_stride;
  int32_t* idx = a.idx + (int64_t)unit * a.budget;
  // the need-th largest key: its digits, and how many of the keys equal to it stay
  int need = kept - sinks - last;
  uint32_t key = 0u, mask = 0u;
  if (need < to - from && need > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = threadIdx.x; i < 256; i += kThreads) bins[i] = 0;
      __syncthreads();
      for (int t = from + (int)threadIdx.x; t < to; t += kThreads) {
        const uint32_t k = weight_key(w[t]);
        if ((k & mask) == key) atomicAdd(&bins[k >> shift & 255], 1);
      }
      __syncthreads();
      if (threadIdx.x == 0) {
        int above = 0, digit = 255;
        while (above + bins[digit] < need) above += bins[digit--];
        found[0] = digit, found[1] = above;
      }
      __syncthreads();
      key |= found[0] << shift;
      mask |= 255u << shift;
      need -= (int)found[1];
      __syncthreads();
    }
  } else if (need > 0) {
    need = 0, key = 0u, mask = 0u;  // all of them stay (below)
  } else {
    mask = 1u;  // none of them
  }
  const bool all = mask == 0u, none = mask == 1u;
  // where each wave's stretch writes
  const int per = ((T + kWaves - 1) / kWaves + 63) & ~63, lo = min(T, wave * per), hi = min(T, lo + per);
  int above = 0, equal = 0;
  for (int t = lo + lane; t < hi; t += 64) {
    const bool always = t < from || t >= to;
    const uint32_t k = always || all || none ? 0u : weight_key(w[t]);
    above += always || all || (!none && k > key);
    equal += !always && !all && !none && k == key;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) above += __shfl_xor(above, o), equal += __shfl_xor(equal, o);
  if (lane == 0) sums[wave] = above, ties[wave] = equal;
  __syncthreads();
  int slot = 0, tied = 0;  // kept positions, equal keys before this stretch
  for (int v = 0; v < wave; ++v) slot += sums[v], tied += ties[v];
  slot += min(tied, need);
  for (int t0 = lo; t0 < hi; t0 += 64) {
    const int t = t0 + lane;
    bool stays = false, tie = false;
    float x = 0.f;
    if (t < hi) {
      const bool always = t < from || t >= to;
      x = w[t];
      const uint32_t k = weight_key(x);
      stays = always || all || (!none && k > key);
      tie = !always && !all && !none && k == key;
    }
    const uint64_t before = (1ull << lane) - 1, tie_set = __ballot(tie);
    stays = stays || (tie && tied + __popcll(tie_set & before) < need);
    const uint64_t set = __ballot(stays);
    if (stays) {
      const int j = slot + __popcll(set & before);
      idx[j] = t;
      out[j] = x;
    }
    slot += __popcll(set);
    tied += __popcll(tie_set);
  }
  for (int j = kept + (int)threadIdx.x; j < a.budget; j += kThreads) idx[j] = -1;
  for (int j = kept + (int)threadIdx.x; j < a.d.t_max; j += kThreads) out[j] = 0.f;
  if (threadIdx.x == 0) {
    a.n_kept[unit] = kept;
    if (a.lens_out && l == 0 && h == 0) a.lens_out[b] = kept;
  }
}

}  // namespace

size_t evict_ws_bytes(const ams_params*) { return 256; }

hipError_t launch_evict_pick(const EvictArgs& a, char*, hipStream_t s) {
  prof_mark("evict_pick", s);
  hipLaunchKernelGGL(evict_pick_kernel, dim3(a.d.units), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace ams
