// Which positions stay by accumulated attention weight (ams_evict): the first and last ones of the rules, and of the others
// the `need` of largest weight, equal ones by lower position.  One workgroup per unit.
//
// 1. The need-th largest weight, by its digits from the top, 11, 11 and 10 bits of an order-preserving integer image of the floats:
//    counts per digit in LDS, one wave finds the digit.  Rows of up to 16 positions a thread stay in registers, so that the
//    weights are read once.
// 2. Two bits a position, above that weight and equal to it, in LDS; sums of their counts say where each group of 64 writes, and which of
//    the equal ones stay.
// Longer rows have two launches before that, since one compute unit reads its row at no more than 15 to 25 GB/s (96 rows of 40000 to
// 131072 positions of which 4096 stay: 316 us with digits of the whole row from one workgroup, 112 with a sample and one
// walk, 53 now): a sample of the row says between which two values the wanted one lies, then many workgroups mark what is above
// and what is between.  The digits are those of what is between.  The sample is wrong once in some thousand rows; the counts
// show it, and the digits of the whole row decide.  So they do where more than 8192 positions lie between two different values: many
// equal weights, and the wanted one so near their first or last that the values take in the others (zeros under a high budget), or equal
// largest ones under a budget so small that the upper value is infinite.  One workgroup then walks the row up to four times (96
// rows of up to 131072: this launch 223 us against 23 with half of the weights equal to the largest and 300 kept; 96 rows of 131072, 60000
// kept, zeros from about there on: 298 against 95).
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 16, kThreads = 64 * kWaves;
constexpr int kBins = 2048;
constexpr int kSample = 4 * kThreads;
constexpr int kMarked = 4096 * 64;  // longest row with marks

// Larger weight, larger key; no number: 0, below every number (-inf: 0x007FFFFF); -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// The value of a key, for comparisons with weights (x > value, x >= value); keys beside the numbers: the nearest number's.
__device__ __forceinline__ float key_weight(uint32_t k) {
  k = min(max(k, 0x007FFFFFu), 0xFF800000u);
  if (k == 0x7FFFFFFFu) k = 0x7FFFFFFEu;  // -0 has the key of 0: the number below
  return __uint_as_float((k & 0x80000000u) ? k & 0x7FFFFFFFu : ~k);
}

// Sum over the lanes above this one.
__device__ __forceinline__ int wave_sum_above(int v, int lane) {
  int s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_down(s, o);
    if (lane + o < 64) s += up;
  }
  return s - v;
}

struct Found {
  int digit, above, equal;  // the bin that holds the need-th largest; keys in higher bins; keys in it
};

// One wave: the bin of the need-th largest key (1 <= need <= all of them).
__device__ __forceinline__ Found find_bin(const int* bins, int need, int lane) {
  constexpr int PER = kBins / 64;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < PER; i += 4) {
    const int4 v = *(const int4*)&bins[lane * PER + i];
    sum += v.x + v.y + v.z + v.w;
  }
  int above = wave_sum_above(sum, lane);
  const uint64_t holds = __ballot(above < need && above + sum >= need);
  const int owner = __ffsll((unsigned long long)holds) - 1;
  above = __shfl(above, owner);
  const int mine = lane < PER ? bins[owner * PER + lane] : 0;
  const int over = above + wave_sum_above(mine, lane);
  const uint64_t here = __ballot(over < need && over + mine >= need);
  const int at = __ffsll((unsigned long long)here) - 1;
  return Found{owner * PER + at, __shfl(over, at), __shfl(mine, at)};
}

template <int PER>
struct PickLds {
  static constexpr int kWords = PER ? 16 * PER : kMarked / 64;  // groups of 64 positions whose bits are here at a time
  static constexpr int kList = PER ? 1 : 16384;                 // kept positions that are written at a time, from a list
  static constexpr int kBetween = PER ? 4 : 8192;               // positions between the sample's bounds
  uint64_t over[kWords], tie[kWords];
  union {
    struct {
      __align__(16) int bins[2][kBins];
      uint32_t key[kBetween];
      int32_t where[kBetween];
    };
    int32_t list[kList];
    int32_t slot[PER ? kWords : 1];  // kept positions before the group
  };
  int sums[kWaves], tie_sums[kWaves];
  Found found;
};

// What precedes evict_pick_kernel for long rows, in the workspace: per unit the sample's bounds, and two bits a position.
struct Marks {
  float2* bounds;          // null: no marks
  uint64_t *over, *between;  // [units, words]
  int words;
};

// How many of the row's candidates [from, to) are wanted.
struct Rule {
  int T, kept, from, to, wanted;
  __device__ __forceinline__ Rule(const EvictArgs& a, int b) {
    T = seq_len(a.d, a.seq_lens, b);
    kept = min(a.budget, T);
    const int sinks = min(a.n_sink, kept), last = min(a.n_last, kept - sinks);
    from = sinks, to = T - last;
    wanted = kept - sinks - last;  // 0 .. to - from
  }
  __device__ __forceinline__ bool marked() const { return wanted > 0 && wanted < to - from && to - from > 4 * kSample; }
};

// Values between which the wanted one lies, from runs of four weights: exact ones of the sample, seven deviations of independent draws
// each way (neighbours resemble each other), fewer where that would leave more than four fifths of what can be kept between.
__global__ __launch_bounds__(kThreads) void evict_bounds_kernel(EvictArgs a, Marks m) {
  __shared__ __align__(16) int bins[2][kBins];
  __shared__ Found found[2];
  const int unit = blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const Rule r(a, b);
  if (!r.marked()) return;
  const float* w = a.weights + (int64_t)unit * a.d.t_stride;
  const int n = r.to - r.from;
  const double share = (double)r.wanted / n, mean = share * kSample;
  const int margin = (int)fmin(7.0 * sqrt(mean * (1 - share)), 0.4 * PickLds<0>::kBetween * kSample / n) + 4;
  const int rank[2] = {(int)mean - margin, (int)mean + margin};
  uint32_t key[4], bound[2] = {0, 0};
  int left[2] = {min(max(rank[0], 1), kSample), min(max(rank[1], 1), kSample)};
  const int run = r.from + (int)((int64_t)threadIdx.x * (n - 4) / kThreads);
#pragma unroll
  for (int i = 0; i < 4; ++i) key[i] = weight_key(w[run + i]);
#pragma unroll
  for (int shift = 21; shift >= 0; shift -= shift == 21 ? 11 : 10) {
    const uint32_t mask = shift == 21 ? 0u : ~0u << (shift == 10 ? 21 : 10);
    for (int i = threadIdx.x; i < 2 * kBins; i += kThreads) bins[0][i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        if ((key[i] & mask) == bound[k]) atomicAdd(&bins[k][key[i] >> shift & (shift == 0 ? 1023 : 2047)], 1);
    __syncthreads();
    if (wave < 2) {
      const Found f = find_bin(bins[wave], wave ? left[1] : left[0], lane);
      if (lane == 0) found[wave] = f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      bound[k] |= (uint32_t)found[k].digit << shift;
      left[k] -= found[k].above;
    }
  }
  if (threadIdx.x == 0)
    m.bounds[unit] = make_float2(rank[1] > kSample ? -INFINITY : key_weight(bound[1]), rank[0] < 1 ? INFINITY : key_weight(bound[0]));
}

constexpr int kMarkThreads = 256, kMarkGroups = 16;                   // groups of 64 positions per wave
constexpr int kMarkPositions = kMarkThreads / 64 * kMarkGroups * 64;  // per workgroup

// The bits of the row.
__global__ __launch_bounds__(kMarkThreads) void evict_mark_kernel(EvictArgs a, Marks m) {
  const int unit = blockIdx.y, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const Rule r(a, b);
  const int t0 = turned_x() * kMarkPositions + wave * kMarkGroups * 64;
  if (!r.marked() || t0 >= r.T) return;
  const float* w = a.weights + (int64_t)unit * a.d.t_stride;
  const float2 bound = m.bounds[unit];
  float x[kMarkGroups];
#pragma unroll
  for (int g = 0; g < kMarkGroups; ++g) x[g] = w[min(t0 + g * 64 + lane, r.T - 1)];
  uint64_t my_over = 0, my_between = 0;
#pragma unroll
  for (int g = 0; g < kMarkGroups; ++g) {
    const int t = t0 + g * 64 + lane;
    const bool in = t >= r.from && t < r.to;
    const uint64_t over = __ballot(in ? x[g] > bound.y : t < r.T), between = __ballot(in && x[g] >= bound.x && !(x[g] > bound.y));
    if (lane == g) my_over = over, my_between = between;
  }
  const int word = t0 / 64 + lane;
  if (lane < kMarkGroups && word < m.words) {
    m.over[(int64_t)unit * m.words + word] = my_over;
    m.between[(int64_t)unit * m.words + word] = my_between;
  }
}

// Zeros behind the kept weights of long rows, by workgroups of their own beside those that pick (they are memory, the others
// latency: 96 rows of up to 131072 positions 105 us an eviction; zeros beside the marks 109, beside the sample 109).
constexpr int kZeros = 64 * kThreads;  // positions per workgroup
__device__ __forceinline__ void write_zeros(const EvictArgs& a, int group) {
  const int groups = (a.d.t_max + kZeros - 1) / kZeros, unit = group / groups;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const Rule r(a, b);
  float* out = a.weights_out + (int64_t)unit * a.d.t_stride;
  const int begin = group % groups * kZeros, end = min(a.d.t_max, begin + kZeros);
  for (int t = max(begin, r.kept) + threadIdx.x; t < end; t += kThreads) out[t] = 0.f;
}

// PER: positions per thread whose weights stay in registers; 0: any length, from memory.
template <int PER>
__global__ __launch_bounds__(kThreads) void evict_pick_kernel(EvictArgs a, Marks m) {
  __shared__ PickLds<PER> s;
  if constexpr (PER == 0) {
    if ((int)blockIdx.x >= a.d.units) return write_zeros(a, (int)blockIdx.x - a.d.units);
  }
  const int unit = blockIdx.x, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const Rule rule(a, b);
  const int T = rule.T, kept = rule.kept, from = rule.from, to = rule.to, wanted = rule.wanted;
  const float* w = a.weights + (int64_t)unit * a.d.t_stride;
  float* out = a.weights_out + (int64_t)unit * a.d.t_stride;
  int32_t* idx = a.idx + (int64_t)unit * a.budget;
  constexpr int kWords = PickLds<PER>::kWords, kPerThread = (kWords + kThreads - 1) / kThreads;

  // f(first position, the lane's weight) for the groups of 64 positions of [begin, end) that are the wave's, whose lengths end at T
  float held[PER ? PER : 1];
  if constexpr (PER > 0) {
#pragma unroll
    for (int g = 0; g < PER; ++g) {
      const int t = (wave * PER + g) * 64 + lane;
      held[g] = t < T ? w[t] : 0.f;
    }
  }
  auto walk = [&](int begin, int end, auto f) __attribute__((always_inline)) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int g = 0; g < PER; ++g)
        if ((wave * PER + g) * 64 < T) f((wave * PER + g) * 64, held[g]);
    } else {
      constexpr int AHEAD = 8;  // groups in flight: one workgroup has the latency of its row to itself
      float next[AHEAD];
      auto fetch = [&](int t0) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) next[g] = w[min(t0 + g * 64 + lane, T - 1)];
      };
      int t0 = begin + wave * AHEAD * 64;
      if (t0 < end) fetch(t0);
      for (; t0 < end; t0 += kWaves * AHEAD * 64) {
        float x[AHEAD];
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) x[g] = next[g];
        fetch(t0 + kWaves * AHEAD * 64);  // (whatever comes: a load under a condition makes every wait one for all loads)
#pragma unroll
        for (int g = 0; g < AHEAD; ++g)
          if (t0 + g * 64 < end) f(t0 + g * 64, x[g]);
      }
    }
  };
  // Counts of one digit are in bins[turn] (the first ones cleared by clear_bins, the others by find, whose other waves have time).
  int turn = 0;
  auto clear_bins = [&]() __attribute__((always_inline)) {
    for (int i = threadIdx.x; i < kBins; i += kThreads) s.bins[0][i] = 0;
    turn = 0;
    __syncthreads();
  };
  auto find = [&](int need) __attribute__((always_inline)) {
    __syncthreads();
    if (wave == 0) {
      const Found f = find_bin(s.bins[turn], need, lane);
      if (lane == 0) s.found = f;
    } else {
      for (int i = threadIdx.x - 64; i < kBins; i += kThreads - 64) s.bins[turn ^ 1][i] = 0;
    }
    turn ^= 1;
    __syncthreads();
    return s.found;
  };
  auto before = [&](int v, int* sums, int& sum) __attribute__((always_inline)) {  // sum over lower threads; over all
    int run = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int down = __shfl_up(run, o);
      if (lane >= o) run += down;
    }
    if (lane == 63) sums[wave] = run;
    __syncthreads();
    int under = 0;
    sum = 0;
    for (int v2 = 0; v2 < kWaves; ++v2) {
      const int x = sums[v2];
      under += v2 < wave ? x : 0;
      sum += x;
    }
    return under + run - v;
  };

  const bool all = wanted == to - from;
  // keys above top stay, and of low .. top the first `ties`
  uint32_t low = 0, top = 0;
  int ties = 0;
  bool done = all || wanted == 0, marked = false;
  if constexpr (PER == 0) {
    if (m.bounds && rule.marked()) {
      const int words = (T + 63) / 64;
      uint64_t between[kPerThread];
      int n_over = 0, n_between = 0, total, n;
#pragma unroll
      for (int i = 0; i < kPerThread; ++i) {
        const int g = threadIdx.x * kPerThread + i;
        between[i] = g < words ? m.between[(int64_t)unit * m.words + g] : 0ull;
        const uint64_t over = g < words ? m.over[(int64_t)unit * m.words + g] : 0ull;
        s.over[g] = over, s.tie[g] = 0ull;
        n_over += __popcll(over), n_between += __popcll(between[i]);
      }
      int at = before(n_between, s.tie_sums, n);
      before(n_over, s.sums, total);
      const int need = kept - total;  // (the bits above hold those that stay whatever their weight)
      const float2 bound = m.bounds[unit];
      if (need >= 1 && need <= n && (n <= PickLds<0>::kBetween || bound.x == bound.y)) {
        marked = done = true;
        ties = need;
        if (bound.x == bound.y) {  // equal ones, all of them
#pragma unroll
          for (int i = 0; i < kPerThread; ++i) s.tie[threadIdx.x * kPerThread + i] = between[i];
        } else {
#pragma unroll
          for (int i = 0; i < kPerThread; ++i)
            for (uint64_t set = between[i]; set; set &= set - 1)
              s.where[at++] = (threadIdx.x * kPerThread + i) * 64 + __ffsll((unsigned long long)set) - 1;
          __syncthreads();
          for (int i = threadIdx.x; i < n; i += kThreads) s.key[i] = weight_key(w[s.where[i]]);
          clear_bins();
#pragma unroll
          for (int shift = 21; shift >= 0; shift -= shift == 21 ? 11 : 10) {
            const uint32_t mask = shift == 21 ? 0u : ~0u << (shift == 10 ? 21 : 10);
            for (int i = threadIdx.x; i < n; i += kThreads)
              if ((s.key[i] & mask) == low) atomicAdd(&s.bins[turn][s.key[i] >> shift & (shift == 0 ? 1023 : 2047)], 1);
            const Found f = find(ties);
            low |= (uint32_t)f.digit << shift;
            ties -= f.above;
          }
          for (int i = threadIdx.x; i < n; i += kThreads) {
            const int t = s.where[i];
            if (s.key[i] >= low)
              atomicOr((unsigned long long*)(s.key[i] > low ? &s.over[t >> 6] : &s.tie[t >> 6]), 1ull << (t & 63));
          }
        }
      }
      __syncthreads();
    }
  }
  if (!done) {
    int need = wanted;
    clear_bins();
    for (int shift = 21;; shift -= shift == 21 ? 11 : 10) {
      const uint32_t mask = shift == 21 ? 0u : ~0u << (shift == 10 ? 21 : 10);
      walk(0, T, [&](int t0, float x) __attribute__((always_inline)) {
        const uint32_t k = weight_key(x);
        if (t0 + lane >= from && t0 + lane < to && (k & mask) == low) atomicAdd(&s.bins[turn][k >> shift & (shift == 0 ? 1023 : 2047)], 1);
      });
      const Found f = find(need);
      low |= (uint32_t)f.digit << shift;
      need -= f.above;
      top = low | (shift == 0 ? 0u : (1u << shift) - 1u);
      ties = need;
      if (f.equal == need || shift == 0) break;  // all that share the digits stay; or there are no more digits
    }
    __syncthreads();  // the bins have been read
  }

  // By value where low and top are numbers' keys; no numbers among the ties: by key.
  const bool some = !all && wanted > 0, odd = some && low < 0x007FFFFFu;
  const float f_low = key_weight(low), f_top = key_weight(top);
  int slot0 = 0, rank0 = 0;  // kept positions, ties before the round
  for (int begin = 0; begin < T; begin += kWords * 64) {
    const int end = min(T, begin + kWords * 64), words = (end - begin + 63) / 64;
    if (!marked) walk(begin, end, [&](int t0, float x) __attribute__((always_inline)) {
      uint64_t over = 0, tie = 0;
      if (some) {
        if (!odd) {
          over = __ballot(x > f_top), tie = __ballot(x >= f_low) & ~over;
        } else {
          const uint32_t k = weight_key(x);
          over = __ballot(k > top), tie = __ballot(k >= low) & ~over;
        }
      }
      if (t0 < from || t0 + 64 > to) {
        const uint64_t always = __ballot(t0 + lane < T && (all || t0 + lane < from || t0 + lane >= to)), in = __ballot(t0 + lane < T);
        over = (over & in) | always, tie = tie & in & ~always;
      } else if (all) {
        over = ~0ull;
      }
      if (lane == 0) s.over[(t0 - begin) >> 6] = over, s.tie[(t0 - begin) >> 6] = tie;
    });
    __syncthreads();
    // ties before every group, then what stays of them, then the kept positions before it
    uint64_t over[kPerThread], tie[kPerThread];
    int n_tie = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int g = threadIdx.x * kPerThread + i;
      over[i] = g < words ? s.over[g] : 0ull, tie[i] = g < words ? s.tie[g] : 0ull;
      n_tie += __popcll(tie[i]);
    }
    int round_ties, round_kept;
    int rank = rank0 + before(n_tie, s.tie_sums, round_ties), n_kept = 0;
#pragma unroll
    for (int i = 0; i < kPerThread; ++i) {
      const int n = __popcll(tie[i]);
      if (rank + n > ties) {  // the first ties - rank of them
        const int stay = max(0, ties - rank);
        uint64_t rest = tie[i];
        for (int k = 0; k < stay; ++k) rest &= rest - 1;
        tie[i] &= ~rest;
      }
      rank += n;
      over[i] |= tie[i];
      n_kept += __popcll(over[i]);
    }
    int slot = slot0 + before(n_kept, s.sums, round_kept);
    if constexpr (PER > 0) {  // the weights are in the registers of the waves that walk the row
      if (threadIdx.x < kWords) s.over[threadIdx.x] = over[0], s.slot[threadIdx.x] = slot;
      __syncthreads();
      walk(begin, end, [&](int t0, float x) __attribute__((always_inline)) {
        const uint64_t set = s.over[t0 >> 6];
        if (set >> lane & 1) {
          const int j = s.slot[t0 >> 6] + __popcll(set & ((1ull << lane) - 1));
          idx[j] = t0 + lane, out[j] = x;
        }
      });
    } else {
      for (int base = 0; base < round_kept; base += PickLds<PER>::kList) {  // through a list of positions, so that loads and stores are dense
        int at = slot - slot0 - base;
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
          const int n = __popcll(over[i]);
          if (at + n > 0 && at < PickLds<PER>::kList) {
            int k = at;
            for (uint64_t set = over[i]; set; set &= set - 1, ++k)
              if (k >= 0 && k < PickLds<PER>::kList) s.list[k] = begin + (threadIdx.x * kPerThread + i) * 64 + __ffsll((unsigned long long)set) - 1;
          }
          at += n;
        }
        __syncthreads();
        for (int j = threadIdx.x; j < min(round_kept - base, PickLds<PER>::kList); j += kThreads) {
          const int t = s.list[j];
          idx[slot0 + base + j] = t, out[slot0 + base + j] = w[t];
        }
        __syncthreads();
      }
    }
    slot0 += round_kept, rank0 += round_ties;
    __syncthreads();  // before the next round's bits
  }
  for (int j = kept + (int)threadIdx.x; j < a.budget; j += kThreads) idx[j] = -1;
  if constexpr (PER > 0)  // else write_zeros
    for (int j = kept + (int)threadIdx.x; j < a.d.t_max; j += kThreads) out[j] = 0.f;
  if (threadIdx.x == 0) {
    a.n_kept[unit] = kept;
    if (a.lens_out && l == 0 && h == 0) a.lens_out[b] = kept;
  }
}

}  // namespace

static size_t mark_words(int t_max) { return t_max > 16 * kThreads && t_max <= kMarked ? (size_t)div_up(t_max, 64) : 0; }

size_t evict_ws_bytes(const ams_params* p) {
  const size_t units = (size_t)p->n_layers * p->batch * p->n_kv_heads;
  return 256 + units * (2 * mark_words(p->t_max) * sizeof(uint64_t) + sizeof(float2));
}

hipError_t launch_evict_pick(const EvictArgs& a, char* ws, hipStream_t s) {
  Marks m{};
  if (const size_t words = mark_words(a.d.t_max)) {
    m.over = (uint64_t*)ws, m.between = m.over + a.d.units * words, m.bounds = (float2*)(m.between + a.d.units * words);
    m.words = (int)words;
    prof_mark("evict_bounds", s);
    hipLaunchKernelGGL(evict_bounds_kernel, dim3(a.d.units), dim3(kThreads), 0, s, a, m);
    prof_mark("evict_mark", s);
    hipLaunchKernelGGL(evict_mark_kernel, dim3(div_up(a.d.t_max, kMarkPositions), a.d.units), dim3(kMarkThreads), 0, s, a, m);
  }
  prof_mark("evict_pick", s);
  if (a.d.t_max <= 4 * kThreads)
    hipLaunchKernelGGL((evict_pick_kernel<4>), dim3(a.d.units), dim3(kThreads), 0, s, a, m);
  else if (a.d.t_max <= 16 * kThreads)
    hipLaunchKernelGGL((evict_pick_kernel<16>), dim3(a.d.units), dim3(kThreads), 0, s, a, m);
  else
    hipLaunchKernelGGL((evict_pick_kernel<0>), dim3(a.d.units * (1 + div_up(a.d.t_max, kZeros))), dim3(kThreads), 0, s, a, m);
  return hipGetLastError();
}

}  // namespace ams
