#include "attend_kernel.h"

namespace ams {
namespace {

__device__ __forceinline__ int splits_of(const AttendArgs& a, int T) { return max(1, (T + a.chunk - 1) / a.chunk); }

// (largest logit, sum) of a query from its splits, for the LANES lanes that ask for it together; loads in batches, since a batch is a
// latency (one unit of 131072 positions: 21 us a pass with half of this batch and of AHEAD below, 18 so).
template <int LANES>
__device__ __forceinline__ float2 joined_stats(const AttendArgs& a, int unit, int n, int n_splits, int lane) {
  constexpr int BATCH = 4;
  const float2* at = a.stats + ((int64_t)unit * a.d.N + n) * a.n_splits;
  float top = kLowest, sum = 0.f;
  for (int s0 = lane; s0 < n_splits; s0 += BATCH * LANES) {
    float2 x[BATCH];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) x[i] = at[min(s0 + i * LANES, n_splits - 1)];
    float now = top;
#pragma unroll
    for (int i = 0; i < BATCH; ++i) now = fmaxf(now, x[i].x);
    sum *= power_of_two(top - now);
    top = now;
#pragma unroll
    for (int i = 0; i < BATCH; ++i)
      if (s0 + i * LANES < n_splits) sum = fmaf(power_of_two(x[i].x - top), x[i].y, sum);
  }
  float all = sixteen_max(top);
  if constexpr (LANES == 64) all = query_max(all);
  sum = sixteen_sum(sum * power_of_two(top - all));
  if constexpr (LANES == 64) sum = query_sum(sum);
  return make_float2(all, sum);
}

// Joins the splits of query n: a wave takes every fourth group of splits, HD / 4 lanes a split, four channels a lane; then the lanes
// and waves of the same channels together.
template <bool BF16, int HD>
__device__ __forceinline__ void join_splits(const AttendArgs& a, int unit, int n, int splits) {
  constexpr int LANES = HD / 4, SIDE = 64 / LANES, AHEAD = 8;
  __shared__ __align__(16) float part[kWaves][HD];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const float2* stats = a.stats + ((int64_t)unit * a.d.N + n) * a.n_splits;
  const float* from = a.part + ((int64_t)unit * a.n_splits * a.d.N + n) * HD + lane % LANES * 4;
  const int64_t step = (int64_t)a.d.N * HD;
  const float2 st = joined_stats<64>(a, unit, n, splits, lane);
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = wave * SIDE + lane / LANES; s0 < splits; s0 += kWaves * SIDE * AHEAD) {
    float4 y[AHEAD];
    float f[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int s = min(s0 + i * kWaves * SIDE, splits - 1);  // (past the last split: that one again, counted 0)
      y[i] = *(const float4*)(from + s * step);
      f[i] = stats[s].x;
    }
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const float w = s0 + i * kWaves * SIDE < splits ? power_of_two(f[i] - st.x) : 0.f;
      x.x = fmaf(w, y[i].x, x.x), x.y = fmaf(w, y[i].y, x.y), x.z = fmaf(w, y[i].z, x.z), x.w = fmaf(w, y[i].w, x.w);
    }
  }
#pragma unroll
  for (int o = LANES; o < 64; o <<= 1) x.x += __shfl_xor(x.x, o), x.y += __shfl_xor(x.y, o), x.z += __shfl_xor(x.z, o), x.w += __shfl_xor(x.w, o);
  if (lane < LANES) *(float4*)&part[wave][lane * 4] = x;
  __syncthreads();
  const int d = threadIdx.x;
  if (d < HD) {
    const float y = (part[0][d] + part[1][d] + part[2][d] + part[3][d]) * (st.y == 0.f ? 0.f : 1.f / st.y);
    const int64_t at = ((int64_t)unit * a.d.N + n) * HD + d;
    if constexpr (BF16)
      *(uint16_t*)(a.out + at * 2) = (uint16_t)bf16_pair(y, 0.f);
    else
      *(float*)(a.out + at * 4) = y;
  }
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[(int64_t)unit * a.d.N + n] = st.y == 0.f ? -INFINITY : (st.x + log2f(st.y)) * kLn2;
    if (a.joined) a.joined[(int64_t)unit * a.d.N + n] = st;
  }
}

constexpr int kStashKeys = 4 * kThreads;  // positions per workgroup that turns stashed logits into weights

// The workgroups of one unit: N of them join the splits (where there is more than one), the others form the weights from stashed logits.
template <bool BF16, int HD>
__global__ __launch_bounds__(kThreads) void attend_join_kernel(AttendArgs a, int joins) {
  __shared__ float2 stat[16];
  const int unit = blockIdx.y, N = a.d.N;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int T = seq_len(a.d, a.seq_lens, b), splits = splits_of(a, T);
  if ((int)blockIdx.x < joins) {  // (first: they take longest)
    join_splits<BF16, HD>(a, unit, blockIdx.x, splits);
    return;
  }
  const int first = turned_x(joins) * kStashKeys;
  if (first >= T) return;
  // The first logits and the weights are on their way while the statistics are joined.
  constexpr int AHEAD = 4;
  const int t = first + 4 * threadIdx.x;
  const float* x = a.stash + (((int64_t)unit * ((a.d.t_max + 15) / 16) + min(t, T - 1) / 16) * N) * 16 + t % 16;
  const int64_t at = (int64_t)unit * a.d.t_stride + t;
  float4 ahead[AHEAD];
  float w[4];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) ahead[i] = *(const float4*)(x + min(i, N - 1) * 16);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = a.weights_in && t + i < T ? a.weights_in[at + i] : 0.f;
  {
    const int n = threadIdx.x >> 4;
    const float2 st = joined_stats<16>(a, unit, min(n, N - 1), splits, threadIdx.x & 15);
    if ((threadIdx.x & 15) == 0) stat[n] = make_float2(st.x, st.y == 0.f ? 0.f : 1.f / st.y);
  }
  __syncthreads();
  if (t >= T) return;
  float more[4] = {0.f, 0.f, 0.f, 0.f};
  auto add = [&](const float4& v, int n) __attribute__((always_inline)) {
    const float s[4] = {v.x, v.y, v.z, v.w};
    const float2 st = stat[n];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (a position that the query does not see has no part in a sum that is no number)
      const float p = power_of_two(s[i] - st.x) * st.y;
      more[i] += s[i] == -INFINITY ? 0.f : p;
    }
  };
#pragma unroll
  for (int i = 0; i < AHEAD; ++i)
    if (i < N) add(ahead[i], i);
#pragma unroll 4
  for (int n = AHEAD; n < N; ++n) add(*(const float4*)(x + n * 16), n);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t + i < T) a.weights_out[at + i] = w[i] + more[i];
}

template <bool BF16, int HD>
void launch_join(const AttendArgs& a, const AttendLayout& lay, hipStream_t s) {
  const int joins = lay.n_splits > 1 ? a.d.N : 0, stash = a.stash ? div_up(a.d.t_max, kStashKeys) : 0;
  prof_mark("attend_join", s);
  hipLaunchKernelGGL((attend_join_kernel<BF16, HD>), dim3(joins + stash, a.d.units), dim3(kThreads), 0, s, a, joins);
}

}  // namespace

AttendLayout attend_layout(const ams_params* p, bool pairs) {
  AttendLayout r;
  const size_t units = (size_t)p->n_layers * p->batch * p->n_kv_heads, N = (size_t)p->group * p->window;
  const int tiles = div_up(N, 16);
  r.row_tiles = tiles <= 1 ? 1 : 2;
  r.row_waves = tiles <= 2 ? 1 : tiles <= 4 ? 2 : 4;
  r.row_groups = div_up(tiles, r.row_tiles * r.row_waves);
  r.stashed = N <= 16;
  // Positions per workgroup: 512 where that fills the chip several times over (ragged sequences end at different times), 2048 with more
  // than 16 queries, whose partial outputs are no longer small beside the cache (4 N / chunk of its bytes, written and read again); else
  // as many as give one round of workgroups, three on a CU (two with more than 16 queries; one fewer with fp32 queries of 128
  // channels, whose three terms take the registers: 64 us with 256 workgroups, 74 with 512, 96 with 1024).  Us a pass, 512 ragged
  // paged units of up to 16384: 324 with 512, 329 with 1024, 349 with 2048, 412 with 4096; 4 units of 131072: 45.6 with 512, 44.7 in
  // one round, 48 in two; 256 ragged units of up to 16384 and 32 queries: 301, 281, 277, 282; 320 and 128 queries: 840, 730, 724, 781;
  // 64 units of 32768 and 32 queries: 201, 187, 178, 172 (the last is one round).
  // Pairs of heads (4 bits): one on a CU, with twice the loads in flight (one, two, three, four on a CU: 4 units of 131072 26, 27, 31, 33 us;
  // 32 units of 16384 23.3, 24.2, 25.9, 27.0, ragged ones 22.4, 22.1, 24.5, 24.3; 128 of 8192 45, 48, 51, 49, ragged ones 35, 34, 31, 35).  That
  // is never more splits than head by head, so the workspace for any cache is that of one head at a time.  Where one round leaves a quarter of
  // the CUs or more without a workgroup, 512 positions again, in no more splits than head by head: 264 units of 7000 91 -> 78 us, ragged ones
  // 86 -> 55; 264 of 4096 57 -> 53 and 53 -> 34, 320 60 -> 58 and 54 -> 39, 384 66 -> 68 and 56 -> 49; 176 of 10000 79 -> 74 and 69 -> 55.
  // Not where more have one: 224 units of 4096 38.6 and 41.2 us, 480 77 and 85.
  r.pairs = pairs;
  const size_t per_split = units * r.row_groups / (pairs ? 2 : 1), resident = pairs ? 1 : (r.row_tiles == 1 ? 3 : 2) - (p->kv_dtype == AMS_F32 && p->head_dim == 128);
  const int fine = r.row_tiles == 1 ? 512 : 2048;
  if (per_split * div_up(p->t_max, fine) >= 2048) {
    r.chunk = fine;
  } else {
    const int splits = (int)max((size_t)1, 256 * resident / per_split);
    r.chunk = div_up(div_up(p->t_max, splits), kWaves * kStep) * kWaves * kStep;
    if (pairs && 4 * splits * per_split <= 3 * 256)
      r.chunk = max(fine, div_up(div_up(p->t_max, attend_layout(p, false).n_splits), kWaves * kStep) * kWaves * kStep);
  }
  while (div_up(p->t_max, r.chunk) > 4096) r.chunk *= 2;  // what the join goes through
  r.n_splits = div_up(p->t_max, r.chunk);
  auto align = [](size_t x) { return (x + 255) & ~(size_t)255; };
  size_t o = 0;
  r.stats = o, o += align(units * r.n_splits * N * sizeof(float2));
  r.joined = o, o += r.n_splits > 1 && !r.stashed ? align(units * N * sizeof(float2)) : 0;
  r.part = o, o += r.n_splits > 1 ? align(units * r.n_splits * N * p->head_dim * sizeof(float)) : 0;
  r.stash = o, o += r.stashed ? align(units * div_up(p->t_max, kBlockRows) * N * kBlockRows * sizeof(float)) : 0;
  r.total = o;
  return r;
}

void launch_attend_join(const AttendArgs& a, const AttendLayout& lay, bool bf16, hipStream_t s) {
  if (a.d.D == 128) return bf16 ? launch_join<true, 128>(a, lay, s) : launch_join<false, 128>(a, lay, s);
  return bf16 ? launch_join<true, 64>(a, lay, s) : launch_join<false, 64>(a, lay, s);
}

hipError_t launch_attend(const AttendArgs& a, const AttendLayout& lay, bool bf16, int el, hipStream_t s) {
  if (el == EL_E2M1) return launch_attend_e2m1(a, lay, bf16, s);
  if (el == EL_INT8) return bf16 ? launch_dim<EL_INT8, true>(a, lay, s) : launch_dim<EL_INT8, false>(a, lay, s);
  return bf16 ? launch_dim<EL_E4M3, true>(a, lay, s) : launch_dim<EL_E4M3, false>(a, lay, s);
}

}  // namespace ams
