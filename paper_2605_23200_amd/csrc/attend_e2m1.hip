// Attention over a cache of 4 bits (ams_attend): the kernels of attend_kernel.h for its codes, and one that takes two heads at a time.
//
// A row of one head is 64 bytes (128 channels), half of a line: read head by head, a pool whose rows hold the heads side by side comes in
// requests of half a line (64 sequences of 4096 to 16384 positions and 8 heads: 11.1 million requests of 64 bytes and a pass of 266 us,
// against 5.6 million of 128 and 209 for slabs).  So, for up to 8 queries a head, a wave takes heads 2 i and 2 i + 1 together, and each of
// its loads both halves of a line:
//   K of 16 positions as two tiles, (positions 0..7 of head 0, the same of head 1) and (positions 8..15 of head 1, the same of head 0); the
//   columns are 8 queries of head 0 and 8 of head 1.  Half of either product is of one head's keys and the other's queries and is left out;
//   the other halves lie in different lanes, so that one select per logit makes them 4 logits a lane, of its query and head.
//   V as words P of positions 0..7 and Q of 8..15, lane groups 0, 1 of P and 2, 3 of Q holding head 0, the others head 1.  Each goes in as it
//   is, with the probabilities of the other head's lanes set to 0: both heads' outputs in the same accumulators.
// As many products as head by head, half of the work on logits.  That pass takes 207 us (206 for slabs), of which 172 are this kernel: 819 MB at
// 4.8 TB/s with the logits it writes.  What bounds it then is memory and how little of a stretch of 512 positions a workgroup spends at
// that rate (the vector ALU is active for 45 %): with 1024 positions a workgroup 204 us and 150 instead of 164 without weights, but 66 instead of
// 63 for 64 sequences of up to 4096, and 62 instead of 59 for 16 of up to 16384.  (512 workgroups that each take an even share of all
// positions: 218; three waves on a SIMD: 218.)  64 channels: half lines also two heads at a time, 157 us against 134 for slabs.
// 9 to 16 queries a head: the same tiles of K with the 16 columns of either head in turn, P and Q likewise: twice the products, none of the
// logits wasted.  64 ragged sequences of up to 16384 positions and 14 queries: a pass of 321 us, 362 head by head (306 in slabs).  222 of it are
// this kernel (vector ALU active for 54 %, matrix cores for 28 %, 24 % of the wave cycles waiting), 99 the join of its logits.
#include "attend_kernel.h"

namespace ams {
namespace {

// Not 0: a byte is 253 or more, a scale under which not every code is a finite bf16 number.
__device__ __forceinline__ uint32_t beyond(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x03030303u) & w & 0x80808080u; }

// SETS of columns: 1, 8 queries of either head; 2, 16 of each.
template <bool BF16, int HD, int SETS>
__global__ __launch_bounds__(kThreads, 2) void attend_pair_kernel(AttendArgs a) {
  constexpr int STEPS = HD / 32, TILES = HD / 16, TERMS = BF16 ? 1 : 3, PTERMS = BF16 ? 2 : 3;
  constexpr int LD = HD + 4;
  __shared__ __align__(16) float joint[kWaves][16][LD];
  __shared__ float2 stat[kWaves][16];
  const int unit0 = 2 * blockIdx.y, split = turned_x();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15, n = SETS == 1 ? c & 7 : c;  // the lane's query
  auto head_of = [&](int set) __attribute__((always_inline)) { return SETS == 1 ? c >> 3 : set; };
  auto first_tile = [&](int set) __attribute__((always_inline)) { return (g < 2) == (head_of(set) == 0); };
  auto group = [&](int set) __attribute__((always_inline)) { return g ^ (2 * head_of(set)); };  // its four positions of a block
  int l, b, h;
  unit_coords(a.d, unit0, l, b, h);
  const int T = seq_len(a.d, a.seq_lens, b), N = a.d.N;
  const int begin = split * a.chunk, end = min(T, begin + a.chunk);
  if (begin >= T && split > 0) return;  // the join knows; split 0 of an empty sequence writes the zeros
  bf16x8 q[SETS][STEPS][TERMS];
  {
    // (rows of the pair's second head follow the first's)
    const char* of_pair = a.q + (int64_t)unit0 * N * HD * (BF16 ? 2 : 4);
#pragma unroll
    for (int set = 0; set < SETS; ++set)
#pragma unroll
      for (int i = 0; i < STEPS; ++i)
        Queries<EL_E2M1, BF16, HD, 1>::load_one(of_pair, n < N ? head_of(set) * N + n : 2 * N, 2 * N, i, lane, q[set][i]);
  }
  const int limit = a.causal ? T - a.d.W + 1 + n % a.d.W : T, fewest = a.causal ? T - a.d.W + 1 : T;
  floatx4 o[SETS][TILES];
  float m[SETS], sum[SETS];
#pragma unroll
  for (int set = 0; set < SETS; ++set) {
    m[set] = kLowest, sum[set] = 0.f;
#pragma unroll
    for (int e = 0; e < TILES; ++e) o[set][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float to_log2 = kLog2E / sqrtf((float)HD);
  const UnitBlocks<EL_E2M1, HD> u(a.k, a.v, l, b, h);
  const uint32_t head_stride = a.k.paged ? HD / 2 : (uint32_t)(a.k.t_capacity * (HD / 2));
  const uint32_t head_scales = (a.k.paged ? 1 : (uint32_t)((a.k.t_capacity + kBlockRows - 1) / kBlockRows)) * kMicroBytes<HD>;
  const int last_blk = (T - 1) / kBlockRows;
  // The lane's byte offsets in a block: tiles of K (row 8 t + c % 8), words P and Q of V (rows 8 t + 4 (g % 2) + 0..3), their scales.
  const int row_stride = u.row_stride;
  uint32_t k_at[2], ks_at[2], v_at[2], vs_at[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const int k_head = (c >> 3) ^ t, v_head = (g >> 1) ^ t, k_row = 8 * t + (c & 7), v_row = 8 * t + 4 * (g & 1);
    k_at[t] = k_row * row_stride + k_head * head_stride + g * (HD / 8);
    ks_at[t] = k_head * head_scales + micro_at<HD>(g * (HD / 4), k_row);
    v_at[t] = v_row * row_stride + v_head * head_stride + c * (HD / 32);
    vs_at[t] = v_head * head_scales + micro_at<HD>(c * TILES, v_row);
  }
  uint32_t kw[2][2][HD / 32], vw[2][8], vs[2][2];
  float ks[2][2];
  int name[2] = {0, 0};
  int64_t slot[2] = {0, 0};
  auto find = [&](int at) __attribute__((always_inline)) {
    name[0] = u.named(min(at / kBlockRows, last_blk));
    name[1] = u.named(min(at / kBlockRows + 1, last_blk));
  };
  auto settle = [&]() __attribute__((always_inline)) { slot[0] = u.slot(name[0]), slot[1] = u.slot(name[1]); };
  // The step at `at`.  CLAMP (a wave's last): rows past the last position are that position again; what is behind it, in the cache or past
  // its end, is not read.
  auto load_k = [&](auto clamp, int at) __attribute__((always_inline)) {
    constexpr bool CLAMP = decltype(clamp)::value;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const char *block = u.k + slot[j] * u.block_bytes, *scales = u.k_scale + slot[j] * u.scale_step;
      const int most = T - 1 - min(at / kBlockRows + j, last_blk) * kBlockRows;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t past = CLAMP ? max(8 * t + (c & 7) - most, 0) : 0;
        const char* from = block + (k_at[t] - past * row_stride);
        if constexpr (HD == 128) {
          const uint4 x = *(const uint4*)from;
          kw[j][t][0] = x.x, kw[j][t][1] = x.y, kw[j][t][2] = x.z, kw[j][t][3] = x.w;
        } else {
          const uint2 x = *(const uint2*)from;
          kw[j][t][0] = x.x, kw[j][t][1] = x.y;
        }
        ks[j][t] = __uint_as_float((uint32_t) * (const uint8_t*)(scales + (ks_at[t] - past)) << 23);
      }
    }
  };
  auto load_v = [&](auto clamp, int at) __attribute__((always_inline)) {
    constexpr bool CLAMP = decltype(clamp)::value;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const char *block = u.v + slot[j] * u.block_bytes, *scales = u.v_scale + slot[j] * u.scale_step;
      const int most = T - 1 - min(at / kBlockRows + j, last_blk) * kBlockRows;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        vs[t][j] = *(const uint32_t*)(scales + vs_at[t]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const char* from;
          if constexpr (CLAMP)
            from = block + (v_at[t] + (min(8 * t + 4 * (g & 1) + i, most) - (8 * t + 4 * (g & 1))) * row_stride);
          else
            from = block + i * row_stride + v_at[t];
          if constexpr (HD == 128)
            vw[t][4 * j + i] = *(const uint32_t*)from;
          else
            vw[t][4 * j + i] = *(const uint16_t*)from;
        }
      }
    }
  };
  const int stride = kWaves * kStep;
  int at = begin + wave * kStep;
  // One step.  MORE: there is another, whose K is loaded when this one's has been used, V likewise; CLAMP: it is the wave's last.
  auto step = [&](auto more, auto clamp) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
    float x[SETS][8];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      floatx4 s[SETS][2];
      auto products = [&](auto ends) __attribute__((always_inline)) {  // ends: of the range of K
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int set = 0; set < SETS; ++set) s[set][t] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int i = 0; i < STEPS; ++i) {
            const bf16x8 k = eight_of_four_bits(kw[j][t][i], ks[j][t]), low = decltype(ends)::value ? without_infinite(k) : k;
#pragma unroll
            for (int set = 0; set < SETS; ++set)
#pragma unroll
              for (int r = TERMS - 1; r >= 0; --r) s[set][t] = mma(r > 0 ? low : k, q[set][i][r], s[set][t]);
          }
        }
      };
      products(std::false_type{});
      if constexpr (TERMS > 1)
        if (__any(max(__float_as_uint(ks[j][0]), __float_as_uint(ks[j][1])) >= kBeyond)) products(std::true_type{});
#pragma unroll
      for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[set][4 * j + i] = (first_tile(set) ? s[set][0][i] : s[set][1][i]) * to_log2;
    }
    const int next = at + stride;
    if constexpr (MORE) {
      settle();
      load_k(clamp, next);
      find(next + stride);
    }
    if (at + kStep > fewest) {
#pragma unroll
      for (int set = 0; set < SETS; ++set)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (at + (j >> 2) * 16 + 4 * group(set) + (j & 3) >= limit) x[set][j] = -INFINITY;
    }
    float top[SETS];
    bool higher = false;
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
      top[set] = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) top[set] = fmaxf(top[set], x[set][j]);
      higher = higher || top[set] > m[set] + kSlack;
    }
    if (__any(higher)) {
#pragma unroll
      for (int set = 0; set < SETS; ++set) {
        const float now = fmaxf(m[set], query_max(top[set])), shrink = power_of_two(m[set] - now);
        m[set] = now;
        sum[set] *= shrink;
#pragma unroll
        for (int e = 0; e < TILES; ++e) o[set][e] *= shrink;
      }
    }
    if (a.stash && n < N) {
#pragma unroll
      for (int set = 0; set < SETS; ++set) {
        float* to = a.stash + (((int64_t)(unit0 + head_of(set)) * ((a.d.t_max + 15) / 16) + at / 16) * N + n) * 16 + 4 * group(set);
        *(float4*)to = make_float4(x[set][0], x[set][1], x[set][2], x[set][3]);
        if (at + 16 < T) *(float4*)(to + N * 16) = make_float4(x[set][4], x[set][5], x[set][6], x[set][7]);
      }
    }
    if constexpr (!MORE) {  // (the sequence's end lies in a last step)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int there = min(max(T - min(at / kBlockRows + j, last_blk) * kBlockRows - (8 * t + 4 * (g & 1)), 0), 4);
          vs[t][j] &= there == 4 ? 0xFFFFFFFFu : (1u << 8 * there) - 1;
        }
    }
    if (__any((beyond(vs[0][0]) | beyond(vs[0][1]) | beyond(vs[1][0]) | beyond(vs[1][1])) != 0)) {
      // Channels of V that are no number: those of the queries that see the position, no others.  Scales under which codes may be infinite: a
      // quarter of them for the position's row, four times the probability, so that 0 times it stays 0.
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int shift = 8 * (j & 3);
          const bool mine = (vs[t][j >> 2] >> shift & 255) == 255;
          const uint64_t bad = __ballot(mine);
          if (mine) vs[t][j >> 2] &= ~(255u << shift);
          const uint32_t byte = vs[t][j >> 2] >> shift & 255;
          if (__ballot(byte >= 253) >> 16 * g & 0xFFFF) {
            vs[t][j >> 2] -= min(byte, 2u) << shift;
#pragma unroll
            for (int set = 0; set < SETS; ++set)
              if (first_tile(set) == (t == 0)) {
                x[set][j] += 2.f;
                sum[set] -= 0.75f * power_of_two(x[set][j] - m[set]);
              }
          }
          if (!bad) continue;
#pragma unroll
          for (int set = 0; set < SETS; ++set) {
            bool hit = false;
#pragma unroll
            for (int i = 0; i < 2; ++i)  // lane groups that hold the column's head, channels of the scale that its outputs have
              hit = hit || ((bad >> (16 * (2 * (head_of(set) ^ t) + i) + 4 * g * TILES / 32 * (32 / TILES)) & 1) &&
                            at + 16 * (j >> 2) + 8 * t + 4 * i + (j & 3) < limit);
            const float no_number = hit ? __uint_as_float(0x7FC00000u) : 0.f;
#pragma unroll
            for (int e = 0; e < TILES; ++e) o[set][e] += no_number;
          }
        }
    }
    // From here on nothing branches: exponentials, conversions and products can be mixed.
    bf16x8 p[SETS][2][PTERMS];
#pragma unroll
    for (int set = 0; set < SETS; ++set) {
      uint32_t t[3][4];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float p0 = power_of_two(x[set][j] - m[set]), p1 = power_of_two(x[set][j + 1] - m[set]);
        sum[set] += p0 + p1;
#pragma unroll
        for (int k = 0; k < PTERMS; ++k) {
          t[k][j >> 1] = bf16_pair(p0, p1);
          if (k + 1 < PTERMS) p0 -= __uint_as_float(t[k][j >> 1] << 16), p1 -= __uint_as_float(t[k][j >> 1] & 0xFFFF0000u);
        }
      }
      const uint32_t in_p = first_tile(set) ? 0xFFFFFFFFu : 0u, in_q = ~in_p;
#pragma unroll
      for (int k = 0; k < PTERMS; ++k) {
        p[set][0][k] = __builtin_bit_cast(bf16x8, make_uint4(t[k][0] & in_p, t[k][1] & in_p, t[k][2] & in_p, t[k][3] & in_p));
        p[set][1][k] = __builtin_bit_cast(bf16x8, make_uint4(t[k][0] & in_q, t[k][1] & in_q, t[k][2] & in_q, t[k][3] & in_q));
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float power[8];
      four_powers(vs[t], power);
#pragma unroll
      for (int w = 0; w < HD / 32; ++w) {
        bf16x8 e[2];
        turn_pair(vw[t], power, w, e[0], e[1]);
#pragma unroll
        for (int set = 0; set < SETS; ++set)
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int r = PTERMS - 1; r >= 0; --r) o[set][2 * w + k] = mma(e[k], p[set][t][r], o[set][2 * w + k]);
      }
    }
    if constexpr (MORE) load_v(clamp, next);
  };
  if (at < end) {
    find(at);
    settle();
    load_k(std::true_type{}, at);
    load_v(std::true_type{}, at);
    find(at + stride);
    for (; at + 2 * stride < end; at += stride) step(std::true_type{}, std::false_type{});
    if (at + stride < end) step(std::true_type{}, std::true_type{}), at += stride;
    step(std::false_type{}, std::true_type{});
  }
  // the waves together: thread (column, stretch of HD / 16 channels)
#pragma unroll
  for (int set = 0; set < SETS; ++set) {
    if (set > 0) __syncthreads();
    const float total = query_sum(sum[set]);
    if (g == 0) stat[wave][c] = make_float2(m[set], total);
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
#pragma unroll
      for (int e = 0; e < TILES; e += 4)
        *(float4*)&joint[wave][c][TILES * (4 * g + q4) + e] = make_float4(o[set][e][q4], o[set][e + 1][q4], o[set][e + 2][q4], o[set][e + 3][q4]);
    __syncthreads();
    const int column = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * TILES, of = SETS == 1 ? column & 7 : column;
    if (of >= N) continue;
    float highest = stat[0][column].x;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) highest = fmaxf(highest, stat[w][column].x);
    float y[TILES], all = 0.f;
#pragma unroll
    for (int e = 0; e < TILES; ++e) y[e] = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = power_of_two(stat[w][column].x - highest);
      all = fmaf(f, stat[w][column].y, all);
#pragma unroll
      for (int e = 0; e < TILES; ++e) y[e] = fmaf(f, joint[w][column][d0 + e], y[e]);
    }
    finish_query<BF16, HD>(a, unit0 + (SETS == 1 ? column >> 3 : set), of, split, highest, all, y, d0);
  }
}

template <bool BF16, int HD>
hipError_t launch_pairs(const AttendArgs& a, const AttendLayout& lay, hipStream_t s) {
  const dim3 grid(lay.n_splits, a.d.units / 2);
  prof_mark("attend", s);
  if (a.d.N <= 8)
    hipLaunchKernelGGL((attend_pair_kernel<BF16, HD, 1>), grid, dim3(kThreads), 0, s, a);
  else if constexpr (BF16 && HD == 128)
    hipLaunchKernelGGL((attend_pair_kernel<BF16, HD, 2>), grid, dim3(kThreads), 0, s, a);
  else
    return hipErrorNotSupported;
  if (lay.n_splits > 1 || a.stash) launch_attend_join(a, lay, BF16, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_attend_e2m1(const AttendArgs& a, const AttendLayout& lay, bool bf16, hipStream_t s) {
  if (lay.pairs) {
    if (a.d.D == 128) return bf16 ? launch_pairs<true, 128>(a, lay, s) : launch_pairs<false, 128>(a, lay, s);
    return bf16 ? launch_pairs<true, 64>(a, lay, s) : launch_pairs<false, 64>(a, lay, s);
  }
  return bf16 ? launch_dim<EL_E2M1, true>(a, lay, s) : launch_dim<EL_E2M1, false>(a, lay, s);
}

}  // namespace ams
