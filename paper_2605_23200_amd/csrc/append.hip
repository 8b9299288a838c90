// New tokens into the cache (ams_append): norms over the head, rotary positions, rows of K and V (in kv_dtype or 8 bits), queries
// in the layout of the window, one pass over what the projections left.
//
// A workgroup takes the new tokens that fall into one block of 16 positions of a sequence and a slice of the heads.  It
// forms the cosines and sines of those tokens once, for all of its heads; a wave then takes a head at a time, eight channels a
// lane (16 lanes a row of 128 channels, four rows a load) and sums the squares over the row's lanes.  The block is the unit because its
// rows share a scale: all of them are in the wave's registers when the largest magnitude is known.
// A lane's eight channels are two runs of four, placed so that a pair's channels are in one lane (halves: 4 i and half + 4 i): no
// exchange, and four cosines and sines in one LDS read each.  (Eight channels in a row, with the other halves and interleaved
// cosines and sines out of LDS, took 35 us for 2036 tokens of 48 heads against 23: every read hit the same banks.)  Halves that are no
// multiple of four channels find the other channel in LDS.
// What bounds it: a launch and its chain of latencies for single tokens (5 us for one, 7 for 64 sequences); 64-bit arithmetic of the
// keys for long pieces (17 us for 2036 tokens of 48 heads to 8 bits, of 10 that the bytes take; 25 for 4096 tokens to bf16, 2048 each).
// Angles: position * (frequency / 2 pi) in 64 bits, whole turns taken off there: at position 10^6 fp32 would be off by 0.06 rad.
// Keys that go to 8 bits are normalised and rotated in 64 bits: a code changes by a whole step where the value
// crosses the middle between two, and fp32 takes about one key element in a million across.
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kPairs = 64;  // most rotated pairs

enum { TURN_NONE = 0, TURN_HALVES = 1, TURN_NEIGHBOURS = 2, TURN_ANY_HALVES = 3 };
struct Rotation {
  int mode, pairs;
  float gain;
  double turns[kPairs];  // per position
};

// To fp32 so that a later rounding to fewer bits comes out as from the 64 bits: towards zero, last bit set if anything was lost.
__device__ __forceinline__ float round_to_odd(double y) {
  const float f = (float)y;
  const double back = (double)f;
  if (back == y) return f;
  uint32_t u = __float_as_uint(f);
  if (fabs(back) > fabs(y)) u -= 1;
  return __uint_as_float(u | 1u);
}

// Cosine and sine of t turns, |t| <= 1/2: the nearest quarter turn off, Taylor's polynomials on |r| <= pi / 4 (the first term left
// out is 1e-15 of 1 in 64 bits; fp32 keeps 2e-9).
template <typename M>
__device__ __forceinline__ void cos_sin(double t, M& c, M& s) {
  const double quarter = rint(4.0 * t);
  const M r = (M)((t - 0.25 * quarter) * 6.283185307179586), z = r * r;
  M pc, ps;
  if constexpr (sizeof(M) == 8) {
    ps = fma(z, fma(z, fma(z, fma(z, fma(z, fma(z, -1.0 / 1307674368000.0, 1.0 / 6227020800.0), -1.0 / 39916800.0), 1.0 / 362880.0), -1.0 / 5040.0),
                    1.0 / 120.0), -1.0 / 6.0);
    pc = fma(z, fma(z, fma(z, fma(z, fma(z, fma(z, fma(z, 1.0 / 20922789888000.0, -1.0 / 87178291200.0), 1.0 / 479001600.0), -1.0 / 3628800.0),
                                  1.0 / 40320.0), -1.0 / 720.0), 1.0 / 24.0), -0.5);
  } else {
    ps = fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
    pc = fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f);
  }
  const M sine = r + r * z * ps, cosine = (M)1 + z * pc;
  const int q = (int)quarter & 3;
  const M a = q & 1 ? sine : cosine, b = q & 1 ? cosine : sine;
  c = (q == 1 || q == 2) ? -a : a;
  s = (q >= 2) ? -b : b;
}

// Sum over the lanes of a row (16 or 8 of them).
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ double moved(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)u, CTRL, 0xF, 0xF, true);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(u >> 32), CTRL, 0xF, 0xF, true);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int LANES, typename M>
__device__ __forceinline__ M row_sum(M x) {
  if constexpr (LANES == 16) x += moved<0x140>(x);  // lane 15 - i of 16
  x += moved<0x141>(x);                             // 7 - i of 8
  x += moved<0x4E>(x);                              // i ^ 2
  return x + moved<0xB1>(x);                        // i ^ 1
}
__device__ __forceinline__ float inverse_root(float v) { return v < 0x1p-100f ? 1.f / sqrtf(v) : __builtin_amdgcn_rsqf(v); }
__device__ __forceinline__ double inverse_root(double v) {
  double y = __builtin_amdgcn_rsq(v);  // 2^-14 or better, doubled twice
  if (v < 0x1p-1000 || !(y < 0x1p600)) return 1.0 / sqrt(v);
  for (int i = 0; i < 2; ++i) y = fma(y, 0.5 * fma(-v * y, y, 1.0), y);
  return y;
}

// Cosines and sines of a block's tokens.
template <typename M>
struct Turns {
  __align__(16) M cos[kBlockRows][kPairs], sin[kBlockRows][kPairs];
};

// First channels of the two runs of four that lane i of a row holds.
__device__ __forceinline__ void lane_runs(const Rotation& rot, int i, int& a, int& b) {
  a = 8 * i, b = 8 * i + 4;
  if (rot.mode == TURN_HALVES) {
    const int lanes = rot.pairs / 4;
    if (i < lanes) a = 4 * i, b = rot.pairs + 4 * i;  // else behind the 8 lanes channels that rotate, in order
  }
}

// Norm and rotation of the wave's rows: channels a .. a + 3 and b .. b + 3 of row x -> y.
template <typename M, int HD, bool ANY>
__device__ __forceinline__ void normed_and_turned(const float (&x)[8], const float (&weight)[8], bool norm, float eps, const Rotation& rot,
                                                  const M* cos_row, const M* sin_row, M* exchange, int i, M (&y)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (M)x[e];
  if (norm) {
    M ss = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fma(y[e], y[e], ss);
    const M inverse = inverse_root(row_sum<HD / 8>(ss) * (M)(1.0 / HD) + (M)eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= inverse * (M)weight[e];
  }
  if constexpr (!ANY) {
    if (rot.mode == TURN_NONE) return;
    // (channels behind the pairs are chosen as they are: turned by nothing, an infinity beside them would make them no number)
    M c[4], s[4];
    bool turns[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) c[e] = cos_row[4 * i + e], s[e] = sin_row[4 * i + e], turns[e] = 4 * i + e < rot.pairs;
    if (rot.mode == TURN_HALVES) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const M p = y[e], q = y[4 + e], first = p * c[e] - q * s[e], second = q * c[e] + p * s[e];
        y[e] = turns[e] ? first : p, y[4 + e] = turns[e] ? second : q;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const M p = y[2 * e], q = y[2 * e + 1], first = p * c[e] - q * s[e], second = q * c[e] + p * s[e];
        y[2 * e] = turns[e] ? first : p, y[2 * e + 1] = turns[e] ? second : q;
      }
    }
  } else {
    const int half = rot.pairs;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own stretch of LDS: its last readers are done
#pragma unroll
    for (int e = 0; e < 8; ++e) exchange[8 * i + e] = y[e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int d = 8 * i + e;
      if (d >= 2 * half) continue;
      const bool second = d >= half;
      const int pair = second ? d - half : d;
      const M c = cos_row[pair], s = sin_row[pair], other = exchange[second ? pair : d + half];
      y[e] = second ? y[e] * c + other * s : y[e] * c - other * s;
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Two runs of four elements of a row.
template <int EL>
__device__ __forceinline__ void load_runs(const char* row, int a, int b, float (&x)[8]) {
  if constexpr (EL == EL_F32) {
    const float4 p = *(const float4*)(row + a * 4), q = *(const float4*)(row + b * 4);
    x[0] = p.x, x[1] = p.y, x[2] = p.z, x[3] = p.w, x[4] = q.x, x[5] = q.y, x[6] = q.z, x[7] = q.w;
  } else if constexpr (EL == EL_BF16) {
    const uint2 p = *(const uint2*)(row + a * 2), q = *(const uint2*)(row + b * 2);
    const uint32_t w[4] = {p.x, p.y, q.x, q.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  } else {
    float lo[4], hi[4];
    unpack_codes<EL>(*(const uint32_t*)(row + a), lo);
    unpack_codes<EL>(*(const uint32_t*)(row + b), hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
  }
}
template <int EL>
__device__ __forceinline__ void store_runs(char* row, int a, int b, const float (&x)[8], float inverse = 1.f) {
  if constexpr (EL == EL_F32) {
    *(float4*)(row + a * 4) = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(row + b * 4) = make_float4(x[4], x[5], x[6], x[7]);
  } else if constexpr (EL == EL_BF16) {
    *(uint2*)(row + a * 2) = make_uint2(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]));
    *(uint2*)(row + b * 2) = make_uint2(bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
  } else {
    const uint2 p = pack_eight<EL>(x, inverse);
    *(uint32_t*)(row + a) = p.x, *(uint32_t*)(row + b) = p.y;
  }
}

// DST: element type of the cache; BF16: of the new rows (and of a cache of kv_dtype); ANY: rot.mode is TURN_ANY_HALVES, and no other
// (a kernel with both takes 180 registers and 40 KB of LDS for int8, two workgroups on a CU; without, 150 and 24 KB, three).
template <int DST, bool BF16, int HD, bool ANY>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, Rotation rot) {
  constexpr int SRC = BF16 ? EL_BF16 : EL_F32, ES = kElBytes<SRC>;
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, PASSES = kBlockRows / ROWS;
  constexpr bool PACK = kPacked<DST>;
  using M = std::conditional_t<PACK, double, float>;  // of keys
  __shared__ Turns<float> turns;
  __shared__ Turns<M> exact;  // (unused where M is float)
  __shared__ __align__(16) M exchange[ANY ? kWaves : 1][ANY ? ROWS : 1][ANY ? HD : 1];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.y % a.d.B, l = blockIdx.y / a.d.B;
  const int len = seq_len(a.d, a.seq_lens, b);
  const int blk = len / kBlockRows + turned_x();
  const int lo = max(len, blk * kBlockRows), hi = min(len + a.n_new, (blk + 1) * kBlockRows);
  if (blockIdx.x == 0 && blockIdx.z == 0 && l == 0 && threadIdx.x == 0 && a.lens_out)
    a.lens_out[b] = min(len + a.n_new, a.d.t_max);
  const int count = hi - lo, kept = min(hi, a.d.t_max) - lo;  // tokens here; those that the cache takes
  if (count <= 0) return;
  const int H = a.d.H, HQ = a.q ? H * a.d.G : 0, n_tasks = HQ + 2 * H;
  const int i = lane % LANES, r0 = lane / LANES;
  M* own = nullptr;
  if constexpr (ANY) own = exchange[wave][r0];
  int run_a, run_b;
  lane_runs(rot, i, run_a, run_b);
  const int64_t token0 = ((int64_t)l * a.d.B + b) * a.n_new + (lo - len);
  // the rows of a head's task: queries, then keys, then values
  float x[PASSES][8];
  auto fetch = [&](int task) __attribute__((always_inline)) {
    const bool is_q = task < HQ, is_k = !is_q && task < HQ + H;
    const int head = is_q ? task : is_k ? task - HQ : task - HQ - H;
    const int64_t step = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
    const char* src = (is_q ? a.q : is_k ? a.k : a.v) + token0 * step + (int64_t)head * HD * ES;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      if (p * ROWS >= count) break;
      load_runs<SRC>(src + min(p * ROWS + r0, count - 1) * step, run_a, run_b, x[p]);  // (rows past the last are that one again)
    }
  };
  int task = wave * gridDim.z + blockIdx.z;  // every workgroup has its share of the keys, which take longest
  const int task_step = kWaves * gridDim.z;
  if (task < n_tasks) fetch(task);  // on its way while the angles are formed
  const int first = a.positions ? a.positions[b] : len;
  for (int k = threadIdx.x; k < count * kPairs; k += kThreads) {
    const int r = k / kPairs, pair = k % kPairs;
    if (pair >= rot.pairs) continue;
    double t = ((double)first + (double)(lo - len + r)) * rot.turns[pair];
    t -= rint(t);
    M s, c;
    cos_sin(t, c, s);
    c *= (M)rot.gain, s *= (M)rot.gain;
    turns.cos[r][pair] = (float)c, turns.sin[r][pair] = (float)s;
    if constexpr (PACK) exact.cos[r][pair] = c, exact.sin[r][pair] = s;
  }
  __syncthreads();
  for (; task < n_tasks; task += task_step, task < n_tasks ? fetch(task) : (void)0) {
    const bool is_q = task < HQ, is_k = !is_q && task < HQ + H;
    const int head = is_q ? task : is_k ? task - HQ : task - HQ - H;
    float weight[8];
    const char* given = is_q ? a.q_weight : is_k ? a.k_weight : nullptr;
    if (given) load_runs<SRC>(given, run_a, run_b, weight);
    if (is_q) {
      char* to = a.q_out + ((((int64_t)l * a.d.B + b) * HQ + head) * a.n_new + (lo - len)) * (HD * ES);
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        if (p * ROWS >= count) break;
        const int r = p * ROWS + r0;
        float y[8];
        normed_and_turned<float, HD, ANY>(x[p], weight, given != nullptr, a.eps, rot, turns.cos[r], turns.sin[r], (float*)own, i, y);
        if (r < count) store_runs<SRC>(to + r * (HD * ES), run_a, run_b, y);
      }
      continue;
    }
    if (kept <= 0) continue;
    if (is_k) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        if (p * ROWS >= count) break;
        M y[8];
        const int r = p * ROWS + r0;
        const M *cos_row, *sin_row;
        if constexpr (PACK)
          cos_row = exact.cos[r], sin_row = exact.sin[r];
        else
          cos_row = turns.cos[r], sin_row = turns.sin[r];
        normed_and_turned<M, HD, ANY>(x[p], weight, given != nullptr, a.eps, rot, cos_row, sin_row, own, i, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if constexpr (PACK)
            x[p][e] = round_to_odd(y[e]);
          else
            x[p][e] = y[e];
        }
      }
    }
    const CacheDev dst = is_k ? a.kd : a.vd;
    const Block to = block_at(dst, l, b, head, blk);
    if (!to.there) continue;
    const int old = lo - blk * kBlockRows;  // rows of the block that were there
    if constexpr (!PACK) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * ROWS + r0;
        if (r < kept) store_runs<SRC>(to.row0 + (old + r) * to.stride, run_a, run_b, x[p]);
      }
    } else {
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
        if (p * ROWS + r0 < kept) top = top_bits(x[p], top);  // (not those past t_max)
      const float need = block_scale<DST>(wave_max(top)), had = old > 0 ? dst.scale[to.scale] : 0.f;
      const bool number = need == need && had == had;
      const float scale = number ? fmaxf(need, had) : __uint_as_float(0x7FC00000u);
      const float inverse = scale_inverse(scale);
      if (old > 0 && !(scale == had)) {  // the rows that were there, rounded again; codes of 0 under a scale that is no number
        const float ratio = number ? had * inverse : 0.f;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          const int r = p * ROWS + r0;
          if (r < old) {
            char* at = to.row0 + r * to.stride;
            float y[8];
            load_runs<DST>(at, run_a, run_b, y);
            store_runs<DST>(at, run_a, run_b, y, ratio);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * ROWS + r0;
        if (r < kept) store_runs<DST>(to.row0 + (old + r) * to.stride, run_a, run_b, x[p], inverse);
      }
      if (lane == 0 && (old == 0 || !(scale == had))) dst.scale[to.scale] = scale;
    }
  }
}

template <int DST, bool BF16, int HD>
hipError_t launch(const AppendArgs& a, const Rotation& rot, hipStream_t s) {
  const int tiles = (a.n_new + 14) / kBlockRows + 1, rows = a.d.L * a.d.B;
  const int tasks = (a.q ? a.d.H * a.d.G : 0) + 2 * a.d.H;
  // Slices of the heads: one round of workgroups, three on a CU where keys are formed in 64 bits (their registers), else four.  2036
  // tokens of 48 heads to 8 bits: 20.0 us with 396 workgroups, 17.3 with 660, 21.9 with 924; 4096 tokens, bf16: 38.5 with 516, 25.3
  // with 1032, 29.5 with 1548.
  const int slices = min(max(1, (kPacked<DST> ? 768 : 1024) / (int)min((int64_t)tiles * rows, (int64_t)1024)), div_up(tasks, kWaves));
  prof_mark("append", s);
  const dim3 grid(tiles, rows, slices);
  if (rot.mode == TURN_ANY_HALVES)
    hipLaunchKernelGGL((append_kernel<DST, BF16, HD, true>), grid, dim3(kThreads), 0, s, a, rot);
  else
    hipLaunchKernelGGL((append_kernel<DST, BF16, HD, false>), grid, dim3(kThreads), 0, s, a, rot);
  return hipGetLastError();
}

template <bool BF16, int HD>
hipError_t launch_to(const AppendArgs& a, const Rotation& rot, int el, hipStream_t s) {
  switch (el) {
    case EL_INT8: return launch<EL_INT8, BF16, HD>(a, rot, s);
    case EL_E4M3: return launch<EL_E4M3, BF16, HD>(a, rot, s);
    default: return launch<BF16 ? EL_BF16 : EL_F32, BF16, HD>(a, rot, s);
  }
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, const ams_rope* rope, bool bf16, int dst_el, hipStream_t s) {
  Rotation rot{};
  if (rope) {
    rot.pairs = rope->rot_dim / 2, rot.gain = rope->gain;
    rot.mode = rot.pairs == 0 ? TURN_NONE : rope->layout == AMS_ROPE_INTERLEAVED ? TURN_NEIGHBOURS : rot.pairs % 4 ? TURN_ANY_HALVES : TURN_HALVES;
    for (int i = 0; i < rot.pairs; ++i) rot.turns[i] = rope->freq[i] / 6.283185307179586;
  }
  if (a.d.D == 128) return bf16 ? launch_to<true, 128>(a, rot, dst_el, s) : launch_to<false, 128>(a, rot, dst_el, s);
  return bf16 ? launch_to<true, 64>(a, rot, dst_el, s) : launch_to<false, 64>(a, rot, dst_el, s);
}

}  // namespace ams
