// New tokens into the cache (ams_append): norms over the head, rotary positions, rows of K and V (in kv_dtype or 8 bits), queries
// in the layout of the window, one pass over what the projections left.
//
// A workgroup takes the new tokens that fall into one block of 16 positions of a sequence and a slice of the heads.  It
// forms the cosines and sines of those tokens once, for all of its heads; a wave then takes a head at a time, eight channels a
// lane (16 lanes a row of 128 channels, four rows a load), sums the squares over the row's lanes, finds the other channel of a pair
// in LDS and writes.  The block is the unit because its rows share a scale: all of them are in the wave's registers when the
// largest magnitude is known.
// Angles: position * (frequency / 2 pi) in 64 bits, whole turns taken off there: at position 10^6 fp32 would be off by 0.06 rad.
// Keys that go to 8 bits are normalised and rotated in 64 bits: a code changes by a whole step where the value
// crosses the middle between two, and fp32 takes about one key element in a million across.
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kPairs = 64;  // most rotated pairs

struct Rotation {
  int layout, rot_dim;
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

template <typename M>
struct Turn {
  M cos, sin;
};

// Norm and rotation of the wave's rows: eight channels 8 i .. 8 i + 7 of row x -> y.
template <typename M, typename TAB, int HD>
__device__ __forceinline__ void normed_and_turned(const float (&x)[8], const float (&weight)[8], bool norm, float eps, const Rotation& rot,
                                                  const Turn<TAB>* row_turns, M* exchange, int i, M (&y)[8]) {
  constexpr int LANES = HD / 8;
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = (M)x[e];
  if (norm) {
    M ss = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += y[e] * y[e];
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    const M inverse = (M)1 / sqrt(ss / (M)HD + (M)eps);
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] *= inverse * (M)weight[e];
  }
  if (rot.rot_dim == 0) return;
  if (rot.layout == AMS_ROPE_INTERLEAVED) {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const int d = 8 * i + e;
      if (d >= rot.rot_dim) continue;
      const M c = (M)row_turns[d / 2].cos, s = (M)row_turns[d / 2].sin;
      const M p = y[e], q = y[e + 1];
      y[e] = p * c - q * s;
      y[e + 1] = q * c + p * s;
    }
    return;
  }
  const int half = rot.rot_dim / 2;
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the wave's own stretch of LDS: its last readers are done
#pragma unroll
  for (int e = 0; e < 8; ++e) exchange[8 * i + e] = y[e];
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = 8 * i + e;
    if (d >= rot.rot_dim) continue;
    const bool second = d >= half;
    const int pair = second ? d - half : d;
    const M c = (M)row_turns[pair].cos, s = (M)row_turns[pair].sin;
    const M other = exchange[second ? pair : d + half];
    y[e] = second ? y[e] * c + other * s : y[e] * c - other * s;
  }
  __builtin_amdgcn_wave_barrier();
}

// DST: element type of the cache; BF16: of the new rows (and of a cache of kv_dtype).
template <int DST, bool BF16, int HD>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a, Rotation rot, int tasks_per_group) {
  constexpr int SRC = BF16 ? EL_BF16 : EL_F32, ES = kElBytes<SRC>;
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, PASSES = kBlockRows / ROWS;
  constexpr bool PACK = kPacked<DST>;
  using M = std::conditional_t<PACK, double, float>;  // of keys, and of the table
  __shared__ Turn<M> turns[kBlockRows][kPairs];
  __shared__ __align__(16) M exchange[kWaves][ROWS][HD];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int b = blockIdx.y % a.d.B, l = blockIdx.y / a.d.B;
  const int len = seq_len(a.d, a.seq_lens, b);
  const int blk = len / kBlockRows + (int)blockIdx.x;
  const int lo = max(len, blk * kBlockRows), hi = min(len + a.n_new, (blk + 1) * kBlockRows);
  if (blockIdx.x == 0 && blockIdx.z == 0 && l == 0 && threadIdx.x == 0 && a.lens_out)
    a.lens_out[b] = min(len + a.n_new, a.d.t_max);
  const int count = hi - lo, kept = min(hi, a.d.t_max) - lo;  // tokens here; those that the cache takes
  if (count <= 0) return;
  const int first = a.positions ? a.positions[b] : len;
  const int pairs = rot.rot_dim / 2;
  for (int k = threadIdx.x; k < count * pairs; k += kThreads) {
    const int r = k / pairs, i = k % pairs;
    double t = ((double)first + (double)(lo - len + r)) * rot.turns[i];
    t -= rint(t);
    M s, c;
    if constexpr (PACK) {
      sincospi(2.0 * t, &s, &c);
    } else {
      sincospif((float)(2.0 * t), &s, &c);
    }
    turns[r][i] = Turn<M>{c * (M)rot.gain, s * (M)rot.gain};
  }
  __syncthreads();
  const int H = a.d.H, HQ = a.q ? H * a.d.G : 0, n_tasks = HQ + 2 * H;
  const int i = lane % LANES, r0 = lane / LANES;
  float qw[8], kw[8];
  if (a.q_weight) load_eight<SRC>(a.q_weight + i * 8 * ES, qw);
  if (a.k_weight) load_eight<SRC>(a.k_weight + i * 8 * ES, kw);
  const int64_t token0 = ((int64_t)l * a.d.B + b) * a.n_new + (lo - len);
  const int end = min(n_tasks, (int)(blockIdx.z + 1) * tasks_per_group);
  for (int task = blockIdx.z * tasks_per_group + wave; task < end; task += kWaves) {
    const bool is_q = task < HQ, is_k = !is_q && task < HQ + H;
    const int head = is_q ? task : is_k ? task - HQ : task - HQ - H;
    const char* src = (is_q ? a.q + token0 * a.q_stride : is_k ? a.k + token0 * a.k_stride : a.v + token0 * a.v_stride) +
                      (int64_t)head * HD * ES + i * 8 * ES;
    const int64_t step = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
    float x[PASSES][8];
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * ROWS + r0;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[p][e] = 0.f;
      if (r < count) load_eight<SRC>(src + r * step, x[p]);
    }
    if (is_q) {
      char* to = a.q_out + ((((int64_t)l * a.d.B + b) * HQ + head) * a.n_new + (lo - len)) * (HD * ES) + i * 8 * ES;
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        if (p * ROWS >= count) break;
        const int r = p * ROWS + r0;
        float y[8];
        normed_and_turned<float, M, HD>(x[p], qw, a.q_weight != nullptr, a.eps, rot, turns[r], (float*)exchange[wave][r0], i, y);
        if (r < count) store_eight<SRC>(to + r * (HD * ES), y);
      }
      continue;
    }
    if (kept <= 0) continue;
    if (is_k) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        if (p * ROWS >= count) break;
        M y[8];
        normed_and_turned<M, M, HD>(x[p], kw, a.k_weight != nullptr, a.eps, rot, turns[p * ROWS + r0], exchange[wave][r0], i, y);
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
        if (r < kept) store_eight<SRC>(to.row0 + (old + r) * to.stride + i * 8 * ES, x[p]);
      }
    } else {
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < PASSES; ++p)
        if (p * ROWS + r0 < kept) top = top_bits(x[p], top);
      const float need = block_scale<DST>(wave_max(top)), had = old > 0 ? dst.scale[to.scale] : 0.f;
      const bool number = need == need && had == had;
      const float scale = number ? fmaxf(need, had) : __uint_as_float(0x7FC00000u);
      const float inverse = scale_inverse(scale);
      if (old > 0 && scale > had) {  // the rows that were there, rounded again
        const float ratio = had * inverse;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
          const int r = p * ROWS + r0;
          if (r < old) {
            char* at = to.row0 + r * to.stride + i * 8;
            float y[8];
            load_eight<DST>(at, y);
            *(uint2*)at = pack_eight<DST>(y, ratio);
          }
        }
      }
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * ROWS + r0;
        if (r < kept) *(uint2*)(to.row0 + (old + r) * to.stride + i * 8) = pack_eight<DST>(x[p], inverse);
      }
      if (lane == 0 && (old == 0 || !(scale == had))) dst.scale[to.scale] = scale;
    }
  }
}

template <int DST, bool BF16, int HD>
hipError_t launch(const AppendArgs& a, const Rotation& rot, hipStream_t s) {
  const int tiles = (a.n_new + 14) / kBlockRows + 1, rows = a.d.L * a.d.B;
  const int tasks = (a.q ? a.d.H * a.d.G : 0) + 2 * a.d.H;
  int per = kWaves;
  while (per < tasks && (int64_t)tiles * rows * div_up(tasks, per) > 2048) per *= 2;
  prof_mark("append", s);
  hipLaunchKernelGGL((append_kernel<DST, BF16, HD>), dim3(tiles, rows, div_up(tasks, per)), dim3(kThreads), 0, s, a, rot, per);
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
    rot.layout = rope->layout, rot.rot_dim = rope->rot_dim, rot.gain = rope->gain;
    for (int i = 0; i < rope->rot_dim / 2; ++i) rot.turns[i] = rope->freq[i] / 6.283185307179586;
  }
  if (a.d.D == 128) return bf16 ? launch_to<true, 128>(a, rot, dst_el, s) : launch_to<false, 128>(a, rot, dst_el, s);
  return bf16 ? launch_to<true, 64>(a, rot, dst_el, s) : launch_to<false, 64>(a, rot, dst_el, s);
}

}  // namespace ams
