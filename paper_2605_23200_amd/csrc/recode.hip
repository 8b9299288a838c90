// Gather of cache rows between element types (ams_recode, ams_evict): rows of kv_dtype to 8 bits, 8 bits to rows, 8 bits to 8 bits, and
// (ams_evict) rows of kv_dtype as they are.
// value = code * scale of its block of 16 positions; a destination block takes the scale of the largest magnitude of ITS 16
// rows, so a block is the unit of work: one wave holds all of it in registers (eight elements per lane and row: 16 lanes a
// row of 128 channels, four rows a load), reduces the largest magnitude over its lanes and writes codes and scale.  Every byte
// moves once; no LDS, no barrier.  Memory is the bound: what a gathered row waits for (index, page, then scale and row) is a
// chain of latencies, so a wave starts all rows of K and V of its block before it looks at the first: 256 units, 2048 of
// 2176 rows, 8 bits to 8 bits: 94 us with a wave for K and one for V that loaded row by row, 52 so (5.2 TB/s); 2048 of 32768 bf16 rows
// to 8 bits: 96 and 83 (4.9 TB/s); 96 paged units, rows of 128 bytes scattered over a pool: 52 (3.9 TB/s).  Rows of kv_dtype as they
// are: an eviction of 256 units to 2048 of 32768 takes 162 us, with a copy that went row by row 164.
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// Eight elements as they lie in memory.
template <int EL>
struct Raw {
  uint32_t w[EL == EL_F32 ? 8 : EL == EL_BF16 ? 4 : 2];
  __device__ __forceinline__ void load(const char* at) {
    if constexpr (kPacked<EL>) {
      const uint2 a = *(const uint2*)at;
      w[0] = a.x, w[1] = a.y;
    } else {
      const uint4 a = *(const uint4*)at;
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
      if constexpr (EL == EL_F32) {
        const uint4 b = *(const uint4*)(at + 16);
        w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
      }
    }
  }
  __device__ __forceinline__ void store(char* at, bool real) const {  // zeros where it is not
    static_assert(!kPacked<EL>, "rows of kv_dtype");
#pragma unroll
    for (int i = 0; i < (EL == EL_F32 ? 8 : 4); i += 4)
      *(uint4*)(at + 4 * i) = real ? make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]) : make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void values(float (&x)[8]) const {
    if constexpr (EL == EL_F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
    } else if constexpr (EL == EL_BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    } else {
      float lo[4], hi[4];
      unpack_codes<EL>(w[0], lo);
      unpack_codes<EL>(w[1], hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
    }
  }
};

template <int SRC, int DST, int HD>
__global__ __launch_bounds__(kThreads) void recode_kernel(RecodeArgs a) {
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, PASSES = kBlockRows / ROWS;
  const int unit = blockIdx.y;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int blk = turned_x() * kWaves + wave;
  const int n = a.idx ? min(a.n_kept[unit], min(a.budget, a.d.t_max)) : seq_len(a.d, a.seq_lens, b);
  if (blk * kBlockRows >= n) return;
  const int32_t* idx = a.idx ? a.idx + (int64_t)unit * a.budget : nullptr;
  const int i = lane % LANES, r0 = lane / LANES;
  int t[PASSES];
  bool real[PASSES];  // false: a row of zeros (an index outside the cache), or none
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int j = min(blk * kBlockRows + p * ROWS + r0, n - 1);
    t[p] = idx ? idx[j] : j;
  }
  if (idx && a.credit_src && a.credit_dst && lane < kBlockRows) {
    const int j = blk * kBlockRows + lane, from = j < n ? idx[j] : -1;
    if (from >= 0 && from < a.d.t_max)
      a.credit_dst[(int64_t)unit * a.credit_dst_stride + j] = a.credit_src[(int64_t)unit * a.d.t_stride + from];
  }
  Raw<SRC> raw[2][PASSES];
  float scale[2][PASSES];
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    real[p] = t[p] >= 0 && t[p] < a.d.t_max;
    const int from = real[p] ? t[p] : 0;
    const Block s = block_at(a.ks, l, b, h, from / kBlockRows);  // V lies in the same places
    const int64_t at = (s.row0 - a.ks.base) + (from % kBlockRows) * s.stride + i * 8 * kElBytes<SRC>;
    raw[0][p].load(a.ks.base + at);
    raw[1][p].load(a.vs.base + at);
    scale[0][p] = kPacked<SRC> ? a.ks.scale[s.scale] : 1.f;
    scale[1][p] = kPacked<SRC> ? a.vs.scale[s.scale] : 1.f;
  }
  const Block to = block_at(a.kd, l, b, h, blk);
  if (!to.there) return;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const CacheDev& dst = kv ? a.vd : a.kd;
    char* rows = dst.base + (to.row0 - a.kd.base) + i * 8 * kElBytes<DST>;
    if constexpr (SRC == DST && !kPacked<DST>) {  // as they are
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * ROWS + r0;
        if (blk * kBlockRows + r < n) raw[kv][p].store(rows + r * to.stride, real[p]);
      }
      continue;
    }
    float x[PASSES][8];
    uint32_t top = 0;
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      raw[kv][p].values(x[p]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (kPacked<SRC>) x[p][e] *= scale[kv][p];
        if (!real[p]) x[p][e] = 0.f;
      }
      if constexpr (kPacked<DST>) top = top_bits(x[p], top);
    }
    float inverse = 1.f;
    if constexpr (kPacked<DST>) {
      const float s = block_scale<DST>(wave_max(top));  // (the last row stands in for those behind it)
      inverse = scale_inverse(s);
      if (lane == 0) dst.scale[to.scale] = s;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * ROWS + r0;
      if (blk * kBlockRows + r >= n) continue;
      if constexpr (kPacked<DST>)
        *(uint2*)(rows + r * to.stride) = pack_eight<DST>(x[p], inverse);
      else
        store_eight<DST>(rows + r * to.stride, x[p]);
    }
  }
}

template <int SRC, int DST>
hipError_t launch(const RecodeArgs& a, hipStream_t s) {
  const int rows = a.idx ? min(a.budget, a.d.t_max) : a.d.t_max;
  const dim3 grid(div_up(rows, kBlockRows * kWaves), a.d.units);
  prof_mark("recode", s);
  if (a.d.D == 128)
    hipLaunchKernelGGL((recode_kernel<SRC, DST, 128>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((recode_kernel<SRC, DST, 64>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

template <int SRC>
hipError_t launch_to(const RecodeArgs& a, int dst_el, hipStream_t s) {
  switch (dst_el) {
    case EL_INT8: return launch<SRC, EL_INT8>(a, s);
    case EL_E4M3: return launch<SRC, EL_E4M3>(a, s);
    case EL_BF16:
      if constexpr (kPacked<SRC> || SRC == EL_BF16) return launch<SRC, EL_BF16>(a, s);
      break;
    case EL_F32:
      if constexpr (kPacked<SRC> || SRC == EL_F32) return launch<SRC, EL_F32>(a, s);
      break;
  }
  return hipErrorNotSupported;
}

}  // namespace

hipError_t launch_recode(const RecodeArgs& a, int src_el, int dst_el, hipStream_t s) {
  switch (src_el) {
    case EL_F32: return launch_to<EL_F32>(a, dst_el, s);
    case EL_BF16: return launch_to<EL_BF16>(a, dst_el, s);
    case EL_INT8: return launch_to<EL_INT8>(a, dst_el, s);
    default: return launch_to<EL_E4M3>(a, dst_el, s);
  }
}

}  // namespace ams
