// Gather of cache rows between element types (ams_recode): rows of kv_dtype to 8 bits, 8 bits to rows, 8 bits to 8 bits.
// value = code * scale of its block of 16 positions; a destination block takes the scale of the largest magnitude of ITS 16
// rows, so a block is the unit of work: one wave holds all of it in registers (eight elements per lane and row: 16 lanes a
// row of 128 channels, four rows a load), reduces the largest magnitude over its lanes and writes codes and scale.  Every byte
// moves once; no LDS, no barrier.  Memory is the bound.
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

template <int SRC, int DST, int HD>
__global__ __launch_bounds__(kThreads) void recode_kernel(RecodeArgs a) {
  constexpr int LANES = HD / 8, ROWS = 64 / LANES, PASSES = kBlockRows / ROWS;
  const int unit = blockIdx.y;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const bool values = wave & 1;
  const int blk = blockIdx.x * (kWaves / 2) + (wave >> 1);
  const int most = min(a.budget, a.d.t_max);
  const int n = a.idx ? min(a.n_kept[unit], most) : seq_len(a.d, a.seq_lens, b);
  if (blk * kBlockRows >= n) return;
  const CacheDev src = values ? a.vs : a.ks, dst = values ? a.vd : a.kd;
  const int32_t* idx = a.idx ? a.idx + (int64_t)unit * a.budget : nullptr;
  const int i = lane % LANES, r0 = lane / LANES;
  float x[PASSES][8];
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int j = blk * kBlockRows + p * ROWS + r0;
    int t = -1;
    if (j < n) t = idx ? idx[j] : j;
    if (t < 0 || t >= a.d.t_max) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[p][e] = 0.f;
      continue;
    }
    const Block s = block_at(src, l, b, h, t / kBlockRows);
    load_eight<SRC>(s.row0 + (t % kBlockRows) * s.stride + i * 8 * kElBytes<SRC>, x[p]);
    if constexpr (kPacked<SRC>) {
      const float scale = src.scale[s.scale];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[p][e] *= scale;
    }
  }
  const Block to = block_at(dst, l, b, h, blk);
  if (to.there) {
    float inverse = 1.f;
    if constexpr (kPacked<DST>) {
#pragma unroll
      for (int p = 0; p < PASSES; ++p) top = top_bits(x[p], top);
      const float scale = block_scale<DST>(wave_max(top));
      inverse = scale_inverse(scale);
      if (lane == 0) dst.scale[to.scale] = scale;
    }
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
      const int r = p * ROWS + r0;
      if (blk * kBlockRows + r >= n) continue;
      char* row = to.row0 + r * to.stride + i * 8 * kElBytes<DST>;
      if constexpr (kPacked<DST>)
        *(uint2*)row = pack_eight<DST>(x[p], inverse);
      else
        store_eight<DST>(row, x[p]);
    }
  }
  if (!values && idx && a.credit_src && a.credit_dst && lane < kBlockRows) {
    const int j = blk * kBlockRows + lane;
    if (j < n && idx[j] >= 0 && idx[j] < a.d.t_max)
      a.credit_dst[(int64_t)unit * a.credit_dst_stride + j] = a.credit_src[(int64_t)unit * a.d.t_stride + idx[j]];
  }
}

template <int SRC, int DST>
hipError_t launch(const RecodeArgs& a, hipStream_t s) {
  const int rows = a.idx ? min(a.budget, a.d.t_max) : a.d.t_max;
  const dim3 grid(div_up(rows, kBlockRows * (kWaves / 2)), a.d.units);
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
      if constexpr (kPacked<SRC>) return launch<SRC, EL_BF16>(a, s);
      break;
    case EL_F32:
      if constexpr (kPacked<SRC>) return launch<SRC, EL_F32>(a, s);
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
