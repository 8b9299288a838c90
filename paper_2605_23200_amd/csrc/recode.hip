// Gather of cache rows between element types (ams_recode, ams_evict): rows of kv_dtype to 8 or 4 bits, these to rows and among themselves, and
// (ams_evict) rows of kv_dtype as they are.
// value = code * scale of its block of 16 positions; a destination block takes the scale of the largest magnitude of ITS 16
// rows, so a block is the unit of work: one wave holds all of it in registers (eight elements per lane and row: 16 lanes a
// row of 128 channels, four rows a load), reduces the largest magnitude over its lanes and writes codes and scale.  Every byte
// moves once; no LDS, no barrier.  Memory is the bound: what a gathered row waits for (index, page, then scale and row) is a
// chain of latencies, so a wave starts all rows of K and V of its block before it looks at the first: 256 units, 2048 of
// 2176 rows, 8 bits to 8 bits: 94 us with a wave for K and one for V that loaded row by row, 52 so (5.2 TB/s); 2048 of 32768 bf16 rows
// to 8 bits: 96 and 83 (4.9 TB/s); 96 paged units, rows of 128 bytes scattered over a pool: 52 (3.9 TB/s).  Rows of kv_dtype as they
// are: an eviction of 256 units to 2048 of 32768 takes 162 us, with a copy that went row by row 164.
// 4 bits: a scale for every 32 channels of a row, which are four lanes; no two rows have anything in common.  2048 of 32768 bf16 rows, 256
// units: 95 us, and 60 back to rows, 680 MB in all at 4.4 TB/s (92 with a conversion that does nothing, 47 without its stores: while it
// reads, the memory-side cache writes back what the kernel before it wrote).  Four or five waves on a SIMD instead of eight win 3 % of that and
// lose 2 % with whole slabs.  4 bits to 4 bits, 2048 of up to 16384 rows of 64 bytes scattered over a pool, 159 MB: 40 us (4.0 TB/s) where the caches hold
// nothing that waits to be written, 45 after its own last pass, 63 after a kernel that wrote 268 MB of bf16 rows (an eviction that is read back).
// (One, two and four rows a lane in flight: 151, 153 and 157 us for the eviction and its reading back.)
#include "cache.h"

namespace ams {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

// Eight elements as they lie in memory.
template <int EL>
struct Raw {
  uint32_t w[kEightBytes<EL> / 4];
  __device__ __forceinline__ void load(const char* at) {
    if constexpr (kMicro<EL>) {
      w[0] = *(const uint32_t*)at;
    } else if constexpr (kPacked<EL>) {
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
    static_assert(!kCodes<EL>, "rows of kv_dtype");
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
    } else if constexpr (kPacked<EL>) {
      float lo[4], hi[4];
      unpack_codes<EL>(w[0], lo);
      unpack_codes<EL>(w[1], hi);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
    }
  }
};

// Over four lanes in a row.
__device__ __forceinline__ uint32_t four_max(uint32_t x) {
  x = max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0x4E, 0xF, 0xF, true));        // i ^ 2
  return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, 0xB1, 0xF, 0xF, true));     // i ^ 1
}

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
  std::conditional_t<kMicro<SRC>, uint32_t, float> scale[2][PASSES];  // in 4 bits the byte of the lane's channels
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    real[p] = t[p] >= 0 && t[p] < a.d.t_max;
    const int from = real[p] ? t[p] : 0;
    const Block s = block_at(a.ks, l, b, h, from / kBlockRows);  // V lies in the same places
    const int64_t at = (s.row0 - a.ks.base) + (from % kBlockRows) * s.stride + i * kEightBytes<SRC>;
    raw[0][p].load(a.ks.base + at);
    raw[1][p].load(a.vs.base + at);
    if constexpr (kMicro<SRC>) {
      const int64_t byte = s.scale * kMicroBytes<HD> + micro_at<HD>(8 * i, from % kBlockRows);
      scale[0][p] = ((const uint8_t*)a.ks.scale)[byte], scale[1][p] = ((const uint8_t*)a.vs.scale)[byte];
    } else {
      scale[0][p] = kPacked<SRC> ? a.ks.scale[s.scale] : 1.f;
      scale[1][p] = kPacked<SRC> ? a.vs.scale[s.scale] : 1.f;
    }
  }
  const Block to = block_at(a.kd, l, b, h, blk);
  if (!to.there) return;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const CacheDev& dst = kv ? a.vd : a.kd;
    char* rows = dst.base + (to.row0 - a.kd.base) + i * kEightBytes<DST>;
    if constexpr (SRC == DST && !kCodes<DST>) {  // as they are
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
      if constexpr (kMicro<SRC>)
        unpack_micro(raw[kv][p].w[0], scale[kv][p], x[p]);
      else
        raw[kv][p].values(x[p]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if constexpr (kPacked<SRC>) x[p][e] *= scale[kv][p];
        if (!real[p]) x[p][e] = 0.f;
      }
      if constexpr (kPacked<DST>) top = top_bits(x[p], top);
    }
    if constexpr (kMicro<DST>) {  // a scale for the four lanes of 32 channels
#pragma unroll
      for (int p = 0; p < PASSES; ++p) {
        const int r = p * ROWS + r0;
        const uint32_t byte = micro_scale(four_max(top_bits(x[p], 0)));
        if (blk * kBlockRows + r >= n) continue;
        *(uint32_t*)(rows + r * to.stride) = pack_eight_micro(x[p], micro_inverse(byte));
        if (i % 4 == 0) ((uint8_t*)dst.scale)[to.scale * kMicroBytes<HD> + micro_at<HD>(8 * i, r)] = (uint8_t)byte;
      }
      continue;
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
      else if constexpr (!kMicro<DST>)
        store_eight<DST>(rows + r * to.stride, x[p]);
    }
  }
}

// Rows of 4 bits to rows of 4 bits, as they are: a lane holds 16 bytes of a row, which are of one scale, and starts its loads of K and V
// before it looks at the first.
template <int HD>
__global__ __launch_bounds__(kThreads) void move_kernel(RecodeArgs a) {
  constexpr int LANES = HD / 32, ROWS = 64 / LANES;
  const int unit = blockIdx.y;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int first = (turned_x() * kWaves + wave) * ROWS;
  const int n = a.idx ? min(a.n_kept[unit], min(a.budget, a.d.t_max)) : seq_len(a.d, a.seq_lens, b);
  if (first >= n) return;
  const int32_t* idx = a.idx ? a.idx + (int64_t)unit * a.budget : nullptr;
  const int i = lane % LANES, j = first + lane / LANES, row = min(j, n - 1);
  const int t = idx ? idx[row] : row;
  const bool real = t >= 0 && t < a.d.t_max;  // else a row of zeros
  const int from = real ? t : 0;
  if (idx && a.credit_src && a.credit_dst && i == 0 && j < n && real)
    a.credit_dst[(int64_t)unit * a.credit_dst_stride + j] = a.credit_src[(int64_t)unit * a.d.t_stride + t];
  const Block s = block_at(a.ks, l, b, h, from / kBlockRows);
  const int64_t at = (s.row0 - a.ks.base) + (from % kBlockRows) * s.stride + i * 16;
  const int64_t at_scale = s.scale * kMicroBytes<HD> + micro_at<HD>(32 * i, from % kBlockRows);
  uint4 k = *(const uint4*)(a.ks.base + at), v = *(const uint4*)(a.vs.base + at);
  uint8_t k_scale = ((const uint8_t*)a.ks.scale)[at_scale], v_scale = ((const uint8_t*)a.vs.scale)[at_scale];
  const Block to = block_at(a.kd, l, b, h, row / kBlockRows);
  if (!to.there || j >= n) return;
  if (!real) k = v = make_uint4(0u, 0u, 0u, 0u), k_scale = v_scale = 0;
  const int64_t put = (to.row0 - a.kd.base) + (j % kBlockRows) * to.stride + i * 16;
  const int64_t put_scale = to.scale * kMicroBytes<HD> + micro_at<HD>(32 * i, j % kBlockRows);
  *(uint4*)(a.kd.base + put) = k, *(uint4*)(a.vd.base + put) = v;
  ((uint8_t*)a.kd.scale)[put_scale] = k_scale, ((uint8_t*)a.vd.scale)[put_scale] = v_scale;
}

template <int SRC, int DST>
hipError_t launch(const RecodeArgs& a, hipStream_t s) {
  const int rows = a.idx ? min(a.budget, a.d.t_max) : a.d.t_max;
  const dim3 grid(div_up(rows, kBlockRows * kWaves), a.d.units);
  prof_mark("recode", s);
  if constexpr (kMicro<SRC> && kMicro<DST>) {
    if (a.d.D == 128)
      hipLaunchKernelGGL((move_kernel<128>), dim3(div_up(rows, 16 * kWaves), a.d.units), dim3(kThreads), 0, s, a);
    else
      hipLaunchKernelGGL((move_kernel<64>), dim3(div_up(rows, 32 * kWaves), a.d.units), dim3(kThreads), 0, s, a);
  } else if (a.d.D == 128) {
    hipLaunchKernelGGL((recode_kernel<SRC, DST, 128>), grid, dim3(kThreads), 0, s, a);
  } else {
    hipLaunchKernelGGL((recode_kernel<SRC, DST, 64>), grid, dim3(kThreads), 0, s, a);
  }
  return hipGetLastError();
}

template <int SRC>
hipError_t launch_to(const RecodeArgs& a, int dst_el, hipStream_t s) {
  switch (dst_el) {
    case EL_INT8: return launch<SRC, EL_INT8>(a, s);
    case EL_E4M3: return launch<SRC, EL_E4M3>(a, s);
    case EL_E2M1: return launch<SRC, EL_E2M1>(a, s);
    case EL_BF16:
      if constexpr (kCodes<SRC> || SRC == EL_BF16) return launch<SRC, EL_BF16>(a, s);
      break;
    case EL_F32:
      if constexpr (kCodes<SRC> || SRC == EL_F32) return launch<SRC, EL_F32>(a, s);
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
    case EL_E4M3: return launch_to<EL_E4M3>(a, dst_el, s);
    default: return launch_to<EL_E2M1>(a, dst_el, s);
  }
}

}  // namespace ams
