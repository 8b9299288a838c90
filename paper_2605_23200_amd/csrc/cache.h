// Caches of 8 and 4 bits on the device: blocks, scales and codes (ams_cache in include/ams.h).
#ifndef AMS_CACHE_H
#define AMS_CACHE_H

#include <type_traits>

#include "ams_internal.h"

namespace ams {

constexpr int kBlockRows = 16;  // positions that share a scale (in 4 bits: whose scales lie together); a page of the paged layout

// Element types as the kernels are instantiated for them.
enum { EL_F32 = AMS_F32, EL_BF16 = AMS_BF16, EL_INT8 = AMS_INT8, EL_E4M3 = AMS_E4M3, EL_E2M1 = AMS_E2M1 };
template <int EL>
constexpr bool kPacked = EL == EL_INT8 || EL == EL_E4M3;  // 8 bits, a scale per block
template <int EL>
constexpr bool kMicro = EL == EL_E2M1;                    // 4 bits, a scale per 32 channels of a row
template <int EL>
constexpr bool kCodes = kPacked<EL> || kMicro<EL>;
template <int EL>
constexpr int kElBytes = EL == EL_F32 ? 4 : EL == EL_BF16 ? 2 : 1;
template <int EL>
constexpr int kEightBytes = kMicro<EL> ? 4 : 8 * kElBytes<EL>;  // of eight elements

// Scales of 4 bits: bytes, those of a block together, its 16 positions for every 32 channels.
constexpr int kMicroChannels = 32;
template <int HD>
constexpr int kMicroBytes = HD / kMicroChannels * kBlockRows;
template <int HD>
__device__ __forceinline__ uint32_t micro_at(int channel, int row) { return channel / kMicroChannels * kBlockRows + row; }

// One of K / V of a cache.
struct CacheDev {
  char* base;
  float* scale;  // null for rows of kv_dtype; bytes in 4 bits
  const int32_t* table;
  int64_t t_capacity;  // dense: rows per unit
  int64_t n_pages;     // paged: pages per layer
  int64_t n_slots;     // paged: rows per layer
  int32_t max_blocks;
  int32_t B, H, row_bytes;
  int32_t paged;
};

// The block of a unit that holds positions 16 blk .. 16 blk + 15.
struct Block {
  char* row0;
  int64_t stride;  // bytes from row to row
  int64_t scale;   // index of its scale
  bool there;      // false: the block table names no page of the pool (row0 is then the nearest page's)
};
__device__ __forceinline__ Block block_at(const CacheDev& c, int l, int b, int h, int blk) {
  Block r;
  if (!c.paged) {
    const int64_t unit = ((int64_t)l * c.B + b) * c.H + h;
    r.row0 = c.base + (unit * c.t_capacity + (int64_t)blk * kBlockRows) * c.row_bytes;
    r.stride = c.row_bytes;
    r.scale = unit * ((c.t_capacity + kBlockRows - 1) / kBlockRows) + blk;
    r.there = true;
    return r;
  }
  const int64_t named = c.table[(int64_t)b * c.max_blocks + blk];
  r.there = named >= 0 && named < c.n_pages;
  const int64_t page = r.there ? named : (named < 0 ? 0 : c.n_pages - 1);
  r.row0 = c.base + (((int64_t)l * c.n_slots + page * kBlockRows) * c.H + h) * c.row_bytes;
  r.stride = (int64_t)c.H * c.row_bytes;
  r.scale = ((int64_t)l * c.n_pages + page) * c.H + h;
  return r;
}

// blockIdx.x, from `first` on, of a (stretch of positions, unit) grid, turned from unit to unit.  Workgroups go to the eight dies in turn: where gridDim.x
// and eight share a factor, the last stretches of all units, which short sequences of a batch leave empty, would fall to the same
// dies.  (ams_attend, 512 units of 4096 to 16384 positions: 348 us without, 321 so; 320 of 1000 to 16384, 128 queries: 884 and 620;
// ams_recode, 1024 ragged units of up to 2048: 396 and 313.)
__device__ __forceinline__ int turned_x(int first = 0) {
  const uint32_t y = blockIdx.y;
  return (int)((blockIdx.x - first + y + (y >> 1) + (y >> 2)) % (gridDim.x - first));
}

// Largest magnitude of a code.
template <int EL>
constexpr float kMostCode = EL == EL_INT8 ? 127.f : 448.f;

// Scale of a block from the bits of its largest magnitude: the least power of two that takes it to kMostCode or less.
// 127 = 1.984375 * 2^6, 448 = 1.75 * 2^8: the mantissa says whether the exponent below suffices.
template <int EL>
__device__ __forceinline__ float block_scale(uint32_t top) {
  if (top == 0) return 0.f;
  if (top >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
  constexpr uint32_t kMantissa = EL == EL_INT8 ? 0x7E0000u : 0x600000u;
  constexpr int kShift = EL == EL_INT8 ? 6 : 8;
  const int e = (int)(top >> 23) - 127 - kShift + ((top & 0x7FFFFFu) > kMantissa);  // subnormal: -127 - kShift, below the least
  return __uint_as_float((uint32_t)(max(e, -120) + 127) << 23);
}
// 1 / scale (exact for powers of two); 0 where the codes are 0 anyway.
__device__ __forceinline__ float scale_inverse(float scale) { return scale >= 0x1p-120f ? 1.f / scale : 0.f; }

// Four values already divided by their scale -> four codes, nearest, ties to even.
template <int EL>
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  constexpr float M = kMostCode<EL>;
  a = fminf(fmaxf(a, -M), M), b = fminf(fmaxf(b, -M), M), c = fminf(fmaxf(c, -M), M), d = fminf(fmaxf(d, -M), M);
  if constexpr (EL == EL_INT8) {
    const int x = (int)rintf(a), y = (int)rintf(b), z = (int)rintf(c), w = (int)rintf(d);
    return (uint32_t)(x & 255) | (uint32_t)(y & 255) << 8 | (uint32_t)(z & 255) << 16 | (uint32_t)w << 24;
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  }
}
template <int EL>
__device__ __forceinline__ void unpack_codes(uint32_t w, float (&x)[4]) {
  if constexpr (EL == EL_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
  }
}

// Scale byte of 32 channels of 4 bits from the bits of their largest magnitude: the least power of two that takes it to 7 = 1.75 * 2^2 or
// less.  (7 and not 6, the largest code: between 6 and 7 a value is as near to 6 as others of that binade may be to their codes.)
__device__ __forceinline__ uint32_t micro_scale(uint32_t top) {
  if (top == 0) return 0;
  if (top >= 0x7F800000u) return 255;
  return (uint32_t)(max((int)(top >> 23) - 127 - 2 + ((top & 0x7FFFFFu) > 0x600000u), -120) + 127);
}
__device__ __forceinline__ float micro_inverse(uint32_t byte) {  // 0 where the codes are 0 anyway
  return byte == 0 || byte == 255 ? 0.f : __uint_as_float((254 - byte) << 23);
}
// Four values, and eight, already divided by their scale -> codes, nearest, ties to even, 6 at most.
__device__ __forceinline__ uint32_t pack_four_bits(float a, float b, float c, float d) {
  const uint32_t lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, 1.f, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, c, d, 1.f, 1);
}
__device__ __forceinline__ uint32_t pack_eight_micro(const float (&x)[8], float inverse) {
  if (inverse == 0.f) return 0u;
  return pack_four_bits(x[0] * inverse, x[1] * inverse, x[2] * inverse, x[3] * inverse) |
         pack_four_bits(x[4] * inverse, x[5] * inverse, x[6] * inverse, x[7] * inverse) << 16;
}
// Eight codes as the values that they stand for.
__device__ __forceinline__ void unpack_micro(uint32_t w, uint32_t byte, float (&x)[8]) {
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  const float scale = __uint_as_float(byte << 23);
  const floatx2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const floatx2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {  // nearest, ties to even
  typedef float floatx2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((floatx2){a, b}, bf16x2));
}

// Eight consecutive elements of a row, as values (codes: not yet times their scale).
template <int EL>
__device__ __forceinline__ void load_eight(const char* at, float (&x)[8]) {
  if constexpr (EL == EL_F32) {
    const float4 a = *(const float4*)at, b = *(const float4*)(at + 16);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  } else if constexpr (EL == EL_BF16) {
    const uint4 a = *(const uint4*)at;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) x[2 * i] = __uint_as_float(w[i] << 16), x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  } else {
    const uint2 a = *(const uint2*)at;
    float lo[4], hi[4];
    unpack_codes<EL>(a.x, lo);
    unpack_codes<EL>(a.y, hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lo[i], x[4 + i] = hi[i];
  }
}
// Eight values of a row of kv_dtype.
template <int EL>
__device__ __forceinline__ void store_eight(char* at, const float (&x)[8]) {
  static_assert(!kPacked<EL>, "rows of kv_dtype");
  if constexpr (EL == EL_F32) {
    *(float4*)at = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(at + 16) = make_float4(x[4], x[5], x[6], x[7]);
  } else {
    *(uint4*)at = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
  }
}
template <int EL>
__device__ __forceinline__ uint2 pack_eight(const float (&x)[8], float inverse) {
  if (inverse == 0.f) return make_uint2(0u, 0u);  // a scale of 0 or NaN
  return make_uint2(pack_codes<EL>(x[0] * inverse, x[1] * inverse, x[2] * inverse, x[3] * inverse),
                    pack_codes<EL>(x[4] * inverse, x[5] * inverse, x[6] * inverse, x[7] * inverse));
}
__device__ __forceinline__ uint32_t top_bits(const float (&x)[8], uint32_t top) {
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  return top;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
  return x;
}

// Where scratch of ams_attend lies.
struct AttendLayout {
  size_t part, stats, joined, stash, total;  // outputs and statistics of the splits, logits
  int chunk, n_splits, row_tiles, row_waves, row_groups;
  bool stashed;  // the logits are kept for the weights
  bool pairs;    // of heads (4 bits)
};

// ---- launchers ----
struct AppendArgs {
  Dims d;
  const char *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // bytes
  const char *q_weight, *k_weight;
  float eps;
  const int32_t *positions, *seq_lens;
  int n_new;
  char* q_out;
  CacheDev kd, vd;
  int32_t* lens_out;
};
hipError_t launch_append(const AppendArgs& a, const ams_rope* rope, bool bf16, int dst_el, hipStream_t s);

struct AttendArgs {
  Dims d;
  CacheDev k, v;
  const int32_t* seq_lens;
  const char* q;
  char* out;
  float* lse;
  const float* weights_in;
  float* weights_out;
  int causal;
  float* part;    // [units, splits, N, D]
  float2* stats;  // [units, N, splits]: largest logit (log2), sum
  float2* joined; // [units, N], where the weights come from K again
  float* stash;   // [units, blocks, N, 16]
  int chunk, n_splits, row_waves;
};
AttendLayout attend_layout(const ams_params* p, bool pairs);
hipError_t launch_attend(const AttendArgs& a, const AttendLayout& lay, bool bf16, int el, hipStream_t s);
hipError_t launch_attend_e2m1(const AttendArgs& a, const AttendLayout& lay, bool bf16, hipStream_t s);
void launch_attend_join(const AttendArgs& a, const AttendLayout& lay, bool bf16, hipStream_t s);

struct RecodeArgs {
  Dims d;
  CacheDev ks, vs, kd, vd;
  const int32_t *seq_lens, *idx, *n_kept;
  int budget;
  const float* credit_src;
  float* credit_dst;
  int64_t credit_dst_stride;
};
hipError_t launch_recode(const RecodeArgs& a, int src_el, int dst_el, hipStream_t s);

struct EvictArgs {
  Dims d;
  const int32_t* seq_lens;
  const float* weights;
  float* weights_out;
  int32_t *idx, *n_kept, *lens_out;
  int budget, n_sink, n_last;
};
struct PagesArgs {
  int batch, t_max, max_blocks, n_pages;
  const int32_t *from, *to, *table;
  int32_t *table_out, *ring;
  const int32_t* state;
  int32_t *state_out, *lens_out, *starts;
  int64_t *slots, n_slots;
};
hipError_t launch_pages(const PagesArgs& a, hipStream_t s);

size_t evict_ws_bytes(const ams_params* p);
hipError_t launch_evict_pick(const EvictArgs& a, char* ws, hipStream_t s);

}  // namespace ams
#endif
