// Attention over a cache of 8 or 4 bits (ams_attend): the kernels of one head.  (Joins and layouts: attend.hip; two heads a wave: attend_e2m1.hip.)
//
// One wave takes 32 positions at a time: K as 16x16x32 tiles with the positions as rows and the queries as columns,
// S^T = K Q^T, so that a lane ends with 2 x 4 logits of ONE query (column lane % 16) at positions 4 (lane / 16) + 0..3 of both
// tiles.  That is already the layout in which the second product, O^T = V^T P^T over the same 32 positions, wants P (its k index
// runs over the positions in any order both operands share), so probabilities never leave the lane.  V is read as bytes of
// 8 positions per lane and turned there: one v_perm per two elements, which the conversion to bf16 needs anyway.  Codes are bf16
// numbers, so q.k has exact products; the scales of the two blocks of 16 positions go to the logits and to the probabilities.
// P goes in as two bf16 terms: one (2^-9) would be an error as large as the rounding of the output, fp16 would lose what a block of
// small values under another of large ones contributes; the second product has room, the kernel is bound by memory.
// Softmax: a running reference per query that is moved (and O rescaled) only when a logit exceeds it by 2^8; P and the
// sums are then at most 2^8 per position, far inside bf16's and fp32's range.
// No LDS until the waves of a workgroup (which take the steps of their split in turn) join their sums, in fixed order.
// The splits of a long axis are joined by attend_join_kernel, again in fixed order.
// What bounds it: the bytes of K and V.  512 paged units of 4096 to 16384 positions: 288 us, 5.1 TB/s with the logits it writes (without
// weights, 256 dense units of 16384: 5.5 TB/s); 4 units of 131072: 33 us of 28 at the rate of a copy.  It reads that fast because
// tables and scales come through the scalar cache, a name of a page two steps before its codes (vector loads of them: 507 us), and
// because no load is under a condition.  More than 32 queries are bound by what follows from one another within a step: 436 vector
// instructions and 48 products for 32 positions and 32 queries, 44 us for 8 units of 32768 positions and 128 queries, in which the
// vector ALU is active for 51 % and the matrix cores for 21 %.  (Sharing the conversions of four waves through
// LDS: 52; the masks as a variant of the step: 44, but 128 against 120 for 64 units and 32 queries.)
//
// Codes of 4 bits: a quarter of a row of K is of one scale and in one lane, a conversion of two codes multiplies by the scale as well, and the
// values are bf16 numbers, so that logits and probabilities need no factors; the rest is the same.  (Pairs of heads run in attend_e2m1.hip: up to 8
// queries, and 9 to 16 of bf16 over 128 channels in pages with positions enough; odd head counts, slabs of 2^24 rows and the other calls of 9 to 16
// queries run here, as all of more.)  64
// ragged sequences of up to 16384 positions and 14 queries a head in slabs: 306 us; 8 units of 32768 and 128 queries: 39 us (345 vector
// instructions for 32 positions and 32 queries, vector ALU active for 57 %, matrix cores for 28 %; with 64 queries a wave 54; with three waves on a SIMD,
// which spill 30 registers, a pass of 61 takes 67).  Not with the matrix cores' own scaled products of 4-bit by 8-bit floats, which take K's codes as they are: inside 32
// channels their sums lose what lies about 2^14 below the largest product (5e-4 of it for codes of any size, measured), and queries would have
// to go in as several terms of 4 bits.
//
// Weights: with up to 16 queries the logits go to scratch (4 N bytes a position, written and read once, against 2 D of K and V)
// and the join turns them into probabilities; beyond that K is read a second time (attend_weights_kernel).  In 4 bits the same: with K again
// for 9 to 16 queries 64 sequences of up to 16384 positions and 14 queries take 431 us against 365.
#ifndef AMS_ATTEND_KERNEL_H
#define AMS_ATTEND_KERNEL_H

#include "cache.h"
#include "score_tile.h"

namespace ams {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kStep = 32;                 // positions per wave and step
constexpr float kSlack = 8.f;             // log2 by which a logit may exceed the reference
constexpr float kLowest = -1e38f;         // reference before any logit
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// Two codes of 8 bits of a word, bytes 2 HALF and 2 HALF + 1, as bf16.
template <int EL, int HALF>
__device__ __forceinline__ uint32_t two_codes(uint32_t w) {
  if constexpr (EL == EL_INT8) {
    const float a = (float)(int8_t)(w >> (16 * HALF)), b = (float)(int8_t)(w >> (16 * HALF + 8));
    return high_halves(__float_as_uint(a), __float_as_uint(b));
  } else {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.f, HALF);
    return __builtin_bit_cast(uint32_t, c);
  }
}
// Two codes of 4 bits of a word, those of its byte `byte`, as bf16; their scale is 2^(x - 127), x the exponent bits of `scale`: 255 makes both no
// number, 0 is 2^-127.
__device__ __forceinline__ uint32_t two_of_four_bits(uint32_t w, float scale, int byte) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 c;
  switch (byte) {  // (the builtin takes a constant)
    case 0: c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0); break;
    case 1: c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1); break;
    case 2: c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2); break;
    default: c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  }
  return __builtin_bit_cast(uint32_t, c);
}
// Scale bytes of 253 and 254: codes under them may be infinite as bf16.
constexpr uint32_t kBeyond = 253u << 23;  // as the scale's bits
// Those of an operand as 0.  Queries of fp32 go in as three terms, of which the lower ones may be 0 or have the other sign: times an infinite
// key they would make a logit no number that the first term makes infinite.  (So products are formed in two ways, by whether a step holds such
// a scale: 8 units of 16384 and 128 queries 65.5 -> 66.2 us; up to 32 queries no difference.)
__device__ __forceinline__ bf16x8 without_infinite(bf16x8 x) {
  uint4 r = __builtin_bit_cast(uint4, x);
  asm volatile("" : "+v"(r.x), "+v"(r.y), "+v"(r.z), "+v"(r.w));  // (formed where it is used: kept over a loop it would take 64 registers)
  auto one = [](uint32_t w) __attribute__((always_inline)) {
    return w & ((w & 0x7FFFu) == 0x7F80u ? 0xFFFF0000u : 0xFFFFFFFFu) & ((w & 0x7FFF0000u) == 0x7F800000u ? 0xFFFFu : 0xFFFFFFFFu);
  };
  r = make_uint4(one(r.x), one(r.y), one(r.z), one(r.w));
  return __builtin_bit_cast(bf16x8, r);
}
// Eight codes -> the operand of one product.
template <int EL>
__device__ __forceinline__ bf16x8 eight_codes(uint32_t lo, uint32_t hi) {
  const uint4 r = make_uint4(two_codes<EL, 0>(lo), two_codes<EL, 1>(lo), two_codes<EL, 0>(hi), two_codes<EL, 1>(hi));
  return __builtin_bit_cast(bf16x8, r);
}
__device__ __forceinline__ bf16x8 eight_of_four_bits(uint32_t w, float scale) {
  const uint4 r = make_uint4(two_of_four_bits(w, scale, 0), two_of_four_bits(w, scale, 1), two_of_four_bits(w, scale, 2), two_of_four_bits(w, scale, 3));
  return __builtin_bit_cast(bf16x8, r);
}
// Word w[j] holds elements 0..3 of position j: the eight positions of element E.
template <int EL, int E>
__device__ __forceinline__ void turn_pair(const uint32_t (&w)[8], bf16x8& first, bf16x8& second) {  // elements 2 E, 2 E + 1
  uint32_t a[4], b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (EL == EL_INT8) {
      a[j] = high_halves(__float_as_uint((float)(int8_t)(w[2 * j] >> (16 * E))), __float_as_uint((float)(int8_t)(w[2 * j + 1] >> (16 * E))));
      b[j] = high_halves(__float_as_uint((float)(int8_t)(w[2 * j] >> (16 * E + 8))),
                         __float_as_uint((float)(int8_t)(w[2 * j + 1] >> (16 * E + 8))));
    } else {
      const uint32_t x = two_codes<EL, E>(w[2 * j]), y = two_codes<EL, E>(w[2 * j + 1]);
      a[j] = low_halves(x, y);
      b[j] = high_halves(x, y);
    }
  }
  first = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
  second = __builtin_bit_cast(bf16x8, make_uint4(b[0], b[1], b[2], b[3]));
}

// Word w[j] holds elements 0..7 of position j in 4 bits: the eight positions of elements 2 byte and 2 byte + 1, with their scales.
__device__ __forceinline__ void turn_pair(const uint32_t (&w)[8], const float (&scale)[8], int byte, bf16x8& first, bf16x8& second) {
  uint32_t a[4], b[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t x = two_of_four_bits(w[2 * j], scale[2 * j], byte), y = two_of_four_bits(w[2 * j + 1], scale[2 * j + 1], byte);
    a[j] = low_halves(x, y);
    b[j] = high_halves(x, y);
  }
  first = __builtin_bit_cast(bf16x8, make_uint4(a[0], a[1], a[2], a[3]));
  second = __builtin_bit_cast(bf16x8, make_uint4(b[0], b[1], b[2], b[3]));
}

// 2^x to an ulp; results below 2^-126 are 0, which no sum here notices.
__device__ __forceinline__ float power_of_two(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ floatx4 mma(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Over the four lanes that hold one query.
__device__ __forceinline__ float query_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float query_sum(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Over the sixteen lanes that hold one position's logits.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sixteen_sum(float x) {
  x += moved<0x140>(x);         // lane 15 - i of 16
  x += moved<0x141>(x);         // 7 - i of 8
  x += moved<0x4E>(x);          // i ^ 2
  return x + moved<0xB1>(x);    // i ^ 1
}

__device__ __forceinline__ float sixteen_max(float x) {
  x = fmaxf(x, moved<0x140>(x));
  x = fmaxf(x, moved<0x141>(x));
  x = fmaxf(x, moved<0x4E>(x));
  return fmaxf(x, moved<0xB1>(x));
}

// Channel of element 0 of the 8 that lane group g feeds to product i of q.k: 16 bytes of a K row per load; in 4 bits a lane has a
// quarter of the row, which is of one scale.
template <int EL, int HD>
__device__ __forceinline__ int k_channel(int i, int g) {
  if constexpr (kMicro<EL>) return HD / 4 * g + 8 * i;
  return 64 * (i >> 1) + 16 * g + 8 * (i & 1);
}

// The query operand of rows row0 + 16 r + lane % 16, as TERMS bf16 terms.
template <int EL, bool BF16, int HD, int R>
struct Queries {
  static constexpr int TERMS = BF16 ? 1 : 3, STEPS = HD / 32;
  bf16x8 x[R][STEPS][TERMS];
  __device__ __forceinline__ void load(const char* unit_q, int row0, int N, int lane) {
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int i = 0; i < STEPS; ++i) load_one(unit_q, row0 + r * 16 + (lane & 15), N, i, lane, x[r][i]);
  }
  static __device__ __forceinline__ void load_one(const char* unit_q, int n, int N, int i, int lane, bf16x8 (&out)[TERMS]) {
    const int d = k_channel<EL, HD>(i, lane >> 4);
    if constexpr (BF16) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (n < N) v = *(const uint4*)(unit_q + ((int64_t)n * HD + d) * 2);
      out[0] = __builtin_bit_cast(bf16x8, v);
    } else {
      float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
      if (n < N) load_eight<EL_F32>(unit_q + ((int64_t)n * HD + d) * 4, v);
      uint32_t t[3][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) split2<true>(v[2 * j], v[2 * j + 1], t[0][j], t[1][j], t[2][j]);
#pragma unroll
      for (int k = 0; k < 3; ++k) out[k] = __builtin_bit_cast(bf16x8, make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]));
    }
  }
};

// Loads of what this kernel does not write and every lane of the wave wants (a block table, scales; other launches write them): through the
// scalar cache.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// The blocks of one unit: slot of a block (the block itself, or its page), bytes and scales from slot to slot, the same for K and V.
template <int EL, int HD>
struct UnitBlocks {
  static constexpr int kScales = kMicro<EL> ? kMicroBytes<HD> : 4;  // bytes of a block's scales
  const char *k, *v, *k_scale, *v_scale;
  const int32_t* table;  // null: dense
  int64_t block_bytes, scale_step, n_pages;
  int row_stride;
  __device__ __forceinline__ UnitBlocks(const CacheDev& kc, const CacheDev& vc, int l, int b, int h) {
    const Block k0 = first(kc, l, b, h), v0 = first(vc, l, b, h);
    k = k0.row0, v = v0.row0, k_scale = (const char*)kc.scale + k0.scale * kScales, v_scale = (const char*)vc.scale + v0.scale * kScales;
    table = kc.paged ? kc.table + (int64_t)b * kc.max_blocks : nullptr;
    row_stride = (int)k0.stride;
    block_bytes = k0.stride * kBlockRows;
    scale_step = (kc.paged ? kc.H : 1) * kScales;
    n_pages = kc.n_pages;
  }
  static __device__ __forceinline__ Block first(const CacheDev& c, int l, int b, int h) {
    Block r;
    const int64_t unit = ((int64_t)l * c.B + b) * c.H + h;
    r.row0 = c.base + (c.paged ? (int64_t)l * c.n_slots * c.H + h : unit * c.t_capacity) * c.row_bytes;
    r.stride = c.paged ? (int64_t)c.H * c.row_bytes : c.row_bytes;
    r.scale = c.paged ? (int64_t)l * c.n_pages * c.H + h : unit * ((c.t_capacity + kBlockRows - 1) / kBlockRows);
    r.there = true;
    return r;
  }
  // The table's word, and the slot that it names: apart, so that the word can be on its way for a while.
  __device__ __forceinline__ int named(int blk) const { return table ? uniform_load(table + blk) : blk; }
  __device__ __forceinline__ int64_t slot(int name) const {
    if (!table) return name;
    return name < 0 ? 0 : name < n_pages ? name : n_pages - 1;
  }
};

// A lane's byte offsets in two blocks: row lane % 16 of K, rows 4 (lane / 16) + 0..3 of V.  Rows past the last position (of the
// sequence's last blocks) are that position again: what is behind it, in the cache or past its end, is not read.  In 4 bits also the
// offset of K's scale, and the bytes of V's scales (four positions a word) that are there: the others are read as 0.
template <int EL, int HD>
struct Offsets {
  uint32_t k[2], v[2][4], k_scale[2], v_there[2];
  __device__ __forceinline__ void set(int row_stride, int lane, int most0, int most1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int most = j ? most1 : most0;
      k[j] = (uint32_t)min(lane & 15, most) * row_stride + (lane >> 4) * (kMicro<EL> ? HD / 8 : 16);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[j][i] = (uint32_t)min((lane >> 4) * 4 + i, most) * row_stride + (lane & 15) * (kMicro<EL> ? HD / 32 : HD / 16);
      if constexpr (kMicro<EL>) {
        k_scale[j] = micro_at<HD>((lane >> 4) * (HD / 4), min(lane & 15, most));
        const int there = min(max(most + 1 - (lane >> 4) * 4, 0), 4);
        v_there[j] = there == 4 ? 0xFFFFFFFFu : (1u << 8 * there) - 1;
      }
    }
  }
};

// A block of K as the wave reads it: lane % 16 is the position, lane / 16 the 16 bytes of every 64 (in 4 bits the quarter of the row).
template <int EL, int HD>
struct KTile {
  static constexpr int WORDS = kMicro<EL> ? HD / 32 : HD / 16;
  uint32_t w[WORDS];
  float scale;  // in 4 bits part of the operands
  __device__ __forceinline__ void load(const UnitBlocks<EL, HD>& u, int64_t slot, uint32_t offset, uint32_t at_scale) {
    const char* scales = u.k_scale + slot * u.scale_step;
    const char* row = u.k + slot * u.block_bytes;
    if constexpr (kMicro<EL>) {
      if constexpr (WORDS == 4) {
        const uint4 x = *(const uint4*)(row + offset);
        w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
      } else {
        const uint2 x = *(const uint2*)(row + offset);
        w[0] = x.x, w[1] = x.y;
      }
      scale = __uint_as_float((uint32_t) * (const uint8_t*)(scales + at_scale) << 23);
    } else {
      scale = uniform_load((const float*)scales);
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) {
        const uint4 x = *(const uint4*)(row + offset + 64 * i);
        w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
      }
    }
  }
  __device__ __forceinline__ bf16x8 operand(int i) const {
    if constexpr (kMicro<EL>)
      return eight_of_four_bits(w[i], scale);
    else
      return eight_codes<EL>(w[2 * i], w[2 * i + 1]);
  }
  __device__ __forceinline__ float of_logits() const { return kMicro<EL> ? 1.f : scale; }
};

// Scale bytes of two times four positions as powers of two.
__device__ __forceinline__ void four_powers(const uint32_t (&scales)[2], float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t b = scales[j >> 2];
    const int up = 23 - 8 * (j & 3);
    x[j] = __uint_as_float((up >= 0 ? b << up : b >> -up) & 0x7F800000u);
  }
}

// Two blocks of V: lane % 16 is the stretch of HD / 16 channels, word [j] of position 4 (lane / 16) + j % 4 of block j / 4.
template <int EL, int HD>
struct VTile {
  static constexpr int WORDS = kMicro<EL> ? 1 : HD / 64;  // of 4 channels; in 4 bits of HD / 16
  uint32_t w[WORDS][8];
  float scale[2];     // of the blocks
  uint32_t scales[2]; // in 4 bits: bytes of the four positions
  __device__ __forceinline__ void load(const UnitBlocks<EL, HD>& u, int64_t slot0, int64_t slot1, const Offsets<EL, HD>& o, uint32_t at_scale) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t slot = j ? slot1 : slot0;
      const char* of_block = u.v_scale + slot * u.scale_step;
      if constexpr (kMicro<EL>)
        scales[j] = *(const uint32_t*)(of_block + at_scale);
      else
        scale[j] = uniform_load((const float*)of_block);
      const char* block = u.v + slot * u.block_bytes;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (kMicro<EL>) {
          if constexpr (HD == 128)
            w[0][4 * j + i] = *(const uint32_t*)(block + o.v[j][i]);
          else
            w[0][4 * j + i] = *(const uint16_t*)(block + o.v[j][i]);
        } else if constexpr (WORDS == 2) {
          const uint2 x = *(const uint2*)(block + o.v[j][i]);
          w[0][4 * j + i] = x.x, w[1][4 * j + i] = x.y;
        } else {
          w[0][4 * j + i] = *(const uint32_t*)(block + o.v[j][i]);
        }
      }
    }
  }
};

// Channels d0 .. d0 + HD / 16 - 1 of a query's sums over a split: the output where there is one split, else for the join.
template <bool BF16, int HD>
__device__ __forceinline__ void finish_query(const AttendArgs& a, int unit, int n, int split, float top, float all, const float (&x)[HD / 16], int d0) {
  const int N = a.d.N;
  const bool last = a.n_splits == 1;
  const int64_t row = ((int64_t)unit * a.n_splits + split) * N + n;
  if (threadIdx.x % 16 == 0) {
    a.stats[((int64_t)unit * N + n) * a.n_splits + split] = make_float2(top, all);
    if (last && a.lse) a.lse[(int64_t)unit * N + n] = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
  }
  if (last) {
    const float inverse = all == 0.f ? 0.f : 1.f / all;
    char* to = a.out + (((int64_t)unit * N + n) * HD + d0) * (BF16 ? 2 : 4);
#pragma unroll
    for (int e = 0; e < HD / 16; e += 4) {
      const float y0 = x[e] * inverse, y1 = x[e + 1] * inverse, y2 = x[e + 2] * inverse, y3 = x[e + 3] * inverse;
      if constexpr (BF16)
        *(uint2*)(to + 2 * e) = make_uint2(bf16_pair(y0, y1), bf16_pair(y2, y3));
      else
        *(float4*)(to + 4 * e) = make_float4(y0, y1, y2, y3);
    }
  } else {
#pragma unroll
    for (int e = 0; e < HD / 16; e += 4) *(float4*)&a.part[row * HD + d0 + e] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
  }
}

// One split of one unit's positions for 16 R row_waves of its queries: row_waves waves side by side take 16 R queries each, the others
// every (4 / row_waves)-th step of the positions.
template <int EL, bool BF16, int HD, int R>
__global__ __launch_bounds__(kThreads, R == 1 ? (BF16 || HD == 64 ? 3 : 2) : (BF16 || HD == 64 ? 2 : 1)) void attend_kernel(AttendArgs a) {
  constexpr int STEPS = HD / 32, TILES = HD / 16, TERMS = BF16 ? 1 : 3, PTERMS = BF16 ? 2 : 3;
  constexpr int LD = HD + 4;  // row of the join in LDS
  __shared__ __align__(16) float joint[kWaves][16][LD];
  __shared__ float2 stat[kWaves][16];
  const int unit = blockIdx.y, split = turned_x();
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15;
  const int row_waves = a.row_waves, key_waves = kWaves / row_waves, stride = key_waves * kStep;
  const int row0 = (blockIdx.z * row_waves + wave % row_waves) * 16 * R;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int T = seq_len(a.d, a.seq_lens, b), N = a.d.N;
  const int begin = split * a.chunk, end = min(T, begin + a.chunk);
  if (begin >= T && split > 0) return;  // the join knows; split 0 of an empty sequence writes the zeros
  Queries<EL, BF16, HD, R> q;
  q.load(a.q + (int64_t)unit * N * HD * (BF16 ? 2 : 4), row0, N, lane);
  int limit[R];  // positions that the lane's query sees
  int fewest = T;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int n = row0 + r * 16 + c;
    limit[r] = a.causal ? T - a.d.W + 1 + n % a.d.W : T;
    if (a.causal) fewest = T - a.d.W + 1;
  }
  floatx4 o[R][TILES];
  float m[R], sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = kLowest, sum[r] = 0.f;
#pragma unroll
    for (int e = 0; e < TILES; ++e) o[r][e] = floatx4{0.f, 0.f, 0.f, 0.f};
  }
  const float to_log2 = kLog2E / sqrtf((float)HD);
  const UnitBlocks<EL, HD> u(a.k, a.v, l, b, h);
  const int last_blk = (T - 1) / kBlockRows;
  Offsets<EL, HD> off;
  off.set(u.row_stride, lane, kBlockRows - 1, kBlockRows - 1);
  const uint32_t v_scale = micro_at<HD>(c * TILES, 4 * g);  // (in 4 bits)
  KTile<EL, HD> kt[2];
  VTile<EL, HD> vt;
  int name[2] = {0, 0};
  int64_t slot[2] = {0, 0};
  // names of the step's two blocks; its offsets where it holds the sequence's end (the wave's last step)
  auto find = [&](int at) __attribute__((always_inline)) {
    name[0] = u.named(min(at / kBlockRows, last_blk));
    name[1] = u.named(min(at / kBlockRows + 1, last_blk));
  };
  auto settle = [&](int at) __attribute__((always_inline)) {
    slot[0] = u.slot(name[0]), slot[1] = u.slot(name[1]);
    if (at + kStep > T) {
      const int blk1 = min(at / kBlockRows + 1, last_blk);
      off.set(u.row_stride, lane, min(T - 1 - at, kBlockRows - 1), T - 1 - blk1 * kBlockRows);
    }
  };
  int at = begin + wave / row_waves * kStep;
  // One step.  MORE: there is another, whose K is loaded when this one's has been used, V likewise.  (Loads under a condition that
  // the compiler cannot follow would make every wait one for all loads.)
  auto step = [&](auto more) __attribute__((always_inline)) {
    constexpr bool MORE = decltype(more)::value;
    const bool whole = at + kStep <= fewest;  // every query sees every position of the step
    floatx4 s[2][R];
    float kscale[2];
    auto products = [&](auto ends) __attribute__((always_inline)) {  // ends: of the range of K
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        kscale[j] = kt[j].of_logits() * to_log2;
#pragma unroll
        for (int r = 0; r < R; ++r) s[j][r] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
          const bf16x8 k = kt[j].operand(i), low = decltype(ends)::value ? without_infinite(k) : k;
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) s[j][r] = mma(t > 0 ? low : k, q.x[r][i][t], s[j][r]);
        }
      }
    };
    products(std::false_type{});
    if constexpr (kMicro<EL> && TERMS > 1)
      if (__any(max(__float_as_uint(kt[0].scale), __float_as_uint(kt[1].scale)) >= kBeyond)) products(std::true_type{});
    const int next = at + stride;
    if constexpr (MORE) {
      settle(next);
      kt[0].load(u, slot[0], off.k[0], off.k_scale[0]);
      kt[1].load(u, slot[1], off.k[1], off.k_scale[1]);
      find(next + stride);
    }
    float x[R][8];  // logits in units of log2; in 4 bits with several tiles still without that factor, which is the same for all
    constexpr bool RAW = kMicro<EL> && R > 1;
    bool higher = false;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[r][j] = RAW ? s[j >> 2][r][j & 3] : s[j >> 2][r][j & 3] * kscale[j >> 2];
    if (!whole) {
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (at + (j >> 2) * 16 + 4 * g + (j & 3) >= limit[r]) x[r][j] = -INFINITY;
    }
    float top[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) top[r] = fmaxf(top[r], x[r][j]);
      if constexpr (RAW) top[r] *= to_log2;
      higher = higher || top[r] > m[r] + kSlack;
    }
    if (__any(higher)) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float now = fmaxf(m[r], query_max(top[r])), shrink = power_of_two(m[r] - now);
        m[r] = now;
        sum[r] *= shrink;
#pragma unroll
        for (int e = 0; e < TILES; ++e) o[r][e] *= shrink;
      }
    }
    if (R == 1 && a.stash && c < N) {
      float* to = a.stash + (((int64_t)unit * ((a.d.t_max + 15) / 16) + at / 16) * N + c) * 16 + 4 * g;
      *(float4*)to = make_float4(x[0][0], x[0][1], x[0][2], x[0][3]);
      if (at + 16 < T) *(float4*)(to + N * 16) = make_float4(x[0][4], x[0][5], x[0][6], x[0][7]);
    }
    float vscale[2], vpower[8];
    if constexpr (kMicro<EL>) {
      if constexpr (!MORE) vt.scales[0] &= off.v_there[0], vt.scales[1] &= off.v_there[1];  // (the sequence's end lies in a last step)
      four_powers(vt.scales, vpower);
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(vpower[j]));
      // Channels of V that are no number: those of the queries that see the position, no others.  Scales from 2^126 on, under which codes may be
      // infinite: a quarter of them for the position's row, four times the probability, so that 0 times it stays 0.
      if (__any(most >= 0x7E800000u)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const uint64_t bad = __ballot(__float_as_uint(vpower[j]) == 0x7F800000u);
          if (__float_as_uint(vpower[j]) == 0x7F800000u) vpower[j] = 0.f;
          if (__ballot(__float_as_uint(vpower[j]) >= 0x7E800000u) >> 16 * g & 0xFFFF) {
            vpower[j] = __uint_as_float(max(__float_as_uint(vpower[j]), 2u << 23) - (2u << 23));
#pragma unroll
            for (int r = 0; r < R; ++r) {
              x[r][j] += RAW ? 2.f / to_log2 : 2.f;
              sum[r] -= 0.75f * power_of_two((RAW ? x[r][j] * to_log2 : x[r][j]) - m[r]);
            }
          }
          if (!bad) continue;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            bool hit = false;  // lane group i's position, channels of the scale that the lane's outputs have
#pragma unroll
            for (int i = 0; i < 4; ++i)
              hit = hit || ((bad >> (16 * i + 4 * g * TILES / 32 * (32 / TILES)) & 1) && at + 16 * (j >> 2) + 4 * i + (j & 3) < limit[r]);
            const float no_number = hit ? __uint_as_float(0x7FC00000u) : 0.f;
#pragma unroll
            for (int e = 0; e < TILES; ++e) o[r][e] += no_number;
          }
        }
      }
    } else {
      vscale[0] = vt.scale[0], vscale[1] = vt.scale[1];
      if (vscale[0] != vscale[0] || vscale[1] != vscale[1]) {  // a block of V that is no number: the outputs of the queries that see it, no others
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (vscale[j] == vscale[j]) continue;
          vscale[j] = 0.f;
#pragma unroll
          for (int r = 0; r < R; ++r) {
            bool seen = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) seen = seen || !(x[r][4 * j + i] == -INFINITY);
            const float no_number = query_max(seen ? 1.f : 0.f) > 0.f ? __uint_as_float(0x7FC00000u) : 0.f;
#pragma unroll
            for (int e = 0; e < TILES; ++e) o[r][e] += no_number;
          }
        }
      }
    }
    // From here on nothing branches: exponentials, conversions and products can be mixed.
    bf16x8 p[R][PTERMS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint32_t t[3][4];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float p0, p1;
        if constexpr (RAW)
          p0 = power_of_two(fmaf(x[r][j], to_log2, -m[r])), p1 = power_of_two(fmaf(x[r][j + 1], to_log2, -m[r]));
        else
          p0 = power_of_two(x[r][j] - m[r]), p1 = power_of_two(x[r][j + 1] - m[r]);
        sum[r] += p0 + p1;
        if constexpr (!kMicro<EL>) p0 *= vscale[j >> 2], p1 *= vscale[j >> 2];
#pragma unroll
        for (int k = 0; k < PTERMS; ++k) {
          t[k][j >> 1] = bf16_pair(p0, p1);
          if (k + 1 < PTERMS) p0 -= __uint_as_float(t[k][j >> 1] << 16), p1 -= __uint_as_float(t[k][j >> 1] & 0xFFFF0000u);
        }
      }
#pragma unroll
      for (int k = 0; k < PTERMS; ++k) p[r][k] = __builtin_bit_cast(bf16x8, make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]));
    }
    if constexpr (kMicro<EL>) {
#pragma unroll
      for (int w = 0; w < HD / 32; ++w) {
        bf16x8 e[2];
        turn_pair(vt.w[0], vpower, w, e[0], e[1]);
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = PTERMS - 1; t >= 0; --t) o[r][2 * w + k] = mma(e[k], p[r][t], o[r][2 * w + k]);
      }
    } else {
#pragma unroll
      for (int w = 0; w < VTile<EL, HD>::WORDS; ++w) {
        bf16x8 e[4];
        turn_pair<EL, 0>(vt.w[w], e[0], e[1]);
        turn_pair<EL, 1>(vt.w[w], e[2], e[3]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = PTERMS - 1; t >= 0; --t) o[r][4 * w + k] = mma(e[k], p[r][t], o[r][4 * w + k]);
      }
    }
    if constexpr (MORE) vt.load(u, slot[0], slot[1], off, v_scale);
  };
  if (at < end && row0 < N) {
    find(at);
    settle(at);
    kt[0].load(u, slot[0], off.k[0], off.k_scale[0]);
    kt[1].load(u, slot[1], off.k[1], off.k_scale[1]);
    vt.load(u, slot[0], slot[1], off, v_scale);
    find(at + stride);
    for (; at + stride < end; at += stride) step(std::true_type{});
    step(std::false_type{});
  }
  // the waves of the same queries together: 16 queries at a time, thread (query, stretch of HD / 16 channels)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (r > 0) __syncthreads();
    const float total = query_sum(sum[r]);
    if (g == 0) stat[wave][c] = make_float2(m[r], total);
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)  // the lane's rows 4 g + q4 of every tile: channels TILES (4 g + q4) + tile
#pragma unroll
      for (int e = 0; e < TILES; e += 4)
        *(float4*)&joint[wave][c][TILES * (4 * g + q4) + e] = make_float4(o[r][e][q4], o[r][e + 1][q4], o[r][e + 2][q4], o[r][e + 3][q4]);
    __syncthreads();
    const int qr = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * TILES;
    for (int q = 0; q < row_waves; ++q) {
      const int n = (blockIdx.z * row_waves + q) * 16 * R + r * 16 + qr;
      if (n >= N) continue;
      float top = stat[q][qr].x;
      for (int w = q + row_waves; w < kWaves; w += row_waves) top = fmaxf(top, stat[w][qr].x);
      float x[TILES], all = 0.f;
#pragma unroll
      for (int e = 0; e < TILES; ++e) x[e] = 0.f;
      for (int w = q; w < kWaves; w += row_waves) {
        const float f = power_of_two(stat[w][qr].x - top);
        all = fmaf(f, stat[w][qr].y, all);
#pragma unroll
        for (int e = 0; e < TILES; ++e) x[e] = fmaf(f, joint[w][qr][d0 + e], x[e]);
      }
      finish_query<BF16, HD>(a, unit, n, split, top, all, x, d0);
    }
  }
}

// Weights from K again, for more queries than the stash is for.  The queries' operands of the whole call lie in LDS; a wave takes two
// blocks of positions at a time, converts them once, runs 32 queries at a time over them, and has the next two on their way.  (One step per
// workgroup, with the queries loaded for it, is latency: 172 us for 64 units of 32768 positions and 32 queries, 80 with several.)
// With fp32 queries four blocks, so that their three terms come out of LDS half as often (a pass of 8 units of 16384 and 128 queries
// 64 us, 69 with two blocks; bf16, 64 units of 32768 and 32 queries 214 with four blocks at two workgroups on a CU, 201 with two at four; a
// pass of 8 units of 32768 and 128 queries in 4 bits 62, 65 and 67 with two, three and four).
constexpr int kWeightRows = 32;
template <bool BF16>
constexpr int kWeightBlocks = BF16 ? 2 : 4;
template <bool BF16>
constexpr int kWeightStep = kWaves * kWeightBlocks<BF16> * kBlockRows;
template <bool BF16, int HD>
constexpr int kWeightGroupBytes = kWeightRows / 16 * (HD / 32) * (BF16 ? 1 : 3) * 64 * 16;

template <int EL, bool BF16, int HD>
__global__ __launch_bounds__(kThreads) void attend_weights_kernel(AttendArgs a, int row_begin, int row_end, int steps) {
  constexpr int R = kWeightRows / 16, STEPS = HD / 32, TERMS = BF16 ? 1 : 3, BLOCKS = kWeightBlocks<BF16>, STEP = kWeightStep<BF16>;
  typedef bf16x8 Group[R][STEPS][TERMS][64];
  extern __shared__ __align__(16) char lds[];
  Group* q = (Group*)lds;
  __shared__ float2 stat[256];
  const int unit = blockIdx.y, N = a.d.N;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4, c = lane & 15;
  int l, b, h;
  unit_coords(a.d, unit, l, b, h);
  const int T = seq_len(a.d, a.seq_lens, b);
  const int start = turned_x() * steps * STEP;
  if (start >= T) return;
  const int groups = (row_end - row_begin + kWeightRows - 1) / kWeightRows, last_blk = (T - 1) / kBlockRows;
  const UnitBlocks<EL, HD> u(a.k, a.v, l, b, h);
  KTile<EL, HD> k[BLOCKS];
  auto fetch = [&](int first) __attribute__((always_inline)) {  // (positions past the last: that one again)
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
      const int blk = min(first / kBlockRows + j, last_blk);
      const int row = min(lane & 15, T - 1 - blk * kBlockRows);
      k[j].load(u, u.slot(u.named(blk)), (uint32_t)row * u.row_stride + (lane >> 4) * (kMicro<EL> ? HD / 8 : 16), micro_at<HD>((lane >> 4) * (HD / 4), row));
    }
  };
  int first = start + wave * BLOCKS * kBlockRows;
  fetch(first);
  // Joined, or of the only split.  In the places of the last 32 that have no query stands the last one again, counted 0: its probabilities are
  // numbers wherever its own are, also under keys that are infinite (zeros in its place would make the weights there NaN).
  {
    const int n = row_begin + threadIdx.x;
    const float2 st = a.joined[(int64_t)unit * N + min(n, row_end - 1)];
    stat[threadIdx.x] = make_float2(st.x, n >= row_end || st.y == 0.f ? 0.f : 1.f / st.y);
  }
  const char* unit_q = a.q + (int64_t)unit * N * HD * (BF16 ? 2 : 4);
  for (int f = wave; f < groups * R * STEPS; f += kWaves) {
    const int group = f / (R * STEPS), r = f / STEPS % R, i = f % STEPS;
    bf16x8 one[TERMS];
    Queries<EL, BF16, HD, R>::load_one(unit_q, min(row_begin + group * kWeightRows + r * 16 + c, row_end - 1), row_end, i, lane, one);
#pragma unroll
    for (int t = 0; t < TERMS; ++t) q[group][r][i][t][lane] = one[t];
  }
  __syncthreads();
  const float to_log2 = kLog2E / sqrtf((float)HD);
  const int fewest = a.causal ? T - a.d.W + 1 : T;  // positions that every query sees
  for (int step = 0; step < steps && first < T; ++step, first += STEP) {
    bf16x8 x[BLOCKS][STEPS];
    float scale[BLOCKS], w[BLOCKS][4];
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
#pragma unroll
      for (int i = 0; i < STEPS; ++i) x[j][i] = k[j].operand(i);
      scale[j] = k[j].of_logits() * to_log2;
      w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0.f;
    }
    bool ends = false;  // of the range of K
    if constexpr (kMicro<EL> && TERMS > 1) {
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < BLOCKS; ++j) most = max(most, __float_as_uint(k[j].scale));
      ends = __any(most >= kBeyond);
    }
    fetch(first + STEP);
    const bool whole = first + BLOCKS * kBlockRows <= fewest;
    auto queries = [&](auto ends) __attribute__((always_inline)) {
      for (int group = 0; group < groups; ++group) {
        floatx4 s[BLOCKS][R];
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
          for (int r = 0; r < R; ++r) s[j][r] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
          for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t) {
              const bf16x8 y = q[group][r][i][t][lane];
#pragma unroll
              for (int j = 0; j < BLOCKS; ++j) s[j][r] = mma(decltype(ends)::value && t > 0 ? without_infinite(x[j][i]) : x[j][i], y, s[j][r]);
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const int m = group * kWeightRows + r * 16 + c, n = row_begin + m;
          const float2 st = stat[m];
          if (whole) {
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) w[j][i] = fmaf(power_of_two(fmaf(s[j][r][i], scale[j], -st.x)), st.y, w[j][i]);
          } else {
            const int limit = n >= row_end ? 0 : a.causal ? T - a.d.W + 1 + n % a.d.W : T;
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const float p = power_of_two(fmaf(s[j][r][i], scale[j], -st.x)) * st.y;
                if (first + 16 * j + 4 * g + i < limit) w[j][i] += p;
              }
          }
        }
      }
    };
    if (ends)
      queries(std::bool_constant<kMicro<EL> && (TERMS > 1)>{});
    else
      queries(std::false_type{});
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[j][i] = sixteen_sum(w[j][i]);
      const int t = first + 16 * j + 4 * g + (c & 3);
      if (c < 4 && t < T) {
        const int64_t at = (int64_t)unit * a.d.t_stride + t;
        const float more = c == 0 ? w[j][0] : c == 1 ? w[j][1] : c == 2 ? w[j][2] : w[j][3];
        a.weights_out[at] = (a.weights_in ? a.weights_in[at] : 0.f) + more;
      }
    }
  }
}

template <int EL, bool BF16, int HD>
hipError_t launch_weights(AttendArgs a, hipStream_t s) {
  constexpr int kMost = 96 * 1024 / kWeightGroupBytes<BF16, HD> * kWeightRows;  // queries whose operands fit LDS (fp32, 128 channels: 128)
  for (int row = 0; row < a.d.N; row += kMost) {
    const int end = min(a.d.N, row + kMost), bytes = div_up(end - row, kWeightRows) * kWeightGroupBytes<BF16, HD>;
    // Steps per workgroup: one round of workgroups where there are more, as many on a CU as its registers and LDS hold (us a pass, 8
    // units of 32768 and 128 queries, 32 KB: 79 with 256 workgroups, 70 with 512, 69 with 1024, 74 with 2048; 256 queries, 64 KB: 69, 64
    // and 71; fp32, 128 queries, 96 KB: 64 with 256, 71 with 512).
    const int resident = min(BF16 ? 4 : 2, 160 * 1024 / (bytes + (int)(256 * sizeof(float2))));
    const int total = div_up(a.d.t_max, kWeightStep<BF16>), steps = max(1, (int)((int64_t)total * a.d.units / (256 * resident)));
    hipError_t e = ensure_lds<attend_weights_kernel<EL, BF16, HD>>(bytes);
    if (e != hipSuccess) return e;
    prof_mark("attend_weights", s);
    hipLaunchKernelGGL((attend_weights_kernel<EL, BF16, HD>), dim3(div_up(total, steps), a.d.units), dim3(kThreads), bytes, s, a, row, end,
                       steps);
    a.weights_in = a.weights_out;  // the next queries' are added
  }
  return hipSuccess;
}

template <int EL, bool BF16, int HD>
hipError_t launch(const AttendArgs& a, const AttendLayout& lay, hipStream_t s) {
  const dim3 grid(lay.n_splits, a.d.units, lay.row_groups);
  prof_mark("attend", s);
  if (lay.row_tiles == 1)
    hipLaunchKernelGGL((attend_kernel<EL, BF16, HD, 1>), grid, dim3(kThreads), 0, s, a);
  else
    hipLaunchKernelGGL((attend_kernel<EL, BF16, HD, 2>), grid, dim3(kThreads), 0, s, a);
  if (lay.n_splits > 1 || a.stash) launch_attend_join(a, lay, BF16, s);
  if (a.weights_out && !a.stash) {
    const hipError_t e = launch_weights<EL, BF16, HD>(a, s);
    if (e != hipSuccess) return e;
  }
  return hipGetLastError();
}

template <int EL, bool BF16>
hipError_t launch_dim(const AttendArgs& a, const AttendLayout& lay, hipStream_t s) {
  return a.d.D == 128 ? launch<EL, BF16, 128>(a, lay, s) : launch<EL, BF16, 64>(a, lay, s);
}

}  // namespace
}  // namespace ams
#endif
