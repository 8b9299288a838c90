// Attention over a cache of 8 bits (ams_attend).
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
// Weights: with up to 16 queries the logits go to scratch (4 N bytes a position, written and read once, against 2 D of K and V)
// and the join turns them into probabilities; beyond that K is read a second time (attend_weights_kernel).
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

// Two codes of a word, bytes 2 HALF and 2 HALF + 1, as bf16.
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
// Eight codes -> the operand of one product.
template <int EL>
__device__ __forceinline__ bf16x8 eight_codes(uint32_t lo, uint32_t hi) {
  const uint4 r = make_uint4(two_codes<EL, 0>(lo), two_codes<EL, 1>(lo), two_codes<EL, 0>(hi), two_codes<EL, 1>(hi));
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

// Channel of element 0 of the 8 that lane group g feeds to product i of q.k: 16 bytes of a K row per load.
__device__ __forceinline__ int k_channel(int i, int g) { return 64 * (i >> 1) + 16 * g + 8 * (i & 1); }

// The query operand of rows row0 + 16 r + lane % 16, as TERMS bf16 terms.
template <bool BF16, int HD, int R>
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
    const int d = k_channel(i, lane >> 4);
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

// Loads of what no kernel here writes and every lane of the wave wants: through the scalar cache.
template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// The blocks of one unit: slot of a block (the block itself, or its page), bytes and scales from slot to slot, the same for K and V.
struct UnitBlocks {
  const char *k, *v;
  const float *k_scale, *v_scale;
  const int32_t* table;  // null: dense
  int64_t block_bytes, scale_step, n_pages;
  int row_stride;
  __device__ __forceinline__ UnitBlocks(const CacheDev& kc, const CacheDev& vc, int l, int b, int h) {
    const Block k0 = first(kc, l, b, h), v0 = first(vc, l, b, h);
    k = k0.row0, v = v0.row0, k_scale = kc.scale + k0.scale, v_scale = vc.scale + v0.scale;
    table = kc.paged ? kc.table + (int64_t)b * kc.max_blocks : nullptr;
    row_stride = (int)k0.stride;
    block_bytes = k0.stride * kBlockRows;
    scale_step = kc.paged ? kc.H : 1;
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
// sequence's last blocks) are that position again: what is behind it, in the cache or past its end, is not read.
template <int HD>
struct Offsets {
  uint32_t k[2], v[2][4];
  __device__ __forceinline__ void set(int row_stride, int lane, int most0, int most1) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int most = j ? most1 : most0;
      k[j] = (uint32_t)min(lane & 15, most) * row_stride + (lane >> 4) * 16;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[j][i] = (uint32_t)min((lane >> 4) * 4 + i, most) * row_stride + (lane & 15) * (HD / 16);
    }
  }
};

// A block of K as the wave reads it: lane % 16 is the position, lane / 16 the 16 bytes of every 64.
template <int HD>
struct KTile {
  uint4 w[HD / 64];
  float scale;
  __device__ __forceinline__ void load(const UnitBlocks& u, int64_t slot, uint32_t offset) {
    scale = uniform_load(u.k_scale + slot * u.scale_step);
    const char* row = u.k + slot * u.block_bytes;
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) w[i] = *(const uint4*)(row + offset + 64 * i);
  }
  template <int EL>
  __device__ __forceinline__ bf16x8 operand(int i) const {
    return (i & 1) ? eight_codes<EL>(w[i >> 1].z, w[i >> 1].w) : eight_codes<EL>(w[i >> 1].x, w[i >> 1].y);
  }
};

// Two blocks of V: lane % 16 is the stretch of HD / 16 channels, word [j] of position 4 (lane / 16) + j % 4 of block j / 4.
template <int HD>
struct VTile {
  static constexpr int WORDS = HD / 64;  // of 4 channels
  uint32_t w[WORDS][8];
  float scale[2];
  __device__ __forceinline__ void load(const UnitBlocks& u, int64_t slot0, int64_t slot1, const Offsets<HD>& o) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t slot = j ? slot1 : slot0;
      scale[j] = uniform_load(u.v_scale + slot * u.scale_step);
      const char* block = u.v + slot * u.block_bytes;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (WORDS == 2) {
          const uint2 x = *(const uint2*)(block + o.v[j][i]);
          w[0][4 * j + i] = x.x, w[1][4 * j + i] = x.y;
        } else {
          w[0][4 * j + i] = *(const uint32_t*)(block + o.v[j][i]);
        }
      }
    }
  }
};

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
  Queries<BF16, HD, R> q;
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
  const UnitBlocks u(a.k, a.v, l, b, h);
  const int last_blk = (T - 1) / kBlockRows;
  Offsets<HD> off;
  off.set(u.row_stride, lane, kBlockRows - 1, kBlockRows - 1);
  KTile<HD> kt[2];
  VTile<HD> vt;
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
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      kscale[j] = kt[j].scale * to_log2;
#pragma unroll
      for (int r = 0; r < R; ++r) s[j][r] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < STEPS; ++i) {
        const bf16x8 k = kt[j].template operand<EL>(i);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int t = TERMS - 1; t >= 0; --t) s[j][r] = mma(k, q.x[r][i][t], s[j][r]);
      }
    }
    const int next = at + stride;
    if constexpr (MORE) {
      settle(next);
      kt[0].load(u, slot[0], off.k[0]);
      kt[1].load(u, slot[1], off.k[1]);
      find(next + stride);
    }
    float x[R][8];
    bool higher = false;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int j = 0; j < 8; ++j) x[r][j] = s[j >> 2][r][j & 3] * kscale[j >> 2];
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
    float vscale[2] = {vt.scale[0], vt.scale[1]};
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
    // From here on nothing branches: exponentials, conversions and products can be mixed.
    bf16x8 p[R][PTERMS];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint32_t t[3][4];
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        float p0 = power_of_two(x[r][j] - m[r]), p1 = power_of_two(x[r][j + 1] - m[r]);
        sum[r] += p0 + p1;
        p0 *= vscale[j >> 2], p1 *= vscale[j >> 2];
#pragma unroll
        for (int k = 0; k < PTERMS; ++k) {
          t[k][j >> 1] = bf16_pair(p0, p1);
          if (k + 1 < PTERMS) p0 -= __uint_as_float(t[k][j >> 1] << 16), p1 -= __uint_as_float(t[k][j >> 1] & 0xFFFF0000u);
        }
      }
#pragma unroll
      for (int k = 0; k < PTERMS; ++k) p[r][k] = __builtin_bit_cast(bf16x8, make_uint4(t[k][0], t[k][1], t[k][2], t[k][3]));
    }
#pragma unroll
    for (int w = 0; w < VTile<HD>::WORDS; ++w) {
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
    if constexpr (MORE) vt.load(u, slot[0], slot[1], off);
  };
  if (at < end && row0 < N) {
    find(at);
    settle(at);
    kt[0].load(u, slot[0], off.k[0]);
    kt[1].load(u, slot[1], off.k[1]);
    vt.load(u, slot[0], slot[1], off);
    find(at + stride);
    for (; at + stride < end; at += stride) step(std::true_type{});
    step(std::false_type{});
  }
  // the waves of the same queries together: 16 queries at a time, thread (query, stretch of HD / 16 channels)
  const bool last = a.n_splits == 1;
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
      const int64_t row = ((int64_t)unit * a.n_splits + split) * N + n;
      if (threadIdx.x % 16 == 0) {
        a.stats[((int64_t)unit * N + n) * a.n_splits + split] = make_float2(top, all);
        if (last && a.lse) a.lse[(int64_t)unit * N + n] = all == 0.f ? -INFINITY : (top + log2f(all)) * kLn2;
      }
      if (last) {
        const float inverse = all == 0.f ? 0.f : 1.f / all;
        char* to = a.out + (((int64_t)unit * N + n) * HD + d0) * (BF16 ? 2 : 4);
#pragma unroll
        for (int e = 0; e < TILES; e += 4) {
          const float y0 = x[e] * inverse, y1 = x[e + 1] * inverse, y2 = x[e + 2] * inverse, y3 = x[e + 3] * inverse;
          if constexpr (BF16)
            *(uint2*)(to + 2 * e) = make_uint2(bf16_pair(y0, y1), bf16_pair(y2, y3));
          else
            *(float4*)(to + 4 * e) = make_float4(y0, y1, y2, y3);
        }
      } else {
#pragma unroll
        for (int e = 0; e < TILES; e += 4) *(float4*)&a.part[row * HD + d0 + e] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      }
    }
  }
}

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
  {
    const int n = threadIdx.x >> 4;
    const float2 st = joined_stats<16>(a, unit, min(n, N - 1), splits, threadIdx.x & 15);
    if ((threadIdx.x & 15) == 0) stat[n] = make_float2(st.x, st.y == 0.f ? 0.f : 1.f / st.y);
  }
  __syncthreads();
  const int t = first + 4 * threadIdx.x;
  if (t >= T) return;
  const float* x = a.stash + (((int64_t)unit * ((a.d.t_max + 15) / 16) + t / 16) * N) * 16 + t % 16;
  float w[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int n = 0; n < N; ++n) {
    const float4 v = *(const float4*)(x + n * 16);
    const float s[4] = {v.x, v.y, v.z, v.w};
    const float2 st = stat[n];
#pragma unroll
    for (int i = 0; i < 4; ++i) {  // (a position that the query does not see has no part in a sum that is no number)
      const float p = power_of_two(s[i] - st.x) * st.y;
      w[i] += s[i] == -INFINITY ? 0.f : p;
    }
  }
  const int64_t at = (int64_t)unit * a.d.t_stride + t;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t + i < T) a.weights_out[at + i] = (a.weights_in ? a.weights_in[at + i] : 0.f) + w[i];
}

// Weights from K again, for more queries than the stash is for.  The queries' operands of the whole call lie in LDS; a wave takes two
// blocks of positions at a time, converts them once, runs 32 queries at a time over them, and has the next two on their way.  (One step per
// workgroup, with the queries loaded for it, is latency: 172 us for 64 units of 32768 positions and 32 queries, 80 with several.)
// With fp32 queries four blocks, so that their three terms come out of LDS half as often (a pass of 8 units of 16384 and 128 queries
// 64 us, 69 with two blocks; bf16, 64 units of 32768 and 32 queries 214 with four blocks at two workgroups on a CU, 201 with two at four).
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
  const UnitBlocks u(a.k, a.v, l, b, h);
  KTile<HD> k[BLOCKS];
  auto fetch = [&](int first) __attribute__((always_inline)) {  // (positions past the last: that one again)
#pragma unroll
    for (int j = 0; j < BLOCKS; ++j) {
      const int blk = min(first / kBlockRows + j, last_blk);
      k[j].load(u, u.slot(u.named(blk)), (uint32_t)min(lane & 15, T - 1 - blk * kBlockRows) * u.row_stride + (lane >> 4) * 16);
    }
  };
  int first = start + wave * BLOCKS * kBlockRows;
  fetch(first);
  {  // joined, or of the only split; a query that is not there counts nothing
    const int n = row_begin + threadIdx.x;
    const float2 st = n < row_end ? a.joined[(int64_t)unit * N + n] : make_float2(0.f, 0.f);
    stat[threadIdx.x] = make_float2(st.x, st.y == 0.f ? 0.f : 1.f / st.y);
  }
  const char* unit_q = a.q + (int64_t)unit * N * HD * (BF16 ? 2 : 4);
  for (int f = wave; f < groups * R * STEPS; f += kWaves) {
    const int group = f / (R * STEPS), r = f / STEPS % R, i = f % STEPS;
    bf16x8 one[TERMS];
    Queries<BF16, HD, R>::load_one(unit_q, row_begin + group * kWeightRows + r * 16 + c, row_end, i, lane, one);
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
      for (int i = 0; i < STEPS; ++i) x[j][i] = k[j].template operand<EL>(i);
      scale[j] = k[j].scale * to_log2;
      w[j][0] = w[j][1] = w[j][2] = w[j][3] = 0.f;
    }
    fetch(first + STEP);
    const bool whole = first + BLOCKS * kBlockRows <= fewest;
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
            for (int j = 0; j < BLOCKS; ++j) s[j][r] = mma(x[j][i], y, s[j][r]);
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
  const int joins = lay.n_splits > 1 ? a.d.N : 0, stash = a.stash ? div_up(a.d.t_max, kStashKeys) : 0;
  if (joins + stash > 0) {
    prof_mark("attend_join", s);
    hipLaunchKernelGGL((attend_join_kernel<BF16, HD>), dim3(joins + stash, a.d.units), dim3(kThreads), 0, s, a, joins);
  }
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

AttendLayout attend_layout(const ams_params* p) {
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
  const size_t per_split = units * r.row_groups, resident = (r.row_tiles == 1 ? 3 : 2) - (p->kv_dtype == AMS_F32 && p->head_dim == 128);
  const int fine = r.row_tiles == 1 ? 512 : 2048;
  if (per_split * div_up(p->t_max, fine) >= 2048) {
    r.chunk = fine;
  } else {
    const int splits = (int)max((size_t)1, 256 * resident / per_split);
    r.chunk = div_up(div_up(p->t_max, splits), kWaves * kStep) * kWaves * kStep;
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

hipError_t launch_attend(const AttendArgs& a, const AttendLayout& lay, bool bf16, int el, hipStream_t s) {
  if (el == EL_INT8) return bf16 ? launch_dim<EL_INT8, true>(a, lay, s) : launch_dim<EL_INT8, false>(a, lay, s);
  return bf16 ? launch_dim<EL_E4M3, true>(a, lay, s) : launch_dim<EL_E4M3, false>(a, lay, s);
}

}  // namespace ams
