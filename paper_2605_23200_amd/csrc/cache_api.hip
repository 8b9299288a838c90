// Host side of the entry points around a bounded cache (ams_append, ams_attend, ams_recode, ams_evict): argument checks and the order
// of the launches.  Nothing here touches device memory or waits for the stream.
#include <math.h>

#include "cache.h"

namespace ams {
namespace {

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

// The sizes that every call here goes by.
int check_sizes(const ams_params* p) {
  if (!p) return AMS_ERR_INVALID_ARG;
  if (p->n_layers < 1 || p->batch < 1 || p->n_kv_heads < 1 || p->group < 1 || p->window < 1 || p->t_max < 1 || p->t_stride < p->t_max)
    return AMS_ERR_INVALID_ARG;
  if (p->kv_dtype != AMS_F32 && p->kv_dtype != AMS_BF16) return AMS_ERR_INVALID_ARG;
  if (p->head_dim < 1) return AMS_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return AMS_ERR_UNSUPPORTED;
  // (three factors of 31 bits: no product of two overflows 64)
  const int64_t rows = (int64_t)p->n_layers * p->batch;
  if (rows > 65535 || rows * p->n_kv_heads > 65535) return AMS_ERR_UNSUPPORTED;
  if ((int64_t)p->n_kv_heads * p->group > 65535 || p->t_max > (1 << 30)) return AMS_ERR_UNSUPPORTED;
  return AMS_OK;
}
int check_attend(const ams_params* p) {
  const int rc = check_sizes(p);
  if (rc) return rc;
  if (p->causal != 0 && p->causal != 1) return AMS_ERR_INVALID_ARG;
  return (int64_t)p->group * p->window > 256 ? AMS_ERR_UNSUPPORTED : AMS_OK;
}
int check_evict(const ams_params* p) {
  const int rc = check_sizes(p);
  if (rc) return rc;
  if (p->budget < 1 || p->n_sink < 0 || p->n_last < 0) return AMS_ERR_INVALID_ARG;
  return p->budget > (1 << 30) ? AMS_ERR_UNSUPPORTED : AMS_OK;
}

bool packed(const ams_cache* c) { return c->dtype == AMS_INT8 || c->dtype == AMS_E4M3; }

// rows: positions per sequence that the call may touch.
int check_cache(const ams_params* p, const ams_cache* c, int64_t rows) {
  if (!c || !c->kv.k || !c->kv.v || !aligned(c->kv.k) || !aligned(c->kv.v)) return AMS_ERR_INVALID_ARG;
  if (!packed(c) && c->dtype != p->kv_dtype) return AMS_ERR_INVALID_ARG;
  if (packed(c) && (!c->k_scale || !c->v_scale)) return AMS_ERR_INVALID_ARG;
  if (c->kv.layout == AMS_LAYOUT_DENSE) return c->kv.t_capacity < rows ? AMS_ERR_INVALID_ARG : AMS_OK;
  if (c->kv.layout != AMS_LAYOUT_PAGED) return AMS_ERR_INVALID_ARG;
  if (!c->kv.block_table || c->kv.max_blocks_per_seq < 1 || c->kv.n_slots < kBlockRows) return AMS_ERR_INVALID_ARG;
  if (c->kv.block_size != kBlockRows) return AMS_ERR_UNSUPPORTED;
  if (packed(c) && c->kv.n_slots % kBlockRows) return AMS_ERR_INVALID_ARG;
  return (int64_t)c->kv.max_blocks_per_seq * kBlockRows < rows ? AMS_ERR_INVALID_ARG : AMS_OK;
}
bool same_slab(const ams_cache* a, const ams_cache* b) {  // paged views may share a pool (other blocks)
  return a->kv.layout == AMS_LAYOUT_DENSE && b->kv.layout == AMS_LAYOUT_DENSE && (a->kv.k == b->kv.k || a->kv.v == b->kv.v);
}

Dims dims(const ams_params* p) {
  Dims d;
  d.L = p->n_layers, d.B = p->batch, d.H = p->n_kv_heads, d.G = p->group, d.W = p->window, d.D = p->head_dim;
  d.N = p->group * p->window;
  d.units = p->n_layers * p->batch * p->n_kv_heads;
  d.t_max = p->t_max, d.t_stride = p->t_stride;
  return d;
}
CacheDev device(const ams_params* p, const ams_cache* c, bool values) {
  CacheDev r;
  r.base = (char*)(values ? c->kv.v : c->kv.k);
  r.scale = packed(c) ? (values ? c->v_scale : c->k_scale) : nullptr;
  r.table = c->kv.block_table;
  r.t_capacity = c->kv.t_capacity;
  r.n_pages = c->kv.n_slots / kBlockRows;
  r.n_slots = c->kv.n_slots;
  r.max_blocks = c->kv.max_blocks_per_seq;
  r.B = p->batch, r.H = p->n_kv_heads;
  r.row_bytes = p->head_dim * (packed(c) ? 1 : c->dtype == AMS_BF16 ? 2 : 4);
  r.paged = c->kv.layout == AMS_LAYOUT_PAGED;
  return r;
}
int status(hipError_t e, hipStream_t s) {
  prof_mark("end", s);
  if (e == hipSuccess) return AMS_OK;
  return e == hipErrorNotSupported ? AMS_ERR_UNSUPPORTED : AMS_ERR_HIP;
}

}  // namespace
}  // namespace ams

using namespace ams;

extern "C" {

int ams_rope_init(ams_rope* out, int32_t layout, int32_t rot_dim, double base, int32_t scaling, double factor,
                  int32_t original_len, double slow, double fast, float gain) {
  if (!out || (layout != AMS_ROPE_HALF && layout != AMS_ROPE_INTERLEAVED) || rot_dim < 0 || rot_dim > 128 || rot_dim % 2)
    return AMS_ERR_INVALID_ARG;
  if (scaling < AMS_ROPE_PLAIN || scaling > AMS_ROPE_BY_PARTS || !(base > 0) || isinf(base) || !isfinite(gain)) return AMS_ERR_INVALID_ARG;
  if (scaling != AMS_ROPE_PLAIN && (!(factor >= 1) || isinf(factor))) return AMS_ERR_INVALID_ARG;
  if (scaling == AMS_ROPE_BASE && rot_dim == 2) return AMS_ERR_INVALID_ARG;
  if (scaling == AMS_ROPE_BY_PARTS && (original_len < 1 || !(fast > slow) || !isfinite(fast) || !isfinite(slow))) return AMS_ERR_INVALID_ARG;
  *out = ams_rope{};
  out->layout = layout, out->rot_dim = rot_dim, out->gain = gain;
  if (scaling == AMS_ROPE_BASE && rot_dim > 0) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    if (scaling == AMS_ROPE_LINEAR) f /= factor;
    if (scaling == AMS_ROPE_BY_PARTS) {
      const double turns = original_len * f / 6.283185307179586;
      const double keep = fmin(fmax((turns - slow) / (fast - slow), 0.0), 1.0);
      f *= keep + (1 - keep) / factor;
    }
    out->freq[i] = f;
  }
  return AMS_OK;
}

int ams_append(const ams_params* p, const ams_new_tokens* x, const ams_rope* rope, const int32_t* seq_lens, void* q_out,
               const ams_cache* dst, int32_t* lens_out, void* stream) {
  int rc = check_sizes(p);
  if (rc) return rc;
  if ((rc = check_cache(p, dst, p->t_max))) return rc;
  if (!x || !x->k || !x->v || !seq_lens || (x->q == nullptr) != (q_out == nullptr) || (q_out && q_out == x->q) || lens_out == seq_lens)
    return AMS_ERR_INVALID_ARG;
  if (x->n_new < 1 || !(x->norm_eps >= 0.f) || isinf(x->norm_eps)) return AMS_ERR_INVALID_ARG;
  if (x->n_new > (1 << 20)) return AMS_ERR_UNSUPPORTED;
  const int es = p->kv_dtype == AMS_BF16 ? 2 : 4;
  const int64_t k_row = (int64_t)p->n_kv_heads * p->head_dim, q_row = k_row * p->group;
  if (x->k_stride < k_row || x->v_stride < k_row || (x->q && x->q_stride < q_row)) return AMS_ERR_INVALID_ARG;
  if (x->k_stride * es % 16 || x->v_stride * es % 16 || (x->q && x->q_stride * es % 16)) return AMS_ERR_INVALID_ARG;
  if (!aligned(x->q) || !aligned(x->k) || !aligned(x->v) || !aligned(q_out) || !aligned(x->q_weight) || !aligned(x->k_weight))
    return AMS_ERR_INVALID_ARG;
  if (rope) {
    if ((rope->layout != AMS_ROPE_HALF && rope->layout != AMS_ROPE_INTERLEAVED) || rope->rot_dim < 0 || rope->rot_dim % 2 ||
        rope->rot_dim > p->head_dim || !isfinite(rope->gain))
      return AMS_ERR_INVALID_ARG;
    for (int i = 0; i < rope->rot_dim / 2; ++i)
      if (!isfinite(rope->freq[i])) return AMS_ERR_INVALID_ARG;
  }
  AppendArgs a;
  a.d = dims(p);
  a.q = (const char*)x->q, a.k = (const char*)x->k, a.v = (const char*)x->v;
  a.q_stride = x->q_stride * es, a.k_stride = x->k_stride * es, a.v_stride = x->v_stride * es;
  a.q_weight = (const char*)x->q_weight, a.k_weight = (const char*)x->k_weight;
  a.eps = x->norm_eps;
  a.positions = x->positions, a.seq_lens = seq_lens, a.n_new = x->n_new;
  a.q_out = (char*)q_out;
  a.kd = device(p, dst, false), a.vd = device(p, dst, true);
  a.lens_out = lens_out;
  return status(launch_append(a, rope, p->kv_dtype == AMS_BF16, dst->dtype, (hipStream_t)stream), (hipStream_t)stream);
}

size_t ams_attend_workspace_bytes(const ams_params* p) { return check_attend(p) == AMS_OK ? attend_layout(p).total : 0; }
size_t ams_evict_workspace_bytes(const ams_params* p) { return check_evict(p) == AMS_OK ? evict_ws_bytes(p) : 0; }

int ams_attend(const ams_params* p, const ams_cache* src, const int32_t* seq_lens, const void* q, void* out, float* lse,
               const float* weights_in, float* weights_out, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_attend(p);
  if (rc) return rc;
  if ((rc = check_cache(p, src, p->t_max))) return rc;
  if (!packed(src)) return AMS_ERR_UNSUPPORTED;
  if (!seq_lens || !q || !out || !ws || (weights_in && !weights_out)) return AMS_ERR_INVALID_ARG;
  if (!aligned(q) || !aligned(out) || !aligned(ws) || q == out) return AMS_ERR_INVALID_ARG;
  const AttendLayout lay = attend_layout(p);
  if (ws_bytes < lay.total) return AMS_ERR_WORKSPACE_TOO_SMALL;
  AttendArgs a;
  a.d = dims(p);
  a.k = device(p, src, false), a.v = device(p, src, true);
  a.seq_lens = seq_lens;
  a.q = (const char*)q, a.out = (char*)out, a.lse = lse;
  a.weights_in = weights_in, a.weights_out = weights_out;
  a.causal = p->causal;
  a.part = (float*)((char*)ws + lay.part);
  a.stats = (float2*)((char*)ws + lay.stats);
  a.joined = lay.stashed ? nullptr : lay.n_splits > 1 ? (float2*)((char*)ws + lay.joined) : a.stats;
  a.stash = weights_out && lay.stashed ? (float*)((char*)ws + lay.stash) : nullptr;
  a.chunk = lay.chunk, a.n_splits = lay.n_splits, a.row_waves = lay.row_waves;
  return status(launch_attend(a, lay, p->kv_dtype == AMS_BF16, src->dtype, (hipStream_t)stream), (hipStream_t)stream);
}

int ams_recode(const ams_params* p, const ams_cache* src, const int32_t* seq_lens, const int32_t* idx, const int32_t* n_kept,
               const ams_cache* dst, const float* credit_src, float* credit_dst, void* stream) {
  int rc = check_sizes(p);
  if (rc) return rc;
  if (idx && p->budget < 1) return AMS_ERR_INVALID_ARG;
  const int64_t rows = idx && p->budget < p->t_max ? p->budget : p->t_max;
  if ((rc = check_cache(p, src, p->t_max))) return rc;
  if ((rc = check_cache(p, dst, rows))) return rc;
  if (!(idx ? n_kept : seq_lens) || same_slab(src, dst)) return AMS_ERR_INVALID_ARG;
  if (!packed(src) && !packed(dst)) return AMS_ERR_UNSUPPORTED;
  RecodeArgs a{dims(p), device(p, src, false), device(p, src, true), device(p, dst, false), device(p, dst, true),
               seq_lens, idx, n_kept, p->budget, credit_src, credit_dst, p->budget};
  return status(launch_recode(a, src->dtype, dst->dtype, (hipStream_t)stream), (hipStream_t)stream);
}

int ams_evict(const ams_params* p, const ams_cache* src, const int32_t* seq_lens, const float* weights, const ams_cache* dst,
              float* weights_out, int32_t* idx, int32_t* n_kept, int32_t* lens_out, void* ws, size_t ws_bytes, void* stream) {
  int rc = check_evict(p);
  if (rc) return rc;
  const int64_t keep = p->budget < p->t_max ? p->budget : p->t_max;
  if ((rc = check_cache(p, src, p->t_max))) return rc;
  if ((rc = check_cache(p, dst, keep))) return rc;
  if (!seq_lens || !weights || !weights_out || !idx || !n_kept || !ws || !aligned(ws) || weights == weights_out || lens_out == seq_lens || same_slab(src, dst))
    return AMS_ERR_INVALID_ARG;
  if (ws_bytes < evict_ws_bytes(p)) return AMS_ERR_WORKSPACE_TOO_SMALL;
  const Dims d = dims(p);
  const EvictArgs e{d, seq_lens, weights, weights_out, idx, n_kept, lens_out, p->budget, p->n_sink, p->n_last};
  hipStream_t s = (hipStream_t)stream;
  const hipError_t err = launch_evict_pick(e, (char*)ws, s);
  if (err != hipSuccess) return status(err, s);
  const CacheDev ks = device(p, src, false), vs = device(p, src, true), kd = device(p, dst, false), vd = device(p, dst, true);
  const RecodeArgs a{d, ks, vs, kd, vd, nullptr, idx, n_kept, p->budget, nullptr, nullptr, p->budget};
  return status(launch_recode(a, src->dtype, dst->dtype, s), s);
}

}  // extern "C"
