// C ABI of the operators around the attention (declared in include/vc_attn.h): argument validation on the
// host, workspace carve-up and launches of the norms with the rotation and of the attention to another sequence.
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "vc_attn.h"
#include "vc_internal.hpp"

namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// A view of [B, H, n] rows of d channels; outputs must not overlap themselves
vc_status check_view(const vc_view* v, int B, int H, int n, int d, bool output) {
  if (!v || !v->data) return VC_ERR_NULL;
  if (!aligned(v->data, 16)) return VC_ERR_ALIGN;
  int64_t stride[3] = {v->sb, v->sh, v->sn}, extent[3] = {B, H, n};
  for (int i = 0; i < 3; ++i) {
    if (extent[i] == 1) continue;
    if (stride[i] < 0 || stride[i] > (1LL << 40) / (extent[i] - 1)) return VC_ERR_SHAPE;
    if (stride[i] % 8 != 0) return VC_ERR_ALIGN;
  }
  if (!output) return VC_OK;
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] < stride[i]) {
        const int64_t s = stride[i], e = extent[i];
        stride[i] = stride[j], extent[i] = extent[j];
        stride[j] = s, extent[j] = e;
      }
  int64_t span = d;
  for (int i = 0; i < 3; ++i) {
    if (extent[i] == 1) continue;
    if (stride[i] < span) return VC_ERR_SHAPE;
    span += stride[i] * (extent[i] - 1);
  }
  return VC_OK;
}

// strides of axes of extent 1 are not used
void strides(const vc_view* v, int B, int H, int n, int64_t& sb, int64_t& sh, int64_t& sn) {
  sb = B == 1 ? 0 : v->sb;
  sh = H == 1 ? 0 : v->sh;
  sn = n == 1 ? 0 : v->sn;
}

vc_status check_norm_rope(const vc_norm_rope_shape* s, const vc_norm_rope_opts* o) {
  if (!s || !o) return VC_ERR_NULL;
  if (s->B < 1 || s->N < 1 || s->Hq < 1 || s->Hk < 0 || (s->d != 64 && s->d != 128)) return VC_ERR_SHAPE;
  if ((int64_t)s->B * s->N >= (1LL << 31) || ((int64_t)s->Hq + s->Hk) * s->d > (1 << 20)) return VC_ERR_SHAPE;
  if (o->dtype != VC_BF16 && o->dtype != VC_FP16) return VC_ERR_UNSUPPORTED;
  if (o->norm != VC_NORM_NONE && o->norm != VC_NORM_HEAD && o->norm != VC_NORM_TOKEN) return VC_ERR_UNSUPPORTED;
  if (o->layout != VC_ROPE_NONE && o->layout != VC_ROPE_INTERLEAVED && o->layout != VC_ROPE_HALF)
    return VC_ERR_UNSUPPORTED;
  if (o->norm == VC_NORM_NONE && o->layout == VC_ROPE_NONE) return VC_ERR_UNSUPPORTED;
  if (o->norm != VC_NORM_NONE && !(o->eps >= FLT_MIN && std::isfinite(o->eps))) return VC_ERR_UNSUPPORTED;
  if (o->norm == VC_NORM_TOKEN && (s->Hq * s->d > 8192 || s->Hk * s->d > 8192)) return VC_ERR_SHAPE;
  if (o->layout == VC_ROPE_NONE) return o->rot == 0 ? VC_OK : VC_ERR_UNSUPPORTED;
  if (o->rot < 16 || o->rot > s->d || o->rot % 16 != 0) return VC_ERR_UNSUPPORTED;
  if (o->F == 0 && o->Ht == 0 && o->Wd == 0) return o->rows >= 1 ? VC_OK : VC_ERR_UNSUPPORTED;
  if (o->F < 1 || o->Ht < 1 || o->Wd < 1) return VC_ERR_UNSUPPORTED;
  const int64_t fh = (int64_t)o->F * o->Ht;
  if (fh > s->N || fh * o->Wd != s->N) return VC_ERR_SHAPE;
  if ((int64_t)o->F + o->Ht + o->Wd >= (1 << 25)) return VC_ERR_SHAPE;   // the kernels' indexes into the tables
  if (s->d != 128 || o->rot != 128) return VC_ERR_UNSUPPORTED;
  return VC_OK;
}

// columns of a tensor's weights
int norm_weights(const vc_norm_rope_opts* o, int H, int d) { return o->norm == VC_NORM_TOKEN ? H * d : d; }

vc_status norm_rope_args(const vc_norm_rope_shape* s, const vc_norm_rope_opts* o, const float* cos_t,
                         const float* sin_t, const int32_t* pos, vc::NormRopeArgs& a) {
  const bool turned = o->layout != VC_ROPE_NONE, grid = turned && o->F > 0;
  if (turned && (!cos_t || !sin_t)) return VC_ERR_NULL;
  if (turned && (!aligned(cos_t, 16) || !aligned(sin_t, 16))) return VC_ERR_ALIGN;
  if (pos && !aligned(pos, 4)) return VC_ERR_ALIGN;
  if (grid && pos) return VC_ERR_UNSUPPORTED;
  if (turned && !grid && !pos && o->rows < s->N) return VC_ERR_SHAPE;
  a.ntensors = s->Hk > 0 ? 2 : 1;
  a.tokens = (int64_t)s->B * s->N;
  a.N = s->N;
  a.d = s->d;
  a.dtype = o->dtype;
  a.norm = o->norm;
  a.layout = o->layout;
  a.rot = o->rot;
  a.eps = o->eps;
  a.sign = 1.f;
  a.cos_t = cos_t;
  a.sin_t = sin_t;
  a.pos = turned ? pos : nullptr;
  a.rows = o->rows;
  a.grid = grid;
  a.F = o->F;
  a.Ht = o->Ht;
  a.Wd = o->Wd;
  return VC_OK;
}

vc_status check_cross(const vc_cross_shape* s, const vc_cross_opts* o) {
  if (!s || !o) return VC_ERR_NULL;
  if (s->B < 1 || s->Hq < 1 || s->Hk < 1 || s->M < 1 || s->N < 1 || (s->d != 64 && s->d != 128)) return VC_ERR_SHAPE;
  if (s->Hq % s->Hk != 0) return VC_ERR_SHAPE;
  const int64_t top = 1LL << 31;
  if ((int64_t)s->B * s->Hq >= top || (int64_t)s->B * s->Hq * s->M >= top || (int64_t)s->B * s->Hk * s->N >= top)
    return VC_ERR_SHAPE;
  const int64_t rows = (int64_t)(s->Hq / s->Hk) * s->M, heads = (int64_t)s->B * s->Hk;
  if (rows > (1 << 30) || s->N > (1 << 30)) return VC_ERR_SHAPE;
  // workgroups of 128 rows or keys, or of 1024 threads for 4096 keys of an item: a launch has fewer than 2^32 threads
  if (s->B >= (1 << 22) || (rows + 127) / 128 * heads >= (1 << 24) || ((int64_t)s->N + 127) / 128 * heads >= (1 << 24)) return VC_ERR_SHAPE;
  if (o->dtype != VC_BF16 && o->dtype != VC_FP16) return VC_ERR_UNSUPPORTED;
  if (!(o->sm_scale >= 0.f) || !std::isfinite(o->sm_scale * 1.4426950408889634f)) return VC_ERR_UNSUPPORTED;
  if (o->masked != 0 && o->masked != 1) return VC_ERR_UNSUPPORTED;
  return VC_OK;
}

inline size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

// The shape, the plan and the workspace of a call: fills a, returns the bytes that the workspace at `ws` takes
size_t cross_args(const vc_cross_shape* s, const vc_cross_opts* o, bool backward, void* ws, vc::CrossArgs& a) {
  a.B = s->B;
  a.Hq = s->Hq;
  a.Hk = s->Hk;
  a.G = s->Hq / s->Hk;
  a.M = s->M;
  a.N = s->N;
  a.R = a.G * a.M;
  a.d = s->d;
  a.dtype = o->dtype;
  const double scale = o->sm_scale > 0.f ? (double)o->sm_scale : 1.0 / std::sqrt((double)s->d);
  a.scale = (float)scale;
  a.c = (float)(scale * 1.4426950408889634074);
  if (backward) vc::cross_plan_backward(a);
  else vc::cross_plan(a);
  size_t end = 0;
  auto part = [&](size_t bytes) {
    const size_t at = end;
    end += align256(bytes);
    return static_cast<char*>(ws) + at;
  };
  const size_t rows = (size_t)a.B * a.Hk * a.R, keys = (size_t)a.B * a.Hk * a.N;
  if (o->masked) {
    a.idx = reinterpret_cast<int32_t*>(part((size_t)a.B * a.N * 4));
    a.count = reinterpret_cast<int32_t*>(part((size_t)a.B * 4));
  }
  if (a.splits > 1) {
    a.part_o = reinterpret_cast<float*>(part(a.splits * rows * a.d * 4));
    a.part_ml = reinterpret_cast<float*>(part(a.splits * rows * 8));
  }
  if (backward) {
    a.stats = reinterpret_cast<float*>(part((size_t)a.B * a.Hq * vc::cross_stat_rows(a.M) * 8));
    if (a.row_splits > 1) a.part_kv = reinterpret_cast<float*>(part(a.row_splits * 2 * keys * a.d * 4));
  }
  return end;
}

vc_status cross_view(const vc_view* v, int B, int H, int n, int d, bool output, vc::Strided& t) {
  const vc_status st = check_view(v, B, H, n, d, output);
  if (st != VC_OK) return st;
  t.p = static_cast<uint16_t*>(v->data);
  strides(v, B, H, n, t.sb, t.sh, t.sn);
  if (n == 1) t.sn = d;   // a single row: what would follow it lies behind its buffer
  return VC_OK;
}

// The arguments that both directions share
vc_status cross_inputs(const vc_cross_shape* s, const vc_cross_opts* o, const vc_view* Q, const vc_view* K,
                       const vc_view* V, const int32_t* k_len, const uint8_t* k_mask, int64_t stride, void* ws,
                       size_t ws_bytes, bool backward, vc::CrossArgs& a) {
  vc_status st = check_cross(s, o);
  if (st != VC_OK) return st;
  if ((st = cross_view(Q, s->B, s->Hq, s->M, s->d, false, a.Q)) != VC_OK) return st;
  if ((st = cross_view(K, s->B, s->Hk, s->N, s->d, false, a.K)) != VC_OK) return st;
  if ((st = cross_view(V, s->B, s->Hk, s->N, s->d, false, a.V)) != VC_OK) return st;
  if (k_len && !aligned(k_len, 4)) return VC_ERR_ALIGN;
  if (o->masked && !k_mask) return VC_ERR_NULL;
  if (!o->masked && k_mask) return VC_ERR_UNSUPPORTED;
  if (k_mask && s->B > 1 && stride != 0 && stride < s->N) return VC_ERR_SHAPE;
  a.k_len = k_len;
  const size_t need = cross_args(s, o, backward, ws, a);
  if (need > 0 && (!ws || ws_bytes < need)) return VC_ERR_WORKSPACE;
  if (need > 0 && !aligned(ws, 16)) return VC_ERR_ALIGN;
  return VC_OK;
}

// the list of the keys that count, where there is a mask
vc_status cross_keys(const vc::CrossArgs& a, const uint8_t* k_mask, int64_t stride, hipStream_t s) {
  if (!k_mask) return VC_OK;
  return vc::hip_status(vc::launch_cross_keys(k_mask, stride, a.k_len, a.B, a.N, const_cast<int32_t*>(a.idx),
                                              const_cast<int32_t*>(a.count), s));
}

}  // namespace

extern "C" {

size_t vc_cross_attn_workspace_size(const vc_cross_shape* shape, const vc_cross_opts* opts, int32_t backward) {
  if (check_cross(shape, opts) != VC_OK) return (size_t)-1;
  vc::CrossArgs a{};
  return cross_args(shape, opts, backward != 0, nullptr, a);
}

vc_status vc_cross_attn_forward(const vc_cross_shape* shape, const vc_cross_opts* opts, const vc_view* Q,
                                const vc_view* K, const vc_view* V, const int32_t* k_len, const uint8_t* k_mask,
                                int64_t k_mask_stride, const vc_view* O, float* lse, void* ws, size_t ws_bytes,
                                void* stream) {
  vc::CrossArgs a{};
  vc_status st = cross_inputs(shape, opts, Q, K, V, k_len, k_mask, k_mask_stride, ws, ws_bytes, false, a);
  if (st != VC_OK) return st;
  if ((st = cross_view(O, shape->B, shape->Hq, shape->M, shape->d, true, a.O)) != VC_OK) return st;
  if (lse && !aligned(lse, 4)) return VC_ERR_ALIGN;
  a.lse = lse;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if ((st = cross_keys(a, k_mask, k_mask_stride, s)) != VC_OK) return st;
  return vc::hip_status(vc::launch_cross_forward(a, s));
}

vc_status vc_cross_attn_backward(const vc_cross_shape* shape, const vc_cross_opts* opts, const vc_view* Q,
                                 const vc_view* K, const vc_view* V, const int32_t* k_len, const uint8_t* k_mask,
                                 int64_t k_mask_stride, const vc_view* O, const float* lse, const vc_view* dO,
                                 const vc_view* dQ, const vc_view* dK, const vc_view* dV, void* ws, size_t ws_bytes,
                                 void* stream) {
  vc::CrossArgs a{};
  vc_status st = cross_inputs(shape, opts, Q, K, V, k_len, k_mask, k_mask_stride, ws, ws_bytes, true, a);
  if (st != VC_OK) return st;
  const int B = shape->B, Hq = shape->Hq, Hk = shape->Hk, M = shape->M, N = shape->N, d = shape->d;
  if (O && (st = cross_view(O, B, Hq, M, d, false, a.O)) != VC_OK) return st;
  if ((st = cross_view(dO, B, Hq, M, d, false, a.dO)) != VC_OK) return st;
  if ((st = cross_view(dQ, B, Hq, M, d, true, a.dQ)) != VC_OK) return st;
  if ((st = cross_view(dK, B, Hk, N, d, true, a.dK)) != VC_OK) return st;
  if ((st = cross_view(dV, B, Hk, N, d, true, a.dV)) != VC_OK) return st;
  if (!lse) return VC_ERR_NULL;
  if (!aligned(lse, 4)) return VC_ERR_ALIGN;
  a.lse = const_cast<float*>(lse);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  if ((st = cross_keys(a, k_mask, k_mask_stride, s)) != VC_OK) return st;
  return vc::hip_status(vc::launch_cross_backward(a, s));
}

vc_status vc_norm_rope(const vc_norm_rope_shape* shape, const vc_norm_rope_opts* opts, const vc_view* q,
                       const vc_view* k, const float* q_weight, const float* k_weight, const float* rope_cos,
                       const float* rope_sin, const int32_t* pos, const vc_view* q_out, const vc_view* k_out,
                       void* stream) {
  vc_status st = check_norm_rope(shape, opts);
  if (st != VC_OK) return st;
  vc::NormRopeArgs a{};
  if ((st = norm_rope_args(shape, opts, rope_cos, rope_sin, pos, a)) != VC_OK) return st;
  const int B = shape->B, N = shape->N, d = shape->d, heads[2] = {shape->Hq, shape->Hk};
  const vc_view *in[2] = {q, k}, *out[2] = {q_out, k_out};
  const float* weight[2] = {q_weight, k_weight};
  for (int i = 0; i < a.ntensors; ++i) {
    vc::NormRopeTensor& t = a.t[i];
    if ((st = check_view(in[i], B, heads[i], N, d, false)) != VC_OK) return st;
    if ((st = check_view(out[i], B, heads[i], N, d, true)) != VC_OK) return st;
    if (weight[i] && !aligned(weight[i], 16)) return VC_ERR_ALIGN;
    t.in = static_cast<const uint16_t*>(in[i]->data);
    t.out = static_cast<uint16_t*>(out[i]->data);
    strides(in[i], B, heads[i], N, t.in_sb, t.in_sh, t.in_sn);
    strides(out[i], B, heads[i], N, t.out_sb, t.out_sh, t.out_sn);
    t.weight = opts->norm == VC_NORM_NONE ? nullptr : weight[i];
    t.H = heads[i];
    t.weights = norm_weights(opts, t.H, d);
    t.inv_span = 1.f / (float)t.weights;
  }
  return vc::hip_status(vc::launch_norm_rope(a, static_cast<hipStream_t>(stream)));
}

size_t vc_norm_rope_workspace_size(const vc_norm_rope_shape* shape, const vc_norm_rope_opts* opts) {
  if (check_norm_rope(shape, opts) != VC_OK) return (size_t)-1;
  if (opts->norm == VC_NORM_NONE) return 0;
  const size_t C = norm_weights(opts, shape->Hq, shape->d) + (shape->Hk ? norm_weights(opts, shape->Hk, shape->d) : 0);
  return C * 4 * vc::norm_rope_parts((int64_t)shape->B * shape->N, shape->Hk ? 2 : 1);
}

vc_status vc_norm_rope_backward(const vc_norm_rope_shape* shape, const vc_norm_rope_opts* opts, const vc_view* q,
                                const vc_view* k, const float* q_weight, const float* k_weight, const float* rope_cos,
                                const float* rope_sin, const int32_t* pos, const vc_view* dq_out,
                                const vc_view* dk_out, const vc_view* dq, const vc_view* dk, float* dq_weight,
                                float* dk_weight, void* ws, size_t ws_bytes, void* stream) {
  vc_status st = check_norm_rope(shape, opts);
  if (st != VC_OK) return st;
  vc::NormRopeArgs a{};
  if ((st = norm_rope_args(shape, opts, rope_cos, rope_sin, pos, a)) != VC_OK) return st;
  const bool norm = opts->norm != VC_NORM_NONE;
  if (!norm && (dq_weight || dk_weight)) return VC_ERR_UNSUPPORTED;
  const int B = shape->B, N = shape->N, d = shape->d, heads[2] = {shape->Hq, shape->Hk};
  const vc_view *in[2] = {q, k}, *grad[2] = {dq_out, dk_out}, *out[2] = {dq, dk};
  const float* weight[2] = {q_weight, k_weight};
  float* dw[2] = {dq_weight, dk_weight};
  if (dq_weight || (dk_weight && a.ntensors == 2)) {
    if (!ws || ws_bytes < vc_norm_rope_workspace_size(shape, opts)) return VC_ERR_WORKSPACE;
    if (!aligned(ws, 16)) return VC_ERR_ALIGN;
  }
  float* part = static_cast<float*>(ws);
  for (int i = 0; i < a.ntensors; ++i) {
    vc::NormRopeTensor& t = a.t[i];
    if (norm && (st = check_view(in[i], B, heads[i], N, d, false)) != VC_OK) return st;
    if ((st = check_view(grad[i], B, heads[i], N, d, false)) != VC_OK) return st;
    if ((st = check_view(out[i], B, heads[i], N, d, true)) != VC_OK) return st;
    if ((weight[i] && !aligned(weight[i], 16)) || (dw[i] && !aligned(dw[i], 16))) return VC_ERR_ALIGN;
    if (norm) {
      t.in = static_cast<const uint16_t*>(in[i]->data);
      strides(in[i], B, heads[i], N, t.in_sb, t.in_sh, t.in_sn);
    }
    t.grad = static_cast<const uint16_t*>(grad[i]->data);
    t.out = static_cast<uint16_t*>(out[i]->data);
    strides(grad[i], B, heads[i], N, t.grad_sb, t.grad_sh, t.grad_sn);
    strides(out[i], B, heads[i], N, t.out_sb, t.out_sh, t.out_sn);
    t.weight = norm ? weight[i] : nullptr;
    t.H = heads[i];
    t.weights = norm_weights(opts, t.H, d);
    t.inv_span = 1.f / (float)t.weights;
    t.dw = dw[i];
    if (dw[i]) {
      t.dw_part = part;
      part += (size_t)t.weights * vc::norm_rope_parts(a.tokens, a.ntensors);
    }
  }
  if (!norm) {
    // the rotation's gradient: the rotation with the sines negated
    for (int i = 0; i < a.ntensors; ++i) {
      vc::NormRopeTensor& t = a.t[i];
      t.in = t.grad;
      t.in_sb = t.grad_sb, t.in_sh = t.grad_sh, t.in_sn = t.grad_sn;
    }
    a.sign = -1.f;
    return vc::hip_status(vc::launch_norm_rope(a, static_cast<hipStream_t>(stream)));
  }
  return vc::hip_status(vc::launch_norm_rope_backward(a, static_cast<hipStream_t>(stream)));
}

vc_status vc_rope_line_tables(int32_t rows, int32_t rot, double theta, const vc_rope_scaling* scaling, float* cos_t,
                              float* sin_t) {
  if (!cos_t || !sin_t) return VC_ERR_NULL;
  if (rows < 1 || rot < 16 || rot > 128 || rot % 16 != 0 || (int64_t)rows * (rot / 2) >= (1LL << 31))
    return VC_ERR_SHAPE;
  if (!(theta > 0.0) || !std::isfinite(theta)) return VC_ERR_SHAPE;
  const int half = rot / 2;
  double magnitude = 1.0, freq[64];
  for (int i = 0; i < half; ++i) freq[i] = std::pow(theta, -2.0 * i / rot);
  if (scaling) {
    const vc_rope_scaling& c = *scaling;
    if (c.kind < VC_SCALE_NONE || c.kind > VC_SCALE_PARTS) return VC_ERR_UNSUPPORTED;
    if (c.kind != VC_SCALE_NONE && !(c.factor >= 1.0 && std::isfinite(c.factor))) return VC_ERR_UNSUPPORTED;
    if (!(c.magnitude >= 0.0) || !std::isfinite(c.magnitude)) return VC_ERR_UNSUPPORTED;
    if (c.magnitude > 0.0) magnitude = c.magnitude;
    if (c.kind == VC_SCALE_LINEAR)
      for (int i = 0; i < half; ++i) freq[i] /= c.factor;
    if (c.kind == VC_SCALE_BASE) {
      const double base = theta * std::pow(c.factor, (double)rot / (rot - 2));
      for (int i = 0; i < half; ++i) freq[i] = std::pow(base, -2.0 * i / rot);
    }
    if (c.kind == VC_SCALE_PARTS) {
      if (!(c.trained >= 1.0 && std::isfinite(c.trained) && c.slow >= 0.0 && c.fast > c.slow && std::isfinite(c.fast)))
        return VC_ERR_UNSUPPORTED;
      for (int i = 0; i < half; ++i) {
        const double turns = c.trained * freq[i] / 6.283185307179586476925;
        double keep = (turns - c.slow) / (c.fast - c.slow);
        keep = keep < 0.0 ? 0.0 : (keep > 1.0 ? 1.0 : keep);
        freq[i] = freq[i] * keep + freq[i] / c.factor * (1.0 - keep);
      }
    }
  }
  for (int p = 0; p < rows; ++p)
    for (int i = 0; i < half; ++i) {
      const double ang = (double)p * freq[i];
      cos_t[(size_t)p * half + i] = (float)(std::cos(ang) * magnitude);
      sin_t[(size_t)p * half + i] = (float)(std::sin(ang) * magnitude);
    }
  return VC_OK;
}

}  // extern "C"
