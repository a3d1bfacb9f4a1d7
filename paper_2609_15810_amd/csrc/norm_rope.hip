// RMS norms of queries and keys with the rotation by position in the same pass, and their gradients.
//
// A row is one head of one token, x of d channels. With the norm's span S (the head's d channels, or all
// H d channels of the token) and weights w,
//   r = 1 / sqrt(mean_S(x^2) + eps),  y = x r w,  z = R(pos) y,
// where R turns the pairs of the first `rot` channels by the token's angles. With g = R^T dz,
//   dw = sum over rows of g x r,  dx = r (g w - x r^2 mean_S(g w x)).
// R^T is R with the sines negated (also where the tables carry a factor), so the gradient of the rotation
// alone is the forward kernel with that sign.
//
// Everything is bound by memory: 2 bytes read and 2 written per element (backward: 4 and 2), and the tables.
// So a lane holds 16 channels of a row as two 16-byte pieces, d/16 lanes a row, chosen such that both channels
// of every pair are in one lane: in the half layout pieces j and j + rot/16, which hold channels c and
// c + rot/2; in the interleaved layout pieces j and j + d/16. The sums of a norm are exchanges among the lanes of
// the row (or token). A wave works on 64/(16 or 8) = 8 or more rows at once: P slots of d/16 lanes each belong to
// one token, the remaining factor is over tokens, so that a token's table row is read once per wave and
// held for its heads. All sums are fp32, outputs are rounded once.
#include "vc_common.hpp"
#include "vc_internal.hpp"

namespace vc {
namespace {

constexpr int WAVES = 4;   // of a workgroup; they share nothing but the backward's weight sums

template <int DT>
__device__ __forceinline__ void unpack8(const u4& raw, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT == VC_BF16) {
      x[2 * i] = bf16_lo(raw[i]);
      x[2 * i + 1] = bf16_hi(raw[i]);
    } else {
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      const uint32_t w = raw[i];   // a bit cast of the element itself is compiled into one of element 0
      const v2f f = __builtin_convertvector(__builtin_bit_cast(h2, w), v2f);
      x[2 * i] = f[0];
      x[2 * i + 1] = f[1];
    }
  }
}

template <int DT>
__device__ __forceinline__ u4 pack8(const float* x) {
  u4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
  return out;
}

__device__ __forceinline__ void load8f(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// The channels of a lane: two pieces of 8, starting at c0 and c1; which of its pairs are turned
struct Lane {
  int c0, c1;       // first channels of its pieces
  bool turn0, turn1;
};
template <int D, int LAYOUT>
__device__ __forceinline__ Lane lane_channels(int j, int rot) {
  constexpr int G = D / 16;
  Lane l;
  if (LAYOUT == VC_ROPE_HALF) {
    const int rc = rot / 16;
    l.turn0 = l.turn1 = j < rc;
    l.c0 = j < rc ? 8 * j : 16 * j;            // behind the turned part the pieces stand in order
    l.c1 = j < rc ? 8 * (j + rc) : 16 * j + 8;
  } else {
    l.c0 = 8 * j;
    l.c1 = 8 * (j + G);
    l.turn0 = l.c0 < rot;
    l.turn1 = l.c1 < rot;
  }
  return l;
}

// cos and sin of a lane's eight pairs (1 and 0 where its channels are not turned). Pair p stands in column p of
// the table row of its axis; on a line all axes are the one row. Pairs of a lane: half layout c0 .. c0 + 7;
// interleaved c0/2 .. + 3 and c1/2 .. + 3.
template <int LAYOUT>
__device__ __forceinline__ void load_angles(const NormRopeArgs& a, const Lane& l, int n, int b, float sign, float* cs,
                                            float* sn) {
#pragma unroll
  for (int i = 0; i < 8; ++i) cs[i] = 1.f, sn[i] = 0.f;
  if (LAYOUT == VC_ROPE_NONE) return;
  const int p0 = LAYOUT == VC_ROPE_HALF ? l.c0 : l.c0 >> 1;
  const int p1 = LAYOUT == VC_ROPE_HALF ? l.c0 + 4 : l.c1 >> 1;
  const int half = a.rot >> 1;
  if (!a.grid) {
    const int64_t row = clamp_index(a.pos ? a.pos[(size_t)b * a.N + n] : n, a.rows);
    const float *c = a.cos_t + row * half, *s = a.sin_t + row * half;
    if (l.turn0) {
      const float4 v = *reinterpret_cast<const float4*>(c + p0), w = *reinterpret_cast<const float4*>(s + p0);
      cs[0] = v.x, cs[1] = v.y, cs[2] = v.z, cs[3] = v.w;
      sn[0] = w.x, sn[1] = w.y, sn[2] = w.z, sn[3] = w.w;
    }
    if (l.turn1) {
      const float4 v = *reinterpret_cast<const float4*>(c + p1), w = *reinterpret_cast<const float4*>(s + p1);
      cs[4] = v.x, cs[5] = v.y, cs[6] = v.z, cs[7] = v.w;
      sn[4] = w.x, sn[5] = w.y, sn[6] = w.z, sn[7] = w.w;
    }
  } else {
    // frame, row and column of the token; a group of four pairs meets at most two axes
    const int hw = a.Ht * a.Wd, f = n / hw, rest = n - f * hw, y = rest / a.Wd, x = rest - y * a.Wd;
    const int at[3] = {f * 64, (a.F + y) * 64, (a.F + a.Ht + x) * 64};
    auto pick = [&](int axis) { return axis == 0 ? at[0] : (axis == 1 ? at[1] : at[2]); };
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int p = q ? p1 : p0;
      const int first = rope_axis(p), last = rope_axis(p + 3);
      const int ra = pick(first) + p, rb = pick(last) + p;
      const float4 ca = *reinterpret_cast<const float4*>(a.cos_t + ra), sa = *reinterpret_cast<const float4*>(a.sin_t + ra);
      const float4 cb = *reinterpret_cast<const float4*>(a.cos_t + rb), sb = *reinterpret_cast<const float4*>(a.sin_t + rb);
      const bool s1 = rope_axis(p + 1) == first, s2 = rope_axis(p + 2) == first;
      cs[4 * q] = ca.x, sn[4 * q] = sa.x;
      cs[4 * q + 1] = s1 ? ca.y : cb.y, sn[4 * q + 1] = s1 ? sa.y : sb.y;
      cs[4 * q + 2] = s2 ? ca.z : cb.z, sn[4 * q + 2] = s2 ? sa.z : sb.z;
      cs[4 * q + 3] = cb.w, sn[4 * q + 3] = sb.w;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sn[i] *= sign;
}

// turn the pairs of x (16 channels: piece 0, then piece 1)
template <int LAYOUT>
__device__ __forceinline__ void turn(float* x, const float* cs, const float* sn) {
  if (LAYOUT == VC_ROPE_NONE) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int ia = LAYOUT == VC_ROPE_HALF ? i : 2 * i, ib = LAYOUT == VC_ROPE_HALF ? i + 8 : 2 * i + 1;
    const float u = x[ia], v = x[ib];
    x[ia] = __builtin_fmaf(u, cs[i], -v * sn[i]);
    x[ib] = __builtin_fmaf(u, sn[i], v * cs[i]);
  }
}

// sum over the `n` lanes (a power of two) that a lane shares a span with
__device__ __forceinline__ float lanes_sum(float v, int n) {
  for (int o = 1; o < n; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Where a wave's slots stand: slot = lane / (d/16); token slot / P of the wave's 64/(d/16)/P, head slot % P
struct Place {
  int j, b, n, head;   // lane in its row, batch item, token, first head
  bool live;
};
template <int D>
__device__ __forceinline__ Place place(const NormRopeArgs& a, int P, int64_t group, int head0) {
  constexpr int G = D / 16, SLOTS = 64 / G;
  const int lane = threadIdx.x & 63, slot = lane / G;
  Place p;
  p.j = lane % G;
  const int tokens = SLOTS / P;
  const int64_t t = group * tokens + slot / P;
  p.head = head0 + (slot & (P - 1));
  p.live = t < a.tokens;
  const int64_t tt = p.live ? t : a.tokens - 1;
  p.b = (int)(tt / a.N);
  p.n = (int)(tt - (int64_t)p.b * a.N);
  return p;
}

// One wave: the heads head0, head0 + P, .. of its tokens, at most `heads` iterations, NB of them in flight at once.
// A norm over the token needs all heads in one batch (heads <= NB).
template <int DT, int D, int NORM, int LAYOUT, int NB>
__global__ __launch_bounds__(64 * WAVES) void norm_rope_fwd(NormRopeArgs a) {
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t w = (int64_t)blockIdx.x * WAVES + wave;
  const int64_t group = w / x.parts;   // tokens of the wave; part of the heads
  const int part = (int)(w - group * x.parts);
  constexpr int G = D / 16, SLOTS = 64 / G;
  const int P = x.P;
  if (group * (SLOTS / P) >= a.tokens) return;
  const Place p = place<D>(a, P, group, part * x.iters * P);
  const int end = min(x.H, (part + 1) * x.iters * P);
  const Lane l = lane_channels<D, LAYOUT>(p.j, a.rot);
  const uint16_t* in = x.in + p.b * x.in_sb + p.n * x.in_sn;
  uint16_t* out = x.out + p.b * x.out_sb + p.n * x.out_sn;
  float cs[8], sn[8], wt[16];
  u4 raw[NB][2];
  auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = h0 + i * P;
      if (p.live && h < end) {
        const uint16_t* row = in + h * x.in_sh;
        raw[i][0] = *reinterpret_cast<const u4*>(row + l.c0);
        raw[i][1] = *reinterpret_cast<const u4*>(row + l.c1);
      } else {
        raw[i][0] = raw[i][1] = u4{0, 0, 0, 0};
      }
    }
  };
  load(p.head);
  load_angles<LAYOUT>(a, l, p.n, p.b, a.sign, cs, sn);
  if (NORM == VC_NORM_HEAD && x.weight) {
    load8f(x.weight + l.c0, wt);
    load8f(x.weight + l.c1, wt + 8);
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) wt[e] = 1.f;
  }
  for (int h0 = p.head; ; ) {
    float ss = 0.f;
    if (NORM == VC_NORM_TOKEN) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        float v[16];
        unpack8<DT>(raw[i][0], v);
        unpack8<DT>(raw[i][1], v + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss = __builtin_fmaf(v[e], v[e], ss);
      }
      ss = lanes_sum(ss, G * P);
    }
    float r = NORM == VC_NORM_TOKEN ? __builtin_amdgcn_rsqf(__builtin_fmaf(ss, x.inv_span, a.eps)) : 1.f;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = h0 + i * P;
      float v[16];
      unpack8<DT>(raw[i][0], v);
      unpack8<DT>(raw[i][1], v + 8);
      if (NORM == VC_NORM_HEAD) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s = __builtin_fmaf(v[e], v[e], s);
        r = __builtin_amdgcn_rsqf(__builtin_fmaf(lanes_sum(s, G), x.inv_span, a.eps));
      }
      const bool on = p.live && h < end;
      if (NORM == VC_NORM_TOKEN && x.weight && on) {
        load8f(x.weight + h * D + l.c0, wt);
        load8f(x.weight + h * D + l.c1, wt + 8);
      }
      if (NORM != VC_NORM_NONE) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] * r * wt[e];
      }
      turn<LAYOUT>(v, cs, sn);
      if (on) {
        uint16_t* row = out + h * x.out_sh;
        *reinterpret_cast<u4*>(row + l.c0) = pack8<DT>(v);
        *reinterpret_cast<u4*>(row + l.c1) = pack8<DT>(v + 8);
      }
    }
    h0 += NB * P;
    if (NORM == VC_NORM_TOKEN || h0 - p.head + part * x.iters * P >= end) break;   // the same for all lanes
    load(h0);
  }
}

// Gradients. Waves walk over the tokens (groups wave, wave + waves of the grid, ..), so that the sums of the
// weights' gradients stay in registers; a workgroup's waves add theirs in LDS one after the other, in a fixed order,
// and write one row of partial sums, which norm_rope_join adds up in a fixed order.
template <int DT, int D, int NORM, int LAYOUT, int NB>
__global__ __launch_bounds__(64 * WAVES) void norm_rope_bwd(NormRopeArgs a) {
  extern __shared__ float acc[];
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int G = D / 16, SLOTS = 64 / G;
  constexpr int ND = NORM == VC_NORM_TOKEN ? NB : 1;   // weights that a lane meets: its 16 channels of so many heads
  const int P = x.P, tokens = SLOTS / P;
  const int64_t groups = (a.tokens + tokens - 1) / tokens;
  float dw[ND][16], wt[16];
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f;
  const int lane = threadIdx.x & 63, j = lane % G;
  const Lane l = lane_channels<D, LAYOUT>(j, a.rot);
#pragma unroll
  for (int e = 0; e < 16; ++e) wt[e] = 1.f;
  if (NORM == VC_NORM_HEAD && x.weight) {
    load8f(x.weight + l.c0, wt);
    load8f(x.weight + l.c1, wt + 8);
  }
  for (int64_t group = (int64_t)blockIdx.x * WAVES + wave; group < groups; group += (int64_t)gridDim.x * WAVES) {
    const Place p = place<D>(a, P, group, 0);
    const uint16_t* in = x.in + p.b * x.in_sb + p.n * x.in_sn;
    const uint16_t* gin = x.grad + p.b * x.grad_sb + p.n * x.grad_sn;
    uint16_t* out = x.out + p.b * x.out_sb + p.n * x.out_sn;
    float cs[8], sn[8];
    bool angles = false;
    for (int h0 = p.head;;) {
      u4 raw[NB][2], gr[NB][2];
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int h = h0 + i * P;
        raw[i][0] = raw[i][1] = gr[i][0] = gr[i][1] = u4{0, 0, 0, 0};
        if (p.live && h < x.H) {
          raw[i][0] = *reinterpret_cast<const u4*>(in + h * x.in_sh + l.c0);
          raw[i][1] = *reinterpret_cast<const u4*>(in + h * x.in_sh + l.c1);
          gr[i][0] = *reinterpret_cast<const u4*>(gin + h * x.grad_sh + l.c0);
          gr[i][1] = *reinterpret_cast<const u4*>(gin + h * x.grad_sh + l.c1);
        }
      }
      if (!angles) load_angles<LAYOUT>(a, l, p.n, p.b, -1.f, cs, sn);
      angles = true;
      auto weights = [&](int h) __attribute__((always_inline)) {
        if (NORM == VC_NORM_TOKEN && x.weight && h < x.H) {
          load8f(x.weight + h * D + l.c0, wt);
          load8f(x.weight + h * D + l.c1, wt + 8);
        }
      };
      auto values = [&](int i, float* v, float* g) __attribute__((always_inline)) {
        unpack8<DT>(raw[i][0], v);
        unpack8<DT>(raw[i][1], v + 8);
        unpack8<DT>(gr[i][0], g);
        unpack8<DT>(gr[i][1], g + 8);
        turn<LAYOUT>(g, cs, sn);
      };
      float r = 0.f, k = 0.f;   // r, and r^3 mean(g w x)
      auto sums = [&](float ss, float dot, int lanes) __attribute__((always_inline)) {
        ss = lanes_sum(ss, lanes);
        dot = lanes_sum(dot, lanes);
        r = __builtin_amdgcn_rsqf(__builtin_fmaf(ss, x.inv_span, a.eps));
        k = r * r * r * (dot * x.inv_span);
      };
      if (NORM == VC_NORM_TOKEN) {
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          float v[16], g[16];
          values(i, v, g);
          weights(h0 + i * P);
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            ss = __builtin_fmaf(v[e], v[e], ss);
            dot = __builtin_fmaf(v[e] * wt[e], g[e], dot);
          }
        }
        sums(ss, dot, G * P);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int h = h0 + i * P;
        float v[16], g[16];
        values(i, v, g);
        weights(h);
        if (NORM == VC_NORM_HEAD) {
          float ss = 0.f, dot = 0.f;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            ss = __builtin_fmaf(v[e], v[e], ss);
            dot = __builtin_fmaf(v[e] * wt[e], g[e], dot);
          }
          sums(ss, dot, G);
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int id = NORM == VC_NORM_TOKEN ? i : 0;
          dw[id][e] = __builtin_fmaf(g[e] * r, v[e], dw[id][e]);
          g[e] = __builtin_fmaf(-k, v[e], g[e] * wt[e] * r);
        }
        if (p.live && h < x.H) {
          *reinterpret_cast<u4*>(out + h * x.out_sh + l.c0) = pack8<DT>(g);
          *reinterpret_cast<u4*>(out + h * x.out_sh + l.c1) = pack8<DT>(g + 8);
        }
      }
      h0 += NB * P;
      if (NORM == VC_NORM_TOKEN || h0 - p.head >= x.H) break;
    }
  }
  if (!x.dw_part) return;
  // slots that share their channels: all of the wave (a head's norm), or those of its other tokens
  const int share = NORM == VC_NORM_HEAD ? G : G * P;
#pragma unroll
  for (int i = 0; i < ND; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      for (int o = share; o < 64; o <<= 1) dw[i][e] += __shfl_xor(dw[i][e], o, 64);
  const int C = NORM == VC_NORM_HEAD ? D : x.H * D;
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave && lane < share) {
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        const int h = NORM == VC_NORM_HEAD ? 0 : lane / G + i * P;
        if (NORM == VC_NORM_HEAD || h < x.H) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int c = h * D + (e < 8 ? l.c0 + e : l.c1 + e - 8);
            acc[c] = w == 0 ? dw[i][e] : acc[c] + dw[i][e];
          }
        }
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < C; c += 64 * WAVES) x.dw_part[(size_t)blockIdx.x * C + c] = acc[c];
}

// dw[c] = sum of the partial rows: 16 channels a workgroup, 16 threads a channel walk the rows, a tree adds them
__global__ __launch_bounds__(256) void norm_rope_join(NormRopeArgs a, int parts) {
  __shared__ float s[16][17];
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int C = x.weights;
  const int cc = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + cc;
  float v = 0.f;
  if (x.dw_part && c < C)
    for (int p = row; p < parts; p += 16) v += x.dw_part[(size_t)p * C + c];
  s[row][cc] = v;
  __syncthreads();
  for (int o = 8; o > 0; o >>= 1) {
    if (row < o) s[row][cc] += s[row + o][cc];
    __syncthreads();
  }
  if (row == 0 && x.dw_part && c < C) x.dw[c] = s[0][cc];
}

template <int DT, int D, int NORM, int LAYOUT, int NB, bool BWD>
hipError_t launch(const NormRopeArgs& a, int grid, size_t lds, hipStream_t s) {
  const dim3 g((unsigned)grid, (unsigned)a.ntensors);
  if constexpr (BWD) norm_rope_bwd<DT, D, NORM, LAYOUT, NB><<<g, 64 * WAVES, lds, s>>>(a);
  else norm_rope_fwd<DT, D, NORM, LAYOUT, NB><<<g, 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

template <int DT, int D, int NORM, int LAYOUT, bool BWD>
hipError_t launch_nb(const NormRopeArgs& a, int nb, int grid, size_t lds, hipStream_t s) {
  if constexpr (NORM == VC_NORM_TOKEN) {
    if (nb <= 1) return launch<DT, D, NORM, LAYOUT, 1, BWD>(a, grid, lds, s);
    if (nb <= 2) return launch<DT, D, NORM, LAYOUT, 2, BWD>(a, grid, lds, s);
    if (nb <= 4) return launch<DT, D, NORM, LAYOUT, 4, BWD>(a, grid, lds, s);
    if (nb <= 5) return launch<DT, D, NORM, LAYOUT, 5, BWD>(a, grid, lds, s);
    return launch<DT, D, NORM, LAYOUT, 8, BWD>(a, grid, lds, s);
  } else {
    if (nb <= 1) return launch<DT, D, NORM, LAYOUT, 1, BWD>(a, grid, lds, s);
    return launch<DT, D, NORM, LAYOUT, 2, BWD>(a, grid, lds, s);
  }
}

template <int DT, int D, int NORM, bool BWD>
hipError_t launch_layout(const NormRopeArgs& a, int nb, int grid, size_t lds, hipStream_t s) {
  if (a.layout == VC_ROPE_HALF) return launch_nb<DT, D, NORM, VC_ROPE_HALF, BWD>(a, nb, grid, lds, s);
  if (a.layout == VC_ROPE_INTERLEAVED) return launch_nb<DT, D, NORM, VC_ROPE_INTERLEAVED, BWD>(a, nb, grid, lds, s);
  if constexpr (NORM != VC_NORM_NONE) return launch_nb<DT, D, NORM, VC_ROPE_NONE, BWD>(a, nb, grid, lds, s);
  return hipErrorInvalidValue;
}

template <int DT, int D, bool BWD>
hipError_t launch_norm(const NormRopeArgs& a, int nb, int grid, size_t lds, hipStream_t s) {
  if (a.norm == VC_NORM_HEAD) return launch_layout<DT, D, VC_NORM_HEAD, BWD>(a, nb, grid, lds, s);
  if (a.norm == VC_NORM_TOKEN) return launch_layout<DT, D, VC_NORM_TOKEN, BWD>(a, nb, grid, lds, s);
  if constexpr (!BWD) return launch_layout<DT, D, VC_NORM_NONE, BWD>(a, nb, grid, lds, s);
  return hipErrorInvalidValue;
}

template <bool BWD>
hipError_t dispatch(const NormRopeArgs& a, int nb, int grid, size_t lds, hipStream_t s) {
  if (a.d == 128)
    return a.dtype == VC_BF16 ? launch_norm<VC_BF16, 128, BWD>(a, nb, grid, lds, s)
                              : launch_norm<VC_FP16, 128, BWD>(a, nb, grid, lds, s);
  return a.dtype == VC_BF16 ? launch_norm<VC_BF16, 64, BWD>(a, nb, grid, lds, s)
                            : launch_norm<VC_FP16, 64, BWD>(a, nb, grid, lds, s);
}

// slots of a wave that a token's heads take: as many as there are heads, up to the whole wave
int slots_of(int H, int d) {
  const int most = 64 / (d / 16);
  int P = 1;
  while (P < most && P < H) P *= 2;
  return P;
}

}  // namespace

int norm_rope_parts(int64_t tokens) {
  // workgroups of the backward kernel, each of which leaves a row of partial weight sums
  const int64_t w = (tokens + 4 * WAVES - 1) / (4 * WAVES);
  return (int)(w < 1 ? 1 : (w > 1024 ? 1024 : w));
}

hipError_t launch_norm_rope(NormRopeArgs a, hipStream_t s) {
  int64_t grid = 1;
  int nb = 1;
  for (int i = 0; i < a.ntensors; ++i) {
    NormRopeTensor& t = a.t[i];
    t.P = slots_of(t.H, a.d);
    const int tokens = 64 / (a.d / 16) / t.P, iters = (t.H + t.P - 1) / t.P;
    const int64_t groups = (a.tokens + tokens - 1) / tokens;
    // few tokens: the heads of a token go to several waves
    t.parts = a.norm != VC_NORM_TOKEN && groups * iters <= 4096 ? iters : 1;
    t.iters = (iters + t.parts - 1) / t.parts;
    nb = t.iters > nb ? t.iters : nb;
    const int64_t g = (groups * t.parts + WAVES - 1) / WAVES;
    grid = g > grid ? g : grid;
  }
  return dispatch<false>(a, nb, (int)grid, 0, s);
}

hipError_t launch_norm_rope_backward(NormRopeArgs a, hipStream_t s) {
  int nb = 1, C = 0;
  bool weights = false;
  for (int i = 0; i < a.ntensors; ++i) {
    NormRopeTensor& t = a.t[i];
    t.P = slots_of(t.H, a.d);
    t.parts = 1;
    t.iters = (t.H + t.P - 1) / t.P;
    nb = t.iters > nb ? t.iters : nb;
    C = t.weights > C ? t.weights : C;
    weights = weights || t.dw_part;
  }
  const int parts = norm_rope_parts(a.tokens);
  hipError_t e = dispatch<true>(a, nb, parts, (size_t)C * 4, s);
  if (e != hipSuccess || !weights) return e;
  norm_rope_join<<<dim3((unsigned)((C + 15) / 16), (unsigned)a.ntensors), 256, 0, s>>>(a, parts);
  return hipGetLastError();
}

}  // namespace vc
