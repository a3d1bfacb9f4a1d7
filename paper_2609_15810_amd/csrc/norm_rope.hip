// RMS norms of queries and keys with the rotation by position in the same pass, and their gradients.
//
// A row is one head of one token, x of d channels. With the norm's span S (the head's d channels, or all
// H d channels of the token) and weights w,
//   r = 1 / sqrt(mean_S(x^2) + eps),  y = x r w,  z = R(pos) y,
// where R turns the pairs of the first `rot` channels by the token's angles. With g = R^T dz,
//   dw = sum over rows of g u,  dx = r (g w - u mean_S(g w u)),  u = x r.
// R^T is R with the sines negated (also where the tables carry a factor), so the gradient of the rotation
// alone is the forward kernel with that sign.
//
// Everything is bound by memory: 2 bytes read and 2 written per element (backward: 4 and 2), and the tables.
// So a lane holds 16 channels of a row as two 16-byte pieces, d/16 lanes a row, chosen such that both channels
// of every pair are in one lane: in the half layout pieces j and j + rot/16, which hold channels c and
// c + rot/2; in the interleaved layout pieces j and j + d/16. The sums of a norm are exchanges among the lanes of
// the row (or token). A wave works on 8 rows (d = 128; 16 of d = 64) at once: P slots of d/16 lanes each belong to one
// token, the remaining factor is over tokens, so that a token's table row is read once and held for its heads. A norm
// over more heads than two rounds of a wave's slots takes 2 or 4 waves a token, whose sums meet in LDS. All sums are
// fp32, outputs are rounded once.
#include "lanes.hpp"
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

// The channels of a lane: two pieces of 8, starting at c0 and c1; which of its pairs are turned
struct Lane {
  int c0, c1;       // first channels of its pieces
  bool turn0, turn1;
};

// A row's two pieces. Results of large calls are stored past the caches (past_caches)
__device__ __forceinline__ void store_row(uint16_t* row, const Lane& l, u4 lo, u4 hi, int past) {
  if (past) {
    asm volatile("" ::: "memory");   // without these, both branches become one of plain stores
    __builtin_nontemporal_store(lo, reinterpret_cast<u4*>(row + l.c0));
    __builtin_nontemporal_store(hi, reinterpret_cast<u4*>(row + l.c1));
    asm volatile("" ::: "memory");
  } else {
    *reinterpret_cast<u4*>(row + l.c0) = lo;
    *reinterpret_cast<u4*>(row + l.c1) = hi;
  }
}

__device__ __forceinline__ void load8f(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
  x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

template <int D, int LAYOUT>
__device__ __forceinline__ Lane lane_channels(int j, int rot) {
  constexpr int G = D / 16;
  Lane l;
  if (LAYOUT == VC_ROPE_HALF) {
    const int rc = rot / 16;
    l.turn0 = l.turn1 = j < rc;
    l.c0 = 8 * (j < rc ? j : j + rc);           // the pieces behind the turned part: the first half of them
    l.c1 = 8 * (j < rc ? j + rc : j + G);       // in the first pieces, the others in the second
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
      const int ra = pick(first) + p;
      const float4 ca = *reinterpret_cast<const float4*>(a.cos_t + ra), sa = *reinterpret_cast<const float4*>(a.sin_t + ra);
      float *c = cs + 4 * q, *s = sn + 4 * q;
      c[0] = ca.x, c[1] = ca.y, c[2] = ca.z, c[3] = ca.w;
      s[0] = sa.x, s[1] = sa.y, s[2] = sa.z, s[3] = sa.w;
      if (first != last) {   // in two of a row's sixteen groups: a load of few lanes
        const int rb = pick(last) + p;
        const float4 cb = *reinterpret_cast<const float4*>(a.cos_t + rb), sb = *reinterpret_cast<const float4*>(a.sin_t + rb);
        const bool s1 = rope_axis(p + 1) == first, s2 = rope_axis(p + 2) == first;
        c[1] = s1 ? c[1] : cb.y, s[1] = s1 ? s[1] : sb.y;
        c[2] = s2 ? c[2] : cb.z, s[2] = s2 ? s[2] : sb.z;
        c[3] = cb.w, s[3] = sb.w;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) sn[i] *= sign;
}

// turn the pairs of x (16 channels: piece 0, then piece 1); the channels that are not turned stay as they are (a product with
// a sine of 0 would carry an infinity or NaN from one into another)
template <int LAYOUT>
__device__ __forceinline__ void turn(float* x, const Lane& l, const float* cs, const float* sn) {
  if (LAYOUT == VC_ROPE_NONE) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int ia = LAYOUT == VC_ROPE_HALF ? i : 2 * i, ib = LAYOUT == VC_ROPE_HALF ? i + 8 : 2 * i + 1;
    const bool on = i < 4 ? l.turn0 : l.turn1;
    const float u = x[ia], v = x[ib];
    const float s = __builtin_fmaf(u, cs[i], -v * sn[i]), t = __builtin_fmaf(u, sn[i], v * cs[i]);
    x[ia] = on ? s : u;
    x[ib] = on ? t : v;
  }
}

// sum over the n lanes (4, 8, .., 64) that a lane shares a span with: exchanges in quads, mirrored in 8 and 16 lanes
// (where all lanes of a half have the same sum by then), and of the wave's quarters and halves
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lanes_sum(float v, int n) {
  v = dpp_add<0xb1>(v);                // quad_perm 1 0 3 2
  v = dpp_add<0x4e>(v);                // quad_perm 2 3 0 1
  if (n > 4) v = dpp_add<0x141>(v);    // row_half_mirror
  if (n > 8) v = dpp_add<0x140>(v);    // row_mirror
  if (n > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    uint32_t x = r[0], y = r[1];
    lanes::pin(x);
    lanes::pin(y);
    v = __uint_as_float(x) + __uint_as_float(y);
  }
  if (n > 32) v = lanes::half_sum(v);
  return v;
}

// Where a wave's slots stand. A workgroup's waves form WAVES / W teams of W waves; a team works on one group of
// tokens: one token where P, the slots of a token, is all of the team's, else 64 / (d/16) / P of them.
struct Place {
  int b, n, head;   // batch item, token, first head
  int live;         // 0: behind the last token
};
template <int D>
__device__ __forceinline__ Place place(const NormRopeArgs& a, const NormRopeTensor& x, int wave, uint32_t group, int head0) {
  constexpr int G = D / 16, SLOTS = 64 / G;
  const int slot = (wave & (x.W - 1)) * SLOTS + (threadIdx.x & 63) / G;
  Place p;
  const uint32_t t = group * (SLOTS * x.W / x.P) + slot / x.P;   // below 2^31 + 32
  p.head = head0 + (slot & (x.P - 1));
  p.live = t < (uint32_t)a.tokens;
  const uint32_t tt = p.live ? t : (uint32_t)a.tokens - 1;
  p.b = a.N == (int)a.tokens ? 0 : tt / (uint32_t)a.N;
  p.n = tt - p.b * a.N;
  return p;
}

// Sums over a token of the waves of its team (each lane of a wave has its wave's); `red` alternates between two rounds, so
// one barrier a round is enough
template <int K>
__device__ __forceinline__ void team_sum(float (&v)[K], float (&red)[WAVES][K], int wave, int W) {
  if (W == 1) return;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) red[wave][k] = v[k];
  }
  __syncthreads();
  const int first = wave & ~(W - 1);
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v[k] = red[first][k];
    for (int w = 1; w < W; ++w) v[k] += red[first + w][k];
  }
}

// The teams of a tensor walk over its units: a group of tokens with the heads h, h + P, .. of one batch of NB heads a
// slot (a norm over the token has all heads in one batch). The rows of the next unit are loaded while the present one
// is worked on; the weights stay in registers.
template <int DT, int D, int NORM, int LAYOUT, int NB>
__global__ __launch_bounds__(64 * WAVES, 3) void norm_rope_fwd(NormRopeArgs a) {
  __shared__ float red[2][WAVES][1];
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int G = D / 16;
  constexpr int NW = NORM == VC_NORM_TOKEN ? NB : 1;   // weights that a lane meets: its channels of so many heads
  const int P = x.P, per = NB * P, teams = WAVES / x.W;
  const uint32_t batches = (x.H + per - 1) / per;
  const uint64_t units = (uint64_t)x.groups * batches;
  uint64_t first = (uint64_t)blockIdx.x * teams;   // of the workgroup: the same for its waves, which share barriers
  if (first >= units) return;
  const Lane l = lane_channels<D, LAYOUT>(threadIdx.x & (G - 1), a.rot);
  auto at = [&](uint64_t u) __attribute__((always_inline)) {
    u += wave / x.W;
    if (batches == 1) return place<D>(a, x, wave, (uint32_t)u, 0);
    const uint32_t group = u / batches;
    return place<D>(a, x, wave, group, (int)(u - (uint64_t)group * batches) * per);
  };
  auto load = [&](const Place& p, u4 (&raw)[NB][2]) __attribute__((always_inline)) {
    const uint16_t* in = x.in + p.b * x.in_sb + p.n * x.in_sn;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = p.head + i * P;
      raw[i][0] = raw[i][1] = u4{0, 0, 0, 0};
      if (p.live && h < x.H) {
        const uint16_t* row = in + h * x.in_sh;
        raw[i][0] = *reinterpret_cast<const u4*>(row + l.c0);
        raw[i][1] = *reinterpret_cast<const u4*>(row + l.c1);
      }
    }
  };
  Place p = at(first);
  u4 raw[NB][2];
  load(p, raw);
  float wt[NW][16];
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const int h = NORM == VC_NORM_TOKEN ? p.head + i * P : 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) wt[i][e] = 1.f;
    if (NORM != VC_NORM_NONE && x.weight && h < x.H) {
      load8f(x.weight + h * D + l.c0, wt[i]);
      load8f(x.weight + h * D + l.c1, wt[i] + 8);
    }
  }
  for (int round = 0;; round ^= 1) {
    float cs[8], sn[8];
    load_angles<LAYOUT>(a, l, p.n, p.b, a.sign, cs, sn);
    first += (uint64_t)gridDim.x * teams;
    const bool more = first < units;
    Place np = p;
    u4 next[NB][2];
    if (more) {
      np = at(first);
      load(np, next);
    }
    float r = 1.f;
    if (NORM == VC_NORM_TOKEN) {
      float ss[1] = {0.f};
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        float v[16];
        unpack8<DT>(raw[i][0], v);
        unpack8<DT>(raw[i][1], v + 8);
#pragma unroll
        for (int e = 0; e < 16; ++e) ss[0] = __builtin_fmaf(v[e], v[e], ss[0]);
      }
      ss[0] = lanes_sum(ss[0], min(G * P, 64));
      team_sum(ss, red[round], wave, x.W);
      r = __builtin_amdgcn_rsqf(__builtin_fmaf(ss[0], x.inv_span, a.eps));
    }
    uint16_t* out = x.out + p.b * x.out_sb + p.n * x.out_sn;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = p.head + i * P;
      float v[16];
      unpack8<DT>(raw[i][0], v);
      unpack8<DT>(raw[i][1], v + 8);
      if (NORM == VC_NORM_HEAD) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 16; ++e) s = __builtin_fmaf(v[e], v[e], s);
        r = __builtin_amdgcn_rsqf(__builtin_fmaf(lanes_sum(s, G), x.inv_span, a.eps));
      }
      if (NORM != VC_NORM_NONE) {
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = v[e] * r * wt[NORM == VC_NORM_TOKEN ? i : 0][e];
      }
      turn<LAYOUT>(v, l, cs, sn);
      if (p.live && h < x.H) {
        store_row(out + h * x.out_sh, l, pack8<DT>(v), pack8<DT>(v + 8), a.past);
      }
    }
    if (!more) break;
    p = np;
#pragma unroll
    for (int i = 0; i < NB; ++i) raw[i][0] = next[i][0], raw[i][1] = next[i][1];
  }
}

// Gradients. The teams walk over the units as in the forward kernel (all batches of a group of tokens by the same team), so
// that the sums of the weights' gradients stay in registers; a workgroup's waves add theirs in LDS one after the other, in a
// fixed order, and write one row of partial sums, which norm_rope_join adds up in a fixed order.
template <int DT, int D, int NORM, int LAYOUT, int NB>
__global__ __launch_bounds__(64 * WAVES, 2) void norm_rope_bwd(NormRopeArgs a) {
  extern __shared__ float acc[];
  __shared__ float red[2][WAVES][2];
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  constexpr int G = D / 16;
  constexpr int NW = NORM == VC_NORM_TOKEN ? NB : 1;
  const int P = x.P, teams = WAVES / x.W, lane = threadIdx.x & 63;
  const Lane l = lane_channels<D, LAYOUT>(lane % G, a.rot);
  const int head0 = place<D>(a, x, wave, 0, 0).head;   // a slot's heads are the same in all groups
  float dw[NW][16], wt[NW][16];
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const int h = NORM == VC_NORM_TOKEN ? head0 + i * P : 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f, wt[i][e] = 1.f;
    if (x.weight && h < x.H) {
      load8f(x.weight + h * D + l.c0, wt[i]);
      load8f(x.weight + h * D + l.c1, wt[i] + 8);
    }
  }
  const int per = NB * P;
  struct Unit {
    Place p;
    int h0;
    uint64_t first;
  };
  auto load = [&](const Unit& u, u4 (&raw)[NB][2], u4 (&gr)[NB][2]) __attribute__((always_inline)) {
    const uint16_t* in = x.in + u.p.b * x.in_sb + u.p.n * x.in_sn;
    const uint16_t* gin = x.grad + u.p.b * x.grad_sb + u.p.n * x.grad_sn;
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const int h = u.h0 + i * P;
      raw[i][0] = raw[i][1] = gr[i][0] = gr[i][1] = u4{0, 0, 0, 0};
      if (u.p.live && h < x.H) {
        raw[i][0] = *reinterpret_cast<const u4*>(in + h * x.in_sh + l.c0);
        raw[i][1] = *reinterpret_cast<const u4*>(in + h * x.in_sh + l.c1);
        gr[i][0] = *reinterpret_cast<const u4*>(gin + h * x.grad_sh + l.c0);
        gr[i][1] = *reinterpret_cast<const u4*>(gin + h * x.grad_sh + l.c1);
      }
    }
  };
  Unit u;
  u.first = (uint64_t)blockIdx.x * teams;
  u.h0 = head0;
  u4 raw[NB][2], gr[NB][2];
  if (u.first < x.groups) {
    u.p = place<D>(a, x, wave, (uint32_t)(u.first + wave / x.W), 0);
    load(u, raw, gr);
    float cs[8], sn[8];
    for (int round = 0;; round ^= 1) {
      if (u.h0 == head0) load_angles<LAYOUT>(a, l, u.p.n, u.p.b, -1.f, cs, sn);
      // the next batch of the heads, or the next tokens
      Unit v = u;
      v.h0 += per;
      if (v.h0 - head0 >= x.H) {
        v.h0 = head0;
        v.first += (uint64_t)gridDim.x * teams;
        v.p = place<D>(a, x, wave, (uint32_t)(v.first + wave / x.W), 0);
      }
      const bool more = v.first < x.groups;
      u4 raw_next[NB][2], gr_next[NB][2];
      if (more) load(v, raw_next, gr_next);
      uint16_t* out = x.out + u.p.b * x.out_sb + u.p.n * x.out_sn;
      auto values = [&](int i, float* v, float* g) __attribute__((always_inline)) {
        unpack8<DT>(raw[i][0], v);
        unpack8<DT>(raw[i][1], v + 8);
        unpack8<DT>(gr[i][0], g);
        unpack8<DT>(gr[i][1], g + 8);
        turn<LAYOUT>(g, l, cs, sn);
      };
      float t[2] = {0.f, 0.f};   // sums of x^2 and of g w x
      auto add = [&](int i, const float* v, const float* g) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          t[0] = __builtin_fmaf(v[e], v[e], t[0]);
          t[1] = __builtin_fmaf(v[e] * wt[NORM == VC_NORM_TOKEN ? i : 0][e], g[e], t[1]);
        }
      };
      if (NORM == VC_NORM_TOKEN) {
#pragma unroll
        for (int i = 0; i < NB; ++i) {
          float v[16], g[16];
          values(i, v, g);
          add(i, v, g);
        }
        t[0] = lanes_sum(t[0], min(G * P, 64));
        t[1] = lanes_sum(t[1], min(G * P, 64));
        team_sum(t, red[round], wave, x.W);
      }
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const int h = u.h0 + i * P, iw = NORM == VC_NORM_TOKEN ? i : 0;
        float v[16], g[16];
        values(i, v, g);
        if (NORM == VC_NORM_HEAD) {
          t[0] = t[1] = 0.f;
          add(i, v, g);
          t[0] = lanes_sum(t[0], G);
          t[1] = lanes_sum(t[1], G);
        }
        const float r = __builtin_amdgcn_rsqf(__builtin_fmaf(t[0], x.inv_span, a.eps));
        const float k = t[1] * x.inv_span * r;   // mean(g w u) with u = x r: of the size of g w, whatever r is
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float u = v[e] * r;
          dw[iw][e] = __builtin_fmaf(g[e], u, dw[iw][e]);
          g[e] = __builtin_fmaf(-k, u, g[e] * wt[iw][e]) * r;
        }
        if (u.p.live && h < x.H) {
          store_row(out + h * x.out_sh, l, pack8<DT>(g), pack8<DT>(g + 8), a.past);
        }
      }
      if (!more) break;
      u = v;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) raw[i][e] = raw_next[i][e], gr[i][e] = gr_next[i][e];
    }
  }
  if (!x.dw_part) return;
  // slots that share their channels: all of the wave (a head's norm), or those of its other tokens
  const int share = NORM == VC_NORM_HEAD ? G : min(G * P, 64);
#pragma unroll
  for (int i = 0; i < NW; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e)
      for (int o = share; o < 64; o <<= 1) dw[i][e] += __shfl_xor(dw[i][e], o, 64);
  const int C = NORM == VC_NORM_HEAD ? D : x.H * D;
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave && lane < share) {
#pragma unroll
      for (int i = 0; i < NW; ++i) {
        const int h = NORM == VC_NORM_HEAD ? 0 : head0 + i * P;
        if (NORM == VC_NORM_HEAD || h < x.H) {
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int c = h * D + (e < 8 ? l.c0 + e : l.c1 + e - 8);
            acc[c] = w < x.W ? dw[i][e] : acc[c] + dw[i][e];   // the first team's waves have all channels
          }
        }
      }
    }
    __syncthreads();
  }
  for (int c = threadIdx.x; c < C; c += 64 * WAVES) x.dw_part[(size_t)blockIdx.x * C + c] = acc[c];
}

// dw[c] = sum of the partial rows: 8 channels a workgroup, 128 threads a channel walk the rows, a tree adds them
// (with 16 threads a channel, 64 loads one behind the other: 25 us for 128 channels of 1024 rows)
__global__ __launch_bounds__(1024) void norm_rope_join(NormRopeArgs a, int parts) {
  __shared__ float s[128][9];
  const NormRopeTensor& x = a.t[blockIdx.y];
  const int C = x.weights;
  const int cc = threadIdx.x & 7, row = threadIdx.x >> 3, c = blockIdx.x * 8 + cc;
  float v = 0.f;
  if (x.dw_part && c < C) {
#pragma unroll 4
    for (int p = row; p < parts; p += 128) v += x.dw_part[(size_t)p * C + c];
  }
  s[row][cc] = v;
  __syncthreads();
  for (int o = 64; o > 0; o >>= 1) {
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
  if (nb <= 1) return launch<DT, D, NORM, LAYOUT, 1, BWD>(a, grid, lds, s);
  if constexpr (NORM != VC_NORM_TOKEN && !BWD)
    if (nb > 2) return launch<DT, D, NORM, LAYOUT, 4, BWD>(a, grid, lds, s);
  return launch<DT, D, NORM, LAYOUT, 2, BWD>(a, grid, lds, s);
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

// Waves of a team, slots of a token and groups of tokens of a tensor; returns the rounds of the slots over its heads
int set_teams(const NormRopeArgs& a, NormRopeTensor& t) {
  const int slots = 64 / (a.d / 16);   // of a wave
  t.W = 1;
  if (a.norm == VC_NORM_TOKEN)
    while (t.W < WAVES && t.H > 2 * slots * t.W) t.W *= 2;   // two rounds at most (8192 channels)
  t.P = t.W * slots;
  if (t.W == 1)
    while (t.P / 2 >= t.H) t.P /= 2;
  const int tokens = slots * t.W / t.P;
  t.groups = (uint32_t)((a.tokens + tokens - 1) / tokens);
  return (t.H + t.P - 1) / t.P;
}

// Calls whose tensors do not stay in the 256 MB memory-side cache anyway store their results past the caches. Measured (us,
// with / without, inputs from memory): 12 heads of 32760 tokens (200 MB in, 200 MB out) 82 / 87 the rotation alone, 86 / 91
// norms per head, 81 / 85 norms per token, gradients 132 / 139 and 142 / 148. Smaller results stay for the step that reads
// them next.
int past_caches(const NormRopeArgs& a, int tensors) {
  int64_t values = 0;
  for (int i = 0; i < a.ntensors; ++i) values += a.tokens * a.t[i].H * a.d;
  return values * 2 * tensors > (256LL << 20);
}

}  // namespace

int norm_rope_parts(int64_t tokens, int ntensors) {
  // workgroups of the backward kernel, each of which leaves a row of partial weight sums: as many as fit the CUs at once, two
  // each, and no more than have a token each. Measured (us, this / twice as many): 12 + 12 heads of 32760 tokens, norms per head
  // 141 / 140, per token 148 / 156; of 16000 tokens 71 / 75, 74 / 84. With 16 tokens each instead of one, 40 + 40 heads of 16
  // tokens take 28 instead of 13 per head and 52 instead of 14 per token.
  const int64_t most = 512 / ntensors;
  return (int)(tokens < most ? tokens : most);
}

hipError_t launch_norm_rope(NormRopeArgs a, hipStream_t s) {
  a.past = past_caches(a, 2);
  int64_t rounds = 1, units = 0;
  for (int i = 0; i < a.ntensors; ++i) {
    const int64_t r = set_teams(a, a.t[i]);
    rounds = r > rounds ? r : rounds;
    units += a.t[i].groups * r;
  }
  // heads of a slot that a wave has in flight: more of them for large calls; one, so that the heads of a token go to
  // several waves, where there are few tokens. Measured (us, the rotation alone, one / more): 40 heads of 16 tokens 3.9 / 4.5, of
  // 256 tokens (2560 units) 5.1 / 5.4; 12 heads of 2000 tokens (8000 units) 8.5 / 7.8, of 16000 52 / 43
  const int nb = a.norm == VC_NORM_TOKEN ? (int)rounds : units <= 4096 ? 1 : rounds <= 2 ? (int)rounds : 4;
  int64_t grid = 1;
  for (int i = 0; i < a.ntensors; ++i) {
    const NormRopeTensor& t = a.t[i];
    const int64_t u = (int64_t)t.groups * ((t.H + nb * t.P - 1) / (nb * t.P)), teams = WAVES / t.W;
    grid = (u + teams - 1) / teams > grid ? (u + teams - 1) / teams : grid;
  }
  // workgroups: half of them with 12 + 12 heads of 32760 tokens take 73 instead of 68 us for the rotation alone, 81 instead of 77
  // with norms per token; twice as many 66 and 80, and 54 instead of 50 for 16000 tokens with these norms
  const int64_t most = 4096 / a.ntensors;
  return dispatch<false>(a, nb, (int)(grid < most ? grid : most), 0, s);
}

hipError_t launch_norm_rope_backward(NormRopeArgs a, hipStream_t s) {
  a.past = past_caches(a, 3);
  int nb = 1, C = 0;
  bool weights = false;
  for (int i = 0; i < a.ntensors; ++i) {
    NormRopeTensor& t = a.t[i];
    const int r = set_teams(a, t);
    nb = r > nb ? r : nb;
    C = t.weights > C ? t.weights : C;
    weights = weights || t.dw_part;
  }
  const int parts = norm_rope_parts(a.tokens, a.ntensors);
  hipError_t e = dispatch<true>(a, nb, parts, (size_t)C * 4, s);
  if (e != hipSuccess || !weights) return e;
  norm_rope_join<<<dim3((unsigned)((C + 7) / 8), (unsigned)a.ntensors), 1024, 0, s>>>(a, parts);
  return hipGetLastError();
}

}  // namespace vc
