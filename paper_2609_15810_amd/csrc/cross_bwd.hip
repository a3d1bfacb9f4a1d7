// Gradients of the attention to the states of another sequence (cross_fwd.hip), from lse of the forward pass:
//
//   P = exp(c' Q K^T - lse),  dV = P^T dO,  dP = dO V^T,  delta_i = sum_j P_ij dP_ij / sum_j P_ij,
//   dS = P (dP - delta),  dQ = c' dS K,  dK = c' dS^T Q,
//
// with dK and dV summed over the query heads of a key head. Two kernels form S and dP each, so that every sum is
// formed in a fixed order in registers (one kernel would have to add dQ or dK, dV in memory, in the order in which
// workgroups come):
//   cross_dq   a wave owns 32 rows (queries), keys in tiles of 64 from LDS: S^T = K Q^T, dP^T = V dO^T,
//              dQ^T += K^T dS^T;
//   cross_dkv  a wave owns 32 keys, rows in tiles of 32 from LDS: S = Q K^T, dP = dO V^T, dV^T += dO^T P,
//              dK^T += Q^T dS.
// In both a lane owns one column of the products, the probabilities and dS of a lane are already in operand
// order for the next product, whose other operand is read from LDS by transposing reads. P and dS are rounded to the
// operands' 16 bits, as the matrix instructions take them; sums are fp32.
//
// Two things cost matrix products for the sake of dQ and dK. delta is formed from P and dP, in a first walk over the keys. It
// equals sum_c dO_ic O_ic, which costs no walk, but O comes rounded to 16 bits, and an error of delta does not average out: dS
// of a row is off by P times it. (The sum of P is 1 but for the error of lse, which dS then does not see.) And for dQ, dS is
// taken as two 16-bit numbers: the dS of a row add up to 0, which takes out of dQ what all keys have in common, but their
// roundings do not, and keys tend to have large means. Measured on 12 heads of 32760 rows and 512 keys in bf16, rms errors of dQ
// and dK relative to their size (a rounding of them alone: 0.0017) and the time of cross_dq:
//   delta from O                          0.0038, 0.0030   190 us
//   delta from P and dP                   0.0025, 0.0024   261 us
//   and dS in two numbers for dQ          0.0017, 0.0023   310 us
#include <type_traits>

#include "cross_common.hpp"

namespace vc {
namespace cross {
namespace {

constexpr int NW = 4;          // waves of a workgroup
constexpr int QR = 32 * NW;    // rows of a workgroup of cross_dq
constexpr int KT = 64;         // keys of its tiles
constexpr int KB = 32 * NW;    // keys of a workgroup of cross_dkv
constexpr int RT = 32;         // rows of its tiles

// rows of a query head's statistics: whole tiles of cross_dkv
__host__ __device__ __forceinline__ int stat_rows(int M) { return (M + RT - 1) / RT * RT; }

template <int DT>
__device__ __forceinline__ u4 pack_half(const v16f& s, int h) {
  u4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2<DT>(s[8 * h + 2 * i], s[8 * h + 2 * i + 1]);
  return r;
}
// what that rounded off
template <int DT>
__device__ __forceinline__ u4 pack_rest(const v16f& s, int h, const u4& rounded) {
  u4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = rounded[i];
    float x, y;
    if constexpr (DT == VC_BF16) {
      x = bf16_lo(w), y = bf16_hi(w);
    } else {
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      const h2 f = __builtin_bit_cast(h2, w);
      x = f[0], y = f[1];
    }
    r[i] = pack2<DT>(s[8 * h + 2 * i] - x, s[8 * h + 2 * i + 1] - y);
  }
  return r;
}

// In cross_dkv probabilities are 2^shift times themselves: fp16's normal range ends at 2^-14, which the probabilities of
// many keys fall below
template <int DT>
constexpr float P_SHIFT = DT == VC_FP16 ? 15.f : 0.f;
template <int DT>
constexpr float P_UNIT = DT == VC_FP16 ? 1.f / 32768.f : 1.f;

// What a launch of cross_dq forms: delta and dQ in two walks over all keys; or over a part of the keys its part of delta, and in
// a second launch its part of dQ
enum { WHOLE, PART_DELTA, PART_DQ };

// GATHER: addresses per key (the keys are those of a list, or off_buffer)
template <int DT, int D, bool GATHER, int MODE>
__global__ __launch_bounds__(64 * NW, 2) void cross_dq(CrossArgs a) {
  using T = Tile<D>;
  using C = Copier<D, KT, NW>;
  constexpr int TB = KT * T::ROW, KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t kt[4][TB];   // two tiles of K, two of V
  uint8_t(*const vt)[TB] = kt + 2;

  const uint32_t wg = xcd_order(blockIdx.x, gridDim.x), blocks = (uint32_t)(a.R + QR - 1) / QR;
  const uint32_t rest = wg / blocks, bh = rest / (uint32_t)a.splits;
  const int rb = wg - rest * blocks, split = rest - bh * a.splits;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk;
  const int lane = threadIdx.x & 63, col = lane & 31, kh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = keys_of(a, b);
  const int k0 = MODE == WHOLE ? 0 : split * a.chunk, k1 = MODE == WHOLE ? n : min(n, k0 + a.chunk);
  const int tiles = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0;
  const int steps = MODE == WHOLE ? 2 * tiles : tiles;   // tiles in the order of both walks

  const uint16_t *kbase = a.K.p + b * a.K.sb + hk * a.K.sh, *vbase = a.V.p + b * a.V.sb + hk * a.V.sh;
  const int crow = lane / T::CH;
  const C kc(a.K.sn, wave, lane), vc(a.V.sn, wave, lane);
  int next[C::COPIES];
  auto fetch = [&](int u) __attribute__((always_inline)) {
    if (GATHER) {
      const int t = u < tiles ? u : u - tiles;
#pragma unroll
      for (int c = 0; c < C::COPIES; ++c) {
        const int j = k0 + t * KT + (c * NW + wave) * T::ROWS_PER_COPY + crow;
        next[c] = u < steps && j < k1 ? (a.idx ? a.idx[(size_t)b * a.N + j] : j) : -1;
      }
    }
  };
  auto copy_tile = [&](int u, int buf) __attribute__((always_inline)) {
    if (GATHER) {
#pragma unroll
      for (int c = 0; c < C::COPIES; ++c) {
        const int q = c * NW + wave, ch = (lane % T::CH) ^ T::key(q * T::ROWS_PER_COPY + crow);
        const int64_t src = next[c];
        copy16(src >= 0 ? (const void*)(kbase + src * a.K.sn + 8 * ch) : (const void*)&zero16, kt[buf] + q * 1024);
        copy16(src >= 0 ? (const void*)(vbase + src * a.V.sn + 8 * ch) : (const void*)&zero16, vt[buf] + q * 1024);
      }
    } else {
      const int j = k0 + (u < tiles ? u : u - tiles) * KT;
      kc.copy(kbase + j * a.K.sn, k1 - j, kt[buf], wave);
      vc.copy(vbase + j * a.V.sn, k1 - j, vt[buf], wave);
    }
  };
  if (tiles > 0) {
    fetch(0);
    copy_tile(0, 0);
    fetch(1);
  }

  const int r0 = rb * QR + 32 * wave, row = r0 + col;
  const bool active = r0 < a.R;
  const QueryRow qr = query_row(a, hk, min(row, a.R - 1));
  u4 q[KS], g[KS];
  {
    const uint16_t* pq = a.Q.p + b * a.Q.sb + qr.h * a.Q.sh + qr.i * a.Q.sn + 8 * kh;
    const uint16_t* pg = a.dO.p + b * a.dO.sb + qr.h * a.dO.sh + qr.i * a.dO.sn + 8 * kh;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = *reinterpret_cast<const u4*>(pq + 16 * s);
      g[s] = *reinterpret_cast<const u4*>(pg + 16 * s);
    }
  }
  const float l2 = a.lse[((size_t)b * a.Hq + qr.h) * a.M + qr.i] * 1.4426950408889634f;
  const size_t heads = (size_t)a.B * a.Hk;
  float delta = 0.f, sum = 0.f;   // sums of P dP and of P over the keys; then delta
  if (MODE == PART_DQ && row < a.R)
    for (int s = 0; s < a.splits; ++s) {
      const float2 x = *reinterpret_cast<const float2*>(a.part_ml + 2 * ((s * heads + bh) * a.R + row));
      delta += x.x, sum += x.y;
    }
  const RowOperands<D> rows0(lane);
  const ColOperands<D> cols0(lane);
  v16f acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = v16f{};

  // S^T and dP^T of the 32 keys from row 32 x of a tile, of which `valid` count; S becomes P
  auto products = [&](uint32_t at, int x, int valid, v16f& s, v16f& dp) __attribute__((always_inline)) {
    const RowOperands<D> rows = rows0.move(lds_addr(kt[0]) + at);
    s = v16f{};
    dp = v16f{};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = mma<DT>(rows.get(32 * x * T::ROW, i), q[i], s);
      dp = mma<DT>(rows.get(2 * TB + 32 * x * T::ROW, i), g[i], dp);
    }
    issue_reads<6>();
    issue_products<2 * KS - 6, 1>();
    issue_products<6, 0>();
    __builtin_amdgcn_sched_barrier(0);
    if (valid < 32 * x + 32) mask_scores(s, valid - 32 * x, kh);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -l2));
  };
  // tile u (of both walks) is there, the next on its way
  auto arrive = [&](int u) __attribute__((always_inline)) {
    wait_copies<0>();
    barrier();
    if (u + 1 < steps) {
      copy_tile(u + 1, (u + 1) & 1);
      fetch(u + 2);
    }
  };
  // (The second half of a tile without keys is left out: 40 heads of 75600 rows over 77 keys, all gradients, 1176 -> 1105 us.)
  int u = 0;
  if (MODE != PART_DQ) {
    float part[8] = {};   // in four chains each: the operations of one wait for each other
    for (; u < tiles; ++u) {
      arrive(u);
      if (!active) continue;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (k1 - k0 - u * KT <= 32 * x) break;
        v16f s, dp;
        products((u & 1) * TB, x, k1 - k0 - u * KT, s, dp);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          part[r & 3] = __builtin_fmaf(s[r], dp[r], part[r & 3]);
          part[4 + (r & 3)] += s[r];
        }
      }
    }
    delta = half_sum((part[0] + part[1]) + (part[2] + part[3]));
    sum = half_sum((part[4] + part[5]) + (part[6] + part[7]));
  }
  if (MODE == PART_DELTA) {
    if (row < a.R && kh == 0)
      *reinterpret_cast<float2*>(a.part_ml + 2 * ((split * heads + bh) * a.R + row)) = make_float2(delta, sum);
    return;
  }
  delta = sum > 0.f ? delta / sum : 0.f;
  for (int t = 0; t < tiles; ++t, ++u) {
    arrive(u);
    if (!active) continue;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (k1 - k0 - t * KT <= 32 * x) break;
      v16f s, dp;
      products((u & 1) * TB, x, k1 - k0 - t * KT, s, dp);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] *= dp[r] - delta;
      const u4 ds[2] = {pack_half<DT>(s, 0), pack_half<DT>(s, 1)};
      const u4 rest[2] = {pack_rest<DT>(s, 0, ds[0]), pack_rest<DT>(s, 1, ds[1])};
      __builtin_amdgcn_sched_barrier(0);
      const ColOperands<D> cols = cols0.move(lds_addr(kt[0]) + (u & 1) * TB);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          const u4 k = cols.get((32 * x + 16 * h) * T::ROW, db);
          acc[db] = mma<DT>(k, ds[h], acc[db]);
          acc[db] = mma<DT>(k, rest[h], acc[db]);
        }
      issue_reads<8>();
      issue_products<4 * DB - 8, 1>();
      issue_products<8, 0>();
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  // what cross_dkv needs of a row; the rows that fill a head's last tile get probabilities of 0
  if (split == 0 && kh == 0 && row < a.R) {
    const int fill = stat_rows(a.M);
    float* st = a.stats + 2 * (((size_t)b * a.Hq + qr.h) * fill + qr.i);
    *reinterpret_cast<float2*>(st) = make_float2(l2 - P_SHIFT<DT>, delta * P_UNIT<DT>);
    if (qr.i == a.M - 1)
      for (int i = 1; i < fill - qr.i; ++i) *reinterpret_cast<float2*>(st + 2 * i) = make_float2(INFINITY, 0.f);
  }
  if (MODE == PART_DQ) {
    if (row < a.R) {
      float* p = a.part_o + ((split * heads + bh) * a.R + row) * D + 4 * kh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<float4*>(p + 32 * db + 8 * x) =
              make_float4(acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]);
    }
    return;
  }
  store_row<DT, D>(acc, a.scale, row < a.R ? a.dQ.p + b * a.dQ.sb + qr.h * a.dQ.sh + qr.i * a.dQ.sn : nullptr, lane);
}

// The sums of a wave's 32 keys take half of its registers, their K operand an eighth; V of the workgroup's keys stands in LDS,
// so that two waves fit a SIMD, of two workgroups that are not in step: one's products and the other's vector work overlap.
// (One wave a SIMD with V in registers: the products then leave their results in accumulation registers, 32 to 96 copies a
// step; 283 us for 12 heads of 32760 rows and 512 keys.)
// FAR: addresses per row (off_buffer); SPLIT: leave parts
template <int DT, int D, bool FAR, bool SPLIT>
__global__ __launch_bounds__(64 * NW, 2) void cross_dkv(CrossArgs a) {
  using T = Tile<D>;
  using C = Copier<D, RT, NW>;
  constexpr int TB = RT * T::ROW, KS = D / 16, DB = D / 32;
  // V of the keys; of two row tiles Q, then dO; their statistics
  __shared__ __attribute__((aligned(256))) uint8_t vt[KB * T::ROW], tile[2][2 * TB];
  __shared__ __attribute__((aligned(16))) float st[2][2 * RT];

  const uint32_t wg = xcd_order(blockIdx.x, gridDim.x), blocks = (uint32_t)(a.N + KB - 1) / KB;
  const uint32_t rest = wg / blocks, bh = rest / (uint32_t)a.row_splits;
  const int block = wg - rest * blocks, split = rest - bh * a.row_splits;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk;
  const int lane = threadIdx.x & 63, col = lane & 31, kh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = keys_of(a, b);
  if (SPLIT && block * KB >= n) return;   // the join writes the zeros of keys that do not count
  // row tiles, each of one query head: tile x of head g is g * per_head + x
  const int per_head = (a.M + RT - 1) / RT;
  const int t0 = SPLIT ? split * a.row_chunk : 0, t1 = SPLIT ? min(a.G * per_head, t0 + a.row_chunk) : a.G * per_head;
  const int tiles = block * KB < n ? t1 - t0 : 0;

  const C qc(a.Q.sn, wave, lane), gc(a.dO.sn, wave, lane);
  int head = hk * a.G + t0 / per_head, m0 = t0 % per_head * RT;   // of the next tile to copy
  auto copy_tile = [&](int to) __attribute__((always_inline)) {
    const uint16_t *q = a.Q.p + b * a.Q.sb + head * a.Q.sh + m0 * a.Q.sn;
    const uint16_t *g = a.dO.p + b * a.dO.sb + head * a.dO.sh + m0 * a.dO.sn;
    if (FAR) {
#pragma unroll
      for (int u = 0; u < C::COPIES; ++u) {
        const int x = u * NW + wave, r = x * T::ROWS_PER_COPY + lane / T::CH, ch = (lane % T::CH) ^ T::key(r);
        const bool in = m0 + r < a.M;
        copy16(in ? (const void*)(q + r * a.Q.sn + 8 * ch) : (const void*)&zero16, tile[to] + x * 1024);
        copy16(in ? (const void*)(g + r * a.dO.sn + 8 * ch) : (const void*)&zero16, tile[to] + TB + x * 1024);
      }
    } else {
      qc.copy(q, a.M - m0, tile[to], wave);
      gc.copy(g, a.M - m0, tile[to] + TB, wave);
    }
    if (wave == 0 && lane < RT / 2)
      copy16(a.stats + 2 * (((size_t)b * a.Hq + head) * stat_rows(a.M) + m0) + 4 * lane, st[to]);
    m0 += RT;
    if (m0 >= a.M) m0 = 0, ++head;
  };
  if (tiles > 0) copy_tile(0);

  // this lane's key, in the order of the list; its K in registers, its V in LDS in the place of row `col` of the wave's
  const int j = block * KB + 32 * wave + col;
  const bool counts = j < n;
  const bool active = block * KB + 32 * wave < n;
  const int64_t key = j < a.N ? (a.idx ? a.idx[(size_t)b * a.N + j] : j) : 0;
  u4 k[KS];
  {
    const uint16_t *pk = a.K.p + b * a.K.sb + hk * a.K.sh + key * a.K.sn + 8 * kh;
    const uint16_t *pv = a.V.p + b * a.V.sb + hk * a.V.sh + key * a.V.sn + 8 * kh;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      k[s] = counts ? *reinterpret_cast<const u4*>(pk + 16 * s) : u4{0, 0, 0, 0};
      *reinterpret_cast<u4*>(vt + T::at(32 * wave + col, 2 * s + kh)) =
          counts ? *reinterpret_cast<const u4*>(pv + 16 * s) : u4{0, 0, 0, 0};
    }
  }
  v16f dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = v16f{};
  const RowOperands<D> vrows = RowOperands<D>(lane).move(lds_addr(vt) + 32 * wave * T::ROW);
  RowOperands<D> rows = RowOperands<D>(lane).move(lds_addr(tile));
  ColOperands<D> cols = ColOperands<D>(lane).move(lds_addr(tile));
  const uint32_t st0 = lds_addr(st) + 32 * kh;

  for (int t = 0; t < tiles; ++t) {
    wait_copies<0>();
    barrier();
    if (t + 1 < tiles) copy_tile((t + 1) & 1);
    if (!active) continue;
    v16f s = {}, dp = {};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = mma<DT>(rows.get(0, i), k[i], s);
      dp = mma<DT>(rows.get(TB, i), vrows.get(0, i), dp);
    }
    issue_reads<6>();
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      issue_products<1, 1>();
      issue_products<1, 2>();
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      typedef float f4 __attribute__((ext_vector_type(4)));
      typedef const __attribute__((address_space(3))) f4* at;
      const f4 x = *(at)(st0 + (t & 1) * 8 * RT + 64 * g), y = *(at)(st0 + (t & 1) * 8 * RT + 64 * g + 16);
      const float l2[4] = {x[0], x[2], y[0], y[2]}, dl[4] = {x[1], x[3], y[1], y[3]};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -l2[e]));
        dp[r] = s[r] * __builtin_fmaf(dp[r], P_UNIT<DT>, -dl[e]);
      }
    }
    u4 p[2], ds[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) p[h] = pack_half<DT>(s, h), ds[h] = pack_half<DT>(dp, h);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        dv[db] = mma<DT>(cols.get(TB + 16 * h * T::ROW, db), p[h], dv[db]);
        dk[db] = mma<DT>(cols.get(16 * h * T::ROW, db), ds[h], dk[db]);
      }
    issue_reads<10>();
    issue_products<4 * DB - 5, 2>();
    issue_products<5, 0>();
    __builtin_amdgcn_sched_barrier(0);
    rows.shift((t & 1) ? -2 * TB : 2 * TB);
    cols.shift((t & 1) ? -2 * TB : 2 * TB);
  }

  if (SPLIT) {
    if (counts) {
      const size_t each = (size_t)a.B * a.Hk * a.N * D;
      float* p = a.part_kv + 2 * split * each + ((size_t)bh * a.N + j) * D + 4 * kh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          *reinterpret_cast<float4*>(p + 32 * db + 8 * x) =
              make_float4(dk[db][4 * x], dk[db][4 * x + 1], dk[db][4 * x + 2], dk[db][4 * x + 3]);
          *reinterpret_cast<float4*>(p + each + 32 * db + 8 * x) =
              make_float4(dv[db][4 * x], dv[db][4 * x + 1], dv[db][4 * x + 2], dv[db][4 * x + 3]);
        }
    }
    return;
  }
  // keys that do not count have gradients of 0
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      dk[db][r] = counts ? dk[db][r] : 0.f;
      dv[db][r] = counts ? dv[db][r] : 0.f;
    }
  auto row_of = [&](const Strided& t) __attribute__((always_inline)) -> uint16_t* {
    return j < a.N ? t.p + b * t.sb + hk * t.sh + key * t.sn : nullptr;
  };
  store_row<DT, D>(dk, a.scale, row_of(a.dK), lane);
  store_row<DT, D>(dv, P_UNIT<DT>, row_of(a.dV), lane);
}

// Sums of parts [part][row][D] at p (rows * D apart by `step`): as cross_join, d / 4 lanes and `groups` of them a row;
// the sum is complete in the lanes of group 0
template <int D>
__device__ __forceinline__ float4 join_parts(const float* p, size_t step, int parts, int groups, bool in) {
  constexpr int L = D / 4, ALL = 256 / L;
  __shared__ __attribute__((aligned(16))) float so[ALL][D];
  const int slot = threadIdx.x / L, g = slot & (groups - 1), c = threadIdx.x % L * 4;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float4 v) __attribute__((always_inline)) { o.x += v.x, o.y += v.y, o.z += v.z, o.w += v.w; };
  if (in) {
#pragma unroll 4
    for (int s = g; s < parts; s += groups) add(*reinterpret_cast<const float4*>(p + s * step + c));
  }
  if (groups > 1) {
    *reinterpret_cast<float4*>(&so[slot][c]) = o;
    __syncthreads();
    if (g == 0)
      for (int i = 1; i < groups; ++i) add(*reinterpret_cast<const float4*>(&so[slot + i][c]));
  }
  return o;
}

// dQ from the parts of split keys
template <int DT, int D>
__global__ __launch_bounds__(256) void cross_join_dq(CrossArgs a, int groups) {
  constexpr int L = D / 4, ALL = 256 / L;
  const int slot = threadIdx.x / L, c = threadIdx.x % L * 4;
  const int64_t rows = (int64_t)a.B * a.Hk * a.R, at = (int64_t)blockIdx.x * (ALL / groups) + slot / groups;
  const float4 o = join_parts<D>(a.part_o + at * D, rows * D, a.splits, groups, at < rows);
  if ((slot & (groups - 1)) != 0 || at >= rows) return;
  const uint32_t bh = at / a.R;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk;
  const QueryRow w = query_row(a, hk, (int)(at - (int64_t)bh * a.R));
  const float f = a.scale;
  *reinterpret_cast<u2*>(a.dQ.p + b * a.dQ.sb + w.h * a.dQ.sh + w.i * a.dQ.sn + c) =
      u2{pack2<DT>(o.x * f, o.y * f), pack2<DT>(o.z * f, o.w * f)};
}

// dK and dV from the parts of split rows; zeros for keys that do not count
template <int DT, int D>
__global__ __launch_bounds__(256) void cross_join_dkv(CrossArgs a, int groups) {
  constexpr int L = D / 4, ALL = 256 / L;
  const int slot = threadIdx.x / L, c = threadIdx.x % L * 4, which = blockIdx.y;
  const int64_t keys = (int64_t)a.B * a.Hk * a.N, at = (int64_t)blockIdx.x * (ALL / groups) + slot / groups;
  const bool in = at < keys;
  const uint32_t bh = (in ? at : 0) / a.N;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk, j = in ? (int)(at - (int64_t)bh * a.N) : 0;
  const float4 o = join_parts<D>(a.part_kv + (which * keys + at) * D, 2 * keys * D, a.row_splits, groups,
                                 in && j < keys_of(a, b));
  if ((slot & (groups - 1)) != 0 || !in) return;
  const float f = which ? P_UNIT<DT> : a.scale;
  const Strided& t = which ? a.dV : a.dK;
  const int64_t i = a.idx ? a.idx[(size_t)b * a.N + j] : j;
  *reinterpret_cast<u2*>(t.p + b * t.sb + hk * t.sh + i * t.sn + c) =
      u2{pack2<DT>(o.x * f, o.y * f), pack2<DT>(o.z * f, o.w * f)};
}

template <int DT, int D>
hipError_t backward(const CrossArgs& a, hipStream_t s) {
  const int gj = join_groups(a.splits), gkj = join_groups(a.row_splits);
  const int64_t jq = 256 / (D / 4) / gj, jk = 256 / (D / 4) / gkj;   // joined rows of a workgroup
  const int64_t heads = (int64_t)a.B * a.Hk;
  const unsigned gq = (unsigned)((int64_t)(a.R + QR - 1) / QR * heads * a.splits);
  const unsigned gk = (unsigned)((int64_t)(a.N + KB - 1) / KB * heads * a.row_splits);
  const bool gather = a.idx || off_buffer(a.K, D) || off_buffer(a.V, D);
  const bool far = off_buffer(a.Q, D) || off_buffer(a.dO, D);
  hipError_t e;
  if (a.splits > 1) {
    if (gather) cross_dq<DT, D, true, PART_DELTA><<<gq, 64 * NW, 0, s>>>(a);
    else cross_dq<DT, D, false, PART_DELTA><<<gq, 64 * NW, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (gather) cross_dq<DT, D, true, PART_DQ><<<gq, 64 * NW, 0, s>>>(a);
    else cross_dq<DT, D, false, PART_DQ><<<gq, 64 * NW, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    cross_join_dq<DT, D><<<(unsigned)((heads * a.R + jq - 1) / jq), 256, 0, s>>>(a, gj);
  } else {
    if (gather) cross_dq<DT, D, true, WHOLE><<<gq, 64 * NW, 0, s>>>(a);
    else cross_dq<DT, D, false, WHOLE><<<gq, 64 * NW, 0, s>>>(a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.row_splits > 1) {
    if (far) cross_dkv<DT, D, true, true><<<gk, 64 * NW, 0, s>>>(a);
    else cross_dkv<DT, D, false, true><<<gk, 64 * NW, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    cross_join_dkv<DT, D><<<dim3((unsigned)((heads * a.N + jk - 1) / jk), 2), 256, 0, s>>>(a, gkj);
  } else {
    if (far) cross_dkv<DT, D, true, false><<<gk, 64 * NW, 0, s>>>(a);
    else cross_dkv<DT, D, false, false><<<gk, 64 * NW, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace cross

void cross_plan_backward(CrossArgs& a) {
  using namespace cross;
  cross_plan(a);
  // Row tiles are split where the keys alone do not give every CU two workgroups, into as many parts as fit at once (12 heads of
  // 32760 rows and 512 keys: 10 parts 218 us, one workgroup a CU 302, 21 parts 227)
  const int64_t base = (int64_t)(a.N + KB - 1) / KB * a.B * a.Hk, tiles = (int64_t)a.G * ((a.M + RT - 1) / RT);
  int64_t splits = base >= 256 ? 1 : 512 / base;
  if (splits > tiles) splits = tiles;
  const int64_t per = (tiles + splits - 1) / splits;
  a.row_chunk = (int)per;
  a.row_splits = (int)((tiles + per - 1) / per);
}

int cross_stat_rows(int M) { return cross::stat_rows(M); }

hipError_t launch_cross_backward(const CrossArgs& a, hipStream_t s) {
  if (a.d == 128) return a.dtype == VC_BF16 ? cross::backward<VC_BF16, 128>(a, s) : cross::backward<VC_FP16, 128>(a, s);
  return a.dtype == VC_BF16 ? cross::backward<VC_BF16, 64>(a, s) : cross::backward<VC_FP16, 64>(a, s);
}

}  // namespace vc
