// Gradients of the attention to the states of another sequence (cross_fwd.hip), from lse and O of the forward pass:
//
//   P = exp(c' Q K^T - lse),  dV = P^T dO,  dP = dO V^T,  delta_i = sum_j P_ij dP_ij,
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
// delta is sum_c dO_ic O_ic with O as the forward pass rounded it, an error of half a step of O per term. Where all keys of a
// batch item are in one tile, it is formed from P and dP instead, which cancels exactly in dS where a row has few
// keys (with one key dS is 0).
#include "cross_common.hpp"

namespace vc {
namespace cross {
namespace {

constexpr int NW = 4;          // waves of a workgroup
constexpr int QR = 32 * NW;    // rows of a workgroup of cross_dq
constexpr int KT = 64;         // keys of its tiles
constexpr int KB = 32 * NW;    // keys of a workgroup of cross_dkv
constexpr int RT = 32;         // rows of its tiles

// rows of the row statistics per key head: whole workgroups of cross_dq
__host__ __device__ __forceinline__ int64_t stat_rows(int R) { return ((int64_t)R + QR - 1) / QR * QR; }

// A wave's 32 rows of D channels held as 32x32 results (column = row), times f: through its part of LDS, so that each
// row is stored as a whole. dst(r) is row r's address, or null.
template <int DT, int D, typename F>
__device__ __forceinline__ void store_rows(const v16f (&o)[D / 32], float f, uint8_t* lds, int lane, F dst) {
  using T = Tile<D>;
  const int col = lane & 31, kh = lane >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<u2*>(lds + T::at(col, 4 * db + g) + 8 * kh) =
          u2{pack2<DT>(o[db][4 * g] * f, o[db][4 * g + 1] * f), pack2<DT>(o[db][4 * g + 2] * f, o[db][4 * g + 3] * f)};
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
  for (int u = 0; u < 32 / T::ROWS_PER_COPY; ++u) {
    const int r = u * T::ROWS_PER_COPY + lane / T::CH, ch = lane % T::CH;
    uint16_t* p = dst(r);
    if (p) *reinterpret_cast<u4*>(p + 8 * ch) = *reinterpret_cast<const u4*>(lds + T::at(r, ch));
  }
}

template <int DT>
__device__ __forceinline__ float dot8(u4 a, u4 b, float s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t x = a[i], y = b[i];
    if constexpr (DT == VC_BF16) {
      s = __builtin_fmaf(bf16_lo(x), bf16_lo(y), s);
      s = __builtin_fmaf(bf16_hi(x), bf16_hi(y), s);
    } else {
      typedef _Float16 h2 __attribute__((ext_vector_type(2)));
      const h2 u = __builtin_bit_cast(h2, x), v = __builtin_bit_cast(h2, y);
      s = __builtin_fmaf((float)u[0], (float)v[0], s);
      s = __builtin_fmaf((float)u[1], (float)v[1], s);
    }
  }
  return s;
}

template <int DT>
__device__ __forceinline__ u4 pack_half(const v16f& s, int h) {
  u4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = pack2<DT>(s[8 * h + 2 * i], s[8 * h + 2 * i + 1]);
  return r;
}

template <int DT, int D, bool IDX, bool SPLIT>
__global__ __launch_bounds__(64 * NW, 2) void cross_dq(CrossArgs a) {
  using T = Tile<D>;
  constexpr int TB = KT * T::ROW, COPIES = KT / T::ROWS_PER_COPY / NW, KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t kt[2][TB], vt[2][TB];

  const uint32_t wg = xcd_order(blockIdx.x, gridDim.x), blocks = (uint32_t)(a.R + QR - 1) / QR;
  const uint32_t rest = wg / blocks, bh = rest / (uint32_t)a.splits;
  const int rb = wg - rest * blocks, split = rest - bh * a.splits;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk;
  const int lane = threadIdx.x & 63, col = lane & 31, kh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = keys_of(a, b);
  const int k0 = SPLIT ? split * a.chunk : 0, k1 = SPLIT ? min(n, k0 + a.chunk) : n;
  const int tiles = k1 > k0 ? (k1 - k0 + KT - 1) / KT : 0;

  const uint16_t *kbase = a.K.p + b * a.K.sb + hk * a.K.sh, *vbase = a.V.p + b * a.V.sb + hk * a.V.sh;
  const int crow = lane / T::CH;
  int next[COPIES];
  auto fetch = [&](int t) __attribute__((always_inline)) {
    if (IDX) {
#pragma unroll
      for (int u = 0; u < COPIES; ++u) {
        const int j = k0 + t * KT + (u * NW + wave) * T::ROWS_PER_COPY + crow;
        next[u] = j < k1 ? a.idx[(size_t)b * a.N + j] : -1;
      }
    }
  };
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < COPIES; ++u) {
      const int q = u * NW + wave, r = q * T::ROWS_PER_COPY + crow;
      const int j = k0 + t * KT + r, ch = (lane % T::CH) ^ T::key(r);
      const int64_t src = IDX ? next[u] : j;
      const bool in = IDX ? next[u] >= 0 : j < k1;
      copy16(in ? (const void*)(kbase + src * a.K.sn + 8 * ch) : (const void*)&zero16, kt[buf] + q * 1024);
      copy16(in ? (const void*)(vbase + src * a.V.sn + 8 * ch) : (const void*)&zero16, vt[buf] + q * 1024);
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
  float delta = 0.f;
  {
    const uint16_t* pq = a.Q.p + b * a.Q.sb + qr.h * a.Q.sh + qr.i * a.Q.sn + 8 * kh;
    const uint16_t* pg = a.dO.p + b * a.dO.sb + qr.h * a.dO.sh + qr.i * a.dO.sn + 8 * kh;
    const uint16_t* po = a.O.p + b * a.O.sb + qr.h * a.O.sh + qr.i * a.O.sn + 8 * kh;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      q[s] = *reinterpret_cast<const u4*>(pq + 16 * s);
      g[s] = *reinterpret_cast<const u4*>(pg + 16 * s);
      delta = dot8<DT>(g[s], *reinterpret_cast<const u4*>(po + 16 * s), delta);
    }
  }
  delta = half_sum(delta);
  const float l2 = a.lse[((size_t)b * a.Hq + qr.h) * a.M + qr.i] * 1.4426950408889634f;
  v16f acc[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) acc[db] = v16f{};

  for (int t = 0; t < tiles; ++t) {
    wait_copies();
    barrier();
    if (t + 1 < tiles) {
      copy_tile(t + 1, (t + 1) & 1);
      fetch(t + 2);
    }
    if (!active) continue;
    const uint8_t *kb = kt[t & 1], *vb = vt[t & 1];
    v16f s[2], dp[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      s[x] = v16f{};
      dp[x] = v16f{};
#pragma unroll
      for (int i = 0; i < KS; ++i) {
        s[x] = mma<DT>(T::rows(kb, 32 * x, i, lane), q[i], s[x]);
        dp[x] = mma<DT>(T::rows(vb, 32 * x, i, lane), g[i], dp[x]);
      }
    }
    const int valid = k1 - k0 - t * KT;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const bool in = 32 * x + 8 * (r >> 2) + 4 * kh + (r & 3) < valid;
        s[x][r] = in ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][r], a.c, -l2)) : 0.f;
      }
    if (n <= KT) {
      float d = 0.f;
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int r = 0; r < 16; ++r) d = __builtin_fmaf(s[x][r], dp[x][r], d);
      delta = half_sum(d);
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[x][r] *= dp[x][r] - delta;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const u4 ds = pack_half<DT>(s[x], h);
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = mma<DT>(T::cols(kb, 32 * x + 16 * h, db, lane), ds, acc[db]);
      }
    }
  }

  // what cross_dkv needs of a row; rows behind the last get probabilities of 0
  if (split == 0 && kh == 0)
    *reinterpret_cast<float2*>(a.stats + 2 * (bh * stat_rows(a.R) + row)) =
        row < a.R ? make_float2(l2, delta) : make_float2(INFINITY, 0.f);
  if (SPLIT) {
    if (row < a.R) {
      float* p = a.part_o + (((size_t)split * a.B * a.Hk + bh) * a.R + row) * D + 4 * kh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          *reinterpret_cast<float4*>(p + 32 * db + 8 * x) =
              make_float4(acc[db][4 * x], acc[db][4 * x + 1], acc[db][4 * x + 2], acc[db][4 * x + 3]);
    }
    return;
  }
  barrier();
  store_rows<DT, D>(acc, a.scale, kt[0] + wave * 32 * T::ROW, lane, [&](int r) __attribute__((always_inline)) -> uint16_t* {
    if (r0 + r >= a.R) return nullptr;
    const QueryRow w = query_row(a, hk, r0 + r);
    return a.dQ.p + b * a.dQ.sb + w.h * a.dQ.sh + w.i * a.dQ.sn;
  });
}

template <int DT, int D, bool SPLIT>
__global__ __launch_bounds__(64 * NW, 1) void cross_dkv(CrossArgs a) {
  using T = Tile<D>;
  constexpr int TB = RT * T::ROW, COPIES = RT / T::ROWS_PER_COPY / NW, KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t qt[2][TB], gt[2][TB];
  __shared__ __attribute__((aligned(16))) float st[2][2 * RT];

  const uint32_t wg = xcd_order(blockIdx.x, gridDim.x), blocks = (uint32_t)(a.N + KB - 1) / KB;
  const uint32_t rest = wg / blocks, bh = rest / (uint32_t)a.row_splits;
  const int block = wg - rest * blocks, split = rest - bh * a.row_splits;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk;
  const int lane = threadIdx.x & 63, col = lane & 31, kh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = keys_of(a, b);
  if (SPLIT && block * KB >= n) return;   // the join writes the zeros of keys that do not count
  const int r0 = SPLIT ? split * a.row_chunk : 0, r1 = SPLIT ? min(a.R, r0 + a.row_chunk) : a.R;
  const int tiles = block * KB < n ? (r1 - r0 + RT - 1) / RT : 0;

  const uint16_t *qbase = a.Q.p + b * a.Q.sb, *gbase = a.dO.p + b * a.dO.sb;
  const float* stats = a.stats + 2 * bh * stat_rows(a.R);
  const int crow = lane / T::CH;
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < COPIES; ++u) {
      const int x = u * NW + wave, r = x * T::ROWS_PER_COPY + crow;
      const int i = r0 + t * RT + r, ch = (lane % T::CH) ^ T::key(r);
      const bool in = i < a.R;
      const QueryRow w = query_row(a, hk, min(i, a.R - 1));
      copy16(in ? (const void*)(qbase + w.h * a.Q.sh + w.i * a.Q.sn + 8 * ch) : (const void*)&zero16, qt[buf] + x * 1024);
      copy16(in ? (const void*)(gbase + w.h * a.dO.sh + w.i * a.dO.sn + 8 * ch) : (const void*)&zero16, gt[buf] + x * 1024);
    }
    // row chunks are multiples of the tile, so a tile's statistics are in the padded array
    if (wave == 0 && lane < RT / 2) copy16(stats + 2 * (r0 + t * RT) + 4 * lane, st[buf]);
  };
  if (tiles > 0) copy_tile(0, 0);

  const int j = block * KB + 32 * wave + col;   // this lane's key, in the order of the list
  const bool counts = j < n;
  const bool active = block * KB + 32 * wave < n;
  const int64_t key = j < a.N ? (a.idx ? a.idx[(size_t)b * a.N + j] : j) : 0;
  u4 k[KS], v[KS];
  {
    const uint16_t *pk = a.K.p + b * a.K.sb + hk * a.K.sh + key * a.K.sn + 8 * kh;
    const uint16_t *pv = a.V.p + b * a.V.sb + hk * a.V.sh + key * a.V.sn + 8 * kh;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      k[s] = counts ? *reinterpret_cast<const u4*>(pk + 16 * s) : u4{0, 0, 0, 0};
      v[s] = counts ? *reinterpret_cast<const u4*>(pv + 16 * s) : u4{0, 0, 0, 0};
    }
  }
  v16f dk[DB], dv[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) dk[db] = dv[db] = v16f{};

  for (int t = 0; t < tiles; ++t) {
    wait_copies();
    barrier();
    if (t + 1 < tiles) copy_tile(t + 1, (t + 1) & 1);
    if (!active) continue;
    const uint8_t *qb = qt[t & 1], *gb = gt[t & 1];
    v16f s = {}, dp = {};
#pragma unroll
    for (int i = 0; i < KS; ++i) {
      s = mma<DT>(T::rows(qb, 0, i, lane), k[i], s);
      dp = mma<DT>(T::rows(gb, 0, i, lane), v[i], dp);
    }
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const float4 x = *reinterpret_cast<const float4*>(&st[t & 1][2 * (8 * g + 4 * kh)]);
      const float4 y = *reinterpret_cast<const float4*>(&st[t & 1][2 * (8 * g + 4 * kh) + 4]);
      const float l2[4] = {x.x, x.z, y.x, y.z}, dl[4] = {x.y, x.w, y.y, y.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.c, -l2[e]));
        dp[r] = s[r] * (dp[r] - dl[e]);
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const u4 p = pack_half<DT>(s, h), ds = pack_half<DT>(dp, h);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        dv[db] = mma<DT>(T::cols(gb, 16 * h, db, lane), p, dv[db]);
        dk[db] = mma<DT>(T::cols(qb, 16 * h, db, lane), ds, dk[db]);
      }
    }
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
  barrier();
  uint8_t* lds = (wave < 2 ? qt[wave] : gt[wave - 2]);
  static_assert(TB >= 32 * T::ROW, "a wave's keys fit one row tile");
  const int j0 = block * KB + 32 * wave;
  auto row_of = [&](const Strided& t, int r) __attribute__((always_inline)) -> uint16_t* {
    if (j0 + r >= a.N) return nullptr;
    const int64_t i = a.idx ? a.idx[(size_t)b * a.N + j0 + r] : j0 + r;
    return t.p + b * t.sb + hk * t.sh + i * t.sn;
  };
  store_rows<DT, D>(dk, a.scale, lds, lane, [&](int r) __attribute__((always_inline)) { return row_of(a.dK, r); });
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  store_rows<DT, D>(dv, 1.f, lds, lane, [&](int r) __attribute__((always_inline)) { return row_of(a.dV, r); });
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
  const float f = which ? 1.f : a.scale;
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
  hipError_t e;
  if (a.splits > 1) {
    if (a.idx) cross_dq<DT, D, true, true><<<gq, 64 * NW, 0, s>>>(a);
    else cross_dq<DT, D, false, true><<<gq, 64 * NW, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    cross_join_dq<DT, D><<<(unsigned)((heads * a.R + jq - 1) / jq), 256, 0, s>>>(a, gj);
  } else {
    if (a.idx) cross_dq<DT, D, true, false><<<gq, 64 * NW, 0, s>>>(a);
    else cross_dq<DT, D, false, false><<<gq, 64 * NW, 0, s>>>(a);
  }
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.row_splits > 1) {
    cross_dkv<DT, D, true><<<gk, 64 * NW, 0, s>>>(a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    cross_join_dkv<DT, D><<<dim3((unsigned)((heads * a.N + jk - 1) / jk), 2), 256, 0, s>>>(a, gkj);
  } else {
    cross_dkv<DT, D, false><<<gk, 64 * NW, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace cross

void cross_plan_backward(CrossArgs& a) {
  using namespace cross;
  cross_plan(a);
  // rows are split where the keys alone do not give every CU a workgroup
  const int64_t base = (int64_t)(a.N + KB - 1) / KB * a.B * a.Hk, tiles = ((int64_t)a.R + RT - 1) / RT;
  int64_t splits = base >= 256 ? 1 : 256 / base;
  if (splits > tiles) splits = tiles;
  const int64_t per = (tiles + splits - 1) / splits;
  a.row_chunk = (int)(per * RT);
  a.row_splits = (int)((tiles + per - 1) / per);
}

int64_t cross_stat_rows(int R) { return cross::stat_rows(R); }

hipError_t launch_cross_backward(const CrossArgs& a, hipStream_t s) {
  if (a.d == 128) return a.dtype == VC_BF16 ? cross::backward<VC_BF16, 128>(a, s) : cross::backward<VC_FP16, 128>(a, s);
  return a.dtype == VC_BF16 ? cross::backward<VC_BF16, 64>(a, s) : cross::backward<VC_FP16, 64>(a, s);
}

}  // namespace vc
