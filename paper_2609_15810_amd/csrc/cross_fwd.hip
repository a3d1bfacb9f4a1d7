// Attention of queries to the states of another sequence, 16-bit operands, forward.
//
//   O_i = sum_j p_ij v_j,  p_ij = exp(c' q_i k_j - lse_i),  lse_i = log sum_j exp(c' q_i k_j)
//
// over the keys j that count for the batch item. Keys are visited in tiles of 64 with a running maximum and sum; exponents
// are in log2 units (c = c' log2 e). Both products are computed transposed so that a lane owns one query (column
// lane % 32 of a 32x32 product): S^T = K Q^T with keys from LDS and the wave's 32 queries in registers, then
// O^T += V^T P^T, for which the probabilities of a lane are already in operand order and V is read from LDS by
// transposing reads. A workgroup's four waves share the tiles (128 rows); tiles are copied straight into LDS, one
// tile ahead.
//
// The rows of a key head are those of all its query heads, one head behind the other, so that grouped heads share
// tiles and a token's few queries share one. Calls of 128 channels with rows for 256 workgroups of 256 take cross_fwd_wide
// instead, whose workgroups walk over blocks of rows of a head. Measured (us, this kernel / wide): 12 heads of 32760 rows over
// 64 keys 44 / 42, over 512 keys 129 / 122, over 1024 keys 232 / 214; 40 heads of 75600 rows over 512 keys 1099 / 1036 (1.5 GB,
// 793 GFLOP); with 192 workgroups (12 heads of 4096 rows) 26 / 26, below that it loses CUs. Of 64 channels, four waves of this
// kernel fit a SIMD, and the wide one has two: 12 heads of 32760 rows over 64 keys 23 / 28, over 512 66 / 88, over 2048 222 / 291.
//
// What bounds it: 16 bytes of LDS are read per product and lane, exponentials and products take about the same time, and the
// card lowers its clock under the matrix cores' load (1.7 GHz at their full rate on random operands); the sustained rate of
// a large library product here is 1.06 to 1.35 PFLOP/s, of this kernel 0.85.
//
// Few rows and long keys: the keys are split over workgroups (cross_plan), each leaves unnormalised fp32 outputs with its
// maximum and sum, and cross_join adds them up in a fixed order.
#include <type_traits>

#include "cross_common.hpp"

namespace vc {
namespace cross {
namespace {

constexpr int NW = 4;           // waves of a workgroup
constexpr int QR = 32 * NW;     // its rows
constexpr int KT = 64;          // keys of a tile

// A row's exponents are relative to a reference that follows its running maximum at a distance of at most LAG (log2
// units): it moves, and the sums are rescaled, only where the maximum has left it by more. Probabilities then reach 2^LAG,
// which the 16-bit types and the fp32 sums hold with the same relative errors. In fp16 the reference starts SHIFT below the
// maximum, so that probabilities reach 2^15 and those down to 2^-21 of the largest are normal numbers.
constexpr float LAG = 8.f;
template <int DT>
constexpr float SHIFT = DT == VC_FP16 ? 7.f : 0.f;

// A lane's row: O = o / l and lse
template <int DT, int D>
__device__ __forceinline__ void finish_row(const CrossArgs& a, int b, int hk, int row, int n, const v16f (&o)[D / 32], float m,
                                           float l, int lane) {
  const QueryRow w = query_row(a, hk, min(row, a.R - 1));
  // no key counts: O = 0, lse = -inf
  const float inv = n > 0 ? 1.f / l : 0.f;
  if (a.lse && row < a.R && lane < 32)
    a.lse[((size_t)b * a.Hq + w.h) * a.M + w.i] = n > 0 ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
  store_row<DT, D>(o, inv, row < a.R ? a.O.p + b * a.O.sb + w.h * a.O.sh + w.i * a.O.sn : nullptr, lane);
}

// GATHER: addresses per key (the keys are those of a list, or off_buffer);
// SPLIT: leave parts
template <int DT, int D, bool GATHER, bool SPLIT>
__global__ __launch_bounds__(64 * NW, 2) void cross_fwd(CrossArgs a) {
  using T = Tile<D>;
  using C = Copier<D, KT, NW>;
  constexpr int TB = KT * T::ROW;                                // bytes of a tile
  constexpr int KS = D / 16, DB = D / 32;
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
  const C kc(a.K.sn, wave, lane), vc(a.V.sn, wave, lane);
  int next[C::COPIES];   // GATHER: keys of the next tile to copy
  auto fetch = [&](int t) __attribute__((always_inline)) {
    if (GATHER) {
#pragma unroll
      for (int u = 0; u < C::COPIES; ++u) {
        const int j = k0 + t * KT + (u * NW + wave) * T::ROWS_PER_COPY + crow;
        next[u] = j < k1 ? (a.idx ? a.idx[(size_t)b * a.N + j] : j) : -1;
      }
    }
  };
  auto copy_tile = [&](int t, int buf) __attribute__((always_inline)) {
    if (GATHER) {
#pragma unroll
      for (int u = 0; u < C::COPIES; ++u) {
        const int q = u * NW + wave, ch = (lane % T::CH) ^ T::key(q * T::ROWS_PER_COPY + crow);
        const int64_t src = next[u];
        copy16(src >= 0 ? (const void*)(kbase + src * a.K.sn + 8 * ch) : (const void*)&zero16, kt[buf] + q * 1024);
        copy16(src >= 0 ? (const void*)(vbase + src * a.V.sn + 8 * ch) : (const void*)&zero16, vt[buf] + q * 1024);
      }
    } else {
      const int j = k0 + t * KT;
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
  const bool active = r0 < a.R;   // waves without rows only copy
  const QueryRow qr = query_row(a, hk, min(row, a.R - 1));
  u4 q[KS];
  {
    const uint16_t* p = a.Q.p + b * a.Q.sb + qr.h * a.Q.sh + qr.i * a.Q.sn + 8 * kh;
#pragma unroll
    for (int s = 0; s < KS; ++s) q[s] = *reinterpret_cast<const u4*>(p + 16 * s);
  }
  v16f o[DB];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db] = v16f{};
  const RowOperands<D> rows0(lane);
  const ColOperands<D> cols0(lane);
  float m = -INFINITY, l = 0.f;   // the reference; the sum of this lane's keys

  for (int t = 0; t < tiles; ++t) {
    wait_copies();
    barrier();
    if (t + 1 < tiles) {
      copy_tile(t + 1, (t + 1) & 1);
      fetch(t + 2);
    }
    if (!active) continue;
    const RowOperands<D> rows = rows0.move(lds_addr(kt[0]) + (t & 1) * TB);
    const ColOperands<D> cols = cols0.move(lds_addr(vt[0]) + (t & 1) * TB);
    v16f s[2];
#pragma unroll
    for (int g = 0; g < 2; ++g) s[g] = v16f{};
#pragma unroll
    for (int i = 0; i < KS; ++i)
#pragma unroll
      for (int g = 0; g < 2; ++g) s[g] = mma<DT>(rows.get(32 * g * T::ROW, i), q[i], s[g]);
    issue_reads<6>();
    issue_products<2 * KS - 6, 1>();
    issue_products<6, 0>();
    __builtin_amdgcn_sched_barrier(0);
    const int valid = k1 - k0 - t * KT;
    if (valid < KT) mask_scores(s, valid, kh);
    float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, s[0][r]), s[1][r]);
    top = half_max(top) * a.c;
    if (__builtin_amdgcn_ballot_w64(top > m + (LAG + SHIFT<DT>))) {
      const float up = top > m + (LAG + SHIFT<DT>) ? top - SHIFT<DT> : m, alpha = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.f : up));
      m = up;
      l *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    }
    const float off = m == -INFINITY ? 0.f : m;   // scores of -inf alone so far
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g][8 * h + e], a.c, -off));
          l += p[e];
        }
        const u4 pp = {pack2<DT>(p[0], p[1]), pack2<DT>(p[2], p[3]), pack2<DT>(p[4], p[5]), pack2<DT>(p[6], p[7])};
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = mma<DT>(cols.get((32 * g + 16 * h) * T::ROW, db), pp, o[db]);
      }
  }
  l = half_sum(l);

  if (SPLIT) {
    if (row < a.R) {
      const size_t at = ((size_t)split * a.B * a.Hk + bh) * a.R + row;
      if (kh == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m, l);
      float* p = a.part_o + at * D + 4 * kh;
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *reinterpret_cast<float4*>(p + 32 * db + 8 * g) =
              make_float4(o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]);
    }
    return;
  }
  finish_row<DT, D>(a, b, hk, row, n, o, m, l, lane);
}

// Many rows: a workgroup on each CU, of eight waves of 32 rows that share the tiles, two on each SIMD, in two groups that are
// half a step apart: while one group's waves issue products (the values of a tile, then the scores of the next), those of
// the other form probabilities; a barrier ends each half step, so that the matrix cores always have one group's products.
// The workgroup walks over blocks of 256 rows of a query head, those of a head without a break: their tiles are one sequence,
// copied two steps ahead (pair g: K of tile g and V of tile g - 1, both first read by the products of step g), the next
// block's queries are copied into LDS a block ahead, and a block's rows are stored in the first step of the next.
constexpr int WW = 8;           // waves
constexpr int WR = 32 * WW;     // rows of a block
constexpr int RING = 3;         // tiles of K and of V in LDS

template <int DT, int D, bool GATHER>
__global__ __launch_bounds__(64 * WW, 2) void cross_fwd_wide(CrossArgs a, int total) {
  using T = Tile<D>;
  using C = Copier<D, KT, WW>;
  constexpr int TB = KT * T::ROW, KS = D / 16, DB = D / 32;
  __shared__ __attribute__((aligned(16))) uint8_t kt[RING][TB], vt[RING][TB], qt[WR * T::ROW];

  const int blocks = (a.M + WR - 1) / WR;   // of a query head
  const uint32_t wg = xcd_order(blockIdx.x, gridDim.x);
  const int end = (int)((int64_t)total * (wg + 1) / gridDim.x);
  const int lane = threadIdx.x & 63, col = lane & 31, kh = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool late = wave >= WW / 2;
  const C kc(a.K.sn, wave, lane), vc(a.V.sn, wave, lane);

  uint8_t* const mine = qt + wave * 32 * T::ROW;   // this wave's queries of the next block

  for (int block = (int)((int64_t)total * wg / gridDim.x); block < end;) {
    // the blocks of one query head from here on
    const uint32_t bh = block / (uint32_t)blocks;
    const int b = bh / (uint32_t)a.Hq, h = bh - b * a.Hq;
    const int rb = block - bh * blocks, count = min(end - block, blocks - rb);
    block += count;
    const int n = __builtin_amdgcn_readfirstlane(keys_of(fresh_args(), b)), tiles = (n + KT - 1) / KT;

    u4 q[KS], p[4];
    v16f o[DB], s[2];
    float m = -INFINITY, l = 0.f;   // the reference; the sum of this lane's keys
    // The rows of a finished block; the sums start anew where the reference is -inf. As many stores in every call: one per
    // piece of a row and one of lse.
    constexpr int STORES = D / 16;
    auto finish = [&](int x) __attribute__((always_inline)) {
      const CrossArgs f = fresh_args();
      const int r0 = (rb + x) * WR, rows = min(WR, f.M - r0);
      const float sum = half_sum(l), inv = n > 0 ? 1.f / sum : 0.f;
      const auto out = buffer_of(f.O.p + b * f.O.sb + h * f.O.sh + r0 * f.O.sn, (uint32_t)(rows - 1) * 2 * f.O.sn + 2 * D);
      const int at = (32 * wave + col) * 2 * (int)f.O.sn;
      row_pieces<DT, D>(o, inv, lane, [&](int c, u4 w) __attribute__((always_inline)) {
        __builtin_amdgcn_raw_buffer_store_b128(w, out, at + 2 * c, 0, 0);
      });
      // (without an lse: a buffer of no bytes)
      const auto lse = buffer_of(f.lse ? f.lse + ((size_t)b * f.Hq + h) * f.M + r0 : nullptr, f.lse ? 4 * rows : 0);
      const float value = n > 0 ? (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f : -INFINITY;
      __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(value), lse, 4 * (32 * wave + col), 0, 0);
      m = -INFINITY;
    };
    if (n == 0) {
#pragma unroll
      for (int db = 0; db < DB; ++db) o[db] = v16f{};
      for (int x = 0; x < count; ++x) finish(x);
      continue;
    }

    const CrossArgs f = fresh_args();
    const uint32_t hk = (uint32_t)h / (uint32_t)f.G;
    const uint16_t *kbase = f.K.p + b * f.K.sb + hk * f.K.sh, *vbase = f.V.p + b * f.V.sb + hk * f.V.sh;
    auto copy_one = [&](const uint16_t* base, int64_t sn, const C& c, int t, uint8_t* to) __attribute__((always_inline)) {
      if (GATHER) {
#pragma unroll
        for (int u = 0; u < C::COPIES; ++u) {
          const int x = u * WW + wave, r = x * T::ROWS_PER_COPY + lane / T::CH, j = t * KT + r;
          const int64_t src = j < n ? (a.idx ? a.idx[(size_t)b * a.N + j] : j) : -1;
          copy16(src >= 0 ? (const void*)(base + src * sn + 8 * ((lane % T::CH) ^ T::key(r))) : (const void*)&zero16,
                 to + x * 1024);
        }
      } else {
        c.copy(base + (int64_t)t * KT * sn, n - t * KT, to, wave);
      }
    };
    // the next pair to copy: K of tile `ahead` of a block, of `left` blocks still to come; V of tile `behind`
    int left = count, pair = 0, ahead = 0, behind = -1;
    auto copy_pair = [&]() __attribute__((always_inline)) {
      if (behind >= 0) copy_one(vbase, a.V.sn, vc, behind, vt[(pair + RING - 1) % RING]);
      behind = -1;
      if (left > 0) {
        copy_one(kbase, a.K.sn, kc, ahead, kt[pair % RING]);
        behind = ahead;
        ++ahead;
        if (ahead == tiles) ahead = 0, --left;
      }
      pair = (pair + 1) % RING;
    };
    // this wave's queries of block x: on their way into LDS, and from there
    auto copy_queries = [&](int x) __attribute__((always_inline)) {
      const CrossArgs f = fresh_args();
      const int r0 = (rb + x) * WR + 32 * wave;
      int l = lane;
      lanes::pin(l);   // (seldom: its addresses are not to be held)
      Copier<D, 32, 1>(f.Q.sn, 0, l).copy(f.Q.p + b * f.Q.sb + h * f.Q.sh + r0 * f.Q.sn, f.M - r0, mine, 0);
    };
    auto load_queries = [&]() __attribute__((always_inline)) {
      wait_copies<0>();
      int l = lane;
      lanes::pin(l);
      const RowOperands<D> at = RowOperands<D>(l).move(lds_addr(mine));
#pragma unroll
      for (int s = 0; s < KS; ++s) q[s] = at.get(0, s);
#pragma unroll
      for (int s = 0; s < KS; ++s) lanes::pin(q[s]);
    };
    // operands of the tile whose scores, and of that whose values come next
    RowOperands<D> rows = RowOperands<D>(lane).move(lds_addr(kt[0]));
    ColOperands<D> cols = ColOperands<D>(lane).move(lds_addr(vt[0]));
    auto scores = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < 2; ++x) s[x] = v16f{};
#pragma unroll
      for (int i = 0; i < KS; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) s[x] = mma<DT>(rows.get(32 * x * T::ROW, i), q[i], s[x]);
    };
    auto values = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] = mma<DT>(cols.get(16 * i * T::ROW, db), p[i], o[db]);
    };
    auto probabilities = [&](bool first, int valid) __attribute__((always_inline)) {
      if (valid < KT) mask_scores(s, valid, kh);
      float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
      for (int r = 1; r < 16; ++r) top = fmaxf(fmaxf(top, s[0][r]), s[1][r]);
      top = half_max(top) * a.c;
      if (first || __builtin_amdgcn_ballot_w64(top > m + (LAG + SHIFT<DT>))) {   // (the first tile of a block always clears its sums)
        const float up = top > m + (LAG + SHIFT<DT>) ? top - SHIFT<DT> : m, alpha = __builtin_amdgcn_exp2f(m - (up == -INFINITY ? 0.f : up));
        const bool anew = m == -INFINITY;   // (selected, not multiplied: what stands there may not be finite)
        m = up;
        l = anew ? 0.f : l * alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[db][r] = anew ? 0.f : o[db][r] * alpha;
      }
      const float off = m == -INFINITY ? 0.f : m;   // scores of -inf alone so far
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float e[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          e[x] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i >> 1][8 * (i & 1) + x], a.c, -off));
          l += e[x];
        }
        p[i] = u4{pack2<DT>(e[0], e[1]), pack2<DT>(e[2], e[3]), pack2<DT>(e[4], e[5]), pack2<DT>(e[6], e[7])};
      }
    };

    copy_queries(0);
    for (int x = 0; x < RING - 1; ++x) copy_pair();
    load_queries();
    if (count > 1) copy_queries(1);
    barrier();
    if (late) barrier();
    scores();
    barrier();
    int slot = 0, x = 0, t = 0;   // of the tile at work: its place in the ring, its block, its place in the block
    rows.shift(TB);
    bool stored = false;
    for (;;) {
      // probabilities
      copy_pair();
      if (stored) finish(x - 1);   // the block before the one at work is complete
      const bool last = t + 1 == tiles;
      probabilities(t == 0, n - t * KT);
      if (last && x + 1 < count) {
        load_queries();
        if (x + 2 < count) copy_queries(x + 2);
      }
      barrier();
      if (last && x + 1 == count) break;
      // products: values of this tile, scores of the next
      
      values();
      scores();
      // operands are read six products ahead of their use
      issue_reads<12>();
      issue_products<4 * DB - 6, 2>();
      issue_products<6, 1>();
      issue_products<2 * KS - 6, 1>();
      issue_products<6, 0>();
      
      cols.shift(slot < RING - 1 ? TB : -(RING - 1) * TB);
      slot = slot + 1 < RING ? slot + 1 : 0;
      rows.shift(slot < RING - 1 ? TB : -(RING - 1) * TB);
      // the next pair is there; rows that were stored behind it may be on their way
      if (stored && !last) wait_copies<STORES + 1>();
      else wait_copies<0>();
      barrier();
      stored = last;
      ++t;
      if (last) {
        ++x;
        t = 0;
      }
    }
    values();
    finish(x);
    if (!late) barrier();   // the groups meet again
    barrier();              // and the tiles are read no more
  }
}

// The parts of a row joined: d / 4 lanes and `groups` (a power of two) of them share a row, group g taking the
// parts g, g + groups, ..; the groups' sums meet in LDS. (One group walking 24 parts of the 32 rows of a token: 12 us, the
// loads of a part waiting for the one before.)
template <int DT, int D>
__global__ __launch_bounds__(256) void cross_join(CrossArgs a, int groups) {
  constexpr int L = D / 4, ALL = 256 / L;
  __shared__ __attribute__((aligned(16))) float so[ALL][D];
  __shared__ float2 sml[ALL];
  const int lane = threadIdx.x % L, slot = threadIdx.x / L, g = slot & (groups - 1), c = 4 * lane;
  const int64_t rows = (int64_t)a.B * a.Hk * a.R, at = (int64_t)blockIdx.x * (ALL / groups) + slot / groups;
  float m = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](float2 ml, float4 v) __attribute__((always_inline)) {
    const float up = fmaxf(m, ml.x), off = up == -INFINITY ? 0.f : up;
    const float x = __builtin_amdgcn_exp2f(m - off), w = __builtin_amdgcn_exp2f(ml.x - off);
    m = up;
    l = __builtin_fmaf(w, ml.y, l * x);
    o.x = __builtin_fmaf(w, v.x, o.x * x), o.y = __builtin_fmaf(w, v.y, o.y * x);
    o.z = __builtin_fmaf(w, v.z, o.z * x), o.w = __builtin_fmaf(w, v.w, o.w * x);
  };
  if (at < rows) {
#pragma unroll 4
    for (int s = g; s < a.splits; s += groups)
      add(*reinterpret_cast<const float2*>(a.part_ml + 2 * (s * rows + at)),
          *reinterpret_cast<const float4*>(a.part_o + (s * rows + at) * D + c));
  }
  if (groups > 1) {
    *reinterpret_cast<float4*>(&so[slot][c]) = o;
    if (lane == 0) sml[slot] = make_float2(m, l);
    __syncthreads();
    if (g == 0)
      for (int i = 1; i < groups; ++i) add(sml[slot + i], *reinterpret_cast<const float4*>(&so[slot + i][c]));
  }
  if (g != 0 || at >= rows) return;
  const uint32_t bh = at / a.R;
  const int b = bh / (uint32_t)a.Hk, hk = bh - b * a.Hk, n = keys_of(a, b);
  const QueryRow w = query_row(a, hk, (int)(at - (int64_t)bh * a.R));
  const float inv = n > 0 ? 1.f / l : 0.f;
  *reinterpret_cast<u2*>(a.O.p + b * a.O.sb + w.h * a.O.sh + w.i * a.O.sn + c) =
      u2{pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv)};
  if (a.lse && c == 0)
    a.lse[((size_t)b * a.Hq + w.h) * a.M + w.i] = n > 0 ? (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : -INFINITY;
}

// The list of the keys that count: keys in ascending order, those that count first. A workgroup lists LIST keys of a batch
// item, four a thread; it counts those of the whole item and those before its own by itself (16 bytes of the mask a
// load), so that no workgroup waits for another: 6 us for 32760 keys of two items, 3 us for 1000 (one workgroup an item,
// 1024 keys at a time: 29 us).
constexpr int LIST = 4096;
__global__ __launch_bounds__(1024) void cross_keys(const uint8_t* mask, int64_t stride, const int32_t* k_len, int N,
                                                   int32_t* idx, int32_t* count) {
  __shared__ int sums[3][16];   // of the waves
  const uint32_t parts = ((uint32_t)N + LIST - 1) / LIST;
  const int b = blockIdx.x / parts, j0 = (blockIdx.x - b * parts) * LIST;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint8_t* mb = mask + b * stride;
  const int len = k_len ? max(0, min(k_len[b], N)) : N;
  // this thread's keys (a bit each)
  const int j = j0 + 4 * tid;
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < len && mb[j + e] != 0) bits |= 1u << e;
  // keys that count in the item and before j0
  int all = 0, prior = 0;
  if (parts > 1)
    for (int64_t i = 16 * tid; i < len; i += 16 * 1024) {
      int here = 0;
      if (i + 16 <= len) {
        uint32_t w[4];
        __builtin_memcpy(w, mb + i, 16);
#pragma unroll
        for (int e = 0; e < 16; ++e) here += (w[e / 4] >> (8 * (e % 4)) & 0xff) != 0;
      } else {
        for (int64_t e = i; e < len; ++e) here += mb[e] != 0;
      }
      all += here;
      if (i < j0) prior += here;
    }
  int mine = __popc(bits), up = mine;   // up: of the wave's lanes to this one
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(up, o, 64);
    up += lane >= o ? v : 0;
  }
  if (parts > 1)
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o, 64), prior += __shfl_xor(prior, o, 64);
  if (lane == 63) sums[0][wave] = up, sums[1][wave] = all, sums[2][wave] = prior;
  __syncthreads();
  int before = up - mine, total = 0;
  for (int w = 0; w < 16; ++w) {
    before += (w < wave ? sums[0][w] : 0) + sums[2][w];
    total += sums[parts > 1 ? 1 : 0][w];
  }
  int32_t* out = idx + (size_t)b * N;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (j + e < N) {
      const int on = bits >> e & 1;
      out[on ? before : total + (j + e - before)] = j + e;
      before += on;
    }
  if (j0 == 0 && tid == 0) count[b] = total;
}

template <int DT, int D>
hipError_t forward(const CrossArgs& a, hipStream_t s) {
  const unsigned grid = (unsigned)((int64_t)(a.R + QR - 1) / QR * a.B * a.Hk * a.splits);
  const bool gather = a.idx || off_buffer(a.K, D) || off_buffer(a.V, D);
  const int wide = (int)((int64_t)(a.M + WR - 1) / WR * a.B * a.Hq);
  if constexpr (D == 128)
    if (a.splits == 1 && wide >= 256 && a.M >= WR && a.Q.sn < FAR_STRIDE && a.O.sn < FAR_STRIDE) {
      if (gather) cross_fwd_wide<DT, D, true><<<256, 64 * WW, 0, s>>>(a, wide);
      else cross_fwd_wide<DT, D, false><<<256, 64 * WW, 0, s>>>(a, wide);
      return hipGetLastError();
    }
  if (a.splits > 1) {
    if (gather) cross_fwd<DT, D, true, true><<<grid, 64 * NW, 0, s>>>(a);
    else cross_fwd<DT, D, false, true><<<grid, 64 * NW, 0, s>>>(a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int groups = join_groups(a.splits), rows = 256 / (D / 4) / groups;
    cross_join<DT, D><<<(unsigned)(((int64_t)a.B * a.Hk * a.R + rows - 1) / rows), 256, 0, s>>>(a, groups);
  } else {
    if (gather) cross_fwd<DT, D, true, false><<<grid, 64 * NW, 0, s>>>(a);
    else cross_fwd<DT, D, false, false><<<grid, 64 * NW, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace cross

hipError_t launch_cross_keys(const uint8_t* k_mask, int64_t stride, const int32_t* k_len, int B, int N, int32_t* idx,
                             int32_t* count, hipStream_t s) {
  const unsigned parts = ((unsigned)N + cross::LIST - 1) / cross::LIST;
  cross::cross_keys<<<B * parts, 1024, 0, s>>>(k_mask, stride, k_len, N, idx, count);
  return hipGetLastError();
}

void cross_plan(CrossArgs& a) {
  using namespace cross;
  // Keys are split where the rows alone do not give every CU two workgroups, into as many parts as fit the CUs at once (with
  // four workgroups more than that, 64 rows of 12 heads over 32760 keys take 55 us instead of 46), and only where that shortens
  // a workgroup's walk by more than the joining launch costs: a tile takes 1.3 us alone, the join 4 to 5 us
  const int64_t base = (int64_t)(a.R + QR - 1) / QR * a.B * a.Hk;
  const int64_t tiles = (a.N + KT - 1) / KT;
  int64_t splits = base >= 256 ? 1 : 512 / base;
  if (splits > tiles) splits = tiles;
  int64_t per = (tiles + splits - 1) / splits;
  if (tiles - per < 5) per = tiles;
  a.chunk = (int)(per * KT);
  a.splits = (int)((tiles + per - 1) / per);
}

hipError_t launch_cross_forward(const CrossArgs& a, hipStream_t s) {
  if (a.d == 128) return a.dtype == VC_BF16 ? cross::forward<VC_BF16, 128>(a, s) : cross::forward<VC_FP16, 128>(a, s);
  return a.dtype == VC_BF16 ? cross::forward<VC_BF16, 64>(a, s) : cross::forward<VC_FP16, 64>(a, s);
}

}  // namespace vc
