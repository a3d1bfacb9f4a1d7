// Device helpers shared by the cross attention's forward and backward kernels (not part of the public ABI).
#pragma once
#include "lanes.hpp"
#include "vc_common.hpp"
#include "vc_internal.hpp"

namespace vc {
namespace cross {

using lanes::half_max;
using lanes::half_sum;

constexpr int NXCD = 8;   // accelerator complex dies (each with its own L2)

// A source of zeros for rows that do not exist, so that a tile's padding is finite whatever the tensors hold
static __device__ const u4 zero16 = {0, 0, 0, 0};

// c += a b with 16 steps of k: 16-bit operands of 8 values a lane (row or column lane % 32, k = 8 (lane / 32) ..),
// 32x32 fp32 results (column lane % 32, register r is row 8 (r / 4) + 4 (lane / 32) + r % 4)
template <int DT>
__device__ __forceinline__ v16f mma(u4 a, u4 b, v16f c) {
  typedef __bf16 b8 __attribute__((ext_vector_type(8)));
  typedef _Float16 f8 __attribute__((ext_vector_type(8)));
  if constexpr (DT == VC_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f8, a), __builtin_bit_cast(f8, b), c, 0, 0, 0);
}

// Tiles of rows of D 16-bit values in LDS, without padding: the 16-byte piece `ch` of row `r` stands in place
// ch ^ key(r). 256 bytes of LDS are read in a cycle: by rows, the same piece of 16 rows, whose keys therefore differ; by
// columns (transposing reads), four neighbouring pieces of four rows, so the keys of four rows differ in the bits above
// the lowest two. (With key(r) = r, in which four rows' pieces stand in the same banks, LDS was busy for 1.9 times as
// long in the kernel of dK and dV.)
template <int D>
struct Tile {
  static constexpr int CH = D / 8;              // pieces of a row
  static constexpr int ROW = 2 * D;             // bytes of a row
  static constexpr int ROWS_PER_COPY = 64 / CH; // rows that one wave's copy moves
  // (of 64 channels, two rows fill the 256 bytes)
  __device__ static __forceinline__ int key(int r) {
    return D == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
  }
  __device__ static __forceinline__ int at(int r, int ch) { return r * ROW + ((ch ^ key(r)) << 4); }
};

// A lane's addresses of operands in a tile. move() puts them to a tile; loads then name rows of it by a constant offset
// `off`, the bytes of its row r0 (a multiple of 16).
template <int D>
struct RowOperands {
  using T = Tile<D>;
  uint32_t at[D / 16];
  __device__ __forceinline__ RowOperands() = default;
  __device__ __forceinline__ explicit RowOperands(int lane) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) at[s] = T::at(lane & 31, 2 * s + (lane >> 5));
  }
  __device__ __forceinline__ RowOperands move(uint32_t lds) const {
    RowOperands r;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      r.at[s] = at[s] + lds;
      lanes::pin(r.at[s]);   // formed here, once
    }
    return r;
  }
  // from one tile of a ring to the next
  __device__ __forceinline__ void shift(uint32_t by) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) at[s] += by;
  }
  // rows r0 .. r0 + 31 at k-step s: lane (l % 32, h) gets channels 16 s + 8 h .. + 7 of its row
  __device__ __forceinline__ u4 get(uint32_t off, int s) const {
    return *(const __attribute__((address_space(3))) u4*)(at[s] + off);
  }
};
template <int D>
struct ColOperands {
  using T = Tile<D>;
  uint32_t lo[D / 32], hi[D / 32];
  __device__ __forceinline__ ColOperands() = default;
  __device__ __forceinline__ explicit ColOperands(int lane) {
    const int r = 4 * (lane >> 5) + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      lo[db] = T::at(r, 4 * db + ch) + 8 * (lane & 1);
      hi[db] = T::at(r + 8, 4 * db + ch) + 8 * (lane & 1);
    }
  }
  __device__ __forceinline__ ColOperands move(uint32_t lds) const {
    ColOperands r;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      r.lo[db] = lo[db] + lds, r.hi[db] = hi[db] + lds;
      lanes::pin(r.lo[db]);
      lanes::pin(r.hi[db]);
    }
    return r;
  }
  __device__ __forceinline__ void shift(uint32_t by) {
#pragma unroll
    for (int db = 0; db < D / 32; ++db) lo[db] += by, hi[db] += by;
  }
  // channels 32 db .. + 31 (lane % 32) with 16 rows from r0 as the k, in the order in which a lane's results of a 32x32
  // product hold them: element e of half h is row r0 + 8 (e / 4) + 4 h + e % 4. The reads transpose: of 16 lanes, lane i
  // brings 4 values at piece-half i % 4 of row i / 4, and receives value i of the 4 rows.
  __device__ __forceinline__ u4 get(uint32_t off, int db) const {
    const u2 x = read_tr(lo[db] + off), y = read_tr(hi[db] + off);
    return u4{x[0], x[1], y[0], y[1]};
  }
  __device__ static __forceinline__ u2 read_tr(uint32_t lds) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(lds)));
  }
};

// Order of issue from here to the next barrier or scheduling fence: groups of LDS reads and matrix instructions, so that
// operands are read several products ahead of their use. (Left alone, the compiler waits for each operand where it is used.)
template <int READS>
__device__ __forceinline__ void issue_reads() {
  __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
}
template <int PRODUCTS, int READS>
__device__ __forceinline__ void issue_products() {
#pragma unroll
  for (int i = 0; i < PRODUCTS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    if (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
}

__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)p));
}

// One wave's copy of 16 bytes a lane from memory straight into LDS at lds + 16 lane. Issued as asm so that the compiler
// adds no waits of its own: copies are waited for (wait_copies) before the barrier that precedes their first use.
__device__ __forceinline__ void copy16(const void* src, const void* lds) {
  const uint32_t to = __builtin_amdgcn_readfirstlane(
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)lds)));
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(to) : "memory", "m0");
}

// Scores of the keys (rows of a 32x32 result) behind the first `valid` become -inf. For a branch that is taken once a row
// block at most; the pin keeps the comparisons in it.
__device__ __forceinline__ void mask_scores(v16f& s, int valid, int kh) {
  int rest = valid - 4 * kh;
  lanes::pin(rest);
#pragma unroll
  for (int r = 0; r < 16; ++r)
    if (8 * (r >> 2) + (r & 3) >= rest) s[r] = -INFINITY;
}
__device__ __forceinline__ void mask_scores(v16f (&s)[2], int valid, int kh) {
  mask_scores(s[0], valid, kh);
  mask_scores(s[1], valid - 32, kh);
}

// The copies of a tile of ROWS rows at a constant stride (in elements, below FAR_STRIDE) by the NW waves of a workgroup,
// through a buffer descriptor: a lane's offset from the tile's first row is the same for all tiles, and rows behind
// the `valid` first are out of the buffer's range, which reads as zero without an access.
constexpr int64_t FAR_STRIDE = 1 << 22;   // 256 rows of less than this stay below 2^31 bytes
// Strides that a buffer does not serve: too far, or rows that overlap (shared ones: 0), of which those behind the last
// would not be out of range
inline bool off_buffer(const Strided& t, int d) { return t.sn >= FAR_STRIDE || t.sn < d; }
template <int D, int ROWS, int NW>
struct Copier {
  using T = Tile<D>;
  static constexpr int COPIES = ROWS / T::ROWS_PER_COPY / NW;
  static constexpr int STEP = NW * T::ROWS_PER_COPY;   // rows between two copies of a wave
  uint32_t off, row_bytes;
  int r, ch;
  __device__ __forceinline__ Copier(int64_t stride, int wave, int lane) {
    row_bytes = 2 * (uint32_t)stride;
    r = wave * T::ROWS_PER_COPY + lane / T::CH;
    ch = lane % T::CH;
    off = place(0);
  }
  __device__ __forceinline__ uint32_t place(int u) const {
    return (r + u * STEP) * row_bytes + 16 * (ch ^ T::key(r + u * STEP));
  }
  // tile: address of the tile's first row, the same for all lanes
  __device__ __forceinline__ void copy(const uint16_t* tile, int valid, const uint8_t* lds, int wave) const {
    typedef int v4i __attribute__((ext_vector_type(4)));
    const uint64_t p = reinterpret_cast<uint64_t>(tile);
    const uint32_t bytes = valid > 0 ? (min(valid, ROWS) - 1) * row_bytes + T::ROW : 0u;
    const v4i rsrc = {(int)(uint32_t)p, (int)(uint32_t)(p >> 32), (int)bytes, 0x00020000};
    const uint32_t to = lds_addr(lds) + wave * 1024;
#pragma unroll
    for (int u = 0; u < COPIES; ++u)   // (keys repeat every 16 rows)
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(
                       STEP % 16 == 0 ? off + u * STEP * row_bytes : place(u)),
                   "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(to + u * NW * 1024))
                   : "memory", "m0");
  }
};

// at most N of this wave's memory operations are in flight (they end in order)
template <int N = 0>
__device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Workgroup barrier; the wave's LDS operations are done before it, copies in flight stay in flight
__device__ __forceinline__ void barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
}

// The dispatcher deals workgroups to the XCDs round-robin; this bijection gives each a contiguous range, so that its
// L2 holds the keys and values of few heads
__device__ __forceinline__ uint32_t xcd_order(uint32_t id, uint32_t total) {
  const uint32_t x = id % NXCD, q = total / NXCD, r = total % NXCD;
  return x * q + min(x, r) + id / NXCD;
}

// groups of lanes that share a joined row: up to eight, with four parts or fewer each
inline int join_groups(int parts) { return parts <= 4 ? 1 : parts <= 8 ? 2 : parts <= 16 ? 4 : 8; }

// A lane's row of D channels held as results of 32x32 products (column = row; the other half of the channels in lane
// l ^ 32), times f, handed to `put` in pieces: put(c, w) stores the 8 channels from c on. Halves exchange four channels of
// every eight, so that a lane stores 16 bytes and its row's two lanes 32 bytes side by side.
template <int DT, int D, typename F>
__device__ __forceinline__ void row_pieces(const v16f (&o)[D / 32], float f, int lane, F put) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      u4 w;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t x = pack2<DT>(o[db][4 * g + 2 * i] * f, o[db][4 * g + 2 * i + 1] * f);
        const uint32_t y = pack2<DT>(o[db][4 * g + 4 + 2 * i] * f, o[db][4 * g + 4 + 2 * i + 1] * f);
        const auto r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
        w[i] = r[0];
        w[2 + i] = r[1];
      }
      put(32 * db + 8 * g + 8 * (lane >> 5), w);
    }
}
// stored at p (null: not at all)
template <int DT, int D>
__device__ __forceinline__ void store_row(const v16f (&o)[D / 32], float f, uint16_t* p, int lane) {
  row_pieces<DT, D>(o, f, lane, [&](int c, u4 w) __attribute__((always_inline)) {
    if (p) *reinterpret_cast<u4*>(p + c) = w;
  });
}

// A buffer of `bytes` at p (the same for all lanes): accesses behind its end are left out, and every store is one
// instruction whatever lanes take part, so that the operations in flight can be counted
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(p, 0, (int)bytes, 0x00020000);
}

// The kernel's arguments (its first parameter) read anew from memory: for what a loop needs seldom, which would otherwise
// hold scalar registers throughout
__device__ __forceinline__ CrossArgs fresh_args() {
  auto p = (const __attribute__((address_space(4))) CrossArgs*)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return *(const CrossArgs*)p;
}

// keys of batch item b that count
__device__ __forceinline__ int keys_of(const CrossArgs& a, int b) {
  if (a.count) return a.count[b];
  if (a.k_len) return max(0, min(a.k_len[b], a.N));
  return a.N;
}

// Row r of key head hk: query head hk G + r / M, query r % M
struct QueryRow {
  int h, i;
};
__device__ __forceinline__ QueryRow query_row(const CrossArgs& a, int hk, int r) {
  if (a.G == 1) return {hk, r};
  const int g = (uint32_t)r / (uint32_t)a.M;
  return {hk * a.G + g, r - g * a.M};
}

}  // namespace cross
}  // namespace vc
