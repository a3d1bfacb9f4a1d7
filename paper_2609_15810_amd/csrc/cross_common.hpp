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
// ch ^ key(r), so that the pieces that 16 lanes read from 16 consecutive rows lie in different banks.
template <int D>
struct Tile {
  static constexpr int CH = D / 8;              // pieces of a row
  static constexpr int ROW = 2 * D;             // bytes of a row
  static constexpr int ROWS_PER_COPY = 64 / CH; // rows that one wave's copy moves
  __device__ static __forceinline__ int key(int r) { return (D == 128 ? r : r >> 1) & (CH - 1); }
  __device__ static __forceinline__ int at(int r, int ch) { return r * ROW + ((ch ^ key(r)) << 4); }

  // operand of rows r0 .. r0 + 31 at k-step s: lane (l % 32, h) holds channels 16 s + 8 h .. + 7 of its row
  __device__ static __forceinline__ u4 rows(const uint8_t* t, int r0, int s, int lane) {
    return *reinterpret_cast<const u4*>(t + at(r0 + (lane & 31), 2 * s + (lane >> 5)));
  }
  // operand of channels 32 db .. + 31 (lane % 32) with 16 rows from r0 as its k, in the order in which a lane's
  // results of a 32x32 product hold them: element e of half h is row r0 + 8 (e / 4) + 4 h + e % 4. The reads
  // transpose: of 16 lanes, lane i brings 4 values at piece-half i % 4 of row i / 4, and receives value i of the 4 rows.
  __device__ static __forceinline__ u4 cols(const uint8_t* t, int r0, int db, int lane) {
    const int r = r0 + 4 * (lane >> 5) + ((lane & 15) >> 2);
    const int ch = 4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
    const u2 lo = read_tr(t + at(r, ch) + 8 * (lane & 1)), hi = read_tr(t + at(r + 8, ch) + 8 * (lane & 1));
    return u4{lo[0], lo[1], hi[0], hi[1]};
  }
  __device__ static __forceinline__ u2 read_tr(const uint8_t* p) {
    typedef short s4 __attribute__((ext_vector_type(4)));
    const s4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(p));
    return __builtin_bit_cast(u2, v);
  }
};

// One wave's copy of 16 bytes a lane from memory straight into LDS at lds + 16 lane. Issued as asm so that the compiler
// adds no waits of its own: copies are waited for (wait_copies) before the barrier that precedes their first use.
__device__ __forceinline__ void copy16(const void* src, const void* lds) {
  const uint32_t to = __builtin_amdgcn_readfirstlane(
      static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)lds)));
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(to) : "memory", "m0");
}

// The copies of a tile of ROWS rows at a constant stride (in elements, below FAR_STRIDE) by the NW waves of a workgroup,
// through a buffer descriptor: a lane's offset from the tile's first row is the same for all tiles, and rows behind
// the `valid` first are out of the buffer's range, which reads as zero without an access.
constexpr int64_t FAR_STRIDE = 1 << 24;   // 64 rows of less than this stay below 2^32 bytes
template <int D, int ROWS, int NW>
struct Copier {
  using T = Tile<D>;
  static constexpr int COPIES = ROWS / T::ROWS_PER_COPY / NW;
  uint32_t off, step, row_bytes;
  __device__ __forceinline__ Copier(int64_t stride, int wave, int lane) {
    const int r = wave * T::ROWS_PER_COPY + lane / T::CH;   // the places of its other rows have the same key
    row_bytes = 2 * (uint32_t)stride;
    off = r * row_bytes + 16 * ((lane % T::CH) ^ T::key(r));
    step = NW * T::ROWS_PER_COPY * row_bytes;
  }
  // tile: address of the tile's first row, the same for all lanes
  __device__ __forceinline__ void copy(const uint16_t* tile, int valid, const uint8_t* lds, int wave) const {
    typedef int v4i __attribute__((ext_vector_type(4)));
    const uint64_t p = reinterpret_cast<uint64_t>(tile);
    const uint32_t bytes = valid > 0 ? (min(valid, ROWS) - 1) * row_bytes + T::ROW : 0u;
    const v4i rsrc = {(int)(uint32_t)p, (int)(uint32_t)(p >> 32), (int)bytes, 0x00020000};
    const uint32_t to = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void*)lds)) +
                        wave * 1024;
#pragma unroll
    for (int u = 0; u < COPIES; ++u)
      asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off + u * step), "s"(rsrc),
                   "s"(__builtin_amdgcn_readfirstlane(to + u * NW * 1024))
                   : "memory", "m0");
  }
};

// all of this wave's memory operations are done
__device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

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
