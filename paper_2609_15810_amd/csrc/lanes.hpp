// Exchanges between the halves of a wave (not part of the public ABI).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vc {
namespace lanes {

// Empty asm that reads and rewrites x: what the compiler knows of x's value ends here
template <typename V>
__device__ __forceinline__ void pin(V& x) {
  asm volatile("" : "+v"(x));
}

// sum and maximum of v over lanes l and l ^ 32. The swap's two results are both halves' values; they are pinned, since a
// maximum over them has been compiled into one over a single one.
__device__ __forceinline__ float half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  uint32_t x = r[0], y = r[1];
  pin(x);
  pin(y);
  return __uint_as_float(x) + __uint_as_float(y);
}
__device__ __forceinline__ float half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  uint32_t x = r[0], y = r[1];
  pin(x);
  pin(y);
  return fmaxf(__uint_as_float(x), __uint_as_float(y));
}

}  // namespace lanes
}  // namespace vc
