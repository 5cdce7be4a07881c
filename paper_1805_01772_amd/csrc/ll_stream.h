// Loads and stores of what nothing reads again soon (device side).
#pragma once

#include "ll_device.h"

namespace ll {

// 16 bytes past the caches: for arrays larger than the last-level cache, which they
// would only sweep.
constexpr long kLastLevelBytes = 256L << 20;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
__device__ __forceinline__ void st16_stream(void* p, uint4 v) {
  __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p));
}
__device__ __forceinline__ uint4 ld16_stream(const void* p) {
  const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
  return make_uint4(v[0], v[1], v[2], v[3]);
}

}  // namespace ll
