// Float operands of the bfloat16 matrix instructions as sums of pieces, and the
// work-group's barriers over LDS (device side).
#pragma once

#include "ll_device.h"

namespace ll {

typedef bf16x8_t frag;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;

__device__ __forceinline__ f32x4 zero_acc() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
__device__ __forceinline__ f32x4 mfma(frag a, frag b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ frag as_frag(uint4 u) { return __builtin_bit_cast(frag, u); }

// acc += A B for operands in NA and NB pieces, smallest products first.
template <int NA, int NB, int LIM>
__device__ __forceinline__ void mma(const frag* a, const frag* b, f32x4& acc) {
#pragma unroll
  for (int s = LIM; s >= 0; --s)
#pragma unroll
    for (int i = 0; i < NA; ++i) {
      const int j = s - i;
      if (j >= 0 && j < NB) acc = mfma(a[i], b[j], acc);
    }
}

// Two floats to two bfloat16 (round to nearest even).
__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const f32x2 v = {x, y};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

// x, y = sum of N bfloat16 pairs.
template <int N>
__device__ __forceinline__ void split2(float x, float y, uint32_t* p) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    p[i] = pack2(x, y);
    if (i + 1 < N) {
      x -= __uint_as_float(p[i] << 16);
      y -= __uint_as_float(p[i] & 0xffff0000u);
    }
  }
}

// Four floats to N pieces of four bfloat16, stored at dst + i * stride (elements).
template <int N>
__device__ __forceinline__ void split4_store(f32x4 x, bf16_t* dst, int stride) {
  uint32_t a[N], b[N];
  split2<N>(x[0], x[1], a);
  split2<N>(x[2], x[3], b);
#pragma unroll
  for (int i = 0; i < N; ++i) *reinterpret_cast<uint2*>(dst + i * stride) = make_uint2(a[i], b[i]);
}

// Eight floats to N pieces.
template <int N>
__device__ __forceinline__ void split8(const float* x, uint4* p) {
  uint32_t w[4][N];
#pragma unroll
  for (int e = 0; e < 4; ++e) split2<N>(x[2 * e], x[2 * e + 1], w[e]);
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = make_uint4(w[0][i], w[1][i], w[2][i], w[3][i]);
}

__device__ __forceinline__ frag lds_frag(const bf16_t* p) { return as_frag(ld16(p)); }

// Barrier of the work-group that orders LDS only: loads and stores of global
// memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// LDS written by other lanes of the same wave is read next.
__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

}  // namespace ll
