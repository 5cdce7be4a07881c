// Argument blocks of the gated delta rule's kernels (internal).
#pragma once

#include "ll_device.h"

namespace ll {

constexpr int kDeltaChunk = 64;      // tokens per chunk
constexpr int kDeltaMaxDk = 128;
constexpr int kDeltaMaxDv = 512;

// Chunk n of (row b, value head h) is item (b * Hv + h) * nch + n.
struct DeltaArgs {
  int T, B, Hk, Hv, Dk, Dv, nch;
  float scale;
  long q_ld, k_ld, v_ld, dq_ld, dk_ld, dv_ld;
  const void *q, *k, *v, *dy;
  const float *g, *beta, *S0, *dST;
  const int* seq_len;
  void *y, *dq, *dk, *dv;
  float *ST, *dg, *dbeta, *dS0;
  int* err;
  // per item: T = (I + A)^-1 and P [64][64], decays of its tokens
  float *tm, *pm;
  double* G;                         // [64] sums of g from the chunk's start
  float4* tok;                       // [64] e^G, e^{G_end - G}, beta, -
  // per item, kept for the gradient
  float *st, *u;                     // entering state [Dk][Dv], U [64][Dv]
  float *dst, *dr;                   // gradient of the leaving state, of R
};

__device__ __forceinline__ int delta_len(const DeltaArgs& a, int b) {
  const int L = a.seq_len ? a.seq_len[b] : a.T;
  return L < 0 || L > a.T ? 0 : L;
}

template <typename T> hipError_t delta_launch_fwd(const DeltaArgs& a, bool save, hipStream_t s);
template <typename T> hipError_t delta_launch_bwd(const DeltaArgs& a, hipStream_t s);

}  // namespace ll
