// Argument blocks of the gated delta rule's kernels (internal).
#pragma once

#include "ll_device.h"

namespace ll {

constexpr int kDeltaChunk = 64;      // tokens per chunk
constexpr int kDeltaDots = 10 * 2 * 256;   // products of a chunk's q and k on and below the diagonal, tiles of 16
constexpr int kDeltaMaxDk = 128;
constexpr int kDeltaMaxDv = 512;

// Head size of the keys in 32-element steps of a matrix instruction, rounded
// up to a power of two (1, 2, 4).
inline int delta_ksteps(int Dk) { return Dk <= 32 ? 1 : Dk <= 64 ? 2 : 4; }
// Pieces of bfloat16 that hold an operand of the call's type.
inline int delta_pieces(bool bf16) { return bf16 ? 1 : 3; }

// Chunk n of (row b, value head h) is item (b * Hv + h) * nch + n; of key head
// hk item (b * Hk + hk) * nch + n.
//
// Matrices that a matrix instruction reads are stored by fragments, 16 rows x 32
// columns of one piece in the order in which a wave's lanes hold them: a lane's
// eight elements lie together, 1 KB is one load of a wave (read by rows instead,
// four neighbouring lanes touch four cache lines and a load takes four times as
// long).  Order: row tile, step of 32 columns, piece.
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
  // made by prep, per item: T = (I + A)^-1 and P with their transposes, 64 x
  // 64 in three pieces; decays of the tokens
  bf16_t *tp, *pp, *ttp, *ptp;
  double* G;                         // [64] sums of g from the chunk's start
  float4* tok;                       // [64] e^G, e^{G_end - G}, beta, -
  // per item of a key head, zeros past the row's end and Dk: K and Q, 64 x
  // (32 ksteps), and their transposes
  bf16_t *kp, *qp, *ktp, *qtp;
  // per item of a key head, kept for the gradient: q_i.k_j and k_i.k_j, tile by tile
  // (row tile w, column tile m <= w: number w (w + 1) / 2 + m) as the accumulators hold them
  float* dots;
  // per item, kept for the gradient
  float *st, *u;                     // entering state [Dk][Dv], U [64][Dv]
  float *dst, *dr;                   // gradient of the leaving state, of R
};

// Fragment (row tile, step, piece) of a matrix of `steps` steps and `pieces`
// pieces, in elements.
__device__ __forceinline__ constexpr int frag_at(int tile, int step, int piece, int steps, int pieces) {
  return ((tile * steps + step) * pieces + piece) * 512;
}

__device__ __forceinline__ int delta_len(const DeltaArgs& a, int b) {
  const int L = a.seq_len ? a.seq_len[b] : a.T;
  return L < 0 || L > a.T ? 0 : L;
}

template <typename T> hipError_t delta_launch_fwd(const DeltaArgs& a, bool save, int cus, hipStream_t s);
template <typename T> hipError_t delta_launch_bwd(const DeltaArgs& a, int cus, hipStream_t s);

}  // namespace ll
