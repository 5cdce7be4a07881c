// The gated delta rule over chunks of 64 tokens, forward and gradient.
//
// Within a chunk with entering state S0, G_i = g_1 + .. + g_i and
//   A_ij = beta_i e^{G_i - G_j} k_i.k_j  (j < i),     T = (I + A)^-1
//   P_ij = scale e^{G_i - G_j} q_i.k_j   (j <= i)
// the recurrence of the chunk's tokens is
//   R = V - diag(e^G) K S0,   U = T diag(beta) R
//   Y = scale diag(e^G) Q S0 + P U,   S' = e^{G_end} S0 + (diag(e^{G_end - G}) K)^T U
// and its gradient, from dY and dS',
//   dU = P^T dY + diag(e^{G_end - G}) K dS',   Z = T^T dU,   dV = dR = beta Z
//   dS0 = scale (diag(e^G) Q)^T dY + e^{G_end} dS' - (diag(e^G) K)^T dR
//   F = scale tril(e^{G_i - G_j} dY_i.U_j),  H = -stril(e^{G_i - G_j} dR_i.U_j)
//   dQ = scale diag(e^G) dY S0^T + F K
//   dK = F^T Q + diag(e^{G_end - G}) U dS'^T - diag(e^G) dR S0^T + (H + H^T) K
//   dbeta_i = Z_i.U_i / beta_i
//   dg_t = sum_{i >= t} (dq_i.q_i - dv_i.v_i) + <dS', S'>   (i within the chunk)
// beta counts as at least 2^-40 in magnitude, so that U_i / beta_i exists.
//
// Kernels: prep (T, P of every chunk at once), state_fwd (S, U, Y from chunk to
// chunk, 32 columns of the state per work-group), state_bwd (dS, dR backwards,
// the same split), grads (dQ, dK, dbeta, dg of every chunk at once).
#include "ll_delta.h"
#include "ll_kernels.h"

namespace ll {

namespace {

constexpr int CT = kDeltaChunk;
constexpr int NT = 32;               // columns of the state per work-group
constexpr int SC = CT + 4, SN = NT + 4;   // LDS row pitches

__device__ __forceinline__ f32x4 zero_acc() { return f32x4{0.f, 0.f, 0.f, 0.f}; }

// acc[n] += A[16 rows of the wave][K] B[K][16 n ..]: element (i, k) of A at
// A[i * ar + k * ak], (k, c) of B at B[k * bk + c * bc].
template <int N>
__device__ __forceinline__ void mm(const float* A, int ar, int ak, const float* B, int bk, int bc, int K,
                                   f32x4* acc) {
  const int l = threadIdx.x & 63, lo = l & 15, hi = l >> 4;
  for (int k = hi; k < K; k += 4) {
    const float a = A[lo * ar + k * ak];
#pragma unroll
    for (int n = 0; n < N; ++n)
      acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, B[k * bk + (16 * n + lo) * bc], acc[n], 0, 0, 0);
  }
}

// rows [64][D] of a token array into LDS (pitch p, D padded to Dp by zeros),
// zeros past the row's end
template <typename T>
__device__ void load_rows(float* dst, int p, const void* src, long ld, long head_off, int c0, int D, int Dp,
                          int t0, int len, int b, int B) {
  for (int i = threadIdx.x; i < CT * Dp; i += 256) {
    const int r = i / Dp, c = i % Dp;
    const int t = t0 + r;
    float v = 0.f;
    if (t < len && c < D)
      v = Op<T>::to_f32(static_cast<const T*>(src)[((long)t * B + b) * ld + head_off + c0 + c]);
    dst[r * p + c] = v;
  }
}

__device__ void load_square(float* dst, const float* src) {
  for (int i = threadIdx.x; i < CT * CT; i += 256) dst[(i / CT) * SC + i % CT] = src[i];
}

__device__ __forceinline__ int pad16(int d) { return (d + 15) & ~15; }

}  // namespace

template <typename T>
__global__ __launch_bounds__(256) void delta_prep_kernel(DeltaArgs a) {
  extern __shared__ float lds[];
  const int n = blockIdx.x % a.nch, bh = blockIdx.x / a.nch;
  const int b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
  const int len = delta_len(a, b), t0 = n * CT;
  if (n == 0 && h == 0 && threadIdx.x == 0 && a.seq_len && (a.seq_len[b] < 0 || a.seq_len[b] > a.T))
    atomicOr(a.err, LL_DEVERR_SEQ_LEN_BIT);
  if (t0 >= len) return;
  const int Dp = pad16(a.Dk), p = Dp + 4;
  float* ks = lds;
  float* qs = ks + CT * p;
  float* am = qs + CT * p;
  float* tm = am + CT * SC;
  double* G = reinterpret_cast<double*>(tm + CT * SC);
  float* be = reinterpret_cast<float*>(G + CT);
  load_rows<T>(ks, p, a.k, a.k_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
  load_rows<T>(qs, p, a.q, a.q_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
  const long item = blockIdx.x;
  if (threadIdx.x < CT) {
    const int i = threadIdx.x, t = t0 + i;
    float g = 0.f, bt = 0.f;
    if (t < len) {
      const long at = ((long)t * a.B + b) * a.Hv + h;
      g = a.g[at];
      bt = a.beta[at];
      if (g < -200.f) g = -200.f;          // e^g is 0 all the same
    }
    if (fabsf(bt) < 0x1p-40f) bt = copysignf(0x1p-40f, bt);
    be[i] = bt;
    double s = g;
    for (int d = 1; d < 64; d <<= 1) {
      const double o = __shfl_up(s, d, 64);
      if (i >= d) s += o;
    }
    G[i] = s;
    const double end = __shfl(s, 63, 64);
    a.G[item * CT + i] = s;
    a.tok[item * CT + i] = make_float4(expf((float)s), expf((float)(end - s)), bt, 0.f);
  }
  __syncthreads();
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, lo = l & 15, hi = l >> 4;
  f32x4 kk[4], qk[4];
  for (int i = 0; i < 4; ++i) kk[i] = qk[i] = zero_acc();
  mm<4>(ks + 16 * w * p, p, 1, ks, 1, p, Dp, kk);
  mm<4>(qs + 16 * w * p, p, 1, ks, 1, p, Dp, qk);
  for (int m = 0; m < 4; ++m)
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * w + 4 * hi + r, j = 16 * m + lo;
      const float d = j <= i ? expf((float)(G[i] - G[j])) : 0.f;
      am[i * SC + j] = j < i ? be[i] * d * kk[m][r] : 0.f;
      a.pm[item * CT * CT + i * CT + j] = j <= i ? a.scale * d * qk[m][r] : 0.f;
    }
  __syncthreads();
  if (threadIdx.x < CT) {
    const int c = threadIdx.x;
    for (int i = 0; i < CT; ++i) {
      float x = i == c ? 1.f : 0.f;
      for (int j = c; j < i; ++j) x -= am[i * SC + j] * tm[j * SC + c];
      tm[i * SC + c] = x;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < CT * CT; i += 256) a.tm[item * CT * CT + i] = tm[(i / CT) * SC + i % CT];
}

template <typename T, bool SAVE>
__global__ __launch_bounds__(256) void delta_state_fwd_kernel(DeltaArgs a) {
  extern __shared__ float lds[];
  const int ntile = (a.Dv + NT - 1) / NT;
  const int ct = blockIdx.x % ntile, bh = blockIdx.x / ntile;
  const int b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
  const int len = delta_len(a, b), live = (len + CT - 1) / CT;
  const int Dp = pad16(a.Dk), p = Dp + 4, c0 = ct * NT;
  float* ks = lds;
  float* qs = ks + CT * p;
  float* S = qs + CT * p;              // [Dp][NT]
  float* tm = S + Dp * SN;
  float* pm = tm + CT * SC;
  float* R = pm + CT * SC;             // [64][NT]
  float* U = R + CT * SN;
  float4* tok = reinterpret_cast<float4*>(U + CT * SN);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lo = l & 15, hi = l >> 4;
  const long head = (long)bh * a.Dk * a.Dv;
  for (int i = tid; i < Dp * NT; i += 256) {
    const int d = i / NT, c = i % NT;
    S[d * SN + c] = a.S0 && d < a.Dk && c0 + c < a.Dv ? a.S0[head + (long)d * a.Dv + c0 + c] : 0.f;
  }
  for (int n = 0; n < live; ++n) {
    const long item = (long)bh * a.nch + n;
    const int t0 = n * CT;
    __syncthreads();
    load_rows<T>(ks, p, a.k, a.k_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
    load_rows<T>(qs, p, a.q, a.q_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
    load_rows<T>(R, SN, a.v, a.v_ld, (long)h * a.Dv, c0, min(NT, a.Dv - c0), NT, t0, len, b, a.B);
    load_square(tm, a.tm + item * CT * CT);
    load_square(pm, a.pm + item * CT * CT);
    if (tid < CT) tok[tid] = a.tok[item * CT + tid];
    if (SAVE)
      for (int i = tid; i < a.Dk * NT; i += 256) {
        const int d = i / NT, c = i % NT;
        if (c0 + c < a.Dv) a.st[item * a.Dk * a.Dv + (long)d * a.Dv + c0 + c] = S[d * SN + c];
      }
    __syncthreads();
    f32x4 acc[2] = {zero_acc(), zero_acc()};
    mm<2>(ks + 16 * w * p, p, 1, S, SN, 1, Dp, acc);
#pragma unroll
    for (int m = 0; m < 2; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r, c = 16 * m + lo;
        R[i * SN + c] = tok[i].z * (R[i * SN + c] - tok[i].x * acc[m][r]);
      }
    __syncthreads();
    f32x4 u[2] = {zero_acc(), zero_acc()};
    mm<2>(tm + 16 * w * SC, SC, 1, R, SN, 1, CT, u);
#pragma unroll
    for (int m = 0; m < 2; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r, c = 16 * m + lo;
        U[i * SN + c] = u[m][r];
        if (SAVE && c0 + c < a.Dv) a.u[(item * CT + i) * a.Dv + c0 + c] = u[m][r];
      }
    __syncthreads();
    f32x4 y0[2] = {zero_acc(), zero_acc()}, y1[2] = {zero_acc(), zero_acc()};
    mm<2>(qs + 16 * w * p, p, 1, S, SN, 1, Dp, y0);
    mm<2>(pm + 16 * w * SC, SC, 1, U, SN, 1, CT, y1);
#pragma unroll
    for (int m = 0; m < 2; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r, c = 16 * m + lo, t = t0 + i;
        if (t < a.T && c0 + c < a.Dv)
          static_cast<T*>(a.y)[(((long)t * a.B + b) * a.Hv + h) * a.Dv + c0 + c] =
              Op<T>::from_f32(t < len ? a.scale * tok[i].x * y0[m][r] + y1[m][r] : 0.f);
      }
    __syncthreads();
    for (int i = tid; i < CT * NT; i += 256) U[(i / NT) * SN + i % NT] *= tok[i / NT].y;
    __syncthreads();
    const float end = tok[CT - 1].x;
    for (int mt = w; mt < Dp / 16; mt += 4) {
      f32x4 s[2] = {zero_acc(), zero_acc()};
      mm<2>(ks + 16 * mt, 1, p, U, SN, 1, CT, s);
  #pragma unroll
    for (int m = 0; m < 2; ++m)
        for (int r = 0; r < 4; ++r) {
          float& x = S[(16 * mt + 4 * hi + r) * SN + 16 * m + lo];
          x = end * x + s[m][r];
        }
    }
  }
  __syncthreads();
  if (a.ST)
    for (int i = tid; i < a.Dk * NT; i += 256) {
      const int d = i / NT, c = i % NT;
      if (c0 + c < a.Dv) a.ST[head + (long)d * a.Dv + c0 + c] = S[d * SN + c];
    }
  for (int t = live * CT + tid / NT; t < a.T; t += 256 / NT)
    if (c0 + tid % NT < a.Dv)
      static_cast<T*>(a.y)[(((long)t * a.B + b) * a.Hv + h) * a.Dv + c0 + tid % NT] = Op<T>::from_f32(0.f);
}

template <typename T>
__global__ __launch_bounds__(256) void delta_state_bwd_kernel(DeltaArgs a) {
  extern __shared__ float lds[];
  const int ntile = (a.Dv + NT - 1) / NT;
  const int ct = blockIdx.x % ntile, bh = blockIdx.x / ntile;
  const int b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
  const int len = delta_len(a, b), live = (len + CT - 1) / CT;
  const int Dp = pad16(a.Dk), p = Dp + 4, c0 = ct * NT;
  float* ks = lds;
  float* qs = ks + CT * p;
  float* S = qs + CT * p;              // dS [Dp][NT]
  float* tm = S + Dp * SN;
  float* pm = tm + CT * SC;
  float* dY = pm + CT * SC;            // [64][NT]
  float* U = dY + CT * SN;             // dU, then dR
  float4* tok = reinterpret_cast<float4*>(U + CT * SN);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lo = l & 15, hi = l >> 4;
  const long head = (long)bh * a.Dk * a.Dv;
  for (int i = tid; i < Dp * NT; i += 256) {
    const int d = i / NT, c = i % NT;
    S[d * SN + c] = a.dST && d < a.Dk && c0 + c < a.Dv ? a.dST[head + (long)d * a.Dv + c0 + c] : 0.f;
  }
  for (int n = live - 1; n >= 0; --n) {
    const long item = (long)bh * a.nch + n;
    const int t0 = n * CT;
    __syncthreads();
    load_rows<T>(ks, p, a.k, a.k_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
    load_rows<T>(qs, p, a.q, a.q_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
    load_rows<T>(dY, SN, a.dy, (long)a.Hv * a.Dv, (long)h * a.Dv, c0, min(NT, a.Dv - c0), NT, t0, len, b, a.B);
    load_square(tm, a.tm + item * CT * CT);
    load_square(pm, a.pm + item * CT * CT);
    if (tid < CT) tok[tid] = a.tok[item * CT + tid];
    for (int i = tid; i < a.Dk * NT; i += 256) {
      const int d = i / NT, c = i % NT;
      if (c0 + c < a.Dv) a.dst[item * a.Dk * a.Dv + (long)d * a.Dv + c0 + c] = S[d * SN + c];
    }
    __syncthreads();
    f32x4 u0[2] = {zero_acc(), zero_acc()}, u1[2] = {zero_acc(), zero_acc()};
    mm<2>(pm + 16 * w, 1, SC, dY, SN, 1, CT, u0);
    mm<2>(ks + 16 * w * p, p, 1, S, SN, 1, Dp, u1);
#pragma unroll
    for (int m = 0; m < 2; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r;
        U[i * SN + 16 * m + lo] = u0[m][r] + tok[i].y * u1[m][r];
      }
    __syncthreads();
    f32x4 z[2] = {zero_acc(), zero_acc()};
    mm<2>(tm + 16 * w, 1, SC, U, SN, 1, CT, z);
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 2; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r, c = 16 * m + lo, t = t0 + i;
        const float dr = tok[i].z * z[m][r];
        U[i * SN + c] = tok[i].x * dr;
        if (c0 + c < a.Dv) {
          a.dr[(item * CT + i) * a.Dv + c0 + c] = dr;
          if (t < a.T)
            static_cast<T*>(a.dv)[((long)t * a.B + b) * a.dv_ld + (long)h * a.Dv + c0 + c] =
                Op<T>::from_f32(t < len ? dr : 0.f);
        }
        dY[i * SN + c] *= a.scale * tok[i].x;
      }
    __syncthreads();
    const float end = tok[CT - 1].x;
    for (int mt = w; mt < Dp / 16; mt += 4) {
      f32x4 s0[2] = {zero_acc(), zero_acc()}, s1[2] = {zero_acc(), zero_acc()};
      mm<2>(qs + 16 * mt, 1, p, dY, SN, 1, CT, s0);
      mm<2>(ks + 16 * mt, 1, p, U, SN, 1, CT, s1);
  #pragma unroll
    for (int m = 0; m < 2; ++m)
        for (int r = 0; r < 4; ++r) {
          float& x = S[(16 * mt + 4 * hi + r) * SN + 16 * m + lo];
          x = end * x + s0[m][r] - s1[m][r];
        }
    }
  }
  __syncthreads();
  if (a.dS0)
    for (int i = tid; i < a.Dk * NT; i += 256) {
      const int d = i / NT, c = i % NT;
      if (c0 + c < a.Dv) a.dS0[head + (long)d * a.Dv + c0 + c] = S[d * SN + c];
    }
  for (int t = live * CT + tid / NT; t < a.T; t += 256 / NT)
    if (c0 + tid % NT < a.Dv)
      static_cast<T*>(a.dv)[((long)t * a.B + b) * a.dv_ld + (long)h * a.Dv + c0 + tid % NT] = Op<T>::from_f32(0.f);
}

template <typename T>
__global__ __launch_bounds__(256) void delta_grads_kernel(DeltaArgs a) {
  extern __shared__ float lds[];
  const int n = blockIdx.x % a.nch, bk = blockIdx.x / a.nch;
  const int b = bk / a.Hk, hk = bk % a.Hk, grp = a.Hv / a.Hk;
  const int len = delta_len(a, b), t0 = n * CT;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lo = l & 15, hi = l >> 4;
  T* dq = static_cast<T*>(a.dq);
  T* dk = static_cast<T*>(a.dk);
  if (t0 >= len) {
    for (int r = tid >> 6; r < CT && t0 + r < a.T; r += 4) {
      const long tok = (long)(t0 + r) * a.B + b;
      for (int c = l; c < a.Dk; c += 64) {
        dq[tok * a.dq_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(0.f);
        dk[tok * a.dk_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(0.f);
      }
      for (int c = l; c < grp; c += 64) {
        a.dg[tok * a.Hv + hk * grp + c] = 0.f;
        a.dbeta[tok * a.Hv + hk * grp + c] = 0.f;
      }
    }
    return;
  }
  const int Dp = pad16(a.Dk), p = Dp + 4;
  float* ks = lds;
  float* qs = ks + CT * p;
  float* S = qs + CT * p;              // [Dp][NT]; F after the column loop
  float* dS = S + kDeltaMaxDk * SN;    // [Dp][NT]; H after it
  float* dY = dS + kDeltaMaxDk * SN;
  float* U = dY + CT * SN;
  float* dR = U + CT * SN;
  float4* tok = reinterpret_cast<float4*>(dR + CT * SN);
  double* G = reinterpret_cast<double*>(tok + CT);
  float* dG = reinterpret_cast<float*>(G + CT);
  float* part = dG + CT;               // [4]
  load_rows<T>(ks, p, a.k, a.k_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
  load_rows<T>(qs, p, a.q, a.q_ld, (long)hk * a.Dk, 0, a.Dk, Dp, t0, len, b, a.B);
  f32x4 tq[8], tk[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) tq[i] = tk[i] = zero_acc();
  for (int hh = 0; hh < grp; ++hh) {
    const int h = hk * grp + hh;
    const long bh = (long)b * a.Hv + h, item = bh * a.nch + n;
    f32x4 aq[8], ku[8], kr[8], F[4], H[4];
  #pragma unroll
  for (int i = 0; i < 8; ++i) aq[i] = ku[i] = kr[i] = zero_acc();
    for (int i = 0; i < 4; ++i) F[i] = H[i] = zero_acc();
    float ss = 0.f, ub = 0.f, vr = 0.f;
    const int row = tid >> 2, q4 = (tid & 3) * 8;
    for (int c0 = 0; c0 < a.Dv; c0 += NT) {
      __syncthreads();
      const int nc = min(NT, a.Dv - c0);
      load_rows<T>(dY, SN, a.dy, (long)a.Hv * a.Dv, (long)h * a.Dv, c0, nc, NT, t0, len, b, a.B);
      for (int i = tid; i < CT * NT; i += 256) {
        const int r = i / NT, c = i % NT;
        const long at = (item * CT + r) * a.Dv + c0 + c;
        U[r * SN + c] = c < nc ? a.u[at] : 0.f;
        dR[r * SN + c] = c < nc ? a.dr[at] : 0.f;
      }
      for (int i = tid; i < Dp * NT; i += 256) {
        const int d = i / NT, c = i % NT;
        const long at = item * a.Dk * a.Dv + (long)d * a.Dv + c0 + c;
        const bool in = d < a.Dk && c < nc;
        const float s = in ? a.st[at] : 0.f, ds = in ? a.dst[at] : 0.f;
        S[d * SN + c] = s;
        dS[d * SN + c] = ds;
        ss += s * ds;
      }
      if (c0 == 0 && tid < CT) {
        tok[tid] = a.tok[item * CT + tid];
        G[tid] = a.G[item * CT + tid];
      }
      __syncthreads();
      for (int e = 0; e < 8; ++e) {
        const int c = q4 + e;
        const float r = dR[row * SN + c];
        ub += r * U[row * SN + c];
        if (t0 + row < len && c < nc)
          vr += r * Op<T>::to_f32(static_cast<const T*>(a.v)[((long)(t0 + row) * a.B + b) * a.v_ld +
                                                             (long)h * a.Dv + c0 + c]);
      }
      mm<4>(dY + 16 * w * SN, SN, 1, U, 1, SN, NT, F);
      mm<4>(dR + 16 * w * SN, SN, 1, U, 1, SN, NT, H);
    #pragma unroll
  for (int i = 0; i < 8; ++i)
        if (16 * i < Dp) {
          mm<1>(dY + 16 * w * SN, SN, 1, S + 16 * i * SN, 1, SN, NT, aq + i);
          mm<1>(U + 16 * w * SN, SN, 1, dS + 16 * i * SN, 1, SN, NT, ku + i);
          mm<1>(dR + 16 * w * SN, SN, 1, S + 16 * i * SN, 1, SN, NT, kr + i);
        }
    }
    __syncthreads();
    float* Fm = S;
    float* Hm = dS;
    for (int m = 0; m < 4; ++m)
      for (int r = 0; r < 4; ++r) {
        const int i = 16 * w + 4 * hi + r, j = 16 * m + lo;
        const float d = j <= i ? expf((float)(G[i] - G[j])) : 0.f;
        Fm[i * SC + j] = a.scale * d * F[m][r];
        Hm[i * SC + j] = j < i ? -d * H[m][r] : 0.f;
      }
    // <dS', S'> without the part of U
    const float end = tok[CT - 1].x;
    ss *= end;
    float dots[4] = {0.f, 0.f, 0.f, 0.f};
  #pragma unroll
  for (int i = 0; i < 8; ++i)
      if (16 * i < Dp)
        for (int r = 0; r < 4; ++r) {
          const int j = 16 * w + 4 * hi + r;
          ku[i][r] *= tok[j].y;
          ss += ku[i][r] * ks[j * p + 16 * i + lo];
          aq[i][r] *= a.scale * tok[j].x;
          kr[i][r] *= tok[j].x;
        }
    for (int d = 1; d < 64; d <<= 1) ss += __shfl_xor(ss, d, 64);
    if (l == 0) part[w] = ss;
    __syncthreads();
  #pragma unroll
  for (int i = 0; i < 8; ++i)
      if (16 * i < Dp) {
        mm<1>(Fm + 16 * w * SC, SC, 1, ks + 16 * i, p, 1, CT, aq + i);
        f32x4 x = zero_acc();
        mm<1>(Fm + 16 * w, 1, SC, qs + 16 * i, p, 1, CT, &x);
        mm<1>(Hm + 16 * w * SC, SC, 1, ks + 16 * i, p, 1, CT, &x);
        mm<1>(Hm + 16 * w, 1, SC, ks + 16 * i, p, 1, CT, &x);
        for (int r = 0; r < 4; ++r) {
          const int j = 16 * w + 4 * hi + r;
          dots[r] += aq[i][r] * qs[j * p + 16 * i + lo];
          tq[i][r] += aq[i][r];
          tk[i][r] += x[r] + ku[i][r] - kr[i][r];
        }
      }
    for (int d = 1; d < 4; d <<= 1) {
      ub += __shfl_xor(ub, d, 64);
      vr += __shfl_xor(vr, d, 64);
    }
    for (int r = 0; r < 4; ++r) {
      for (int d = 1; d < 16; d <<= 1) dots[r] += __shfl_xor(dots[r], d, 64);
      if (lo == 0) dG[16 * w + 4 * hi + r] = dots[r];
    }
    __syncthreads();
    if ((tid & 3) == 0) {
      dG[row] -= vr;
      const float bt = tok[row].z;
      if (t0 + row < a.T)
        a.dbeta[((long)(t0 + row) * a.B + b) * a.Hv + h] = t0 + row < len ? ub / (bt * bt) : 0.f;
    }
    __syncthreads();
    if (tid < CT) {
      float s = dG[CT - 1 - tid];        // sums from the chunk's end
      for (int d = 1; d < 64; d <<= 1) {
        const float o = __shfl_up(s, d, 64);
        if (tid >= d) s += o;
      }
      const int t = t0 + CT - 1 - tid;
      if (t < a.T)
        a.dg[((long)t * a.B + b) * a.Hv + h] = t < len ? s + ((part[0] + part[1]) + (part[2] + part[3])) : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    for (int r = 0; r < 4; ++r) {
      const int t = t0 + 16 * w + 4 * hi + r, c = 16 * i + lo;
      if (t < a.T && c < a.Dk) {
        const long at = (long)t * a.B + b;
        dq[at * a.dq_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(t < len ? tq[i][r] : 0.f);
        dk[at * a.dk_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(t < len ? tk[i][r] : 0.f);
      }
    }
}

namespace {

template <typename K>
hipError_t launch(K kernel, long grid, size_t lds, const DeltaArgs& a, hipStream_t s) {
  hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                     hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)grid), dim3(256), lds, s>>>(a);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t delta_launch_fwd(const DeltaArgs& a, bool save, hipStream_t s) {
  const int Dp = (a.Dk + 15) & ~15, p = Dp + 4;
  const long bh = (long)a.B * a.Hv, ntile = (a.Dv + NT - 1) / NT;
  hipError_t e = launch(delta_prep_kernel<T>, bh * a.nch,
                        sizeof(float) * (2 * CT * p + 2 * CT * SC + 3 * CT), a, s);
  if (e != hipSuccess) return e;
  const size_t lds = sizeof(float) * (2 * CT * p + Dp * SN + 2 * CT * SC + 2 * CT * SN + 4 * CT);
  return save ? launch(delta_state_fwd_kernel<T, true>, bh * ntile, lds, a, s)
              : launch(delta_state_fwd_kernel<T, false>, bh * ntile, lds, a, s);
}

template <typename T>
hipError_t delta_launch_bwd(const DeltaArgs& a, hipStream_t s) {
  const int Dp = (a.Dk + 15) & ~15, p = Dp + 4;
  const long bh = (long)a.B * a.Hv, ntile = (a.Dv + NT - 1) / NT;
  hipError_t e = launch(delta_state_bwd_kernel<T>, bh * ntile,
                        sizeof(float) * (2 * CT * p + Dp * SN + 2 * CT * SC + 2 * CT * SN + 4 * CT), a, s);
  if (e != hipSuccess) return e;
  return launch(delta_grads_kernel<T>, (long)a.B * a.Hk * a.nch,
                sizeof(float) * (2 * CT * p + 2 * kDeltaMaxDk * SN + 3 * CT * SN + 4 * CT + 3 * CT + 4), a, s);
}

template hipError_t delta_launch_fwd<float>(const DeltaArgs&, bool, hipStream_t);
template hipError_t delta_launch_fwd<bf16_t>(const DeltaArgs&, bool, hipStream_t);
template hipError_t delta_launch_bwd<float>(const DeltaArgs&, hipStream_t);
template hipError_t delta_launch_bwd<bf16_t>(const DeltaArgs&, hipStream_t);

}  // namespace ll
