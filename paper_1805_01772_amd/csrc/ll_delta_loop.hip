// The gated delta rule over chunks of 64 tokens, forward and gradient.
//
// Within a chunk with entering state S0, G_i = g_1 + .. + g_i and
//   A_ij = beta_i e^{G_i - G_j} k_i.k_j  (j < i),     T = (I + A)^-1
//   P_ij = scale e^{G_i - G_j} q_i.k_j   (j <= i)
// the recurrence of the chunk's tokens is
//   R = V - diag(e^G) K S0,   U = T diag(beta) R
//   Y = scale diag(e^G) Q S0 + P U,   S' = e^{G_end} S0 + K^T diag(e^{G_end - G}) U
// and its gradient, from dY and dS',
//   dU = P^T dY + diag(e^{G_end - G}) K dS',   Z = T^T dU,   dV = dR = beta Z
//   dS0 = Q^T (scale diag(e^G) dY) + e^{G_end} dS' - K^T (diag(e^G) dR)
//   F = scale tril(e^{G_i - G_j} dY_i.U_j),  H = -stril(e^{G_i - G_j} dR_i.U_j)
//   dQ = scale diag(e^G) dY S0^T + F K
//   dK = F^T Q + diag(e^{G_end - G}) U dS'^T - diag(e^G) dR S0^T + (H + H^T) K
//   dbeta_i = Z_i.U_i / beta_i
//   X_ij = F_ij q_i.k_j + H_ij k_i.k_j  (j < i),  what the pair's decay is worth
//   dg_t = sum_{i >= t > j} X_ij + sum_{i >= t} (q_i.(scale e^{G_i} S0 dY_i) - k_i.(e^{G_i} S0 dR_i))
//          + sum_{j < t} k_j.(e^{G_end - G_j} dS' U_j) + e^{G_end} <dS', S0>
// and nothing that does not straddle t is in the sum, to be taken out again: it would leave
// its rounding where e^{g_t} is small
// beta counts as at least 2^-40 in magnitude, so that U_i / beta_i exists.
//
// Kernels: prep (T, P and the transposes of every chunk at once), state_fwd (S,
// U, Y from chunk to chunk), state_bwd (dS, dR backwards), grads (dQ, dK, dbeta,
// dg of every chunk at once).  The columns of the state do not meet in the two
// loops, so each work-group has 16 or 32 of them (cols_of).
//
// Arithmetic.  The bfloat16 matrix instructions run at sixteen times the rate of
// the float32 ones, so a float operand is taken as the sum of three bfloat16
// pieces (24 bits, exactly), a bfloat16 one is its own piece, and a product of
// pieces i and j is taken while i + j <= 2: what is dropped is below 2^-24 of the
// term.  Sums are float32.  (Two pieces, 17 bits, of what only y and dK read would
// round one bfloat16 result in five hundred the other way and lose small differences of
// large terms; they save 2 to 6 %: 8 rows, forward and gradient, 784 us against 818 when measured.)
//
// Sizes that the figures below are for: "8 rows", lengths 256 to 2048, and "one
// row" of 16384 tokens, 16 value heads of 128 x 128 in bfloat16 (8 and 16 key
// heads), forward and gradient; "prompts", 4 rows of 100 to 1000 tokens, the same
// heads, inference.
#include "ll_delta.h"
#include "ll_exchange.h"
#include "ll_kernels.h"

namespace ll {

namespace {

constexpr int CT = kDeltaChunk;
constexpr int SC = CT + 4;           // row pitch of float [64][64] in LDS
constexpr int RC = CT + 8;           // of bfloat16 [..][64]: 16 rows hit all banks
constexpr int SQ = CT * CT;

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

// Raw eight elements of an operand, and their pieces.
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = zero4(); }
  __device__ __forceinline__ void load(const bf16_t* p) { u = ld16(p); }
  __device__ __forceinline__ void pieces(uint4* f) const { f[0] = u; }
};
template <> struct Raw8<float> {
  uint4 u, v;
  __device__ __forceinline__ void zero() { u = v = zero4(); }
  __device__ __forceinline__ void load(const float* p) {
    u = ld16(p);
    v = ld16(p + 4);
  }
  __device__ __forceinline__ void pieces(uint4* f) const {
    const float x[8] = {__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w),
                        __uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w)};
    split8<3>(x, f);
  }
};

template <typename T> struct Pieces { static constexpr int n = 3; };
template <> struct Pieces<bf16_t> { static constexpr int n = 1; };

__device__ __forceinline__ frag lds_frag(const bf16_t* p) { return as_frag(ld16(p)); }

// A fragment's read of 16 bytes a lane serves lanes 0-3, 12-15, 20-27 together
// (4-11, 16-19, 28-31; the same from 32), each from 64 banks: rows 4-11 of every 16
// hold their neighbouring groups of eight columns exchanged, so that with an odd
// number of groups to a row the 16 lanes meet different banks.
__device__ __forceinline__ int swap8(int row) { return ((row >> 2) ^ (row >> 3)) & 1 ? 8 : 0; }

// Sums over the 8 or 16 neighbouring lanes that hold a row, in every one of them,
// by moves inside the rows of 16 lanes.
template <int CTRL>
__device__ __forceinline__ float moved(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum8(float x) {
  x += moved<0xb1>(x);                                   // pairs
  x += moved<0x4e>(x);                                   // quads
  return x + moved<0x141>(x);                            // the half row mirrored
}
__device__ __forceinline__ float sum16(float x) {
  x = sum8(x);
  return x + moved<0x128>(x);                            // the row turned by 8
}

// The same in double, by two moves of 32 bits.
template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ double moved2(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t a = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
  const uint32_t b = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)b << 32 | a);
}
__device__ __forceinline__ double sum16(double x) {
  x += moved2<0xb1>(x);
  x += moved2<0x4e>(x);
  x += moved2<0x141>(x);
  return x + moved2<0x128>(x);
}
// Sum over the lanes lo, lo + 16, lo + 32, lo + 48, in every one of them.
__device__ __forceinline__ float sum_rows(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(__uint_as_float(a[0]) + __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sums over the lanes up to this one: of its row of 16, of all 64.
constexpr int kUpOne = 0x111;                            // the lane below's, 0 in a row's first
__device__ __forceinline__ float scan16(float x) {
  x += moved<kUpOne>(x);
  x += moved<0x112>(x);                                  // by 2, 4, 8
  x += moved<0x114>(x);
  return x + moved<0x118>(x);
}
__device__ __forceinline__ double scan16(double x) {
  x += moved2<kUpOne>(x);
  x += moved2<0x112>(x);
  x += moved2<0x114>(x);
  return x + moved2<0x118>(x);
}
__device__ __forceinline__ double scan64(double x) {
  x = scan16(x);
  x += moved2<0x142, 0xa>(x);                            // a row's last lane to the next row, odd rows
  return x + moved2<0x143, 0xc>(x);                      // lane 31 to the upper half
}

// Rows crow .. crow + 3 of column lo (a tile of the accumulators) to dst: float as
// they are, bfloat16 two columns a store, even lanes the even rows.
template <typename T>
__device__ __forceinline__ void store_tile(T* dst, long pitch, f32x4 x, int lo, int rows) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (r < rows) dst[r * pitch + lo] = x[r];
  } else {
    const bool odd = lo & 1;
#pragma unroll
    for (int r = 0; r < 4; r += 2) {
      const float got = moved<0xb1>(odd ? x[r] : x[r + 1]);
      const uint32_t two = odd ? pack2(got, x[r + 1]) : pack2(x[r], got);
      if (r + odd < rows) *reinterpret_cast<uint32_t*>(dst + (r + odd) * pitch + (lo & ~1)) = two;
    }
  }
}

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

}  // namespace

// ---------------------------------------------------------------------------
// prep: one work-group per item.  k k^T and q k^T on the matrix cores, the
// inverse of I + A by blocks of 16 (each diagonal block by substitution, the
// blocks below by float32 products: T_rc = -T_rr sum_k A_rk T_kc, a wave per
// block column), then everything the loops read in the order in which a lane
// reads it, 16 bytes at a time.
// Bound: HBM, for what it writes (K, Q, T and P, plain and transposed, in pieces):
// 8 rows 110 us, 0.6 GB; one row 146 us; prompts 27 us.  (float32 keeps k and q in LDS in
// pieces, 73 KB at 64 columns and 122 KB at 128: two work-groups and one a compute unit.)
// ---------------------------------------------------------------------------
template <typename T, int KS, bool SAVE>
__global__ __launch_bounds__(256) void delta_prep_kernel(DeltaArgs a) {
  constexpr int NP = Pieces<T>::n, DP = 32 * KS, KP = DP + 8;
  constexpr int kOps = 2 * NP * CT * KP * 2, kMats = 2 * CT * SC * 4;
  __shared__ __align__(16) unsigned char raw[kOps > kMats ? kOps : kMats];
  __shared__ __align__(16) float tm[CT * SC];
  __shared__ double G[CT];
  __shared__ float be[CT];
  const int n = blockIdx.x % a.nch, bh = blockIdx.x / a.nch;
  const int b = bh / a.Hv, h = bh % a.Hv, grp = a.Hv / a.Hk, hk = h / grp;
  const int len = delta_len(a, b), t0 = n * CT;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, lo = l & 15, hi = l >> 4;
  if (n == 0 && h == 0 && tid == 0 && a.seq_len && (a.seq_len[b] < 0 || a.seq_len[b] > a.T))
    atomicOr(a.err, LL_DEVERR_SEQ_LEN_BIT);
  if (t0 >= len) return;
  const long item = blockIdx.x, kitem = ((long)b * a.Hk + hk) * a.nch + n;
  const bool first = h == hk * grp;                      // what the key head's value heads share is written once
  bf16_t* kp = reinterpret_cast<bf16_t*>(raw);           // [NP][64][KP]
  bf16_t* qp = kp + NP * CT * KP;
  for (int i = tid; i < CT * DP / 8; i += 256) {
    const int r = i / (DP / 8), c = (i % (DP / 8)) * 8, t = t0 + r;
    Raw8<T> x, y;
    if (t < len && c < a.Dk) {
      const long tok = (long)t * a.B + b;
      x.load(static_cast<const T*>(a.k) + tok * a.k_ld + (long)hk * a.Dk + c);
      y.load(static_cast<const T*>(a.q) + tok * a.q_ld + (long)hk * a.Dk + c);
    } else {
      x.zero();
      y.zero();
    }
    uint4 p[NP], q[NP];
    x.pieces(p);
    y.pieces(q);
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      *reinterpret_cast<uint4*>(kp + (e * CT + r) * KP + c) = p[e];
      *reinterpret_cast<uint4*>(qp + (e * CT + r) * KP + c) = q[e];
    }
  }
  if (tid < CT) {
    const int t = t0 + tid;
    float g = 0.f, bt = 0.f;
    if (t < len) {
      const long at = ((long)t * a.B + b) * a.Hv + h;
      g = a.g[at];
      bt = a.beta[at];
      if (g < -200.f) g = -200.f;          // e^g is 0 all the same, and sums stay finite
    }
    if (fabsf(bt) < 0x1p-40f) bt = copysignf(0x1p-40f, bt);
    be[tid] = bt;
    double s = g;                          // differences of the sums keep float's bits
    for (int d = 1; d < 64; d <<= 1) {
      const double o = __shfl_up(s, d, 64);
      if (tid >= d) s += o;
    }
    G[tid] = s;
    const double end = __shfl(s, 63, 64);
    if (SAVE) a.G[item * CT + tid] = s;
    a.tok[item * CT + tid] = make_float4(expf((float)s), expf((float)(end - s)), bt, 0.f);
  }
  lds_barrier();
  f32x4 kk[4], qk[4];
#pragma unroll
  for (int m = 0; m < 4; ++m) kk[m] = qk[m] = zero_acc();
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    frag ka[NP], qa[NP];
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      ka[e] = lds_frag(kp + (e * CT + 16 * w + lo) * KP + 32 * s + 8 * hi);
      qa[e] = lds_frag(qp + (e * CT + 16 * w + lo) * KP + 32 * s + 8 * hi);
    }
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (m <= w) {
        frag kb[NP];
#pragma unroll
        for (int e = 0; e < NP; ++e) kb[e] = lds_frag(kp + (e * CT + 16 * m + lo) * KP + 32 * s + 8 * hi);
        mma<NP, NP, 2>(ka, kb, kk[m]);
        mma<NP, NP, 2>(qa, kb, qk[m]);
      }
  }
  if (SAVE && first) {
    f32x4* x = reinterpret_cast<f32x4*>(a.dots + kitem * kDeltaDots) + w * (w + 1) * 64 + l;
#pragma unroll
    for (int m = 0; m < 4; ++m)
      if (m <= w) {
        x[m * 128] = qk[m];
        x[m * 128 + 64] = kk[m];
      }
  }
  if (first) {
    // wave by wave one fragment: lane l has row 16 tile + lo, columns 32 step + 8 hi ..
    const long base = kitem * NP * CT * DP + 8 * l;
    for (int f = w; f < 4 * KS * NP; f += 4) {
      const int e = f % NP, s = f / NP % KS, t = f / (NP * KS);
      const int at = (e * CT + 16 * t + lo) * KP + 32 * s + 8 * hi;
      *reinterpret_cast<uint4*>(a.kp + base + f * 512) = ld16(kp + at);
      *reinterpret_cast<uint4*>(a.qp + base + f * 512) = ld16(qp + at);
    }
    for (int f = w; f < 4 * KS * NP; f += 4) {           // 2 KS row tiles of two steps
      const int e = f % NP, s = f / NP % 2, t = f / (NP * 2);
      uint32_t x[4], y[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const int at = (e * CT + 32 * s + 8 * hi + 2 * m) * KP + 16 * t + lo;
        x[m] = (uint32_t)kp[at] | (uint32_t)kp[at + KP] << 16;
        if (SAVE) y[m] = (uint32_t)qp[at] | (uint32_t)qp[at + KP] << 16;
      }
      *reinterpret_cast<uint4*>(a.ktp + base + f * 512) = make_uint4(x[0], x[1], x[2], x[3]);
      if (SAVE) *reinterpret_cast<uint4*>(a.qtp + base + f * 512) = make_uint4(y[0], y[1], y[2], y[3]);
    }
  }
  lds_barrier();
  float* am = reinterpret_cast<float*>(raw);
  float* pm = am + CT * SC;
#pragma unroll
  for (int m = 0; m < 4; ++m)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = 16 * w + 4 * hi + r, j = 16 * m + lo;
      const float d = j <= i ? expf((float)(G[i] - G[j])) : 0.f;
      am[i * SC + j] = j < i ? be[i] * d * kk[m][r] : 0.f;
      pm[i * SC + j] = j <= i ? a.scale * d * qk[m][r] : 0.f;
    }
  lds_barrier();
  {
    // diagonal block w: column lo by substitution, in registers
    const float* A = am + 16 * w * SC + 16 * w;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float s = i == lo ? 1.f : 0.f;
#pragma unroll
      for (int j = 0; j < i; ++j) s -= A[i * SC + j] * x[j];
      x[i] = s;
    }
    if (hi == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) tm[(16 * w + i) * SC + 16 * w + lo] = x[i];
    }
    // above the diagonal: zero
    for (int m = 0; m < w; ++m)
#pragma unroll
      for (int r = 0; r < 4; ++r) tm[(16 * m + 4 * hi + r) * SC + 16 * w + lo] = 0.f;
  }
  lds_barrier();
  for (int r = w + 1; r < 4; ++r) {
    f32x4 x = zero_acc(), z = zero_acc();
    for (int k = w; k < r; ++k)
#pragma unroll
      for (int s = 0; s < 4; ++s)
        x = __builtin_amdgcn_mfma_f32_16x16x4f32(am[(16 * r + lo) * SC + 16 * k + 4 * s + hi],
                                                 tm[(16 * k + 4 * s + hi) * SC + 16 * w + lo], x, 0, 0, 0);
    float* blk = tm + 16 * r * SC + 16 * w;
#pragma unroll
    for (int e = 0; e < 4; ++e) blk[(4 * hi + e) * SC + lo] = -x[e];
    wave_lds_fence();
#pragma unroll
    for (int s = 0; s < 4; ++s)
      z = __builtin_amdgcn_mfma_f32_16x16x4f32(tm[(16 * r + lo) * SC + 16 * r + 4 * s + hi],
                                               blk[(4 * s + hi) * SC + lo], z, 0, 0, 0);
    wave_lds_fence();
#pragma unroll
    for (int e = 0; e < 4; ++e) blk[(4 * hi + e) * SC + lo] = z[e];
    wave_lds_fence();
  }
  lds_barrier();
  // fragments (row tile, step) of T and P and, for the gradient, the transposes
  for (int f = w; f < 8; f += 4) {
    const int r = 16 * (f / 2) + lo, j = 32 * (f % 2) + 8 * hi;
    const long at = item * 3 * SQ + (long)f * 3 * 512 + 8 * l;
    float x[8];
    uint4 p[3];
    // (the fragments right of a lower and left of an upper triangle are never read)
    const bool low = f % 2 == 0 || f / 2 >= 2, up = f % 2 == 1 || f / 2 < 2;
    auto put = [&](bf16_t* dst, int n, bool some) {
      if (some)
        for (int e = 0; e < n; ++e) *reinterpret_cast<uint4*>(dst + at + e * 512) = p[e];
    };
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = tm[r * SC + j + e];
    split8<3>(x, p);
    put(a.tp, 3, low);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = pm[r * SC + j + e];
    split8<3>(x, p);
    put(a.pp, 3, low);
    if (SAVE) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = tm[(j + e) * SC + r];
      split8<3>(x, p);
      put(a.ttp, 3, up);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = pm[(j + e) * SC + r];
      split8<3>(x, p);
      put(a.ptp, 3, up);
    }
  }
}

namespace {

// The loops' loads and stores go through buffer descriptors made for each
// chunk: what lies past a row's end, past Dk or past Dv is out of the buffer's
// range (read as 0, not written), so there is no branch around any of them
// and the wait for one counts exactly what was issued after it.  A lane that
// has no place at all gets an offset past every range; a time step spans at most
// 2^26 bytes (validated), so the offsets of 32 of them stay below it.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
constexpr unsigned kNowhere = 0x80000000u;

// `rows` rows of `cols` elements, `ld` apart (none: an empty range).
template <typename T>
__device__ __forceinline__ rsrc_t rows_rsrc(const T* base, int rows, long ld, int cols) {
  return make_rsrc(base, rows > 0 ? (unsigned)(((rows - 1) * ld + cols) * (long)sizeof(T)) : 0u);
}
__device__ __forceinline__ uint4 bload16(rsrc_t r, unsigned off) {
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
}
template <typename T> __device__ __forceinline__ T bload(rsrc_t r, unsigned off);
template <> __device__ __forceinline__ float bload<float>(rsrc_t r, unsigned off) {
  return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, off, 0, 0));
}
template <> __device__ __forceinline__ bf16_t bload<bf16_t>(rsrc_t r, unsigned off) {
  return __builtin_bit_cast(bf16_t, __builtin_amdgcn_raw_buffer_load_b16(r, off, 0, 0));
}
__device__ __forceinline__ void bstore(rsrc_t r, unsigned off, float v) {
  __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, off, 0, 0);
}
__device__ __forceinline__ void bstore(rsrc_t r, unsigned off, bf16_t v) {
  __builtin_amdgcn_raw_buffer_store_b16(v, r, off, 0, 0);
}

// One row and head's walk by a wave of the two loops.
struct Walk {
  int b, h, len, live, c0, nc, w, lane, lo, hi, crow;
  long head, item0, kitem0;
  bool none;                           // no head for this work-group
  __device__ Walk(const DeltaArgs& a, int NT) {
    // work-groups go to the XCDs in turn: a head's columns to one of them, whose
    // L2 then reads the head's operands once
    const int ntile = (a.Dv + NT - 1) / NT, at = (int)(blockIdx.x >> 3);
    const int bh = (int)(blockIdx.x & 7) + 8 * (at / ntile);
    none = bh >= a.B * a.Hv;
    if (none) return;
    c0 = at % ntile * NT;
    nc = min(NT, a.Dv - c0);
    b = bh / a.Hv;
    h = bh % a.Hv;
    len = delta_len(a, b);
    live = (len + CT - 1) / CT;
    head = (long)bh * a.Dk * a.Dv;
    item0 = (long)bh * a.nch;
    kitem0 = ((long)b * a.Hk + h / (a.Hv / a.Hk)) * a.nch;
    lane = threadIdx.x & 63;
    w = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6) & 3);
    lo = lane & 15;
    hi = lane >> 4;
    crow = 16 * w + 4 * hi;            // first of the four rows of a result
  }
  // Byte offset of the lane's first row and column 16 q + lo in rows ld apart,
  // from the wave's first row.
  template <typename T>
  __device__ __forceinline__ unsigned place(int q, long ld) const {
    return 16 * q + lo < nc ? (unsigned)((4 * hi * ld + 16 * q + lo) * (long)sizeof(T)) : kNowhere;
  }
};

// A wave's fragments into registers: rows 16 w .. of K or Q of a chunk ..
template <int NP, int KS>
__device__ __forceinline__ void load_rows16(uint4 (*x)[KS], const bf16_t* base, const Walk& k) {
  const rsrc_t r = make_rsrc(base, NP * CT * 32 * KS * 2);
#pragma unroll
  for (int s = 0; s < KS; ++s)
#pragma unroll
    for (int e = 0; e < NP; ++e)
      x[e][s] = bload16(r, (frag_at(0, s, e, KS, NP) + k.w * KS * NP * 512) * 2 + k.lane * 16);
}

// .. of a 64 x 64 in three pieces, N of them (a triangular one: tiles 0 and 1
// of a lower and 2 and 3 of an upper one have nothing in one of the steps) ..
template <int N, bool LOW>
__device__ __forceinline__ void load_square16(uint4 (*x)[2], const bf16_t* base, const Walk& k) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const bool some = LOW ? s == 0 || k.w >= 2 : s == 1 || k.w < 2;
    const rsrc_t r = make_rsrc(base, some ? 3 * SQ * 2 : 0);
#pragma unroll
    for (int e = 0; e < N; ++e) x[e][s] = bload16(r, (frag_at(0, s, e, 2, 3) + k.w * 2 * 3 * 512) * 2 + k.lane * 16);
  }
}

// .. and the wave's MT row tiles of K^T or Q^T (tiles past the last read 0).
template <int NP, int MT, int DP>
__device__ __forceinline__ void load_transposed(uint4 (*x)[MT][2], const bf16_t* base, const Walk& k, bool own) {
  const rsrc_t r = make_rsrc(base, own ? NP * DP * CT * 2 : 0);
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int e = 0; e < NP; ++e)
        x[e][m][s] = bload16(r, (frag_at(m, s, e, 2, NP) + k.w * MT * 2 * NP * 512) * 2 + k.lane * 16);
}

// B operand: NN pieces of a column, from LDS [piece][NT][pitch].
template <int NN>
__device__ __forceinline__ void load_b(frag* f, const bf16_t* p, int stride) {
#pragma unroll
  for (int e = 0; e < NN; ++e) f[e] = lds_frag(p + e * stride);
}

// The wave's rows of the state: tiles of 16 from 16 w MT on.
template <int MT, int NL>
struct State {
  f32x4 x[MT][NL];
  __device__ __forceinline__ rsrc_t range(const Walk& k, const DeltaArgs& a, const float* p) const {
    const int d0 = 16 * k.w * MT;
    return rows_rsrc(p + (long)d0 * a.Dv + k.c0, min(16 * MT, a.Dk - d0), a.Dv, k.nc);
  }
  // from [Dk][Dv] floats at p; zeros without one
  __device__ __forceinline__ void load(const Walk& k, const DeltaArgs& a, const float* p) {
    const rsrc_t rs = range(k, a, p);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < NL; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          x[m][q][r] = p ? bload<float>(rs, k.place<float>(q, a.Dv) + (16 * m + r) * a.Dv * 4) : 0.f;
  }
  __device__ __forceinline__ void store(const Walk& k, const DeltaArgs& a, float* p) const {
    const rsrc_t rs = range(k, a, p);
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < NL; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) bstore(rs, k.place<float>(q, a.Dv) + (16 * m + r) * a.Dv * 4, x[m][q][r]);
  }
  // in pieces, column-major, for the products that read it
  __device__ __forceinline__ void publish(const Walk& k, bf16_t* Sp, int KP) const {
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int q = 0; q < NL; ++q)
        split4_store<3>(x[m][q], Sp + (16 * q + k.lo) * KP + ((16 * (k.w * MT + m) + 4 * k.hi) ^ swap8(k.lo)), 16 * NL * KP);
  }
};

template <typename T, int NT>
__device__ void zero_rest(T* out, long tok_ld, const DeltaArgs& a, const Walk& k) {
  const int tid = threadIdx.x, c = k.c0 + tid % NT;
  if (c < a.Dv)
    for (int t = k.live * CT + tid / NT; t < a.T; t += 512 / NT)
      out[((long)t * a.B + k.b) * tok_ld + (long)k.h * a.Dv + c] = Op<T>::from_f32(0.f);
}

}  // namespace

// ---------------------------------------------------------------------------
// state_fwd: the loop over a row's chunks for 16 NL columns of one head's state.
// Waves 0-3 carry the recurrence: K S, T R, K^T U, each wave 16 of the 64 tokens
// (and a quarter of the state's rows, which stay in its accumulators in float32);
// what the next product needs of the other waves goes through LDS in pieces.
// Waves 4-7 make Y beside them from the same pieces.  Three barriers a chunk.
// The operands that do not depend on the state are loaded a chunk ahead, each into
// its own registers as soon as the last product that reads them has been issued
// (two register sets in turn need 60 registers more: prompts 54 us against 45, 8
// rows 240 against 224).  The waves that make Y load in the phase in which they
// have nothing to multiply, and S and U are stored in the second phase: 8 rows 226
// -> 215 us, one row 657 -> 630.
// Bound: with few heads a chunk's three products one after the other, 2.6 us a chunk
// with 16 columns (1.5 of them when nothing else runs on the compute unit): one
// row 655 us for 256 chunks, on half of the compute units; with many the traffic of the operands and of what is
// kept for the gradient: 8 rows 227 us, 0.85 GB, 3.7 TB/s; prompts 46 us.
// ---------------------------------------------------------------------------
template <typename T, int KS, int NL, bool SAVE>
__global__ __launch_bounds__(512) void delta_state_fwd_kernel(DeltaArgs a) {
  constexpr int NP = Pieces<T>::n, DP = 32 * KS, KP = DP + 8, NT = 16 * NL;
  constexpr int MT = KS == 4 ? 2 : 1;                  // 16-row tiles of the state per wave
  __shared__ __align__(16) bf16_t Sp[3 * NT * KP];     // state, column-major pieces
  __shared__ __align__(16) bf16_t Rp[3 * NT * RC], Up[3 * NT * RC], Uy[3 * NT * RC];
  const Walk k(a, NT);
  if (k.none) return;
  const int lo = k.lo, h8 = 8 * k.hi ^ swap8(k.lo), wc = k.crow ^ swap8(k.lo);   // columns read, written in LDS
  const long vrow = (long)a.B * a.v_ld, yrow = (long)a.B * a.Hv * a.Dv;
  if (threadIdx.x < 256) {
    struct Ops {
      uint4 rows[NP][KS], sq[3][2], kt[NP][MT][2];
      float4 tok[4];
      float end;
      T v[4][NL];
    };
    const bool own = k.w * MT * 16 < DP;               // this wave holds rows of the state
    State<MT, NL> S;
    S.load(k, a, a.S0 && own ? a.S0 + k.head : nullptr);
    if (own) S.publish(k, Sp, KP);
    auto load_t = [&](Ops& o, int n) { load_square16<3, true>(o.sq, a.tp + (k.item0 + n) * 3 * SQ, k); };
    auto load_kt = [&](Ops& o, int n) {
      load_transposed<NP, MT, DP>(o.kt, a.ktp + (k.kitem0 + n) * NP * DP * CT, k, own);
      o.end = bload<float>(make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16), (CT - 1) * 16);
    };
    auto load_k = [&](Ops& o, int n) {
      load_rows16<NP, KS>(o.rows, a.kp + (k.kitem0 + n) * NP * CT * DP, k);
    };
    auto load_v = [&](Ops& o, int n) {
      const int t0 = n * CT + 16 * k.w;
      const rsrc_t rt = make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16);
      const rsrc_t rv = rows_rsrc(static_cast<const T*>(a.v) + ((long)t0 * a.B + k.b) * a.v_ld + (long)k.h * a.Dv + k.c0,
                                  min(16, k.len - t0), vrow, k.nc);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        o.tok[r] = __builtin_bit_cast(float4, bload16(rt, (k.crow + r) * 16));
#pragma unroll
        for (int q = 0; q < NL; ++q)
          o.v[r][q] = bload<T>(rv, k.place<T>(q, vrow) + (unsigned)(r * vrow * (long)sizeof(T)));
      }
    };
    auto chunk = [&](int n, Ops& o) {
      const long item = k.item0 + n;
      const int next = min(n + 1, k.live - 1);
      f32x4 ks[NL][2];                                 // two sums: the products wait for each other less
#pragma unroll
      for (int q = 0; q < NL; ++q) ks[q][0] = ks[q][1] = zero_acc();
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int q = 0; q < NL; ++q) {
          frag sb[3], ra[NP];
          load_b<3>(sb, Sp + (16 * q + lo) * KP + 32 * s + h8, NT * KP);
#pragma unroll
          for (int e = 0; e < NP; ++e) ra[e] = as_frag(o.rows[e][s]);
          mma<NP, 3, 2>(ra, sb, ks[q][s & 1]);
        }
      load_k(o, next);
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 rr;
#pragma unroll
        for (int r = 0; r < 4; ++r) rr[r] = o.tok[r].z * (Op<T>::to_f32(o.v[r][q]) - o.tok[r].x * (ks[q][0][r] + ks[q][1][r]));
        split4_store<3>(rr, Rp + (16 * q + lo) * RC + wc, NT * RC);
      }
      lds_barrier();
      const rsrc_t ru = rows_rsrc(a.u + (item * CT + 16 * k.w) * a.Dv + k.c0, SAVE ? 16 : 0, a.Dv, k.nc);
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 us, part[2] = {zero_acc(), zero_acc()};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          frag rb[3], tf[3];
          load_b<3>(rb, Rp + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
          for (int e = 0; e < 3; ++e) tf[e] = as_frag(o.sq[e][s]);
          mma<3, 3, 2>(tf, rb, part[s]);
        }
        const f32x4 u = part[0] + part[1];
#pragma unroll
        for (int r = 0; r < 4; ++r) us[r] = o.tok[r].y * u[r];
        split4_store<3>(us, Up + (16 * q + lo) * RC + wc, NT * RC);
        split4_store<3>(u, Uy + (16 * q + lo) * RC + wc, NT * RC);
        if (SAVE) {
#pragma unroll
          for (int r = 0; r < 4; ++r) bstore(ru, k.place<float>(q, a.Dv) + r * a.Dv * 4, u[r]);
        }
      }
      if (SAVE) S.store(k, a, a.st + item * a.Dk * a.Dv);
      load_t(o, next);
      load_v(o, next);
      lds_barrier();
      if (own) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int q = 0; q < NL; ++q) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S.x[m][q][r] *= o.end;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              frag ub[3], kf[NP];
              load_b<3>(ub, Up + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
              for (int e = 0; e < NP; ++e) kf[e] = as_frag(o.kt[e][m][s]);
              mma<NP, 3, 2>(kf, ub, S.x[m][q]);
            }
          }
        S.publish(k, Sp, KP);
      }
      load_kt(o, next);
      lds_barrier();
    };
    Ops A;
    if (k.live > 0) {
      load_k(A, 0);
      load_v(A, 0);
      load_t(A, 0);
      load_kt(A, 0);
    }
    lds_barrier();
    for (int n = 0; n < k.live; ++n) chunk(n, A);
    if (own && a.ST) S.store(k, a, a.ST + k.head);
  } else {
    struct Ops {
      uint4 rows[NP][KS], sq[3][2];
      float tok[4];
    };
    auto load_p = [&](Ops& o, int n) { load_square16<3, true>(o.sq, a.pp + (k.item0 + n) * 3 * SQ, k); };
    auto load_q = [&](Ops& o, int n) {
      load_rows16<NP, KS>(o.rows, a.qp + (k.kitem0 + n) * NP * CT * DP, k);
      const rsrc_t rt = make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) o.tok[r] = bload<float>(rt, (k.crow + r) * 16);
    };
    auto chunk = [&](int n, Ops& o) {
      const int next = min(n + 1, k.live - 1);
      f32x4 y[NL];
#pragma unroll
      for (int q = 0; q < NL; ++q) y[q] = zero_acc();
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int q = 0; q < NL; ++q) {
          frag sb[3], ra[NP];
          load_b<3>(sb, Sp + (16 * q + lo) * KP + 32 * s + h8, NT * KP);
#pragma unroll
          for (int e = 0; e < NP; ++e) ra[e] = as_frag(o.rows[e][s]);
          mma<NP, 3, 2>(ra, sb, y[q]);
        }
#pragma unroll
      for (int q = 0; q < NL; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) y[q][r] *= a.scale * o.tok[r];
      lds_barrier();
      load_q(o, next);
      lds_barrier();
      const int t0 = n * CT + 16 * k.w;
      const rsrc_t ry = rows_rsrc(static_cast<T*>(a.y) + ((long)t0 * a.B + k.b) * a.Hv * a.Dv + (long)k.h * a.Dv + k.c0,
                                  min(16, a.T - t0), yrow, k.nc);
#pragma unroll
      for (int q = 0; q < NL; ++q) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          frag ub[3], pf[3];
          load_b<3>(ub, Uy + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
          for (int e = 0; e < 3; ++e) pf[e] = as_frag(o.sq[e][s]);
          mma<3, 3, 2>(pf, ub, y[q]);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r)
          bstore(ry, k.place<T>(q, yrow) + (unsigned)(r * yrow * (long)sizeof(T)),
                 Op<T>::from_f32(n * CT + k.crow + r < k.len ? y[q][r] : 0.f));
      }
      load_p(o, next);
      lds_barrier();
    };
    Ops A;
    if (k.live > 0) {
      load_q(A, 0);
      load_p(A, 0);
    }
    lds_barrier();
    for (int n = 0; n < k.live; ++n) chunk(n, A);
  }
  zero_rest<T, NT>(static_cast<T*>(a.y), (long)a.Hv * a.Dv, a, k);
}

// ---------------------------------------------------------------------------
// state_bwd: the gradient loop, the same split.  Waves 0-3 carry dS: K dS, T^T dU,
// K^T dR.  Waves 4-7 make what does not depend on it, P^T dY and Q^T (scale e^G
// dY), one chunk ahead, each for the chain wave of its rows (through LDS, in the
// accumulators' order).  Bound as state_fwd: 8 rows 231 us, one row 650 us.
// ---------------------------------------------------------------------------
template <typename T, int KS, int NL>
__global__ __launch_bounds__(512) void delta_state_bwd_kernel(DeltaArgs a) {
  constexpr int NP = Pieces<T>::n, DP = 32 * KS, KP = DP + 8, NT = 16 * NL;
  constexpr int MT = KS == 4 ? 2 : 1;
  __shared__ __align__(16) bf16_t Sp[3 * NT * KP];
  __shared__ __align__(16) bf16_t Rp[3 * NT * RC], Up[3 * NT * RC];
  __shared__ __align__(16) bf16_t Yp[NP * NT * RC], Ys[3 * NT * RC];   // dY, scale e^G dY of the next chunk
  __shared__ f32x4 mail[2][4][(MT + 1) * NL][64];
  const Walk k(a, NT);
  if (k.none) return;
  const int lo = k.lo, l = threadIdx.x & 63;
  const int h8 = 8 * k.hi ^ swap8(lo), wc = k.crow ^ swap8(lo);   // columns read, written in LDS
  const bool own = k.w * MT * 16 < DP;
  const long vrow = (long)a.B * a.dv_ld, yrow = (long)a.B * a.Hv * a.Dv;
  if (threadIdx.x < 256) {
    struct Ops {
      uint4 rows[NP][KS], sq[3][2], kt[NP][MT][2];
      float4 tok[4];
      float end;
    };
    State<MT, NL> S;
    S.load(k, a, a.dST && own ? a.dST + k.head : nullptr);
    if (own) S.publish(k, Sp, KP);
    auto load_t = [&](Ops& o, int n) { load_square16<3, false>(o.sq, a.ttp + (k.item0 + n) * 3 * SQ, k); };
    auto load_kt = [&](Ops& o, int n) {
      load_transposed<NP, MT, DP>(o.kt, a.ktp + (k.kitem0 + n) * NP * DP * CT, k, own);
      o.end = bload<float>(make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16), (CT - 1) * 16);
    };
    auto load_k = [&](Ops& o, int n) {
      load_rows16<NP, KS>(o.rows, a.kp + (k.kitem0 + n) * NP * CT * DP, k);
    };
    auto load_tok = [&](Ops& o, int n) {
      const rsrc_t rt = make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16);
#pragma unroll
      for (int r = 0; r < 4; ++r) o.tok[r] = __builtin_bit_cast(float4, bload16(rt, (k.crow + r) * 16));
    };
    auto chunk = [&](int n, Ops& o) {
      const long item = k.item0 + n;
      const int slot = n & 1, next = max(n - 1, 0);
      f32x4 du[NL][2];
#pragma unroll
      for (int q = 0; q < NL; ++q) du[q][0] = du[q][1] = zero_acc();
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int q = 0; q < NL; ++q) {
          frag sb[3], ra[NP];
          load_b<3>(sb, Sp + (16 * q + lo) * KP + 32 * s + h8, NT * KP);
#pragma unroll
          for (int e = 0; e < NP; ++e) ra[e] = as_frag(o.rows[e][s]);
          mma<NP, 3, 2>(ra, sb, du[q][s & 1]);
        }
      load_k(o, next);
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 x = mail[slot][k.w][q][l];
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] += o.tok[r].y * (du[q][0][r] + du[q][1][r]);
        split4_store<3>(x, Rp + (16 * q + lo) * RC + wc, NT * RC);
      }
      S.store(k, a, a.dst + item * a.Dk * a.Dv);
      lds_barrier();
      const int t0 = n * CT + 16 * k.w;
      const rsrc_t rr = rows_rsrc(a.dr + (item * CT + 16 * k.w) * a.Dv + k.c0, 16, a.Dv, k.nc);
      const rsrc_t rv = rows_rsrc(static_cast<T*>(a.dv) + ((long)t0 * a.B + k.b) * a.dv_ld + (long)k.h * a.Dv + k.c0,
                                  min(16, a.T - t0), vrow, k.nc);
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 zs, part[2] = {zero_acc(), zero_acc()};
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          frag rb[3], tf[3];
          load_b<3>(rb, Rp + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
          for (int e = 0; e < 3; ++e) tf[e] = as_frag(o.sq[e][s]);
          mma<3, 3, 2>(tf, rb, part[s]);
        }
        f32x4 z = part[0] + part[1];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          z[r] *= o.tok[r].z;                            // dR
          zs[r] = -o.tok[r].x * z[r];
        }
        split4_store<3>(zs, Up + (16 * q + lo) * RC + wc, NT * RC);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          bstore(rr, k.place<float>(q, a.Dv) + r * a.Dv * 4, z[r]);
          bstore(rv, k.place<T>(q, vrow) + (unsigned)(r * vrow * (long)sizeof(T)),
                 Op<T>::from_f32(n * CT + k.crow + r < k.len ? z[r] : 0.f));
        }
      }
      load_t(o, next);
      load_tok(o, next);
      lds_barrier();
      if (own) {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int q = 0; q < NL; ++q) {
            const f32x4 x = mail[slot][k.w][NL + m * NL + q][l];
#pragma unroll
            for (int r = 0; r < 4; ++r) S.x[m][q][r] = o.end * S.x[m][q][r] + x[r];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              frag ub[3], kf[NP];
              load_b<3>(ub, Up + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
              for (int e = 0; e < NP; ++e) kf[e] = as_frag(o.kt[e][m][s]);
              mma<NP, 3, 2>(kf, ub, S.x[m][q]);
            }
          }
        S.publish(k, Sp, KP);
      }
      load_kt(o, next);
      lds_barrier();
    };
    Ops A;
    if (k.live > 0) {
      load_k(A, k.live - 1);
      load_tok(A, k.live - 1);
      load_t(A, k.live - 1);
      load_kt(A, k.live - 1);
    }
    lds_barrier();
    lds_barrier();
    for (int n = k.live - 1; n >= 0; --n) chunk(n, A);
    if (own && a.dS0) S.store(k, a, a.dS0 + k.head);
  } else {
    struct Ops {
      uint4 sq[3][2], qt[NP][MT][2];
      float tok[4];
      T y[4][NL];
    };
    auto load_dy = [&](Ops& o, int n) {
      const int t0 = n * CT + 16 * k.w;
      const rsrc_t rt = make_rsrc(a.tok + (k.item0 + n) * CT, CT * 16);
      const rsrc_t ry = rows_rsrc(static_cast<const T*>(a.dy) + ((long)t0 * a.B + k.b) * a.Hv * a.Dv + (long)k.h * a.Dv + k.c0,
                                  min(16, k.len - t0), yrow, k.nc);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        o.tok[r] = bload<float>(rt, (k.crow + r) * 16);
#pragma unroll
        for (int q = 0; q < NL; ++q)
          o.y[r][q] = bload<T>(ry, k.place<T>(q, yrow) + (unsigned)(r * yrow * (long)sizeof(T)));
      }
    };
    auto load_sq = [&](Ops& o, int n) {
      load_square16<3, false>(o.sq, a.ptp + (k.item0 + n) * 3 * SQ, k);
      load_transposed<NP, MT, DP>(o.qt, a.qtp + (k.kitem0 + n) * NP * DP * CT, k, own);
    };
    // dY of the fetched chunk into LDS ..
    auto lay_dy = [&](const Ops& o) {
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 y, ys;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          y[r] = Op<T>::to_f32(o.y[r][q]);
          ys[r] = a.scale * o.tok[r] * y[r];
        }
        split4_store<NP>(y, Yp + (16 * q + lo) * RC + wc, NT * RC);
        split4_store<3>(ys, Ys + (16 * q + lo) * RC + wc, NT * RC);
      }
    };
    // .. and the two products into the mailbox
    auto products = [&](int slot, const Ops& o) {
#pragma unroll
      for (int q = 0; q < NL; ++q) {
        f32x4 x = zero_acc();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          frag yb[NP], pa[3];
          load_b<NP>(yb, Yp + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
          for (int e = 0; e < 3; ++e) pa[e] = as_frag(o.sq[e][s]);
          mma<3, NP, 2>(pa, yb, x);
        }
        mail[slot][k.w][q][l] = x;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          f32x4 z = zero_acc();
#pragma unroll
          for (int s = 0; s < 2; ++s) {
            frag yb[3], qa[NP];
            load_b<3>(yb, Ys + (16 * q + lo) * RC + 32 * s + h8, NT * RC);
#pragma unroll
            for (int e = 0; e < NP; ++e) qa[e] = as_frag(o.qt[e][m][s]);
            mma<NP, 3, 2>(qa, yb, z);
          }
          mail[slot][k.w][NL + m * NL + q][l] = z;
        }
      }
    };
    Ops A;
    if (k.live > 0) {
      load_dy(A, k.live - 1);
      load_sq(A, k.live - 1);
      lay_dy(A);
      load_dy(A, max(k.live - 2, 0));
    }
    lds_barrier();
    if (k.live > 0) {
      products((k.live - 1) & 1, A);
      load_sq(A, max(k.live - 2, 0));
    }
    lds_barrier();
    // in the chain's chunk n: chunk n - 1's products, loads of chunk n - 2
    for (int n = k.live - 1; n >= 0; --n) {
      const int next = max(n - 2, 0);
      lay_dy(A);
      load_dy(A, next);
      lds_barrier();
      products((n - 1) & 1, A);
      lds_barrier();
      load_sq(A, next);
      lds_barrier();
    }
  }
  zero_rest<T, NT>(static_cast<T*>(a.dv), a.dv_ld, a, k);
}

// ---------------------------------------------------------------------------
// grads: one work-group of eight waves per item of a key head; wave = 16 of the 64
// tokens x half of the columns.  The value columns are walked 32 at a time, the
// states' rows 64 at a time within: dY, U, dR and the two states go through LDS
// in pieces.  A step's products read one of two buffers while the next step is
// split into the other and the one after it is on its way into registers.  F, H
// and the three products with the states stay in accumulators.  The value heads
// of a key head follow one another, so dQ and dK are summed in a fixed order.
// After the walk K^T and Q^T come through LDS once for all eight waves: read by each
// wave for itself from global memory they took 10 of 52 thousand cycles a head's
// chunk.  Bound: HBM in the walk (U, dR and both states of every chunk, 5 TB/s),
// which stands still while F, H and what follows are made, since LDS holds one
// work-group (139 KB): 8 rows 330 to 346 us, 1.2 GB, 3.5 TB/s; one row 379 us.
// ---------------------------------------------------------------------------
template <typename T, int KS>
__global__ __launch_bounds__(512) void delta_grads_kernel(DeltaArgs a) {
  constexpr int NP = Pieces<T>::n;
  constexpr int DP = 32 * KS, NC = 32, CP = NC + 8, ND = DP / 32;
  constexpr int TPS = ND < 2 ? ND : 2, HS = ND / TPS, DR = 32 * TPS;   // column tiles of a wave, row halves, rows a step
  constexpr int kTok = (NP + 6) * CT * CP, kState = 6 * DR * CP, kSq = 9 * CT * RC;
  // after the walk: F and H, K^T and Q^T (all of them, or half the column tiles at a
  // time where LDS does not hold them)
  constexpr int NS = NP == 3 && KS == 4 ? 2 : 1, kTr = NP * DP * CT / NS;
  constexpr int kPool = 2 * (kTok + kState), kEnd = kSq + 2 * kTr;
  __shared__ __align__(16) bf16_t pool[kPool > kEnd ? kPool : kEnd];
  __shared__ float4 tok[CT];
  __shared__ double G[CT];
  __shared__ float part[8][4], sbeta[CT];
  // sums of X: of row i over column tile jt < its own; for column t over the rows >= t of
  // row tile w and the columns below t of t's tile
  __shared__ float rowsX[3][CT], colsX[4][CT];
  __shared__ float nearS[2][CT], farS[2][CT];            // the tokens' terms with S0, with dS'
  // tokens' buffer: dY [NP][64][CP], U [3][64][CP], dR [3][64][CP]; states': S
  // [3][DR][CP], dS [3][DR][CP]
  constexpr int kU = NP * CT * CP, kR = kU + 3 * CT * CP, kD = 3 * DR * CP;
  bf16_t* Fp = pool;                   // [3][64][RC] F, rows i          (after the walk)
  bf16_t* Ft = Fp + 3 * CT * RC;       // [3][64][RC] F^T
  bf16_t* Hp = Ft + 3 * CT * RC;      // [3][64][RC] H + H^T
  bf16_t* Kt = Hp + 3 * CT * RC;      // K^T, Q^T in fragments
  bf16_t* Qt = Kt + kTr;
  // the wave's column tile i of the results
  auto tile = [](int i, int half) { return i / TPS * 2 * TPS + half * TPS + i % TPS; };
  const int n = blockIdx.x % a.nch, bk = blockIdx.x / a.nch;
  const int b = bk / a.Hk, hk = bk % a.Hk, grp = a.Hv / a.Hk;
  const int len = delta_len(a, b), t0 = n * CT;
  const int tid = threadIdx.x, l = tid & 63, lo_ = l & 15, hi_ = l >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), w = wave & 3, half = wave >> 2;
  T* dq = static_cast<T*>(a.dq);
  T* dk = static_cast<T*>(a.dk);
  if (t0 >= len) {
    for (int r = wave; r < CT && t0 + r < a.T; r += 8) {
      const long at = (long)(t0 + r) * a.B + b;
      for (int c = l; c < a.Dk; c += 64) {
        dq[at * a.dq_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(0.f);
        dk[at * a.dk_ld + (long)hk * a.Dk + c] = Op<T>::from_f32(0.f);
      }
      for (int c = l; c < grp; c += 64) {
        a.dg[at * a.Hv + hk * grp + c] = 0.f;
        a.dbeta[at * a.Hv + hk * grp + c] = 0.f;
      }
    }
    return;
  }
  f32x4 tq[ND], tkk[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) tq[i] = tkk[i] = zero_acc();
  const long kitem = bk * (long)a.nch + n;
  const rsrc_t rk = make_rsrc(a.ktp + kitem * NP * DP * CT, NP * DP * CT * 2);
  const rsrc_t rq = make_rsrc(a.qtp + kitem * NP * DP * CT, NP * DP * CT * 2);
  const rsrc_t rx = make_rsrc(a.dots + kitem * kDeltaDots, kDeltaDots * 4);
  // K or Q at the results' places (rows crow .. crow + 3 of a column), as the
  // transposes hold them: four neighbours of one fragment
  auto column = [&](const bf16_t* tr, int i) {
    f32x4 v = zero_acc();
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const uint2 u = *reinterpret_cast<const uint2*>(tr + frag_at(i, w >> 1, e, 2, NP) +
                                                      ((2 * (w & 1) + (hi_ >> 1)) * 16 + lo_) * 8 + 4 * (hi_ & 1));
      v += f32x4{__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                 __uint_as_float(u.y & 0xffff0000u)};
    }
    return v;
  };
  // loads of a step, four columns a thread: a row of each state and, with the
  // first rows, a token (descriptors as in the loops: uniform bases, so that few
  // addresses live in registers)
  const int h8 = 8 * hi_ ^ swap8(lo_);
  const int row = tid >> 3, rc = (tid & 7) * 4, wc = rc ^ swap8(row);
  const long yrow = (long)a.B * a.Hv * a.Dv;
  struct alignas(4 * sizeof(T)) Four { T x[4]; };
  f32x4 fs, fd, fu, fr;
  Four fy;
  auto load4 = [&](rsrc_t r, unsigned off, Four& f) {
    if constexpr (NP == 1) f = __builtin_bit_cast(Four, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, 0));
    else f = __builtin_bit_cast(Four, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, 0));
  };
  auto fetch = [&](int h, int c0, int hs) {
    const long item = ((long)b * a.Hv + h) * a.nch + n;
    const bool in = c0 + rc < a.Dv;
    const rsrc_t rs = make_rsrc(a.st + item * a.Dk * a.Dv, a.Dk * a.Dv * 4), rd = make_rsrc(a.dst + item * a.Dk * a.Dv, a.Dk * a.Dv * 4);
    const unsigned at = in && row < DR ? ((hs * DR + row) * a.Dv + c0 + rc) * 4 : kNowhere;
    fs = __builtin_bit_cast(f32x4, bload16(rs, at));
    fd = __builtin_bit_cast(f32x4, bload16(rd, at));
    if (hs == 0) {
      const rsrc_t ru = make_rsrc(a.u + item * CT * a.Dv, CT * a.Dv * 4), rr = make_rsrc(a.dr + item * CT * a.Dv, CT * a.Dv * 4);
      const unsigned off = in ? (row * a.Dv + c0 + rc) * 4 : kNowhere;
      fu = __builtin_bit_cast(f32x4, bload16(ru, off));
      fr = __builtin_bit_cast(f32x4, bload16(rr, off));
      const int tv = min(8, len - t0 - 8 * wave);          // the wave's eight rows: its tokens
      const long tok0 = (long)(t0 + 8 * wave) * a.B + b;
      const rsrc_t ry = rows_rsrc(static_cast<const T*>(a.dy) + (tok0 * a.Hv + h) * a.Dv, tv, yrow, a.Dv);
      load4(ry, in ? (unsigned)(((row & 7) * yrow + c0 + rc) * (long)sizeof(T)) : kNowhere, fy);
    }
  };
  fetch(hk * grp, 0, 0);
  for (int hh = 0; hh < grp; ++hh) {
    const int h = hk * grp + hh;
    const long item = ((long)b * a.Hv + h) * a.nch + n;
    f32x4 aq[ND], ku[ND], kr[ND], F[2], H[2];
#pragma unroll
    for (int i = 0; i < ND; ++i) aq[i] = ku[i] = kr[i] = zero_acc();
    F[0] = F[1] = H[0] = H[1] = zero_acc();
    float ss = 0.f, ub = 0.f;
    // the fetched step into the buffers (cb: of the tokens, sb: of the states)
    auto split = [&](int hs, int cb, int sb) {
      bf16_t* S = pool + 2 * kTok + sb * kState;
      if (row < DR) {
#pragma unroll
        for (int e = 0; e < 4; ++e) ss += fs[e] * fd[e];
        split4_store<3>(fs, S + row * CP + wc, DR * CP);
        split4_store<3>(fd, S + kD + row * CP + wc, DR * CP);
      }
      if (hs == 0) {
        bf16_t* X = pool + cb * kTok;
        f32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y[e] = Op<T>::to_f32(fy.x[e]);
          ub += fr[e] * fu[e];
        }
        split4_store<NP>(y, X + row * CP + wc, CT * CP);
        split4_store<3>(fu, X + kU + row * CP + wc, CT * CP);
        split4_store<3>(fr, X + kR + row * CP + wc, CT * CP);
      }
    };
    lds_barrier();
    if (tid < CT) {
      tok[tid] = a.tok[item * CT + tid];
      G[tid] = a.G[item * CT + tid];
    }
    split(0, 0, 0);
    if (HS > 1) fetch(h, 0, 1);
    else if (NC < a.Dv) fetch(h, NC, 0);
    else if (hh + 1 < grp) fetch(h + 1, 0, 0);
    for (int ct = 0; ct * NC < a.Dv; ++ct) {
      const int c0 = ct * NC;
      const bool more = c0 + NC < a.Dv;
#pragma unroll
      for (int hs = 0; hs < HS; ++hs) {
        const int sb = HS == 2 ? hs : ct & 1, cb = ct & 1;
        lds_barrier();
        // the next step's pieces, the loads of the one after it
        if (hs + 1 < HS) {
          split(1, cb, 1 - sb);
          if (more) fetch(h, c0 + NC, 0);
          else if (hh + 1 < grp) fetch(h + 1, 0, 0);
        } else if (more) {
          split(0, 1 - cb, 1 - sb);
          if (HS == 2) fetch(h, c0 + NC, 1);
          else if (c0 + 2 * NC < a.Dv) fetch(h, c0 + 2 * NC, 0);
          else if (hh + 1 < grp) fetch(h + 1, 0, 0);
        }
        const bf16_t* X = pool + cb * kTok + (16 * w + lo_) * CP + h8;
        const bf16_t* S = pool + 2 * kTok + sb * kState + lo_ * CP + h8;
        frag ya[NP], ua[3], ra[3];
#pragma unroll
        for (int e = 0; e < NP; ++e) ya[e] = lds_frag(X + e * CT * CP);
#pragma unroll
        for (int e = 0; e < 3; ++e) ua[e] = lds_frag(X + kU + e * CT * CP);
#pragma unroll
        for (int e = 0; e < 3; ++e) ra[e] = lds_frag(X + kR + e * CT * CP);
        if (hs == 0) {
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const int j = 2 * half + m;
            if (j <= w) {
              frag un[3];
#pragma unroll
              for (int e = 0; e < 3; ++e) un[e] = lds_frag(pool + cb * kTok + kU + (e * CT + 16 * j + lo_) * CP + h8);
              mma<NP, 3, 2>(ya, un, F[m]);
              mma<3, 3, 2>(ra, un, H[m]);
            }
          }
        }
#pragma unroll
        for (int i = 0; i < TPS; ++i) {
          frag sf[3], df[3];
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            sf[e] = lds_frag(S + (e * DR + 16 * (half * TPS + i)) * CP);
            df[e] = lds_frag(S + kD + (e * DR + 16 * (half * TPS + i)) * CP);
          }
          mma<NP, 3, 2>(ya, sf, aq[hs * TPS + i]);
          mma<3, 3, 2>(ua, df, ku[hs * TPS + i]);
          mma<3, 3, 2>(ra, sf, kr[hs * TPS + i]);
        }
      }
    }
    // K^T and Q^T on their way while F and H are made
    constexpr int NL = (kTr / 8 + 511) / 512;
    uint4 kraw[NL], qraw[NL];
    auto load_kq = [&](int st) {
#pragma unroll
      for (int x = 0; x < NL; ++x) {
        const unsigned at = (tid + 512 * x) * 8 < kTr ? (st * kTr + (tid + 512 * x) * 8) * 2 : kNowhere;
        kraw[x] = bload16(rk, at);
        qraw[x] = bload16(rq, at);
      }
    };
    auto lay_kq = [&]() {
#pragma unroll
      for (int x = 0; x < NL; ++x)
        if ((tid + 512 * x) * 8 < kTr) {
          *reinterpret_cast<uint4*>(Kt + (tid + 512 * x) * 8) = kraw[x];
          *reinterpret_cast<uint4*>(Qt + (tid + 512 * x) * 8) = qraw[x];
        }
    };
    // q_i.k_j and k_i.k_j at F's and H's places
    f32x4 qk[2], kk[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const unsigned at = 2 * half + m <= w ? (w * (w + 1) / 2 + 2 * half + m) * 2048 + l * 16 : kNowhere;
      qk[m] = __builtin_bit_cast(f32x4, bload16(rx, at));
      kk[m] = __builtin_bit_cast(f32x4, bload16(rx, at + 1024));
    }
    load_kq(0);
    // (places computed anew for every head: kept over the walk they would spill)
    int lo = lo_, hi = hi_;
    asm volatile("" : "+v"(lo), "+v"(hi));
    const int arow = 16 * w + lo, crow = 16 * w + 4 * hi;
    lds_barrier();
    // F, F^T and H + H^T in pieces (F_ij of tile (w, jt), jt <= w; zero above)
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const int jt = 2 * half + m, j = 16 * jt + lo;
      f32x4 f, hm;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = crow + r;
        const float d = j <= i ? expf((float)(G[i] - G[j])) : 0.f;
        f[r] = j <= i ? a.scale * d * F[m][r] : 0.f;
        hm[r] = j < i ? -d * H[m][r] : 0.f;
      }
      {
        float below = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float x = scan16(j < crow + r ? f[r] * qk[m][r] + hm[r] * kk[m][r] : 0.f);
          if (jt < w && lo == 15) rowsX[jt][crow + r] = x;
          below += j <= crow + r ? moved<kUpOne>(x) : 0.f;
        }
        below = sum_rows(below);
        if (hi == 0) colsX[w][j] = below;
      }
      // rows i .. i + 3 of column j: consecutive in the transpose
      split4_store<3>(f, Ft + j * RC + (crow ^ swap8(lo)), CT * RC);
      uint32_t p0[3], p1[3];
      split2<3>(f[0], f[1], p0);
      split2<3>(f[2], f[3], p1);
#pragma unroll
      for (int e = 0; e < 3; ++e) {
        bf16_t* x = Fp + (e * CT + crow) * RC + (j ^ swap8(4 * hi));
        x[0] = (bf16_t)p0[e];
        x[RC] = (bf16_t)(p0[e] >> 16);
        x[2 * RC] = (bf16_t)p1[e];
        x[3 * RC] = (bf16_t)(p1[e] >> 16);
      }
      // H below the diagonal, its mirror above (the diagonal is 0): a tile below
      // writes both, a diagonal one its lower entries and their mirrors
      if (jt < w) split4_store<3>(hm, Hp + j * RC + (crow ^ swap8(lo)), CT * RC);
      if (jt <= w) {
        split2<3>(hm[0], hm[1], p0);
        split2<3>(hm[2], hm[3], p1);
#pragma unroll
        for (int e = 0; e < 3; ++e) {
          const bf16_t q[4] = {(bf16_t)p0[e], (bf16_t)(p0[e] >> 16), (bf16_t)p1[e], (bf16_t)(p1[e] >> 16)};
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = crow + r;
            if (j <= i) {
              Hp[(e * CT + i) * RC + (j ^ swap8(4 * hi))] = q[r];
              if (jt == w) Hp[(e * CT + j) * RC + (i ^ swap8(lo))] = q[r];
            }
          }
        }
      }
    }
    ss *= tok[CT - 1].x;
    float nr[4] = {0.f, 0.f, 0.f, 0.f}, fs4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float4 tk = tok[crow + r];
#pragma unroll
      for (int i = 0; i < ND; ++i) {
        ku[i][r] *= tk.y;
        aq[i][r] *= a.scale * tk.x;
        kr[i][r] *= tk.x;
      }
    }
    ub = sum8(ub);
    if ((tid & 7) == 0) sbeta[row] = ub;
#pragma unroll
    for (int st = 0; st < NS; ++st) {
      if (st > 0) lds_barrier();
      lay_kq();
      lds_barrier();
      if (st + 1 < NS) load_kq(st + 1);
#pragma unroll
      for (int i = st * ND / NS; i < (st + 1) * ND / NS; ++i) {
        const int ti = tile(i, half) - st * (2 * KS / NS);
        const f32x4 kc = column(Kt, ti), qc = column(Qt, ti);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          nr[r] += aq[i][r] * qc[r] - kr[i][r] * kc[r];
          fs4[r] += ku[i][r] * kc[r];
        }
        f32x4 x = zero_acc();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
          frag fa[3], ta[3], ha[3], kb[NP], qb[NP];
#pragma unroll
          for (int e = 0; e < NP; ++e) {
            kb[e] = lds_frag(Kt + frag_at(ti, s, e, 2, NP) + 8 * (16 * hi + lo));
            qb[e] = lds_frag(Qt + frag_at(ti, s, e, 2, NP) + 8 * (16 * hi + lo));
          }
#pragma unroll
          for (int e = 0; e < 3; ++e) fa[e] = lds_frag(Fp + (e * CT + arow) * RC + 32 * s + (8 * hi ^ swap8(lo)));
#pragma unroll
          for (int e = 0; e < 3; ++e) {
            ta[e] = lds_frag(Ft + (e * CT + arow) * RC + 32 * s + (8 * hi ^ swap8(lo)));
            ha[e] = lds_frag(Hp + (e * CT + arow) * RC + 32 * s + (8 * hi ^ swap8(lo)));
          }
          mma<3, NP, 2>(fa, kb, aq[i]);
          mma<3, NP, 2>(ta, qb, x);
          mma<3, NP, 2>(ha, kb, x);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          tq[i][r] += aq[i][r];
          tkk[i][r] += x[r] + ku[i][r] - kr[i][r];
        }
        __builtin_amdgcn_sched_barrier(0);               // (tiles mixed by the compiler would spill)
      }
    }
    ss = sum16(ss);
    if (lo == 0) part[wave][hi] = ss;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      nr[r] = sum16(nr[r]);
      fs4[r] = sum16(fs4[r]);
      if (lo == 0) {
        nearS[half][crow + r] = nr[r];
        farS[half][crow + r] = fs4[r];
      }
    }
    lds_barrier();
    if (tid < CT) {
      const float bt = tok[tid].z;
      if (t0 + tid < a.T)
        a.dbeta[((long)(t0 + tid) * a.B + b) * a.Hv + h] = t0 + tid < len ? sbeta[tid] / (bt * bt) : 0.f;
      // lane by lane from the chunk's end: token at, of tile jt
      const int at = CT - 1 - tid, jt = at >> 4;
      double all = scan64((double)nearS[0][at] + nearS[1][at]);
      const double c = scan64((double)farS[0][tid] + farS[1][tid]), before = __shfl(c, at - 1, 64);
      if (at > 0) all += before;
      // pairs in t's column tile, then those of the tiles before it: rows of t's own tile, of later ones
      for (int i = jt; i < 4; ++i) all += colsX[i][at];
      const double r0 = jt > 0 ? rowsX[0][at] : 0., r1 = jt > 1 ? rowsX[1][at] : 0., r2 = jt > 2 ? rowsX[2][at] : 0.;
      all += scan16(r0 + r1 + r2);
      const double s0 = sum16(r0), s1 = sum16(r1);
      const double s03 = __shfl(s0, 0, 64), s02 = __shfl(s0, 16, 64), s13 = __shfl(s1, 0, 64);
      if (jt == 1) all += s02 + s03;
      if (jt == 2) all += s03 + s13;
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) all += part[i][j];
      if (t0 + at < a.T) a.dg[((long)(t0 + at) * a.B + b) * a.Hv + h] = t0 + at < len ? (float)all : 0.f;
    }
  }
  const int crow = 16 * w + 4 * hi_, rows = a.T - t0 - crow;
  const long at = (long)(t0 + crow) * a.B + b;
#pragma unroll
  for (int i = 0; i < ND; ++i) {
    const int c = 16 * tile(i, half);
    if (c + lo_ >= a.Dk) continue;                       // (Dk is even: pairs of lanes agree)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (t0 + crow + r >= len) tq[i][r] = tkk[i][r] = 0.f;
    store_tile(dq + at * a.dq_ld + (long)hk * a.Dk + c, (long)a.B * a.dq_ld, tq[i], lo_, rows);
    store_tile(dk + at * a.dk_ld + (long)hk * a.Dk + c, (long)a.B * a.dk_ld, tkk[i], lo_, rows);
  }
}

namespace {

// Columns of the state per work-group, in 16s: 32 where that still gives every
// compute unit a work-group (16 read the chunk's operands twice as often).  32 against
// 16 columns, 16 heads of 128 columns: inference over 1000 tokens takes 280 against 322
// us for 16 whole rows and 800 against 920 for 64 of 100 to 1000 tokens (8 of those:
// 105 against 95), 8 rows' forward and gradient 816 against 897, as many of 2048 tokens
// 990 against 1215; for 2 rows' inference it is 59 against 46, for one row of 16384,
// forward and gradient, 2127 against 1800.
int cols_of(const DeltaArgs& a, int cus) {
  return a.Dv > 16 && (long)a.B * a.Hv * ((a.Dv + 31) / 32) >= cus ? 2 : 1;
}

template <typename T, int KS, int NL>
hipError_t launch_state(const DeltaArgs& a, bool save, bool bwd, hipStream_t s) {
  const dim3 grid((unsigned)(((long)a.B * a.Hv + 7) / 8 * 8 * ((a.Dv + 16 * NL - 1) / (16 * NL))));
  if (bwd) delta_state_bwd_kernel<T, KS, NL><<<grid, dim3(512), 0, s>>>(a);
  else if (save) delta_state_fwd_kernel<T, KS, NL, true><<<grid, dim3(512), 0, s>>>(a);
  else delta_state_fwd_kernel<T, KS, NL, false><<<grid, dim3(512), 0, s>>>(a);
  return hipGetLastError();
}

template <typename T, int KS>
hipError_t launch_cols(const DeltaArgs& a, bool save, bool bwd, int cus, hipStream_t s) {
  return cols_of(a, cus) == 2 ? launch_state<T, KS, 2>(a, save, bwd, s) : launch_state<T, KS, 1>(a, save, bwd, s);
}

template <typename T, int KS>
hipError_t launch_fwd(const DeltaArgs& a, bool save, int cus, hipStream_t s) {
  const dim3 items((unsigned)((long)a.B * a.Hv * a.nch));
  if (save) delta_prep_kernel<T, KS, true><<<items, dim3(256), 0, s>>>(a);
  else delta_prep_kernel<T, KS, false><<<items, dim3(256), 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  return launch_cols<T, KS>(a, save, false, cus, s);
}

template <typename T, int KS>
hipError_t launch_bwd(const DeltaArgs& a, int cus, hipStream_t s) {
  hipError_t e = launch_cols<T, KS>(a, true, true, cus, s);
  if (e != hipSuccess) return e;
  delta_grads_kernel<T, KS><<<dim3((unsigned)((long)a.B * a.Hk * a.nch)), dim3(512), 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

template <typename T>
hipError_t delta_launch_fwd(const DeltaArgs& a, bool save, int cus, hipStream_t s) {
  switch (delta_ksteps(a.Dk)) {
    case 1: return launch_fwd<T, 1>(a, save, cus, s);
    case 2: return launch_fwd<T, 2>(a, save, cus, s);
    default: return launch_fwd<T, 4>(a, save, cus, s);
  }
}

template <typename T>
hipError_t delta_launch_bwd(const DeltaArgs& a, int cus, hipStream_t s) {
  switch (delta_ksteps(a.Dk)) {
    case 1: return launch_bwd<T, 1>(a, cus, s);
    case 2: return launch_bwd<T, 2>(a, cus, s);
    default: return launch_bwd<T, 4>(a, cus, s);
  }
}

template hipError_t delta_launch_fwd<float>(const DeltaArgs&, bool, int, hipStream_t);
template hipError_t delta_launch_fwd<bf16_t>(const DeltaArgs&, bool, int, hipStream_t);
template hipError_t delta_launch_bwd<float>(const DeltaArgs&, int, hipStream_t);
template hipError_t delta_launch_bwd<bf16_t>(const DeltaArgs&, int, hipStream_t);

}  // namespace ll
