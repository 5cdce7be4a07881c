// Linear attention with a decay for each head: forward, gradient, one-token step.
//
//   S_t = l S_{t-1} + k_t v_t^T,  y_t = scale S_t^T q_t,  l = e^g of the head
// and, with D_t = dL/dS_t (all of it), D_t = l D_{t+1} + scale q_t dy_t^T,
//   dq_t = scale S_t dy_t,  dk_t = D_t v_t,  dv_t = D_t^T k_t,  dS0 = l D_1
// are the same recurrence four times (LinPass): rows a ask, rows b and c make the state
//   out_i = w_P sum_{j <= i} l^{i-j} (a_i.b_j) c_j + w_A l^{i+e} a_i S
//   S'    = l^m S + w_U sum_j l^{m-j-e} b_j c_j^T          over m tokens, S entering
//   y:  a, b, c = q, k, v     dq: dy, v, k (state S^T)           e = 1
//   dv: a, b, c = k, q, dy    dk: v, dy, q (state D^T)   e = 0, tokens from the last on
#include <algorithm>
#include <cmath>
#include <new>

#include "ll_host.h"
#include "ll_kernels.h"
#include "ll_pieces.h"

using ll::bf16_t;
using ll::fail;

namespace ll {

constexpr int kLinMaxD = 128;
constexpr int kLinStepCols = 32;

__device__ __forceinline__ float uniform(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// Tokens of a chunk: 16 KB of 128 columns in either type.  The state is rounded to float
// once a chunk.  (bfloat16 chunks of 32: 5.3 us for 64 tokens and head of a compute unit
// instead of 5.1.)
template <typename T> struct LinChunk { static constexpr int n = 64; };
template <> struct LinChunk<float> { static constexpr int n = 32; };

struct LinPass {
  const void *a, *b, *c;
  void* out;                           // NULL: this pass is not made
  long a_ld, b_ld, c_ld, o_ld;         // elements from token to token
  int ag, bg, cg, og;                  // value heads to a head of the array
  int Dr, Dc;                          // sizes of a and b, of c and out
  const float* st;                     // entering states, part by part; NULL: zeros
  float* keep;                         // where the parts' states go: LOCAL's, or a copy of st; or NULL
  float* last;                         // the state after the last token, or NULL
  int rs, cs;                          // distances of the rows (Dr) and columns (Dc) of st,
  int krs, kcs;                        // of keep
  int lrs, lcs;                        // and of last
  float wP, wA, wU;
  int e, rev;
  int wide;                            // out is float whatever the call's type
};

struct LinArgs {
  LinPass p[3];
  int T, B, H, Dk, Dv;                 // H: value heads
  int parts, per, npass;               // parts of a row, chunks of a part
  const float* g;
  const int* seq_len;
  int* err;
};

__device__ __forceinline__ int lin_len(const LinArgs& a, int b) {
  const int L = a.seq_len ? a.seq_len[b] : a.T;
  return L < 0 || L > a.T ? 0 : L;
}
// The logarithm of a decay: l^n is 0 in float well before -200, and l^0 stays 1.
__device__ __forceinline__ float lin_log(const float* g, int h) {
  const float x = g[h];
  return x < -200.f ? -200.f : x;
}

// What a decay l = e^x leaves of a state.  Near 1 as S + (l - 1) S, because a rounded l would
// err the same way in every chunk; else as l S, because S + (l - 1) S would leave roundings
// of S itself, and l S may be less than those.
struct LinLeft {
  float f;                             // l - 1 or l
  bool near;
  __device__ __forceinline__ explicit LinLeft(float x) : f(x > -0.69f ? expm1f(x) : expf(x)), near(x > -0.69f) {}
  __device__ __forceinline__ float of(float s) const { return near ? __builtin_fmaf(s, f, s) : s * f; }
};

// Rows in LDS have UP units of 16 bytes, a power of two, and hold unit u at u ^ turn(row):
// 16 lanes that read the same unit of 16 rows, or two units of 8 rows, meet 16 different
// places of the banks.
template <int UP>
__device__ __forceinline__ int lin_turn(int row) {
  if (UP >= 16) return (row & 7) << 1 | (row >> 3 & 1);
  if (UP == 8) return (row >> 1 & 3) << 1 | (row >> 3 & 1);
  return (row >> 2 & 1) << 1 | (row >> 3 & 1);
}

// Operands over 32 of what a product sums over: a lane holds the four of its group hi
// in each of two tiles of 16, the four that an accumulator tile gives it.  So states and
// the chunk's products go from accumulators into the next product as they lie.
//
// The bfloat16 matrix instructions run at sixteen times the rate of the float ones: a
// float operand is the sum of three bfloat16 pieces (24 bits, exactly), a bfloat16 one of
// the call its own piece, and a product takes pieces i and j while i + j <= 2; what is
// dropped is below 2^-24 of the term.  (float32 calls on the float instructions: 8 rows of
// 2048 tokens, 16 heads of 128, 972 us instead of 793.)
// NR: pieces of an operand of the call; CT: rows of it in LDS, a plane for each piece.
template <int NR, int CT>
struct Lin {
  static constexpr int NS = 3;
  struct Raw { uint4 p[NR]; };
  struct Split { uint4 p[NS]; };
  // terms of a product with a float operand, the smallest first
  static constexpr int NP = NR == 1 ? 3 : 6;
  __device__ static constexpr int raw_of(int n) { return NR == 1 ? 0 : n == 0 ? 2 : n == 1 || n == 3 ? 1 : 0; }
  __device__ static constexpr int split_of(int n) { return NR == 1 ? 2 - n : n == 2 ? 2 : n == 1 || n == 4 ? 1 : 0; }

  // Row `row` (16 i + lo), steps k: columns 32 k + 4 hi .. and 16 further on.
  template <int UP>
  __device__ static __forceinline__ Raw rows(const bf16_t* m, int row, int k, int hi) {
    const bf16_t* p = m + row * UP * 8 + 4 * (hi & 1);
    const int u = (hi >> 1) ^ lin_turn<UP>(row);
    Raw r;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const uint2 x = *reinterpret_cast<const uint2*>(p + i * CT * UP * 8 + 8 * (u ^ (4 * k)));
      const uint2 y = *reinterpret_cast<const uint2*>(p + i * CT * UP * 8 + 8 * (u ^ (4 * k + 2)));
      r.p[i] = make_uint4(x.x, x.y, y.x, y.y);
    }
    return r;
  }
  // Rows row0 .. row0 + 31 down column `col` + Q (lo / 4) + lo % 4 (the transposing load
  // takes four rows' fours from 16 lanes).
  template <int UP, int Q>
  __device__ static __forceinline__ Raw cols(const bf16_t* m, int row0, int col, int lo, int hi) {
    typedef __attribute__((ext_vector_type(4))) short s4;
    typedef __attribute__((address_space(3))) s4* lds4;
    const int row = 4 * hi + (lo >> 2), c = col + Q * (lo & 3);
    Raw r;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const bf16_t* at = m + (i * CT + row0 + row) * UP * 8 + 8 * ((c >> 3) ^ lin_turn<UP>(row)) + (c & 7);
      const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)at);
      const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at + 16 * UP * 8));
      const uint2 u = __builtin_bit_cast(uint2, x), v = __builtin_bit_cast(uint2, y);
      r.p[i] = make_uint4(u.x, u.y, v.x, v.y);
    }
    return r;
  }
  // 16 bytes of the call's type, number u of row `row`.
  template <int UP>
  __device__ static __forceinline__ void put_row(bf16_t* m, int row, int u, uint4 x) {
    if constexpr (NR == 1) {
      *reinterpret_cast<uint4*>(m + (row * UP + (u ^ lin_turn<UP>(row))) * 8) = x;
    } else {
      const f32x4 f = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w)};
      split4_store<NR>(f, m + (row * UP + (u >> 1 ^ lin_turn<UP>(row))) * 8 + 4 * (u & 1), CT * UP * 8);
    }
  }
  __device__ static __forceinline__ Split split(f32x4 x, f32x4 y) {
    const float f[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    Split s;
    split8<NS>(f, s.p);
    return s;
  }
  // A float operand in LDS: `half` 0 or 1 of fragment `at` as its four floats say, and the
  // whole of it.
  static constexpr int kHeld = NS * 1024;
  __device__ static __forceinline__ void put(unsigned char* lds, int at, int half, int l, f32x4 x) {
    split4_store<NS>(x, reinterpret_cast<bf16_t*>(lds + at * kHeld + l * 16 + half * 8), 512);
  }
  __device__ static __forceinline__ Split get(const unsigned char* lds, int at, int l) {
    Split s;
#pragma unroll
    for (int i = 0; i < NS; ++i) s.p[i] = ld16(lds + at * kHeld + i * 1024 + l * 16);
    return s;
  }
  __device__ static __forceinline__ void floats(const Raw& r, f32x4& x, f32x4& y) {
    x = y = zero_acc();
#pragma unroll
    for (int n = NR - 1; n >= 0; --n) {
      const uint32_t w[4] = {r.p[n].x, r.p[n].y, r.p[n].z, r.p[n].w};
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const f32x4 f = {__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u), __uint_as_float(w[2 + i] << 16),
                         __uint_as_float(w[2 + i] & 0xffff0000u)};
        x[2 * i] = n == NR - 1 ? f[0] : x[2 * i] + f[0];
        x[2 * i + 1] = n == NR - 1 ? f[1] : x[2 * i + 1] + f[1];
        y[2 * i] = n == NR - 1 ? f[2] : y[2 * i] + f[2];
        y[2 * i + 1] = n == NR - 1 ? f[3] : y[2 * i + 1] + f[3];
      }
    }
  }
  __device__ static __forceinline__ f32x4 mm(const Raw& a, const Raw& b, f32x4 c) {
#pragma unroll
    for (int n = NR == 1 ? 2 : 0; n < NP; ++n) c = mfma(as_frag(a.p[raw_of(n)]), as_frag(b.p[NR == 1 ? 0 : split_of(n)]), c);
    return c;
  }
  // Term n of a product with a float operand: those of different accumulators in turn,
  // because one waits for the one before.
  __device__ static __forceinline__ f32x4 mm(const Raw& a, const Split& b, f32x4 c, int n) {
    return mfma(as_frag(a.p[raw_of(n)]), as_frag(b.p[split_of(n)]), c);
  }
  __device__ static __forceinline__ f32x4 mm(const Split& a, const Raw& b, f32x4 c, int n) {
    return mfma(as_frag(a.p[split_of(n)]), as_frag(b.p[raw_of(n)]), c);
  }
};

// N floats, neighbours, to dst as the call's type or as floats.
template <typename T, int N>
__device__ __forceinline__ void lin_store(void* dst, long at, const float* x, bool wide) {
  if (sizeof(T) == 4 || wide) {
    f32x4* p = reinterpret_cast<f32x4*>(static_cast<float*>(dst) + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) p[i] = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  } else {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack2(x[2 * i], x[2 * i + 1]);
    bf16_t* p = static_cast<bf16_t*>(dst) + at;
    if (N == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[N / 2 - 2], w[N / 2 - 1]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  }
}

// ---------------------------------------------------------------------------
// One part of a row, head and pass, up to 64 NV columns of the state: chunk after chunk.  A
// wave has 16 NV columns of the state in its accumulators, and a share of the chunk's
// products a_i.b_j, which go to the others through LDS as the next product takes them.
// LOCAL: only the state of the part's tokens alone.
// KD: rows of the state in steps of 32.
//
// Bound by the instructions between the products: 64 tokens of a head of 128 x 128 in
// bfloat16 take a compute unit 5.1 us forward and 14 for the three passes of the gradient,
// where their bytes take 3.05 at the rate of a copy; the matrix unit works in 37 % of the
// cycles (one row of 16384 tokens, gradient) and others, a float's pieces first of all, are
// issued in 45 %.  That kernel has all 256 registers of two waves a SIMD and keeps 12 more
// in scratch.  (With two pieces for y's products 4.65; eight waves of 16 columns 6.0; 64
// columns a work-group 6.4; three waves a SIMD keep more there, 8.7.)  One launch
// makes all passes at the widest one's KD and NV: the gradient for heads of 64 x 72 has
// states of 96 x 128, 2.7 times theirs.
// ---------------------------------------------------------------------------
template <typename T, int KD, int NV, bool LOCAL>
__global__ __launch_bounds__(256, 2) void lin_kernel(LinArgs args) {
  constexpr int NR = sizeof(T) == 2 ? 1 : 3, CT = LinChunk<T>::n;
  typedef Lin<NR, CT> L;
  constexpr int NI = CT / 16, NM = CT / 32, NC = 64 * NV, Q = 4 * NV;
  constexpr int E = 16 / sizeof(T);                      // elements of a load's 16 bytes
  constexpr int UP = KD == 3 ? 16 : 4 * KD, UQ = NC / 8;  // units of 8 bfloat16 of a row in LDS
  constexpr int UR = UP * 8 / E, UC = UQ * 8 / E;        // loads of a row
  constexpr int RR = 256 / UR, RC = 256 / UC;            // rows that the work-group loads at once
  constexpr int LR = CT / RR, LC = CT / RC;              // loads of a thread
  __shared__ __align__(16) bf16_t as[LOCAL ? 8 : NR * CT * UP * 8];
  __shared__ __align__(16) bf16_t bs[NR * CT * UP * 8];
  __shared__ __align__(16) bf16_t cs[NR * CT * UQ * 8];
  // the chunk's products a_i.b_j: pairs of tiles (rows 32 j .., columns 16 i ..)
  constexpr int NF = NI == 4 ? 6 : 2;
  auto pair = [](int i, int j) { return i + (i > 2 ? 1 : 0) + j; };   // 0 | 1 | 2 3 | 4 5
  __shared__ __align__(16) unsigned char ps[LOCAL ? 16 : NF * L::kHeld];
  // passes that read the same tokens lie 8 work-groups apart: on one XCD, one after the other
  const int parts = LOCAL ? args.parts - 1 : args.parts;  // nothing follows the last part's own
  const int items = args.B * args.H * parts;
  int id = blockIdx.x;
  const int full = items / 8 * 8 * args.npass;
  int item, which;
  if (id < full) {
    item = id / (8 * args.npass) * 8 + id % 8;
    which = id / 8 % args.npass;
  } else {
    id -= full;
    item = items / 8 * 8 + id % (items % 8);
    which = id / (items % 8);
  }
  const LinPass& p = args.p[which];
  const int part = item % parts, bh = item / parts, h = bh % args.H, b = bh / args.H;
  const int len = lin_len(args, b), per = args.per * CT;
  const int t_lo = part * per, t_hi = min(args.T, t_lo + per);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lo_ = tid & 15, hi_ = tid >> 4 & 3;
  if (!LOCAL && h == 0 && part == 0 && which == 0 && tid == 0 && args.seq_len &&
      (args.seq_len[b] < 0 || args.seq_len[b] > args.T))
    atomicOr(args.err, LL_DEVERR_SEQ_LEN_BIT);
  // token number i of the pass is token len - 1 - i where it runs backwards
  auto token = [&](int i) { return (long)(p.rev ? len - 1 - i : i) * args.B + b; };
  const int cw = 16 * NV * w;                            // the wave's columns; a lane's: cw + 4 NV hi_ + ..
  const int mine = cw + Q * hi_;
  const T* pa = static_cast<const T*>(p.a) + (long)(h / p.ag) * p.Dr;
  const T* pb = static_cast<const T*>(p.b) + (long)(h / p.bg) * p.Dr;
  const T* pc = static_cast<const T*>(p.c) + (long)(h / p.cg) * p.Dc;
  const long oh = (long)(h / p.og) * p.Dc;

  // the state: rows 16 d + 4 hi_ + r, column of tile t: cw + 4 NV (lo_ / 4) + 4 t + lo_ % 4
  f32x4 S[2 * KD][NV];
  const long stride = (long)args.Dk * args.Dv, slot = ((long)bh * args.parts + part) * stride;
  auto each_state = [&](int rs, int cs, auto f) __attribute__((always_inline)) {
    const int c1 = cw + Q * (lo_ >> 2) + (lo_ & 3);
    const long at = (long)(4 * hi_) * rs + (long)c1 * cs;
#pragma unroll
    for (int d = 0; d < 2 * KD; ++d)
#pragma unroll
      for (int t = 0; t < NV; ++t)
        f(S[d][t], at + 16l * d * rs + 4l * t * cs, 16 * d + 4 * hi_ < p.Dr && c1 + 4 * t < p.Dc);
  };
  each_state(p.rs, p.cs, [&](f32x4& s, long at, bool in) __attribute__((always_inline)) {
    s = zero_acc();
    if (LOCAL || !p.st || !in) return;
    const float* x = p.st + slot + at;
    if (p.rs == 1) s = *reinterpret_cast<const f32x4*>(x);
    else s = f32x4{x[0], x[p.rs], x[2l * p.rs], x[3l * p.rs]};
  });
  auto put_state = [&](float* to, int rs, int cs) __attribute__((always_inline)) {
    each_state(rs, cs, [&](f32x4& s, long at, bool in) __attribute__((always_inline)) {
      if (!in) return;
      float* x = to + at;
      if (rs == 1) {
        *reinterpret_cast<f32x4*>(x) = s;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[(long)e * rs] = s[e];
      }
    });
  };
  if (!LOCAL && p.keep) put_state(p.keep + slot, p.krs, p.kcs);

  // (what lies above the diagonal in a pair's second tile stays zero)
  if constexpr (!LOCAL)
    for (int i = tid; i < NF * L::kHeld / 16; i += 256) reinterpret_cast<uint4*>(ps)[i] = zero4();
  const float g = lin_log(args.g, h);
  // weights: of pairs on the diagonal tiles, of pairs one tile apart (more apart: times
  // l^16 each), of a token's place in its tile, and of what a full chunk's tokens leave
  f32x4 near, far, leave;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int d = lo_ - 4 * hi_ - r;
    near[r] = d < 0 ? 0.f : p.wP * expf(g * d);
    far[r] = p.wP * expf(g * (16 + d));
    leave[r] = p.wU * expf(g * (16 - 4 * hi_ - r - p.e));
  }
  const float place = p.wA * expf(g * (lo_ + p.e));
  float l16[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) l16[i] = uniform(expf(g * (16 * i)));

  // where this thread loads from: rows ur + RR i of a and b, uc + RC i of c, 16 bytes each
  const int ur_ = tid / UR, ux_ = tid % UR, uc_ = tid / UC, cx_ = tid % UC;
  const long dir = p.rev ? -args.B : args.B;
  const long tok0 = token(0), ahead = tok0 + dir * t_lo;
  const bool in_r = ux_ * E < p.Dr, in_c = cx_ * E < p.Dc;
  const T* la = pa + (ahead + dir * ur_) * p.a_ld + ux_ * E;
  const T* lb = pb + (ahead + dir * ur_) * p.b_ld + ux_ * E;
  const T* lc = pc + (ahead + dir * uc_) * p.c_ld + cx_ * E;
  LinLeft left_all(g * CT);
  left_all.f = uniform(left_all.f);
  uint4 ra[LR], rb[LR], rc[LC];
#pragma unroll
  for (int i = 0; i < LR; ++i) ra[i] = rb[i] = zero4();
#pragma unroll
  for (int i = 0; i < LC; ++i) rc[i] = zero4();
  // (columns past the operand's stay the zeros that they are)
  auto load = [&](int t0, int ur, int uc) __attribute__((always_inline)) {
    if (t0 + CT <= len) {
      if (in_r) {
#pragma unroll
        for (int i = 0; i < LR; ++i) {
          if (!LOCAL) ra[i] = ld16(la + dir * RR * i * p.a_ld);
          rb[i] = ld16(lb + dir * RR * i * p.b_ld);
        }
      }
      if (in_c) {
#pragma unroll
        for (int i = 0; i < LC; ++i) rc[i] = ld16(lc + dir * RC * i * p.c_ld);
      }
    } else {
#pragma unroll
      for (int i = 0; i < LR; ++i) {
        const bool in = t0 + ur + RR * i < len && in_r;
        if (!LOCAL) ra[i] = in ? ld16(la + dir * RR * i * p.a_ld) : zero4();
        rb[i] = in ? ld16(lb + dir * RR * i * p.b_ld) : zero4();
      }
#pragma unroll
      for (int i = 0; i < LC; ++i) rc[i] = t0 + uc + RC * i < len && in_c ? ld16(lc + dir * RC * i * p.c_ld) : zero4();
    }
    la += dir * CT * p.a_ld;
    lb += dir * CT * p.b_ld;
    lc += dir * CT * p.c_ld;
  };
  long out_at = (ahead + dir * lo_) * p.o_ld + oh + mine;
  const int t_end = min(t_hi, len);
  if (t_lo < t_end) load(t_lo, ur_, uc_);
  for (int t0 = t_lo; t0 < t_end; t0 += CT) {
    // the places in LDS are made anew for every chunk: kept, they and the weights' products
    // would not fit the registers, and a reload from scratch waits for the chunk's loads
    int me = tid;
    asm volatile("" : "+v"(me));
    const int l = me & 63, lo = me & 15, hi = me >> 4 & 3, ur = me / UR, ux = me % UR, uc = me / UC, cx = me % UC;
#pragma unroll
    for (int r = 0; r < 4; ++r) asm volatile("" : "+v"(leave[r]));
    lds_barrier();                                       // the chunk before has been read
#pragma unroll
    for (int i = 0; i < LR; ++i) {
      if (!LOCAL) L::template put_row<UP>(as, ur + RR * i, ux, ra[i]);
      L::template put_row<UP>(bs, ur + RR * i, ux, rb[i]);
    }
#pragma unroll
    for (int i = 0; i < LC; ++i) L::template put_row<UQ>(cs, uc + RC * i, cx, rc[i]);
    lds_barrier();
    if (LOCAL && t0 + CT < t_end) load(t0 + CT, ur, uc);
    const int m = min(CT, len - t0);
    if constexpr (!LOCAL) {
      // the chunk's products, tiles of 16 x 16 (rows j, columns i >= j) a wave in turn
      constexpr int NT = NI * (NI + 1) / 2, PT = (NT + 3) / 4;
      int ti[PT], tj[PT];
      f32x4 x[PT];
#pragma unroll
      for (int n = 0; n < PT; ++n) {
        const int at = min(w + 4 * n, NT - 1);
        ti[n] = at >= 6 ? 3 : at >= 3 ? 2 : at >= 1 ? 1 : 0;
        tj[n] = at - ti[n] * (ti[n] + 1) / 2;
        x[n] = zero_acc();
      }
#pragma unroll
      for (int k = 0; k < KD; ++k)
#pragma unroll
        for (int n = 0; n < PT; ++n)
          x[n] = L::mm(L::template rows<UP>(bs, 16 * tj[n] + lo, k, hi), L::template rows<UP>(as, 16 * ti[n] + lo, k, hi), x[n]);
#pragma unroll
      for (int n = 0; n < PT; ++n) {
        const int d = ti[n] - tj[n];
        const float f = d > 2 ? l16[2] : d > 1 ? l16[1] : 1.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float on = lo >= 4 * hi + r ? x[n][r] * near[r] : 0.f, off = x[n][r] * (far[r] * f);
          x[n][r] = d == 0 ? on : off;
        }
        if (w + 4 * n < NT) L::put(ps, pair(ti[n], tj[n] / 2), tj[n] & 1, l, x[n]);
      }
      f32x4 y[NI][NV];
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int t = 0; t < NV; ++t) y[i][t] = zero_acc();
#pragma unroll
      for (int k = 0; k < KD; ++k) {
        typename L::Split s[NV];
#pragma unroll
        for (int t = 0; t < NV; ++t) s[t] = L::split(S[2 * k][t], S[2 * k + 1][t]);
        typename L::Raw fa[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) fa[i] = L::template rows<UP>(as, 16 * i + lo, k, hi);
#pragma unroll
        for (int n = 0; n < L::NP; ++n)
#pragma unroll
          for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int t = 0; t < NV; ++t) y[i][t] = L::mm(s[t], fa[i], y[i][t], n);
      }
      lds_barrier();                                     // the products are there
      if (t0 + CT < t_end) load(t0 + CT, ur, uc);
      typename L::Raw cf[NM][NV];
#pragma unroll
      for (int j = 0; j < NM; ++j)
#pragma unroll
        for (int t = 0; t < NV; ++t) cf[j][t] = L::template cols<UQ, Q>(cs, 32 * j, 16 * NV * w + 4 * t, lo, hi);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const float f = place * l16[i];
#pragma unroll
        for (int t = 0; t < NV; ++t) y[i][t] *= f;
#pragma unroll
        for (int j = 0; j <= i / 2; ++j) {
          const typename L::Split s = L::get(ps, pair(i, j), l);
#pragma unroll
          for (int n = 0; n < L::NP; ++n)
#pragma unroll
            for (int t = 0; t < NV; ++t) y[i][t] = L::mm(cf[j][t], s, y[i][t], n);
        }
      }
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (16 * i + lo < m && mine < p.Dc) {
          float o[4 * NV];
#pragma unroll
          for (int t = 0; t < NV; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[4 * t + r] = y[i][t][r];
          lin_store<T, 4 * NV>(p.out, out_at + dir * 16 * i * p.o_ld, o, p.wide);
        }
      }
      out_at += dir * CT * p.o_ld;
    }
    // S' = l^m S + ..
    // (LOCAL: from zero, so every token's weight is what the part's end leaves of it)
    f32x4 wt[NI];
    const float after = LOCAL ? uniform(expf(g * max(0, t_end - t0 - CT))) : 1.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) wt[i] = leave * (l16[NI - 1 - i] * after);
    LinLeft left = left_all;
    if (m != CT) {
      left = LinLeft(g * m);
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)                      // (tokens past the end are zeros)
          wt[i][r] = p.wU * expf(g * max(0, m - 16 * i - 4 * hi - r - p.e));
    }
    if (!LOCAL) {
      auto each = [&](auto f) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < 2 * KD; ++d)
#pragma unroll
          for (int t = 0; t < NV; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[d][t][r] = f(S[d][t][r]);
      };
      if (left.near) each([&](float x) { return __builtin_fmaf(x, left.f, x); });
      else each([&](float x) { return x * left.f; });
    }
#pragma unroll
    for (int j = 0; j < NM; ++j) {
      typename L::Split cv[NV];
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        f32x4 x, y;
        L::floats(L::template cols<UQ, Q>(cs, 32 * j, 16 * NV * w + 4 * t, lo, hi), x, y);
        cv[t] = L::split(x * wt[2 * j], y * wt[2 * j + 1]);
      }
#pragma unroll
      for (int d = 0; d < 2 * KD; d += 2) {
        typename L::Raw f[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) f[e] = L::template cols<UP, 4>(bs, 32 * j, 16 * (d + e), lo, hi);
#pragma unroll
        for (int n = 0; n < L::NP; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int t = 0; t < NV; ++t) S[d + e][t] = L::mm(f[e], cv[t], S[d + e][t], n);
      }
    }
  }
  if constexpr (LOCAL) {
    put_state(p.keep + slot, p.krs, p.kcs);
  } else {
    // tokens past the row's end
    if (mine < p.Dc) {
      const float zero[4 * NV] = {};
      for (int t = max(t_lo, len) + lo_; t < t_hi; t += 16)
        lin_store<T, 4 * NV>(p.out, ((long)t * args.B + b) * p.o_ld + oh + mine, zero, p.wide);
    }
    // the part that holds the last token has the last state (the first one of an empty row)
    if (p.last && (part == 0 || t_lo < len) && t_lo + per >= len) put_state(p.last + bh * stride, p.lrs, p.lcs);
  }
}

// The parts' states from their tokens' own: E_0 as given, E_{p+1} = l^n E_p + local_p.  They
// lie as [Dv][Dk], S0 as [Dk][Dv].  Bound by the states' bytes, in and out: 64 heads of
// 8 parts of 128 x 128, 67 MB, in 10.9 us, 6.2 TB/s.
__global__ __launch_bounds__(256) void lin_scan_kernel(LinArgs a, float* states, const float* S0, int chunk) {
  const long size = (long)a.Dk * a.Dv;
  const int blocks = (int)((size / 4 + 255) / 256);
  const int bh = blockIdx.x / blocks;
  const long at = ((long)(blockIdx.x % blocks) * 256 + threadIdx.x) * 4;
  if (at >= size) return;
  const int len = lin_len(a, bh / a.H), per = a.per * chunk;
  const float g = lin_log(a.g, bh % a.H);
  f32x4 e = zero_acc();
  if (S0) {
    const float* x = S0 + bh * size + at % a.Dk * a.Dv + at / a.Dk;
    e = f32x4{x[0], x[a.Dv], x[2l * a.Dv], x[3l * a.Dv]};
  }
  float* st = states + (long)bh * a.parts * size + at;
  constexpr int R = 4;                                   // parts read at once
  for (int p = 0; p < a.parts; p += R) {
    f32x4 own[R];
#pragma unroll
    for (int i = 0; i < R; ++i)
      own[i] = p + i < a.parts - 1 ? *reinterpret_cast<const f32x4*>(st + (p + i) * size) : zero_acc();
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (p + i >= a.parts) break;
      *reinterpret_cast<f32x4*>(st + (p + i) * size) = e;
      const LinLeft left(g * min(per, max(0, len - (p + i) * per)));
#pragma unroll
      for (int r = 0; r < 4; ++r) e[r] = left.of(e[r]) + own[i][r];
    }
  }
}

// Sums over the r value heads that share a key head: two gradients of a token, [Hk r][D]
// floats each, to [Hk][D] of the call's type, in the heads' order.  Bound by its bytes:
// 6400 tokens of 8 heads of 64 floats, two arrays, 39 MB in 6.8 us.
struct LinSum {
  const float* from[2];
  void* to[2];
  long ld[2];
  long tokens;
  int Hk, r, D;
};
template <typename T>
__global__ __launch_bounds__(256) void lin_sum_kernel(LinSum a) {
  const int per = a.Hk * a.D / 4;                        // groups of four of a token
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const long tok = i / per;
  if (tok >= a.tokens) return;
  const int u = (int)(i % per) * 4, h = u / a.D, c = u % a.D;
  const float* x = a.from[blockIdx.y] + (tok * a.Hk + h) * a.r * a.D + c;
  f32x4 s = *reinterpret_cast<const f32x4*>(x);
  for (int j = 1; j < a.r; ++j) s += *reinterpret_cast<const f32x4*>(x + (long)j * a.D);
  const float o[4] = {s[0], s[1], s[2], s[3]};
  lin_store<T, 4>(a.to[blockIdx.y], tok * a.ld[blockIdx.y] + u, o, false);
}

// One token.  A work-group has 32 columns of one head's state: thread (row group tid / 8,
// column group tid % 8) holds rows r, r + 32, .. and four columns of them.  Bound by the
// state, read and written: 256 rows of 32 heads of 128 x 128, 1.07 GB, in 222 us, 4.8 TB/s;
// 4 rows of 4 heads of 32 x 32 take 3.7 us, a launch's time.
struct LinStepArgs {
  int B, Hk, H, Dk, Dv, n_slots;
  float scale;
  long q_ld, k_ld, v_ld;
  const void *q, *k, *v;
  const float* g;
  float* S;
  const int* slots;
  void* y;
  int* err;
};

template <typename T>
__global__ __launch_bounds__(256) void lin_step_kernel(LinStepArgs a) {
  __shared__ float4 red[4][8];
  const int ntile = (a.Dv + kLinStepCols - 1) / kLinStepCols;
  const int ct = blockIdx.x % ntile, bh = blockIdx.x / ntile;
  const int b = bh / a.H, h = bh % a.H, hk = h / (a.H / a.Hk);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  const int c = ct * kLinStepCols + (tid & 7) * 4, r0 = tid >> 3;
  const bool in = c < a.Dv;                              // Dv is a multiple of 8: all four columns or none
  const long yat = ((long)b * a.H + h) * a.Dv + c;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    const float zero[4] = {};
    if (in && r0 == 0) lin_store<T, 4>(a.y, yat, zero, false);
    if ((slot < -1 || slot >= a.n_slots) && a.err && h == 0 && ct == 0 && tid == 0) atomicOr(a.err, LL_DEVERR_SLOT);
    return;
  }
  const T* k = static_cast<const T*>(a.k) + b * a.k_ld + (long)hk * a.Dk;
  const T* q = static_cast<const T*>(a.q) + b * a.q_ld + (long)hk * a.Dk;
  const T* v = static_cast<const T*>(a.v) + b * a.v_ld + (long)h * a.Dv + c;
  float* S = a.S + ((long)slot * a.H + h) * a.Dk * a.Dv + c;
  const LinLeft left(lin_log(a.g, h));
  f32x4 s[4];
  float kd[4], qd[4], vc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = r0 + 32 * i;
    const bool has = in && d < a.Dk;
    s[i] = has ? *reinterpret_cast<const f32x4*>(S + (long)d * a.Dv) : zero_acc();
    kd[i] = has ? Op<T>::to_f32(k[d]) : 0.f;
    qd[i] = has ? Op<T>::to_f32(q[d]) : 0.f;
    vc[i] = in ? Op<T>::to_f32(v[i]) : 0.f;
  }
  f32x4 o = zero_acc();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = r0 + 32 * i;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[i][e] = __builtin_fmaf(kd[i], vc[e], left.of(s[i][e]));
      o[e] = __builtin_fmaf(qd[i], s[i][e], o[e]);
    }
    if (in && d < a.Dk) *reinterpret_cast<f32x4*>(S + (long)d * a.Dv) = s[i];
  }
#pragma unroll
  for (int m = 8; m < 64; m <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], m, 64);
  if (l < 8) red[w][l] = make_float4(o[0], o[1], o[2], o[3]);
  __syncthreads();
  if (in && r0 == 0) {
    const float4 x = red[0][tid], y = red[1][tid], z = red[2][tid], u = red[3][tid];
    const float f[4] = {a.scale * ((x.x + y.x) + (z.x + u.x)), a.scale * ((x.y + y.y) + (z.y + u.y)),
                        a.scale * ((x.z + y.z) + (z.z + u.z)), a.scale * ((x.w + y.w) + (z.w + u.w))};
    lin_store<T, 4>(a.y, yat, f, false);
  }
}

}  // namespace ll

struct ll_linattn_plan {
  ll_linattn_desc d;
  int device = 0, cus = 0;
  ll::LinArgs a{};                     // sizes and the error word
  long ld[6] = {};                     // q, k, v, dq, dk, dv
  float scale = 0.f;
  float *st = nullptr, *dst = nullptr, *wide = nullptr;
  int64_t bytes = 0;
  bool saved = false, has_state = false;
  const void *q = nullptr, *k = nullptr, *v = nullptr;
  const float* g = nullptr;
  const int* seq_len = nullptr;
  long saved_ld[3] = {};
};

namespace {

ll_status validate(const ll_linattn_desc* d, bool step) {
  if (!d) return fail(LL_EINVAL, "desc is NULL");
  if (d->T_max < 1 || d->B < 1 || d->Hk < 1 || d->Hv < 1 || d->Dk < 1 || d->Dv < 1)
    return fail(LL_EINVAL, "T_max, B, Hk, Hv, Dk and Dv must be at least 1 (got %d, %d, %d, %d, %d, %d)",
                d->T_max, d->B, d->Hk, d->Hv, d->Dk, d->Dv);
  if (step && d->T_max != 1) return fail(LL_EINVAL, "the step takes one token: T_max must be 1 (got %d)", d->T_max);
  if (d->dtype != LL_F32 && d->dtype != LL_BF16) return fail(LL_EINVAL, "dtype must be LL_F32 or LL_BF16");
  if (d->Hv % d->Hk) return fail(LL_EINVAL, "Hv = %d is not a multiple of Hk = %d", d->Hv, d->Hk);
  if (d->reserved) return fail(LL_EINVAL, "reserved must be 0");
  if (!std::isfinite(d->scale)) return fail(LL_EINVAL, "scale is not finite");
  if (d->Dk % 8 || d->Dv % 8 || d->Dk > ll::kLinMaxD || d->Dv > ll::kLinMaxD)
    return fail(LL_EUNSUPPORTED, "Dk = %d and Dv = %d must be multiples of 8, at most %d", d->Dk, d->Dv, ll::kLinMaxD);
  const int es = d->dtype == LL_BF16 ? 2 : 4;
  const int64_t qk = (int64_t)d->Hk * d->Dk, v = (int64_t)d->Hv * d->Dv;
  const int64_t ld[6] = {d->q_ld, d->k_ld, d->v_ld, d->dq_ld, d->dk_ld, d->dv_ld};
  const int64_t need[6] = {qk, qk, v, qk, qk, v};
  const char* names[6] = {"q_ld", "k_ld", "v_ld", "dq_ld", "dk_ld", "dv_ld"};
  for (int i = 0; i < (step ? 3 : 6); ++i)
    if (ld[i] && (ld[i] < need[i] || ld[i] * es % 16 || ld[i] > (int64_t)1 << 31))
      return fail(LL_EINVAL, "%s = %lld must be 0, or at least %lld, at most 2^31 and a multiple of 16 bytes",
                  names[i], (long long)ld[i], (long long)need[i]);
  if (d->T_max > 1 << 30) return fail(LL_EUNSUPPORTED, "T_max = %d is more than 2^30", d->T_max);
  // work-groups: three passes of each head and part (rows have parts only where heads are
  // few); the step's column tiles
  const int64_t heads = (int64_t)d->B * d->Hv;
  const int64_t groups = heads * (step ? (d->Dv + ll::kLinStepCols - 1) / ll::kLinStepCols : 3);
  const int64_t most = ll::max_groups(256);
  if (heads >= 1 << (step ? 24 : 22) || groups > most)
    return fail(LL_EUNSUPPORTED, "B * Hv = %lld: %lld work-groups, a launch holds %lld", (long long)heads,
                (long long)groups, (long long)most);
  if (!step && (int64_t)d->T_max * d->B * qk / 4 > most * 256)
    return fail(LL_EUNSUPPORTED, "T_max * B * Hk * Dk = %lld is too large for one launch",
                (long long)d->T_max * d->B * (long long)qk);
  return LL_OK;
}

void distances(ll_linattn_plan* p) {
  const ll_linattn_desc& d = p->d;
  const long qk = (long)d.Hk * d.Dk, v = (long)d.Hv * d.Dv;
  p->ld[0] = d.q_ld ? d.q_ld : qk;
  p->ld[1] = d.k_ld ? d.k_ld : qk;
  p->ld[2] = d.v_ld ? d.v_ld : v;
  p->ld[3] = d.dq_ld ? d.dq_ld : qk;
  p->ld[4] = d.dk_ld ? d.dk_ld : qk;
  p->ld[5] = d.dv_ld ? d.dv_ld : v;
}

float scale_of(const ll_linattn_desc& d) { return d.scale != 0.f ? d.scale : (float)(1.0 / std::sqrt((double)d.Dk)); }
int chunk_of(const ll_linattn_desc& d) { return d.dtype == LL_BF16 ? ll::LinChunk<bf16_t>::n : ll::LinChunk<float>::n; }

void release(ll_linattn_plan* p) {
  void* all[] = {p->st, p->dst, p->wide, p->a.err};
  for (void* m : all)
    if (m) (void)hipFree(m);
}

template <typename T, int KD>
void launch(const ll::LinArgs& a, int nv, bool local, unsigned grid, hipStream_t s) {
  if (local) {
    if (nv == 1) ll::lin_kernel<T, KD, 1, true><<<dim3(grid), dim3(256), 0, s>>>(a);
    else ll::lin_kernel<T, KD, 2, true><<<dim3(grid), dim3(256), 0, s>>>(a);
  } else {
    if (nv == 1) ll::lin_kernel<T, KD, 1, false><<<dim3(grid), dim3(256), 0, s>>>(a);
    else ll::lin_kernel<T, KD, 2, false><<<dim3(grid), dim3(256), 0, s>>>(a);
  }
}

// The passes a.p[0 .. npass) over all parts.
hipError_t launch_passes(ll::LinArgs a, bool bf16, bool local, hipStream_t s) {
  int dr = 0, dc = 0;
  for (int i = 0; i < a.npass; ++i) {
    dr = std::max(dr, a.p[i].Dr);
    dc = std::max(dc, a.p[i].Dc);
  }
  const int nv = dc > 64 ? 2 : 1;
  const unsigned grid = (unsigned)a.B * a.H * (local ? a.parts - 1 : a.parts) * a.npass;
  const int kd = (dr + 31) / 32;
  if (bf16) {
    if (kd == 1) launch<bf16_t, 1>(a, nv, local, grid, s);
    else if (kd == 2) launch<bf16_t, 2>(a, nv, local, grid, s);
    else if (kd == 3) launch<bf16_t, 3>(a, nv, local, grid, s);
    else launch<bf16_t, 4>(a, nv, local, grid, s);
  } else {
    if (kd == 1) launch<float, 1>(a, nv, local, grid, s);
    else if (kd == 2) launch<float, 2>(a, nv, local, grid, s);
    else if (kd == 3) launch<float, 3>(a, nv, local, grid, s);
    else launch<float, 4>(a, nv, local, grid, s);
  }
  return hipGetLastError();
}

// The parts' entering states into `to` from the first one; a.p[0] says what makes them.
hipError_t launch_states(ll::LinArgs a, float* to, const float* first, bool bf16, int chunk, hipStream_t s) {
  a.p[0].keep = to;
  a.p[0].krs = 1;
  a.p[0].kcs = a.Dk;
  a.npass = 1;
  if (hipError_t e = launch_passes(a, bf16, true, s); e != hipSuccess) return e;
  const long blocks = ((long)a.Dk * a.Dv / 4 + 255) / 256;
  ll::lin_scan_kernel<<<dim3((unsigned)(blocks * a.B * a.H)), dim3(256), 0, s>>>(a, to, first, chunk);
  return hipGetLastError();
}

}  // namespace

extern "C" {

ll_status ll_linattn_plan_create(const ll_linattn_desc* desc, int device, ll_linattn_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  LL_STATUS(validate(desc, false));
  LL_STATUS(ll::check_device(device));
  ll::DeviceGuard guard(device);
  ll_linattn_plan* p = new (std::nothrow) ll_linattn_plan();
  if (!p) return fail(LL_ENOMEM, "host allocation of the plan failed");
  p->d = *desc;
  p->device = device;
  distances(p);
  p->scale = scale_of(*desc);
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, device) != hipSuccess) {
    delete p;
    return fail(LL_EHIP, "hipGetDeviceProperties failed");
  }
  p->cus = prop.multiProcessorCount;
  ll::LinArgs& a = p->a;
  a.T = desc->T_max; a.B = desc->B; a.H = desc->Hv; a.Dk = desc->Dk; a.Dv = desc->Dv;
  const int chunk = chunk_of(*desc), nch = (desc->T_max + chunk - 1) / chunk;
  const long heads = (long)desc->B * desc->Hv;
  // Parts of a row: two work-groups for a compute unit, as many as it holds, two chunks each
  // at least; short rows stay whole, because two launches make the parts' states.  (8 rows of 256 to
  // 2048 tokens, 16 heads, training: 1 part 444 us, 4 381, 5 353, 8 433; one row of 16384:
  // 16 parts 447, 32 423, 37 487, 64 494; 64 rows of 100, 8 heads, float32: 1 107, 2 182.)
  const int want = nch < 8 ? 1 : (int)std::max(1L, std::min(2L * p->cus / heads, nch / 2L));
  a.per = (nch + want - 1) / want;
  a.parts = (nch + a.per - 1) / a.per;
  const size_t st = sizeof(float) * heads * a.parts * desc->Dk * desc->Dv;
  const size_t wide = sizeof(float) * 2 * (size_t)desc->T_max * heads * desc->Dk;
  const bool train = !desc->inference;
  struct { void** at; size_t bytes; const char* what; bool want; } bufs[] = {
      {(void**)&p->st, st, "the parts' states", train || a.parts > 1},
      {(void**)&p->dst, st, "the gradients of the parts' states", train && a.parts > 1},
      {(void**)&p->wide, wide, "the heads' gradients of q and k", train && desc->Hv > desc->Hk},
      {(void**)&a.err, sizeof(int), "the error word", true},
  };
  ll_status status = LL_OK;
  for (auto& b : bufs)
    if (b.want && status == LL_OK) {
      status = ll::dalloc(b.at, b.bytes, b.what);
      p->bytes += (int64_t)b.bytes;
    }
  if (status == LL_OK && hipMemset(a.err, 0, sizeof(int)) != hipSuccess)
    status = fail(LL_EHIP, "hipMemset of the error word failed");
  if (status == LL_OK) status = ll::wait_created();
  if (status != LL_OK) {
    release(p);
    delete p;
    return status;
  }
  *out = p;
  return LL_OK;
}

ll_status ll_linattn_plan_destroy(ll_linattn_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_linattn_plan_bytes(const ll_linattn_plan* p, int64_t* device_bytes) {
  if (!p || !device_bytes) return fail(LL_EINVAL, "plan and device_bytes are required");
  *device_bytes = p->bytes;
  return LL_OK;
}

ll_status ll_linattn_plan_set_ld(ll_linattn_plan* p, const int64_t* ld) {
  if (!p || !ld) return fail(LL_EINVAL, "plan and ld are required");
  ll_linattn_desc d = p->d;
  d.q_ld = ld[0]; d.k_ld = ld[1]; d.v_ld = ld[2]; d.dq_ld = ld[3]; d.dk_ld = ld[4]; d.dv_ld = ld[5];
  LL_STATUS(validate(&d, false));
  p->d = d;
  distances(p);
  return LL_OK;
}

ll_status linattn_loop_fwd(ll_linattn_plan* p, void* stream, const void* q, const void* k, const void* v,
                           const float* g, const int32_t* seq_len, const float* S0, void* y, float* ST,
                           int32_t save_for_backward) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (!q || !k || !v || !g || !y) return fail(LL_EINVAL, "q, k, v, g and y are required");
  if (save_for_backward && p->d.inference)
    return fail(LL_EINVAL, "the plan was created for inference: it keeps nothing for the gradient");
  LL_ALIGNED(q, 16); LL_ALIGNED(k, 16); LL_ALIGNED(v, 16); LL_ALIGNED(y, 16); LL_ALIGNED(S0, 16); LL_ALIGNED(ST, 16);
  LL_ALIGNED(g, 4); LL_ALIGNED(seq_len, 4);
  ll::DeviceGuard guard(p->device);
  const ll_linattn_desc& d = p->d;
  const int r = d.Hv / d.Hk;
  ll::LinArgs a = p->a;
  a.g = g; a.seq_len = seq_len; a.npass = 1;
  ll::LinPass& f = a.p[0];
  f.a = q; f.b = k; f.c = v; f.out = y;
  f.a_ld = p->ld[0]; f.b_ld = p->ld[1]; f.c_ld = p->ld[2]; f.o_ld = (long)d.Hv * d.Dv;
  f.ag = f.bg = r; f.cg = f.og = 1;
  f.Dr = d.Dk; f.Dc = d.Dv; f.lrs = d.Dv; f.lcs = 1;
  f.wP = f.wA = p->scale; f.wU = 1.f; f.e = 1;
  f.last = ST;
  p->saved = false;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool bf16 = d.dtype == LL_BF16;
  if (a.parts > 1) {
    LL_HIP(launch_states(a, p->st, S0, bf16, chunk_of(d), s));
    f.st = p->st; f.rs = 1; f.cs = d.Dk;
  } else {
    f.st = S0; f.rs = d.Dv; f.cs = 1;
    f.keep = save_for_backward && S0 ? p->st : nullptr;
    f.krs = 1; f.kcs = d.Dk;
  }
  LL_HIP(launch_passes(a, bf16, false, s));
  if (save_for_backward) {
    p->saved = true;
    p->has_state = f.st != nullptr;
    p->q = q; p->k = k; p->v = v; p->g = g; p->seq_len = seq_len;
    for (int i = 0; i < 3; ++i) p->saved_ld[i] = p->ld[i];
  }
  return LL_OK;
}

ll_status linattn_loop_bwd(ll_linattn_plan* p, void* stream, const void* q, const void* k, const void* v,
                           const float* g, const int32_t* seq_len, const void* dy, const float* dST, void* dq,
                           void* dk, void* dv, float* dS0) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (!p->saved)
    return fail(LL_ESTATE, "no saved forward on this plan (call linattn_loop_fwd with save_for_backward=1 first)");
  for (int i = 0; i < 3; ++i)
    if (p->ld[i] != p->saved_ld[i])
      return fail(LL_ESTATE, "the saved forward's q, k or v had their tokens at other distances than the plan now");
  if (q != p->q || k != p->k || v != p->v || g != p->g || seq_len != p->seq_len)
    return fail(LL_EINVAL, "q, k, v, g or seq_len differs from the saved forward's");
  if (!dy || !dq || !dk || !dv) return fail(LL_EINVAL, "dy, dq, dk and dv are required");
  if (dS0 && dS0 == dST) return fail(LL_EINVAL, "dS0 must be another array than dST");
  LL_ALIGNED(dy, 16); LL_ALIGNED(dST, 16); LL_ALIGNED(dq, 16); LL_ALIGNED(dk, 16); LL_ALIGNED(dv, 16);
  LL_ALIGNED(dS0, 16);
  ll::DeviceGuard guard(p->device);
  const ll_linattn_desc& d = p->d;
  const int r = d.Hv / d.Hk;
  const bool bf16 = d.dtype == LL_BF16;
  const long qw = (long)d.Hv * d.Dk, y_ld = (long)d.Hv * d.Dv;
  ll::LinArgs a = p->a;
  a.g = g; a.seq_len = seq_len;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  p->saved = false;
  float* wide_k = p->wide ? p->wide + (long)d.T_max * d.B * qw : nullptr;
  ll::LinPass v_, q_, k_;
  v_ = ll::LinPass{};
  v_.a = k; v_.b = q; v_.c = dy; v_.out = dv;
  v_.a_ld = p->ld[1]; v_.b_ld = p->ld[0]; v_.c_ld = y_ld; v_.o_ld = p->ld[5];
  v_.ag = v_.bg = r; v_.cg = v_.og = 1;
  v_.Dr = d.Dk; v_.Dc = d.Dv; v_.lrs = d.Dv; v_.lcs = 1;
  v_.wP = v_.wU = p->scale; v_.wA = 1.f; v_.e = 0; v_.rev = 1;
  v_.last = dS0;
  v_.st = dST; v_.rs = d.Dv; v_.cs = 1;
  if (a.parts > 1) {
    a.p[0] = v_;
    LL_HIP(launch_states(a, p->dst, dST, bf16, chunk_of(d), s));
    v_.st = p->dst; v_.rs = 1; v_.cs = d.Dk;
  }
  k_ = v_;
  k_.a = v; k_.b = dy; k_.c = q;
  k_.a_ld = p->ld[2]; k_.b_ld = y_ld; k_.c_ld = p->ld[0];
  k_.ag = k_.bg = 1; k_.cg = r;
  k_.Dr = d.Dv; k_.Dc = d.Dk;
  std::swap(k_.rs, k_.cs);
  k_.last = nullptr;
  k_.out = r > 1 ? wide_k : dk; k_.o_ld = r > 1 ? qw : p->ld[4]; k_.og = 1; k_.wide = r > 1;
  q_ = k_;
  q_.a = dy; q_.b = v; q_.c = k;
  q_.a_ld = y_ld; q_.b_ld = p->ld[2]; q_.c_ld = p->ld[1];
  q_.wP = q_.wA = p->scale; q_.wU = 1.f; q_.e = 1; q_.rev = 0;
  q_.st = p->has_state ? p->st : nullptr; q_.rs = d.Dk; q_.cs = 1;
  q_.out = r > 1 ? p->wide : dq; q_.o_ld = r > 1 ? qw : p->ld[3];
  a.p[0] = v_; a.p[1] = k_; a.p[2] = q_;
  a.npass = 3;
  LL_HIP(launch_passes(a, bf16, false, s));
  if (r > 1) {
    ll::LinSum m{};
    m.from[0] = p->wide; m.from[1] = wide_k;
    m.to[0] = dq; m.to[1] = dk;
    m.ld[0] = p->ld[3]; m.ld[1] = p->ld[4];
    m.tokens = (long)d.T_max * d.B;
    m.Hk = d.Hk; m.r = r; m.D = d.Dk;
    const dim3 grid((unsigned)((m.tokens * (d.Hk * d.Dk / 4) + 255) / 256), 2);
    if (bf16) ll::lin_sum_kernel<bf16_t><<<grid, dim3(256), 0, s>>>(m);
    else ll::lin_sum_kernel<float><<<grid, dim3(256), 0, s>>>(m);
    LL_HIP(hipGetLastError());
  }
  return LL_OK;
}

ll_status ll_linattn_status_sync(ll_linattn_plan* p, int32_t* device_error) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  ll::DeviceGuard guard(p->device);
  return ll::read_error_word(p->a.err, device_error);
}

ll_status linattn_loop_step(const ll_linattn_desc* desc, void* stream, const void* q, const void* k, const void* v,
                            const float* g, float* S, const int32_t* slots, int32_t n_slots, void* y,
                            int32_t* device_error) {
  LL_STATUS(validate(desc, true));
  if (!q || !k || !v || !g || !S || !y) return fail(LL_EINVAL, "q, k, v, g, S and y are required");
  if (n_slots < 1 || (!slots && n_slots < desc->B))
    return fail(LL_EINVAL, "n_slots = %d is too small for B = %d rows", n_slots, desc->B);
  LL_ALIGNED(q, 16); LL_ALIGNED(k, 16); LL_ALIGNED(v, 16); LL_ALIGNED(y, 16); LL_ALIGNED(S, 16);
  LL_ALIGNED(g, 4); LL_ALIGNED(slots, 4); LL_ALIGNED(device_error, 4);
  ll::LinStepArgs a{};
  const long qk = (long)desc->Hk * desc->Dk, vw = (long)desc->Hv * desc->Dv;
  a.B = desc->B; a.Hk = desc->Hk; a.H = desc->Hv; a.Dk = desc->Dk; a.Dv = desc->Dv; a.n_slots = n_slots;
  a.scale = scale_of(*desc);
  a.q_ld = desc->q_ld ? desc->q_ld : qk;
  a.k_ld = desc->k_ld ? desc->k_ld : qk;
  a.v_ld = desc->v_ld ? desc->v_ld : vw;
  a.q = q; a.k = k; a.v = v; a.g = g; a.S = S; a.slots = slots; a.y = y; a.err = device_error;
  const long grid = (long)a.B * a.H * ((a.Dv + ll::kLinStepCols - 1) / ll::kLinStepCols);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (desc->dtype == LL_BF16) ll::lin_step_kernel<bf16_t><<<dim3((unsigned)grid), dim3(256), 0, s>>>(a);
  else ll::lin_step_kernel<float><<<dim3((unsigned)grid), dim3(256), 0, s>>>(a);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

}  // extern "C"
