// Rows of logits: their sums and their largest values in one walk (device side).
#pragma once

#include "ll_device.h"
#include "lstmloop.h"

namespace ll {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLowest = -3.402823466e38f;
constexpr int kTopMax = LL_LOGPROB_TOP_MAX;
constexpr int kPartsMax = 32;          // work-groups per row

// The chunks of a row that a part walks, and its single elements.
struct Span {
  int head;                            // elements before the first chunk
  int c0, c1;                          // chunks
  int tail0;                           // first element after the chunks
  bool first, last;                    // does the head / the tail
};

template <typename T>
__device__ __forceinline__ Span span_of(const T* row, int V, int part, int parts) {
  constexpr int E = Op<T>::kPerChunk;
  Span s;
  const int mis = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
  s.head = min(mis ? E - mis : 0, V);
  const int nc = (V - s.head) / E;
  s.c0 = (int)((long)nc * part / parts);
  s.c1 = (int)((long)nc * (part + 1) / parts);
  s.tail0 = s.head + nc * E;
  s.first = part == 0;
  s.last = part == parts - 1;
  return s;
}

template <typename T> __device__ __forceinline__ void unpack(uint4 u, float* f);
template <> __device__ __forceinline__ void unpack<float>(uint4 u, float* f) {
  f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y);
  f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void unpack<bf16_t>(uint4 u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
template <typename T> __device__ __forceinline__ uint4 pack(const float* f);
template <> __device__ __forceinline__ uint4 pack<float>(const float* f) {
  return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 pack<bf16_t>(const float* f) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (uint32_t)f32_to_bf16(f[2 * i]) | (uint32_t)f32_to_bf16(f[2 * i + 1]) << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Stats {
  float m, s, t;
};

__device__ __forceinline__ float exp_diff(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }

// Both sums moved to the reference m2 >= a.m.  The differences stay finite, so
// an empty part (s = 0) adds nothing.
__device__ __forceinline__ void rebase(Stats& a, float m2) {
  const float d = fmaxf(a.m - m2, -1e30f), f = exp_diff(d);
  a.t = f * (a.t + a.s * d);
  a.s *= f;
  a.m = m2;
}
__device__ __forceinline__ Stats join(Stats a, Stats b) {
  const float m = fmaxf(a.m, b.m);
  rebase(a, m);
  rebase(b, m);
  return Stats{m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ void add_one(Stats& a, float x) {
  if (x > a.m) rebase(a, x);
  const float d = x - a.m, e = exp_diff(d);
  a.s += e;
  a.t += fmaxf(d, -1e4f) * e;          // minus infinity times 0
}

// Largest value of the float order, ties by lower index; NaN below everything.
__device__ __forceinline__ unsigned long long key_of(float x, int index) {
  uint32_t u = __float_as_uint(x + 0.f);
  u = (u & 0x80000000u) ? ~u : u | 0x80000000u;
  if (x != x) u = 0;
  return (unsigned long long)u << 32 | (uint32_t)~index;
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }
__device__ __forceinline__ float key_value(unsigned long long k) {
  const uint32_t u = (uint32_t)(k >> 32);
  return __uint_as_float(u == 0 ? 0x7fc00000u : u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ unsigned long long shfl_xor_u64(unsigned long long v, int d) {
  const uint32_t lo = __shfl_xor((int)(uint32_t)v, d, 64), hi = __shfl_xor((int)(uint32_t)(v >> 32), d, 64);
  return (unsigned long long)hi << 32 | lo;
}

template <int NTHR>
struct Shared {
  float st[3][NTHR / 64];
  unsigned long long group[64];
  unsigned long long bound;
  int count, cands, last;
  unsigned long long top[kTopMax];
  int cand[NTHR];
  unsigned long long buf[NTHR == 256 ? 1024 : 4096];
};

template <int NTHR>
__device__ __forceinline__ Stats join_group(Stats a, float (*st)[NTHR / 64]) {
  const int tid = threadIdx.x, w = tid >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
    a = join(a, Stats{__shfl_xor(a.m, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)});
  if ((tid & 63) == 0) {
    st[0][w] = a.m;
    st[1][w] = a.s;
    st[2][w] = a.t;
  }
  __syncthreads();
  constexpr int NW = NTHR / 64;
  const int i = tid & (NW - 1);
  a = Stats{st[0][i], st[1][i], st[2][i]};
#pragma unroll
  for (int d = 1; d < NW; d <<= 1)
    a = join(a, Stats{__shfl_xor(a.m, d, 64), __shfl_xor(a.s, d, 64), __shfl_xor(a.t, d, 64)});
  return a;
}

// The n <= capacity keys of sh.buf: the `top` largest into sh.top, in order
// (0 where there are fewer).
template <int NTHR>
__device__ void rank_buffer(Shared<NTHR>& sh, int n, int top) {
  const int tid = threadIdx.x;
  if (tid < kTopMax) sh.top[tid] = 0;
  __syncthreads();
  if (n <= 512) {
    for (int e = tid; e < n; e += NTHR) {
      const unsigned long long k = sh.buf[e];
      int rank = 0;
#pragma unroll 8
      for (int j = 0; j < n; ++j) rank += sh.buf[j] > k;
      if (rank < top) sh.top[rank] = k;
    }
    __syncthreads();
    return;
  }
  // many ties at the bound: one maximum after the other
  unsigned long long below = ~0ull;
  for (int j = 0; j < top; ++j) {
    unsigned long long best = 0;
    for (int e = tid; e < n; e += NTHR) {
      const unsigned long long k = sh.buf[e];
      if (k < below && k > best) best = k;
    }
    for (int d = 1; d < 64; d <<= 1) best = max(best, shfl_xor_u64(best, d));
    if ((tid & 63) == 0) sh.group[tid >> 6] = best;
    __syncthreads();
    for (int i = 0; i < NTHR / 64; ++i) best = max(best, sh.group[i]);
    __syncthreads();
    if (tid == 0) sh.top[j] = best;
    below = best;
  }
  __syncthreads();
}

// The `top` largest keys of the part's span into sh.top.  (own: the chunk of this
// thread's that holds its largest value, the first of them; own_c: which one,
// -1: the thread has none.)
template <typename T, int NTHR>
__device__ void select_top(const T* row, const Span& sp, int V, int top, uint4 own, int own_c, Shared<NTHR>& sh) {
  constexpr int E = Op<T>::kPerChunk, G = NTHR / 64, CAP = NTHR == 256 ? 1024 : 4096;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  unsigned long long key = 0;
  if (own_c >= 0) {
    float f[E];
    unpack<T>(own, f);
#pragma unroll
    for (int e = 0; e < E; ++e) key = max(key, key_of(f[e], sp.head + own_c * E + e));
  }
  unsigned long long g = key;
  for (int d = 1; d < G; d <<= 1) g = max(g, shfl_xor_u64(g, d));
  if ((tid & (G - 1)) == 0) sh.group[tid / G] = g;
  if (tid == 0) {
    sh.bound = 0;
    sh.count = 0;
    sh.cands = 0;
  }
  __syncthreads();
  if (w == 0) {
    const unsigned long long mine = sh.group[l];
    int rank = 0;
#pragma unroll 16
    for (int i = 0; i < 64; ++i) rank += sh.group[i] > mine;
    // (groups without a chunk have key 0 and share a rank: then every element
    // counts, and there are few)
    if (rank == top - 1 && mine != 0) sh.bound = mine;
  }
  __syncthreads();
  const unsigned long long bound = sh.bound;
  if (own_c >= 0 && key >= bound) sh.cand[atomicAdd(&sh.cands, 1)] = tid;
  auto offer = [&](float x, int i) {
    const unsigned long long k = key_of(x, i);
    if (k >= bound) {
      const int at = atomicAdd(&sh.count, 1);
      if (at < CAP) sh.buf[at] = k;
    }
  };
  if (sp.first && tid < sp.head) offer(Op<T>::to_f32(row[tid]), tid);
  if (sp.last && tid < V - sp.tail0) offer(Op<T>::to_f32(row[sp.tail0 + tid]), sp.tail0 + tid);
  __syncthreads();
  const int nc = sh.cands;
  // a wave per candidate, its chunks over the lanes; four candidates' loads at once
  const int per = (sp.c1 - sp.c0 + NTHR - 1) / NTHR;     // chunks of a thread at most
  for (int j = w; j < nc; j += 4 * (NTHR / 64))
    for (int i = l; i < per; i += 64) {
      uint4 u[4];
      int c[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int jq = j + q * (NTHR / 64);
        c[q] = jq < nc ? sp.c0 + sh.cand[jq] + i * NTHR : sp.c1;
        u[q] = ld16(row + sp.head + (long)min(c[q], sp.c1 - 1) * E);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (c[q] < sp.c1) {
          float f[E];
          unpack<T>(u[q], f);
#pragma unroll
          for (int e = 0; e < E; ++e) offer(f[e], sp.head + c[q] * E + e);
        }
    }
  __syncthreads();
  const int n = sh.count;
  if (n <= CAP) {
    rank_buffer<NTHR>(sh, n, top);
    return;
  }
  // a few threads hold more above the bound than the buffer: one maximum of
  // the whole span after the other
  if (tid < kTopMax) sh.top[tid] = 0;
  __syncthreads();
  unsigned long long below = ~0ull;
  for (int j = 0; j < top; ++j) {
    unsigned long long best = 0;
    auto see = [&](float x, int i) {
      const unsigned long long k = key_of(x, i);
      if (k < below && k > best) best = k;
    };
    if (sp.first && tid < sp.head) see(Op<T>::to_f32(row[tid]), tid);
    if (sp.last && tid < V - sp.tail0) see(Op<T>::to_f32(row[sp.tail0 + tid]), sp.tail0 + tid);
    for (long c = sp.c0 + tid; c < sp.c1; c += NTHR) {
      float f[E];
      unpack<T>(ld16(row + sp.head + c * E), f);
#pragma unroll
      for (int e = 0; e < E; ++e) see(f[e], sp.head + (int)c * E + e);
    }
    for (int d = 1; d < 64; d <<= 1) best = max(best, shfl_xor_u64(best, d));
    if (l == 0) sh.group[w] = best;
    __syncthreads();
    for (int i = 0; i < NTHR / 64; ++i) best = max(best, sh.group[i]);
    __syncthreads();
    if (tid == 0) sh.top[j] = best;
    below = best;
  }
  __syncthreads();
}

// The part's sums (per thread), and with TOP its thread's largest chunk.  With
// KEEP the thread's first chunks stay in LDS (keep[i][tid]).  Chunks are loaded
// four at a time, past the end the last one again: one wait for four.  Without T_SUM
// the sum that the entropy needs is left out.
template <typename T, int NTHR, bool TOP, int KEEP = 0, bool T_SUM = true>
__device__ __forceinline__ Stats walk(const T* row, const Span& sp, int V, uint4* own, int* own_c,
                                      uint4 (*keep)[NTHR] = nullptr) {
  constexpr int E = Op<T>::kPerChunk;
  const int tid = threadIdx.x;
  Stats a{kLowest, 0.f, 0.f};
  float best = -__builtin_inff();
  int best_c = -1;
  uint4 best_u = zero4();
  auto eat = [&](uint4 u, int c) {
    float f[E];
    unpack<T>(u, f);
    float cm = f[0];
#pragma unroll
    for (int e = 1; e < E; ++e) cm = fmaxf(cm, f[e]);
    if (cm > a.m) rebase(a, cm);
    if (TOP && (cm > best || best_c < 0)) {
      best = cm > best ? cm : best;    // (a first chunk of NaN: anything is more)
      best_c = c;
      best_u = u;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = f[e] - a.m, x = exp_diff(d);
      a.s += x;
      if (T_SUM) a.t += fmaxf(d, -1e4f) * x;
    }
  };
  const T* body = row + sp.head;
  float single = 0.f;
  const bool in_head = sp.first && tid < sp.head, in_tail = sp.last && tid < V - sp.tail0;
  if (in_head) single = Op<T>::to_f32(row[tid]);
  float single2 = 0.f;
  if (in_tail) single2 = Op<T>::to_f32(row[sp.tail0 + tid]);
  int slot = 0;
  for (int c = sp.c0 + tid; c < sp.c1; c += 4 * NTHR) {
    uint4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = ld16(body + (long)min(c + i * NTHR, sp.c1 - 1) * E);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i * NTHR < sp.c1) {
        if (KEEP && slot + i < KEEP) keep[slot + i][tid] = u[i];
        eat(u[i], c + i * NTHR);
      }
    slot += 4;
  }
  if (in_head) add_one(a, single);
  if (in_tail) add_one(a, single2);
  *own = best_u;
  *own_c = best_c;
  return a;
}

}  // namespace ll
