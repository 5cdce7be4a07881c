// Embedding: x_n = scale W[token_n], and the gradient of the table
//   dW_r = scale sum over n with token_n = r of dx_n
// in the tokens' order, without atomics on sums: the places are sorted by token (stable,
// radix), the sorted places are cut into pieces of equal length, each piece sums its runs
// of equal tokens, and a run that goes over pieces is joined from their partial sums.  So
// a token that is every tenth one costs no more than ten that are every hundredth, and
// the same call gives the same bits.  Sums are float: up to 64 terms at a time and those
// sums after that, so that n equal tokens are off by at most (64 + n / 64 + 2) 2^-24 of
// their terms' magnitudes; wider ones would take registers that the sums lack.
//
// Rows need an element's alignment only: a thread moves eight elements by vector accesses
// of that alignment.
#include <algorithm>
#include <cmath>
#include <new>

#include "ll_host.h"
#include "ll_pieces.h"
#include "ll_stream.h"

using ll::bf16_t;
using ll::fail;

namespace ll {

constexpr int kEmbSmall = 4096;        // places that one work-group sorts
constexpr int kEmbThreads = 512, kEmbWaves = kEmbThreads / 64;
constexpr int kEmbBits = 10;           // of a digit at most
constexpr int kEmbTiles = 128;         // work-groups of a sorting pass at most
constexpr int kEmbHeld = 4;            // keys of a thread that stay in registers
constexpr int kEmbUnit = 8;            // elements of a thread
constexpr int kEmbJoin = 256;          // threads that join a run
constexpr int kEmbSums = 2048;         // waves that sum, where there are places enough

struct EmbedArgs {
  int N, V, D;
  float scale;
  long w_ld, x_ld, dx_ld, dw_ld;
  const int* tokens;
  const void *w, *dx;
  void *x, *dw;
  int accumulate;
  int* err;
  // sorted places: tokens (V: none), and where they stand
  int *key[2], *pos[2];
  int* hist;                           // [tile][digit]
  int bits, tiles, tile;               // of a digit; work-groups and places of a pass
  int piece, pieces;
  float* part;                         // [piece][2][D]: a run's sum that the piece before, or this one, began
  int *heads, *count;                  // pieces whose last run goes on
  int fill;                            // work-groups that clear the table's gradient beside the sort
};

// Eight elements at an element's alignment, as they are and as floats.
template <typename T> struct Eight;
template <> struct Eight<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    typedef f32x4 any __attribute__((aligned(4)));
    a = *reinterpret_cast<const any*>(p);
    b = *reinterpret_cast<const any*>(p + 4);
  }
  __device__ __forceinline__ void load_few(const float* p, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = i < n ? p[i] : 0.f;
      b[i] = 4 + i < n ? p[4 + i] : 0.f;
    }
  }
  __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = a[i];
      f[4 + i] = b[i];
    }
  }
};
template <> struct Eight<bf16_t> {
  u32x4 a;
  __device__ __forceinline__ void load(const bf16_t* p) {
    typedef u32x4 any __attribute__((aligned(2)));
    a = *reinterpret_cast<const any*>(p);
  }
  __device__ __forceinline__ void load_few(const bf16_t* p, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a[i] = (2 * i < n ? (uint32_t)p[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)p[2 * i + 1] << 16 : 0u);
  }
  __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(a[i] << 16);
      f[2 * i + 1] = __uint_as_float(a[i] & 0xffff0000u);
    }
  }
};
template <typename T> __device__ __forceinline__ void store8(T* p, const float* f);
template <> __device__ __forceinline__ void store8<float>(float* p, const float* f) {
  typedef f32x4 any __attribute__((aligned(4)));
  *reinterpret_cast<any*>(p) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<any*>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}
template <> __device__ __forceinline__ void store8<bf16_t>(bf16_t* p, const float* f) {
  typedef u32x4 any __attribute__((aligned(2)));
  *reinterpret_cast<any*>(p) = u32x4{pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7])};
}

// The columns of a thread: eight from `col` on, of which it answers for those from `skip` on
// (the last thread of a row whose size is no multiple of eight moves back to have eight).
// A row of fewer than eight is one thread's, element by element.
struct Columns {
  int col, skip, size;
  bool any;
  __device__ __forceinline__ Columns(int u, int D) {
    any = u < D;
    size = D;
    col = D < kEmbUnit ? 0 : min(u, D - kEmbUnit);
    skip = any ? u - col : kEmbUnit;
  }
};
// (every load goes out before the first is waited for, where there are eight columns)
template <typename T, int R, typename At>
__device__ __forceinline__ void load_rows(const Columns& c, At row, Eight<T>* x) {
  if (c.size >= kEmbUnit) {
#pragma unroll
    for (int j = 0; j < R; ++j) x[j].load(row(j) + c.col);
  } else {
#pragma unroll
    for (int j = 0; j < R; ++j) x[j].load_few(row(j), c.size);
  }
}
template <typename T>
__device__ __forceinline__ void store_row(const Columns& c, T* row, const float* f) {
  if (c.size >= kEmbUnit && c.skip == 0) {
    store8(row + c.col, f);
    return;
  }
#pragma unroll
  for (int e = 0; e < kEmbUnit; ++e)
    if (e >= c.skip && c.col + e < c.size) row[c.col + e] = Op<T>::from_f32(f[e]);
}

// Rows of a work-group of 256: `lanes` threads (a power of two) a row.  Bound by its bytes:
// 131072 rows of 1024 bfloat16, 537 MB with what is read, in 77 us; 128 rows in 3.5 us.
template <typename TW, typename TX>
__global__ __launch_bounds__(256) void embed_fwd_kernel(EmbedArgs a, int lanes, int rows) {
  constexpr int R = 4;                 // rows of a thread under way at once
  const int lane = threadIdx.x & (lanes - 1), grp = threadIdx.x / lanes, groups = 256 / lanes;
  const long n0 = (long)blockIdx.x * rows;
  const TW* w = static_cast<const TW*>(a.w);
  for (int u = lane * kEmbUnit; u < a.D; u += lanes * kEmbUnit) {
    const Columns c(u, a.D);
    for (int i = grp; i < rows; i += R * groups) {
      int t[R];
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const long n = n0 + i + j * groups;
        t[j] = i + j * groups < rows && n < a.N ? a.tokens[n] : -1;
      }
      Eight<TW> x[R];
      // (without a token: row 0, and it counts for nothing)
      load_rows<TW, R>(c, [&](int j) { return w + (t[j] >= 0 && t[j] < a.V ? t[j] : 0) * a.w_ld; }, x);
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const long n = n0 + i + j * groups;
        if (i + j * groups >= rows || n >= a.N) continue;
        const bool has = t[j] >= 0 && t[j] < a.V;
        if (!has && t[j] != -1 && u == 0) atomicOr(a.err, LL_DEVERR_TOKEN);
        float f[kEmbUnit];
        x[j].floats(f);
#pragma unroll
        for (int e = 0; e < kEmbUnit; ++e) f[e] = has ? f[e] * a.scale : 0.f;
        store_row(c, static_cast<TX*>(a.x) + n * a.x_ld, f);
      }
    }
  }
}

// Clears share `index` of `shares` of the table's gradient.
template <typename TG>
__device__ void embed_clear(const EmbedArgs& a, long index, long shares, int threads) {
  TG* dw = static_cast<TG*>(a.dw);
  const long at = index * threads + threadIdx.x, all = shares * threads;
  const float zero[kEmbUnit] = {};
  if (a.dw_ld == a.D) {
    // (16 bytes a lane, neighbours side by side)
    constexpr int E = 16 / sizeof(TG);
    typedef u32x4 any __attribute__((aligned(2)));
    const long n = (long)a.V * a.D, units = n / E;
    for (long u = at; u < units; u += all) *reinterpret_cast<any*>(dw + u * E) = u32x4{0, 0, 0, 0};
    if (at < n - units * E) dw[units * E + at] = 0;
    return;
  }
  const int units = (a.D + kEmbUnit - 1) / kEmbUnit;
  for (long u = at; u < (long)a.V * units; u += all) {
    store_row(Columns((int)(u % units) * kEmbUnit, a.D), dw + u / units * a.dw_ld, zero);
  }
}

// The key of a place: its token, or V where it has none.
__device__ __forceinline__ int embed_key(const EmbedArgs& a, int n) {
  const int t = a.tokens[n];
  if (t < -1 || t >= a.V) atomicOr(a.err, LL_DEVERR_TOKEN);
  return t < 0 || t >= a.V ? a.V : t;
}

struct EmbedSort {
  int cnt[kEmbWaves][1 << kEmbBits];
  int wave[kEmbWaves];
};

// A pass waits for memory and LDS more than it moves: 131072 places in 64 tiles take 4.8
// us to count and 11.7 to place, 1 MB each way; places a wave puts down together find their
// rank by a ballot for each bit of the digit, without atomics.
//
// One pass over the digit at `shift` for tile `tile`: places [n0, n1) of the source go to
// where the tiles' counts say, equal digits in their order.  `first`: the source is the
// tokens.  `alone`: there is one tile, which counts for itself.
__device__ void embed_pass(const EmbedArgs& a, EmbedSort& sh, int tile, int shift, bool first, bool alone,
                           const int* key_in, const int* pos_in, int* key_out, int* pos_out) {
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63, digits = 1 << a.bits, mask = digits - 1;
  const int n0 = tile * a.tile, n1 = min(a.N, n0 + a.tile);
  const int share = ((n1 - n0 + kEmbWaves - 1) / kEmbWaves + 63) & ~63;
  const int lo = min(n1, n0 + w * share), hi = min(n1, lo + share);
  for (int d = tid; d < kEmbWaves << a.bits; d += kEmbThreads) sh.cnt[d >> a.bits][d & mask] = 0;
  __syncthreads();
  // (the first rounds' keys stay in registers between the two walks over them)
  int held[kEmbHeld];
#pragma unroll
  for (int i = 0; i < kEmbHeld; ++i) {
    const int n = lo + 64 * i + l;
    held[i] = n < hi ? (first ? embed_key(a, n) : key_in[n]) : a.V;
  }
#pragma unroll
  for (int i = 0; i < kEmbHeld; ++i)
    if (lo + 64 * i + l < hi) atomicAdd(&sh.cnt[w][held[i] >> shift & mask], 1);
  for (int n = lo + 64 * kEmbHeld + l; n < hi; n += 64)
    atomicAdd(&sh.cnt[w][((first ? embed_key(a, n) : key_in[n]) >> shift) & mask], 1);
  __syncthreads();
  // a thread's two digits: all before them, then in tile and wave order
  constexpr int PER = (1 << kEmbBits) / kEmbThreads;
  static_assert(PER == 2, "two digits a thread, read at once");
  int total[PER], before[PER], sum = 0;
#pragma unroll
  for (int i = 0; i < PER; ++i) total[i] = before[i] = 0;
  if (tid * PER < digits) {            // (digits is a multiple of PER)
    if (alone) {
#pragma unroll
      for (int i = 0; i < PER; ++i)
        for (int j = 0; j < kEmbWaves; ++j) total[i] += sh.cnt[j][tid * PER + i];
    } else {
#pragma unroll 16
      for (int t = 0; t < a.tiles; ++t) {
        const int2 c = *reinterpret_cast<const int2*>(a.hist + (long)t * digits + tid * PER);
        total[0] += c.x;
        total[1] += c.y;
        before[0] += t < tile ? c.x : 0;
        before[1] += t < tile ? c.y : 0;
      }
    }
    sum = total[0] + total[1];
  }
  int scan = sum;
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(scan, d, 64);
    if (l >= d) scan += o;
  }
  if (l == 63) sh.wave[w] = scan;
  __syncthreads();
  int at = scan - sum;
  for (int j = 0; j < w; ++j) at += sh.wave[j];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int d = tid * PER + i;
    if (d >= digits) continue;
    int start = at + before[i];
    for (int j = 0; j < kEmbWaves; ++j) {
      const int c = sh.cnt[j][d];
      sh.cnt[j][d] = start;
      start += c;
    }
    at += total[i];
  }
  __syncthreads();
  // (an address in LDS: accesses through a general one wait for the stores to memory too,
  // 14 us instead of 11.7 for 131072 places)
  typedef __attribute__((address_space(3))) volatile int* lds_int;
  lds_int next = (lds_int)sh.cnt[w];
  auto place = [&](int n, int key, int pos) {
    const bool in = n + l < hi;
    const int d = (key >> shift) & mask;
    unsigned long long same = __ballot(in);
    for (int i = 0; i < a.bits; ++i) {
      const bool bit = d >> i & 1;
      const unsigned long long m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    if (in) {
      const int rank = __popcll(same & ((1ull << l) - 1));
      const int to = next[d] + rank;
      key_out[to] = key;
      pos_out[to] = pos;
      wave_lds_fence();
      if (rank == 0) next[d] = to + __popcll(same);
    }
    wave_lds_fence();
  };
  int from[kEmbHeld];
#pragma unroll
  for (int i = 0; i < kEmbHeld; ++i) {
    const int n = lo + 64 * i + l;
    from[i] = first || n >= hi ? n : pos_in[n];
  }
#pragma unroll
  for (int i = 0; i < kEmbHeld; ++i)
    if (lo + 64 * i < hi) place(lo + 64 * i, held[i], from[i]);
  for (int n = lo + 64 * kEmbHeld; n < hi; n += 64) {
    int key = a.V, pos = n + l;
    if (n + l < hi) {
      key = first ? embed_key(a, n + l) : key_in[n + l];
      pos = first ? n + l : pos_in[n + l];
    }
    place(n, key, pos);
  }
}

// All passes of a few places by one work-group; the others clear the gradient.
template <typename TG>
__global__ __launch_bounds__(kEmbThreads) void embed_sort_small_kernel(EmbedArgs a, int passes) {
  __shared__ EmbedSort sh;
  if (blockIdx.x > 0) {
    embed_clear<TG>(a, blockIdx.x - 1, a.fill, kEmbThreads);
    return;
  }
  if (threadIdx.x == 0) *a.count = 0;
  for (int i = 0; i < passes; ++i) {
    embed_pass(a, sh, 0, i * a.bits, i == 0, true, a.key[(i + 1) & 1], a.pos[(i + 1) & 1], a.key[i & 1], a.pos[i & 1]);
    __threadfence_block();
    __syncthreads();
  }
}

// Digits of every tile.
template <typename TG>
__global__ __launch_bounds__(kEmbThreads) void embed_count_kernel(EmbedArgs a, int pass, long clear0, long shares) {
  __shared__ int cnt[1 << kEmbBits];
  if ((int)blockIdx.x >= a.tiles) {
    embed_clear<TG>(a, clear0 + blockIdx.x - a.tiles, shares, kEmbThreads);
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = 0;
  const int digits = 1 << a.bits, mask = digits - 1, tile = blockIdx.x;
  for (int d = threadIdx.x; d < digits; d += kEmbThreads) cnt[d] = 0;
  __syncthreads();
  const int n0 = tile * a.tile, n1 = min(a.N, n0 + a.tile);
  const int* in = a.key[(pass + 1) & 1];
  for (int n = n0 + threadIdx.x; n < n1; n += kEmbThreads)
    atomicAdd(&cnt[((pass == 0 ? embed_key(a, n) : in[n]) >> pass * a.bits) & mask], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < digits; d += kEmbThreads) a.hist[(long)tile * digits + d] = cnt[d];
}

template <typename TG>
__global__ __launch_bounds__(kEmbThreads) void embed_place_kernel(EmbedArgs a, int pass, long clear0, long shares) {
  __shared__ EmbedSort sh;
  if ((int)blockIdx.x >= a.tiles) {
    embed_clear<TG>(a, clear0 + blockIdx.x - a.tiles, shares, kEmbThreads);
    return;
  }
  embed_pass(a, sh, blockIdx.x, pass * a.bits, pass == 0, false, a.key[(pass + 1) & 1], a.pos[(pass + 1) & 1],
             a.key[pass & 1], a.pos[pass & 1]);
}

// scale * acc to the row of token t, or added to it: to `old`, where that has been read.
template <typename TG, bool ADD>
__device__ __forceinline__ void embed_put(const EmbedArgs& a, int t, const Columns& c, const float* acc,
                                          const Eight<TG>* old = nullptr) {
  TG* to = static_cast<TG*>(a.dw) + t * a.dw_ld;
  float f[kEmbUnit];
  if (ADD) {
    Eight<TG> x[1];
    if (old) x[0] = *old;
    else load_rows<TG, 1>(c, [&](int) { return to; }, x);
    x[0].floats(f);
  }
#pragma unroll
  for (int e = 0; e < kEmbUnit; ++e) f[e] = ADD ? __builtin_fmaf(a.scale, acc[e], f[e]) : a.scale * acc[e];
  store_row(c, to, f);
}

// The runs of a piece: `lanes` threads and as many eights of columns.  Bound by the rows of
// dx that it gathers and the rows it writes: 131072 places of 1024 bfloat16, onto old
// floats (ADD), in 142 us, 3.7 TB/s (152 when a run's old row was read at its end, one
// after the other; its 183 registers leave two waves a SIMD); 25600 places of 1024 floats,
// 19200 of them with a token, in 27 us, 3.9 TB/s with the 25 MB written (47 when the places
// were fetched with their rows).
template <typename TX, typename TG, bool ADD>
__global__ __launch_bounds__(256) void embed_sum_kernel(EmbedArgs a, int lanes, int cols, const int* key, const int* pos) {
  constexpr int R = 8;
  const int lane = threadIdx.x & (lanes - 1), groups = 256 / lanes;
  const int piece = (int)(blockIdx.x / cols) * groups + threadIdx.x / lanes;
  const Columns c(((int)(blockIdx.x % cols) * lanes + lane) * kEmbUnit, a.D);
  if (piece >= a.pieces) return;
  const int n0 = piece * a.piece, n1 = min(a.N, n0 + a.piece);
  int cur = key[n0];
  if (cur == a.V) return;
  const bool begun = n0 > 0 && key[n0 - 1] == cur;
  const int after = n1 < a.N ? key[n1] : -1;
  bool first = true;
  float acc[kEmbUnit] = {};
  auto flush = [&](bool goes_on, const Eight<TG>* old) __attribute__((always_inline)) {
    if (!c.any) return;
    const bool before = first && begun;
    if (before || goes_on) store_row(c, a.part + (2l * piece + (before ? 0 : 1)) * a.D, acc);
    else embed_put<TG, ADD>(a, cur, c, acc, old);
  };
  // eight places at a time (a piece is a multiple of that, and the arrays are padded to
  // one): their tokens and rows' numbers a step ahead of the rows, the rows without
  // conditions (what stands behind the last token has a row too, which counts for nothing)
  const TX* dx = static_cast<const TX*>(a.dx);
  auto fetch = [&](int n, int* k, int* at) {
#pragma unroll
    for (int j = 0; j < R; j += 4) {
      const int4 x = *reinterpret_cast<const int4*>(key + n + j), y = *reinterpret_cast<const int4*>(pos + n + j);
      k[j] = x.x; k[j + 1] = x.y; k[j + 2] = x.z; k[j + 3] = x.w;
      at[j] = y.x; at[j + 1] = y.y; at[j + 2] = y.z; at[j + 3] = y.w;
    }
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (n + j >= n1) {
        k[j] = a.V;
        at[j] = at[0];
      }
  };
  int k[R], at[R], k2[R], at2[R];
  fetch(n0, k, at);
  for (int n = n0; n < n1 && cur != a.V; n += R) {
    Eight<TX> x[R];
    load_rows<TX, R>(c, [&](int j) { return dx + at[j] * a.dx_ld; }, x);
    // the old rows of the runs that end here, beside them
    Eight<TG> old[ADD ? R : 1];
    if (ADD) {
#pragma unroll
      for (int j = 0; j < R; ++j) {
        const int t = j ? k[j - 1] : cur;
        if (t != k[j] && t != a.V && n + j < n1)
          load_rows<TG, 1>(c, [&](int) { return static_cast<const TG*>(a.dw) + t * a.dw_ld; }, old + j);
      }
    }
    if (n + R < n1) fetch(n + R, k2, at2);
#pragma unroll
    for (int j = 0; j < R; ++j) {
      if (cur == a.V) break;
      if (k[j] != cur) {
        if (n + j >= n1) break;        // the piece's end: below
        flush(false, ADD ? old + j : nullptr);
        first = false;
        cur = k[j];
#pragma unroll
        for (int e = 0; e < kEmbUnit; ++e) acc[e] = 0.f;
        if (cur == a.V) break;
      }
      float f[kEmbUnit];
      x[j].floats(f);
#pragma unroll
      for (int e = 0; e < kEmbUnit; ++e) acc[e] += f[e];
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      k[j] = k2[j];
      at[j] = at2[j];
    }
  }
  if (cur == a.V) return;
  const bool goes_on = after == cur;
  flush(goes_on, nullptr);
  if (goes_on && !(first && begun) && c.any && c.col + c.skip == 0) a.heads[atomicAdd(a.count, 1)] = piece;
}

// Runs that go over pieces: the waves' shares of the partial sums, joined in order (7 us
// for 25600 places in pieces of 16, 13 for 131072 in pieces of 64: a few long runs).
template <typename TG, bool ADD>
__global__ __launch_bounds__(kEmbJoin) void embed_join_kernel(EmbedArgs a, const int* key) {
  constexpr int NW = kEmbJoin / 64, R = 8;
  __shared__ int more;
  __shared__ float sums[NW][64 * kEmbUnit];
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  const int count = *a.count;
  const Columns c(((int)blockIdx.y * 64 + l) * kEmbUnit, a.D);
  for (int i = blockIdx.x; i < count; i += gridDim.x) {
    const int head = a.heads[i], t = key[(head + 1) * a.piece];
    if (tid == 0) more = 0;
    __syncthreads();
    // pieces that begin with this token, sorted as they are: a run of them
    for (int p0 = head + 1; p0 < a.pieces; p0 += kEmbJoin) {
      const bool in = p0 + tid < a.pieces && key[(p0 + tid) * a.piece] == t;
      const int n = __popcll(__ballot(in));
      if (l == 0 && n) atomicAdd(&more, n);
      __syncthreads();
      if (more < p0 + kEmbJoin - head - 1) break;
    }
    const int n = more + 1;            // partial sums: the head's second, the others' first
    const int share = (n + NW - 1) / NW, lo = min(n, w * share), hi = min(n, lo + share);
    float acc[kEmbUnit] = {};
    if (c.any)
      for (int j = lo; j < hi; j += R) {
        Eight<float> x[R];
        load_rows<float, R>(c, [&](int q) {
          const int k = min(j + q, hi - 1);
          return a.part + (2l * (head + k) + (k == 0 ? 1 : 0)) * a.D;
        }, x);
#pragma unroll
        for (int q = 0; q < R; ++q) {
          if (j + q >= hi) break;
          float f[kEmbUnit];
          x[q].floats(f);
#pragma unroll
          for (int e = 0; e < kEmbUnit; ++e) acc[e] += f[e];
        }
      }
#pragma unroll
    for (int e = 0; e < kEmbUnit; ++e) sums[w][e * 64 + l] = acc[e];
    __syncthreads();
    if (w == 0 && c.any) {
#pragma unroll
      for (int e = 0; e < kEmbUnit; ++e) {
        float s = sums[0][e * 64 + l];
        for (int j = 1; j < NW; ++j) s += sums[j][e * 64 + l];
        acc[e] = s;
      }
      embed_put<TG, ADD>(a, t, c, acc);
    }
    __syncthreads();
  }
}

}  // namespace ll

struct ll_embed_plan {
  ll_embed_desc d;
  int device = 0, cus = 0, passes = 0;
  ll::EmbedArgs a{};
  int64_t bytes = 0;
};

namespace {

int bytes_of(int dtype) { return dtype == LL_BF16 ? 2 : 4; }

void release(ll_embed_plan* p) {
  void* all[] = {p->a.key[0], p->a.key[1], p->a.pos[0], p->a.pos[1], p->a.hist, p->a.part, p->a.heads, p->a.count, p->a.err};
  for (void* m : all)
    if (m) (void)hipFree(m);
}

// Threads for a row of D: eight elements each, a power of two.
int lanes_of(int D) {
  int lanes = 1;
  while (lanes < 256 && lanes * ll::kEmbUnit < D) lanes *= 2;
  return lanes;
}

// Places of a piece for n of them: long ones leave fewer partial sums, as long as there
// are waves enough.  (Sums and joins of 25600 places of 1024 floats: pieces of 64 places
// 40.4 + 4.9 us, 32 33.0 + 6.2, 16 26.9 + 7.4, 8 26.5 + 13.1; of 131072 places of bfloat16,
// before old rows were read ahead: 64 152 + 12.7, 32 145 + 22.7.)
int piece_of(int n, int D) {
  const int lanes = lanes_of(D), cols = (D + lanes * ll::kEmbUnit - 1) / (lanes * ll::kEmbUnit);
  int piece = 64;
  while (piece > 8 && (long)(n / piece) * cols * lanes < 64L * ll::kEmbSums) piece /= 2;
  return piece;
}

ll_status validate(const ll_embed_desc* d) {
  if (!d) return fail(LL_EINVAL, "desc is NULL");
  if (d->N < 1 || d->N > 1 << 24 || d->V < 1 || d->V >= 1 << 30 || d->D < 1 || d->D > 1 << 16)
    return fail(LL_EINVAL, "N = %d must be 1 .. 2^24, V = %d 1 .. 2^30 - 1 and D = %d 1 .. 2^16", d->N, d->V, d->D);
  for (int t : {d->table_dtype, d->x_dtype, d->dx_dtype, d->grad_dtype})
    if (t != LL_F32 && t != LL_BF16) return fail(LL_EINVAL, "the types must be LL_F32 or LL_BF16");
  for (int64_t ld : {d->table_ld, d->x_ld, d->dx_ld, d->grad_ld})
    if (ld && (ld < d->D || ld > (int64_t)1 << 31))
      return fail(LL_EINVAL, "a distance of rows is %lld: it must be 0, or D = %d .. 2^31", (long long)ld, d->D);
  if (!std::isfinite(d->scale)) return fail(LL_EINVAL, "scale is not finite");
  if (d->reserved) return fail(LL_EINVAL, "reserved must be 0");
  // work-groups of the sums (a piece of 64 places and 512 columns each) at most
  const int64_t groups = ((int64_t)(d->N + 63) / 64) * ((d->D + 511) / 512);
  if (groups > ll::max_groups(256))
    return fail(LL_EUNSUPPORTED, "N = %d with D = %d: %lld work-groups, a launch holds %lld", d->N, d->D,
                (long long)groups, (long long)ll::max_groups(256));
  return LL_OK;
}

ll_status count_ok(const ll_embed_plan* p, int32_t n) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (n < 0 || n > p->d.N) return fail(LL_EINVAL, "n = %d must be 0 .. %d", n, p->d.N);
  return LL_OK;
}

template <typename TW, typename TX>
void launch_fwd(const ll::EmbedArgs& a, int lanes, int rows, hipStream_t s) {
  const unsigned grid = (unsigned)((a.N + rows - 1) / rows);
  ll::embed_fwd_kernel<TW, TX><<<dim3(grid), dim3(256), 0, s>>>(a, lanes, rows);
}

template <typename TX, typename TG>
void launch_bwd(const ll::EmbedArgs& a, int passes, hipStream_t s) {
  const int threads = ll::kEmbThreads;
  if (a.N <= ll::kEmbSmall) {
    ll::embed_sort_small_kernel<TG><<<dim3(1 + a.fill), dim3(threads), 0, s>>>(a, passes);
  } else {
    // the clearing work-groups go out with the sort's launches, three quarters of them beside
    // the longer one of a pass (131 MB with 25600 places: 41 us of sort, 3 more in equal
    // shares)
    const int launches = 2 * passes;
    long done = 0;
    for (int i = 0; i < launches; ++i) {
      const long upto = (long)a.fill * (i & 1 ? 4 * (i / 2 + 1) : 4 * (i / 2) + 1) / (4 * passes);
      const dim3 grid((unsigned)(a.tiles + upto - done));
      if (i & 1) ll::embed_place_kernel<TG><<<grid, dim3(threads), 0, s>>>(a, i / 2, done, a.fill);
      else ll::embed_count_kernel<TG><<<grid, dim3(threads), 0, s>>>(a, i / 2, done, a.fill);
      done = upto;
    }
  }
  if (a.pieces == 0) return;
  const int* key = a.key[(passes - 1) & 1];
  const int* pos = a.pos[(passes - 1) & 1];
  const int lanes = lanes_of(a.D), cols = (a.D + lanes * ll::kEmbUnit - 1) / (lanes * ll::kEmbUnit);
  const int groups = 256 / lanes;
  const unsigned grid = (unsigned)((a.pieces + groups - 1) / groups) * cols;
  const dim3 joins((unsigned)std::min(a.pieces - 1, 2048),
                   (unsigned)((a.D + 64 * ll::kEmbUnit - 1) / (64 * ll::kEmbUnit)));
  if (a.accumulate) {
    ll::embed_sum_kernel<TX, TG, true><<<dim3(grid), dim3(256), 0, s>>>(a, lanes, cols, key, pos);
    if (a.pieces > 1) ll::embed_join_kernel<TG, true><<<joins, dim3(ll::kEmbJoin), 0, s>>>(a, key);
  } else {
    ll::embed_sum_kernel<TX, TG, false><<<dim3(grid), dim3(256), 0, s>>>(a, lanes, cols, key, pos);
    if (a.pieces > 1) ll::embed_join_kernel<TG, false><<<joins, dim3(ll::kEmbJoin), 0, s>>>(a, key);
  }
}

}  // namespace

extern "C" {

ll_status ll_embed_plan_create(const ll_embed_desc* d, int device, ll_embed_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  LL_STATUS(validate(d));
  LL_STATUS(ll::check_device(device));
  ll::DeviceGuard guard(device);
  ll_embed_plan* p = new (std::nothrow) ll_embed_plan();
  if (!p) return fail(LL_ENOMEM, "host allocation of the plan failed");
  p->d = *d;
  p->device = device;
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, device) != hipSuccess) {
    delete p;
    return fail(LL_EHIP, "hipGetDeviceProperties failed");
  }
  p->cus = prop.multiProcessorCount;
  ll::EmbedArgs& a = p->a;
  a.V = d->V; a.D = d->D;
  a.scale = d->scale != 0.f ? d->scale : 1.f;
  a.w_ld = d->table_ld ? d->table_ld : d->D;
  a.x_ld = d->x_ld ? d->x_ld : d->D;
  a.dx_ld = d->dx_ld ? d->dx_ld : d->D;
  a.dw_ld = d->grad_ld ? d->grad_ld : d->D;
  int key_bits = 1;
  while ((long)1 << key_bits <= d->V) ++key_bits;        // the key V is a place without a token
  p->passes = (key_bits + ll::kEmbBits - 1) / ll::kEmbBits;
  a.bits = (key_bits + p->passes - 1) / p->passes;
  // partial sums: two a piece; the most pieces that any number of places up to N has
  // (fewer than twice those of the smallest number that takes longer ones)
  const int lanes = lanes_of(d->D), cols = (d->D + lanes * ll::kEmbUnit - 1) / (lanes * ll::kEmbUnit);
  const long full = 64L * ll::kEmbSums / ((long)cols * lanes) + 1;
  const long pieces = std::max((long)(d->N + 63) / 64, std::min((long)(d->N + 7) / 8, 2 * full + 2));
  const size_t n4 = sizeof(int) * ((size_t)(d->N + 7) / 8 * 8);  // (read eight at a time)
  const bool train = !d->inference;
  struct { void** at; size_t bytes; const char* what; bool want; } bufs[] = {
      {(void**)&a.key[0], n4, "the sorted tokens", train},
      {(void**)&a.key[1], n4, "the sorted tokens", train},
      {(void**)&a.pos[0], n4, "the sorted places", train},
      {(void**)&a.pos[1], n4, "the sorted places", train},
      {(void**)&a.hist, sizeof(int) * ((size_t)ll::kEmbTiles << a.bits), "the tiles' counts", train && d->N > ll::kEmbSmall},
      {(void**)&a.part, sizeof(float) * 2 * pieces * d->D, "the pieces' sums", train},
      {(void**)&a.heads, sizeof(int) * pieces, "the runs over pieces", train},
      {(void**)&a.count, sizeof(int), "their number", train},
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

ll_status ll_embed_plan_destroy(ll_embed_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_embed_plan_bytes(const ll_embed_plan* p, int64_t* device_bytes) {
  if (!p || !device_bytes) return fail(LL_EINVAL, "plan and device_bytes are required");
  *device_bytes = p->bytes;
  return LL_OK;
}

ll_status ll_embed_fwd(ll_embed_plan* p, void* stream, int32_t n, const void* table, const int32_t* tokens, void* x) {
  LL_STATUS(count_ok(p, n));
  if (n == 0) return LL_OK;
  if (!table || !tokens || !x) return fail(LL_EINVAL, "table, tokens and x are required");
  LL_ALIGNED(table, bytes_of(p->d.table_dtype)); LL_ALIGNED(x, bytes_of(p->d.x_dtype)); LL_ALIGNED(tokens, 4);
  ll::DeviceGuard guard(p->device);
  ll::EmbedArgs a = p->a;
  a.N = n; a.w = table; a.tokens = tokens; a.x = x;
  const int lanes = lanes_of(a.D);
  // four rows a thread where there are rows enough for all compute units
  const int groups = 256 / lanes;
  const int rows = (long)n >= 8L * p->cus * groups ? 4 * groups : groups;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool wb = p->d.table_dtype == LL_BF16, xb = p->d.x_dtype == LL_BF16;
  if (wb && xb) launch_fwd<bf16_t, bf16_t>(a, lanes, rows, s);
  else if (wb) launch_fwd<bf16_t, float>(a, lanes, rows, s);
  else if (xb) launch_fwd<float, bf16_t>(a, lanes, rows, s);
  else launch_fwd<float, float>(a, lanes, rows, s);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_embed_bwd(ll_embed_plan* p, void* stream, int32_t n, const int32_t* tokens, const void* dx, void* dtable,
                       int32_t accumulate) {
  LL_STATUS(count_ok(p, n));
  if (p->d.inference) return fail(LL_EINVAL, "the plan was created for inference: it has nothing to sort with");
  if (n == 0 && accumulate) return LL_OK;
  if (!dtable || (n > 0 && (!tokens || !dx))) return fail(LL_EINVAL, "tokens, dx and dtable are required");
  LL_ALIGNED(dx, bytes_of(p->d.dx_dtype)); LL_ALIGNED(dtable, bytes_of(p->d.grad_dtype)); LL_ALIGNED(tokens, 4);
  ll::DeviceGuard guard(p->device);
  ll::EmbedArgs a = p->a;
  a.N = n; a.tokens = tokens; a.dx = dx; a.dw = dtable; a.accumulate = accumulate != 0;
  a.piece = piece_of(n, a.D);
  a.pieces = (n + a.piece - 1) / a.piece;
  if (n <= ll::kEmbSmall) {
    a.tiles = 1;
    a.tile = n;
  } else {
    // (131072 places: 128 tiles take 3 us longer to place than 64, each reads all counts)
    a.tiles = std::min(ll::kEmbTiles, (n + 2047) / 2048);
    a.tile = (n + a.tiles - 1) / a.tiles;
  }
  // a work-group of 512 threads clears 64 KB or more
  const long bytes = (long)a.V * a.D * bytes_of(p->d.grad_dtype);
  a.fill = accumulate ? 0 : (int)std::min((bytes + 65535) / 65536, 4L * p->cus);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  const bool xb = p->d.dx_dtype == LL_BF16, gb = p->d.grad_dtype == LL_BF16;
  if (xb && gb) launch_bwd<bf16_t, bf16_t>(a, p->passes, s);
  else if (xb) launch_bwd<bf16_t, float>(a, p->passes, s);
  else if (gb) launch_bwd<float, bf16_t>(a, p->passes, s);
  else launch_bwd<float, float>(a, p->passes, s);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_embed_status_sync(ll_embed_plan* p, int32_t* device_error) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  ll::DeviceGuard guard(p->device);
  return ll::read_error_word(p->a.err, device_error);
}

}  // extern "C"
