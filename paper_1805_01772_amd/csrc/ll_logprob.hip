// Log probabilities of given tokens, entropy, the most likely alternatives,
// and their gradient.
//
// One pass over a row keeps, per thread, the running maximum m, s = sum e^{x-m}
// and t = sum (x - m) e^{x-m}; joined over the work-group
//     lse = m + log s,  logp = (x_target - m) - log s,  entropy = log s - t / s.
// m and log s stay apart wherever both are at hand: their sum as one float loses log s
// where |m| is large (of a row at the type's lowest value all of it).
// Alternatives: each of 64 thread groups knows its largest (value, index); the
// top_k-th largest of those bounds the row's top_k-th from below, so only the
// threads that hold at least that much are read again (about top_k of them),
// and what they hold above the bound is ranked.  Equal values rank by index, so
// all keys differ.
// Gradient, with c = dlogp (if there is a target) + sum_j dtop_j:
//     dx = -p (c + dentropy (log p + entropy)) + dlogp [target] + dtop_j [id_j]
// the marked entries are few and written after the row.  The call of its own has lse
// as a float: where that is 32 or more in magnitude it sums the row again first
// (lse_rest).
//
// Rows are walked in 16-byte chunks from the first aligned element; up to 7
// elements before and after are done singly.
// Bound: HBM.  Forward: one pass, 2047 rows of 50001 floats in 72 us (5.7 TB/s), with 16
// alternatives in 97.  Gradient in a call of its own: two passes, 4096 rows of 131072
// bfloat16 in 423 us (5.1 TB/s), 1024 of 100000 floats in 166 (4.9).  Both in one: the
// first 64 KB of a long row (16 KB of a short one) stay in LDS, the rest is read again
// from the last-level cache on the whole; 4096 rows of 131072 bfloat16 in 445 to 461 us,
// 2.1 GB of traffic that cannot be saved at 4.7 TB/s, 4096 of 32000 floats in 193 (5.4).
// A few rows: latency, 8 rows of 32000 bfloat16 with 8 alternatives in 10 us.
#include <algorithm>
#include <new>

#include "ll_host.h"
#include "ll_rows.h"
#include "ll_stream.h"

using ll::bf16_t;
using ll::fail;

namespace ll {

struct LogprobArgs {
  int V, top, parts;
  long ld;
  const void* x;
  const int* targets;
  float *logp, *entropy, *lse;
  int* top_ids;
  float* top_logp;
  // gradient
  const float *lse_in, *ent_in, *dlogp, *dentropy, *dtop;
  const int* ids_in;
  void* dx;
  bool stream;                         // dx goes past the caches
  bool apart;                          // dx's rows do not lie as x's do between 16-byte borders
  int* err;
  // rows split over work-groups: m, s, t per part, its keys, arrivals per row
  float4* part;
  unsigned long long* keys;
  unsigned* arrived;
  float* rest;                         // lse_rest by row, where a kernel of its own made it
};

struct RowResult {
  float m, ls, ent;                    // log p = (x - m) - ls
  bool empty, sound;                   // nothing is allowed; no NaN
  __device__ __forceinline__ float logp(float x) const {
    return x == -__builtin_inff() && sound ? x : (x - m) - ls;
  }
};

// The row's target and its logit, read while the row is (thread 0's are used).
struct Target {
  int id;
  float x;
};
template <typename T>
__device__ __forceinline__ Target target_of(const LogprobArgs& a, const T* row, long r) {
  Target t{-1, 0.f};
  if (a.targets && threadIdx.x == 0) {
    t.id = a.targets[r];
    if (t.id >= 0 && t.id < a.V) t.x = Op<T>::to_f32(row[t.id]);
  }
  return t;
}

// The row's outputs from its sums (one thread writes).
__device__ __forceinline__ RowResult row_result(const LogprobArgs& a, long r, Stats st, Target t) {
  RowResult res;
  res.empty = st.s == 0.f;
  res.m = res.empty ? 0.f : st.m;
  res.ls = res.empty ? -__builtin_inff() : logf(st.s);
  res.ent = res.empty ? 0.f : res.ls - st.t / st.s;
  const float lse = res.m + res.ls;
  res.sound = lse == lse;
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = res.ent;
    if (a.targets && a.logp) {
      float lp = 0.f;
      if (t.id >= 0 && t.id < a.V) {
        lp = res.logp(t.x);
      } else if (t.id != -1) {
        atomicOr(a.err, LL_DEVERR_TARGET);
      }
      a.logp[r] = lp;
    }
  }
  return res;
}

template <typename T, int NTHR, bool TOP>
__global__ __launch_bounds__(NTHR) void logprob_fwd_kernel(LogprobArgs a) {
  __shared__ Shared<NTHR> sh;
  const int tid = threadIdx.x;
  const long r = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  const Span sp = span_of(row, a.V, part, a.parts);
  const Target target = target_of(a, row, r);
  uint4 own;
  int own_c;
  Stats st = walk<T, NTHR, TOP>(row, sp, a.V, &own, &own_c);
  st = join_group<NTHR>(st, sh.st);
  if (TOP) {
    if (st.s == 0.f) {
      // nothing is allowed here: all equal, the first ones
      const int first = sp.first ? 0 : sp.head + sp.c0 * Op<T>::kPerChunk;
      if (tid < a.top) sh.top[tid] = key_of(-__builtin_inff(), first + tid);
      __syncthreads();
    } else {
      select_top<T, NTHR>(row, sp, a.V, a.top, own, own_c, sh);
    }
  }
  if (a.parts > 1) {
    // the last work-group of the row to arrive joins the parts
    const long at = r * a.parts + part;
    // (the first wave writes and arrives, and it alone fences: a fence writes back
    // or drops the L2 of the XCD, and one from each of 16 waves took 50 us more where
    // 64 rows were split in two)
    if (tid < 64) {
      if (tid == 0) a.part[at] = make_float4(st.m, st.s, st.t, 0.f);
      if (TOP && tid < a.top) a.keys[at * kTopMax + tid] = sh.top[tid];
      __threadfence();
      if (tid == 0) {
        sh.last = atomicAdd(&a.arrived[r], 1u) == (unsigned)a.parts - 1;
        if (sh.last) {
          __threadfence();
          a.arrived[r] = 0;            // for the next call
        }
      }
    }
    __syncthreads();
    if (!sh.last) return;
    static_assert(kPartsMax == 32, "a part for each of 32 lanes");
    const int i = tid & 31;
    const volatile float* ps = reinterpret_cast<const volatile float*>(a.part + r * a.parts + min(i, a.parts - 1));
    st = Stats{ps[0], ps[1], ps[2]};
    if (i >= a.parts) st = Stats{kLowest, 0.f, 0.f};
#pragma unroll
    for (int d = 1; d < 32; d <<= 1)
      st = join(st, Stats{__shfl_xor(st.m, d, 32), __shfl_xor(st.s, d, 32), __shfl_xor(st.t, d, 32)});
    if (TOP) {
      const int n = a.parts * a.top;
      const volatile unsigned long long* keys = a.keys + r * a.parts * kTopMax;
      for (int e = tid; e < n; e += NTHR) sh.buf[e] = keys[(long)(e / a.top) * kTopMax + e % a.top];
      __syncthreads();
      rank_buffer<NTHR>(sh, n, a.top);
    }
  }
  const RowResult res = row_result(a, r, st, target);
  if (TOP && tid < a.top) {
    a.top_ids[r * a.top + tid] = key_index(sh.top[tid]);
    a.top_logp[r * a.top + tid] = res.logp(key_value(sh.top[tid]));
  }
}

// log sum e^{x - lse} of a row: what the rounding of its lse to a float took away, at
// most a unit of lse.  More than that is no rounding (the lse of more logits than these,
// a vocabulary in several parts): 0, lse is taken as it is.
template <typename T, int NTHR>
__device__ float lse_rest(const T* row, int V, float lse, float* part) {
  constexpr int E = Op<T>::kPerChunk, NW = NTHR / 64;
  const int tid = threadIdx.x;
  const Span sp = span_of(row, V, 0, 1);
  float s = 0.f;
  if (tid < sp.head) s += exp_diff(Op<T>::to_f32(row[tid]) - lse);
  if (tid < V - sp.tail0) s += exp_diff(Op<T>::to_f32(row[sp.tail0 + tid]) - lse);
  for (int c = tid; c < sp.c1; c += 4 * NTHR) {
    uint4 u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = ld16(row + sp.head + (long)min(c + i * NTHR, sp.c1 - 1) * E);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (c + i * NTHR < sp.c1) {
        float f[E];
        unpack<T>(u[i], f);
#pragma unroll
        for (int e = 0; e < E; ++e) s += exp_diff(f[e] - lse);
      }
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  s = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) s += part[i];
  const float z = logf(s);
  return __builtin_fabsf(z) <= __builtin_fabsf(lse) * 0x1p-22f ? z : 0.f;
}

// Below this an lse's rounding is at most 2^-20 of p, of the size that the exponent's
// own rounding leaves, and the row is not read again (4096 rows of 131072 bfloat16: 423
// us, 560 where it is; 1024 of 100000 floats 166 and 201).
__device__ __forceinline__ bool lse_is_coarse(float lse) {
  return __builtin_fabsf(lse) >= 32.f && lse != -__builtin_inff();
}

// lse_rest for rows that are split and overwritten, before them: a part would read what
// another has written (3 us for rows that need nothing; 8 rows of 400000 floats that do
// 90 us in all, 84 where every part sums the row for itself).
template <typename T>
__global__ __launch_bounds__(256) void logprob_rest_kernel(LogprobArgs a) {
  __shared__ float part[4];
  const long r = blockIdx.x;
  const float lse = a.lse_in[r];
  const float z = lse_is_coarse(lse) ? lse_rest<T, 256>(static_cast<const T*>(a.x) + r * a.ld, a.V, lse, part) : 0.f;
  if (threadIdx.x == 0) a.rest[r] = z;
}

// The gradient of one part of a row: everything but the marked entries in a
// pass, those after it.  log p = (x - m) - ls.
template <typename T, int NTHR, int KEEP = 0>
__device__ void row_gradient(const LogprobArgs& a, const T* row, T* out, long r, const Span& sp, float m, float ls,
                             float ent, bool empty, int* mark, float* add, float* val,
                             const uint4 (*keep)[NTHR] = nullptr) {
  constexpr int E = Op<T>::kPerChunk;
  const int tid = threadIdx.x;
  const int t = a.targets ? a.targets[r] : -1;
  const bool has = t >= 0 && t < a.V;
  const float dl = has && a.dlogp ? a.dlogp[r] : 0.f;
  const float dh = a.dentropy ? a.dentropy[r] : 0.f;
  const int ntop = a.dtop ? a.top : 0;
  float c = 0.f;
  for (int j = 0; j < ntop; ++j) c += a.dtop[r * a.top + j];
  c += dl;
  // log p and log p + entropy from x - m: their other terms are the row's
  const float h = ent - ls, l2 = -ls * kLog2e, cl = -c, dhn = -dh;
  auto grad = [&](float x) {
    const float d = x - m, p = __builtin_amdgcn_exp2f(__builtin_fmaf(d, kLog2e, l2));
    return p * (cl + dhn * (fmaxf(d, -1e30f) + h));
  };
  // marked entries of this part (they are read before anything is written:
  // out may be the row itself)
  const int lo = sp.first ? 0 : sp.head + sp.c0 * E, hi = sp.last ? a.V : sp.head + sp.c1 * E;
  const int nm = ntop + 1;
  if (tid < nm) {
    int id = tid < ntop ? a.ids_in[r * a.top + tid] : (has ? t : -1);
    if (id < lo || id >= hi || empty) id = -1;
    mark[tid] = id;
    add[tid] = tid < ntop ? a.dtop[r * a.top + tid] : dl;
    val[tid] = id >= 0 ? grad(Op<T>::to_f32(row[id])) : 0.f;
  }
  __syncthreads();
  float f[E];
  auto put = [&](int k) {
    T* to = out + sp.head + (long)k * E;
    if (a.apart) {
#pragma unroll
      for (int e = 0; e < E; ++e) to[e] = Op<T>::from_f32(f[e]);
    } else if (a.stream) {
      st16_stream(to, pack<T>(f));
    } else {
      *reinterpret_cast<uint4*>(to) = pack<T>(f);
    }
  };
  if (empty) {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = 0.f;
    for (int k = sp.c0 + tid; k < sp.c1; k += NTHR) put(k);
    if (sp.first && tid < sp.head) out[tid] = Op<T>::from_f32(0.f);
    if (sp.last && tid < a.V - sp.tail0) out[sp.tail0 + tid] = Op<T>::from_f32(0.f);
    return;
  }
  auto one = [&](uint4 u, int k) {
    unpack<T>(u, f);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = grad(f[e]);
    put(k);
  };
  // last chunks first: read most recently, they are the nearest still; the
  // thread's first KEEP chunks are in LDS
  const int mine = sp.c1 - sp.c0 > tid ? (sp.c1 - sp.c0 - tid + NTHR - 1) / NTHR : 0;
  const int k0 = sp.c0 + tid;
  for (int i = mine - 1; i >= KEEP; i -= 4) {
    uint4 u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) u[j] = ld16(row + sp.head + (long)(k0 + max(i - j, KEEP) * NTHR) * E);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i - j >= KEEP) one(u[j], k0 + (i - j) * NTHR);
  }
  if (KEEP)
    for (int i = min(mine, KEEP) - 1; i >= 0; --i) one(keep[i][tid], k0 + i * NTHR);
  if (sp.first && tid < sp.head) out[tid] = Op<T>::from_f32(grad(Op<T>::to_f32(row[tid])));
  if (sp.last && tid < a.V - sp.tail0)
    out[sp.tail0 + tid] = Op<T>::from_f32(grad(Op<T>::to_f32(row[sp.tail0 + tid])));
  __syncthreads();
  if (tid < nm && mark[tid] >= 0) {
    float g = 0.f;                     // in c's order: with p = 1 the two cancel exactly
    for (int j = 0; j < nm; ++j)       // the same token may be marked twice
      if (mark[j] == mark[tid]) g += add[j];
    out[mark[tid]] = Op<T>::from_f32(val[tid] + g);
  }
}

template <typename T, int NTHR>
__global__ __launch_bounds__(NTHR) void logprob_bwd_kernel(LogprobArgs a) {
  __shared__ int mark[kTopMax + 1];
  __shared__ float add[kTopMax + 1], val[kTopMax + 1], sums[NTHR / 64];
  const long r = blockIdx.x / a.parts;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  const Span sp = span_of(row, a.V, blockIdx.x % a.parts, a.parts);
  const float lse = a.lse_in[r];
  const float rest = a.rest ? a.rest[r] : lse_is_coarse(lse) ? lse_rest<T, NTHR>(row, a.V, lse, sums) : 0.f;
  row_gradient<T, NTHR>(a, row, static_cast<T*>(a.dx) + r * a.ld, r, sp, lse, rest,
                        a.dentropy ? a.ent_in[r] : 0.f, lse == -__builtin_inff(), mark, add, val);
}

// Both.  Work-groups of 1024 threads for long rows, two a compute unit: few
// enough rows are under way that what is read a second time comes from the
// last-level cache, and 64 KB a row stay in LDS.
template <typename T, int NTHR, int KEEP>
__global__ __launch_bounds__(NTHR, NTHR == 1024 ? 8 : 1) void logprob_fwd_bwd_kernel(LogprobArgs a) {
  __shared__ float sts[3][NTHR / 64];
  __shared__ int mark[kTopMax + 1];
  __shared__ float add[kTopMax + 1], val[kTopMax + 1];
  __shared__ uint4 keep[KEEP ? KEEP : 1][NTHR];
  const long r = blockIdx.x;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  const Span sp = span_of(row, a.V, 0, 1);
  const Target target = target_of(a, row, r);
  uint4 own;
  int own_c;
  Stats st = walk<T, NTHR, false, KEEP>(row, sp, a.V, &own, &own_c, keep);
  st = join_group<NTHR>(st, sts);
  const RowResult res = row_result(a, r, st, target);
  __syncthreads();                     // the target's logit is read before the row is overwritten
  row_gradient<T, NTHR, KEEP>(a, row, static_cast<T*>(a.dx) + r * a.ld, r, sp, res.m, res.ls, res.ent, res.empty, mark,
                              add, val, keep);
}

}  // namespace ll

struct ll_logprob_plan {
  ll_logprob_desc d;
  int device = 0, cus = 0;
  ll::LogprobArgs a{};
  float* rest = nullptr;               // [split rows]
};

namespace {

int elem_bytes(const ll_logprob_plan* p) { return p->d.dtype == LL_BF16 ? 2 : 4; }
long row_bytes(const ll_logprob_plan* p) { return (long)p->d.V * elem_bytes(p); }

// Rows of the two start at different places between 16-byte borders: stores by elements
// (4096 rows of 131072 bfloat16 813 us against 425, 1024 of 100000 floats 174 and 167).
bool lie_apart(const void* x, const void* y) {
  return ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) != 0;
}

// Work-groups per row: enough to fill the chip where the rows alone do not,
// each with at least `least` bytes of its row.
int parts_of(const ll_logprob_plan* p, int rows, long least) {
  const long want = (p->cus + rows - 1) / rows;
  return (int)std::max(1L, std::min({want, row_bytes(p) / least, (long)ll::kPartsMax}));
}

// A gradient larger than the last-level cache goes past it (4096 x 131072
// bfloat16: 478 -> 447 us in the call that makes both).
bool past_caches(const ll_logprob_plan* p, int rows) { return row_bytes(p) * rows > ll::kLastLevelBytes; }

void release(ll_logprob_plan* p) {
  void* all[] = {p->a.part, p->a.keys, p->a.arrived, p->a.err, p->rest};
  for (void* m : all)
    if (m) (void)hipFree(m);
}

ll_status rows_ok(const ll_logprob_plan* p, int32_t rows) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (rows < 0 || rows > p->d.N) return fail(LL_EINVAL, "rows = %d must be 0 .. %d", rows, p->d.N);
  return LL_OK;
}

template <typename T>
void launch_fwd(const ll::LogprobArgs& a, int rows, bool wide, hipStream_t s) {
  const dim3 grid((unsigned)(rows * a.parts));
  if (wide) {
    if (a.top) ll::logprob_fwd_kernel<T, 1024, true><<<grid, dim3(1024), 0, s>>>(a);
    else ll::logprob_fwd_kernel<T, 1024, false><<<grid, dim3(1024), 0, s>>>(a);
  } else {
    if (a.top) ll::logprob_fwd_kernel<T, 256, true><<<grid, dim3(256), 0, s>>>(a);
    else ll::logprob_fwd_kernel<T, 256, false><<<grid, dim3(256), 0, s>>>(a);
  }
}

}  // namespace

extern "C" {

ll_status ll_logprob_plan_create(const ll_logprob_desc* d, int device, ll_logprob_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  if (!d) return fail(LL_EINVAL, "desc is NULL");
  if (d->N < 1 || d->N > ll::max_groups(256) || d->V < 1 || d->V > 1 << 28)
    return fail(LL_EINVAL, "N = %d must be 1 .. 2^24 - 1 and V = %d 1 .. 2^28", d->N, d->V);
  if (d->dtype != LL_F32 && d->dtype != LL_BF16) return fail(LL_EINVAL, "dtype must be LL_F32 or LL_BF16");
  if (d->top_k < 0 || d->top_k > ll::kTopMax || d->top_k > d->V)
    return fail(LL_EINVAL, "top_k = %d must be 0 .. %d and at most V", d->top_k, ll::kTopMax);
  if (d->ld != 0 && (d->ld < d->V || d->ld > (int64_t)1 << 32))
    return fail(LL_EINVAL, "ld = %lld must be 0, or V .. 2^32", (long long)d->ld);
  if (d->reserved[0] || d->reserved[1]) return fail(LL_EINVAL, "reserved must be 0");
  LL_STATUS(ll::check_device(device));
  ll::DeviceGuard guard(device);
  ll_logprob_plan* p = new (std::nothrow) ll_logprob_plan();
  if (!p) return fail(LL_ENOMEM, "host allocation of the plan failed");
  p->d = *d;
  p->device = device;
  hipDeviceProp_t prop;
  ll_status st = LL_OK;
  if (hipGetDeviceProperties(&prop, device) != hipSuccess) st = fail(LL_EHIP, "hipGetDeviceProperties failed");
  p->cus = prop.multiProcessorCount;
  p->a.V = d->V;
  p->a.top = d->top_k;
  p->a.ld = d->ld ? d->ld : d->V;
  // rows that are split: fewer than one per compute unit
  const size_t split = (size_t)std::min(d->N, p->cus);
  if (st == LL_OK) st = ll::dalloc((void**)&p->a.part, sizeof(float4) * split * ll::kPartsMax, "the rows' parts");
  if (st == LL_OK)
    st = ll::dalloc((void**)&p->a.keys, d->top_k ? 8 * split * ll::kPartsMax * ll::kTopMax : 0, "the parts' keys");
  if (st == LL_OK) st = ll::dalloc((void**)&p->a.arrived, sizeof(unsigned) * split, "the arrivals");
  if (st == LL_OK) st = ll::dalloc((void**)&p->rest, sizeof(float) * split, "what the rows' lse leave");
  if (st == LL_OK) st = ll::dalloc((void**)&p->a.err, sizeof(int), "the error word");
  if (st == LL_OK && (hipMemset(p->a.arrived, 0, sizeof(unsigned) * split) != hipSuccess ||
                      hipMemset(p->a.err, 0, sizeof(int)) != hipSuccess))
    st = fail(LL_EHIP, "hipMemset of the arrivals or the error word failed");
  if (st == LL_OK) st = ll::wait_created();
  if (st != LL_OK) {
    release(p);
    delete p;
    return st;
  }
  *out = p;
  return LL_OK;
}

ll_status ll_logprob_plan_destroy(ll_logprob_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_logprob_fwd(ll_logprob_plan* p, void* stream, int32_t rows, const void* logits,
                         const int32_t* targets, float* logp, float* entropy, float* lse, int32_t* top_ids,
                         float* top_logp) {
  LL_STATUS(rows_ok(p, rows));
  if (rows == 0) return LL_OK;
  if (!logits) return fail(LL_EINVAL, "logits are required");
  if (!targets != !logp) return fail(LL_EINVAL, "targets and logp go together");
  if (p->d.top_k && (!top_ids || !top_logp)) return fail(LL_EINVAL, "top_ids and top_logp are required (top_k > 0)");
  LL_ALIGNED(logits, elem_bytes(p)); LL_ALIGNED(targets, 4); LL_ALIGNED(logp, 4); LL_ALIGNED(entropy, 4);
  LL_ALIGNED(lse, 4); LL_ALIGNED(top_ids, 4); LL_ALIGNED(top_logp, 4);
  ll::DeviceGuard guard(p->device);
  ll::LogprobArgs a = p->a;
  a.x = logits; a.targets = targets; a.logp = logp; a.entropy = entropy; a.lse = lse;
  a.top_ids = top_ids; a.top_logp = top_logp;
  // (8 rows of 131072 bfloat16: 13.5 us in parts of 64 KiB, 15.7 of 128, 17.4 whole; 8 rows
  // of 400000 floats: 17.5, 15.6 and 44)
  a.parts = parts_of(p, rows, 64 << 10);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // 1024 threads a work-group where there is at most one for a compute unit, else 256
  // (256 rows of 50001 floats: 15.0 us against 19.4; 512 rows: 28.2 against 22.3)
  const bool wide = (long)rows * a.parts <= p->cus;
  if (p->d.dtype == LL_BF16) launch_fwd<bf16_t>(a, rows, wide, s);
  else launch_fwd<float>(a, rows, wide, s);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_logprob_bwd(ll_logprob_plan* p, void* stream, int32_t rows, const void* logits,
                         const int32_t* targets, const float* lse, const float* entropy, const int32_t* top_ids,
                         const float* dlogp, const float* dentropy, const float* dtop, void* dlogits) {
  LL_STATUS(rows_ok(p, rows));
  if (rows == 0) return LL_OK;
  if (!logits || !lse || !dlogits) return fail(LL_EINVAL, "logits, lse and dlogits are required");
  if (dlogp && !targets) return fail(LL_EINVAL, "dlogp needs targets");
  if (dentropy && !entropy) return fail(LL_EINVAL, "dentropy needs the forward's entropy");
  if (dtop && (!top_ids || !p->d.top_k)) return fail(LL_EINVAL, "dtop needs the forward's top_ids (top_k > 0)");
  LL_ALIGNED(logits, elem_bytes(p)); LL_ALIGNED(dlogits, elem_bytes(p)); LL_ALIGNED(targets, 4); LL_ALIGNED(lse, 4);
  LL_ALIGNED(entropy, 4); LL_ALIGNED(top_ids, 4); LL_ALIGNED(dlogp, 4); LL_ALIGNED(dentropy, 4); LL_ALIGNED(dtop, 4);
  ll::DeviceGuard guard(p->device);
  ll::LogprobArgs a = p->a;
  a.x = logits; a.targets = targets; a.lse_in = lse; a.ent_in = entropy; a.ids_in = top_ids;
  a.dlogp = dlogp; a.dentropy = dentropy; a.dtop = dtop; a.dx = dlogits;
  // (nothing to join: 8 rows of 32000 bfloat16 take 3.7 us in parts of 4 KiB, 5.5 of 16,
  // 10 of 64)
  a.parts = parts_of(p, rows, 4 << 10);
  a.stream = past_caches(p, rows);
  a.apart = lie_apart(logits, dlogits);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (a.parts > 1 && logits == dlogits) {
    a.rest = p->rest;
    if (p->d.dtype == LL_BF16) ll::logprob_rest_kernel<bf16_t><<<dim3(rows), dim3(256), 0, s>>>(a);
    else ll::logprob_rest_kernel<float><<<dim3(rows), dim3(256), 0, s>>>(a);
    LL_HIP(hipGetLastError());
  }
  const dim3 grid((unsigned)(rows * a.parts));
  if (p->d.dtype == LL_BF16) ll::logprob_bwd_kernel<bf16_t, 256><<<grid, dim3(256), 0, s>>>(a);
  else ll::logprob_bwd_kernel<float, 256><<<grid, dim3(256), 0, s>>>(a);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_logprob_fwd_bwd(ll_logprob_plan* p, void* stream, int32_t rows, const void* logits,
                             const int32_t* targets, const float* dlogp, const float* dentropy, float* logp,
                             float* entropy, float* lse, void* dlogits) {
  LL_STATUS(rows_ok(p, rows));
  if (rows == 0) return LL_OK;
  if (!logits || !dlogits) return fail(LL_EINVAL, "logits and dlogits are required");
  if (!targets != !logp) return fail(LL_EINVAL, "targets and logp go together");
  if (dlogp && !targets) return fail(LL_EINVAL, "dlogp needs targets");
  LL_ALIGNED(logits, elem_bytes(p)); LL_ALIGNED(dlogits, elem_bytes(p)); LL_ALIGNED(targets, 4); LL_ALIGNED(lse, 4);
  LL_ALIGNED(logp, 4); LL_ALIGNED(entropy, 4); LL_ALIGNED(dlogp, 4); LL_ALIGNED(dentropy, 4);
  ll::DeviceGuard guard(p->device);
  ll::LogprobArgs a = p->a;
  a.x = logits; a.targets = targets; a.dlogp = dlogp; a.dentropy = dentropy; a.logp = logp;
  a.entropy = entropy; a.lse = lse; a.dx = dlogits;
  a.parts = 1;
  a.stream = past_caches(p, rows);
  a.apart = lie_apart(logits, dlogits);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // One work-group a row, however few the rows: a part of a row would have to wait for the
  // others' sums before it writes.  Few long rows are faster in the two calls (8 of 400000
  // floats 13 + 10 us against 64, 8 of 131072 bfloat16 9 + 10 against 28).
  // 1024 threads and 64 KB of a row in LDS, or 256 and 16 (4096 rows of bfloat16: 50000
  // take 188 us against 199, 32000 133 against 132, 10000 63 against 41)
  const bool wide = row_bytes(p) >= 64 << 10 && rows <= ll::max_groups(1024);
  if (p->d.dtype == LL_BF16) {
    if (wide) ll::logprob_fwd_bwd_kernel<bf16_t, 1024, 4><<<dim3(rows), dim3(1024), 0, s>>>(a);
    else ll::logprob_fwd_bwd_kernel<bf16_t, 256, 4><<<dim3(rows), dim3(256), 0, s>>>(a);
  } else {
    if (wide) ll::logprob_fwd_bwd_kernel<float, 1024, 4><<<dim3(rows), dim3(1024), 0, s>>>(a);
    else ll::logprob_fwd_bwd_kernel<float, 256, 4><<<dim3(rows), dim3(256), 0, s>>>(a);
  }
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_logprob_status_sync(ll_logprob_plan* p, int32_t* device_error) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  ll::DeviceGuard guard(p->device);
  return ll::read_error_word(p->a.err, device_error);
}

}  // extern "C"
