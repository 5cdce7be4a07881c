// Beam search: the K best continuations of each search's K beams, and the states of the
// beams in the order of their successors.
//
// Selection.  A candidate (beam k, token v) has the score s = score_k + log p_kv and the
// rank s / ((5 + length) / 6)^alpha; a finished beam is one candidate, as it is.  The K
// best of all candidates of a search are among the K best logits of its beams, so one
// walk over the logits (ll_rows.h) keeps each row's sum and its K largest, and a second,
// small kernel compares those.  Scores of one beam can lie as close as its logits' rounding:
// they are made and compared in double from the walk's m and s.  s is a float's sum, so
// that candidates of different beams nearer than some 1e-6 may change places.
// Equal ranks: lower beam, then lower token.
//
// Reordering in place: a thread has the same few bytes of all K rows, so it reads what it
// needs before it writes.  In a pool (rows by slots) no row moves that need not: a beam's
// first successor takes its slot over, the further ones copy the state into the slots of
// beams without a successor.  A beam without a state (slot -1) has successors without one.
#include <algorithm>
#include <cmath>
#include <new>

#include "ll_host.h"
#include "ll_rows.h"
#include "ll_stream.h"

using ll::bf16_t;
using ll::fail;

namespace ll {

constexpr int kBeamMax = LL_BEAM_MAX;
static_assert(kBeamMax <= kTopMax, "a row's largest are the walk's");

struct BeamArgs {
  int K, V, top, parts, eos;
  long ld;
  double alpha;
  const void* x;
  const float* scores;
  const int *finished, *lengths;
  int *parents, *tokens;
  float* scores_out;
  int *finished_out, *lengths_out;
  float2* part;                        // [row, part] m, s
  unsigned long long* keys;            // [row, part, top]
  int* err;
};

// Whether a row's logits count: its beam goes on.
__device__ __forceinline__ bool beam_live(const BeamArgs& a, long r) {
  return a.scores[r] > -__builtin_inff() && !(a.finished && a.finished[r]);
}

// A part of a row: its sum and its K largest.  Bound by the walk over the logits: its
// bytes, and beside them 13 vector instructions an element, which are issued in 72 % of the
// cycles in which a compute unit has a wave; what comes before and after the walk overlaps
// with nothing where a work-group has a compute unit to itself.  256 rows of 131072
// bfloat16, of which 209 are read, in 19.1 us, 2.9 TB/s (21.1 when the walk made the
// entropy's sum too); 240 of 50001 floats, 198 read, in 14.9, 2.7 TB/s.
template <typename T, int NTHR>
__global__ __launch_bounds__(NTHR) void beam_rows_kernel(BeamArgs a) {
  __shared__ Shared<NTHR> sh;
  const int tid = threadIdx.x, part = blockIdx.x % a.parts;
  const long r = blockIdx.x / a.parts;
  if (!beam_live(a, r)) return;
  const T* row = static_cast<const T*>(a.x) + r * a.ld;
  const Span sp = span_of(row, a.V, part, a.parts);
  uint4 own;
  int own_c;
  Stats st = walk<T, NTHR, true, 0, false>(row, sp, a.V, &own, &own_c);
  st = join_group<NTHR>(st, sh.st);
  const long at = r * a.parts + part;
  if (tid == 0) a.part[at] = make_float2(st.m, st.s);
  const bool some = st.s > 0.f;        // (a NaN's row offers nothing)
  if (some) select_top<T, NTHR>(row, sp, a.V, a.top, own, own_c, sh);
  if (tid < a.top) a.keys[at * a.top + tid] = some ? sh.top[tid] : 0;
}

struct BeamKey {
  double rank;
  unsigned long long at;               // beam << 32 | token
};
__device__ __forceinline__ bool better(BeamKey a, BeamKey b) { return a.rank > b.rank || (a.rank == b.rank && a.at < b.at); }
constexpr unsigned long long kBeamNone = ~0ull;          // no candidate, its rank below all
constexpr int kBeamJoin = 512;         // threads
// How many of x[0, n) are better than each of them: the threads share the comparisons.
template <typename Use>
__device__ __forceinline__ void beam_places(const BeamKey* x, int n, Use use) {
  int share = 1;
  while (share < 64 && 2 * share * n <= kBeamJoin) share *= 2;
  const int first = threadIdx.x & (share - 1);
  for (int i0 = 0; i0 < n * share; i0 += kBeamJoin) {
    const int i = (i0 + (int)threadIdx.x) / share;
    const BeamKey c = x[min(i, n - 1)];
    int place = 0;
#pragma unroll 4
    for (int j = first; j < n; j += share) place += better(x[j], c);
    for (int d = 1; d < share; d <<= 1) place += __shfl_xor(place, d, 64);
    if (i < n && first == 0) use(c, place);
  }
}

// The K best of a search's candidates.  What the first step reads goes out at once, also
// for beams that turn out to offer nothing: the kernel is a handful of trips to memory.
// 32 searches of 8 beams take 5.8 us (9.5 when a thread made all of a candidate's
// comparisons, 14.4 with each beam's values one after the other).
__global__ __launch_bounds__(kBeamJoin) void beam_join_kernel(BeamArgs a) {
  __shared__ float2 all[kBeamMax];
  __shared__ double base[kBeamMax], off[kBeamMax], sum[kBeamMax], pen[kBeamMax];
  __shared__ int kind[kBeamMax], len[kBeamMax];          // 0: offers nothing, 1: its tokens, 2: itself
  __shared__ BeamKey head[kBeamMax * kPartsMax], found[kBeamMax * kBeamMax], bound;
  __shared__ int count;
  const int tid = threadIdx.x, K = a.K, lists = K * a.parts;
  const long r0 = (long)blockIdx.x * K;
  const unsigned long long* keys = a.keys + r0 * a.parts * a.top;
  const unsigned long long early = tid < lists * a.top ? keys[tid] : 0;
  float score = 0.f;
  bool done = false;
  int old = 0;
  if (tid < K) {
    score = a.scores[r0 + tid];
    done = a.finished && a.finished[r0 + tid];
    old = a.lengths ? a.lengths[r0 + tid] : 0;
  }
  for (int k = tid / kPartsMax; k < K; k += kBeamJoin / kPartsMax) {
    const int l = tid % kPartsMax;
    const float2 p = a.part[(r0 + k) * a.parts + min(l, a.parts - 1)];
    Stats st = l < a.parts ? Stats{p.x, p.y, 0.f} : Stats{kLowest, 0.f, 0.f};
#pragma unroll
    for (int d = 1; d < kPartsMax; d <<= 1)
      st = join(st, Stats{__shfl_xor(st.m, d, 64), __shfl_xor(st.s, d, 64), 0.f});
    if (l == 0) all[k] = make_float2(st.m, st.s);
  }
  __syncthreads();
  if (tid < K) {
    const bool live = score > -__builtin_inff() && !done;          // as beam_live
    const float2 st = live ? all[tid] : make_float2(0.f, 0.f);
    const bool bad = score != score || st.y != st.y;
    if (bad) atomicOr(a.err, LL_DEVERR_BEAM);
    const bool walked = live && !bad && st.y > 0.f;
    kind[tid] = walked ? 1 : !bad && done && score > -__builtin_inff() ? 2 : 0;
    len[tid] = done ? max(0, old) : min(max(0, old), 0x7ffffffe) + 1;
    base[tid] = score;
    off[tid] = walked ? (double)st.x : 0.0;
    sum[tid] = walked ? log((double)st.y) : 0.0;
    pen[tid] = a.alpha != 0.0 ? pow((5.0 + len[tid]) / 6.0, a.alpha) : 1.0;
  }
  if (tid == 0) {
    count = 0;
    bound = BeamKey{-__builtin_inf(), kBeamNone};
  }
  __syncthreads();
  // entry j of list i = beam * parts + part, whose key is given
  auto entry = [&](int i, int j, unsigned long long key) {
    const int k = i / a.parts;
    BeamKey c{-__builtin_inf(), kBeamNone};
    if (kind[k] == 2) {
      if (i % a.parts == 0 && j == 0) c = BeamKey{base[k] / pen[k], (unsigned long long)k << 32 | max(a.eos, 0)};
    } else if (kind[k] == 1) {
      const float x = key_value(key);
      if (key != 0 && x > -__builtin_inff())
        c = BeamKey{(base[k] + (((double)x - off[k]) - sum[k])) / pen[k],
                    (unsigned long long)k << 32 | (unsigned)key_index(key)};
    }
    return c;
  };
  const bool few = lists * a.top <= kBeamJoin;           // a candidate a thread: all compared at once
  if (!few) {
    for (int i = tid; i < lists; i += kBeamJoin) head[i] = entry(i, 0, keys[i * a.top]);
    __syncthreads();
    // the K-th best of the lists' first ones bounds the K-th best of all
    beam_places(head, lists, [&](BeamKey c, int place) {
      if (place == K - 1 && c.at != kBeamNone) bound = c;
    });
    __syncthreads();
  }
  const BeamKey least = bound;
  for (int i = tid; i < lists * a.top; i += kBeamJoin) {
    if (!few && better(least, head[i / a.top])) continue;
    const BeamKey c = entry(i / a.top, i % a.top, few ? early : keys[i]);
    if (c.at != kBeamNone && !better(least, c)) found[atomicAdd(&count, 1)] = c;
  }
  __syncthreads();
  const int n = count;
  beam_places(found, n, [&](BeamKey c, int place) {
    if (place >= K) return;
    const long at = r0 + place;
    const int k = (int)(c.at >> 32), t = (int)(unsigned)c.at;
    a.parents[at] = k;
    a.tokens[at] = kind[k] == 2 ? a.eos : t;
    a.scores_out[at] = (float)(c.rank * pen[k]);
    if (a.finished_out) a.finished_out[at] = kind[k] == 2 || t == a.eos;
    if (a.lengths_out) a.lengths_out[at] = len[k];
  });
  // places for which there is no candidate
  if (tid >= n && tid < K) {
    a.parents[r0 + tid] = tid;
    a.tokens[r0 + tid] = -1;
    a.scores_out[r0 + tid] = -__builtin_inff();
    if (a.finished_out) a.finished_out[r0 + tid] = 0;
    if (a.lengths_out) a.lengths_out[r0 + tid] = old;
  }
}

constexpr int kBeamTensors = 32;       // of a launch
constexpr int kBeamSlice = 32 << 10;   // bytes of a row that a work-group moves in a pool
struct BeamMove {
  int B, K, n, n_slots;
  const int *parents, *slots;
  int* slots_out;
  int* err;
  struct {
    char* data;
    long row;                          // bytes
    int unit, first;                   // bytes moved at once; number of its first slice
  } t[kBeamTensors];
};

// The parent of place k; one outside [0, K) counts as k itself.
__device__ __forceinline__ int beam_parent(const BeamMove& a, int b, int k, bool tell) {
  const int p = a.parents[(long)b * a.K + k];
  if (p >= 0 && p < a.K) return p;
  if (tell && a.err) atomicOr(a.err, LL_DEVERR_BEAM);
  return k;
}

template <typename U, int KM>
__device__ void beam_rows_in_place(const BeamMove& a, char* data, long row, int K, const int* from, long u0) {
  const long units = row / (long)sizeof(U), u = u0 + threadIdx.x;
  if (u >= units) return;
  U* x = reinterpret_cast<U*>(data) + u;
  U v[KM];
#pragma unroll
  for (int k = 0; k < KM; ++k)
    if (k < K && from[k] != k) v[k] = x[from[k] * units];
#pragma unroll
  for (int k = 0; k < KM; ++k)
    if (k < K && from[k] != k) x[k * units] = v[k];
}

template <int KM>
__global__ __launch_bounds__(256) void beam_rows_move_kernel(BeamMove a) {
  __shared__ int from[KM];
  const int b = blockIdx.y + gridDim.y * blockIdx.z, tid = threadIdx.x;
  if (b >= a.B) return;
  if (tid < a.K) from[tid] = beam_parent(a, b, tid, blockIdx.x == 0);
  __syncthreads();
  int i = 0;
  while (i + 1 < a.n && (int)blockIdx.x >= a.t[i + 1].first) ++i;
  const long u0 = (long)(blockIdx.x - a.t[i].first) * 256, row = a.t[i].row;
  char* data = a.t[i].data + (long)b * a.K * row;
  switch (a.t[i].unit) {
    case 16: beam_rows_in_place<u32x4, KM>(a, data, row, a.K, from, u0); break;
    case 4: beam_rows_in_place<uint32_t, KM>(a, data, row, a.K, from, u0); break;
    case 2: beam_rows_in_place<uint16_t, KM>(a, data, row, a.K, from, u0); break;
    default: beam_rows_in_place<uint8_t, KM>(a, data, row, a.K, from, u0); break;
  }
}

template <typename U>
__device__ void beam_copy(char* to, const char* from, long bytes) {
  constexpr int R = 8;
  const int n = (int)(bytes / (long)sizeof(U));
  const U* x = reinterpret_cast<const U*>(from);
  U* y = reinterpret_cast<U*>(to);
  for (int i = threadIdx.x; i < n; i += R * 256) {
    U v[R];
#pragma unroll
    for (int j = 0; j < R; ++j) v[j] = x[min(i + j * 256, n - 1)];
#pragma unroll
    for (int j = 0; j < R; ++j)
      if (i + j * 256 < n) y[i + j * 256] = v[j];
  }
}

// Place k of search b, one slice of a tensor's row.  Bound by the copies: 256 places of
// 1 MiB of which 105 move take 33 us, 6.7 TB/s read and written; what does not
// move costs its work-group three trips to memory (4 us where nothing moves).
__global__ __launch_bounds__(256) void beam_pool_move_kernel(BeamMove a) {
  const int place = blockIdx.y + gridDim.y * blockIdx.z;
  if (place >= a.B * a.K) return;
  const int b = place / a.K, k = place % a.K, l = threadIdx.x & 63;
  const bool in = l < a.K, tell = blockIdx.x == 0 && k == 0 && threadIdx.x < 64;
  const bool tell_place = blockIdx.x == 0 && threadIdx.x == 0;
  const int* slots = a.slots + (long)b * a.K;
  const int slot = in ? slots[l] : -1, p = in ? beam_parent(a, b, l, tell) : -1;
  if (tell && in && (slot < -1 || slot >= a.n_slots) && a.err) atomicOr(a.err, LL_DEVERR_SLOT);
  // places after the first successor of their beam, and beams without any
  unsigned long long again = 0, childless = 0;
  for (int j = 0; j < a.K; ++j) {
    const unsigned long long m = __ballot(p == j);
    if (m) again |= m & (m - 1);
    else childless |= 1ull << j;
  }
  // the former need a slot where their beam has a state, the latter offer theirs, in order
  const int old = __shfl(slot, p, 64);
  const unsigned long long needs = again & __ballot(in && old >= 0 && old < a.n_slots);
  childless &= ~__ballot(slot == -1);
  const int src = __shfl(old, k, 64);
  int dst = src;
  if (again >> k & 1) {
    for (int j = __popcll(needs & ((1ull << k) - 1)); j > 0; --j) childless &= childless - 1;
    const bool some = needs >> k & 1 && childless != 0;
    const int free = __shfl(slot, some ? __ffsll(childless) - 1 : 0, 64);
    dst = some ? free : -1;
    if (tell_place && needs >> k & 1 && !some && a.err) atomicOr(a.err, LL_DEVERR_SLOT);
  }
  if (tell_place && a.slots_out) a.slots_out[place] = dst;
  if (dst == src || a.n == 0 || src < 0 || dst < 0 || src >= a.n_slots || dst >= a.n_slots) return;
  int i = 0;
  while (i + 1 < a.n && (int)blockIdx.x >= a.t[i + 1].first) ++i;
  const long row = a.t[i].row, at = (long)(blockIdx.x - a.t[i].first) * kBeamSlice;
  const long bytes = min((long)kBeamSlice, row - at);
  char* to = a.t[i].data + dst * row + at;
  const char* from = a.t[i].data + src * row + at;
  switch (a.t[i].unit) {
    case 16: beam_copy<u32x4>(to, from, bytes); break;
    case 4: beam_copy<uint32_t>(to, from, bytes); break;
    case 2: beam_copy<uint16_t>(to, from, bytes); break;
    default: beam_copy<uint8_t>(to, from, bytes); break;
  }
}

}  // namespace ll

struct ll_beam_plan {
  ll_beam_desc d;
  int device = 0, cus = 0;
  ll::BeamArgs a{};
};

namespace {

int elem_bytes(const ll_beam_plan* p) { return p->d.dtype == LL_BF16 ? 2 : 4; }

void release(ll_beam_plan* p) {
  void* all[] = {p->a.part, p->a.keys, p->a.err};
  for (void* m : all)
    if (m) (void)hipFree(m);
}

template <typename T>
void launch_rows(const ll::BeamArgs& a, int rows, bool wide, hipStream_t s) {
  const dim3 grid((unsigned)(rows * a.parts));
  if (wide) ll::beam_rows_kernel<T, 1024><<<grid, dim3(1024), 0, s>>>(a);
  else ll::beam_rows_kernel<T, 256><<<grid, dim3(256), 0, s>>>(a);
}

// Bytes of a tensor of `rows` rows (more than there are addresses: all of them).
uint64_t bytes_of(const ll_beam_tensor& t, uint64_t rows) {
  uint64_t n;
  return __builtin_mul_overflow(rows, (uint64_t)t.row_bytes, &n) ? ~0ull : n;
}
bool overlap(const void* x, uint64_t nx, const void* y, uint64_t ny) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
  return a <= b ? b - a < nx : a - b < ny;
}

// Bytes moved at once, and the work-groups that move a row.
int unit_of(const ll_beam_tensor& t) {
  const uintptr_t both = reinterpret_cast<uintptr_t>(t.data) | (uintptr_t)t.row_bytes;
  return both % 16 == 0 ? 16 : both % 4 == 0 ? 4 : both % 2 == 0 ? 2 : 1;
}
int64_t slices_of(const ll_beam_tensor& t, bool pool) {
  const int64_t each = pool ? ll::kBeamSlice : 256 * unit_of(t);
  return (t.row_bytes + each - 1) / each;
}

template <int KM>
void launch_in_place(const ll::BeamMove& m, dim3 grid, hipStream_t s) {
  ll::beam_rows_move_kernel<KM><<<grid, dim3(256), 0, s>>>(m);
}

}  // namespace

extern "C" {

ll_status ll_beam_plan_create(const ll_beam_desc* d, int device, ll_beam_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  if (!d) return fail(LL_EINVAL, "desc is NULL");
  if (d->K < 1 || d->K > ll::kBeamMax || d->B < 1 || (int64_t)d->B * d->K > 1 << 20 || d->V < 1 || d->V > 1 << 28)
    return fail(LL_EINVAL, "K = %d must be 1 .. %d, B = %d at least 1 with B * K at most 2^20, V = %d 1 .. 2^28", d->K,
                ll::kBeamMax, d->B, d->V);
  if (d->dtype != LL_F32 && d->dtype != LL_BF16) return fail(LL_EINVAL, "dtype must be LL_F32 or LL_BF16");
  if (d->ld != 0 && (d->ld < d->V || d->ld > (int64_t)1 << 32))
    return fail(LL_EINVAL, "ld = %lld must be 0, or V .. 2^32", (long long)d->ld);
  if (d->eos < -1 || d->eos >= d->V) return fail(LL_EINVAL, "eos = %d must be -1, or a token below V = %d", d->eos, d->V);
  if (!(std::fabs(d->length_penalty) <= 16.f))
    return fail(LL_EINVAL, "length_penalty = %g must be -16 .. 16", (double)d->length_penalty);
  if (d->reserved[0] || d->reserved[1]) return fail(LL_EINVAL, "reserved must be 0");
  LL_STATUS(ll::check_device(device));
  ll::DeviceGuard guard(device);
  ll_beam_plan* p = new (std::nothrow) ll_beam_plan();
  if (!p) return fail(LL_ENOMEM, "host allocation of the plan failed");
  p->d = *d;
  p->device = device;
  hipDeviceProp_t prop;
  ll_status st = LL_OK;
  if (hipGetDeviceProperties(&prop, device) != hipSuccess) st = fail(LL_EHIP, "hipGetDeviceProperties failed");
  p->cus = prop.multiProcessorCount;
  ll::BeamArgs& a = p->a;
  a.K = d->K; a.V = d->V; a.eos = d->eos;
  a.top = std::min(d->K, d->V);
  a.ld = d->ld ? d->ld : d->V;
  a.alpha = d->length_penalty;
  const size_t parts = (size_t)d->B * d->K + p->cus;     // rows times parts of a call, at most
  if (st == LL_OK) st = ll::dalloc((void**)&a.part, sizeof(float2) * parts, "the rows' parts");
  if (st == LL_OK) st = ll::dalloc((void**)&a.keys, 8 * parts * a.top, "the parts' keys");
  if (st == LL_OK) st = ll::dalloc((void**)&a.err, sizeof(int), "the error word");
  if (st == LL_OK && hipMemset(a.err, 0, sizeof(int)) != hipSuccess)
    st = fail(LL_EHIP, "hipMemset of the error word failed");
  if (st == LL_OK) st = ll::wait_created();
  if (st != LL_OK) {
    release(p);
    delete p;
    return st;
  }
  *out = p;
  return LL_OK;
}

ll_status ll_beam_plan_destroy(ll_beam_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_beam_select(ll_beam_plan* p, void* stream, int32_t searches, const void* logits, const float* scores,
                         const int32_t* finished, const int32_t* lengths, int32_t* parents, int32_t* tokens,
                         float* scores_out, int32_t* finished_out, int32_t* lengths_out) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (searches < 0 || searches > p->d.B) return fail(LL_EINVAL, "searches = %d must be 0 .. %d", searches, p->d.B);
  if (searches == 0) return LL_OK;
  if (!logits || !scores || !parents || !tokens || !scores_out)
    return fail(LL_EINVAL, "logits, scores, parents, tokens and scores_out are required");
  if (!lengths && p->d.length_penalty != 0.f) return fail(LL_EINVAL, "the length penalty needs the beams' lengths");
  LL_ALIGNED(logits, elem_bytes(p)); LL_ALIGNED(scores, 4); LL_ALIGNED(finished, 4); LL_ALIGNED(lengths, 4);
  LL_ALIGNED(parents, 4); LL_ALIGNED(tokens, 4); LL_ALIGNED(scores_out, 4); LL_ALIGNED(finished_out, 4);
  LL_ALIGNED(lengths_out, 4);
  ll::DeviceGuard guard(p->device);
  ll::BeamArgs a = p->a;
  a.x = logits; a.scores = scores; a.finished = finished; a.lengths = lengths;
  a.parents = parents; a.tokens = tokens; a.scores_out = scores_out;
  a.finished_out = finished_out; a.lengths_out = lengths_out;
  const int rows = searches * p->d.K;
  // A work-group a compute unit, none of less than 32 KiB.  (Rows, join: 4 rows of 32000
  // floats 8.0 + 4.2 us, in parts of 64 KiB 9.3 + 3.9, of 16 KiB 8.7 + 6.0; 256 rows of
  // 131072 bfloat16, 209 of them read, 19.1 us, with two work-groups a compute unit 20.7.)
  const long want = (p->cus + rows - 1) / rows, row = (long)p->d.V * elem_bytes(p);
  a.parts = (int)std::max(1L, std::min({want, row / (32 << 10), (long)ll::kPartsMax}));
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  // (240 rows of 50001 floats in two parts: 14.6 us by 256 threads, 19.8 by 1024)
  const bool wide = (long)rows * a.parts <= p->cus;
  if (p->d.dtype == LL_BF16) launch_rows<bf16_t>(a, rows, wide, s);
  else launch_rows<float>(a, rows, wide, s);
  LL_HIP(hipGetLastError());
  ll::beam_join_kernel<<<dim3(searches), dim3(ll::kBeamJoin), 0, s>>>(a);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

ll_status ll_beam_reorder(void* stream, int32_t searches, int32_t K, const int32_t* parents, int32_t n_tensors,
                          const ll_beam_tensor* tensors, const int32_t* slots, int32_t n_slots, int32_t* slots_out,
                          int32_t* device_error) {
  if (searches < 0 || K < 1 || K > ll::kBeamMax || (int64_t)searches * K > 1 << 20)
    return fail(LL_EINVAL, "searches = %d must be at least 0 and K = %d 1 .. %d, their product at most 2^20", searches, K,
                ll::kBeamMax);
  if (n_tensors < 0 || n_tensors > LL_BEAM_TENSORS)
    return fail(LL_EINVAL, "n_tensors = %d must be 0 .. %d", n_tensors, LL_BEAM_TENSORS);
  if (!parents || (n_tensors && !tensors)) return fail(LL_EINVAL, "parents and tensors are required");
  if (!slots != !slots_out) return fail(LL_EINVAL, "slots and slots_out go together");
  if (slots && n_slots < 1) return fail(LL_EINVAL, "n_slots = %d must be at least 1", n_slots);
  LL_ALIGNED(parents, 4); LL_ALIGNED(slots, 4); LL_ALIGNED(slots_out, 4); LL_ALIGNED(device_error, 4);
  const uint64_t rows = slots ? n_slots : (int64_t)searches * K, list = 4ull * searches * K;
  if (slots && (overlap(slots_out, list, slots, list) || overlap(slots_out, list, parents, list)))
    return fail(LL_EINVAL, "slots_out overlaps slots or parents: it must be another array");
  for (int i = 0; i < n_tensors; ++i) {
    const ll_beam_tensor& t = tensors[i];
    if (!t.data || t.row_bytes < 1 || t.row_bytes > (int64_t)1 << 36)
      return fail(LL_EINVAL, "tensors[%d]: data is NULL or row_bytes = %lld is not 1 .. 2^36", i, (long long)t.row_bytes);
    const uint64_t bytes = bytes_of(t, rows);
    for (const int32_t* x : {parents, slots, (const int32_t*)slots_out})
      if (x && overlap(t.data, bytes, x, list))
        return fail(LL_EINVAL, "tensors[%d] overlaps %s", i, x == parents ? "parents" : x == slots ? "slots" : "slots_out");
    for (int j = 0; j < i; ++j)
      if (overlap(t.data, bytes, tensors[j].data, bytes_of(tensors[j], rows)))
        return fail(LL_EINVAL, "tensors[%d] and tensors[%d] overlap", j, i);
  }
  if (searches == 0) return LL_OK;
  // blocks times searches (places) in 2^32 work-items; tensors go to as many launches as
  // hold them, all of them counted before the first
  const int64_t outer = slots ? (int64_t)searches * K : searches;
  const int64_t z = (outer + 32767) / 32768, y = (outer + z - 1) / z;
  const int64_t most = ll::max_groups(256) / (y * z);
  int first[LL_BEAM_TENSORS + 1] = {0}, launches = 0;
  int64_t blocks = 0;
  for (int i = 0; i < n_tensors; ++i) {
    const int64_t n = slices_of(tensors[i], slots != nullptr);
    if (n > most)
      return fail(LL_EUNSUPPORTED, "tensors[%d]: %lld slices of %lld rows are more than a launch holds (%lld)", i,
                  (long long)n, (long long)(y * z), (long long)ll::max_groups(256));
    if (i - first[launches] == ll::kBeamTensors || blocks + n > most) {
      first[++launches] = i;
      blocks = 0;
    }
    blocks += n;
  }
  if (n_tensors || slots) first[++launches] = n_tensors;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  for (int j = 0; j < launches; ++j) {
    ll::BeamMove m{};
    m.B = searches; m.K = K; m.n_slots = n_slots;
    m.parents = parents; m.slots = slots; m.slots_out = j == 0 ? slots_out : nullptr; m.err = device_error;
    m.n = first[j + 1] - first[j];
    blocks = 0;
    for (int i = 0; i < m.n; ++i) {
      const ll_beam_tensor& t = tensors[first[j] + i];
      m.t[i].data = static_cast<char*>(t.data);
      m.t[i].row = t.row_bytes;
      m.t[i].unit = unit_of(t);
      m.t[i].first = (int)blocks;
      blocks += slices_of(t, slots != nullptr);
    }
    const dim3 grid((unsigned)std::max<int64_t>(blocks, 1), (unsigned)y, (unsigned)z);
    if (slots) ll::beam_pool_move_kernel<<<grid, dim3(256), 0, s>>>(m);
    else if (K <= 4) launch_in_place<4>(m, grid, s);
    else if (K <= 8) launch_in_place<8>(m, grid, s);
    else if (K <= 16) launch_in_place<16>(m, grid, s);
    else launch_in_place<32>(m, grid, s);
    LL_HIP(hipGetLastError());
  }
  return LL_OK;
}

ll_status ll_beam_status_sync(ll_beam_plan* p, int32_t* device_error) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  ll::DeviceGuard guard(p->device);
  return ll::read_error_word(p->a.err, device_error);
}

}  // extern "C"
