// The gated delta rule's entry points: plan, argument checks, the launch
// sequence of the chunked forward and gradient, and the one-token step.
#include <algorithm>
#include <cmath>
#include <new>

#include "ll_delta.h"
#include "ll_host.h"

using ll::bf16_t;
using ll::DeltaArgs;
using ll::fail;

struct ll_delta_plan {
  ll_delta_desc d;
  int device = 0, cus = 0;
  DeltaArgs a{};                       // sizes and the plan's buffers
  int64_t bytes = 0;
  bool saved = false;
  long saved_ld[3] = {0, 0, 0};        // of the saved forward's q, k and v
};

namespace ll {

struct DeltaStepArgs {
  int B, Hk, Hv, Dk, Dv, n_slots;
  float scale;
  long q_ld, k_ld, v_ld;
  const void *q, *k, *v;
  const float *g, *beta;
  float* S;
  const int* slots;
  void* y;
  int* err;
};

constexpr int kStepCols = 32;

// One token.  A work-group has 32 columns of one head's state: thread (row
// group r = tid / 8, column group tid % 8) holds rows r, r + 32, .. and four
// columns of them in registers.  Two sums over the rows (S^T k, then S^T q)
// are all that the columns exchange.
// Bound: HBM, the state read and written: 256 rows, 32 heads of 128 x 128 in 225 us,
// 1.08 GB, 4.8 TB/s (a copy of that size: 5.2).  A few rows: the launch, 4 rows of 4
// heads of 32 x 32 in 4 us.
template <typename T>
__global__ __launch_bounds__(256) void delta_step_kernel(DeltaStepArgs a) {
  __shared__ float ks[kDeltaMaxDk], qs[kDeltaMaxDk];
  __shared__ float4 red[2][4][8];
  const int ntile = (a.Dv + kStepCols - 1) / kStepCols;
  const int ct = blockIdx.x % ntile, bh = blockIdx.x / ntile;
  const int b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  const int c = ct * kStepCols + (tid & 7) * 4, r0 = tid >> 3;
  const bool in = c < a.Dv;            // Dv is a multiple of 8: all four columns or none
  T* y = static_cast<T*>(a.y) + ((long)b * a.Hv + h) * a.Dv + c;
  const int slot = a.slots ? a.slots[b] : b;
  if (slot < 0 || slot >= a.n_slots) {
    if (in && r0 == 0)
      for (int e = 0; e < 4; ++e) y[e] = Op<T>::from_f32(0.f);
    if ((slot < -1 || slot >= a.n_slots) && a.err && h == 0 && ct == 0 && tid == 0) atomicOr(a.err, LL_DEVERR_SLOT);
    return;
  }
  if (tid < a.Dk) {
    ks[tid] = Op<T>::to_f32(static_cast<const T*>(a.k)[b * a.k_ld + (long)hk * a.Dk + tid]);
    qs[tid] = Op<T>::to_f32(static_cast<const T*>(a.q)[b * a.q_ld + (long)hk * a.Dk + tid]);
  }
  float* S = a.S + ((long)slot * a.Hv + h) * a.Dk * a.Dv + c;
  const float eg = expf(a.g[(long)b * a.Hv + h]), beta = a.beta[(long)b * a.Hv + h];
  float4 s[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = r0 + 32 * i;
    s[i] = in && d < a.Dk ? *reinterpret_cast<const float4*>(S + (long)d * a.Dv) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  float v[4];
  for (int e = 0; e < 4; ++e)
    v[e] = in ? Op<T>::to_f32(static_cast<const T*>(a.v)[b * a.v_ld + (long)h * a.Dv + c + e]) : 0.f;
  __syncthreads();
  auto over_rows = [&](const float* x, int slot_) {
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = r0 + 32 * i;
      const float f = d < a.Dk ? x[d] : 0.f;
      t.x += f * s[i].x; t.y += f * s[i].y; t.z += f * s[i].z; t.w += f * s[i].w;
    }
    for (int m = 8; m < 64; m <<= 1) {
      t.x += __shfl_xor(t.x, m, 64); t.y += __shfl_xor(t.y, m, 64);
      t.z += __shfl_xor(t.z, m, 64); t.w += __shfl_xor(t.w, m, 64);
    }
    if (l < 8) red[slot_][w][l] = t;
    __syncthreads();
    const int g = tid & 7;
    const float4 p = red[slot_][0][g], q = red[slot_][1][g], u = red[slot_][2][g], z = red[slot_][3][g];
    return make_float4((p.x + q.x) + (u.x + z.x), (p.y + q.y) + (u.y + z.y), (p.z + q.z) + (u.z + z.z),
                       (p.w + q.w) + (u.w + z.w));
  };
#pragma unroll
  for (int i = 0; i < 4; ++i) { s[i].x *= eg; s[i].y *= eg; s[i].z *= eg; s[i].w *= eg; }
  const float4 sk = over_rows(ks, 0);
  const float u0 = beta * (v[0] - sk.x), u1 = beta * (v[1] - sk.y), u2 = beta * (v[2] - sk.z),
              u3 = beta * (v[3] - sk.w);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int d = r0 + 32 * i;
    const float f = d < a.Dk ? ks[d] : 0.f;
    s[i].x += f * u0; s[i].y += f * u1; s[i].z += f * u2; s[i].w += f * u3;
    if (in && d < a.Dk) *reinterpret_cast<float4*>(S + (long)d * a.Dv) = s[i];
  }
  const float4 o = over_rows(qs, 1);
  if (in && r0 == 0) {
    y[0] = Op<T>::from_f32(a.scale * o.x);
    y[1] = Op<T>::from_f32(a.scale * o.y);
    y[2] = Op<T>::from_f32(a.scale * o.z);
    y[3] = Op<T>::from_f32(a.scale * o.w);
  }
}

}  // namespace ll

namespace {

ll_status validate(const ll_delta_desc* d, bool step) {
  if (!d) return fail(LL_EINVAL, "desc is NULL");
  if (d->T_max < 1 || d->B < 1 || d->Hk < 1 || d->Hv < 1 || d->Dk < 1 || d->Dv < 1)
    return fail(LL_EINVAL, "T_max, B, Hk, Hv, Dk and Dv must be at least 1 (got %d, %d, %d, %d, %d, %d)",
                d->T_max, d->B, d->Hk, d->Hv, d->Dk, d->Dv);
  if (step && d->T_max != 1) return fail(LL_EINVAL, "the step takes one token: T_max must be 1 (got %d)", d->T_max);
  if (d->dtype != LL_F32 && d->dtype != LL_BF16) return fail(LL_EINVAL, "dtype must be LL_F32 or LL_BF16");
  if (d->Hv % d->Hk) return fail(LL_EINVAL, "Hv = %d is not a multiple of Hk = %d", d->Hv, d->Hk);
  if (d->reserved) return fail(LL_EINVAL, "reserved must be 0");
  if (!std::isfinite(d->scale)) return fail(LL_EINVAL, "scale is not finite");
  if (d->Dk % 8 || d->Dv % 8 || d->Dk > ll::kDeltaMaxDk || d->Dv > ll::kDeltaMaxDv)
    return fail(LL_EUNSUPPORTED, "Dk = %d (at most %d) and Dv = %d (at most %d) must be multiples of 8", d->Dk,
                ll::kDeltaMaxDk, d->Dv, ll::kDeltaMaxDv);
  const int es = d->dtype == LL_BF16 ? 2 : 4;
  const int64_t qk = (int64_t)d->Hk * d->Dk, v = (int64_t)d->Hv * d->Dv;
  const int64_t ld[6] = {d->q_ld, d->k_ld, d->v_ld, d->dq_ld, d->dk_ld, d->dv_ld};
  const int64_t need[6] = {qk, qk, v, qk, qk, v};
  const char* names[6] = {"q_ld", "k_ld", "v_ld", "dq_ld", "dk_ld", "dv_ld"};
  for (int i = 0; i < (step ? 3 : 6); ++i)
    if (ld[i] && (ld[i] < need[i] || ld[i] * es % 16 || ld[i] > (int64_t)1 << 31))
      return fail(LL_EINVAL, "%s = %lld must be 0, or at least %lld, at most 2^31 and a multiple of 16 bytes",
                  names[i], (long long)ld[i], (long long)need[i]);
  const int64_t widest = std::max({d->v_ld, step ? 0 : d->dv_ld, v});
  if (!step && widest * d->B * es > (int64_t)1 << 26)
    return fail(LL_EUNSUPPORTED, "a time step of v, y or dv spans %lld bytes (at most 2^26)",
                (long long)(widest * d->B * es));
  const int64_t nch = (d->T_max + ll::kDeltaChunk - 1) / ll::kDeltaChunk;
  // work-groups of the largest launch: a chunk and head each (512 threads), or the step's column tiles
  const int64_t groups = step ? (int64_t)d->B * d->Hv * ((d->Dv + ll::kStepCols - 1) / ll::kStepCols)
                              : (int64_t)d->B * d->Hv * nch;
  const int64_t most = ll::max_groups(step ? 256 : 512);
  if ((int64_t)d->B * d->Hv > 1 << 24 || groups > most)
    return fail(LL_EUNSUPPORTED, "B * Hv = %lld with T_max = %d and Dv = %d: %lld work-groups, a launch holds %lld",
                (long long)d->B * d->Hv, d->T_max, d->Dv, (long long)groups, (long long)most);
  return LL_OK;
}

DeltaArgs sizes(const ll_delta_desc& d) {
  DeltaArgs a{};
  a.T = d.T_max; a.B = d.B; a.Hk = d.Hk; a.Hv = d.Hv; a.Dk = d.Dk; a.Dv = d.Dv;
  a.nch = (d.T_max + ll::kDeltaChunk - 1) / ll::kDeltaChunk;
  a.scale = d.scale != 0.f ? d.scale : (float)(1.0 / std::sqrt((double)d.Dk));
  const long qk = (long)d.Hk * d.Dk, v = (long)d.Hv * d.Dv;
  a.q_ld = d.q_ld ? d.q_ld : qk;
  a.k_ld = d.k_ld ? d.k_ld : qk;
  a.v_ld = d.v_ld ? d.v_ld : v;
  a.dq_ld = d.dq_ld ? d.dq_ld : qk;
  a.dk_ld = d.dk_ld ? d.dk_ld : qk;
  a.dv_ld = d.dv_ld ? d.dv_ld : v;
  return a;
}

void release(ll_delta_plan* p) {
  void* all[] = {p->a.tp, p->a.pp, p->a.ttp, p->a.ptp, p->a.kp, p->a.qp, p->a.ktp, p->a.qtp, p->a.dots, p->a.G, p->a.tok, p->a.st, p->a.u, p->a.dst, p->a.dr, p->a.err};
  for (void* m : all)
    if (m) (void)hipFree(m);
}

}  // namespace

extern "C" {

ll_status ll_delta_plan_create(const ll_delta_desc* desc, int device, ll_delta_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  LL_STATUS(validate(desc, false));
  LL_STATUS(ll::check_device(device));
  ll::DeviceGuard guard(device);
  ll_delta_plan* p = new (std::nothrow) ll_delta_plan();
  if (!p) return fail(LL_ENOMEM, "host allocation of the plan failed");
  p->d = *desc;
  p->device = device;
  p->a = sizes(*desc);
  const size_t items = (size_t)desc->B * desc->Hv * p->a.nch, C = ll::kDeltaChunk;
  const size_t sq = sizeof(bf16_t) * 3 * items * C * C, st = sizeof(float) * items * desc->Dk * desc->Dv,
               rows = sizeof(float) * items * C * desc->Dv;
  const size_t tr = sizeof(bf16_t) * ll::delta_pieces(desc->dtype == LL_BF16) * 32 * ll::delta_ksteps(desc->Dk) *
                    C * desc->B * desc->Hk * p->a.nch;
  hipDeviceProp_t prop;
  if (hipGetDeviceProperties(&prop, device) != hipSuccess) {
    delete p;
    return fail(LL_EHIP, "hipGetDeviceProperties failed");
  }
  p->cus = prop.multiProcessorCount;
  struct { void** at; size_t bytes; const char* what; bool grad; } bufs[] = {
      {(void**)&p->a.tp, sq, "the chunks' T", false},
      {(void**)&p->a.pp, sq, "the chunks' P", false},
      {(void**)&p->a.kp, tr, "the chunks' K", false},
      {(void**)&p->a.qp, tr, "the chunks' Q", false},
      {(void**)&p->a.ktp, tr, "the chunks' K^T", false},
      {(void**)&p->a.ttp, sq, "the chunks' T^T", true},
      {(void**)&p->a.ptp, sq, "the chunks' P^T", true},
      {(void**)&p->a.qtp, tr, "the chunks' Q^T", true},
      {(void**)&p->a.dots, sizeof(float) * ll::kDeltaDots * desc->B * desc->Hk * p->a.nch, "the chunks' products", true},
      {(void**)&p->a.G, sizeof(double) * items * C, "the sums of g", true},
      {(void**)&p->a.tok, sizeof(float4) * items * C, "the tokens' decays", false},
      {(void**)&p->a.err, sizeof(int), "the error word", false},
      {(void**)&p->a.st, st, "the chunks' states", true},
      {(void**)&p->a.u, rows, "the chunks' U", true},
      {(void**)&p->a.dst, st, "the gradients of the chunks' states", true},
      {(void**)&p->a.dr, rows, "the gradients of R", true},
  };
  for (auto& b : bufs) {
    if (b.grad && desc->inference) continue;
    ll_status s = ll::dalloc(b.at, b.bytes, b.what);
    if (s != LL_OK) {
      release(p);
      delete p;
      return s;
    }
    p->bytes += (int64_t)b.bytes;
  }
  if (hipMemset(p->a.err, 0, sizeof(int)) != hipSuccess) {
    release(p);
    delete p;
    return fail(LL_EHIP, "hipMemset of the error word failed");
  }
  if (const ll_status s = ll::wait_created(); s != LL_OK) {
    release(p);
    delete p;
    return s;
  }
  *out = p;
  return LL_OK;
}

ll_status ll_delta_plan_destroy(ll_delta_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_delta_plan_set_ld(ll_delta_plan* p, const int64_t* ld) {
  if (!p || !ld) return fail(LL_EINVAL, "plan and ld are required");
  ll_delta_desc d = p->d;
  d.q_ld = ld[0]; d.k_ld = ld[1]; d.v_ld = ld[2]; d.dq_ld = ld[3]; d.dk_ld = ld[4]; d.dv_ld = ld[5];
  LL_STATUS(validate(&d, false));
  const DeltaArgs z = sizes(d);
  p->d = d;
  p->a.q_ld = z.q_ld; p->a.k_ld = z.k_ld; p->a.v_ld = z.v_ld;
  p->a.dq_ld = z.dq_ld; p->a.dk_ld = z.dk_ld; p->a.dv_ld = z.dv_ld;
  return LL_OK;
}

ll_status ll_delta_plan_bytes(const ll_delta_plan* p, int64_t* device_bytes) {
  if (!p || !device_bytes) return fail(LL_EINVAL, "plan and device_bytes are required");
  *device_bytes = p->bytes;
  return LL_OK;
}

ll_status delta_loop_fwd(ll_delta_plan* p, void* stream, const void* q, const void* k, const void* v,
                         const float* g, const float* beta, const int32_t* seq_len, const float* S0,
                         void* y, float* ST, int32_t save_for_backward) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (!q || !k || !v || !g || !beta || !y) return fail(LL_EINVAL, "q, k, v, g, beta and y are required");
  if (save_for_backward && p->d.inference)
    return fail(LL_EINVAL, "the plan was created for inference: it keeps nothing for the gradient");
  LL_ALIGNED(q, 16); LL_ALIGNED(k, 16); LL_ALIGNED(v, 16); LL_ALIGNED(y, 16); LL_ALIGNED(S0, 16); LL_ALIGNED(ST, 16);
  LL_ALIGNED(g, 4); LL_ALIGNED(beta, 4); LL_ALIGNED(seq_len, 4);
  ll::DeviceGuard guard(p->device);
  DeltaArgs a = p->a;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.seq_len = seq_len; a.S0 = S0; a.y = y; a.ST = ST;
  p->saved = false;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  LL_HIP(p->d.dtype == LL_BF16 ? ll::delta_launch_fwd<bf16_t>(a, save_for_backward != 0, p->cus, s)
                               : ll::delta_launch_fwd<float>(a, save_for_backward != 0, p->cus, s));
  if (save_for_backward) {
    p->saved = true;
    p->saved_ld[0] = a.q_ld; p->saved_ld[1] = a.k_ld; p->saved_ld[2] = a.v_ld;
    p->a.q = q; p->a.k = k; p->a.v = v; p->a.g = g; p->a.beta = beta; p->a.seq_len = seq_len;
  }
  return LL_OK;
}

ll_status delta_loop_bwd(ll_delta_plan* p, void* stream, const void* q, const void* k, const void* v,
                         const float* g, const float* beta, const int32_t* seq_len, const void* dy,
                         const float* dST, void* dq, void* dk, void* dv, float* dg, float* dbeta,
                         float* dS0) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (!p->saved)
    return fail(LL_ESTATE, "no saved forward on this plan (call delta_loop_fwd with save_for_backward=1 first)");
  if (p->a.q_ld != p->saved_ld[0] || p->a.k_ld != p->saved_ld[1] || p->a.v_ld != p->saved_ld[2])
    return fail(LL_ESTATE, "the saved forward's q, k or v had their tokens at other distances than the plan now");
  if (q != p->a.q || k != p->a.k || v != p->a.v || g != p->a.g || beta != p->a.beta || seq_len != p->a.seq_len)
    return fail(LL_EINVAL, "q, k, v, g, beta or seq_len differs from the saved forward's");
  if (!dy || !dq || !dk || !dv || !dg || !dbeta)
    return fail(LL_EINVAL, "dy, dq, dk, dv, dg and dbeta are required");
  LL_ALIGNED(dy, 16); LL_ALIGNED(dST, 16); LL_ALIGNED(dq, 16); LL_ALIGNED(dk, 16); LL_ALIGNED(dv, 16);
  LL_ALIGNED(dS0, 16);
  LL_ALIGNED(dg, 4); LL_ALIGNED(dbeta, 4);
  ll::DeviceGuard guard(p->device);
  DeltaArgs a = p->a;
  a.dy = dy; a.dST = dST; a.dq = dq; a.dk = dk; a.dv = dv; a.dg = dg; a.dbeta = dbeta; a.dS0 = dS0;
  p->saved = false;
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  LL_HIP(p->d.dtype == LL_BF16 ? ll::delta_launch_bwd<bf16_t>(a, p->cus, s)
                               : ll::delta_launch_bwd<float>(a, p->cus, s));
  return LL_OK;
}

ll_status ll_delta_status_sync(ll_delta_plan* p, int32_t* device_error) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  ll::DeviceGuard guard(p->device);
  return ll::read_error_word(p->a.err, device_error);
}

ll_status delta_loop_step(const ll_delta_desc* desc, void* stream, const void* q, const void* k,
                          const void* v, const float* g, const float* beta, float* S,
                          const int32_t* slots, int32_t n_slots, void* y, int32_t* device_error) {
  LL_STATUS(validate(desc, true));
  if (!q || !k || !v || !g || !beta || !S || !y)
    return fail(LL_EINVAL, "q, k, v, g, beta, S and y are required");
  if (n_slots < 1 || (!slots && n_slots < desc->B))
    return fail(LL_EINVAL, "n_slots = %d is too small for B = %d rows", n_slots, desc->B);
  LL_ALIGNED(q, 16); LL_ALIGNED(k, 16); LL_ALIGNED(v, 16); LL_ALIGNED(y, 16); LL_ALIGNED(S, 16);
  LL_ALIGNED(g, 4); LL_ALIGNED(beta, 4); LL_ALIGNED(slots, 4); LL_ALIGNED(device_error, 4);
  const DeltaArgs z = sizes(*desc);
  ll::DeltaStepArgs a{};
  a.B = z.B; a.Hk = z.Hk; a.Hv = z.Hv; a.Dk = z.Dk; a.Dv = z.Dv; a.n_slots = n_slots;
  a.scale = z.scale; a.q_ld = z.q_ld; a.k_ld = z.k_ld; a.v_ld = z.v_ld;
  a.q = q; a.k = k; a.v = v; a.g = g; a.beta = beta; a.S = S; a.slots = slots; a.y = y; a.err = device_error;
  const long grid = (long)z.B * z.Hv * ((z.Dv + ll::kStepCols - 1) / ll::kStepCols);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (desc->dtype == LL_BF16)
    ll::delta_step_kernel<bf16_t><<<dim3((unsigned)grid), dim3(256), 0, s>>>(a);
  else
    ll::delta_step_kernel<float><<<dim3((unsigned)grid), dim3(256), 0, s>>>(a);
  LL_HIP(hipGetLastError());
  return LL_OK;
}

}  // extern "C"
