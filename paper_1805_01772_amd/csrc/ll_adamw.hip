// AdamW over many tensors in one launch.
//
// Bound: HBM.  A parameter moves 28 bytes with 32-bit states (30 with a
// bfloat16 copy), 14 to 18 with 8-bit ones.  The tensors are cut into chunks
// of 4096 elements, one per work-group, through a table made with the plan, so
// that many small tensors cost one launch; a thread has the loads of 16
// elements in flight.  Gradients move from step to step, so their pointers
// travel in the kernel's arguments, kGradsPerLaunch of them a launch.
// Measured: 247 million parameters in 40 tensors, 32-bit states and the copy 1355 us
// (7.4 GB, 5.5 TB/s; a copy of 8 GB reaches 4.7), 8-bit states and bfloat16 gradients 837 us
// (4.0 GB, 4.7 TB/s; the roots and hashes of the codes keep it from the rest); 48 tensors
// of 0.4 million in 7 us.
//
// An 8-bit row of 256 elements is one wave's: four elements a lane, the row's
// largest magnitude by six exchanges.  Everything that a code depends on is
// rounded operation by operation (no contraction), so that the same state and
// gradient give the same codes on any path that does the same.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ll_host.h"
#include "ll_stream.h"

using ll::bf16_t;
using ll::fail;

namespace ll {

constexpr int kAdamChunk = 4096;
constexpr int kGradsPerLaunch = 256;

struct AdamTensor {
  float* p;
  bf16_t* copy;
  void *m, *v;
  float *ms, *vs;
  long n;
  int chunk0;                          // its first chunk
  float decay;
};

struct AdamArgs {
  const AdamTensor* tensors;
  const int* tensor_of;                // per chunk
  const float* grad_scale;
  int chunk0, tensor0;                 // of this launch
  float b1, c1, b2, c2, r1, r2, eps, lr;
  float lift;                          // power of two that makes eps a normal number
  uint32_t seed;
  const void* grads[kGradsPerLaunch];
};

struct Adam1 {
  float p, m, v;
};

__device__ __forceinline__ Adam1 adam_one(const AdamArgs& a, float p, float m, float v, float g, float keep) {
#pragma clang fp contract(off)
  Adam1 r;
  r.m = m * a.b1 + g * a.c1;
  r.v = v * a.b2 + (g * g) * a.c2;
  // Root and reciprocal by the instructions, one unit off at most.  They take subnormal
  // numbers for 0, so v is lifted out of them, and den where eps is that small.  (The
  // exact root and quotient: 920 us against 837 of the large 8-bit case.)
  const bool sub = r.v < 0x1p-126f;
  float root = __builtin_amdgcn_sqrtf(sub ? r.v * 0x1p24f : r.v);
  root = sub ? root * 0x1p-12f : root;
  const float den = root * a.r2 + a.eps;
  const float step = (r.m * a.r1 * a.lift) * __builtin_amdgcn_rcpf(den * a.lift);
  r.p = p * keep - step * a.lr;
  return r;
}

// 32 random bits of an element: its place in its tensor, the tensor, the seed.
__device__ __forceinline__ uint32_t adam_hash(uint32_t place, uint32_t index, uint32_t seed) {
  uint32_t h = place + (index + 1u) * 0xBB67AE85u + seed * 0x9E3779B9u;
  h = (h ^ (h >> 16)) * 0x6A09E667u;
  h = (h ^ (h >> 15)) * 0xBB67AE85u;
  h = (h ^ (h >> 13)) * 0x9E3779B9u;
  return h ^ (h >> 16);
}

// Code of w = |x| / scale in [0, 1]: (code / TOP)^POWER = w, up or down at
// random (rnd in [0, 1)) so that the mean is w.  The root only finds the
// neighbours: one that is off at a code's own value gives the same code.
template <int POWER, int TOP>
__device__ __forceinline__ float adam_code(float w, float rnd) {
#pragma clang fp contract(off)
  float root = __builtin_amdgcn_sqrtf(w);
  if (POWER == 4) root = __builtin_amdgcn_sqrtf(root);
  const float y = fminf(floorf(root * (float)TOP), (float)(TOP - 1));
  float lo = y * y, hi = (y + 1.f) * (y + 1.f), full = (float)TOP * (float)TOP;
  if (POWER == 4) {
    lo = lo * lo;
    hi = hi * hi;
    full = 4228250625.0f;
  }
  return y + ((w * full - lo) > rnd * (hi - lo) ? 1.f : 0.f);
}

// Largest value over the wave; NaN if any is.
__device__ __forceinline__ float wave_max_nan(float x) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const float o = __shfl_xor(x, d, 64);
    x = (o > x || o != o) ? o : x;
  }
  return x;
}

template <typename G> struct Quad;
template <> struct Quad<float> {
  template <bool STREAM>
  __device__ static __forceinline__ float4 load(const float* p) {
    return __builtin_bit_cast(float4, STREAM ? ld16_stream(p) : ld16(p));
  }
};
template <> struct Quad<bf16_t> {
  template <bool STREAM>
  __device__ static __forceinline__ float4 load(const bf16_t* p) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u),
                       __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u));
  }
};

// four elements from i on, zeros past n
template <bool STREAM, typename G>
__device__ __forceinline__ float4 load4(const G* p, long i, long n) {
  if (i + 4 <= n) return Quad<G>::template load<STREAM>(p + i);
  float4 r = make_float4(0.f, 0.f, 0.f, 0.f);
  if (i < n) r.x = Op<G>::to_f32(p[i]);
  if (i + 1 < n) r.y = Op<G>::to_f32(p[i + 1]);
  if (i + 2 < n) r.z = Op<G>::to_f32(p[i + 2]);
  return r;
}
template <bool STREAM>
__device__ __forceinline__ void store4(float* p, long i, long n, float4 x) {
  if (i + 4 <= n) {
    if (STREAM) st16_stream(p + i, __builtin_bit_cast(uint4, x));
    else *reinterpret_cast<float4*>(p + i) = x;
    return;
  }
  if (i < n) p[i] = x.x;
  if (i + 1 < n) p[i + 1] = x.y;
  if (i + 2 < n) p[i + 2] = x.z;
}
__device__ __forceinline__ void store4(bf16_t* p, long i, long n, float4 x) {
  const bf16_t h[4] = {f32_to_bf16(x.x), f32_to_bf16(x.y), f32_to_bf16(x.z), f32_to_bf16(x.w)};
  if (i + 4 <= n) {
    *reinterpret_cast<uint2*>(p + i) =
        make_uint2((uint32_t)h[0] | (uint32_t)h[1] << 16, (uint32_t)h[2] | (uint32_t)h[3] << 16);
    return;
  }
  for (int e = 0; e < 3; ++e)
    if (i + e < n) p[i + e] = h[e];
}
__device__ __forceinline__ uint32_t load4_codes(const void* base, long i, long n) {
  const unsigned char* p = static_cast<const unsigned char*>(base);
  if (i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p + i);
  uint32_t r = 0;
  for (int e = 0; e < 3; ++e)
    if (i + e < n) r |= (uint32_t)p[i + e] << (8 * e);
  return r;
}
__device__ __forceinline__ void store4_codes(void* base, long i, long n, uint32_t x) {
  unsigned char* p = static_cast<unsigned char*>(base);
  if (i + 4 <= n) {
    *reinterpret_cast<uint32_t*>(p + i) = x;
    return;
  }
  for (int e = 0; e < 3; ++e)
    if (i + e < n) p[i + e] = (unsigned char)(x >> (8 * e));
}

template <typename G, bool Q8, bool STREAM>
__global__ __launch_bounds__(256) void adamw_kernel(AdamArgs a) {
#pragma clang fp contract(off)
  const int chunk = a.chunk0 + blockIdx.x, index = a.tensor_of[chunk];
  const AdamTensor t = a.tensors[index];
  const G* grad = static_cast<const G*>(a.grads[index - a.tensor0]);
  const float gs = a.grad_scale ? *a.grad_scale : 1.f;
  if (!grad || !(__builtin_fabsf(gs) < __builtin_inff())) return;
  const long base = (long)(chunk - t.chunk0) * kAdamChunk;
  const float keep = 1.f - a.lr * t.decay;
  const int tid = threadIdx.x, w = tid >> 6, l = tid & 63;
  if (!Q8) {
    float* pm = static_cast<float*>(t.m);
    float* pv = static_cast<float*>(t.v);
    float4 p[4], m[4], v[4], g[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long at = base + (i * 256 + tid) * 4;
      g[i] = load4<STREAM>(grad, at, t.n);
      p[i] = load4<STREAM>(t.p, at, t.n);
      m[i] = load4<STREAM>(pm, at, t.n);
      v[i] = load4<STREAM>(pv, at, t.n);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const long at = base + (i * 256 + tid) * 4;
      const Adam1 x = adam_one(a, p[i].x, m[i].x, v[i].x, g[i].x * gs, keep),
                  y = adam_one(a, p[i].y, m[i].y, v[i].y, g[i].y * gs, keep),
                  z = adam_one(a, p[i].z, m[i].z, v[i].z, g[i].z * gs, keep),
                  u = adam_one(a, p[i].w, m[i].w, v[i].w, g[i].w * gs, keep);
      const float4 np = make_float4(x.p, y.p, z.p, u.p);
      store4<STREAM>(t.p, at, t.n, np);
      store4<STREAM>(pm, at, t.n, make_float4(x.m, y.m, z.m, u.m));
      store4<STREAM>(pv, at, t.n, make_float4(x.v, y.v, z.v, u.v));
      if (t.copy) store4(t.copy, at, t.n, np);
    }
    return;
  }
  // 8 bits: rows of 256, four of the chunk's sixteen per wave
  float4 p[4], g[4];
  uint32_t cm[4], cv[4];
  float ms[4], vs[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long row = base + (w * 4 + i) * 256, at = row + l * 4;
    g[i] = load4<STREAM>(grad, at, t.n);
    p[i] = load4<STREAM>(t.p, at, t.n);
    cm[i] = load4_codes(t.m, at, t.n);
    cv[i] = load4_codes(t.v, at, t.n);
    ms[i] = row < t.n ? t.ms[row >> 8] : 0.f;
    vs[i] = row < t.n ? t.vs[row >> 8] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const long row = base + (w * 4 + i) * 256, at = row + l * 4;
    if (row >= t.n) break;
    const float sm = ms[i] * (float)(1.0 / 16129.0), sv = vs[i] * (float)(1.0 / 4228250625.0);
    const float gp[4] = {g[i].x, g[i].y, g[i].z, g[i].w}, pp[4] = {p[i].x, p[i].y, p[i].z, p[i].w};
    Adam1 r[4];
    float am = 0.f, av = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float c = (float)(int8_t)(cm[i] >> (8 * e)), d = (float)(uint8_t)(cv[i] >> (8 * e));
      const float d2 = d * d;
      r[e] = adam_one(a, pp[e], (c * __builtin_fabsf(c)) * sm, (d2 * d2) * sv, gp[e] * gs, keep);
      const float x = __builtin_fabsf(r[e].m);
      am = (x > am || x != x) ? x : am;
      av = (r[e].v > av || r[e].v != r[e].v) ? r[e].v : av;
    }
    am = wave_max_nan(am);
    av = wave_max_nan(av);
    const float im = am >= 0x1p-126f ? 1.f / am : 0.f, iv = av >= 0x1p-126f ? 1.f / av : 0.f;
    uint32_t om = 0, ov = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t bits = adam_hash((uint32_t)(at + e), (uint32_t)index, a.seed);
      const float xm = adam_code<2, 127>(__builtin_fabsf(r[e].m) * im, (float)(bits & 0xffffu) * 0x1p-16f);
      const float xv = adam_code<4, 255>(r[e].v * iv, (float)(bits >> 16) * 0x1p-16f);
      const int c = r[e].m < 0.f ? -(int)xm : (int)xm;
      int d = (int)xv;
      if (r[e].v > 0.f && d < 1) d = 1;
      om |= (uint32_t)(c & 0xff) << (8 * e);
      ov |= (uint32_t)(d & 0xff) << (8 * e);
    }
    const float4 np = make_float4(r[0].p, r[1].p, r[2].p, r[3].p);
    store4<STREAM>(t.p, at, t.n, np);
    if (t.copy) store4(t.copy, at, t.n, np);
    store4_codes(t.m, at, t.n, om);
    store4_codes(t.v, at, t.n, ov);
    if (l == 0) {
      t.ms[row >> 8] = am;
      t.vs[row >> 8] = av;
    }
  }
}

}  // namespace ll

struct ll_adamw_plan {
  ll_adamw_desc d;
  int device = 0;
  std::vector<int> chunk0;             // per tensor, and the end
  long bytes = 0;                      // that a step moves
  ll::AdamTensor* tensors = nullptr;
  int* tensor_of = nullptr;
};

namespace {

void release(ll_adamw_plan* p) {
  if (p->tensors) (void)hipFree(p->tensors);
  if (p->tensor_of) (void)hipFree(p->tensor_of);
}

ll_status build(ll_adamw_plan* p, const ll_adamw_tensor* ts) {
  const bool q8 = p->d.state_bits == 8;
  std::vector<ll::AdamTensor> recs;
  std::vector<int> of;
  long chunks = 0;
  for (int i = 0; i < p->d.n_tensors; ++i) {
    const ll_adamw_tensor& t = ts[i];
    if (t.n < 0 || t.n > (int64_t)1 << 40) return fail(LL_EINVAL, "tensor %d: n = %lld", i, (long long)t.n);
    if (t.reserved) return fail(LL_EINVAL, "tensor %d: reserved must be 0", i);
    if (!std::isfinite(t.weight_decay) || t.weight_decay < 0.f)
      return fail(LL_EINVAL, "tensor %d: weight_decay must be at least 0", i);
    if (t.n > 0 && (!t.p || !t.m || !t.v || (q8 && (!t.m_scale || !t.v_scale))))
      return fail(LL_EINVAL, "tensor %d: p, m, v%s are required", i, q8 ? ", m_scale and v_scale" : "");
    const void* ptrs[] = {t.p, t.copy, t.m, t.v};
    for (const void* x : ptrs)
      if (!ll::aligned16(x)) return fail(LL_EINVAL, "tensor %d: %p is not 16-byte aligned", i, x);
    if (q8 && (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3))
      return fail(LL_EINVAL, "tensor %d: the scales are not 4-byte aligned", i);
    const long c = (long)((t.n + ll::kAdamChunk - 1) / ll::kAdamChunk);
    if (chunks + c > ll::max_groups(256))
      return fail(LL_EUNSUPPORTED, "more than 2^24 - 1 chunks of %d elements in one plan (at tensor %d)",
                  ll::kAdamChunk, i);
    recs.push_back(ll::AdamTensor{t.p, static_cast<bf16_t*>(t.copy), t.m, t.v, t.m_scale, t.v_scale, (long)t.n,
                                  (int)chunks, t.weight_decay});
    p->chunk0.push_back((int)chunks);
    p->bytes += (long)t.n * (8 + (p->d.grad_dtype == LL_BF16 ? 2 : 4) + (q8 ? 4 : 16) + (t.copy ? 2 : 0));
    of.insert(of.end(), (size_t)c, i);
    chunks += c;
  }
  p->chunk0.push_back((int)chunks);
  LL_STATUS(ll::check_device(p->device));
  ll::DeviceGuard guard(p->device);
  LL_STATUS(ll::dalloc((void**)&p->tensors, sizeof(ll::AdamTensor) * recs.size(), "the tensor table"));
  LL_STATUS(ll::dalloc((void**)&p->tensor_of, sizeof(int) * of.size(), "the chunk table"));
  LL_HIP(hipMemcpy(p->tensors, recs.data(), sizeof(ll::AdamTensor) * recs.size(), hipMemcpyHostToDevice));
  if (!of.empty()) LL_HIP(hipMemcpy(p->tensor_of, of.data(), sizeof(int) * of.size(), hipMemcpyHostToDevice));
  return ll::wait_created();
}

}  // namespace

extern "C" {

ll_status ll_adamw_plan_create(const ll_adamw_desc* desc, const ll_adamw_tensor* tensors, int device,
                               ll_adamw_plan** out) {
  if (!out) return fail(LL_EINVAL, "out is NULL");
  *out = nullptr;
  if (!desc || !tensors) return fail(LL_EINVAL, "desc and tensors are required");
  if (desc->n_tensors < 1 || desc->n_tensors > 65536)
    return fail(LL_EINVAL, "n_tensors = %d must be 1 .. 65536", desc->n_tensors);
  if (desc->state_bits != 32 && desc->state_bits != 8)
    return fail(LL_EINVAL, "state_bits must be 32 or 8 (got %d)", desc->state_bits);
  if (desc->grad_dtype != LL_F32 && desc->grad_dtype != LL_BF16)
    return fail(LL_EINVAL, "grad_dtype must be LL_F32 or LL_BF16");
  if (desc->reserved) return fail(LL_EINVAL, "reserved must be 0");
  ll_adamw_plan* p = nullptr;
  ll_status st;
  try {
    p = new ll_adamw_plan();
    p->d = *desc;
    p->device = device;
    st = build(p, tensors);
  } catch (const std::bad_alloc&) {
    st = fail(LL_ENOMEM, "host allocation of the plan failed");
  }
  if (st != LL_OK) {
    if (p) release(p);
    delete p;
    return st;
  }
  *out = p;
  return LL_OK;
}

ll_status ll_adamw_plan_destroy(ll_adamw_plan* p) {
  if (!p) return LL_OK;
  ll::DeviceGuard guard(p->device);
  (void)hipDeviceSynchronize();
  release(p);
  delete p;
  return LL_OK;
}

ll_status ll_adamw_step(ll_adamw_plan* p, void* stream, const void* const* grads, const ll_adamw_hyper* h,
                        const float* grad_scale) {
  if (!p) return fail(LL_EINVAL, "plan is NULL");
  if (!grads || !h) return fail(LL_EINVAL, "grads and hyper are required");
  if (!(h->lr >= 0.0) || !std::isfinite(h->lr) || !(h->beta1 >= 0.0 && h->beta1 < 1.0) ||
      !(h->beta2 >= 0.0 && h->beta2 < 1.0) || !(h->eps > 0.0) || !std::isfinite(h->eps) || h->step < 1)
    return fail(LL_EINVAL, "lr >= 0, 0 <= beta < 1, eps > 0 and step >= 1 are required "
                           "(got %g, %g, %g, %g, %lld)", h->lr, h->beta1, h->beta2, h->eps, (long long)h->step);
  if (h->reserved) return fail(LL_EINVAL, "reserved must be 0");
  const int n = p->d.n_tensors;
  for (int i = 0; i < n; ++i)
    if (!ll::aligned16(grads[i])) return fail(LL_EINVAL, "grads[%d] = %p is not 16-byte aligned", i, grads[i]);
  ll::DeviceGuard guard(p->device);
  ll::AdamArgs a{};
  a.tensors = p->tensors;
  a.tensor_of = p->tensor_of;
  a.grad_scale = grad_scale;
  a.b1 = (float)h->beta1;
  a.c1 = (float)(1.0 - h->beta1);
  a.b2 = (float)h->beta2;
  a.c2 = (float)(1.0 - h->beta2);
  a.r1 = (float)(1.0 / (1.0 - std::pow(h->beta1, (double)h->step)));
  a.r2 = (float)(1.0 / std::sqrt(1.0 - std::pow(h->beta2, (double)h->step)));
  a.eps = std::max((float)h->eps, 0x1p-149f);
  a.lr = (float)h->lr;
  a.lift = a.eps < 0x1p-100f ? 0x1p48f : 1.f;
  a.seed = h->seed;
  hipStream_t hs = reinterpret_cast<hipStream_t>(stream);
  for (int t0 = 0; t0 < n; t0 += ll::kGradsPerLaunch) {
    const int t1 = std::min(n, t0 + ll::kGradsPerLaunch);
    const int blocks = p->chunk0[t1] - p->chunk0[t0];
    if (blocks == 0) continue;
    a.tensor0 = t0;
    a.chunk0 = p->chunk0[t0];
    for (int i = t0; i < t1; ++i) a.grads[i - t0] = grads[i];
    const bool bf = p->d.grad_dtype == LL_BF16, q8 = p->d.state_bits == 8;
    // a step that sweeps the last-level cache goes past it (247 M parameters,
    // 32-bit states 1397 -> 1355 us, 8-bit ones 870 -> 855; 0.4 M: no difference)
    const bool past = p->bytes > ll::kLastLevelBytes;
    auto* kernel = past ? (q8 ? (bf ? ll::adamw_kernel<bf16_t, true, true> : ll::adamw_kernel<float, true, true>)
                                : (bf ? ll::adamw_kernel<bf16_t, false, true> : ll::adamw_kernel<float, false, true>))
                          : (q8 ? (bf ? ll::adamw_kernel<bf16_t, true, false> : ll::adamw_kernel<float, true, false>)
                                : (bf ? ll::adamw_kernel<bf16_t, false, false> : ll::adamw_kernel<float, false, false>));
    kernel<<<dim3((unsigned)blocks), dim3(256), 0, hs>>>(a);
    LL_HIP(hipGetLastError());
  }
  return LL_OK;
}

}  // extern "C"
