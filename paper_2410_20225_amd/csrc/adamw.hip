// AdamW over many tensors in one launch, states in 32 or in 8 bits.
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,  p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// 8 bits: m is the signed square of a whole number, v the fourth power of one, in units of the largest of 128 elements.  Both spread
// their numbers over many orders of magnitude (m: 1 .. 127^2, v: 1 .. 255^4, the range of g^2 that belongs to m's and more), finest
// where the values are large.  They are rounded up or down by chance, with the value as the mean: beta2 is so close to one that a
// step changes v by less than half of what separates two stored numbers, and rounding to nearest would hold v where it is for good.
// The operations that lead to the stored numbers are rounded one by one, none contracted, so that a number next to a border falls
// the same way wherever the formula is computed.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "rows.h"

namespace tdf {
namespace {

using namespace rows;

constexpr int BLOCK = 128;          // elements that share a scale
constexpr int64_t CHUNK = 4096;     // elements of a workgroup's piece of a tensor
constexpr int64_t MOST_CHUNKS = (1 << 24) - 1;   // a workgroup of 256 threads each: less than 2^32 threads

struct AdamTensor {
  int64_t n;
  int64_t first_chunk;
  void* param;
  const void* grad;
  __bf16* copy;
  void *m, *v;
  float *m_scale, *v_scale;
  int32_t param_dtype, grad_dtype, bits;
  float weight_decay;
  int32_t whole, reserved;          // whole: everything begins at a place that eight elements are aligned to
};

struct AdamArgs {
  const AdamTensor* tensors;
  const uint32_t* tensor_of;        // of each chunk
  float beta1, rest1, beta2, rest2; // rest = 1 - beta
  float lr;                         // lr / (1 - beta1^step)
  float root;                       // 1 / sqrt(1 - beta2^step)
  float eps;
  float plain_lr;
  const float* grad_scale;
  uint32_t seed;
};

__device__ __forceinline__ uint32_t mix(uint32_t x) {
  x = (x ^ (x >> 16)) * 0xBB67AE85u;
  x = (x ^ (x >> 13)) * 0x6A09E667u;
  return x ^ (x >> 16);
}

// Eight elements beside each other, `n` of them there.
constexpr int EACH = 8;
typedef float Four __attribute__((ext_vector_type(4)));
typedef __bf16 Eight __attribute__((ext_vector_type(8)));
typedef unsigned int Two __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void load8(const float* p, int n, bool whole, float* x) {
  if (whole && n == EACH) {
    const Four a = ((const Four*)p)[0], b = ((const Four*)p)[1];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e], x[4 + e] = b[e];
  } else {
#pragma unroll
    for (int e = 0; e < EACH; ++e) x[e] = e < n ? p[e] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const __bf16* p, int n, bool whole, float* x) {
  if (whole && n == EACH) {
    const Eight a = *(const Eight*)p;
#pragma unroll
    for (int e = 0; e < EACH; ++e) x[e] = (float)a[e];
  } else {
#pragma unroll
    for (int e = 0; e < EACH; ++e) x[e] = e < n ? (float)p[e] : 0.0f;
  }
}
__device__ __forceinline__ void load8(const uint8_t* p, int n, bool whole, uint32_t* x) {
  if (whole && n == EACH) {
    const Two a = *(const Two*)p;
    x[0] = a[0], x[1] = a[1];
  } else {
    x[0] = x[1] = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (e < n) x[e / 4] |= (uint32_t)p[e] << (e % 4 * 8);
  }
}
__device__ __forceinline__ void store8(float* p, int n, bool whole, const float* x) {
  if (whole && n == EACH) {
    ((Four*)p)[0] = Four{x[0], x[1], x[2], x[3]};
    ((Four*)p)[1] = Four{x[4], x[5], x[6], x[7]};
  } else {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (e < n) p[e] = x[e];
  }
}
__device__ __forceinline__ void store8(__bf16* p, int n, bool whole, const float* x) {
  if (whole && n == EACH) {
    Eight a;
#pragma unroll
    for (int e = 0; e < EACH; ++e) a[e] = (__bf16)x[e];
    *(Eight*)p = a;
  } else {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (e < n) p[e] = (__bf16)x[e];
  }
}
__device__ __forceinline__ void store8(uint8_t* p, int n, bool whole, const uint32_t* x) {
  if (whole && n == EACH) {
    *(Two*)p = Two{x[0], x[1]};
  } else {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (e < n) p[e] = (uint8_t)(x[e / 4] >> (e % 4 * 8));
  }
}

// A block's scale from the bits of its largest magnitude (as whole numbers, NaN is above infinity): too small ones are zero.
__device__ __forceinline__ float scale_of(uint32_t top) { return top < 0x12800000u /* 2^-90 */ ? 0.0f : __uint_as_float(top); }

// Products and sums that are not contracted into one operation.
__device__ __forceinline__ float mul(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}
__device__ __forceinline__ float add(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}

// The whole number q whose square is y, or one of the two around it.  (The root is the hardware's, which may be off in its last place and
// so may be the whole number below it next to a square; but there the number that is taken is the same from either side.)
__device__ __forceinline__ float stored_m(float y, float u) {
  const float lo = fminf(floorf(__builtin_amdgcn_sqrtf(y)), 126.0f);
  return mul(u, add(mul(2.0f, lo), 1.0f)) < add(y, -mul(lo, lo)) ? lo + 1.0f : lo;
}
// The same for the fourth power; (lo + 1)^4 - lo^4 = (2 lo + 1) (lo^2 + (lo + 1)^2).
__device__ __forceinline__ float stored_v(float y, float u) {
  const float lo = fminf(floorf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(y))), 254.0f), lo2 = mul(lo, lo), hi = lo + 1.0f;
  const float gap = mul(add(mul(2.0f, lo), 1.0f), add(lo2, mul(hi, hi)));
  const float q = mul(u, gap) < add(y, -mul(lo2, lo2)) ? hi : lo;
  return y > 0.0f ? fmaxf(q, 1.0f) : q;
}

// What a thread reads for its eight elements.
struct Before {
  float p[EACH], g[EACH], m[EACH], v[EACH], m_scale, v_scale;
  uint32_t qm[2], qv[2];
};

// One workgroup a chunk; a thread has eight elements beside each other, twice, and 16 threads share a scale.  Memory bounds it: 28 bytes an
// element (states of 32 bits, all fp32), 16.1 with states of 8; the latter with about 90 instructions, which keep the
// vector units busy for 86 % of the time that the bytes take: 153 M elements in 451 us, 5.45 TB/s; 5.8 M with 32 bits 33 us, 5.3 TB/s; a few
// chunks 5.7 us.
__global__ void __launch_bounds__(256) k_adamw(AdamArgs a) {
  typedef const __attribute__((address_space(4))) AdamTensor* Table;
  typedef const __attribute__((address_space(4))) uint32_t* Numbers;
  constexpr int PASSES = CHUNK / (256 * EACH);
  const uint32_t k = ((Numbers)a.tensor_of)[blockIdx.x];
  const Table t = (Table)(a.tensors + k);
  const int64_t first = ((int64_t)blockIdx.x - t->first_chunk) * CHUNK + threadIdx.x * EACH, size = t->n;
  const bool whole = t->whole, small = t->bits == 8, p16 = t->param_dtype == TDF_BF16, g16 = t->grad_dtype == TDF_BF16;
  int left = (int)min(max(size - first, (int64_t)0), (int64_t)CHUNK);     // elements from the thread's first on
  asm("" : "+v"(left));                                                   // (compared as 32 bits)
  Before in[PASSES];
#pragma unroll
  for (int j = 0; j < PASSES; ++j) {
    const int64_t i = first + j * 256 * EACH;
    const int n = min(max(left - j * 256 * EACH, 0), EACH);
    if (p16) load8((const __bf16*)t->param + i, n, whole, in[j].p);
    else load8((const float*)t->param + i, n, whole, in[j].p);
    if (g16) load8((const __bf16*)t->grad + i, n, whole, in[j].g);
    else load8((const float*)t->grad + i, n, whole, in[j].g);
    if (small) {
      load8((const uint8_t*)t->m + i, n, whole, in[j].qm);
      load8((const uint8_t*)t->v + i, n, whole, in[j].qv);
      in[j].m_scale = n ? t->m_scale[i / BLOCK] : 0.0f;
      in[j].v_scale = n ? t->v_scale[i / BLOCK] : 0.0f;
    } else {
      load8((const float*)t->m + i, n, whole, in[j].m);
      load8((const float*)t->v + i, n, whole, in[j].v);
    }
  }
  const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
  const float decay = a.plain_lr * t->weight_decay;
  const uint32_t key = mix(a.seed ^ (0x9E3779B9u * (k + 1)));
#pragma unroll
  for (int j = 0; j < PASSES; ++j) {
    const int64_t i = first + j * 256 * EACH;
    const int n = min(max(left - j * 256 * EACH, 0), EACH);
    Before& o = in[j];
    const float um = mul(o.m_scale, (float)(1.0 / (127.0 * 127.0))), uv = mul(o.v_scale, (float)(1.0 / (255.0 * 255.0 * 255.0 * 255.0)));
    uint32_t tm = 0, tv = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      if (small) {
        const float qm = (float)(int8_t)(o.qm[e / 4] >> (e % 4 * 8)), qv = (float)(uint8_t)(o.qv[e / 4] >> (e % 4 * 8)), q2 = qv * qv;
        o.m[e] = mul(qm * fabsf(qm), um);
        o.v[e] = mul(mul(q2, q2), uv);
      }
      const float g = mul(o.g[e], gs);
      o.m[e] = add(mul(o.m[e], a.beta1), mul(g, a.rest1));
      o.v[e] = add(mul(o.v[e], a.beta2), mul(mul(g, g), a.rest2));
      const float root = fmaf(__builtin_amdgcn_sqrtf(o.v[e]), a.root, a.eps);
      // (1 - decay would be rounded to a multiple of 2^-24, so that a small decay were none or a larger one, the same way in every step)
      o.p[e] -= fmaf(o.p[e], decay, o.m[e] * a.lr * __builtin_amdgcn_rcpf(root));
      // (elements that are not there are zeros and stay zeros, unless a NaN scale makes them one, as all of the block)
      tm = max(tm, __float_as_uint(o.m[e]) & 0x7FFFFFFFu);
      tv = max(tv, __float_as_uint(o.v[e]) & 0x7FFFFFFFu);
    }
    if (p16) store8((__bf16*)t->param + i, n, whole, o.p);
    else store8((float*)t->param + i, n, whole, o.p);
    if (t->copy) store8(t->copy + i, n, whole, o.p);
    if (!small) {
      store8((float*)t->m + i, n, whole, o.m);
      store8((float*)t->v + i, n, whole, o.v);
      continue;
    }
#pragma unroll
    for (int d = BLOCK / EACH / 2; d; d >>= 1) {
      tm = max(tm, (uint32_t)__shfl_xor((int)tm, d));
      tv = max(tv, (uint32_t)__shfl_xor((int)tv, d));
    }
    const float ms = scale_of(tm), vs = scale_of(tv);
    const float im = ms == 0.0f ? 0.0f : 16129.0f / ms, iv = vs == 0.0f ? 0.0f : 4228250625.0f / vs;
    const uint32_t start = (uint32_t)i * 0x9E3779B1u + key + (uint32_t)(i >> 32) * 0x85EBCA77u;   // (eight elements do not cross 2^32)
    uint32_t qm[2] = {0, 0}, qv[2] = {0, 0};
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const uint32_t u = mix(start + e * 0x9E3779B1u);
      const float m = stored_m(mul(fabsf(o.m[e]), im), (float)(u & 0xFFFFu) * 0x1p-16f);
      const float v = stored_v(mul(o.v[e], iv), (float)(u >> 16) * 0x1p-16f);
      qm[e / 4] |= ((uint32_t)(int)(o.m[e] < 0 ? -m : m) & 0xFFu) << (e % 4 * 8);
      qv[e / 4] |= ((uint32_t)v & 0xFFu) << (e % 4 * 8);
    }
    store8((uint8_t*)t->m + i, n, whole, qm);
    store8((uint8_t*)t->v + i, n, whole, qv);
    if (n && threadIdx.x % (BLOCK / EACH) == 0) {
      t->m_scale[i / BLOCK] = ms;
      t->v_scale[i / BLOCK] = vs;
    }
  }
}

size_t table_bytes(size_t n) { return (n * sizeof(AdamTensor) + 255) / 256 * 256; }

}  // namespace
}  // namespace tdf

using namespace tdf;

struct tdf_adamw_plan {
  std::vector<AdamTensor> tensors;
  std::vector<uint32_t> tensor_of;
  void* workspace = nullptr;
  int device = -1;
};

extern "C" tdf_status tdf_adamw_build(const tdf_adamw_tensor* tensors, int64_t n_tensors, tdf_adamw_plan** out) {
  const char* who = "tdf_adamw_build";
  try {
    if (!out) return refuse(who, "out is NULL");
    *out = nullptr;
    if (n_tensors < 1 || n_tensors > (1 << 24) || !tensors) return refuse(who, "no tensors, or too many");
    tdf_adamw_plan plan;
    std::vector<std::pair<uintptr_t, uintptr_t>> written;
    int64_t chunks = 0;
    for (int64_t k = 0; k < n_tensors; ++k) {
      const tdf_adamw_tensor& t = tensors[k];
      const std::string at = "tensor " + std::to_string(k) + ": ";
      const auto bad = [&](const char* what) { return refuse(who, (at + what).c_str()); };
      if (t.n < 0 || t.n > (1ll << 40)) return bad("n out of range");
      if (!known_type(t.param_dtype) || !known_type(t.grad_dtype)) return bad("bad dtype");
      if (t.state_bits != 8 && t.state_bits != 32) return bad("state_bits must be 8 or 32");
      if (!(fabsf(t.weight_decay) <= 3.0e38f)) return bad("weight_decay is not finite");
      if (t.copy && t.param_dtype != TDF_F32) return bad("only a float parameter has a copy in bf16");
      if ((t.state_bits == 8) != (t.m_scale != nullptr) || (t.state_bits == 8) != (t.v_scale != nullptr))
        if (t.n) return bad("scales go with states of 8 bits");
      if (t.n && (!t.param || !t.grad || !t.m || !t.v)) return bad("NULL pointer");
      const size_t ps = element_size(t.param_dtype), gs = element_size(t.grad_dtype), ss = t.state_bits / 8;
      if ((uintptr_t)t.param % ps || (uintptr_t)t.grad % gs || (uintptr_t)t.copy % 2 || (ss == 4 && ((uintptr_t)t.m % 4 || (uintptr_t)t.v % 4)) ||
          bad_floats(t.m_scale) || bad_floats(t.v_scale))
        return bad("a pointer is not aligned to its elements");
      if (t.n) {
        const size_t blocks = (size_t)((t.n + BLOCK - 1) / BLOCK);
        const std::pair<const void*, size_t> outs[] = {{t.param, t.n * ps}, {t.copy, t.n * 2}, {t.m, t.n * ss}, {t.v, t.n * ss},
                                                       {t.m_scale, blocks * 4}, {t.v_scale, blocks * 4}};
        for (const auto& o : outs)
          if (o.first) written.emplace_back((uintptr_t)o.first, (uintptr_t)o.first + o.second);
      }
      plan.tensors.push_back({t.n, chunks, t.param, t.grad, (__bf16*)t.copy, t.m, t.v, t.m_scale, t.v_scale, t.param_dtype, t.grad_dtype, t.state_bits, t.weight_decay,
                              ((uintptr_t)t.param | (uintptr_t)t.grad | (uintptr_t)t.copy) % 16 == 0 && ((uintptr_t)t.m | (uintptr_t)t.v) % (t.state_bits == 8 ? 8 : 16) == 0, 0});
      const int64_t more = (t.n + CHUNK - 1) / CHUNK;
      chunks += more;
      if (chunks > MOST_CHUNKS) return bad("too many elements");
      plan.tensor_of.insert(plan.tensor_of.end(), (size_t)more, (uint32_t)k);
    }
    std::sort(written.begin(), written.end());
    for (size_t i = 1; i < written.size(); ++i)
      if (written[i].first < written[i - 1].second) return refuse(who, "two outputs overlap");
    *out = new tdf_adamw_plan(std::move(plan));
    return TDF_OK;
  } catch (const std::exception& e) {
    return refuse(who, e.what());
  }
}

extern "C" void tdf_adamw_destroy(tdf_adamw_plan* plan) { delete plan; }

extern "C" tdf_status tdf_adamw_workspace_size(const tdf_adamw_plan* plan, size_t* bytes) {
  if (!plan || !bytes) return refuse("tdf_adamw_workspace_size", "NULL argument");
  *bytes = std::max<size_t>(256, table_bytes(plan->tensors.size()) + plan->tensor_of.size() * sizeof(uint32_t));
  return TDF_OK;
}

extern "C" tdf_status tdf_adamw_prepare(tdf_adamw_plan* plan, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const char* who = "tdf_adamw_prepare";
  if (!plan) return refuse(who, "plan is NULL");
  size_t need = 0;
  tdf_adamw_workspace_size(plan, &need);
  if (!workspace || workspace_bytes < need || (uintptr_t)workspace % 256) {
    set_error("tdf_adamw_prepare: workspace too small or misaligned");
    return TDF_ERR_WORKSPACE;
  }
  const hipStream_t s = (hipStream_t)hip_stream;
  int device = -1;
  hipError_t err = hipGetDevice(&device);
  if (err == hipSuccess) err = hipMemcpyAsync(workspace, plan->tensors.data(), plan->tensors.size() * sizeof(AdamTensor), hipMemcpyHostToDevice, s);
  if (err == hipSuccess && !plan->tensor_of.empty())
    err = hipMemcpyAsync((char*)workspace + table_bytes(plan->tensors.size()), plan->tensor_of.data(), plan->tensor_of.size() * sizeof(uint32_t), hipMemcpyHostToDevice, s);
  if (err == hipSuccess) err = hipStreamSynchronize(s);
  if (err != hipSuccess) {
    set_error(std::string(who) + ": " + hipGetErrorString(err));
    return TDF_ERR_DEVICE;
  }
  plan->workspace = workspace;
  plan->device = device;
  return TDF_OK;
}

extern "C" tdf_status tdf_adamw(const tdf_adamw_plan* plan, const tdf_adamw_step* h, void* hip_stream) {
  const char* who = "tdf_adamw";
  if (!plan || !h) return refuse(who, "NULL argument");
  if (!plan->workspace) return refuse(who, "the plan has not been prepared (tdf_adamw_prepare)");
  if (h->step < 1) return refuse(who, "step must be positive");
  if (!(h->beta1 >= 0 && h->beta1 < 1 && h->beta2 >= 0 && h->beta2 < 1)) return refuse(who, "betas must be in [0, 1)");
  if (!(fabs(h->lr) < 1e30) || !(h->eps >= 0)) return refuse(who, "bad lr or eps");
  if (bad_floats(h->grad_scale)) return refuse(who, "grad_scale is not aligned");
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != plan->device) return refuse(who, "the plan was prepared on another device");
  if (plan->tensor_of.empty()) return TDF_OK;
  const AdamArgs a{(const AdamTensor*)plan->workspace,
                   (const uint32_t*)((const char*)plan->workspace + table_bytes(plan->tensors.size())),
                   (float)h->beta1, (float)(1 - h->beta1), (float)h->beta2, (float)(1 - h->beta2),
                   (float)(h->lr / (1 - pow(h->beta1, (double)h->step))), (float)(1 / sqrt(1 - pow(h->beta2, (double)h->step))), (float)h->eps,
                   (float)h->lr, h->grad_scale, h->seed};
  k_adamw<<<(unsigned)plan->tensor_of.size(), 256, 0, (hipStream_t)hip_stream>>>(a);
  return launched(who);
}
