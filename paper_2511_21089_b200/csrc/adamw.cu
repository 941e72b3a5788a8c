// One AdamW step over many tensors (mlpmoe_adamw), per element, with the step's number i:
//     g = grad * grad_scale;   m = b1 m + (1 - b1) g;   v = b2 v + (1 - b2) g^2;
//     p = p - lr wd p - lr / (1 - b1^i) * m / (sqrt(v) / sqrt(1 - b2^i) + eps).
// HBM-bound with moments in fp32 (28 to 30 bytes an element for 40 instructions).  In 8 bits a moment is e4m3 with a scale per 128
// elements, the second as its root: e4m3 spans 2^17 in the root, 2^34 in v.  A root above zero never becomes zero, which would make
// the next quotient m / eps.  Stochastic rounding there, because a step moves v by 1 - b2 of itself, far below half a step of e4m3,
// so that rounding to nearest would leave most elements where they are.
// The tensors' records travel as the kernel's parameters: nothing to copy or to keep for a captured graph.
#include <cuda_fp8.h>
#include <math.h>

#include <cfloat>
#include <vector>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamTurns = 2;                                  // chunks of eight elements of a thread
constexpr int kAdamBlock = kAdamThreads * 8 * kAdamTurns;      // elements of a block
constexpr int kStateBlock = 128;                               // elements of a scale
constexpr float kE4m3Max = 448.0f;
constexpr float kScaleMin = 1.17549435e-38f;                   // 2^-126
constexpr float kRootMin = 1.0f / 512.0f;                      // the smallest e4m3 above zero

struct AdamTensor {
  void* p;
  const void* g;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  __nv_bfloat16* copy;
  int64_t n;
  float decay;
  uint32_t first;       // the tensor's first block
  uint32_t index;       // its place in the caller's list
  uint32_t flags;
};
constexpr uint32_t kParamBf16 = 1, kGradBf16 = 2, kWide = 4;

struct AdamSettings {
  float lr, b1, b2, one_b1, one_b2, eps, log_b1, log_b2;
  const float* lr_device;
  const int64_t* step_device;
  const float* grad_scale;
  int64_t step;
  uint32_t key;         // of the seed
};

template <int K>
struct AdamArgs {
  AdamSettings s;
  int count;
  AdamTensor t[K];
};

// The 32-bit finaliser of MurmurHash3.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
  h ^= h >> 16;
  h *= 0x85EBCA6Bu;
  h ^= h >> 13;
  h *= 0xC2B2AE35u;
  return h ^ (h >> 16);
}

__device__ __forceinline__ void load8(const void* base, bool bf16, int64_t i, int64_t n, bool wide, float (&v)[8]) {
  const int kind = bf16 ? MLPMOE_BF16 : MLPMOE_FP32;
  const char* p = static_cast<const char*>(base) + i * bytes_of(kind);
  if (wide && i + 8 <= n) {
    to_f32(load_chunk<true>(p, kind, 0, 8), kind, v);
  } else {
    to_f32(load_chunk<false>(p, kind, 0, static_cast<int>(n - i < 8 ? n - i : 8)), kind, v);
  }
}
__device__ __forceinline__ void store_to(void* base, bool bf16, int64_t i, int64_t n, bool wide, const float (&v)[8]) {
  const int kind = bf16 ? MLPMOE_BF16 : MLPMOE_FP32;
  char* p = static_cast<char*>(base) + i * bytes_of(kind);
  if (wide && i + 8 <= n) {
    store8<true>(p, kind, 0, 8, v);
  } else {
    store8<false>(p, kind, 0, static_cast<int>(n - i < 8 ? n - i : 8), v);
  }
}

// Eight e4m3 codes as their values.
__device__ __forceinline__ void load_codes(const void* base, int64_t i, int64_t n, bool wide, float (&v)[8]) {
  const uint8_t* p = static_cast<const uint8_t*>(base) + i;
  uint32_t w[2] = {0u, 0u};
  if (wide && i + 8 <= n) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x;
    w[1] = u.y;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < n) w[e / 4] |= static_cast<uint32_t>(p[e]) << (8 * (e % 4));
  }
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[e / 4] >> (8 * (e % 4))), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[e] = f.x;
    v[e + 1] = f.y;
  }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= FLT_MAX; }

// Eight values of a block of 128 (16 lanes) to codes and the block's scale.  What is not finite becomes a NaN code and stays out of the scale.
template <bool NOISE, bool ROOT>
__device__ __forceinline__ void store_codes(void* base, float* scales, int64_t i, int64_t n, bool wide, const float (&x)[8], const uint32_t (&noise)[8]) {
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, finite(x[e]) ? fabsf(x[e]) : 0.0f);
#pragma unroll
  for (int o = 1; o < kStateBlock / 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  const float scale = fmaxf(top / kE4m3Max, kScaleMin), inv = 1.0f / scale;
  if (i >= n) return;
  if (i % kStateBlock == 0) scales[i / kStateBlock] = scale;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float a = fminf(fabsf(x[e]) * inv, kE4m3Max);
    if (NOISE) {
      // up with the probability of what truncation would cut: 16 random bits (and a half) added below the third bit of the fraction;
      // below 2^-6, where the steps no longer shrink, on the value plus 2^-6
      const float base_of = a < 0.015625f ? 0.015625f : 0.0f;
      const uint32_t bits = __float_as_uint(a + base_of) + (((ROOT ? noise[e] >> 16 : noise[e] & 0xFFFFu) << 4) | 8u);
      a = fminf(__uint_as_float(bits & 0xFFF00000u) - base_of, kE4m3Max);
    }
    if (ROOT && x[e] > 0.0f) a = fmaxf(a, kRootMin);
    y[e] = finite(x[e]) ? copysignf(a, x[e]) : __uint_as_float(0x7FC00000u);
  }
  uint32_t c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = __nv_cvt_float2_to_fp8x2(make_float2(y[2 * e], y[2 * e + 1]), __NV_SATFINITE, __NV_E4M3);
  uint8_t* p = static_cast<uint8_t*>(base) + i;
  if (wide && i + 8 <= n) {
    *reinterpret_cast<uint2*>(p) = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (i + e < n) p[e] = static_cast<uint8_t>(c[e / 2] >> (8 * (e & 1)));
  }
}

template <int K, bool EIGHT, bool NOISE>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamArgs<K> a) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {                        // the last tensor that starts at this block or before it
    const int mid = (lo + hi + 1) / 2;
    if (a.t[mid].first <= blockIdx.x) {
      lo = mid;
    } else {
      hi = mid - 1;
    }
  }
  const AdamTensor& t = a.t[lo];
  const AdamSettings& s = a.s;
  int64_t step = s.step_device != nullptr ? *s.step_device : s.step;
  if (step < 1) step = 1;
  const float lr = s.lr_device != nullptr ? *s.lr_device : s.lr;
  const float gs = s.grad_scale != nullptr ? *s.grad_scale : 1.0f;
  const float fstep = static_cast<float>(step);
  const float rate = lr / -expm1f(fstep * s.log_b1);
  const float inv_root = 1.0f / sqrtf(-expm1f(fstep * s.log_b2));
  const float keep = lr * t.decay;
  const bool p16 = t.flags & kParamBf16, g16 = t.flags & kGradBf16, wide = t.flags & kWide;
  const int64_t start = static_cast<int64_t>(blockIdx.x - t.first) * kAdamBlock;
  uint32_t key = 0;
  if (NOISE) {
    key = mix(t.index ^ mix(s.key ^ static_cast<uint32_t>(step)));
    if (start >> 32) key = mix(key ^ static_cast<uint32_t>(start >> 32));
  }
#pragma unroll
  for (int turn = 0; turn < kAdamTurns; ++turn) {
    const int64_t i = start + (turn * kAdamThreads + threadIdx.x) * 8;
    float p[8] = {}, g[8] = {}, m[8] = {}, v[8] = {};
    if (i < t.n) {
      load8(t.p, p16, i, t.n, wide, p);
      load8(t.g, g16, i, t.n, wide, g);
      if (EIGHT) {
        load_codes(t.m, i, t.n, wide, m);
        load_codes(t.v, i, t.n, wide, v);
        const float ms = t.m_scale[i / kStateBlock], vs = t.v_scale[i / kStateBlock];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          m[e] *= ms;
          v[e] *= vs;
          v[e] *= v[e];
        }
      } else {
        load8(t.m, false, i, t.n, wide, m);
        load8(t.v, false, i, t.n, wide, v);
      }
    }
    float root[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = g[e] * gs;
      m[e] = fmaf(s.b1, m[e], s.one_b1 * x);
      v[e] = fmaf(s.b2, v[e], s.one_b2 * x * x);
      root[e] = sqrtf(v[e]);
      p[e] = p[e] - keep * p[e] - rate * (m[e] / fmaf(root[e], inv_root, s.eps));
    }
    uint32_t noise[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) noise[e] = NOISE ? mix(key + (static_cast<uint32_t>(i) + e) * 0x9E3779B1u) : 0u;
    if (i < t.n) {
      if (t.copy != nullptr) store_to(t.copy, true, i, t.n, wide, p);
      if (NOISE && p16) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (finite(p[e])) p[e] = __uint_as_float((__float_as_uint(p[e]) + (mix(noise[e] ^ 0x9E3779B1u) & 0xFFFFu)) & 0xFFFF0000u);
      }
      store_to(t.p, p16, i, t.n, wide, p);
      if (!EIGHT) {
        store_to(t.m, false, i, t.n, wide, m);
        store_to(t.v, false, i, t.n, wide, v);
      }
    }
    if (EIGHT) {
      store_codes<NOISE, false>(t.m, t.m_scale, i, t.n, wide, m, noise);
      store_codes<NOISE, true>(t.v, t.v_scale, i, t.n, wide, root, noise);
    }
  }
}

// Tensors of one launch: 4 KB of parameters hold 44 records, 32 KB 400.
constexpr int kAdamFew = 44, kAdamMany = 400;
static_assert(sizeof(AdamArgs<kAdamFew>) <= 4096 && sizeof(AdamArgs<kAdamMany>) <= 32764, "kernel parameters");

template <int K>
cudaError_t launch_adamw(const AdamSettings& s, const AdamTensor* t, int count, bool eight, bool noise, cudaStream_t st) {
  AdamArgs<K> a;
  a.s = s;
  a.count = count;
  uint64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    a.t[i] = t[i];
    a.t[i].first = static_cast<uint32_t>(blocks);
    blocks += (t[i].n + kAdamBlock - 1) / kAdamBlock;
  }
  const dim3 grid(static_cast<unsigned>(blocks)), block(kAdamThreads);
  if (eight)
    return noise ? launch_pdl(adamw_kernel<K, true, true>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<K, true, false>, grid, block, 0, st, a);
  return noise ? launch_pdl(adamw_kernel<K, false, true>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<K, false, false>, grid, block, 0, st, a);
}

mlpmoe_status_t check_tensor(const mlpmoe_adamw_tensor_t& t) {
  const bool eight = t.state_dtype == MLPMOE_E4M3;
  if (t.n < 0 || !(t.weight_decay >= 0.0f && t.weight_decay <= FLT_MAX)) return MLPMOE_ERR_INVALID_ARG;
  if ((t.param_dtype != MLPMOE_FP32 && t.param_dtype != MLPMOE_BF16) || (t.grad_dtype != MLPMOE_FP32 && t.grad_dtype != MLPMOE_BF16) ||
      (t.state_dtype != MLPMOE_FP32 && !eight) || (t.param_bf16 && t.param_dtype != MLPMOE_FP32))
    return MLPMOE_ERR_INVALID_ARG;
  if (t.n > (int64_t{1} << 40)) return MLPMOE_ERR_UNSUPPORTED;
  if (t.n == 0) return MLPMOE_OK;
  if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return MLPMOE_ERR_INVALID_ARG;
  const uintptr_t sb = eight ? 1 : 4;
  if (!on(t.param, bytes_of(t.param_dtype)) || !on(t.grad, bytes_of(t.grad_dtype)) || !on(t.m, sb) || !on(t.v, sb) || !on(t.param_bf16, 2) ||
      (eight && (!on(t.m_scale, 4) || !on(t.v_scale, 4))))
    return MLPMOE_ERR_INVALID_ARG;
  return MLPMOE_OK;
}

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" mlpmoe_status_t mlpmoe_adamw(const mlpmoe_adamw_tensor_t* tensors, int32_t n_tensors, const mlpmoe_adamw_settings_t* settings,
                                        void* stream) {
  if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !settings) return MLPMOE_ERR_INVALID_ARG;
  const mlpmoe_adamw_settings_t& o = *settings;
  if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0) || !(o.eps <= FLT_MAX) || !(static_cast<float>(o.eps) > 0.0f))
    return MLPMOE_ERR_INVALID_ARG;
  if (!(fabs(o.lr) <= FLT_MAX) || (!o.step_device && o.step < 1)) return MLPMOE_ERR_INVALID_ARG;
  if (!on(o.lr_device, 4) || !on(o.grad_scale, 4) || !on(o.step_device, 8)) return MLPMOE_ERR_INVALID_ARG;
  for (int32_t i = 0; i < n_tensors; ++i) {
    const mlpmoe_status_t rc = check_tensor(tensors[i]);      // all of them before the first launch
    if (rc != MLPMOE_OK) return rc;
  }
  AdamSettings s = {};
  s.lr = static_cast<float>(o.lr);
  s.b1 = static_cast<float>(o.beta1);
  s.b2 = static_cast<float>(o.beta2);
  s.one_b1 = static_cast<float>(1.0 - o.beta1);
  s.one_b2 = static_cast<float>(1.0 - o.beta2);
  s.eps = static_cast<float>(o.eps);
  s.log_b1 = static_cast<float>(log(o.beta1));
  s.log_b2 = static_cast<float>(log(o.beta2));
  s.lr_device = o.lr_device;
  s.step_device = o.step_device;
  s.grad_scale = o.grad_scale;
  s.step = o.step;
  s.key = mix(mix(static_cast<uint32_t>(o.seed)) ^ static_cast<uint32_t>(o.seed >> 32));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  pdl_overlap_enabled() = true;
  for (const bool eight : {false, true}) {
    AdamTensor batch[kAdamMany];
    int count = 0;
    int64_t blocks = 0;
    auto flush = [&]() {
      if (count == 0) return cudaSuccess;
      const cudaError_t e = count <= kAdamFew ? launch_adamw<kAdamFew>(s, batch, count, eight, o.stochastic != 0, st)
                                              : launch_adamw<kAdamMany>(s, batch, count, eight, o.stochastic != 0, st);
      count = 0;
      blocks = 0;
      return e;
    };
    for (int32_t i = 0; i < n_tensors; ++i) {
      const mlpmoe_adamw_tensor_t& t = tensors[i];
      if (t.n == 0 || (t.state_dtype == MLPMOE_E4M3) != eight) continue;
      const int64_t need = (t.n + kAdamBlock - 1) / kAdamBlock;
      if ((count == kAdamMany || blocks + need > INT32_MAX) && flush() != cudaSuccess) return MLPMOE_ERR_CUDA;
      AdamTensor& r = batch[count++];
      blocks += need;
      r.p = t.param;
      r.g = t.grad;
      r.m = t.m;
      r.v = t.v;
      r.m_scale = t.m_scale;
      r.v_scale = t.v_scale;
      r.copy = static_cast<__nv_bfloat16*>(t.param_bf16);
      r.n = t.n;
      r.decay = t.weight_decay;
      r.index = static_cast<uint32_t>(i);
      const bool wide = on(t.param, 16) && on(t.grad, 16) && on(t.m, 16) && on(t.v, 16) && on(t.param_bf16, 16);
      r.flags = (t.param_dtype == MLPMOE_BF16 ? kParamBf16 : 0u) | (t.grad_dtype == MLPMOE_BF16 ? kGradBf16 : 0u) | (wide ? kWide : 0u);
    }
    if (flush() != cudaSuccess) return MLPMOE_ERR_CUDA;
  }
  return MLPMOE_OK;
}
