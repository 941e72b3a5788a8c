// One AdamW step over many tensors (mlpmoe_adamw), per element, with the step's number i:
//     g = grad * grad_scale;   m = b1 m + (1 - b1) g;   v = b2 v + (1 - b2) g^2;
//     p = p - lr wd p - lr / (1 - b1^i) * m / (sqrt(v) / sqrt(1 - b2^i) + eps).
// HBM-bound with moments in fp32 (100 M elements: 24 to 30 bytes each at 95 to 98 % of a copy).  In 8 bits the instructions come near the
// memory's time: 71 an element with noise, 9 of them the hash (bf16 params, with a hash more, 85); one Llama-shaped layer with fp32 params and a bf16
// copy, 176 M elements: 2.84 GB in 478 to 514 us by the GPU (86 to 92 %), bf16 params and gradients 55 % with noise, 79 % without.  A moment in 8 bits is e4m3 with a scale per 128
// elements, the second as its root: e4m3 spans 2^17 in the root, 2^34 in v.  A root above zero never becomes zero, which would make
// the next quotient m / eps.  Stochastic rounding there, because a step moves v by 1 - b2 of itself, far below half a step of e4m3,
// so that rounding to nearest would leave most elements where they are.
// The tensors' records travel as the kernel's parameters: nothing to copy or to keep for a captured graph.
#include <cuda_fp8.h>
#include <math.h>

#include <cfloat>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kAdamThreads = 256;
constexpr int kAdamStep = kAdamThreads * 8;      // elements of a block's step
constexpr int kAdamSteps = 16;                   // steps of a block at most
constexpr int kSms = 148;
constexpr int kAdamCtas = 3;                     // blocks of an SM
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
  uint32_t index;       // its place in the caller's list
  uint32_t wide;        // all buffers start on 16 bytes
};

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
  int count, steps;      // steps: of a block
  uint32_t first[K];     // a tensor's first block
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

// Eight elements at p, as they stand in memory; `left` of them exist (zeros for the rest), `whole`: all eight, and p is on 16 bytes.
template <int KIND>
__device__ __forceinline__ Chunk fetch(const char* p, bool whole, int left) {
  if (whole) return load_chunk<true>(p, KIND, 0, 8);
  return load_chunk<false>(p, KIND, 0, left);
}
__device__ __forceinline__ uint2 fetch_codes(const char* p, bool whole, int left) {
  if (whole) return *reinterpret_cast<const uint2*>(p);
  uint32_t w[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < left) w[e / 4] |= static_cast<uint32_t>(static_cast<uint8_t>(p[e])) << (8 * (e % 4));
  return make_uint2(w[0], w[1]);
}
template <int KIND>
__device__ __forceinline__ void put(char* p, bool whole, int left, const float (&v)[8]) {
  if (whole) {
    store8<true>(p, KIND, 0, 8, v);
  } else {
    store8<false>(p, KIND, 0, left, v);
  }
}
__device__ __forceinline__ void put_codes(char* p, bool whole, int left, uint2 c) {
  if (whole) {
    *reinterpret_cast<uint2*>(p) = c;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = static_cast<char>((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
  }
}

__device__ __forceinline__ void values_of(uint2 codes, float (&v)[8]) {
  const uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>(w[e / 4] >> (8 * (e % 4))), __NV_E4M3);
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    v[e] = f.x;
    v[e + 1] = f.y;
  }
}

__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= FLT_MAX; }
__device__ __forceinline__ float max_nan(float a, float b) {      // a NaN wins
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float min3(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float sqrt_fast(float x) {             // off by 2^-23 at most; below 2^-126: 0
  float r;
  asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float reciprocal_fast(float x) {       // off by 2^-23 at most, for x from 2^-126 to 2^126
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float min_nan(float a, float b, float c) {      // a NaN wins
  float r;
  asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Root and reciprocal rounded to nearest: a Newton step from the one-instruction value, its residual exact in one fma (Markstein, "Computation of
// elementary functions on the IBM RISC System/6000 processor", 1990).  Compared with the correctly rounded functions for every fp32 of the range: the root
// from 2^-96 on (0, infinity and what is not normal give a NaN), the reciprocal from 2^-126 to 2^121.  With the functions themselves the Llama-shaped
// layer takes 527 us.
__device__ __forceinline__ float sqrt_newton(float x) {
  float y;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  const float r = __fmul_rn(x, y);
  return fmaf(fmaf(-r, r, x), 0.5f * y, r);
}
__device__ __forceinline__ float reciprocal_newton(float x) {
  const float r = reciprocal_fast(x);
  return fmaf(r, fmaf(-x, r, 1.0f), r);
}
// Smallest magnitude of eight values.
__device__ __forceinline__ float low_of(const float (&x)[8]) {
  float low = min3(fabsf(x[0]), fabsf(x[1]), fabsf(x[2]));
  low = min3(low, fabsf(x[3]), fabsf(x[4]));
  low = min3(low, fabsf(x[5]), fabsf(x[6]));
  return fminf(low, fabsf(x[7]));
}

// Eight values of a block of 128 (16 neighbouring lanes) as codes, and the block's scale.  What is not finite becomes a NaN code and
// stays out of the scale.  Stochastic: up with the probability of what truncation cuts off, by adding 16 random bits and a half
// below the third bit of the fraction (the half also keeps the block's largest at 448); below 2^-6, where the steps of e4m3 no
// longer shrink, to the value plus 2^-6.  Few elements lie there, so a thread without any skips that.
template <bool NOISE, bool ROOT>
__device__ __forceinline__ uint2 codes_of(const float (&x)[8], const uint32_t (&noise)[8], float& scale) {
  float top = max_nan(fabsf(x[0]), fabsf(x[1]), fabsf(x[2]));
  top = max_nan(top, fabsf(x[3]), fabsf(x[4]));
  top = max_nan(top, fabsf(x[5]), fabsf(x[6]));
  top = max_nan(top, fabsf(x[7]));
#pragma unroll
  for (int o = 1; o < kStateBlock / 8; o <<= 1) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  const bool fine = top <= FLT_MAX;
  if (!fine) {                             // the same for all lanes of the block
    top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, finite(x[e]) ? fabsf(x[e]) : 0.0f);
    const uint32_t half = 0xFFFFu << (threadIdx.x & 16);
#pragma unroll
    for (int o = 1; o < kStateBlock / 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(half, top, o));
  }
  scale = fmaxf(top * (1.0f / kE4m3Max), kScaleMin);
  const float inv = reciprocal_newton(scale);
  float y[8];
  if (fine && (!(NOISE || ROOT) || low_of(x) >= scale * (NOISE ? 0.0157f : 0.002f))) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      y[e] = x[e] * inv;
      if (NOISE) {
        const uint32_t bits = (((ROOT ? noise[e] >> 12 : noise[e] << 4) & 0x000FFFF0u) | 8u) + __float_as_uint(y[e]);
        y[e] = __uint_as_float(bits & 0xFFF00000u);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float a = fabsf(x[e]) * inv;
      if (NOISE) {
        const float base = a < 0.015625f ? 0.015625f : 0.0f;
        const uint32_t bits = (((ROOT ? noise[e] >> 12 : noise[e] << 4) & 0x000FFFF0u) | 8u) + __float_as_uint(a + base);
        a = __uint_as_float(bits & 0xFFF00000u) - base;
      }
      if (ROOT && x[e] > 0.0f) a = fmaxf(a, kRootMin);
      y[e] = finite(x[e]) ? copysignf(a, x[e]) : __uint_as_float(0x7FC00000u);
    }
  }
  uint32_t c[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = __nv_cvt_float2_to_fp8x2(make_float2(y[2 * e], y[2 * e + 1]), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
}
struct Rates {
  float keep, rate, inv_root, grad_scale;     // lr wd; lr / (1 - b1^i); 1 / sqrt(1 - b2^i)
  uint32_t key;
};

// A thread's elements of one step, as they stand in memory.
template <bool EIGHT>
struct Raw {
  Chunk p, g, m, v;
  uint2 m8, v8;
  float m_scale, v_scale;
};

// A block to a stretch of one tensor, 2048 elements a step; the next step's loads are under way while one is computed.
template <int K, int PK, int GK, bool EIGHT, bool NOISE>
__global__ void __launch_bounds__(kAdamThreads, kAdamCtas) adamw_kernel(const __grid_constant__ AdamArgs<K> a) {
  __shared__ Rates shared_rates;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  int lo = 0, hi = a.count - 1;
  while (lo < hi) {                        // the last tensor that starts at this block or before it
    const int mid = (lo + hi + 1) / 2;
    if (a.first[mid] <= blockIdx.x) {
      lo = mid;
    } else {
      hi = mid - 1;
    }
  }
  const AdamTensor& t = a.t[lo];
  const AdamSettings& s = a.s;
  const int64_t start = static_cast<int64_t>(blockIdx.x - a.first[lo]) * a.steps * kAdamStep, first = start + threadIdx.x * 8;
  const int64_t rest = t.n - start;
  const int count = static_cast<int>(rest < static_cast<int64_t>(a.steps) * kAdamStep ? rest : static_cast<int64_t>(a.steps) * kAdamStep);
  const bool wide = t.wide != 0;
  constexpr int PB = bytes_of(PK), GB = bytes_of(GK), SB = EIGHT ? 1 : 4;
  char* const p_at = static_cast<char*>(t.p) + first * PB;
  const char* const g_at = static_cast<const char*>(t.g) + first * GB;
  char* const m_at = static_cast<char*>(t.m) + first * SB;
  char* const v_at = static_cast<char*>(t.v) + first * SB;
  char* const copy_at = reinterpret_cast<char*>(t.copy + first);
  float* const ms_at = t.m_scale + first / kStateBlock;
  float* const vs_at = t.v_scale + first / kStateBlock;
  const bool copies = PK == MLPMOE_FP32 && t.copy != nullptr;
  const int mine = threadIdx.x * 8;
  // at: of the step; whole: the step is full and its buffers are on 16 bytes
  auto load = [&](int at, Raw<EIGHT>& r) {
    const bool whole = wide && at + kAdamStep <= count;
    const int left = min(8, count - at - mine);
    auto all = [&](bool eight_there) {
      r.p = fetch<PK>(p_at + at * PB, eight_there, left);
      r.g = fetch<GK>(g_at + at * GB, eight_there, left);
      if (EIGHT) {
        r.m8 = fetch_codes(m_at + at, eight_there, left);
        r.v8 = fetch_codes(v_at + at, eight_there, left);
        r.m_scale = ms_at[at / kStateBlock];
        r.v_scale = vs_at[at / kStateBlock];
      } else {
        r.m = fetch<MLPMOE_FP32>(m_at + at * 4, eight_there, left);
        r.v = fetch<MLPMOE_FP32>(v_at + at * 4, eight_there, left);
      }
    };
    if (whole) {                           // one branch a step, not one a buffer
      all(true);
    } else if (left > 0) {
      all(false);
    }
  };
  Raw<EIGHT> next = {};
  load(0, next);
  if (threadIdx.x == 0) {                  // while the loads are under way
    int64_t step = s.step_device != nullptr ? *s.step_device : s.step;
    if (step < 1) step = 1;
    const float lr = s.lr_device != nullptr ? *s.lr_device : s.lr;
    Rates r;
    r.keep = lr * t.decay;
    r.rate = lr / -expm1f(static_cast<float>(step) * s.log_b1);
    r.inv_root = 1.0f / sqrtf(-expm1f(static_cast<float>(step) * s.log_b2));
    r.grad_scale = s.grad_scale != nullptr ? *s.grad_scale : 1.0f;
    r.key = mix(t.index ^ mix(s.key ^ static_cast<uint32_t>(step)));
    shared_rates = r;
  }
  __syncthreads();
  const Rates r = shared_rates;
#pragma unroll 1
  for (int at = 0; at < count; at += kAdamStep) {
    const Raw<EIGHT> now = next;
    if (at + kAdamStep < count) load(at + kAdamStep, next);
    const bool whole = wide && at + kAdamStep <= count;
    const int left = min(8, count - at - mine);
    float p[8], g[8], m[8], v[8];
    to_f32(now.p, PK, p);
    to_f32(now.g, GK, g);
    if (EIGHT) {
      values_of(now.m8, m);
      values_of(now.v8, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        m[e] = __fmul_rn(m[e], now.m_scale);
        v[e] = __fmul_rn(v[e], now.v_scale);
        v[e] = __fmul_rn(v[e], v[e]);
      }
    } else {
      to_f32(now.m, MLPMOE_FP32, m);
      to_f32(now.v, MLPMOE_FP32, v);
    }
    // Each product and sum is rounded by itself, in the formulas' order, and in 8 bits the root too, so that a code can be computed again bit by bit.  With
    // fused sums and the approximate root one code in a million was its neighbour, and where it then was its block's largest, the next step's scale was off by
    // up to 6 %.  8 instructions of the 71; fp32 params 477 -> 478 to 489 us on one GPU, bf16 params with noise 265 -> 290 (105 M elements).
    float root[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = __fmul_rn(g[e], r.grad_scale);
      m[e] = __fadd_rn(__fmul_rn(s.b1, m[e]), __fmul_rn(s.one_b1, y));
      v[e] = __fadd_rn(__fmul_rn(s.b2, v[e]), __fmul_rn(__fmul_rn(s.one_b2, y), y));
      root[e] = EIGHT ? sqrt_newton(v[e]) : sqrt_fast(v[e]);
    }
    // zeros among them; in 8 bits also infinity
    if (EIGHT ? !(min_nan(min_nan(min_nan(root[0], root[1], root[2]), root[3], root[4]), root[5], min_nan(root[6], root[7], root[7])) >= 0x1p-48f) : low_of(v) < FLT_MIN) {
#pragma unroll
      for (int e = 0; e < 8; ++e) root[e] = sqrtf(v[e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      p[e] = fmaf(-r.rate, m[e] * reciprocal_fast(fmaf(root[e], r.inv_root, s.eps)), fmaf(-r.keep, p[e], p[e]));
    uint32_t noise[8];
    if (NOISE) {
      const int64_t i = first + at;
      uint32_t key = r.key;
      if (i >> 32) key = mix(key ^ static_cast<uint32_t>(i >> 32));      // (2048 elements of a step lie in the same 2^32)
#pragma unroll
      for (int e = 0; e < 8; ++e) noise[e] = mix(key + static_cast<uint32_t>(i) * 0x9E3779B1u + e * 0x9E3779B1u);
    }
    uint2 code_m, code_v;
    float scale_m, scale_v;
    if (EIGHT) {
      if (!whole) {                        // what lies behind the end must not reach the last block's scales
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= left) m[e] = root[e] = 0.0f;
      }
      code_m = codes_of<NOISE, false>(m, noise, scale_m);
      code_v = codes_of<NOISE, true>(root, noise, scale_v);
    }
    float rounded[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      rounded[e] = p[e];
      if (NOISE && PK == MLPMOE_BF16 && finite(p[e]))
        rounded[e] = __uint_as_float((__float_as_uint(p[e]) + (mix(noise[e] ^ 0x9E3779B1u) & 0xFFFFu)) & 0xFFFF0000u);
    }
    auto all = [&](bool eight_there) {
      if (copies) put<MLPMOE_BF16>(copy_at + at * 2, eight_there, left, p);
      put<PK>(p_at + at * PB, eight_there, left, rounded);
      if (EIGHT) {
        if (threadIdx.x % (kStateBlock / 8) == 0) {
          ms_at[at / kStateBlock] = scale_m;
          vs_at[at / kStateBlock] = scale_v;
        }
        put_codes(m_at + at, eight_there, left, code_m);
        put_codes(v_at + at, eight_there, left, code_v);
      } else {
        put<MLPMOE_FP32>(m_at + at * 4, eight_there, left, m);
        put<MLPMOE_FP32>(v_at + at * 4, eight_there, left, v);
      }
    };
    if (whole) {
      all(true);
    } else if (left > 0) {
      all(false);
    }
  }
}

// Tensors of one launch: 4 KB of parameters hold 44 records, 32 KB 384; the host pays for what is passed (72 tensors: 13.3 us a call with 32 KB,
// 10.7 with 11).
constexpr int kAdamFew = 44, kAdamSome = 128, kAdamMany = 384;
static_assert(sizeof(AdamArgs<kAdamFew>) <= 4096 && sizeof(AdamArgs<kAdamMany>) <= 32764, "kernel parameters");

// A launch takes tensors of one set of types.
struct Kinds {
  bool p16, g16, eight, noise;
};

template <int K, int PK, int GK>
cudaError_t launch_kinds(const Kinds& k, unsigned blocks, const AdamArgs<K>& a, cudaStream_t st) {
  const dim3 grid(blocks), block(kAdamThreads);
  if (k.eight)
    return k.noise ? launch_pdl(adamw_kernel<K, PK, GK, true, true>, grid, block, 0, st, a) : launch_pdl(adamw_kernel<K, PK, GK, true, false>, grid, block, 0, st, a);
  // moments in fp32: nothing to round but a bf16 param
  return k.noise && PK == MLPMOE_BF16 ? launch_pdl(adamw_kernel<K, PK, GK, false, PK == MLPMOE_BF16>, grid, block, 0, st, a)
                                      : launch_pdl(adamw_kernel<K, PK, GK, false, false>, grid, block, 0, st, a);
}

template <int K>
cudaError_t launch_adamw(const AdamSettings& s, const AdamTensor* t, int count, const Kinds& k, cudaStream_t st) {
  AdamArgs<K> a;
  a.s = s;
  a.count = count;
  // steps of a block: as many as leave every SM its blocks twice over
  int64_t total = 0;
  for (int i = 0; i < count; ++i) total += (t[i].n + kAdamStep - 1) / kAdamStep;
  const int64_t most = total / (2 * kAdamCtas * kSms);
  a.steps = most < 1 ? 1 : (most > kAdamSteps ? kAdamSteps : static_cast<int>(most));
  const int64_t per = static_cast<int64_t>(a.steps) * kAdamStep;
  uint64_t blocks = 0;
  for (int i = 0; i < count; ++i) {
    a.t[i] = t[i];
    a.first[i] = static_cast<uint32_t>(blocks);
    blocks += (t[i].n + per - 1) / per;
  }
  const unsigned grid = static_cast<unsigned>(blocks);
  if (k.p16)
    return k.g16 ? launch_kinds<K, MLPMOE_BF16, MLPMOE_BF16>(k, grid, a, st) : launch_kinds<K, MLPMOE_BF16, MLPMOE_FP32>(k, grid, a, st);
  return k.g16 ? launch_kinds<K, MLPMOE_FP32, MLPMOE_BF16>(k, grid, a, st) : launch_kinds<K, MLPMOE_FP32, MLPMOE_FP32>(k, grid, a, st);
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
  if (!(o.beta1 >= 0.0 && o.beta1 < 1.0) || !(o.beta2 >= 0.0 && o.beta2 < 1.0) || !(o.eps <= FLT_MAX) || !(static_cast<float>(o.eps) >= FLT_MIN))
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
  for (int kind = 0; kind < 8; ++kind) {
    const Kinds k = {(kind & 1) != 0, (kind & 2) != 0, (kind & 4) != 0, o.stochastic != 0};
    AdamTensor batch[kAdamMany];
    int count = 0;
    int64_t blocks = 0;
    auto flush = [&]() {
      if (count == 0) return cudaSuccess;
      const cudaError_t e = count <= kAdamFew    ? launch_adamw<kAdamFew>(s, batch, count, k, st)
                            : count <= kAdamSome ? launch_adamw<kAdamSome>(s, batch, count, k, st)
                                                 : launch_adamw<kAdamMany>(s, batch, count, k, st);
      count = 0;
      blocks = 0;
      return e;
    };
    for (int32_t i = 0; i < n_tensors; ++i) {
      const mlpmoe_adamw_tensor_t& t = tensors[i];
      if (t.n == 0 || (t.param_dtype == MLPMOE_BF16) != k.p16 || (t.grad_dtype == MLPMOE_BF16) != k.g16 || (t.state_dtype == MLPMOE_E4M3) != k.eight) continue;
      const int64_t need = (t.n + kAdamStep - 1) / kAdamStep;      // blocks at most
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
      r.wide = on(t.param, 16) && on(t.grad, 16) && on(t.m, 16) && on(t.v, 16) && on(t.param_bf16, 16);
    }
    if (flush() != cudaSuccess) return MLPMOE_ERR_CUDA;
  }
  return MLPMOE_OK;
}
