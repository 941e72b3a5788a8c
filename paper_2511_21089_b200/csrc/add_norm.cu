// Residual addition + RMSNorm + (optionally) 8-bit output with scales in one pass (mlpmoe_add_rmsnorm):
//     s = x + r,  x_out = s,  v = s / sqrt(mean(s^2) + eps) * gain,  out = v | e4m3(v / scale).
// HBM-bound (a few operations per element): every element of x and r is read once and stays in registers
// between the sum of squares and the output, so a row costs one trip through memory.  16384 x 4096 fp32 + bf16 to fp32 and
// e4m3 with scales: 738 MB in 120 to 129 us over seconds of it, 113 in runs of 30 ms (a copy: 119); one token 2 us (latency of one
// load, a block sum, a store).
#include <cuda_fp8.h>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"

namespace mlpmoe {
namespace {

constexpr int kNone = 2;   // no residual, beside MLPMOE_BF16 (0) and MLPMOE_FP32 (1)
constexpr float kE4m3Max = 448.0f;
constexpr float kScaleMin = 1.17549435e-38f;   // 2^-126: keeps 1 / scale finite; a group of zeros gets it too

struct NormArgs {
  const void* x;
  const void* r;
  const float* gain;
  void* x_out;
  void* out;
  float* scales;
  int64_t x_stride, r_stride, x_out_stride, out_stride, n;
  int d, group;   // group: columns per scale, d for one per row
  float eps;
};

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Eight consecutive elements from column col, as they stand in memory (fp32: the whole of a and b; bf16: a), zeros past the
// row's end.  VEC: the row starts on 16 bytes and d % 8 == 0, so a chunk is whole.
struct Chunk {
  uint4 a, b;
};
template <bool VEC>
__device__ __forceinline__ Chunk load_chunk(const void* row, int kind, int col, int d) {
  Chunk c;
  c.a = c.b = make_uint4(0u, 0u, 0u, 0u);
  if (col >= d) return c;
  if (kind == MLPMOE_FP32) {
    const uint32_t* p = static_cast<const uint32_t*>(row) + col;
    if (VEC) {
      c.a = reinterpret_cast<const uint4*>(p)[0];
      c.b = reinterpret_cast<const uint4*>(p)[1];
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = col + i < d ? p[i] : 0u;
      c.a = make_uint4(w[0], w[1], w[2], w[3]);
      c.b = make_uint4(w[4], w[5], w[6], w[7]);
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(row) + col;
    if (VEC) {
      c.a = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = col + i < d ? p[i] : 0u;
      c.a = make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
    }
  }
  return c;
}
__device__ __forceinline__ void to_f32(const Chunk& c, int kind, float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    v[0] = __uint_as_float(c.a.x), v[1] = __uint_as_float(c.a.y), v[2] = __uint_as_float(c.a.z), v[3] = __uint_as_float(c.a.w);
    v[4] = __uint_as_float(c.b.x), v[5] = __uint_as_float(c.b.y), v[6] = __uint_as_float(c.b.z), v[7] = __uint_as_float(c.b.w);
  } else {
    v[0] = bf16_lo(c.a.x), v[1] = bf16_hi(c.a.x), v[2] = bf16_lo(c.a.y), v[3] = bf16_hi(c.a.y);
    v[4] = bf16_lo(c.a.z), v[5] = bf16_hi(c.a.z), v[6] = bf16_lo(c.a.w), v[7] = bf16_hi(c.a.w);
  }
}

template <bool VEC>
__device__ __forceinline__ void store8(void* row, int kind, int col, int d, const float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    float* p = static_cast<float*>(row) + col;
    if (VEC) {
      __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = v[i];
    }
  } else if (kind == MLPMOE_BF16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(row) + col;
    if (VEC) {
      *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = __float2bfloat16_rn(v[i]);
    }
  } else {
    uint8_t* p = static_cast<uint8_t*>(row) + col;
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    if (VEC) {
      *reinterpret_cast<uint2*>(p) = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = static_cast<uint8_t>(c[i / 2] >> (8 * (i & 1)));
    }
  }
}

// Sum (or maximum) over the T threads of a row, the same bits in all of them.  T = 32: the row's warp; else the block.
template <int T, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xFFFFFFFFu, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  if (T > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) v = MAX ? fmaxf(v, red[i]) : v + red[i];
    __syncthreads();
  }
  return v;
}

// One row per T threads (T = 32: eight rows to a block), NCH chunks of eight consecutive columns per thread.
// A group of 32, 64 or 128 columns lies in 4, 8 or 16 neighbouring lanes of one warp, so its maximum is a few shuffles.
template <int XKIND, int RKIND, int OKIND, bool VEC, int T, int NCH>
__global__ void __launch_bounds__(T == 32 ? 256 : T) add_norm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int tid = T == 32 ? threadIdx.x % 32 : threadIdx.x;
  const int64_t t = T == 32 ? static_cast<int64_t>(blockIdx.x) * 8 + threadIdx.x / 32 : blockIdx.x;
  if (t >= a.n) return;                      // T == 32 only: whole warps leave, no block barrier follows
  constexpr int kXBytes = XKIND == MLPMOE_FP32 ? 4 : 2;
  constexpr int kOBytes = OKIND == MLPMOE_FP32 ? 4 : (OKIND == MLPMOE_BF16 ? 2 : 1);
  const char* xrow = static_cast<const char*>(a.x) + t * a.x_stride * kXBytes;
  const char* rrow = static_cast<const char*>(a.r) + t * a.r_stride * (RKIND == MLPMOE_FP32 ? 4 : 2);
  const int d = a.d;
  float s[NCH][8];
  {
    Chunk x[NCH], r[NCH];               // all of the row's loads before the first use
#pragma unroll
    for (int i = 0; i < NCH; ++i) x[i] = load_chunk<VEC>(xrow, XKIND, (i * T + tid) * 8, d);
    if (RKIND != kNone) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) r[i] = load_chunk<VEC>(rrow, RKIND, (i * T + tid) * 8, d);
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      to_f32(x[i], XKIND, s[i]);
      if (RKIND != kNone) {
        float v[8];
        to_f32(r[i], RKIND, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] += v[j];
      }
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += s[i][j] * s[i][j];
  if (a.x_out != nullptr) {
    char* xo = static_cast<char*>(a.x_out) + t * a.x_out_stride * kXBytes;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int col = (i * T + tid) * 8;
      if (col < d) store8<VEC>(xo, XKIND, col, d, s[i]);
    }
  }
  ss = row_reduce<T, false>(ss, red);
  const float inv = 1.0f / sqrtf(ss / static_cast<float>(d) + a.eps);
  float row_max = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int col = (i * T + tid) * 8;
    float g[8];
    if (a.gain != nullptr) {
      to_f32(load_chunk<VEC>(a.gain, MLPMOE_FP32, col, d), MLPMOE_FP32, g);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[i][j] = s[i][j] * inv * g[j];
      if (OKIND == MLPMOE_E4M3) row_max = fmaxf(row_max, fabsf(s[i][j]));
    }
  }
  char* orow = static_cast<char*>(a.out) + t * a.out_stride * kOBytes;
  if (OKIND == MLPMOE_E4M3) {
    const bool per_row = a.group >= d;
    float row_inv = 0.0f;
    if (per_row) {
      row_max = row_reduce<T, true>(row_max, red);
      const float scale = fmaxf(row_max / kE4m3Max, kScaleMin);
      if (tid == 0) a.scales[t] = scale;
      row_inv = 1.0f / scale;
    }
    const int lanes = a.group / 8;           // lanes of a group: 4, 8 or 16
    const int64_t n_groups = per_row ? 1 : (d + a.group - 1) / a.group;
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int col = (i * T + tid) * 8;
      float ginv = row_inv;
      if (!per_row) {
        float m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) m = fmaxf(m, fabsf(s[i][j]));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        if (lanes > 4) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
        if (lanes > 8) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
        const float scale = fmaxf(m / kE4m3Max, kScaleMin);
        if (col < d && col % a.group == 0) a.scales[t * n_groups + col / a.group] = scale;
        ginv = 1.0f / scale;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) s[i][j] *= ginv;
    }
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int col = (i * T + tid) * 8;
    if (col < d) store8<VEC>(orow, OKIND, col, d, s[i]);
  }
}

// A row to a block whose threads take eight columns each: all loads of a row are in flight at once and none is idle long.  A warp
// to a row (no block barrier) where a row is 512 columns at most and there are many: 65536 x 512 60.6 us against 69.9,
// while at 1200 rows both take 3.1.  Rows of more than 8192 columns that are not aligned spill up to 132 bytes a thread.  Two chunks to a thread for 8-bit output of longer rows, whose scales are half the
// work: 16384 x 4096 111 us against 129 with one (bf16 output: 121 against 117, so it keeps one).
template <int XKIND, int RKIND, int OKIND, bool VEC>
cudaError_t launch_shape(const NormArgs& a, cudaStream_t st) {
  const unsigned n = static_cast<unsigned>(a.n);
  if (a.d <= 512 && a.n > 4096) return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 32, 2>, dim3((n + 7) / 8), dim3(256), 0, st, a);
  if (a.d <= 1024) return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 128, 1>, dim3(n), dim3(128), 0, st, a);
  if (a.d <= 2048) return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 256, 1>, dim3(n), dim3(256), 0, st, a);
  if (a.d <= 4096 && OKIND == MLPMOE_E4M3 && a.n > 1024)
    return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 256, 2>, dim3(n), dim3(256), 0, st, a);
  if (a.d <= 4096) return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 512, 1>, dim3(n), dim3(512), 0, st, a);
  if (a.d <= 8192) return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 512, 2>, dim3(n), dim3(512), 0, st, a);
  return launch_pdl(add_norm_kernel<XKIND, RKIND, OKIND, VEC, 1024, 4>, dim3(n), dim3(1024), 0, st, a);
}

template <int XKIND, int RKIND, int OKIND>
cudaError_t launch_vec(const NormArgs& a, bool vec, cudaStream_t st) {
  return vec ? launch_shape<XKIND, RKIND, OKIND, true>(a, st) : launch_shape<XKIND, RKIND, OKIND, false>(a, st);
}

template <int XKIND, int RKIND>
cudaError_t launch_out(const NormArgs& a, int out_kind, bool vec, cudaStream_t st) {
  if (out_kind == MLPMOE_FP32) return launch_vec<XKIND, RKIND, MLPMOE_FP32>(a, vec, st);
  if (out_kind == MLPMOE_BF16) return launch_vec<XKIND, RKIND, MLPMOE_BF16>(a, vec, st);
  return launch_vec<XKIND, RKIND, MLPMOE_E4M3>(a, vec, st);
}

template <int XKIND>
cudaError_t launch_residual(const NormArgs& a, int r_kind, int out_kind, bool vec, cudaStream_t st) {
  if (r_kind == MLPMOE_FP32) return launch_out<XKIND, MLPMOE_FP32>(a, out_kind, vec, st);
  if (r_kind == MLPMOE_BF16) return launch_out<XKIND, MLPMOE_BF16>(a, out_kind, vec, st);
  return launch_out<XKIND, kNone>(a, out_kind, vec, st);
}

inline bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" mlpmoe_status_t mlpmoe_add_rmsnorm(const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride, const void* r,
                                              mlpmoe_dtype_t r_dtype, int64_t r_stride, const float* gain, void* x_out,
                                              int64_t x_out_stride, void* out, mlpmoe_dtype_t out_dtype, int64_t out_stride,
                                              float* scales, int64_t group, int64_t n_tokens, int64_t d_model, float eps, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0) return MLPMOE_ERR_INVALID_ARG;
  if (x_dtype != MLPMOE_FP32 && x_dtype != MLPMOE_BF16) return MLPMOE_ERR_INVALID_ARG;
  if (r && r_dtype != MLPMOE_FP32 && r_dtype != MLPMOE_BF16) return MLPMOE_ERR_INVALID_ARG;
  if (out_dtype != MLPMOE_FP32 && out_dtype != MLPMOE_BF16 && out_dtype != MLPMOE_E4M3) return MLPMOE_ERR_INVALID_ARG;
  if (out_dtype == MLPMOE_E4M3 && group != 0 && group != 32 && group != 64 && group != 128) return MLPMOE_ERR_INVALID_ARG;
  if (d_model > 32768) return MLPMOE_ERR_UNSUPPORTED;
  if (x_stride == 0) x_stride = d_model;
  if (r_stride == 0) r_stride = d_model;
  if (x_out_stride == 0) x_out_stride = d_model;
  if (out_stride == 0) out_stride = d_model;
  if (x_stride < d_model || (r && r_stride < d_model) || (x_out && x_out_stride < d_model) || out_stride < d_model)
    return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens == 0) return MLPMOE_OK;
  if (!x || !out || (out_dtype == MLPMOE_E4M3 && !scales)) return MLPMOE_ERR_INVALID_ARG;
  if (x_out == x && x_out_stride != x_stride && n_tokens > 1) return MLPMOE_ERR_INVALID_ARG;
  const uintptr_t xb = x_dtype == MLPMOE_FP32 ? 4 : 2, rb = r_dtype == MLPMOE_FP32 ? 4 : 2;
  const uintptr_t ob = out_dtype == MLPMOE_FP32 ? 4 : (out_dtype == MLPMOE_BF16 ? 2 : 1);
  if (!on(x, xb) || (r && !on(r, rb)) || !on(gain, 4) || !on(x_out, xb) || !on(out, ob) || (out_dtype == MLPMOE_E4M3 && !on(scales, 4)))
    return MLPMOE_ERR_INVALID_ARG;
  const bool vec = d_model % 8 == 0 && x_stride % 8 == 0 && on(x, 16) && (!r || (r_stride % 8 == 0 && on(r, 16))) && on(gain, 16) &&
                   (!x_out || (x_out_stride % 8 == 0 && on(x_out, 16))) && out_stride % 8 == 0 && on(out, ob == 1 ? 8 : 16);
  NormArgs a;
  a.x = x;
  a.r = r;
  a.gain = gain;
  a.x_out = x_out;
  a.out = out;
  a.scales = scales;
  a.x_stride = x_stride;
  a.r_stride = r ? r_stride : 0;
  a.x_out_stride = x_out_stride;
  a.out_stride = out_stride;
  a.n = n_tokens;
  a.d = static_cast<int>(d_model);
  a.group = group == 0 ? static_cast<int>(d_model) : static_cast<int>(group);
  a.eps = eps;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int r_kind = r ? static_cast<int>(r_dtype) : kNone;
  pdl_overlap_enabled() = true;
  const cudaError_t e = x_dtype == MLPMOE_FP32 ? launch_residual<MLPMOE_FP32>(a, r_kind, out_dtype, vec, st)
                                               : launch_residual<MLPMOE_BF16>(a, r_kind, out_dtype, vec, st);
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}
