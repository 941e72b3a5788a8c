// The kernel of the residual norms (mlpmoe_add_rmsnorm, mlpmoe_add_layernorm): s = x + r, the norm of s, and its output in fp32, bf16 or
// e4m3 with scales, in one pass over memory.
#pragma once
#include <cuda_fp8.h>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kNone = 2;   // no residual, beside MLPMOE_BF16 (0) and MLPMOE_FP32 (1)
constexpr float kE4m3Max = 448.0f;
constexpr float kScaleMin = 1.17549435e-38f;   // 2^-126: keeps 1 / scale finite; a group of zeros gets it too

struct NormArgs {
  const void* x;
  const void* r;
  const float* gain;
  const float* bias;     // LayerNorm only
  void* x_out;
  void* out;
  float* scales;
  int64_t x_stride, r_stride, x_out_stride, out_stride, n;
  int d, group;   // group: columns per scale, d for one per row
  float eps;
};

// One row per T threads (T = 32: eight rows to a block), NCH chunks of eight consecutive columns per thread.
// A group of 32, 64 or 128 columns lies in 4, 8 or 16 neighbouring lanes of one warp, so its maximum is a few shuffles.
template <bool LAYER, int XKIND, int RKIND, int OKIND, bool VEC, int T, int NCH>
__global__ void __launch_bounds__(T == 32 ? 256 : T) add_norm_kernel(const __grid_constant__ NormArgs a) {
  __shared__ float red[32];
  __shared__ float sums[LAYER ? 2 : 1][T / 32][4];
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
  // LayerNorm on rows that take no wide loads: neighbouring columns to neighbouring threads (8-bit scales need them in one thread)
  constexpr bool SPREAD = LAYER && !VEC && OKIND != MLPMOE_E4M3;
  auto load = [&](const void* row, int kind, int i) {
    return SPREAD ? load_columns<false, T>(row, kind, i, tid, d) : load_chunk<VEC>(row, kind, (i * T + tid) * 8, d);
  };
  auto store = [&](void* row, int kind, int i, const float (&v)[8]) {
    if (SPREAD) {
      store_columns<false, T>(row, kind, i, tid, d, v);
    } else if ((i * T + tid) * 8 < d) {
      store8<VEC>(row, kind, (i * T + tid) * 8, d, v);
    }
  };
  auto values = [&](const Chunk& c, int kind, float (&v)[8]) { columns_f32<!SPREAD>(c, kind, v); };
  float s[NCH][8];
  {
    Chunk x[NCH], r[NCH];               // all of the row's loads before the first use
#pragma unroll
    for (int i = 0; i < NCH; ++i) x[i] = load(xrow, XKIND, i);
    if (RKIND != kNone) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) r[i] = load(rrow, RKIND, i);
    }
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      values(x[i], XKIND, s[i]);
      if (RKIND != kNone) {
        float v[8];
        values(r[i], RKIND, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[i][j] += v[j];
      }
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) ss += LAYER ? s[i][j] : s[i][j] * s[i][j];
  if (a.x_out != nullptr) {
    char* xo = static_cast<char*>(a.x_out) + t * a.x_out_stride * kXBytes;
#pragma unroll
    for (int i = 0; i < NCH; ++i) store(xo, XKIND, i, s[i]);
  }
  if (LAYER) {                               // the mean first, then the squares of what is left: no cancellation
    int turn = 0;
    float sum[1] = {ss};
    row_sums<T, 1>(sum, sums, turn);
    const float mean = sum[0] / static_cast<float>(d);
    ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s[i][j] = (SPREAD ? column<false, T>(i, tid, j) : (i * T + tid) * 8 + (VEC ? 0 : j)) < d ? s[i][j] - mean : 0.0f;
        ss += s[i][j] * s[i][j];
      }
    sum[0] = ss;
    row_sums<T, 1>(sum, sums, turn);
    ss = sum[0];
  } else {
    ss = row_reduce<T, false>(ss, red);
  }
  const float inv = 1.0f / sqrtf(ss / static_cast<float>(d) + a.eps);
  float row_max = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    float g[8];
    if (a.gain != nullptr) {
      to_f32(load(a.gain, MLPMOE_FP32, i), MLPMOE_FP32, g);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    }
    float c[8];
    if (LAYER && a.bias != nullptr) {
      to_f32(load(a.bias, MLPMOE_FP32, i), MLPMOE_FP32, c);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      s[i][j] = s[i][j] * inv * g[j];
      if (LAYER) s[i][j] += c[j];
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
  for (int i = 0; i < NCH; ++i) store(orow, OKIND, i, s[i]);
}

// A row to a block whose threads take eight columns each: all loads of a row are in flight at once and none is idle long.  A warp
// to a row (no block barrier) where a row is 512 columns at most and there are many: 65536 x 512 60.6 us against 69.9,
// while at 1200 rows both take 3.1.  Rows of more than 8192 columns spill: RMSNorm of fp32 + fp32 that is not aligned 48 to 132 bytes a thread, LayerNorm of
// aligned rows 4 to 80 (e4m3 or with an fp32 input) and of fp32 + fp32 to e4m3 that is not aligned 84.  Two chunks to a thread for 8-bit output of longer rows, whose scales are half the
// work: 16384 x 4096 111 us against 129 with one (bf16 output: 121 against 117, so it keeps one).
// LayerNorm, with its second sum, takes two for every output: 16384 x 4096 to bf16 121 us against 139 (four: 129).
template <bool LAYER, int XKIND, int RKIND, int OKIND, bool VEC>
cudaError_t launch_shape(const NormArgs& a, cudaStream_t st) {
  const unsigned n = static_cast<unsigned>(a.n);
  if (a.d <= 512 && a.n > 4096) return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 32, 2>, dim3((n + 7) / 8), dim3(256), 0, st, a);
  if (a.d <= 1024) return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 128, 1>, dim3(n), dim3(128), 0, st, a);
  if (a.d <= 2048) return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 256, 1>, dim3(n), dim3(256), 0, st, a);
  if (a.d <= 4096 && (LAYER || OKIND == MLPMOE_E4M3) && a.n > 1024)
    return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 256, 2>, dim3(n), dim3(256), 0, st, a);
  if (a.d <= 4096) return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 512, 1>, dim3(n), dim3(512), 0, st, a);
  if (a.d <= 8192) return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 512, 2>, dim3(n), dim3(512), 0, st, a);
  return launch_pdl(add_norm_kernel<LAYER, XKIND, RKIND, OKIND, VEC, 1024, 4>, dim3(n), dim3(1024), 0, st, a);
}

template <bool LAYER, int XKIND, int RKIND, int OKIND>
cudaError_t launch_vec(const NormArgs& a, bool vec, cudaStream_t st) {
  return vec ? launch_shape<LAYER, XKIND, RKIND, OKIND, true>(a, st) : launch_shape<LAYER, XKIND, RKIND, OKIND, false>(a, st);
}

template <bool LAYER, int XKIND, int RKIND>
cudaError_t launch_out(const NormArgs& a, int out_kind, bool vec, cudaStream_t st) {
  if (out_kind == MLPMOE_FP32) return launch_vec<LAYER, XKIND, RKIND, MLPMOE_FP32>(a, vec, st);
  if (out_kind == MLPMOE_BF16) return launch_vec<LAYER, XKIND, RKIND, MLPMOE_BF16>(a, vec, st);
  return launch_vec<LAYER, XKIND, RKIND, MLPMOE_E4M3>(a, vec, st);
}

template <bool LAYER, int XKIND>
cudaError_t launch_residual(const NormArgs& a, int r_kind, int out_kind, bool vec, cudaStream_t st) {
  if (r_kind == MLPMOE_FP32) return launch_out<LAYER, XKIND, MLPMOE_FP32>(a, out_kind, vec, st);
  if (r_kind == MLPMOE_BF16) return launch_out<LAYER, XKIND, MLPMOE_BF16>(a, out_kind, vec, st);
  return launch_out<LAYER, XKIND, kNone>(a, out_kind, vec, st);
}

// The checks and the launch of both entry points (bias: LayerNorm only, NULL otherwise).
template <bool LAYER>
mlpmoe_status_t add_norm(const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride, const void* r, mlpmoe_dtype_t r_dtype, int64_t r_stride,
                         const float* gain, const float* bias, void* x_out, int64_t x_out_stride, void* out, mlpmoe_dtype_t out_dtype,
                         int64_t out_stride, float* scales, int64_t group, int64_t n_tokens, int64_t d_model, float eps, void* stream) {
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
  if (!on(x, xb) || (r && !on(r, rb)) || !on(gain, 4) || !on(bias, 4) || !on(x_out, xb) || !on(out, ob) || (out_dtype == MLPMOE_E4M3 && !on(scales, 4)))
    return MLPMOE_ERR_INVALID_ARG;
  const bool vec = d_model % 8 == 0 && x_stride % 8 == 0 && on(x, 16) && (!r || (r_stride % 8 == 0 && on(r, 16))) && on(gain, 16) && on(bias, 16) &&
                   (!x_out || (x_out_stride % 8 == 0 && on(x_out, 16))) && out_stride % 8 == 0 && on(out, ob == 1 ? 8 : 16);
  NormArgs a;
  a.x = x;
  a.r = r;
  a.gain = gain;
  a.bias = bias;
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
  const cudaError_t e = x_dtype == MLPMOE_FP32 ? launch_residual<LAYER, MLPMOE_FP32>(a, r_kind, out_dtype, vec, st)
                                               : launch_residual<LAYER, MLPMOE_BF16>(a, r_kind, out_dtype, vec, st);
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // namespace
}  // namespace mlpmoe
