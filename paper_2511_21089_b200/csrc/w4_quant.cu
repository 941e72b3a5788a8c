// Weights to 4-bit codes with group scales, and back (mlpmoe_w4_quantize, mlpmoe_w4_dequantize).  Both are bound by
// the dense matrix they read or write; a block takes a tile of 32 rows x 128 columns, a warp one row of it at a time
// with four neighbouring columns per lane, so a group of 32, 64 or 128 columns is 8, 16 or 32 lanes.
#include "../../include/mlpmoe.h"
#include "internal.h"
#include "w4.h"

namespace mlpmoe {
namespace {

constexpr int kRows = 32, kCols = 128, kThreads = 256;
constexpr int64_t kMaxDim = int64_t(1) << 20;      // keeps the grid within its limits

struct QuantArgs {
  const void* w_in;
  void* w_out;
  uint8_t* q;
  __nv_bfloat16* scale;
  uint8_t* zero;
  int64_t stride, rows, cols, rows16, pitch;
  int group;
};

template <typename T>
__device__ __forceinline__ float to_f32(T v) { return static_cast<float>(v); }

// PAPER: the source is [cols x rows]; the tile goes through shared memory so that both sides are read along memory.
template <typename T, bool PAPER, bool VEC>
__global__ void __launch_bounds__(kThreads) w4_quantize_kernel(const __grid_constant__ QuantArgs a) {
  __shared__ float tile[PAPER ? kRows * (kCols + 1) : 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kRows, c0 = static_cast<int64_t>(blockIdx.x) * kCols;
  const T* w = static_cast<const T*>(a.w_in);
  if (PAPER) {
    for (int i = threadIdx.x; i < kRows * kCols; i += kThreads) {
      const int64_t r = r0 + i % kRows, c = c0 + i / kRows;
      tile[(i % kRows) * (kCols + 1) + i / kRows] = r < a.rows && c < a.cols ? to_f32(w[c * a.stride + r]) : 0.0f;
    }
    __syncthreads();
  }
  const int lanes = a.group / 4;
  const int64_t col = c0 + 4 * lane;
  for (int i = warp; i < kRows; i += kThreads / 32) {
    const int64_t r = r0 + i;
    if (r >= a.rows) break;
    float v[4];
    if (PAPER) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = tile[i * (kCols + 1) + 4 * lane + j];
    } else if (VEC) {                       // cols % 4 == 0, rows on 16 (fp32) or 8 (bf16) bytes
      v[0] = v[1] = v[2] = v[3] = 0.0f;
      if (col < a.cols) {
        if (sizeof(T) == 4) {
          const float4 u = *reinterpret_cast<const float4*>(w + r * a.stride + col);
          v[0] = u.x, v[1] = u.y, v[2] = u.z, v[3] = u.w;
        } else {
          const uint2 u = *reinterpret_cast<const uint2*>(w + r * a.stride + col);
          v[0] = __uint_as_float(u.x << 16), v[1] = __uint_as_float(u.x & 0xFFFF0000u);
          v[2] = __uint_as_float(u.y << 16), v[3] = __uint_as_float(u.y & 0xFFFF0000u);
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = col + j < a.cols ? to_f32(w[r * a.stride + col + j]) : 0.0f;
    }
    float lo = fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), hi = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3]));
    for (int o = 1; o < lanes; o *= 2) {
      lo = fminf(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, o));
      hi = fmaxf(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, o));
    }
    lo = fminf(lo, 0.0f);
    hi = fmaxf(hi, 0.0f);
    // the scale is rounded to bf16 (2 bytes per group) before the codes are made, so the codes fit the scale that is stored
    const __nv_bfloat16 sb = __float2bfloat16_rn(a.zero != nullptr ? (hi - lo) / 15.0f : fmaxf(-lo, hi) / 7.0f);
    const float s = __bfloat162float(sb);
    const float div = s > 0.0f ? s : 1.0f;
    const float z = a.zero != nullptr ? fminf(fmaxf(rintf(-lo / div), 0.0f), 15.0f) : 8.0f;
    uint32_t code = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (col + j < a.cols) code |= static_cast<uint32_t>(fminf(fmaxf(rintf(v[j] / div) + z, 0.0f), 15.0f)) << (4 * j);
    if (col / 2 < a.pitch) *reinterpret_cast<uint16_t*>(a.q + r * a.pitch + col / 2) = static_cast<uint16_t>(code);
    if (lane % lanes == 0 && col < a.cols) {
      const int64_t at = col / a.group * a.rows16 + r;
      a.scale[at] = sb;
      if (a.zero != nullptr) a.zero[at] = static_cast<uint8_t>(z);
    }
  }
}

template <typename T, bool PAPER, bool VEC>
__global__ void __launch_bounds__(kThreads) w4_dequantize_kernel(const __grid_constant__ QuantArgs a) {
  __shared__ float tile[PAPER ? kRows * (kCols + 1) : 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kRows, c0 = static_cast<int64_t>(blockIdx.x) * kCols;
  T* w = static_cast<T*>(a.w_out);
  const int64_t col = c0 + 4 * lane;
  for (int i = warp; i < kRows; i += kThreads / 32) {
    const int64_t r = r0 + i;
    if (r >= a.rows) break;
    float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < a.cols) {
      const uint32_t code = *reinterpret_cast<const uint16_t*>(a.q + r * a.pitch + col / 2);
      const int64_t at = col / a.group * a.rows16 + r;
      const float s = __bfloat162float(a.scale[at]);
      const int z = a.zero != nullptr ? a.zero[at] : 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = static_cast<float>(static_cast<int>((code >> (4 * j)) & 15u) - z) * s;
    }
    if (PAPER) {
#pragma unroll
      for (int j = 0; j < 4; ++j) tile[i * (kCols + 1) + 4 * lane + j] = v[j];
    } else if (VEC) {
      if (col < a.cols) {
        if (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(w + r * a.stride + col) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          const __nv_bfloat162 x = __floats2bfloat162_rn(v[0], v[1]), y = __floats2bfloat162_rn(v[2], v[3]);
          *reinterpret_cast<uint2*>(w + r * a.stride + col) =
              make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (col + j < a.cols) w[r * a.stride + col + j] = static_cast<T>(v[j]);
    }
  }
  if (PAPER) {
    __syncthreads();
    for (int i = threadIdx.x; i < kRows * kCols; i += kThreads) {
      const int64_t r = r0 + i % kRows, c = c0 + i / kRows;
      if (r < a.rows && c < a.cols) w[c * a.stride + r] = static_cast<T>(tile[(i % kRows) * (kCols + 1) + i / kRows]);
    }
  }
}

template <typename T>
cudaError_t launch(bool back, bool paper, bool vec, const QuantArgs& a, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((a.cols + kCols - 1) / kCols), static_cast<unsigned>((a.rows + kRows - 1) / kRows));
  if (back) {
    if (paper) w4_dequantize_kernel<T, true, false><<<grid, kThreads, 0, st>>>(a);
    else if (vec) w4_dequantize_kernel<T, false, true><<<grid, kThreads, 0, st>>>(a);
    else w4_dequantize_kernel<T, false, false><<<grid, kThreads, 0, st>>>(a);
  } else {
    if (paper) w4_quantize_kernel<T, true, false><<<grid, kThreads, 0, st>>>(a);
    else if (vec) w4_quantize_kernel<T, false, true><<<grid, kThreads, 0, st>>>(a);
    else w4_quantize_kernel<T, false, false><<<grid, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
}

inline bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

mlpmoe_status_t run(bool back, const void* W, mlpmoe_dtype_t dtype, mlpmoe_layout_t layout, int64_t stride, int64_t rows, int64_t cols,
                    int32_t group, const uint8_t* q, const void* scale, const uint8_t* zero, void* stream) {
  if (rows < 0 || cols < 0 || (dtype != MLPMOE_FP32 && dtype != MLPMOE_BF16)) return MLPMOE_ERR_INVALID_ARG;
  if (layout != MLPMOE_LAYOUT_LINEAR && layout != MLPMOE_LAYOUT_PAPER) return MLPMOE_ERR_INVALID_ARG;
  if (group != 32 && group != 64 && group != 128) return MLPMOE_ERR_UNSUPPORTED;
  if (rows > kMaxDim || cols > kMaxDim) return MLPMOE_ERR_UNSUPPORTED;
  const int64_t inner = layout == MLPMOE_LAYOUT_LINEAR ? cols : rows;
  if (stride == 0) stride = inner;
  if (stride < inner) return MLPMOE_ERR_INVALID_ARG;
  if (rows == 0 || cols == 0) return MLPMOE_OK;
  if (!W || !q || !scale || !on(q, 16) || !on(scale, 16) || !on(zero, 16)) return MLPMOE_ERR_INVALID_ARG;
  const uintptr_t elem = dtype == MLPMOE_FP32 ? 4 : 2;
  if (!on(W, elem)) return MLPMOE_ERR_INVALID_ARG;
  QuantArgs a;
  a.w_in = W;
  a.w_out = const_cast<void*>(W);
  a.q = const_cast<uint8_t*>(q);
  a.scale = static_cast<__nv_bfloat16*>(const_cast<void*>(scale));
  a.zero = const_cast<uint8_t*>(zero);
  a.stride = stride;
  a.rows = rows;
  a.cols = cols;
  a.rows16 = w4_rows16(rows);
  a.pitch = w4_pitch(cols);
  a.group = group;
  const bool vec = cols % 4 == 0 && stride % 4 == 0 && on(W, 4 * elem);
  const bool paper = layout == MLPMOE_LAYOUT_PAPER;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == MLPMOE_FP32 ? launch<float>(back, paper, vec, a, st) : launch<__nv_bfloat16>(back, paper, vec, a, st);
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // namespace
}  // namespace mlpmoe

extern "C" {

mlpmoe_status_t mlpmoe_w4_quantize(const void* W, mlpmoe_dtype_t dtype, mlpmoe_layout_t layout, int64_t stride, int64_t rows,
                                   int64_t cols, int32_t group, uint8_t* q, void* scale, uint8_t* zero, void* stream) {
  return mlpmoe::run(false, W, dtype, layout, stride, rows, cols, group, q, scale, zero, stream);
}

mlpmoe_status_t mlpmoe_w4_dequantize(const uint8_t* q, const void* scale, const uint8_t* zero, int64_t rows, int64_t cols, int32_t group,
                                     void* W, mlpmoe_dtype_t dtype, mlpmoe_layout_t layout, int64_t stride, void* stream) {
  return mlpmoe::run(true, W, dtype, layout, stride, rows, cols, group, q, scale, zero, stream);
}

}  // extern "C"
