// Weights to 4-bit codes with group scales, and back (mlpmoe_w4_quantize, mlpmoe_w4_dequantize).  Both are bound by
// the dense matrix they read or write.  A block takes a tile of 32 rows x 256 columns, a warp four neighbouring rows of
// it with eight neighbouring columns per lane and row, all loads under way before the first use; a group of 32, 64 or
// 128 columns is 4, 8 or 16 lanes.
// 14336 x 4096 bf16, group 128 with zeros: codes 45 us of 147 MB (23 for a copy; 76 % of the issue slots are taken: a range, a
// product, a sum, a clamp and a place for each value), back 24 us, where the copy takes 23.
#include "../../include/mlpmoe.h"
#include "internal.h"
#include "w4.h"

namespace mlpmoe {
namespace {

constexpr int kRows = 32, kCols = 256, kThreads = 256, kWarpRows = 4;
constexpr int64_t kMaxDim = int64_t(1) << 20;      // keeps the grid within its limits

struct QuantArgs {
  const void* w_in;
  void* w_out;
  uint8_t* q;
  __nv_bfloat16* scale;
  uint8_t* zero;
  int64_t stride, rows, cols, rows16, pitch;
  int log_group;
};

template <typename T>
__device__ __forceinline__ void load_eight(const T* p, float (&v)[8]) {
  if (sizeof(T) == 4) {
    const float4 lo = reinterpret_cast<const float4*>(p)[0], hi = reinterpret_cast<const float4*>(p)[1];
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  } else {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xFFFF0000u), v[2] = __uint_as_float(w.y << 16),
    v[3] = __uint_as_float(w.y & 0xFFFF0000u), v[4] = __uint_as_float(w.z << 16), v[5] = __uint_as_float(w.z & 0xFFFF0000u),
    v[6] = __uint_as_float(w.w << 16), v[7] = __uint_as_float(w.w & 0xFFFF0000u);
  }
}
template <typename T>
__device__ __forceinline__ void store_eight(T* p, const float (&v)[8]) {
  if (sizeof(T) == 4) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// The codes of eight values, rint(v / div) + z between 0 and 15, four bits each.  The quotient is v * (1 / div), off by less
// than 2^-20; only what lies within 2^-17 of a half needs more, so that the codes are those of the correctly rounded
// quotient.  An fp32 value is divided in full.  A bf16 value is there exactly half way between two whole numbers, and commonly
// (8 bits over 8 bits): with a and b the significands of v and div, both below 256, and v at least div / 2, the distance
// from a half is a multiple of 1 / (4 b).  So the sum with 1.5 * 2^12 first takes the quotient to multiples of 2^-11, which
// makes such a half exact and moves nothing else onto or over one (with the division these values cost a third of the time).
// The sum with 1.5 * 2^23 rounds to even and has the whole number in its low bits.  No code falls below 0: the scale is off by
// 2^-9 at most, z = rint(-lo / div), and rint(lo / div) = -z.
template <bool BF16>
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float div, float inv, int z) {
  constexpr float kMagic = 12582912.0f, kFine = 6144.0f;
  float t[8];
  if constexpr (BF16) {
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = fmaf(v[j], inv, kFine) + (kMagic - kFine);
  } else {
    float off[8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      t[j] = fmaf(v[j], inv, kMagic);
      off[j] = fabsf(fmaf(v[j], inv, kMagic - t[j]));
      most = fmaxf(most, off[j]);
    }
    if (most > 0.49999f) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (off[j] > 0.49999f) t[j] = v[j] / div + kMagic;
    }
  }
  uint32_t code = 0;
  const int shift = z - 0x4B400000;
#pragma unroll
  for (int j = 0; j < 8; ++j) code += static_cast<uint32_t>(min(__float_as_int(t[j]) + shift, 15)) << (4 * j);
  return code;
}

// PAPER: the source is [cols x rows]; the tile goes through shared memory so that both sides are read along memory.
// VEC: cols % 8 == 0 and rows on 16 bytes.
template <typename T, bool PAPER, bool VEC>
__global__ void __launch_bounds__(kThreads, 4) w4_quantize_kernel(const __grid_constant__ QuantArgs a) {
  __shared__ float tile[PAPER ? kRows * (kCols + 1) : 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kRows, c0 = static_cast<int64_t>(blockIdx.x) * kCols;
  const T* w = static_cast<const T*>(a.w_in);
  if (PAPER) {
    for (int i = threadIdx.x; i < kRows * kCols; i += kThreads) {
      const int64_t r = r0 + i % kRows, c = c0 + i / kRows;
      tile[(i % kRows) * (kCols + 1) + i / kRows] = r < a.rows && c < a.cols ? static_cast<float>(w[c * a.stride + r]) : 0.0f;
    }
    __syncthreads();
  }
  const int lanes = 1 << (a.log_group - 3);
  const int64_t col = c0 + 8 * lane, row0 = r0 + warp * kWarpRows;
  const int rows_here = static_cast<int>(min(static_cast<int64_t>(kWarpRows), a.rows - row0));
  const int cols_here = static_cast<int>(min(static_cast<int64_t>(8), a.cols - col));       // of this lane; 0 or less: none
  float v[kWarpRows][8];
  const T* src = w + row0 * a.stride + col;
#pragma unroll
  for (int i = 0; i < kWarpRows; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    if (PAPER) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = tile[(warp * kWarpRows + i) * (kCols + 1) + 8 * lane + j];
    } else if (VEC) {
      if (i < rows_here && cols_here > 0) load_eight(src, v[i]);
    } else if (i < rows_here) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < cols_here) v[i][j] = static_cast<float>(src[j]);
    }
    src += a.stride;
  }
  float lo = 0.0f, hi = 0.0f;           // of row lane % 4 in this lane's group
  {
    float l[kWarpRows], h[kWarpRows];   // the group's range in each row; l negated
    if constexpr (sizeof(T) == 2) {     // two bf16 at a time: a comparison keeps either of its operands as it is
      uint32_t range[kWarpRows];        // (l, h)
#pragma unroll
      for (int i = 0; i < kWarpRows; ++i) {
        __nv_bfloat162 p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) p[j] = __floats2bfloat162_rn(v[i][2 * j], v[i][2 * j + 1]);
        const __nv_bfloat162 most = __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])), least = __hmin2(__hmin2(p[0], p[1]), __hmin2(p[2], p[3]));
        const __nv_bfloat162 both = __halves2bfloat162(__hneg(__hmin(least.x, least.y)), __hmax(most.x, most.y));
        const __nv_bfloat162 from_zero = __hmax2(both, __floats2bfloat162_rn(0.0f, 0.0f));
        range[i] = *reinterpret_cast<const uint32_t*>(&from_zero);
      }
      for (int o = 1; o < lanes; o *= 2) {
#pragma unroll
        for (int i = 0; i < kWarpRows; ++i) {
          const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, range[i], o);
          const __nv_bfloat162 wide = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&range[i]), *reinterpret_cast<const __nv_bfloat162*>(&other));
          range[i] = *reinterpret_cast<const uint32_t*>(&wide);
        }
      }
#pragma unroll
      for (int i = 0; i < kWarpRows; ++i) l[i] = __uint_as_float(range[i] << 16), h[i] = __uint_as_float(range[i] & 0xFFFF0000u);
    } else {
#pragma unroll
      for (int i = 0; i < kWarpRows; ++i) {
        l[i] = h[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) l[i] = fmaxf(l[i], -v[i][j]), h[i] = fmaxf(h[i], v[i][j]);
      }
      for (int o = 1; o < lanes; o *= 2) {
#pragma unroll
        for (int i = 0; i < kWarpRows; ++i) {
          h[i] = fmaxf(h[i], __shfl_xor_sync(0xFFFFFFFFu, h[i], o));
          l[i] = fmaxf(l[i], __shfl_xor_sync(0xFFFFFFFFu, l[i], o));
        }
      }
    }
    if (a.zero == nullptr) {
#pragma unroll
      for (int i = 0; i < kWarpRows; ++i) h[i] = fmaxf(h[i], l[i]);
    }
#pragma unroll
    for (int i = 0; i < kWarpRows; ++i)
      if (lane % kWarpRows == i) lo = -l[i], hi = h[i];
  }
  // The divisions of a group once, in the lane of its row: the scale is rounded to bf16 (2 bytes per group) before the codes
  // are made, so the codes fit the scale that is stored.
  float s_mine = __bfloat162float(__float2bfloat16_rn(a.zero != nullptr ? (hi - lo) / 15.0f : hi / 7.0f));
  if (s_mine < 1.17549435e-38f) s_mine = 0.0f;             // below 2^-126 its reciprocal may be infinite
  const float div_mine = s_mine > 0.0f ? s_mine : 1.0f, inv_mine = 1.0f / div_mine;
  const float z_mine = a.zero != nullptr ? fminf(rintf(-lo / div_mine), 15.0f) : 8.0f;
  const int my_row = lane % kWarpRows;
  if (lane % lanes < kWarpRows && col - 8 * my_row < a.cols && my_row < rows_here) {     // the group's first column is in the matrix
    const int64_t at = (col >> a.log_group) * a.rows16 + row0 + my_row;
    a.scale[at] = __float2bfloat16_rn(s_mine);
    if (a.zero != nullptr) a.zero[at] = static_cast<uint8_t>(z_mine);
  }
  const bool store = col / 2 < a.pitch;
  const uint32_t keep = cols_here >= 8 ? 0xFFFFFFFFu : (cols_here <= 0 ? 0u : (1u << (4 * cols_here)) - 1u);   // columns past the last are coded 0
  uint8_t* q = a.q + row0 * a.pitch + col / 2;
#pragma unroll
  for (int i = 0; i < kWarpRows; ++i) {
    const int from = (lane & ~(kWarpRows - 1)) + i;
    const float div = __shfl_sync(0xFFFFFFFFu, div_mine, from), inv = __shfl_sync(0xFFFFFFFFu, inv_mine, from);
    const float z = __shfl_sync(0xFFFFFFFFu, z_mine, from);
    const uint32_t code = codes_of<sizeof(T) == 2>(v[i], div, inv, static_cast<int>(z));
    if (i < rows_here && store) *reinterpret_cast<uint32_t*>(q) = code & keep;
    q += a.pitch;
  }
}

template <typename T, bool PAPER, bool VEC>
__global__ void __launch_bounds__(kThreads) w4_dequantize_kernel(const __grid_constant__ QuantArgs a) {
  __shared__ float tile[PAPER ? kRows * (kCols + 1) : 1];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t r0 = static_cast<int64_t>(blockIdx.y) * kRows, c0 = static_cast<int64_t>(blockIdx.x) * kCols;
  T* w = static_cast<T*>(a.w_out);
  const int64_t col = c0 + 8 * lane, row0 = r0 + warp * kWarpRows;
  const int rows_here = static_cast<int>(min(static_cast<int64_t>(kWarpRows), a.rows - row0));
  const int cols_here = static_cast<int>(min(static_cast<int64_t>(8), a.cols - col));       // of this lane; 0 or less: none
  const bool in = rows_here > 0 && cols_here > 0;
  uint32_t code[kWarpRows];
  const uint8_t* q = a.q + row0 * a.pitch + col / 2;
#pragma unroll
  for (int i = 0; i < kWarpRows; ++i) {
    code[i] = in && i < rows_here ? *reinterpret_cast<const uint32_t*>(q) : 0u;
    q += a.pitch;
  }
  // four rows' scales and zeros at once: rows16 covers a started four
  const int64_t at = (col >> a.log_group) * a.rows16 + row0;
  const uint2 sw = in ? *reinterpret_cast<const uint2*>(a.scale + at) : make_uint2(0u, 0u);
  const uint32_t zw = in && a.zero != nullptr ? *reinterpret_cast<const uint32_t*>(a.zero + at) : 0x08080808u;
  const float s[kWarpRows] = {__uint_as_float(sw.x << 16), __uint_as_float(sw.x & 0xFFFF0000u), __uint_as_float(sw.y << 16),
                              __uint_as_float(sw.y & 0xFFFF0000u)};
  T* dst = w + row0 * a.stride + col;
#pragma unroll
  for (int i = 0; i < kWarpRows; ++i) {
    float v[8];
    // 2^23 + code, less 2^23 + zero: exact
    const float z = __uint_as_float(((zw >> (8 * i)) & 255u) | 0x4B000000u);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (__uint_as_float(((code[i] >> (4 * j)) & 15u) | 0x4B000000u) - z) * s[i];
    if (PAPER) {
#pragma unroll
      for (int j = 0; j < 8; ++j) tile[(warp * kWarpRows + i) * (kCols + 1) + 8 * lane + j] = v[j];
    } else if (VEC) {
      if (in && i < rows_here) store_eight(dst, v);
    } else if (i < rows_here) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < cols_here) dst[j] = static_cast<T>(v[j]);
    }
    dst += a.stride;
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
  a.log_group = group == 32 ? 5 : (group == 64 ? 6 : 7);
  const bool vec = cols % 8 == 0 && stride % 8 == 0 && on(W, 16);
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
