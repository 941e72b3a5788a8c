// Gradient of the residual norms (mlpmoe_norm_backward), with the sums over tokens for gain and bias:
//     z = s - mean(s) (LayerNorm) or s (RMSNorm);  inv = 1 / sqrt(mean(z^2) + eps);  h = gain * dv;
//     dx = ds + inv * (h - mean(h) - z * inv^2 * mean(h z))   (mean(h): LayerNorm only);
//     dgain = sum_t dv * z * inv;   dbias = sum_t dv.
// HBM-bound: s, dv and ds are read once, a block keeps its columns' sums over all of its rows in registers, the next row's loads are
// under way while a row is reduced, and the blocks' sums are joined by a second launch in a fixed order.
#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kNone = 2;
constexpr int kSms = 148;
constexpr int64_t kMaxD = 32768;
constexpr int64_t kOnePassD = 8192;      // longer rows do not leave room for their columns' sums in registers
constexpr int kSplitRows = 64;           // slices of the rows there, for the sums over tokens

struct NormGradArgs {
  const void* s;
  const void* dv;
  const void* ds;
  const float* gain;
  void* dx;
  float* partial;       // [blocks][2][d]
  float* stats;         // [n][2]: mean, inv (long rows)
  float* dgain;
  float* dbias;
  int64_t s_stride, dv_stride, ds_stride, dx_stride, n;
  int s_kind, dv_kind, ds_kind, dx_kind, d;
  float eps;
};

// Sums of V values over the T threads of a row, the same bits in all of them.  `red`: two sets, used in turn, so that one barrier will do.
template <int T, int V>
__device__ __forceinline__ void row_sums(float (&v)[V], float (*red)[T / 32][4], int& turn) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
  if (T > 32) {
    float(*r)[4] = red[turn];
    turn ^= 1;
    if (threadIdx.x % 32 == 0)
#pragma unroll
      for (int k = 0; k < V; ++k) r[threadIdx.x / 32][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = r[0][k];
#pragma unroll
    for (int i = 1; i < T / 32; ++i)
#pragma unroll
      for (int k = 0; k < V; ++k) v[k] += r[i][k];
  }
}

// T threads to a row (T = 32: eight rows to a block), NCH chunks of eight columns a thread.  SUMS: the columns' sums are kept here;
// else the row's mean and inv go to memory for a kernel of their own.
template <bool LAYER, bool VEC, int T, int NCH, bool SUMS>
__global__ void __launch_bounds__(T == 32 ? 256 : T) norm_backward_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr int R = T == 32 ? 8 : 1;
  __shared__ float red[2][T / 32][4];
  __shared__ float join[T == 32 ? 8 : 1][T == 32 ? 256 : 1];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int tid = T == 32 ? threadIdx.x % 32 : threadIdx.x, d = a.d;
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t t = static_cast<int64_t>(blockIdx.x) * R + (T == 32 ? threadIdx.x / 32 : 0);
  float gain[NCH][8], sum_g[SUMS ? NCH : 1][8], sum_b[SUMS && LAYER ? NCH : 1][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    if (a.gain != nullptr) {
      to_f32(load_chunk<VEC>(a.gain, MLPMOE_FP32, (i * T + tid) * 8, d), MLPMOE_FP32, gain[i]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) gain[i][e] = 1.0f;
    }
    if (SUMS)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum_g[i][e] = 0.0f;
        if (LAYER) sum_b[i][e] = 0.0f;
      }
  }
  Chunk cs[NCH], cv[NCH], cr[NCH];
  auto fetch = [&](int64_t row) {
    const char* ps = static_cast<const char*>(a.s) + row * a.s_stride * bytes_of(a.s_kind);
    const char* pv = static_cast<const char*>(a.dv) + row * a.dv_stride * bytes_of(a.dv_kind);
    const char* pr = static_cast<const char*>(a.ds) + row * a.ds_stride * bytes_of(a.ds_kind);
#pragma unroll
    for (int i = 0; i < NCH; ++i) cs[i] = load_chunk<VEC>(ps, a.s_kind, (i * T + tid) * 8, d);
#pragma unroll
    for (int i = 0; i < NCH; ++i) cv[i] = load_chunk<VEC>(pv, a.dv_kind, (i * T + tid) * 8, d);
    if (a.ds_kind != kNone) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) cr[i] = load_chunk<VEC>(pr, a.ds_kind, (i * T + tid) * 8, d);
    }
  };
  if (t < a.n) fetch(t);
  int turn = 0;
  const float inv_d = 1.0f / static_cast<float>(d);
  for (; t < a.n; t += step) {
    float z[NCH][8], v[NCH][8], r[NCH][8];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      to_f32(cs[i], a.s_kind, z[i]);
      to_f32(cv[i], a.dv_kind, v[i]);
      if (a.ds_kind != kNone) {
        to_f32(cr[i], a.ds_kind, r[i]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[i][e] = 0.0f;
      }
    }
    if (SUMS && t + step < a.n) fetch(t + step);
    float mean = 0.0f, mean_h = 0.0f, ss, hz;
    if (LAYER) {
      float sum[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[0] += z[i][e];
      row_sums<T, 1>(sum, red, turn);
      mean = sum[0] * inv_d;
      float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int col = (i * T + tid) * 8 + (VEC ? 0 : e);
          z[i][e] = col < d ? z[i][e] - mean : 0.0f;
          const float h = gain[i][e] * v[i][e];
          q[0] += z[i][e] * z[i][e];
          q[1] += h * z[i][e];
          q[2] += h;
        }
      row_sums<T, 3>(q, red, turn);
      ss = q[0];
      hz = q[1];
      mean_h = q[2] * inv_d;
    } else {
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q[0] += z[i][e] * z[i][e];
          q[1] += gain[i][e] * v[i][e] * z[i][e];
        }
      row_sums<T, 2>(q, red, turn);
      ss = q[0];
      hz = q[1];
    }
    const float inv = 1.0f / sqrtf(ss * inv_d + a.eps);
    const float along = hz * inv * inv * inv_d;
    if (!SUMS && tid == 0 && a.stats != nullptr) {
      a.stats[2 * t] = mean;
      a.stats[2 * t + 1] = inv;
    }
    char* px = static_cast<char*>(a.dx) + t * a.dx_stride * bytes_of(a.dx_kind);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (SUMS) {
          sum_g[i][e] += v[i][e] * (z[i][e] * inv);
          if (LAYER) sum_b[i][e] += v[i][e];
        }
        r[i][e] += inv * (gain[i][e] * v[i][e] - mean_h - z[i][e] * along);
      }
      const int col = (i * T + tid) * 8;
      if (col < d) store8<VEC>(px, a.dx_kind, col, d, r[i]);
    }
  }
  if (!SUMS || (a.dgain == nullptr && a.dbias == nullptr)) return;
  // the block's sums: to the result where it is the only block
  float* out_g = gridDim.x == 1 ? a.dgain : a.partial + static_cast<int64_t>(blockIdx.x) * 2 * d;
  float* out_b = gridDim.x == 1 ? a.dbias : a.partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * d;
  if (T == 32) {
#pragma unroll
    for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) join[threadIdx.x / 32 % (T == 32 ? 8 : 1)][(tid * 8 + e) % (T == 32 ? 256 : 1)] = which == 0 ? sum_g[0][e] : sum_b[0][e];
      __syncthreads();
      float* out = which == 0 ? out_g : out_b;
      const int col = threadIdx.x;
      if (col < d && out != nullptr) {
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < (T == 32 ? 8 : 1); ++w) sum += join[w][col % (T == 32 ? 256 : 1)];
        out[col] = sum;
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < (SUMS ? NCH : 1); ++i) {
    const int col = (i * T + tid) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (col + e >= d) continue;
      if (out_g != nullptr) out_g[col + e] = sum_g[i][e];
      if (LAYER && out_b != nullptr) out_b[col + e] = sum_b[LAYER ? i : 0][e];
    }
  }
}

// The sums over tokens of long rows, from the rows' mean and inv: a block to 256 columns and a slice of the rows.
__global__ void __launch_bounds__(256) norm_column_sums_kernel(const __grid_constant__ NormGradArgs a, int layer) {
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= a.d) return;
  float sum_g = 0.0f, sum_b = 0.0f;
#pragma unroll 4
  for (int64_t t = blockIdx.y; t < a.n; t += gridDim.y) {
    const int64_t is = t * a.s_stride + col, iv = t * a.dv_stride + col;
    const float s = a.s_kind == MLPMOE_FP32 ? static_cast<const float*>(a.s)[is] : __bfloat162float(static_cast<const __nv_bfloat16*>(a.s)[is]);
    const float v = a.dv_kind == MLPMOE_FP32 ? static_cast<const float*>(a.dv)[iv] : __bfloat162float(static_cast<const __nv_bfloat16*>(a.dv)[iv]);
    sum_g += v * ((s - a.stats[2 * t]) * a.stats[2 * t + 1]);
    sum_b += v;
  }
  a.partial[static_cast<int64_t>(blockIdx.y) * 2 * a.d + col] = sum_g;
  if (layer) a.partial[(static_cast<int64_t>(blockIdx.y) * 2 + 1) * a.d + col] = sum_b;
}

// The blocks' sums joined: 32 columns of one result to a block, a warp to every 32nd of the blocks.
__global__ void __launch_bounds__(1024) norm_join_kernel(const __grid_constant__ NormGradArgs a, int blocks) {
  __shared__ float part[32][33];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, col = blockIdx.x * 32 + lane;
  float* out = blockIdx.y == 0 ? a.dgain : a.dbias;
  if (out == nullptr) return;
  float sum = 0.0f;
  if (col < a.d)
#pragma unroll 4
    for (int i = w; i < blocks; i += 32) sum += a.partial[(static_cast<int64_t>(i) * 2 + blockIdx.y) * a.d + col];
  part[w][lane] = sum;
  __syncthreads();
  if (w == 0 && col < a.d) {
#pragma unroll
    for (int i = 1; i < 32; ++i) sum += part[i][lane];
    out[col] = sum;
  }
}

// Blocks of a call, and the threads of a row: about 1024 threads on every SM, so that few sums are left to join.
struct Shape {
  int threads, rows, blocks;
};
Shape shape_of(int64_t n, int64_t d) {
  Shape s;
  s.rows = d <= 256 ? 8 : 1;
  s.threads = d <= 256 ? 256 : (d <= 1024 ? 128 : (d <= 2048 ? 256 : (d <= 4096 ? 512 : 1024)));
  const int64_t need = (n + s.rows - 1) / s.rows, most = static_cast<int64_t>(kSms) * (1024 / s.threads);
  s.blocks = static_cast<int>(need < most ? need : most);
  return s;
}

template <bool LAYER, bool VEC>
cudaError_t launch_rows(const NormGradArgs& a, cudaStream_t st) {
  if (a.d > kOnePassD) return launch_pdl(norm_backward_kernel<LAYER, VEC, 1024, 4, false>, dim3(static_cast<unsigned>(a.n)), dim3(1024), 0, st, a);
  const Shape s = shape_of(a.n, a.d);
  const dim3 grid(static_cast<unsigned>(s.blocks)), block(static_cast<unsigned>(s.threads));
  if (a.d <= 256) return launch_pdl(norm_backward_kernel<LAYER, VEC, 32, 1, true>, grid, block, 0, st, a);
  if (a.d <= 1024) return launch_pdl(norm_backward_kernel<LAYER, VEC, 128, 1, true>, grid, block, 0, st, a);
  if (a.d <= 2048) return launch_pdl(norm_backward_kernel<LAYER, VEC, 256, 1, true>, grid, block, 0, st, a);
  if (a.d <= 4096) return launch_pdl(norm_backward_kernel<LAYER, VEC, 512, 1, true>, grid, block, 0, st, a);
  return launch_pdl(norm_backward_kernel<LAYER, VEC, 1024, 1, true>, grid, block, 0, st, a);
}

int64_t stats_bytes(int64_t n, int64_t d) { return d > kOnePassD ? (n * 8 + 15) / 16 * 16 : 0; }
int64_t grad_bytes(int64_t n, int64_t d) {
  const int64_t blocks = d > kOnePassD ? kSplitRows : shape_of(n, d).blocks;
  return stats_bytes(n, d) + (blocks > 0 ? blocks : 1) * 2 * d * 4;
}

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" {

mlpmoe_status_t mlpmoe_norm_backward_workspace(int64_t n_tokens, int64_t d_model, int64_t* bytes) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0 || !bytes) return MLPMOE_ERR_INVALID_ARG;
  if (d_model > kMaxD) return MLPMOE_ERR_UNSUPPORTED;
  *bytes = grad_bytes(n_tokens, d_model);
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_norm_backward(mlpmoe_norm_t norm, const void* s, mlpmoe_dtype_t s_dtype, int64_t s_stride, const float* gain,
                                     const void* grad_out, mlpmoe_dtype_t grad_out_dtype, int64_t grad_out_stride, const void* grad_s,
                                     mlpmoe_dtype_t grad_s_dtype, int64_t grad_s_stride, void* grad_x, mlpmoe_dtype_t grad_x_dtype,
                                     int64_t grad_x_stride, float* grad_gain, float* grad_bias, int64_t n_tokens, int64_t d_model,
                                     float eps, void* workspace, int64_t workspace_bytes, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0) return MLPMOE_ERR_INVALID_ARG;
  if (norm != MLPMOE_RMSNORM && norm != MLPMOE_LAYERNORM) return MLPMOE_ERR_INVALID_ARG;
  for (mlpmoe_dtype_t k : {s_dtype, grad_out_dtype, grad_x_dtype})
    if (k != MLPMOE_FP32 && k != MLPMOE_BF16) return MLPMOE_ERR_INVALID_ARG;
  if (grad_s && grad_s_dtype != MLPMOE_FP32 && grad_s_dtype != MLPMOE_BF16) return MLPMOE_ERR_INVALID_ARG;
  if (norm == MLPMOE_RMSNORM && grad_bias) return MLPMOE_ERR_INVALID_ARG;
  if (d_model > kMaxD) return MLPMOE_ERR_UNSUPPORTED;
  if (s_stride == 0) s_stride = d_model;
  if (grad_out_stride == 0) grad_out_stride = d_model;
  if (grad_s_stride == 0) grad_s_stride = d_model;
  if (grad_x_stride == 0) grad_x_stride = d_model;
  if (s_stride < d_model || grad_out_stride < d_model || (grad_s && grad_s_stride < d_model) || grad_x_stride < d_model)
    return MLPMOE_ERR_INVALID_ARG;
  if (!on(grad_gain, 4) || !on(grad_bias, 4) || !on(gain, 4)) return MLPMOE_ERR_INVALID_ARG;
  const bool sums = grad_gain || grad_bias;
  if (sums && (!workspace || workspace_bytes < grad_bytes(n_tokens, d_model) || !on(workspace, 16))) return MLPMOE_ERR_INVALID_ARG;
  NormGradArgs a = {};
  a.d = static_cast<int>(d_model);
  a.n = n_tokens;
  a.dgain = grad_gain;
  a.dbias = grad_bias;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const dim3 join_grid(static_cast<unsigned>((d_model + 31) / 32), norm == MLPMOE_LAYERNORM ? 2 : 1);
  pdl_overlap_enabled() = true;
  if (n_tokens == 0) {
    if (sums && launch_pdl(norm_join_kernel, join_grid, dim3(1024), 0, st, a, 0) != cudaSuccess) return MLPMOE_ERR_CUDA;
    return MLPMOE_OK;
  }
  if (!s || !grad_out || !grad_x || grad_x == s || grad_x == grad_out) return MLPMOE_ERR_INVALID_ARG;
  if (grad_x == grad_s && (grad_x_dtype != grad_s_dtype || (grad_x_stride != grad_s_stride && n_tokens > 1))) return MLPMOE_ERR_INVALID_ARG;
  if (!on(s, bytes_of(s_dtype)) || !on(grad_out, bytes_of(grad_out_dtype)) || !on(grad_x, bytes_of(grad_x_dtype)) ||
      (grad_s && !on(grad_s, bytes_of(grad_s_dtype))))
    return MLPMOE_ERR_INVALID_ARG;
  const bool vec = d_model % 8 == 0 && s_stride % 8 == 0 && on(s, 16) && grad_out_stride % 8 == 0 && on(grad_out, 16) &&
                   grad_x_stride % 8 == 0 && on(grad_x, 16) && (!grad_s || (grad_s_stride % 8 == 0 && on(grad_s, 16))) && on(gain, 16);
  a.s = s;
  a.dv = grad_out;
  a.ds = grad_s;
  a.gain = gain;
  a.dx = grad_x;
  a.s_stride = s_stride;
  a.dv_stride = grad_out_stride;
  a.ds_stride = grad_s ? grad_s_stride : 0;
  a.dx_stride = grad_x_stride;
  a.s_kind = s_dtype;
  a.dv_kind = grad_out_dtype;
  a.ds_kind = grad_s ? static_cast<int>(grad_s_dtype) : kNone;
  a.dx_kind = grad_x_dtype;
  a.eps = eps;
  a.stats = sums && d_model > kOnePassD ? static_cast<float*>(workspace) : nullptr;
  a.partial = sums ? reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + stats_bytes(n_tokens, d_model)) : nullptr;
  cudaError_t e;
  if (norm == MLPMOE_LAYERNORM)
    e = vec ? launch_rows<true, true>(a, st) : launch_rows<true, false>(a, st);
  else
    e = vec ? launch_rows<false, true>(a, st) : launch_rows<false, false>(a, st);
  if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  if (!sums) return MLPMOE_OK;
  int blocks = shape_of(n_tokens, d_model).blocks;
  if (d_model > kOnePassD) {
    blocks = static_cast<int>(n_tokens < kSplitRows ? n_tokens : kSplitRows);
    e = launch_pdl(norm_column_sums_kernel, dim3(static_cast<unsigned>((d_model + 255) / 256), static_cast<unsigned>(blocks)), dim3(256), 0, st, a,
                   norm == MLPMOE_LAYERNORM ? 1 : 0);
    if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  } else if (blocks == 1) {
    return MLPMOE_OK;
  }
  return launch_pdl(norm_join_kernel, join_grid, dim3(1024), 0, st, a, blocks) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
