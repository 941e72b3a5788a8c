// Gradient of the residual norms (mlpmoe_norm_backward), with the sums over tokens for gain and bias:
//     z = s - mean(s) (LayerNorm) or s (RMSNorm);  inv = 1 / sqrt(mean(z^2) + eps);  h = gain * dv;
//     dx = ds + inv * (h - mean(h) - z * inv^2 * mean(h z))   (mean(h): LayerNorm only);
//     dgain = sum_t dv * z * inv;   dbias = sum_t dv.
// HBM-bound: s, dv and ds are read once, a block keeps its columns' sums over all of its rows in registers, the next rows are on
// their way while a row is reduced, and the blocks' sums are joined by a second launch in a fixed order.
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

__device__ __forceinline__ void copy_async16(uint4* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Pieces of 16 bytes that eight elements of a kind take.
__host__ __device__ constexpr int pieces_of(int kind) { return kind == MLPMOE_FP32 ? 2 : (kind == MLPMOE_BF16 ? 1 : 0); }

// T threads to a row (T = 32: eight rows to a block), NCH chunks of eight columns a thread, whose sums over the block's rows stay in
// registers.  The next STAGES - 1 rows are on their way to shared memory meanwhile; a thread reads only what it copied itself, so that
// takes no barrier.  (The rows ahead in registers: 98 of them a thread, one block of 512 per SM, 258 us at 16384 x 4096.)
template <bool LAYER, bool VEC, int T, int NCH, int STAGES, int CTAS>
__global__ void __launch_bounds__(T == 32 ? 256 : T, CTAS) norm_backward_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr int R = T == 32 ? 8 : 1, THREADS = T == 32 ? 256 : T;
  extern __shared__ uint4 staged[];
  __shared__ float red[2][T / 32][4];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int tid = T == 32 ? threadIdx.x % 32 : threadIdx.x, d = a.d;
  const int ps = pieces_of(a.s_kind), pv = pieces_of(a.dv_kind), pr = pieces_of(a.ds_kind), pieces = ps + pv + pr;
  const int64_t step = static_cast<int64_t>(gridDim.x) * R;
  int64_t t = static_cast<int64_t>(blockIdx.x) * R + (T == 32 ? threadIdx.x / 32 : 0);
  float sum_g[NCH][8], sum_b[LAYER ? NCH : 1][8];
#pragma unroll
  for (int i = 0; i < NCH; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum_g[i][e] = 0.0f;
      if (LAYER) sum_b[i][e] = 0.0f;
    }
  auto slot = [&](int stage, int i, int piece) { return staged + ((stage * NCH + i) * pieces + piece) * THREADS + threadIdx.x; };
  auto fetch_one = [&](const void* base, int kind, int64_t offset, int stage, int i, int first) {
    const int col = (i * T + tid) * 8;
    const char* p = static_cast<const char*>(base) + offset * bytes_of(kind);
    if (VEC) {
      if (col >= d) return;
      copy_async16(slot(stage, i, first), p + col * bytes_of(kind));
      if (kind == MLPMOE_FP32) copy_async16(slot(stage, i, first + 1), p + col * 4 + 16);
    } else {
      const Chunk c = load_chunk<false>(p, kind, col, d);
      *slot(stage, i, first) = c.a;
      if (kind == MLPMOE_FP32) *slot(stage, i, first + 1) = c.b;
    }
  };
  auto fetch = [&](int64_t row, int stage) {
    if (row < a.n) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        fetch_one(a.s, a.s_kind, row * a.s_stride, stage, i, 0);
        fetch_one(a.dv, a.dv_kind, row * a.dv_stride, stage, i, ps);
        if (pr != 0) fetch_one(a.ds, a.ds_kind, row * a.ds_stride, stage, i, ps + pv);
      }
    }
    copy_commit();
  };
  auto value = [&](int stage, int i, int first, int kind, float (&v)[8]) {
    Chunk c;
    c.a = c.b = make_uint4(0u, 0u, 0u, 0u);
    if (!VEC || (i * T + tid) * 8 < d) {
      c.a = *slot(stage, i, first);
      if (kind == MLPMOE_FP32) c.b = *slot(stage, i, first + 1);
    }
    to_f32(c, kind, v);
  };
  auto gain_of = [&](int i, float (&g)[8]) {      // from the L1 cache: eight registers a chunk are worth more
    if (a.gain != nullptr) {
      to_f32(load_chunk<VEC>(a.gain, MLPMOE_FP32, (i * T + tid) * 8, d), MLPMOE_FP32, g);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = 1.0f;
    }
  };
#pragma unroll
  for (int k = 0; k < STAGES; ++k) fetch(t + k * step, k);
  int turn = 0, stage = 0;
  const float inv_d = 1.0f / static_cast<float>(d);
  for (; t < a.n; t += step) {
    copy_wait<STAGES - 1>();
    float z[NCH][8], v[NCH][8];
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      value(stage, i, 0, a.s_kind, z[i]);
      value(stage, i, ps, a.dv_kind, v[i]);
    }
    float mean_h = 0.0f, ss, hz;
    if (LAYER) {
      float sum[1] = {0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[0] += z[i][e];
      row_sums<T, 1>(sum, red, turn);
      const float mean = sum[0] * inv_d;
      float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        float gain[8];
        gain_of(i, gain);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int col = (i * T + tid) * 8 + (VEC ? 0 : e);
          z[i][e] = col < d ? z[i][e] - mean : 0.0f;
          const float h = gain[e] * v[i][e];
          q[0] += z[i][e] * z[i][e];
          q[1] += h * z[i][e];
          q[2] += h;
        }
      }
      row_sums<T, 3>(q, red, turn);
      ss = q[0];
      hz = q[1];
      mean_h = q[2] * inv_d;
    } else {
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        float gain[8];
        gain_of(i, gain);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          q[0] += z[i][e] * z[i][e];
          q[1] += gain[e] * v[i][e] * z[i][e];
        }
      }
      row_sums<T, 2>(q, red, turn);
      ss = q[0];
      hz = q[1];
    }
    const float inv = 1.0f / sqrtf(ss * inv_d + a.eps);
    const float along = hz * inv * inv * inv_d;
    char* px = static_cast<char*>(a.dx) + t * a.dx_stride * bytes_of(a.dx_kind);
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      float gain[8], r[8];
      gain_of(i, gain);
      if (pr != 0) {
        value(stage, i, ps + pv, a.ds_kind, r);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum_g[i][e] += v[i][e] * (z[i][e] * inv);
        if (LAYER) sum_b[i][e] += v[i][e];
        r[e] += inv * (gain[e] * v[i][e] - mean_h - z[i][e] * along);
      }
      const int col = (i * T + tid) * 8;
      if (col < d) store8<VEC>(px, a.dx_kind, col, d, r);
    }
    fetch(t + STAGES * step, stage);
    stage = stage + 1 == STAGES ? 0 : stage + 1;
  }
  if (a.dgain == nullptr && a.dbias == nullptr) return;
  // the block's sums: to the result where it is the only block
  float* out_g = gridDim.x == 1 ? a.dgain : a.partial + static_cast<int64_t>(blockIdx.x) * 2 * d;
  float* out_b = gridDim.x == 1 ? a.dbias : a.partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * d;
  if (T == 32) {                           // the eight rows' sums first; the copies are done with shared memory
    float* join = reinterpret_cast<float*>(staged);
#pragma unroll
    for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
      copy_wait<0>();
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 8; ++e) join[threadIdx.x * 8 + e] = which == 0 ? sum_g[0][e] : sum_b[0][e];
      __syncthreads();
      float* out = which == 0 ? out_g : out_b;
      if (threadIdx.x < d && out != nullptr) {
        float sum = join[threadIdx.x];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += join[w * 256 + threadIdx.x];
        out[threadIdx.x] = sum;
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NCH; ++i) {
      const int col = (i * T + tid) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (col + e >= d) continue;
        if (out_g != nullptr) out_g[col + e] = sum_g[i][e];
        if (LAYER && out_b != nullptr) out_b[col + e] = sum_b[LAYER ? i : 0][e];
      }
    }
  }
}

// Rows above 8192 columns, a block to a row: no room for the columns' sums, so the row's mean and inv go to memory for a kernel of
// their own, and grad_out is read a second time (from the L2 cache) instead of being held.
template <bool LAYER, bool VEC>
__global__ void __launch_bounds__(1024, 1) norm_backward_long_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr int T = 1024, NCH = 4;
  __shared__ float red[2][T / 32][4];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int d = a.d;
  const int64_t t = blockIdx.x;
  const char* ps = static_cast<const char*>(a.s) + t * a.s_stride * bytes_of(a.s_kind);
  const char* pv = static_cast<const char*>(a.dv) + t * a.dv_stride * bytes_of(a.dv_kind);
  const char* pr = static_cast<const char*>(a.ds) + t * a.ds_stride * bytes_of(a.ds_kind);
  char* px = static_cast<char*>(a.dx) + t * a.dx_stride * bytes_of(a.dx_kind);
  const float inv_d = 1.0f / static_cast<float>(d);
  int turn = 0;
  float z[NCH][8], mean = 0.0f;
#pragma unroll
  for (int i = 0; i < NCH; ++i) to_f32(load_chunk<VEC>(ps, a.s_kind, (i * T + threadIdx.x) * 8, d), a.s_kind, z[i]);
  if (LAYER) {
    float sum[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NCH; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[0] += z[i][e];
    row_sums<T, 1>(sum, red, turn);
    mean = sum[0] * inv_d;
  }
  auto h_of = [&](int i, float (&h)[8]) {
    const int col = (i * T + threadIdx.x) * 8;
    to_f32(load_chunk<VEC>(pv, a.dv_kind, col, d), a.dv_kind, h);
    if (a.gain != nullptr) {
      float g[8];
      to_f32(load_chunk<VEC>(a.gain, MLPMOE_FP32, col, d), MLPMOE_FP32, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] *= g[e];
    }
  };
  float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    float h[8];
    h_of(i, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (LAYER) z[i][e] = (i * T + threadIdx.x) * 8 + e < d ? z[i][e] - mean : 0.0f;
      q[0] += z[i][e] * z[i][e];
      q[1] += h[e] * z[i][e];
      q[2] += h[e];
    }
  }
  row_sums<T, 3>(q, red, turn);
  const float inv = 1.0f / sqrtf(q[0] * inv_d + a.eps);
  const float along = q[1] * inv * inv * inv_d, mean_h = LAYER ? q[2] * inv_d : 0.0f;
  if (threadIdx.x == 0 && a.stats != nullptr) {
    a.stats[2 * t] = mean;
    a.stats[2 * t + 1] = inv;
  }
#pragma unroll
  for (int i = 0; i < NCH; ++i) {
    const int col = (i * T + threadIdx.x) * 8;
    if (col >= d) continue;
    float h[8], r[8] = {};
    h_of(i, h);
    if (a.ds_kind != kNone) to_f32(load_chunk<VEC>(pr, a.ds_kind, col, d), a.ds_kind, r);
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] += inv * (h[e] - mean_h - z[i][e] * along);
    store8<VEC>(px, a.dx_kind, col, d, r);
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

// How a row of d columns is dealt: threads of a row and chunks of a thread, stages of rows on their way, blocks per SM.  Registers and
// shared memory (40 bytes a chunk of fp32 s, bf16 grad_out, fp32 grad_s, up to 96) allow that many, and few blocks leave few sums to join.
struct Shape {
  int threads, rows, chunks, stages, ctas;
};
constexpr Shape kShapes[] = {{256, 8, 1, 3, 3}, {128, 1, 1, 3, 6}, {256, 1, 1, 3, 3}, {512, 1, 1, 2, 2}, {1024, 1, 1, 2, 1}};
int shape_of(int64_t d) { return d <= 256 ? 0 : (d <= 1024 ? 1 : (d <= 2048 ? 2 : (d <= 4096 ? 3 : 4))); }
int blocks_of(int64_t n, int64_t d) {
  const Shape s = kShapes[shape_of(d)];
  const int64_t need = (n + s.rows - 1) / s.rows, most = static_cast<int64_t>(kSms) * s.ctas;
  return static_cast<int>(need < most ? need : most);
}

template <bool LAYER, bool VEC, int SHAPE>
cudaError_t launch_shape(const NormGradArgs& a, cudaStream_t st) {
  constexpr Shape s = kShapes[SHAPE];
  auto kernel = norm_backward_kernel<LAYER, VEC, s.rows == 8 ? 32 : s.threads, s.chunks, s.stages, s.ctas>;
  const int bytes = s.stages * s.chunks * s.threads * 16, pieces = pieces_of(a.s_kind) + pieces_of(a.dv_kind) + pieces_of(a.ds_kind);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 6 * bytes);      // the same for every call
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks_of(a.n, a.d))), dim3(s.threads), static_cast<size_t>(pieces) * bytes, st, a);
}
template <bool LAYER, bool VEC>
cudaError_t launch_rows(const NormGradArgs& a, cudaStream_t st) {
  if (a.d > kOnePassD) return launch_pdl(norm_backward_long_kernel<LAYER, VEC>, dim3(static_cast<unsigned>(a.n)), dim3(1024), 0, st, a);
  switch (shape_of(a.d)) {
    case 0: return launch_shape<LAYER, VEC, 0>(a, st);
    case 1: return launch_shape<LAYER, VEC, 1>(a, st);
    case 2: return launch_shape<LAYER, VEC, 2>(a, st);
    case 3: return launch_shape<LAYER, VEC, 3>(a, st);
    default: return launch_shape<LAYER, VEC, 4>(a, st);
  }
}

int64_t stats_bytes(int64_t n, int64_t d) { return d > kOnePassD ? (n * 8 + 15) / 16 * 16 : 0; }
int64_t grad_bytes(int64_t n, int64_t d) {
  const int64_t blocks = d > kOnePassD ? kSplitRows : blocks_of(n, d);
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
  int blocks = blocks_of(n_tokens, d_model);
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
