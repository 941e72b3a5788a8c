// Gradient of the residual norms (mlpmoe_norm_backward), with the sums over tokens for gain and bias:
//     z = s - mean(s) (LayerNorm) or s (RMSNorm);  inv = 1 / sqrt(mean(z^2) + eps);  h = gain * dv;
//     dx = ds + inv * (h - mean(h) - z * inv^2 * mean(h z))   (mean(h): LayerNorm only);
//     dgain = sum_t dv * z * inv;   dbias = sum_t dv.
// HBM-bound: s, dv and ds are read once, a block keeps its columns' sums over all of its rows in registers, the next rows are on
// their way while a row is reduced, and the blocks' sums are joined by a second launch in a fixed order (5 us of 16384 x 4096, hidden
// in part; none where one block has all rows).
#include <atomic>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "norm_shapes.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kNone = 2;
constexpr int64_t kMaxD = 32768;

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

// Four consecutive values of a kind as they stand in shared memory (fp32: 16 bytes, bf16: 8).
template <int KIND>
__device__ __forceinline__ void quad_of(const char* p, float (&v)[4]) {
  if (KIND == MLPMOE_FP32) {
    const float4 f = *reinterpret_cast<const float4*>(p);
    v[0] = f.x, v[1] = f.y, v[2] = f.z, v[3] = f.w;
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = bf16_lo(u.x), v[1] = bf16_hi(u.x), v[2] = bf16_lo(u.y), v[3] = bf16_hi(u.y);
  }
}
// Four neighbours on their way to shared memory.
__device__ __forceinline__ void copy_quad(char* to, const char* from, int kind) {
  if (kind == MLPMOE_FP32) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
  } else {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(ptx::smem_u32(to)), "l"(from) : "memory");
  }
}
// A row that starts anywhere, by its T threads: what of it fills whole pieces of 16 bytes goes in those, the rest in words of four, to the same
// place relative to 16 bytes.  What stands beside the row is not read: of a word that only half belongs to it (bf16, its first or
// last value) a thread keeps the value for later, marked 1 or 2 above its 16 bits.
template <int T>
__device__ __forceinline__ uint32_t copy_row(char* to, const char* row, int bytes, int d, int tid) {
  const int lead = static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15), end = lead + d * bytes;
  const char* from = row - lead;
  for (int at = 16 * tid; at + 16 <= end; at += 16 * T)
    if (at >= lead) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ptx::smem_u32(to + at)), "l"(from + at) : "memory");
  uint32_t kept = 0;
  if (tid < 8) {
    const bool some = tid < 4 ? lead > 0 || end < 16 : end >= 16 && end % 16 != 0;      // the first piece, the last
    const int at = (tid < 4 ? 0 : end / 16 * 16) + 4 * (tid % 4);
    if (some && at >= lead && at + 4 <= end) {
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(ptx::smem_u32(to + at)), "l"(from + at) : "memory");
    } else if (some && at + 2 == lead) {
      kept = load_if<2>(row, true) | 1u << 16;
    } else if (some && at >= lead && at + 2 == end) {
      kept = load_if<2>(from + at, true) | 2u << 16;
    }
  }
  return kept;
}
__device__ __forceinline__ void put_kept(char* row, uint32_t kept, int d) {
  if (kept != 0) *reinterpret_cast<uint16_t*>(row + (kept >> 17 ? 2 * (d - 1) : 0)) = static_cast<uint16_t>(kept);
}
__device__ __forceinline__ float row_value(const char* row, int kind, int c) {
  return kind == MLPMOE_FP32 ? reinterpret_cast<const float*>(row)[c] : bf16_lo(reinterpret_cast<const uint16_t*>(row)[c]);
}

constexpr int kStages = 2;

// A row to the block's T threads (T = 32: to each of its eight warps), Q times four neighbouring columns a thread (not WIDE, where they
// start anywhere: columns T apart, so that a warp's accesses are neighbours), whose sums over
// the block's rows stay in registers.  The next row is on its way to shared memory meanwhile; a thread reads only what it
// copied itself, so that takes no barrier (not WIDE: two).  16384 x 4096, fp32 and bf16: 940 MB in
// 157 us with the join over seconds (floor 146).  The row ahead in registers and types told apart as it runs: 258 (98 registers, 512 threads per SM); four
// times four columns a thread: 159 (16 warps per SM).
// Not WIDE the time goes with the elements: past shared memory every value is a load and a store of two or four bytes with a bound of its own. 12288 x 4096
// with rows 4101 apart 173 us (63 % of a copy), 12285 x 4097 241 (46 %), 16384 x 201 22 (33 %); all in bf16 206, 293 and 24 (30, 21 and 17 %).
// Below about 1400 columns a block with one row at a time waits for its sums, and many blocks' column sums go through memory: 16384 x 1100 57 us (68 %),
// x 1000 48 (74 %), x 400 28 (50 %), x 200 14.6 (49 %).
// FULL: ds is there, and it and dx are fp32 (told apart as it runs, the same case takes 11 % more instructions and 167 us over seconds, not 157).
// A stream in bf16 has no such kernel: 16384 x 4096 all in bf16 takes 152 us (RMSNorm 121) for 537 MB, 55 and 69 %.
template <bool LAYER, int T, int Q, int CTAS, bool WIDE, int SK, int VK, bool FULL>
__global__ void __launch_bounds__(T == 32 ? 256 : T, CTAS) norm_backward_kernel(const __grid_constant__ NormGradArgs a) {
  constexpr bool WARP = T == 32;
  constexpr int R = WARP ? 8 : 1, THREADS = WARP ? 256 : T, SB = bytes_of(SK), VB = bytes_of(VK);
  extern __shared__ __align__(16) char staged[];
  __shared__ float red[2][T / 32][4];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int d = a.d, tid = WARP ? threadIdx.x % 32 : threadIdx.x, rb = FULL ? 4 : bytes_of(a.ds_kind), xb = FULL ? 4 : bytes_of(a.dx_kind);
  const bool has_r = FULL || a.ds_kind != kNone, r32 = FULL || a.ds_kind == MLPMOE_FP32, x32 = FULL || a.dx_kind == MLPMOE_FP32;
  const int64_t step = static_cast<int64_t>(gridDim.x) * R, first = static_cast<int64_t>(blockIdx.x) * R + (WARP ? threadIdx.x / 32 : 0);
  const int rows = first < a.n ? static_cast<int>((a.n - first + step - 1) / step) : 0;      // of this block or warp
  const int col = WIDE ? tid * 4 : tid, base = WIDE ? col : 0;      // the thread's first column, and the pointers'
  auto apart = [](int k, int e) { return WIDE ? 4 * T * k + e : (4 * k + e) * T; };      // of value e of quad k
  const char* ps = static_cast<const char*>(a.s) + (first * a.s_stride + base) * SB;
  const char* pv = static_cast<const char*>(a.dv) + (first * a.dv_stride + base) * VB;
  const char* pr = static_cast<const char*>(a.ds) + (first * a.ds_stride + base) * rb;
  char* px = static_cast<char*>(a.dx) + (first * a.dx_stride + base) * xb;
  const int64_t ds = step * a.s_stride * SB, dv = step * a.dv_stride * VB, dr = step * a.ds_stride * rb, dx = step * a.dx_stride * xb;
  // in shared memory: [stage][quad][thread], 4 SB bytes of s, then 4 VB of dv, then room for 16 of ds; not WIDE: [stage][row] of each in turn,
  // with 16 bytes more
  constexpr int V_AT = kStages * Q * THREADS * 4 * SB, R_AT = V_AT + kStages * Q * THREADS * 4 * VB;
  constexpr int S_ROW = Q * T * 4 * SB + 16, V_ROW = Q * T * 4 * VB + 16, R_ROW = Q * T * 16 + 16;
  char* const mine_s = WIDE ? staged + threadIdx.x * 4 * SB : staged + (WARP ? threadIdx.x / 32 : 0) * kStages * (S_ROW + V_ROW + (has_r ? R_ROW : 0));
  char* const mine_v = WIDE ? staged + V_AT + threadIdx.x * 4 * VB : mine_s + kStages * S_ROW;
  char* const mine_r = WIDE ? staged + R_AT + threadIdx.x * 16 : mine_v + kStages * V_ROW;
  // not WIDE: where the rows of s, dv and ds start in their 16 bytes, and the values kept for later; of this row and of the next
  struct Edges {
    uint32_t lead, s, v, r;
  };
  Edges now = {}, next = {}, fetched = {};
  auto sync_row = [&]() {
    if (WARP) {
      __syncwarp();
    } else {
      __syncthreads();
    }
  };
  auto fetch = [&](bool more, int stage) {      // the row at ps, pv, pr; then the one after it in turn
    if (more) {
      if (WIDE) {
#pragma unroll
        for (int k = 0; k < Q; ++k) {
          const int at = stage * Q + k, c = apart(k, 0);
          if (col + c >= d) continue;
          copy_quad(mine_s + at * (THREADS * 4 * SB), ps + c * SB, SK);
          copy_quad(mine_v + at * (THREADS * 4 * VB), pv + c * VB, VK);
          if (has_r) copy_quad(mine_r + at * (THREADS * 16), pr + c * rb, FULL ? MLPMOE_FP32 : a.ds_kind);
        }
      } else {
        fetched.s = copy_row<T>(mine_s + stage * S_ROW, ps, SB, d, tid);
        fetched.v = copy_row<T>(mine_v + stage * V_ROW, pv, VB, d, tid);
        if (has_r) fetched.r = copy_row<T>(mine_r + stage * R_ROW, pr, rb, d, tid);
        fetched.lead = static_cast<uint32_t>((reinterpret_cast<uintptr_t>(ps) & 15) | (reinterpret_cast<uintptr_t>(pv) & 15) << 4 | (reinterpret_cast<uintptr_t>(pr) & 15) << 8);
      }
      ps += ds;
      pv += dv;
      pr += dr;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float gain[Q][4], sum_g[Q][4], sum_b[LAYER ? Q : 1][4];
#pragma unroll
  for (int k = 0; k < Q; ++k)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = col + apart(k, e);
      gain[k][e] = c < d ? (a.gain != nullptr ? a.gain[c] : 1.0f) : 0.0f;
      sum_g[k][e] = 0.0f;
      if (LAYER) sum_b[k][e] = 0.0f;
    }
#pragma unroll
  for (int k = 0; k < kStages; ++k) {
    fetch(k < rows, k);
    now = next;
    next = fetched;
  }
  int turn = 0;
  const float inv_d = 1.0f / static_cast<float>(d);
  for (int i = 0; i < rows; ++i) {
    const int stage = i % kStages;
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    const char* const row_s = mine_s + stage * S_ROW + (now.lead & 15);      // not WIDE
    const char* const row_v = mine_v + stage * V_ROW + (now.lead >> 4 & 15);
    const char* const row_r = mine_r + stage * R_ROW + (now.lead >> 8 & 15);
    if (!WIDE) {
      put_kept(const_cast<char*>(row_s), now.s, d);
      put_kept(const_cast<char*>(row_v), now.v, d);
      put_kept(const_cast<char*>(row_r), now.r, d);
      sync_row();                          // the others' copies too
    }
    float z[Q][4], v[Q][4];
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const int at = stage * Q + k;
      if (!WIDE) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = col + apart(k, e);
          z[k][e] = c < d ? row_value(row_s, SK, c) : 0.0f;
          v[k][e] = c < d ? row_value(row_v, VK, c) : 0.0f;
        }
      } else if (col + apart(k, 0) < d) {
        quad_of<SK>(mine_s + at * (THREADS * 4 * SB), z[k]);
        quad_of<VK>(mine_v + at * (THREADS * 4 * VB), v[k]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[k][e] = v[k][e] = 0.0f;
      }
    }
    float mean_h = 0.0f, ss, hz;
    if (LAYER) {
      float sum[1] = {0.0f};
#pragma unroll
      for (int k = 0; k < Q; ++k) sum[0] += (z[k][0] + z[k][1]) + (z[k][2] + z[k][3]);
      row_sums<T, 1>(sum, red, turn);
      const float mean = sum[0] * inv_d;
      float q[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          z[k][e] = col + apart(k, WIDE ? 0 : e) < d ? z[k][e] - mean : 0.0f;
          const float h = gain[k][e] * v[k][e];
          q[0] = fmaf(z[k][e], z[k][e], q[0]);
          q[1] = fmaf(h, z[k][e], q[1]);
          q[2] += h;
        }
      row_sums<T, 3>(q, red, turn);
      ss = q[0];
      hz = q[1];
      mean_h = q[2] * inv_d;
    } else {
      float q[2] = {0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          q[0] = fmaf(z[k][e], z[k][e], q[0]);
          q[1] = fmaf(gain[k][e] * v[k][e], z[k][e], q[1]);
        }
      row_sums<T, 2>(q, red, turn);
      ss = q[0];
      hz = q[1];
    }
    const float inv = rsqrtf(ss * inv_d + a.eps);
    const float along = hz * inv * inv * inv_d;
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const int c = apart(k, 0), at = stage * Q + k;
      if (col + c >= d) continue;
      float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      if (has_r && !WIDE) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (col + apart(k, e) < d) r[e] = row_value(row_r, a.ds_kind, col + apart(k, e));
      } else if (has_r) {
        if (r32) {
          quad_of<MLPMOE_FP32>(mine_r + at * (THREADS * 16), r);
        } else {
          quad_of<MLPMOE_BF16>(mine_r + at * (THREADS * 16), r);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        sum_g[k][e] = fmaf(v[k][e], z[k][e] * inv, sum_g[k][e]);
        if (LAYER) sum_b[k][e] += v[k][e];
        r[e] = fmaf(inv, fmaf(-z[k][e], along, fmaf(gain[k][e], v[k][e], -mean_h)), r[e]);
      }
      if (x32) {
        float* p = reinterpret_cast<float*>(px) + (WIDE ? c : col + c);
        if (WIDE) {
          __stcs(reinterpret_cast<float4*>(p), make_float4(r[0], r[1], r[2], r[3]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + apart(k, e) < d) p[apart(0, e)] = r[e];
        }
      } else {
        __nv_bfloat16* p = reinterpret_cast<__nv_bfloat16*>(px) + (WIDE ? c : col + c);
        if (WIDE) {
          *reinterpret_cast<uint2*>(p) = make_uint2(pack2(r[0], r[1]), pack2(r[2], r[3]));
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + apart(k, e) < d) p[apart(0, e)] = __float2bfloat16_rn(r[e]);
        }
      }
    }
    px += dx;
    if (!WIDE) sync_row();                 // everybody is done with the stage
    fetch(i + kStages < rows, stage);
    now = next;
    next = fetched;
  }
  if (a.dgain == nullptr && a.dbias == nullptr) return;
  // the block's sums: to the result where it is the only block
  float* out[2] = {gridDim.x == 1 ? a.dgain : a.partial + static_cast<int64_t>(blockIdx.x) * 2 * d,
                   gridDim.x == 1 ? a.dbias : a.partial + (static_cast<int64_t>(blockIdx.x) * 2 + 1) * d};
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  float* join = reinterpret_cast<float*>(staged);      // T = 32: the eight rows' sums first
#pragma unroll
  for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
    if (WARP) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) join[(threadIdx.x / 32) * 256 + col + apart(k, e)] = which == 0 ? sum_g[k][e] : sum_b[LAYER ? k : 0][e];
      __syncthreads();
      if (static_cast<int>(threadIdx.x) < d && out[which] != nullptr) {
        float sum = join[threadIdx.x];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += join[w * 256 + threadIdx.x];
        out[which][threadIdx.x] = sum;
      }
    } else if (out[which] != nullptr) {
#pragma unroll
      for (int k = 0; k < Q; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int c = col + apart(k, e);
          if (c < d) out[which][c] = which == 0 ? sum_g[k][e] : sum_b[LAYER ? k : 0][e];
        }
    }
  }
}

// Rows above 8192 columns, a block to a row: no room for the columns' sums, so the row's mean and inv go to memory for a kernel of
// their own, and grad_out is read a second time (from the L2 cache) instead of being held.  2048 x 20000, fp32 and bf16: 574 MB in 242 us (RMSNorm 218), 37 and
// 41 % of a copy; 4096 x 12288 310 and 282, 35 and 39 %; all in bf16 23 to 29 %, odd rows 16 to 23 %.  The rows alone take 142 us (RMSNorm 129), one
// row a block and SM, its loads alone with their latency; the rest are the sums, which read s and grad_out once more, two or four bytes a load.
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
#pragma unroll 8
    for (int i = w; i < blocks; i += 32) sum += a.partial[(static_cast<int64_t>(i) * 2 + blockIdx.y) * a.d + col];
  part[w][lane] = sum;
  __syncthreads();
  if (w == 0 && col < a.d) {
#pragma unroll
    for (int i = 1; i < 32; ++i) sum += part[i][lane];
    out[col] = sum;
  }
}

// A kernel's shared memory, once on each device: `bytes` of it for a block, and the SM's split between it and the L1 cache at its most.  Both
// kernels of a call ask for the same split: where the join got another, the next call's blocks, which start while it runs, did not
// find room for four to an SM (16384 x 2048, calls one after the other: 101 us, 80 with another kernel between them).
template <typename Kernel>
cudaError_t set_shared(Kernel kernel, int bytes, std::atomic<uint64_t>& done) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const uint64_t bit = device < 64 ? uint64_t{1} << device : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  if (bytes > 0) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

template <bool LAYER, bool WIDE, int SHAPE, int SK, int VK, bool FULL>
cudaError_t launch_kernel(const NormGradArgs& a, cudaStream_t st) {
  constexpr Shape s = kShapes[SHAPE];
  constexpr int threads = s.threads == 32 ? 256 : s.threads, rows = s.threads == 32 ? 8 : 1, more = WIDE ? 0 : kStages * rows * 16;
  constexpr int held = kStages * 4 * s.quads * threads * (bytes_of(SK) + bytes_of(VK)) + 2 * more, most = held + kStages * 16 * s.quads * threads + more;
  auto kernel = norm_backward_kernel<LAYER, s.threads, s.quads, s.ctas, WIDE, SK, VK, FULL>;
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = set_shared(kernel, most, done);      // the same for every call, whatever its own size
  if (e != cudaSuccess) return e;
  return launch_pdl(kernel, dim3(static_cast<unsigned>(blocks_of(a.n, a.d))), dim3(threads), static_cast<size_t>(a.ds_kind == kNone ? held : most), st, a);
}
template <bool LAYER, bool WIDE, int SHAPE, int SK, int VK>
cudaError_t launch_kinds(const NormGradArgs& a, cudaStream_t st) {
  constexpr bool kStream = WIDE && SK == MLPMOE_FP32;      // an fp32 residual stream
  if (kStream && a.ds_kind == MLPMOE_FP32 && a.dx_kind == MLPMOE_FP32) return launch_kernel<LAYER, WIDE, SHAPE, SK, VK, kStream>(a, st);
  return launch_kernel<LAYER, WIDE, SHAPE, SK, VK, false>(a, st);
}
template <bool LAYER, bool WIDE, int SHAPE>
cudaError_t launch_from(const NormGradArgs& a, cudaStream_t st) {
  if (a.s_kind == MLPMOE_FP32)
    return a.dv_kind == MLPMOE_FP32 ? launch_kinds<LAYER, WIDE, SHAPE, MLPMOE_FP32, MLPMOE_FP32>(a, st)
                                    : launch_kinds<LAYER, WIDE, SHAPE, MLPMOE_FP32, MLPMOE_BF16>(a, st);
  return a.dv_kind == MLPMOE_FP32 ? launch_kinds<LAYER, WIDE, SHAPE, MLPMOE_BF16, MLPMOE_FP32>(a, st)
                                  : launch_kinds<LAYER, WIDE, SHAPE, MLPMOE_BF16, MLPMOE_BF16>(a, st);
}
template <bool LAYER, bool WIDE>
cudaError_t launch_rows(const NormGradArgs& a, cudaStream_t st) {
  if (a.d > kOnePassD) return launch_pdl(norm_backward_long_kernel<LAYER, WIDE>, dim3(static_cast<unsigned>(a.n)), dim3(1024), 0, st, a);
  switch (shape_of(a.d)) {
    case 0: return launch_from<LAYER, WIDE, 0>(a, st);
    case 1: return launch_from<LAYER, WIDE, 1>(a, st);
    case 2: return launch_from<LAYER, WIDE, 2>(a, st);
    case 3: return launch_from<LAYER, WIDE, 3>(a, st);
    case 4: return launch_from<LAYER, WIDE, 4>(a, st);
    case 5: return launch_from<LAYER, WIDE, 5>(a, st);
    case 6: return launch_from<LAYER, WIDE, 6>(a, st);
    case 7: return launch_from<LAYER, WIDE, 7>(a, st);
    case 8: return launch_from<LAYER, WIDE, 8>(a, st);
    default: return launch_from<LAYER, WIDE, 9>(a, st);
  }
}

cudaError_t launch_join(const NormGradArgs& a, bool layer, int blocks, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  const cudaError_t e = set_shared(norm_join_kernel, 0, done);
  if (e != cudaSuccess) return e;
  return launch_pdl(norm_join_kernel, dim3(static_cast<unsigned>((a.d + 31) / 32), layer ? 2 : 1), dim3(1024), 0, st, a, blocks);
}

int64_t stats_bytes(int64_t n, int64_t d) { return d > kOnePassD ? (n * 8 + 15) / 16 * 16 : 0; }
int64_t grad_bytes(int64_t n, int64_t d) {
  const int64_t blocks = d > kOnePassD ? kSplitRows : blocks_of(n, d);      // (of long rows always all of them)
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
  const bool layer = norm == MLPMOE_LAYERNORM;
  pdl_overlap_enabled() = true;
  if (n_tokens == 0) {
    if (sums && launch_join(a, layer, 0, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
    return MLPMOE_OK;
  }
  if (!s || !grad_out || !grad_x || grad_x == s || grad_x == grad_out) return MLPMOE_ERR_INVALID_ARG;
  if (grad_x == grad_s && (grad_x_dtype != grad_s_dtype || (grad_x_stride != grad_s_stride && n_tokens > 1))) return MLPMOE_ERR_INVALID_ARG;
  if (!on(s, bytes_of(s_dtype)) || !on(grad_out, bytes_of(grad_out_dtype)) || !on(grad_x, bytes_of(grad_x_dtype)) ||
      (grad_s && !on(grad_s, bytes_of(grad_s_dtype))))
    return MLPMOE_ERR_INVALID_ARG;
  // wide: rows in pieces of four elements, of eight above kOnePassD
  const int64_t piece = d_model > kOnePassD ? 8 : 4;
  auto pieces = [&](const void* p, mlpmoe_dtype_t kind, int64_t stride) {
    return stride % piece == 0 && on(p, kind == MLPMOE_FP32 ? 16 : (piece == 8 ? 16 : 8));
  };
  const bool vec = d_model % piece == 0 && pieces(s, s_dtype, s_stride) && pieces(grad_out, grad_out_dtype, grad_out_stride) &&
                   pieces(grad_x, grad_x_dtype, grad_x_stride) && (!grad_s || pieces(grad_s, grad_s_dtype, grad_s_stride)) && on(gain, 16);
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
  if (layer)
    e = vec ? launch_rows<true, true>(a, st) : launch_rows<true, false>(a, st);
  else
    e = vec ? launch_rows<false, true>(a, st) : launch_rows<false, false>(a, st);
  if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  if (!sums) return MLPMOE_OK;
  const int blocks = blocks_of(n_tokens, d_model);
  if (d_model > kOnePassD) {
    e = launch_pdl(norm_column_sums_kernel, dim3(static_cast<unsigned>((d_model + 255) / 256), static_cast<unsigned>(blocks)), dim3(256), 0, st, a,
                   layer ? 1 : 0);
    if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  } else if (blocks == 1) {
    return MLPMOE_OK;
  }
  return launch_join(a, layer, blocks, st) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
