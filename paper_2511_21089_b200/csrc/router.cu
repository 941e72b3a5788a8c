// The router's selection, its balance loss and the loss's gradient (mlpmoe_route, mlpmoe_route_backward).
//     p[t, :] = softmax of the eligible logits;  S_t = the k largest;  counts[b], prob[b] = mean of p[:, b];
//     loss = B' sum_b f_b prob[b];   d loss / d logit[t, j] = B' / T p[t, j] (f_j - sum_b f_b p[t, b]).
// One pass over the logits each way.  A row belongs to LPR lanes of a warp with VPT neighbouring columns each, so a
// lane's columns never change and the column sums live in its registers until the kernel's end.  Forward: bound by the
// k exchanges of the selection (131072 x 128, top 16: 59 us and 10 for the sums, 75 % of the issue slots, where the logits alone
// take 13; a row has all 32 lanes there, so its k exchanges are the whole warp's).  Backward: 131072 x 128 fp32 34 us, 62 % of a copy; 30
// instructions per logit keep it from the rest, of them the sums over a row's lanes, paid for four columns a lane.
// B above 128 (eight columns a lane) spills 88 bytes a thread in the forward: 131072 x 256, top 16: 115 us.
#include <math.h>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"

namespace mlpmoe {
namespace {

constexpr int kMaxB = 256;
constexpr int kRouteThreads = 1024;    // forward: one block per SM, so that few sums are left to join
constexpr int kRouteWarps = kRouteThreads / 32;
constexpr int kRouteCtas = 148;
constexpr int kRouteRows = 2;          // rows of a segment at a time: two chains of exchanges in flight
constexpr int kBackwardThreads = 256;
constexpr int kBackwardCtas = 148 * 6;   // all resident
constexpr int kBackwardRows = 2;

// One block's contribution: B probability sums, then B counts and the number of routed tokens as int32.
__host__ __device__ inline int64_t partial_words(int B) { return 2 * B + 1; }

struct RouteArgs {
  const void* logits;
  const uint8_t* avail;
  const uint8_t* valid;
  int64_t stride, n;
  int B, k;
  uint8_t* select;
  uint32_t* partial;     // [gridDim.x][2 B + 1]
  int32_t* counts;
  float* prob;
  float* loss;
  // backward
  const int32_t* counts_in;
  const float* grad_loss;
  void* grad;
  int64_t grad_stride;
};

template <int W>
__device__ __forceinline__ float seg_max(float v) {
  if constexpr (W == 32) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(v));
    return r;
  } else {
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
  }
}
template <int W>
__device__ __forceinline__ float seg_sum(float v) {
#pragma unroll
  for (int o = W / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}
// The row's values of one lane; places that are not eligible become -infinity, +infinity the largest finite value.
template <typename T, int VPT, bool VEC>
__device__ __forceinline__ void load_row(const T* row, int c0, int B, uint32_t avail_mask, bool live, float (&x)[VPT]) {
#pragma unroll
  for (int i = 0; i < VPT; ++i) x[i] = -INFINITY;
  if (!live) return;
  if (VEC) {                                       // B % 4 == 0 and rows on 16 (fp32) or 8 (bf16) bytes
#pragma unroll
    for (int i = 0; i < VPT; i += 4) {
      if (c0 + i >= B) continue;
      if (sizeof(T) == 4) {
        const float4 v = *reinterpret_cast<const float4*>(row + c0 + i);
        x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(row + c0 + i);
        x[i] = __uint_as_float(v.x << 16), x[i + 1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[i + 2] = __uint_as_float(v.y << 16), x[i + 3] = __uint_as_float(v.y & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      if (c0 + i < B) x[i] = static_cast<float>(row[c0 + i]);
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    const bool ok = ((avail_mask >> i) & 1u) && x[i] > -INFINITY;   // false for a NaN
    x[i] = ok ? fminf(x[i], 3.402823466e38f) : -INFINITY;
  }
}

template <int VPT>
__device__ __forceinline__ uint32_t avail_mask_of(const uint8_t* avail, int c0, int B) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (c0 + i < B && (avail == nullptr || avail[c0 + i] != 0)) m |= 1u << i;
  return m;
}

// Descending.
template <int VPT>
__device__ __forceinline__ void sort_down(float (&s)[VPT]) {
  auto order = [&](int i, int j) {
    const float hi = fmaxf(s[i], s[j]);
    s[j] = fminf(s[i], s[j]);
    s[i] = hi;
  };
  // odd-even merge networks of 4 and of 8 (Batcher)
  order(0, 1), order(2, 3), order(0, 2), order(1, 3), order(1, 2);
  if constexpr (VPT == 8) {
    order(4, 5), order(6, 7), order(4, 6), order(5, 7), order(5, 6);
    order(0, 4), order(1, 5), order(2, 6), order(3, 7), order(2, 4), order(3, 5), order(1, 2), order(3, 4), order(5, 6);
  }
}

// What is left once the sums of a column over all tokens are in s_prob[b], s_count[b] and the routed tokens in *s_routed: the outputs.
__device__ void route_outputs(const RouteArgs& a, const float* s_prob, const int* s_count, const int* s_routed) {
  const int routed = *s_routed;
  if (threadIdx.x < 32) {
    double dot = 0.0;
    int64_t total = 0;
    int n_avail = 0;
    for (int b = threadIdx.x; b < a.B; b += 32) {
      dot += static_cast<double>(s_count[b]) * static_cast<double>(s_prob[b]);
      total += s_count[b];
      n_avail += a.avail == nullptr || a.avail[b] != 0 ? 1 : 0;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
      total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
      n_avail += __shfl_xor_sync(0xFFFFFFFFu, n_avail, o);
    }
    if (threadIdx.x == 0) {
      a.loss[0] = total > 0 ? static_cast<float>(n_avail * dot / (static_cast<double>(total) * routed)) : 0.0f;
      a.counts[a.B] = routed;
    }
  }
  for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
    a.counts[b] = s_count[b];
    a.prob[b] = routed > 0 ? s_prob[b] / static_cast<float>(routed) : 0.0f;
  }
}

// A block's rows.  Of the k largest, each lane offers the largest of its columns that is not taken yet (they are sorted
// once); every lane that holds the row's largest takes it, until k are taken; that gives the smallest value taken, and
// the selection is what lies above it and, of equals, the first in index order.
template <typename T, int LPR, int VPT, bool VEC>
__global__ void __launch_bounds__(kRouteThreads) route_kernel(const __grid_constant__ RouteArgs a) {
  constexpr int kSegs = 32 / LPR, kCols = LPR * VPT, R = kRouteRows;
  __shared__ float s_prob[kRouteWarps * kCols];     // per warp and column: probabilities, then counts
  __shared__ int s_count[kMaxB];
  __shared__ int s_routed[kRouteWarps];
  ptx::griddep_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int seg = lane / LPR, l = lane % LPR, c0 = l * VPT;
  const uint32_t avail_mask = avail_mask_of<VPT>(a.avail, c0, a.B);
  const uint32_t seg_lanes = (LPR == 32 ? 0xFFFFFFFFu : ((1u << (LPR % 32)) - 1u)) << (seg * LPR);
  const bool byte_vec = a.B % 4 == 0 && reinterpret_cast<uintptr_t>(a.select) % 4 == 0;
  float prob[VPT];
  int count[VPT], routed = 0;
#pragma unroll
  for (int i = 0; i < VPT; ++i) prob[i] = 0.0f, count[i] = 0;

  const int64_t step = static_cast<int64_t>(gridDim.x) * kRouteWarps * kSegs * R;
  for (int64_t base = (static_cast<int64_t>(blockIdx.x) * kRouteWarps + warp) * kSegs * R; base < a.n; base += step) {
    float x[R][VPT], s[R][VPT], least[R];
    int taken[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = base + r * kSegs + seg;
      const bool live = t < a.n && (a.valid == nullptr || a.valid[t] != 0);
      load_row<T, VPT, VEC>(static_cast<const T*>(a.logits) + (t < a.n ? t : 0) * a.stride, c0, a.B, avail_mask, live, x[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      // softmax; a place that is not eligible holds -infinity and gets exp(-infinity) = 0
#pragma unroll
      for (int i = 0; i < VPT; ++i) s[r][i] = x[r][i];
      sort_down(s[r]);
      const float m = seg_max<LPR>(s[r][0]);
      const bool any = m > -INFINITY;
      const float top = any ? m : 0.0f;
      float e[VPT], sum = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        e[i] = expf(x[r][i] - top);
        sum += e[i];
      }
      sum = seg_sum<LPR>(sum);
      const float inv = any ? 1.0f / sum : 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) prob[i] += e[i] * inv;
      routed += any && l == 0 ? 1 : 0;
      taken[r] = 0;
      least[r] = INFINITY;
    }
    // k turns always: a row that has its k earlier, or nothing left (every lane then offers -infinity), only goes on
    // without effect
    for (int turn = 0; turn < a.k; ++turn) {
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const float top = seg_max<LPR>(s[r][0]);
        const bool hit = s[r][0] == top;
        const uint32_t who = __ballot_sync(0xFFFFFFFFu, hit) & seg_lanes;
        if (taken[r] < a.k) least[r] = top;
        taken[r] += __popc(who);
        if (hit) {
#pragma unroll
          for (int i = 0; i + 1 < VPT; ++i) s[r][i] = s[r][i + 1];
          s[r][VPT - 1] = -INFINITY;
        }
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      uint32_t above = 0, equal = 0;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        above |= x[r][i] > least[r] ? 1u << i : 0u;
        equal |= x[r][i] == least[r] && x[r][i] > -INFINITY ? 1u << i : 0u;
      }
      // equals: as many as are wanted, the first in index order (columns ascend with the lane)
      int n_above = __popc(above), n_equal = __popc(equal);
      const int mine = n_equal;
      if constexpr (LPR == 32) {
        n_above = __reduce_add_sync(0xFFFFFFFFu, n_above);
        n_equal = __reduce_add_sync(0xFFFFFFFFu, n_equal);
      } else {
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1) {
          n_above += __shfl_xor_sync(0xFFFFFFFFu, n_above, o);
          n_equal += __shfl_xor_sync(0xFFFFFFFFu, n_equal, o);
        }
      }
      if (__any_sync(0xFFFFFFFFu, n_above + n_equal > a.k)) {
        int before = mine;
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) {
          const int u = __shfl_up_sync(0xFFFFFFFFu, before, o, LPR);
          if (l >= o) before += u;
        }
        int room = a.k - n_above - (before - mine);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
          if ((equal >> i) & 1u) {
            if (room <= 0) equal &= ~(1u << i);
            --room;
          }
        }
      }
      const uint32_t chosen = above | equal;
#pragma unroll
      for (int i = 0; i < VPT; ++i) count[i] += (chosen >> i) & 1u;
      const int64_t t = base + r * kSegs + seg;
      if (t < a.n) {
        uint8_t* out = a.select + t * a.B + c0;
        if (byte_vec) {
#pragma unroll
          for (int i = 0; i < VPT; i += 4) {
            const uint32_t b = chosen >> i;
            if (c0 + i < a.B)
              *reinterpret_cast<uint32_t*>(out + i) = (b & 1u) | ((b & 2u) << 7) | ((b & 4u) << 14) | ((b & 8u) << 21);
          }
        } else {
#pragma unroll
          for (int i = 0; i < VPT; ++i)
            if (c0 + i < a.B) out[i] = (chosen >> i) & 1u;
        }
      }
    }
  }

  // the warp's rows, then the block's in the order of its warps
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
#pragma unroll
    for (int o = 16; o >= LPR; o >>= 1) {
      prob[i] += __shfl_xor_sync(0xFFFFFFFFu, prob[i], o);
      count[i] += __shfl_xor_sync(0xFFFFFFFFu, count[i], o);
    }
    if (seg == 0) s_prob[warp * kCols + c0 + i] = prob[i];
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) routed += __shfl_xor_sync(0xFFFFFFFFu, routed, o);
  if (lane == 0) s_routed[warp] = routed;
  __syncthreads();
  float p = 0.0f;
  const int b = threadIdx.x;
  if (b < a.B)
    for (int w = 0; w < kRouteWarps; ++w) p += s_prob[w * kCols + b];
  __syncthreads();
  int* s_warp_count = reinterpret_cast<int*>(s_prob);
  if (seg == 0) {
#pragma unroll
    for (int i = 0; i < VPT; ++i) s_warp_count[warp * kCols + c0 + i] = count[i];
  }
  __syncthreads();
  int c = 0;
  if (b < a.B)
    for (int w = 0; w < kRouteWarps; ++w) c += s_warp_count[w * kCols + b];
  if (threadIdx.x == 0)
    for (int w = 1; w < kRouteWarps; ++w) s_routed[0] += s_routed[w];
  __syncthreads();
  if (gridDim.x == 1) {
    if (b < a.B) s_prob[b] = p, s_count[b] = c;
    __syncthreads();
    route_outputs(a, s_prob, s_count, s_routed);
  } else {
    uint32_t* out = a.partial + static_cast<int64_t>(blockIdx.x) * partial_words(a.B);
    if (b < a.B) {
      out[b] = __float_as_uint(p);
      out[a.B + b] = static_cast<uint32_t>(c);
    }
    if (threadIdx.x == 0) out[2 * a.B] = static_cast<uint32_t>(s_routed[0]);
  }
}

// Adds the blocks' contributions in a fixed order: thread (part, b) takes every parts-th block's sums of column b.
__global__ void __launch_bounds__(kRouteThreads) route_finish_kernel(const __grid_constant__ RouteArgs a, int n_partial) {
  __shared__ float s_prob[kRouteThreads];
  __shared__ int s_count[kRouteThreads];
  __shared__ int s_routed;
  ptx::griddep_wait();
  const int words = static_cast<int>(partial_words(a.B));
  int cols = 8;
  while (cols < a.B) cols *= 2;
  const int parts = kRouteThreads / cols, b = threadIdx.x % cols, part = threadIdx.x / cols;
  float p = 0.0f;
  int c = 0;
  if (b < a.B) {
#pragma unroll 8
    for (int i = part; i < n_partial; i += parts) {
      p += __uint_as_float(a.partial[i * words + b]);
      c += static_cast<int>(a.partial[i * words + a.B + b]);
    }
  }
  s_prob[threadIdx.x] = p;
  s_count[threadIdx.x] = c;
  __syncthreads();
  if (threadIdx.x < 32) {
    int routed = 0;
    for (int i = threadIdx.x; i < n_partial; i += 32) routed += static_cast<int>(a.partial[i * words + 2 * a.B]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) routed += __shfl_xor_sync(0xFFFFFFFFu, routed, o);
    if (threadIdx.x == 0) s_routed = routed;
  }
  if (part == 0 && b < a.B) {
    p = 0.0f;
    c = 0;
    for (int i = 0; i < parts; ++i) {
      p += s_prob[i * cols + b];
      c += s_count[i * cols + b];
    }
  }
  __syncthreads();
  if (part == 0 && b < a.B) s_prob[b] = p, s_count[b] = c;
  __syncthreads();
  route_outputs(a, s_prob, s_count, &s_routed);
}

// f is taken less the mean count, which changes nothing where the probabilities sum to 1 and keeps the difference exact
// where the load is nearly even (all counts equal: the gradient is 0).
template <typename T, int LPR, int VPT, bool VEC>
__global__ void __launch_bounds__(kBackwardThreads, VPT == 4 ? 6 : 4) route_backward_kernel(const __grid_constant__ RouteArgs a) {
  constexpr int kWarps = kBackwardThreads / 32, kSegs = 32 / LPR, R = kBackwardRows;
  ptx::griddep_wait();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int seg = lane / LPR, l = lane % LPR, c0 = l * VPT;
  const uint32_t avail_mask = avail_mask_of<VPT>(a.avail, c0, a.B);
  int64_t total = 0;                    // up to n_tokens * top_k: past 32 bits
  int n_avail = __popc(avail_mask), cnt[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    cnt[i] = c0 + i < a.B ? a.counts_in[c0 + i] : 0;
    total += cnt[i];
  }
#pragma unroll
  for (int o = LPR / 2; o > 0; o >>= 1) {
    total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    n_avail += __shfl_xor_sync(0xFFFFFFFFu, n_avail, o);
  }
  const int routed = a.counts_in[a.B], mean = n_avail > 0 ? static_cast<int>(total / n_avail) : 0;
  float f[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i) f[i] = total > 0 ? static_cast<float>(cnt[i] - mean) / static_cast<float>(total) : 0.0f;
  const float g = a.grad_loss != nullptr ? a.grad_loss[0] : 1.0f;
  const float scale = routed > 0 ? g * static_cast<float>(n_avail) / static_cast<float>(routed) : 0.0f;

  const int64_t step = static_cast<int64_t>(gridDim.x) * kWarps * kSegs * R;
  for (int64_t base = (static_cast<int64_t>(blockIdx.x) * kWarps + warp) * kSegs * R; base < a.n; base += step) {
    float x[R][VPT];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t t = base + r * kSegs + seg;
      const bool live = t < a.n && (a.valid == nullptr || a.valid[t] != 0);
      load_row<T, VPT, VEC>(static_cast<const T*>(a.logits) + (t < a.n ? t : 0) * a.stride, c0, a.B, avail_mask, live, x[r]);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float m = x[r][0];
#pragma unroll
      for (int i = 1; i < VPT; ++i) m = fmaxf(m, x[r][i]);
      m = seg_max<LPR>(m);
      const bool any = m > -INFINITY;
      const float top = any ? m : 0.0f;
      float sum = 0.0f, dot = 0.0f;
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        x[r][i] = expf(x[r][i] - top);
        sum += x[r][i];
        dot += x[r][i] * f[i];
      }
      sum = seg_sum<LPR>(sum);
      dot = seg_sum<LPR>(dot);
      const float inv = any ? 1.0f / sum : 0.0f;
      const float mean_f = dot * inv, c = scale * inv;
      const int64_t t = base + r * kSegs + seg;
      if (t >= a.n) continue;
      T* out = static_cast<T*>(a.grad) + t * a.grad_stride + c0;
#pragma unroll
      for (int i = 0; i < VPT; ++i) x[r][i] = c * x[r][i] * (f[i] - mean_f);
      if (VEC) {
#pragma unroll
        for (int i = 0; i < VPT; i += 4) {
          if (c0 + i >= a.B) continue;
          if (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(out + i) = make_float4(x[r][i], x[r][i + 1], x[r][i + 2], x[r][i + 3]);
          } else {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(x[r][i], x[r][i + 1]), hi = __floats2bfloat162_rn(x[r][i + 2], x[r][i + 3]);
            *reinterpret_cast<uint2*>(out + i) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < VPT; ++i)
          if (c0 + i < a.B) out[i] = static_cast<T>(x[r][i]);
      }
    }
  }
}

enum Op { FORWARD, BACKWARD };

// Lanes of a row: the narrowest power of two that holds B columns, four to a lane (eight above 128).
int lanes_per_row(int B) {
  int lanes = 2;
  while (lanes < 32 && lanes * 4 < B) lanes *= 2;
  return lanes;
}

// Blocks of the forward: one where its warps need one turn only (the sums need no second launch then; 64 x 32, top 4: 4.0 us).
// For two turns it is slower than two blocks and that launch (512 x 32: 8.7 against 7.4 us; 256 x 128, top 8: 15.2 against 7.7).
int forward_blocks(int64_t n, int B) {
  const int64_t rows = 32 / lanes_per_row(B) * kRouteRows * kRouteWarps;
  const int64_t need = (n + rows - 1) / rows;
  return need <= 1 ? 1 : static_cast<int>(need < kRouteCtas ? need : kRouteCtas);
}
int backward_blocks(int64_t n, int B) {
  const int64_t rows = 32 / lanes_per_row(B) * kBackwardRows * (kBackwardThreads / 32);
  const int64_t need = (n + rows - 1) / rows;
  return static_cast<int>(need < kBackwardCtas ? need : kBackwardCtas);
}

template <typename T, int LPR, int VPT, bool VEC>
cudaError_t launch_op(Op op, const RouteArgs& a, cudaStream_t st) {
  if (op == FORWARD)
    return launch_pdl(route_kernel<T, LPR, VPT, VEC>, dim3(static_cast<unsigned>(forward_blocks(a.n, a.B))), dim3(kRouteThreads), 0, st, a);
  return launch_pdl(route_backward_kernel<T, LPR, VPT, VEC>, dim3(static_cast<unsigned>(backward_blocks(a.n, a.B))), dim3(kBackwardThreads),
                    0, st, a);
}

template <typename T, bool VEC>
cudaError_t launch_width(Op op, const RouteArgs& a, cudaStream_t st) {
  switch (lanes_per_row(a.B)) {
    case 2: return launch_op<T, 2, 4, VEC>(op, a, st);
    case 4: return launch_op<T, 4, 4, VEC>(op, a, st);
    case 8: return launch_op<T, 8, 4, VEC>(op, a, st);
    case 16: return launch_op<T, 16, 4, VEC>(op, a, st);
    default: return a.B <= 128 ? launch_op<T, 32, 4, VEC>(op, a, st) : launch_op<T, 32, 8, VEC>(op, a, st);
  }
}

cudaError_t launch_any(Op op, const RouteArgs& a, mlpmoe_dtype_t dtype, cudaStream_t st) {
  const uintptr_t word = dtype == MLPMOE_FP32 ? 16 : 8;
  bool vec = a.B % 4 == 0 && a.stride % 4 == 0 && reinterpret_cast<uintptr_t>(a.logits) % word == 0;
  if (op == BACKWARD) vec = vec && a.grad_stride % 4 == 0 && reinterpret_cast<uintptr_t>(a.grad) % word == 0;
  if (dtype == MLPMOE_FP32) return vec ? launch_width<float, true>(op, a, st) : launch_width<float, false>(op, a, st);
  return vec ? launch_width<__nv_bfloat16, true>(op, a, st) : launch_width<__nv_bfloat16, false>(op, a, st);
}

mlpmoe_status_t check_router(const void* logits, mlpmoe_dtype_t dtype, int64_t* stride, int64_t n, int32_t B) {
  if (n < 0 || n > INT32_MAX || B <= 0) return MLPMOE_ERR_INVALID_ARG;
  if (dtype != MLPMOE_FP32 && dtype != MLPMOE_BF16) return MLPMOE_ERR_INVALID_ARG;
  if (B > kMaxB) return MLPMOE_ERR_UNSUPPORTED;
  if (*stride == 0) *stride = B;
  if (*stride < B) return MLPMOE_ERR_INVALID_ARG;
  if (n > 0 && (!logits || reinterpret_cast<uintptr_t>(logits) % (dtype == MLPMOE_FP32 ? 4 : 2) != 0)) return MLPMOE_ERR_INVALID_ARG;
  return MLPMOE_OK;
}

inline bool on4(const void* p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" {

mlpmoe_status_t mlpmoe_route_workspace(int64_t n_tokens, int32_t B, int64_t* bytes) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || B <= 0 || !bytes) return MLPMOE_ERR_INVALID_ARG;
  if (B > kMaxB) return MLPMOE_ERR_UNSUPPORTED;
  *bytes = (kRouteCtas * partial_words(B) * 4 + 15) / 16 * 16;
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_route(const void* logits, mlpmoe_dtype_t dtype, int64_t stride, int64_t n_tokens, int32_t B, int32_t top_k,
                             const uint8_t* avail, const uint8_t* valid, uint8_t* select, int32_t* counts, float* prob, float* loss,
                             void* workspace, int64_t workspace_bytes, void* stream) {
  mlpmoe_status_t rc = check_router(logits, dtype, &stride, n_tokens, B);
  if (rc != MLPMOE_OK) return rc;
  if (top_k < 1 || top_k > B) return MLPMOE_ERR_INVALID_ARG;
  if (!counts || !prob || !loss || !on4(counts) || !on4(prob) || !on4(loss) || (n_tokens > 0 && !select)) return MLPMOE_ERR_INVALID_ARG;
  int64_t need = 0;
  mlpmoe_route_workspace(n_tokens, B, &need);
  if (!workspace || workspace_bytes < need || reinterpret_cast<uintptr_t>(workspace) % 16 != 0) return MLPMOE_ERR_INVALID_ARG;
  RouteArgs a = {};
  a.logits = logits;
  a.avail = avail;
  a.valid = valid;
  a.stride = stride;
  a.n = n_tokens;
  a.B = B;
  a.k = top_k;
  a.select = select;
  a.partial = static_cast<uint32_t*>(workspace);
  a.counts = counts;
  a.prob = prob;
  a.loss = loss;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  pdl_overlap_enabled() = true;
  int n_partial = 0;
  if (n_tokens > 0) {
    n_partial = forward_blocks(n_tokens, B);
    if (launch_any(FORWARD, a, dtype, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  }
  if (n_partial != 1 && launch_pdl(route_finish_kernel, dim3(1), dim3(kRouteThreads), 0, st, a, n_partial) != cudaSuccess)
    return MLPMOE_ERR_CUDA;
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_route_backward(const void* logits, mlpmoe_dtype_t dtype, int64_t stride, int64_t n_tokens, int32_t B,
                                      const uint8_t* avail, const uint8_t* valid, const int32_t* counts, const float* grad_loss,
                                      void* grad, int64_t grad_stride, void* stream) {
  mlpmoe_status_t rc = check_router(logits, dtype, &stride, n_tokens, B);
  if (rc != MLPMOE_OK) return rc;
  if (grad_stride == 0) grad_stride = B;
  if (grad_stride < B) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens == 0) return MLPMOE_OK;
  if (!counts || !grad || !on4(counts) || !on4(grad_loss)) return MLPMOE_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(grad) % (dtype == MLPMOE_FP32 ? 4 : 2) != 0) return MLPMOE_ERR_INVALID_ARG;
  if (grad == logits && grad_stride != stride && n_tokens > 1) return MLPMOE_ERR_INVALID_ARG;
  RouteArgs a = {};
  a.logits = logits;
  a.avail = avail;
  a.valid = valid;
  a.stride = stride;
  a.n = n_tokens;
  a.B = B;
  a.counts_in = counts;
  a.grad_loss = grad_loss;
  a.grad = grad;
  a.grad_stride = grad_stride;
  pdl_overlap_enabled() = true;
  return launch_any(BACKWARD, a, dtype, static_cast<cudaStream_t>(stream)) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
