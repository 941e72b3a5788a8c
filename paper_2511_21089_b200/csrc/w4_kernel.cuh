// The layer on 4-bit weights for a few tokens (mlpmoe_w4_forward): one kernel template for both products.
//     gate|up:  h[j, t] = alpha_b silu(sum_k Wg[j, k] x[k, t]) * (sum_k Wu[j, k] x[k, t])
//     down:     y[m, t] = residual + c_t sum_j Wd[m, j] h[j, t]
// with W[r, k] = (code - zero) * scale, one scale and zero per row and group of K.
//
// Bound by HBM: the codes are read once.  Between the copy and the tensor core a code costs about 1.4 integer and
// half-precision operations, which has to stay below the copy's time: a word of eight codes becomes four pairs
// (128 + code) as bf16 with one AND-OR each (the codes slide into the mantissa of 128.0), less (128 + zero), exact in
// bf16; mma.sync then multiplies whole numbers of at most 5 bits with the activations and adds in fp32, and the
// group's scale is applied to the group's sums in fp32.  mma.sync and not tcgen05: the weights would have to go back
// through shared memory as bf16 (four times the bytes) for a product whose time is the copy's anyway.
//
// A warp owns 16 rows (gate|up: the gate and up rows of eight neurons, so that a lane ends with both sums of its
// neurons) and walks K in blocks of 128; warps of a block share rows or K, blocks of a cluster share K (down), and the
// sums are joined in a fixed order.  A pair of codes in a register is (k, k + 4) of eight consecutive k, and the four
// lanes of a row hold different eights: the activations are laid out to match (w4_prepare_kernel and the gate|up
// epilogue), one 16-byte unit for eight consecutive k of one column.
#pragma once
#include <cuda_bf16.h>

#include "ptx.cuh"
#include "w4.h"

namespace mlpmoe {
namespace w4 {

constexpr int kThreads = kW4Warps * 32;
constexpr int kColPitch = 20;          // floats between the 16-row columns of a sum tile: keeps a warp's stores on 32 banks

// Where the unit of k8 (eight consecutive k, 0..15 in a block of 128) stands: word w of lane t of the row's four lanes.
// A group's k have to meet in one mma, so the four lanes together cover one group (GPB groups to a block).
template <int GPB>
__host__ __device__ constexpr int unit_word(int k8) {
  return GPB == 1 ? (k8 & 3) : (GPB == 2 ? 2 * (k8 >> 3) + (k8 & 1) : (k8 >> 2));
}
template <int GPB>
__host__ __device__ constexpr int unit_lane(int k8) {
  return GPB == 1 ? (k8 >> 2) : (GPB == 2 ? ((k8 >> 1) & 3) : (k8 & 3));
}
// Index of the unit of (column, k8) in the fragments of one K-block.
template <int GPB>
__host__ __device__ constexpr int unit_at(int col, int k8) {
  return ((col >> 3) * 4 + unit_word<GPB>(k8)) * 32 + (col & 7) * 4 + unit_lane<GPB>(k8);
}
// Place of element e of a unit: (0, 4), (1, 5), (2, 6), (3, 7).
__host__ __device__ constexpr int unit_pos(int e) { return e < 4 ? 2 * e : 2 * (e - 4) + 1; }

template <int GPB>
__host__ __device__ constexpr int stage_bytes() {   // 16 rows x 64 bytes of codes, then the scales and the zeros of two 8-row halves
  return 1024 + 2 * GPB * 16 + 2 * GPB * 8;
}
constexpr int kStages = 6;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(ok ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Eight codes -> four bf16 pairs code - zero, in the order of unit_pos; bias = (128 + zero) twice.
__device__ __forceinline__ void unpack(uint32_t w, uint32_t bias, uint32_t (&p)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&bias));
    p[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
}

__device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ float ld_cluster_f32(const float* p, uint32_t rank) {
  float v;
  const uint32_t addr = ptx::map_to_cta(ptx::smem_u32(p), rank);
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ int branch_of(const W4Args& a, int neuron) {
  int lo = 0, hi = a.B;                 // off[lo] <= neuron < off[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.off[mid] <= neuron) lo = mid;
    else hi = mid;
  }
  return lo;
}

template <int NT, int GPB>
constexpr int smem_bytes(int sums_floats) {
  const int ring = kW4Warps * kStages * stage_bytes<GPB>();
  const int sums = kW4Warps * NT * 8 * kColPitch * 4 + sums_floats * 4;
  return ring > sums ? ring : sums;
}

// grid: (row tiles / wr, cluster along K, chunks of tokens)
template <int NT, int GPB, bool GATEUP>
__global__ void __launch_bounds__(kThreads) w4_kernel(const __grid_constant__ W4Args a) {
  constexpr int kStage = stage_bytes<GPB>(), kWords = 4 / GPB;
  extern __shared__ __align__(128) uint8_t smem[];
  ptx::griddep_launch_dependents();
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int wk = warp % a.wk, wr = warp / a.wk;
  const int chunk = blockIdx.z;
  const int tile = blockIdx.x * a.wr + wr;
  // The weights do not depend on the kernel before this one (w4_prepare_kernel, or gate|up), only the selection does.
  if (!a.dense) ptx::griddep_wait();
  bool live = tile < a.tiles;
  if (GATEUP && !a.dense && live) live = a.active[branch_of(a, tile * 8)] != 0;
  const int n_list = a.list != nullptr ? a.list[a.kblocks] : a.kblocks;
  const int per = (n_list + gridDim.y - 1) / gridDim.y;
  const int k_begin = blockIdx.y * per + wk, k_end = min(n_list, static_cast<int>(blockIdx.y + 1) * per);
  const int count = live && k_begin < k_end ? (k_end - k_begin + a.wk - 1) / a.wk : 0;

  // copies of one stage: 16 bytes of codes per lane and half, scales and zeros by the first lanes
  const uint8_t* q_src[2];
  bool q_ok[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = (GATEUP ? tile * 8 : tile * 16 + 8 * h) + g;
    q_ok[h] = row < a.rows;
    q_src[h] = a.m[h].q + (q_ok[h] ? row * a.m[h].pitch : 0);
  }
  const int s_half = (lane / GPB) & 1, s_group = lane % GPB;
  const int s_row = GATEUP ? tile * 8 : tile * 16 + 8 * s_half;
  const bool s_ok = lane < 2 * GPB && s_row < a.rows;
  const bool z_ok = s_ok && a.m[s_half].zero != nullptr;
  const uint32_t ring = ptx::smem_u32(smem) + warp * kStages * kStage;
  const uint32_t q_dst = ring + g * 64 + (t ^ ((g >> 1) & 3)) * 16;
  auto block_at = [&](int i) {
    const int at = k_begin + i * a.wk;
    return a.list != nullptr ? a.list[at] : at;
  };
  auto issue = [&](int i, int slot) {
    if (i < count) {
      const int kb = block_at(i);
      const int64_t byte = static_cast<int64_t>(kb) * 64 + t * 16;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bool ok = q_ok[h] && byte < a.m[h].pitch;
        cp_async16(q_dst + slot * kStage + h * 512, ok ? q_src[h] + byte : a.m[h].q, ok);
      }
      if (lane < 2 * GPB) {
        const int64_t group = static_cast<int64_t>(kb) * GPB + s_group;
        const bool in = group < a.m[s_half].n_groups;
        const int64_t at = s_ok && in ? group * a.m[s_half].rows16 + s_row : 0;
        cp_async16(ring + slot * kStage + 1024 + lane * 16, a.m[s_half].scale + at, s_ok && in);
        if (a.m[s_half].zero != nullptr) cp_async8(ring + slot * kStage + 1024 + 2 * GPB * 16 + lane * 8, a.m[s_half].zero + at, z_ok && in);
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) issue(i, i);
  if (a.dense) ptx::griddep_wait();

  // columns 8 nt + g: the lanes of a column that stands for no token keep zeros
  bool col_ok[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = nt * 8 + g;
    col_ok[nt] = c < a.c.pieces * a.c.tokens && chunk * a.c.tokens + c % a.c.tokens < a.n;
  }
  float acc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[nt][i] = 0.0f;
  const uint4* frag = a.frag + static_cast<int64_t>(chunk) * a.kblocks * (NT * 128) + lane;
  const bool scaled = GATEUP && a.x_scale != nullptr && a.x_groups > 1;

  int slot = 0;
  for (int i = 0; i < count; ++i) {
    const int kb = block_at(i);
    const uint4* xp = frag + static_cast<int64_t>(kb) * (NT * 128);
    uint4 xb[NT <= 2 ? NT : 1][4];
    if (NT <= 2) {
#pragma unroll
      for (int nt = 0; nt < (NT <= 2 ? NT : 1); ++nt)
#pragma unroll
        for (int w = 0; w < 4; ++w) xb[nt][w] = col_ok[nt] ? xp[(nt * 4 + w) * 32] : make_uint4(0u, 0u, 0u, 0u);
    }
    cp_async_wait<kStages - 2>();
    __syncwarp();                       // the stage is in shared memory for all lanes, and the slot before it has been read by all
    const uint8_t* st = smem + (warp * kStages + slot) * kStage;
    issue(i + kStages - 1, slot == 0 ? kStages - 1 : slot - 1);
#pragma unroll
    for (int j = 0; j < GPB; ++j) {
      float part[NT][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) part[nt][e] = 0.0f;
      uint32_t q[2][kWords], bias[2];
      float s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // the group's words of this lane: 16 bytes of chunk t (one group per block), 8 bytes, or 4
        const int sw = (g >> 1) & 3;
        const uint8_t* row = st + h * 512 + g * 64;
        if (GPB == 1) {
          const uint4 v = *reinterpret_cast<const uint4*>(row + ((t ^ sw) * 16));
          q[h][0] = v.x, q[h][1 % kWords] = v.y, q[h][2 % kWords] = v.z, q[h][3 % kWords] = v.w;
        } else if (GPB == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(row + (((2 * j + (t >> 1)) ^ sw) * 16) + (t & 1) * 8);
          q[h][0] = v.x, q[h][1 % kWords] = v.y;
        } else {
          q[h][0] = *reinterpret_cast<const uint32_t*>(row + ((j ^ sw) * 16) + t * 4);
        }
        const int piece = h * GPB + j;
        s[h] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(st + 1024 + piece * 16 + g * 2));
        const uint32_t z = a.m[h].zero != nullptr ? st[1024 + 2 * GPB * 16 + piece * 8 + g] : 8u;
        bias[h] = 0x43004300u | z | (z << 16);
      }
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        uint32_t lo[4], hi[4];
        unpack(q[0][w], bias[0], lo);
        unpack(q[1][w], bias[1], hi);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint4 b;
          if (NT <= 2) b = xb[nt < 2 ? nt : 0][j * kWords + w];
          else b = col_ok[nt] ? xp[(nt * 4 + j * kWords + w) * 32] : make_uint4(0u, 0u, 0u, 0u);
          mma(part[nt], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
          mma(part[nt], lo[2], hi[2], lo[3], hi[3], b.z, b.w);
        }
      }
      if (scaled) {
        const int xg = (kb * GPB + j) >> a.x_shift;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int c = nt * 8 + 2 * t + e, token = chunk * a.c.tokens + c;
            const float sx = c < a.c.tokens && token < a.n && xg < a.x_groups ? a.x_scale[static_cast<int64_t>(token) * a.x_groups + xg] : 0.0f;
            acc[nt][e] += part[nt][e] * (s[0] * sx);
            acc[nt][2 + e] += part[nt][2 + e] * (s[1] * sx);
          }
        }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          acc[nt][0] += part[nt][0] * s[0];
          acc[nt][1] += part[nt][1] * s[0];
          acc[nt][2] += part[nt][2] * s[1];
          acc[nt][3] += part[nt][3] * s[1];
        }
      }
    }
    slot = slot + 1 == kStages ? 0 : slot + 1;
  }
  cp_async_wait<0>();
  __syncthreads();                      // the ring becomes the sums: [wk][tile of the block][column][16 rows]
  float* sums = reinterpret_cast<float*>(smem);
  const int tiles_here = a.wr;
  {
    float* p = sums + (wk * tiles_here + wr) * (NT * 8 * kColPitch) + (2 * t) * kColPitch + g;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float* c = p + nt * 8 * kColPitch;
      c[0] = acc[nt][0];
      c[kColPitch] = acc[nt][1];
      c[8] = acc[nt][2];
      c[kColPitch + 8] = acc[nt][3];
    }
  }
  __syncthreads();
  const int tokens = a.c.tokens, pieces = a.c.pieces;
  auto sum_of = [&](int tl, int tok, int row) {
    float v = 0.0f;
    for (int k = 0; k < a.wk; ++k) {
      const float* p = sums + (k * tiles_here + tl) * (NT * 8 * kColPitch) + row;
      for (int c = tok; c < pieces * tokens; c += tokens) v += p[c * kColPitch];
    }
    return v;
  };
  if (GATEUP) {
    for (int i = threadIdx.x; i < tiles_here * tokens * 8; i += kThreads) {
      const int e = i & 7, tok = (i >> 3) % tokens, tl = (i >> 3) / tokens;
      const int tile_e = blockIdx.x * a.wr + tl, token = chunk * tokens + tok;
      if (tile_e >= a.tiles || token >= a.n) continue;
      const int neuron = tile_e * 8 + e, b = branch_of(a, neuron);
      bool on = true;
      if (!a.dense) on = a.active[b] != 0 && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
      float h = 0.0f;
      if (on) {
        float gate = sum_of(tl, tok, e), up = sum_of(tl, tok, 8 + e);
        if (a.x_scale != nullptr && a.x_groups == 1) {
          gate *= a.x_scale[token];
          up *= a.x_scale[token];
        }
        h = gate / (1.0f + expf(-gate)) * up * a.alpha[b];
      }
      // h as bf16 pieces: two keep 2^-17 of it (y is rounded to 2^-9), three all 24 bits
      const int h_chunk = token / a.hc.tokens, h_tok = token % a.hc.tokens;
      __nv_bfloat16* out = a.h_frag + ((static_cast<int64_t>(h_chunk) * a.h_kblocks + neuron / 128) * a.hc.nt) * (128 * 8) + unit_pos(e);
      for (int p = 0; p < a.hc.pieces; ++p) {
        const __nv_bfloat16 piece = __float2bfloat16_rn(h);
        h -= __bfloat162float(piece);
        out[unit_at<GPB>(p * a.hc.tokens + h_tok, (neuron % 128) / 8) * 8] = piece;
      }
    }
  } else {
    auto finish = [&](int tl, int tok, int row, float v) {
      const int m = (blockIdx.x * a.wr + tl) * 16 + row, token = chunk * tokens + tok;
      if (m >= a.rows || token >= a.n) return;
      const int64_t at = static_cast<int64_t>(token) * a.d + m;
      if (a.coef != nullptr) v *= a.coef[token];
      if (a.residual != nullptr) v += a.residual[at];
      if (a.y_bf16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
      else static_cast<float*>(a.y)[at] = v;
    };
    const int total = tiles_here * tokens * 16;
    if (gridDim.y == 1) {
      for (int i = threadIdx.x; i < total; i += kThreads) {
        const int row = i & 15, tok = (i >> 4) % tokens, tl = (i >> 4) / tokens;
        finish(tl, tok, row, sum_of(tl, tok, row));
      }
    } else {
      float* own = sums + kW4Warps * (NT * 8 * kColPitch);
      for (int i = threadIdx.x; i < total; i += kThreads) own[i] = sum_of((i >> 4) / tokens, (i >> 4) % tokens, i & 15);
      __syncthreads();
      ptx::cluster_sync_all();
      for (int i = blockIdx.y * kThreads + threadIdx.x; i < total; i += gridDim.y * kThreads) {
        float v = 0.0f;
        for (uint32_t r = 0; r < gridDim.y; ++r) v += ld_cluster_f32(own + i, r);
        finish((i >> 4) / tokens, (i >> 4) % tokens, i & 15, v);
      }
      __syncthreads();
      ptx::cluster_sync_all();          // no block leaves while another reads its sums
    }
  }
}

template <int NT, int GPB, bool GATEUP>
cudaError_t launch(const W4Args& a, int cluster, cudaStream_t st) {
  auto kernel = w4_kernel<NT, GPB, GATEUP>;
  const int smem = smem_bytes<NT, GPB>(GATEUP ? 0 : a.wr * a.c.tokens * 16);
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.tiles + a.wr - 1) / a.wr), static_cast<unsigned>(cluster), static_cast<unsigned>(a.c.chunks));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = static_cast<size_t>(smem);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 1;
  attr[1].val.clusterDim.y = static_cast<unsigned>(cluster);
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <int GPB, bool GATEUP>
cudaError_t launch_nt(const W4Args& a, int cluster, cudaStream_t st) {
  switch (a.c.nt) {
    case 1: return launch<1, GPB, GATEUP>(a, cluster, st);
    case 2: return launch<2, GPB, GATEUP>(a, cluster, st);
    case 3: return launch<3, GPB, GATEUP>(a, cluster, st);
    case 4: return launch<4, GPB, GATEUP>(a, cluster, st);
    case 6: return launch<6, GPB, GATEUP>(a, cluster, st);
    case 8: return launch<8, GPB, GATEUP>(a, cluster, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace w4
}  // namespace mlpmoe
