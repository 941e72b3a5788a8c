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
// One block per SM takes an equal share of the 16-row tiles (gate|up: the gate and up rows of eight neurons, so that a
// lane ends with both sums of its neurons).  Its steps, (tile, 256 columns of K), are dealt to the 16 warps in equal
// runs; a run may end inside a tile, and the parts of a tile are joined in warp order, so the result is the same
// on every call.  Blocks of a cluster share K where the activations of all of K would not fit in shared memory, or
// where there are few rows.  Every warp keeps its own ring of stages filled by cp.async: no barrier in the loop.
//
// A pair of codes in a register is (k, k + 4) of eight consecutive k, and the four lanes of a row hold different
// eights: the activations stand in shared memory to match, one 16-byte unit for eight consecutive k of one column.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "../../include/mlpmoe.h"
#include "ptx.cuh"
#include "w4.h"

namespace mlpmoe {
namespace w4 {

constexpr int kWarps = 16;
constexpr int kThreads = kWarps * 32;
constexpr int kColPitch = 20;          // floats between the 16-row columns of a sum tile: keeps a warp's stores on 32 banks
constexpr int kSmemMax = 226 * 1024;  // dynamic; the rest of the 227 KB is for the small static arrays

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
// The inverse: k8 of (word, lane).
template <int GPB>
__host__ __device__ constexpr int unit_k8(int w, int t) {
  return GPB == 1 ? 4 * t + w : (GPB == 2 ? 8 * (w >> 1) + 2 * t + (w & 1) : 4 * w + t);
}
// Place of element e of a unit: (0, 4), (1, 5), (2, 6), (3, 7).
__host__ __device__ constexpr int unit_pos(int e) { return e < 4 ? 2 * e : 2 * (e - 4) + 1; }

// A stage: two K-blocks of 16 rows x 64 bytes of codes, then the scales and the zeros of their 8-row halves.
template <int GPB>
__host__ __device__ constexpr int stage_bytes() {
  return 2048 + 4 * GPB * 16 + 4 * GPB * 8;
}
template <int NT>
__host__ __device__ constexpr int stages() {
  return NT == 1 ? 4 : 3;
}

// Dynamic shared memory, in bytes from its start.
struct Smem {
  int x, sx, sums, list, tiles, total;
};
template <int NT, int GPB>
__host__ __device__ inline Smem smem_of(const W4Args& a) {
  Smem s;
  s.x = kWarps * stages<NT>() * stage_bytes<GPB>();                       // activations: [entry][4][cols][4] units
  s.sx = s.x + a.entries * a.c.cols() * 256;                              // their scales: [entry][GPB][8 NT]
  s.sums = s.sx + (a.x_groups > 1 ? a.entries * GPB * NT * 8 * 4 : 0);    // parts of the sums: [warp + tile][column][16 rows]
  s.list = s.sums + (kWarps - 1 + a.tiles_per_block) * NT * 8 * kColPitch * 4;
  s.tiles = s.list + a.entries * 4;                                       // the block's K-blocks, then its tiles
  s.total = s.tiles + a.tiles_per_block * 4;
  return s;
}

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

// Eight consecutive activations of one token -> `pieces` units of bf16 whose sum they are.
__device__ __forceinline__ void stage_activations(const W4Args& a, int64_t at, bool in, uint4* unit, int piece_step) {
  float v[8];
  if (!in) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
  } else if (a.x_kind == MLPMOE_FP32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.x) + at);
    const float4 lo = p[0], hi = p[1];
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  } else if (a.x_kind == MLPMOE_BF16) {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.x) + at);
    v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xFFFF0000u), v[2] = __uint_as_float(w.y << 16),
    v[3] = __uint_as_float(w.y & 0xFFFF0000u), v[4] = __uint_as_float(w.z << 16), v[5] = __uint_as_float(w.z & 0xFFFF0000u),
    v[6] = __uint_as_float(w.w << 16), v[7] = __uint_as_float(w.w & 0xFFFF0000u);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.x) + at);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3))), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[e] = f.x, v[e + 1] = f.y;
    }
  }
  for (int p = 0; p < a.c.pieces; ++p) {
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 pair = __floats2bfloat162_rn(v[e], v[e + 4]);
      v[e] -= __low2float(pair);
      v[e + 4] -= __high2float(pair);
      o[e] = *reinterpret_cast<const uint32_t*>(&pair);
    }
    unit[p * piece_step] = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// grid: (shares of the row tiles, cluster along K, chunks of tokens)
template <int NT, int GPB, bool GATEUP>
__global__ void __launch_bounds__(kThreads, 1) w4_kernel(const __grid_constant__ W4Args a) {
  constexpr int kStages = stages<NT>(), kStage = stage_bytes<GPB>(), kWords = 4 / GPB;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint8_t s_active[kW4MaxBranches];
  __shared__ int s_scan[kWarps];
  __shared__ int s_n[2];                // K-blocks and tiles of this block
  // gate|up waits for everything before it on the stream; by the time all its blocks have passed here only gate|up
  // itself is outstanding, so the down kernel, which then may start, reads weights and selection without a wait.
  if (GATEUP) ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const Smem L = smem_of<NT, GPB>(a);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int chunk = blockIdx.z, rank = blockIdx.y, cluster = gridDim.y;
  const int tokens = a.c.tokens, cols = a.c.cols();
  int* s_list = reinterpret_cast<int*>(smem + L.list);
  int* s_tiles = reinterpret_cast<int*>(smem + L.tiles);

  // ---- this block's K-blocks and tiles
  int n_entries, n_tiles;
  if (a.dense) {
    const int per = (a.kblocks + cluster - 1) / cluster;
    n_entries = max(0, min(per, a.kblocks - rank * per));
    n_tiles = min(a.tiles_per_block, a.tiles - static_cast<int>(blockIdx.x) * a.tiles_per_block);
    for (int i = threadIdx.x; i < a.entries; i += kThreads) s_list[i] = i < n_entries ? rank * per + i : -1;
    for (int i = threadIdx.x; i < n_tiles; i += kThreads) s_tiles[i] = blockIdx.x * a.tiles_per_block + i;
    __syncthreads();
  } else {
    // the branches that a token of this chunk computes
    const int n_here = min(tokens, a.n - chunk * tokens);
    for (int b = threadIdx.x; b < a.B; b += kThreads) s_active[b] = a.select == nullptr && a.alpha[b] != 0.0f;
    __syncthreads();
    if (a.select != nullptr) {
      const uint8_t* sel = a.select + static_cast<int64_t>(chunk) * tokens * a.B;
      for (int i = threadIdx.x; i < n_here * a.B; i += kThreads)
        if (sel[i] != 0 && a.alpha[i % a.B] != 0.0f) s_active[i % a.B] = 1;
    }
    __syncthreads();
    // gate|up: the computed tiles in order, an equal share to every block; down: the K-blocks with a computed neuron
    const int total = GATEUP ? a.tiles : a.kblocks;
    int live_total = 0, share = 0, first = 0;
    for (int pass = 0; pass < 2; ++pass) {              // count, then list this block's share
      int running = 0;
      for (int base = 0; base < total; base += kThreads) {
        const int i = base + threadIdx.x;
        bool live = false;
        if (i < total) {
          if (GATEUP) {
            live = s_active[branch_of(a, i * 8)] != 0;
          } else {
            for (int b = branch_of(a, i * 128); b < a.B && a.off[b] < (i + 1) * 128; ++b) live = live || s_active[b] != 0;
          }
        }
        const unsigned ballot = __ballot_sync(0xFFFFFFFFu, live);
        if (lane == 0) s_scan[warp] = __popc(ballot);
        __syncthreads();
        int before = running, all = running;
        for (int w = 0; w < kWarps; ++w) {
          if (w < warp) before += s_scan[w];
          all += s_scan[w];
        }
        if (pass == 1 && live) {
          const int at = before + __popc(ballot & ((1u << lane) - 1u)) - first;
          if (at >= 0 && at < share) (GATEUP ? s_tiles : s_list)[at] = i;
        }
        running = all;
        __syncthreads();
      }
      if (pass == 0) {
        live_total = running;
        const int shares = GATEUP ? static_cast<int>(gridDim.x) : cluster, mine = GATEUP ? static_cast<int>(blockIdx.x) : rank;
        const int per = (live_total + shares - 1) / shares;
        first = mine * per;
        share = max(0, min(per, live_total - first));
      }
    }
    if (GATEUP) {
      const int per = (a.kblocks + cluster - 1) / cluster;
      n_entries = max(0, min(per, a.kblocks - rank * per));
      n_tiles = share;
      for (int i = threadIdx.x; i < a.entries; i += kThreads) s_list[i] = i < n_entries ? rank * per + i : -1;
    } else {
      n_entries = share;
      n_tiles = min(a.tiles_per_block, a.tiles - static_cast<int>(blockIdx.x) * a.tiles_per_block);
      for (int i = threadIdx.x; i < n_tiles; i += kThreads) s_tiles[i] = blockIdx.x * a.tiles_per_block + i;
      for (int i = share + threadIdx.x; i < a.entries; i += kThreads) s_list[i] = -1;
    }
    __syncthreads();
  }

  // ---- this warp's run of steps (tile, two K-blocks)
  const int steps = (n_entries + 1) / 2;
  const int per_warp = (n_tiles * steps + kWarps - 1) / kWarps;
  const int run_begin = min(n_tiles * steps, warp * per_warp), run_end = min(n_tiles * steps, run_begin + per_warp);
  const int count = run_end - run_begin;

  // ---- copies of one stage: 16 bytes of codes per lane, K-block and half; scales and zeros by the first lanes
  const uint32_t ring = ptx::smem_u32(smem) + warp * kStages * kStage;
  const uint32_t q_dst = ring + g * 64 + (t ^ ((g >> 1) & 3)) * 16;
  const int s_block = (lane / (2 * GPB)) & 1, s_half = (lane / GPB) & 1, s_group = lane % GPB;   // lanes below 4 GPB
  const W4Mat& sm = a.m[s_half];
  const bool s_lane = lane < 4 * GPB, z_lane = s_lane && sm.zero != nullptr;
  const uint8_t* q_src[2];
  bool q_ok[2], s_ok = false;
  int s_row = 0;
  int i_tile = steps > 0 ? run_begin / steps : 0, i_step = steps > 0 ? run_begin % steps : 0, i_left = count;
  auto open_tile = [&]() {
    const int tile = s_tiles[i_tile];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = (GATEUP ? tile * 8 : tile * 16 + 8 * h) + g;
      q_ok[h] = row < a.rows;
      q_src[h] = a.m[h].q + (q_ok[h] ? row * a.m[h].pitch : 0);
    }
    s_row = GATEUP ? tile * 8 : tile * 16 + 8 * s_half;
    s_ok = s_row < a.rows;
  };
  if (i_left > 0) open_tile();
  auto issue = [&](int slot) {
    if (i_left > 0) {
      const int2 kb = *reinterpret_cast<const int2*>(s_list + 2 * i_step);
      const uint32_t dst = q_dst + slot * kStage;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int block = j == 0 ? kb.x : kb.y;
        const int byte = block * 64 + t * 16;
        const bool in = block >= 0 && byte < a.m[0].pitch;
#pragma unroll
        for (int h = 0; h < 2; ++h) cp_async16(dst + (j * 2 + h) * 512, q_src[h] + (in ? byte : 0), in && q_ok[h]);
      }
      if (s_lane) {
        const int block = s_block == 0 ? kb.x : kb.y;
        const int group = block * GPB + s_group;
        const bool in = s_ok && block >= 0 && group < sm.n_groups;
        const int64_t at = in ? group * sm.rows16 + s_row : 0;
        cp_async16(ring + slot * kStage + 2048 + lane * 16, sm.scale + at, in);
        if (z_lane) cp_async8(ring + slot * kStage + 2048 + 4 * GPB * 16 + lane * 8, sm.zero + at, in);
      }
      --i_left;
      if (++i_step == steps && i_left > 0) {
        i_step = 0;
        ++i_tile;
        open_tile();
      }
    }
    cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) issue(i);

  // ---- the activations of this block's K-blocks
  uint4* s_x = reinterpret_cast<uint4*>(smem + L.x);
  float* s_sx = reinterpret_cast<float*>(smem + L.sx);
  const int even_entries = 2 * steps;
  if (GATEUP) {
    for (int i = threadIdx.x; i < even_entries * 16 * tokens; i += kThreads) {
      const int k8 = i & 15, entry = (i >> 4) % even_entries, tok = (i >> 4) / even_entries;
      const int block = s_list[entry], token = chunk * tokens + tok, k = block * 128 + k8 * 8;
      stage_activations(a, token * a.x_stride + k, block >= 0 && k < a.K && token < a.n,
                        s_x + ((entry * 4 + unit_word<GPB>(k8)) * cols + tok) * 4 + unit_lane<GPB>(k8), tokens * 4);
    }
    if (a.x_groups > 1) {
      for (int i = threadIdx.x; i < even_entries * GPB * NT * 8; i += kThreads) {
        const int c = i % (NT * 8), j = i / (NT * 8) % GPB, entry = i / (NT * 8) / GPB, token = chunk * tokens + c;
        const int xg = (s_list[entry] * GPB + j) >> a.x_shift;
        s_sx[i] = s_list[entry] >= 0 && c < tokens && token < a.n && xg < a.x_groups ? a.x_scale[static_cast<int64_t>(token) * a.x_groups + xg] : 0.0f;
      }
    }
  } else {
    ptx::griddep_wait();                // h is complete
    const uint4* h = a.h_in + static_cast<int64_t>(chunk) * a.kblocks * (cols * 16);
    for (int i = threadIdx.x; i < even_entries * cols * 16; i += kThreads) {
      const int entry = i / (cols * 16), u = i % (cols * 16), block = s_list[entry];
      const int neuron = block * 128 + unit_k8<GPB>(u / (cols * 4), u & 3) * 8, token = chunk * tokens + (u >> 2) % cols % tokens;
      bool in = block >= 0 && neuron < a.K && token < a.n;
      if (in && !a.dense) {             // what the token does not compute is 0, and gate|up may have left it unwritten
        const int b = branch_of(a, neuron);
        in = s_active[b] != 0 && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
      }
      cp_async16(ptx::smem_u32(s_x + i), h + (in ? static_cast<int64_t>(block) * (cols * 16) + u : 0), in);
    }
    cp_async_commit();
    cp_async_wait<0>();
  }
  __syncthreads();

  // columns 8 nt + g: the lanes of a column that stands for no token keep zeros
  bool col_ok[NT];
  uint4 xb[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = nt * 8 + g;
    col_ok[nt] = c < cols && chunk * tokens + c % tokens < a.n;
#pragma unroll
    for (int w = 0; w < 4; ++w) xb[nt][w] = make_uint4(0u, 0u, 0u, 0u);
  }
  float acc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[nt][i] = 0.0f;
  float* sums = reinterpret_cast<float*>(smem + L.sums);
  const bool scaled = GATEUP && a.x_groups > 1;

  int slot = 0, c_tile = steps > 0 ? run_begin / steps : 0, c_step = steps > 0 ? run_begin % steps : 0;
  for (int i = 0; i < count; ++i) {
    cp_async_wait<kStages - 2>();
    __syncwarp();                       // the stage is in shared memory for all lanes, and the slot before it has been read by all
    const uint8_t* st = smem + (warp * kStages + slot) * kStage;
    issue(slot == 0 ? kStages - 1 : slot - 1);
#pragma unroll
    for (int j = 0; j < 2 * GPB; ++j) {
      const int block = j / GPB;
      if (j % GPB == 0) {
        const uint4* xp = s_x + (2 * c_step + block) * (cols * 16) + lane;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int w = 0; w < 4; ++w)
            if (col_ok[nt]) xb[nt][w] = xp[w * cols * 4 + nt * 32];
      }
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
        const uint8_t* row = st + (block * 2 + h) * 512 + g * 64;
        if (GPB == 1) {
          const uint4 v = *reinterpret_cast<const uint4*>(row + ((t ^ sw) * 16));
          q[h][0] = v.x, q[h][1 % kWords] = v.y, q[h][2 % kWords] = v.z, q[h][3 % kWords] = v.w;
        } else if (GPB == 2) {
          const uint2 v = *reinterpret_cast<const uint2*>(row + (((2 * (j % GPB) + (t >> 1)) ^ sw) * 16) + (t & 1) * 8);
          q[h][0] = v.x, q[h][1 % kWords] = v.y;
        } else {
          q[h][0] = *reinterpret_cast<const uint32_t*>(row + (((j % GPB) ^ sw) * 16) + t * 4);
        }
        const int piece = (block * 2 + h) * GPB + j % GPB;
        s[h] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(st + 2048 + piece * 16 + g * 2));
        const uint32_t z = a.m[h].zero != nullptr ? st[2048 + 4 * GPB * 16 + piece * 8 + g] : 8u;
        bias[h] = 0x43004300u + z * 0x00010001u;
      }
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        uint32_t lo[4], hi[4];
        unpack(q[0][w], bias[0], lo);
        unpack(q[1][w], bias[1], hi);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 b = xb[nt][(j % GPB) * kWords + w];
          mma(part[nt], lo[0], hi[0], lo[1], hi[1], b.x, b.y);
          mma(part[nt], lo[2], hi[2], lo[3], hi[3], b.z, b.w);
        }
      }
      if (scaled) {
        const float* sx = s_sx + ((2 * c_step) * GPB + j) * (NT * 8) + 2 * t;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const float2 f = *reinterpret_cast<const float2*>(sx + nt * 8);
          acc[nt][0] += part[nt][0] * (s[0] * f.x);
          acc[nt][1] += part[nt][1] * (s[0] * f.y);
          acc[nt][2] += part[nt][2] * (s[1] * f.x);
          acc[nt][3] += part[nt][3] * (s[1] * f.y);
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
    if (++c_step == steps || i + 1 == count) {      // the run leaves this tile: its part of the tile's sums
      float* p = sums + (warp + c_tile) * (NT * 8 * kColPitch) + (2 * t) * kColPitch + g;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float* c = p + nt * 8 * kColPitch;
        c[0] = acc[nt][0];
        c[kColPitch] = acc[nt][1];
        c[8] = acc[nt][2];
        c[kColPitch + 8] = acc[nt][3];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[nt][e] = 0.0f;
      }
      c_step = 0;
      ++c_tile;
    }
  }
  cp_async_wait<0>();
  __syncthreads();

  // ---- sums of a tile: the parts of the warps that worked on it, in order, and the pieces of the token
  auto sum_of = [&](int tile, int tok, int row) {
    float v = 0.0f;
    if (steps == 0) return v;
    const int w0 = tile * steps / per_warp, w1 = ((tile + 1) * steps - 1) / per_warp;
    for (int w = w0; w <= w1; ++w) {
      const float* p = sums + (w + tile) * (NT * 8 * kColPitch) + row;
      for (int c = tok; c < cols; c += tokens) v += p[c * kColPitch];
    }
    return v;
  };
  float* own = reinterpret_cast<float*>(smem);       // of a cluster: this block's sums, over the ring
  if (cluster > 1) {
    for (int i = threadIdx.x; i < n_tiles * tokens * 16; i += kThreads) own[i] = sum_of((i >> 4) / tokens, (i >> 4) % tokens, i & 15);
    __syncthreads();
    ptx::cluster_sync_all();
  }
  auto total_of = [&](int tile, int tok, int row) {
    if (cluster == 1) return sum_of(tile, tok, row);
    float v = 0.0f;
    for (int r = 0; r < cluster; ++r) v += ld_cluster_f32(own + (tile * tokens + tok) * 16 + row, r);
    return v;
  };
  if (GATEUP) {
    for (int i = rank * kThreads + threadIdx.x; i < n_tiles * tokens * 8; i += cluster * kThreads) {
      const int e = i & 7, tok = (i >> 3) % tokens, tile = (i >> 3) / tokens, token = chunk * tokens + tok;
      if (token >= a.n) continue;
      const int neuron = s_tiles[tile] * 8 + e, b = branch_of(a, neuron);
      const bool on = a.dense || (s_active[b] != 0 && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0));
      float h = 0.0f;
      if (on) {
        float gate = total_of(tile, tok, e), up = total_of(tile, tok, 8 + e);
        if (a.x_scale != nullptr && a.x_groups == 1) {
          gate *= a.x_scale[token];
          up *= a.x_scale[token];
        }
        h = gate / (1.0f + expf(-gate)) * up * a.alpha[b];
      }
      // h as bf16 pieces: two keep 2^-16 of it (y is rounded to 2^-8), three all 24 bits
      const int hc = a.hc.cols(), k8 = (neuron % 128) / 8, h_tok = token % a.hc.tokens;
      const int64_t block = static_cast<int64_t>(token / a.hc.tokens) * a.h_kblocks + neuron / 128;
      __nv_bfloat16* out = a.h + ((block * 4 + unit_word<GPB>(k8)) * hc * 4 + unit_lane<GPB>(k8)) * 8 + unit_pos(e);
      for (int p = 0; p < a.hc.pieces; ++p) {
        const __nv_bfloat16 piece = __float2bfloat16_rn(h);
        h -= __bfloat162float(piece);
        out[(p * a.hc.tokens + h_tok) * 32] = piece;
      }
    }
  } else {
    for (int i = rank * kThreads + threadIdx.x; i < n_tiles * tokens * 16; i += cluster * kThreads) {
      const int row = i & 15, tok = (i >> 4) % tokens, tile = (i >> 4) / tokens;
      const int m = s_tiles[tile] * 16 + row, token = chunk * tokens + tok;
      if (m >= a.rows || token >= a.n) continue;
      float v = total_of(tile, tok, row);
      if (a.select != nullptr) {
        // c_t: the quotient and the root in double, rounded once, as the routed forward does
        int k = 0, n_avail = 0;
        for (int b = 0; b < a.B; ++b) {
          const bool avail = a.alpha[b] != 0.0f;
          n_avail += avail ? 1 : 0;
          k += avail && a.select[static_cast<int64_t>(token) * a.B + b] != 0 ? 1 : 0;
        }
        float coef = k > 0 ? 1.0f : 0.0f;
        if (k > 0 && a.compensate) coef = static_cast<float>(sqrt(static_cast<double>(n_avail) / static_cast<double>(k)));
        v *= coef;
      }
      const int64_t at = static_cast<int64_t>(token) * a.rows + m;
      if (a.residual != nullptr) v += a.residual[at];
      if (a.y_bf16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
      else static_cast<float*>(a.y)[at] = v;
    }
  }
  if (cluster > 1) {
    __syncthreads();
    ptx::cluster_sync_all();            // no block leaves while another reads its sums
  }
}

template <int NT, int GPB, bool GATEUP>
cudaError_t launch(const W4Args& a, int cluster, cudaStream_t st) {
  auto kernel = w4_kernel<NT, GPB, GATEUP>;
  const int smem = smem_of<NT, GPB>(a).total;
  if (smem > kSmemMax) return cudaErrorInvalidValue;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.tiles + a.tiles_per_block - 1) / a.tiles_per_block), static_cast<unsigned>(cluster),
                     static_cast<unsigned>(a.c.chunks));
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
  switch ((a.c.cols() + 7) / 8) {
    case 1: return launch<1, GPB, GATEUP>(a, cluster, st);
    case 2: return launch<2, GPB, GATEUP>(a, cluster, st);
    case 3: return launch<3, GPB, GATEUP>(a, cluster, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace w4
}  // namespace mlpmoe
