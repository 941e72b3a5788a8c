// The layer on 4-bit weights for a few tokens (mlpmoe_w4_forward): one kernel template for both products.
//     gate|up:  h[j, t] = alpha_b silu(sum_k Wg[j, k] x[k, t]) * (sum_k Wu[j, k] x[k, t])
//     down:     y[m, t] = residual + c_t sum_j Wd[m, j] h[j, t]
// with W[r, k] = (code - zero) * scale, one scale and zero per row and group of K.
//
// Bound by HBM: the codes are read once.  Between the copy and the result an SM issues only a few operations per code, and
// that is what limits such a kernel, so the products are taken on whole numbers (mma.sync, u8 x s8 in s32, exact): a
// word of eight codes becomes two operand registers with two ANDs and a shift, where a bf16 product needs eleven
// operations (210 against 256 issued per 16 x 128 block of codes even after tuning).  The activations are held as
// fixed point inside each group of K: x = (d0 + 256 d1 + 65536 d2) * unit with digits of 8 bits, unit = the group's
// largest |x| / 8323072; every digit is a column of the product, so up to eight columns (two tokens of three digits)
// cost what one does.  Three digits (an fp32 y) keep 2^-23 of the group's largest, which is what an fp32 sum keeps;
// two (y rounded to bf16, 2^-8) keep 2^-16.  sum (code - zero) x = sum code x - zero sum x exactly, the second sum being
// the group's own; scale and unit are applied to the group's whole-number sum in fp32.
// mma.sync and not tcgen05: a scale per group of K means reading the accumulators back after every 32 to 128 columns of
// K, and for a few tokens the product's time is the copy's anyway.
//
// One block per SM takes an equal share of the 16-row tiles (gate|up: the gate and up rows of eight neurons, so that a
// lane ends with both sums of its neurons).  Its steps, (tile, 256 columns of K), are dealt to the 16 warps in equal
// runs; a run may end inside a tile, and the parts of a tile are joined in warp order, so the result is the same
// on every call.  Blocks of a cluster share K where the activations of all of K would not fit in shared memory, or
// where there are few rows.  Every warp keeps its own ring of stages filled by cp.async: no barrier in the loop.
//
// The four lanes of a row hold different eights of consecutive k, and a register of codes is the even or the odd four of an
// eight: the activations stand in shared memory to match, eight bytes (even four, odd four) for each eight.
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
  int x, unit, sums, list, tiles, total;
};
template <int NT, int GPB>
__host__ __device__ inline Smem smem_of(const W4Args& a) {
  Smem s;
  s.x = kWarps * stages<NT>() * stage_bytes<GPB>();                       // digits: [entry][2][8 NT][4] pairs of eights
  s.unit = s.x + a.entries * NT * 8 * 128;                                // their (unit, - sum of digits): [entry][GPB][8 NT]
  s.sums = s.unit + a.entries * GPB * NT * 8 * 8;                         // parts of the sums: [warp + tile][column][16 rows]
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

// d += a x b on whole numbers: a 16 rows x 32 codes (u8), b 32 digits x 8 columns (s8).
__device__ __forceinline__ void mma(int (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(d[0]), "+r"(d[1]), "+r"(d[2]), "+r"(d[3])
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

// Eight consecutive activations of one token, from element `at` of x (gate|up) or h (down, fp32).
__device__ __forceinline__ void load_eight(const void* x, int kind, int64_t at, float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(x) + at);
    const float4 lo = p[0], hi = p[1];
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  } else if (kind == MLPMOE_BF16) {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(x) + at);
    v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xFFFF0000u), v[2] = __uint_as_float(w.y << 16),
    v[3] = __uint_as_float(w.y & 0xFFFF0000u), v[4] = __uint_as_float(w.z << 16), v[5] = __uint_as_float(w.z & 0xFFFF0000u),
    v[6] = __uint_as_float(w.w << 16), v[7] = __uint_as_float(w.w & 0xFFFF0000u);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(x) + at);
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3))), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[e] = f.x, v[e + 1] = f.y;
    }
  }
}

// grid: (shares of the row tiles, cluster along K, chunks of tokens)
template <int NT, int GPB, bool GATEUP, bool ZERO>
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
  const bool s_lane = lane < 4 * GPB, z_lane = ZERO && s_lane && sm.zero != nullptr;
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
  if (ZERO && s_lane && sm.zero == nullptr) {        // a half without stored zeros beside one with them: 8 in every slot, for good
    for (int i = 0; i < kStages; ++i)
      *reinterpret_cast<uint2*>(smem + (warp * kStages + i) * kStage + 2048 + 4 * GPB * 16 + lane * 8) = make_uint2(0x08080808u, 0x08080808u);
  }
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

  // ---- the activations of this block's K-blocks as digits: a thread takes eight k of one token, the group's 4, 8 or 16
  // threads are neighbours
  uint2* s_x = reinterpret_cast<uint2*>(smem + L.x);
  float2* s_unit = reinterpret_cast<float2*>(smem + L.unit);
  const int even_entries = 2 * steps;
  if (!GATEUP) ptx::griddep_wait();     // h is complete
  for (int i = threadIdx.x; i < even_entries * GPB * NT * 8; i += kThreads)
    if (i % (NT * 8) >= cols) s_unit[i] = make_float2(0.0f, 0.0f);
  for (int i = threadIdx.x; i < even_entries * 16 * tokens; i += kThreads) {      // a multiple of 32 threads take part
    const int k8 = i & 15, entry = (i >> 4) % even_entries, tok = (i >> 4) / even_entries;
    const int block = s_list[entry], token = chunk * tokens + tok, k = block * 128 + k8 * 8;
    bool in = block >= 0 && k < a.K && token < a.n;
    if (!GATEUP && in && !a.dense) {    // what the token does not compute is 0, and gate|up may have left it unwritten
      const int b = branch_of(a, k);
      in = s_active[b] != 0 && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
    }
    float v[8], top = 0.0f;
    if (in) {
      load_eight(a.x, a.x_kind, token * a.x_stride + k, v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
#pragma unroll
    for (int o = 1; o < 16 / GPB; o *= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    // the largest becomes 127 in the highest digit and 0 below; a group all below 2^-100 counts as 0 (its unit would leave
    // the range of fp32)
    const float most = a.c.pieces == 3 ? 8323072.0f : 32512.0f;
    const bool some = top >= 7.8886091e-31f;
    const float inv = some ? most / top : 0.0f;
    float unit = some ? top / most : 0.0f;
    int fixed[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) fixed[e] = __float2int_rn(v[e] * inv);
    const int j = k8 / (16 / GPB);
    if (GATEUP && a.x_scale != nullptr && in) {
      const int xg = a.x_groups == 1 ? 0 : (block * GPB + j) >> a.x_shift;
      unit *= a.x_scale[static_cast<int64_t>(token) * a.x_groups + xg];
    }
    const int word = unit_word<GPB>(k8);
    uint2* out = s_x + (((entry * 2 + (word >> 1)) * (NT * 8) + tok) * 4 + unit_lane<GPB>(k8)) * 2 + (word & 1);
    for (int p = 0; p < a.c.pieces; ++p) {
      // the lowest digit, -128 .. 127, and what is left above it
      uint32_t even = 0, odd = 0;
      int sum = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int digit = static_cast<int8_t>(fixed[e]);
        fixed[e] = (fixed[e] - digit) >> 8;
        sum += digit;
        const uint32_t byte = static_cast<uint32_t>(digit & 255) << (8 * (e / 2));
        if (e & 1) odd |= byte;
        else even |= byte;
      }
#pragma unroll
      for (int o = 1; o < 16 / GPB; o *= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      out[p * tokens * 8] = make_uint2(even, odd);
      if (k8 % (16 / GPB) == 0)
        s_unit[(entry * GPB + j) * (NT * 8) + p * tokens + tok] = make_float2(unit, __int_as_float(-sum));
      unit *= 256.0f;
    }
  }
  __syncthreads();

  // columns 8 nt + g: the lanes of a column that stands for no token keep zeros
  bool col_ok[NT];
  uint4 xb[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int c = nt * 8 + g;
    col_ok[nt] = c < cols && chunk * tokens + c % tokens < a.n;
#pragma unroll
    for (int w = 0; w < 2; ++w) xb[nt][w] = make_uint4(0u, 0u, 0u, 0u);
  }
  float acc[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[nt][i] = 0.0f;
  float* sums = reinterpret_cast<float*>(smem + L.sums);

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
        const uint4* xp = reinterpret_cast<const uint4*>(s_x) + (2 * c_step + block) * (NT * 64) + lane;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int w = 0; w < 2; ++w)
            if (col_ok[nt]) xb[nt][w] = xp[w * (NT * 32) + nt * 32];
      }
      uint32_t q[2][kWords];
      int zero[2];
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
        zero[h] = ZERO ? st[2048 + 4 * GPB * 16 + piece * 8 + g] : 8;
      }
      // - zero * sum of digits first, then the codes' products
      const float4* up = reinterpret_cast<const float4*>(s_unit + ((2 * c_step) * GPB + j) * (NT * 8)) + t;
      int part[NT][4];
      float2 unit[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float4 u = up[nt * 4];
        unit[nt] = make_float2(u.x, u.z);
        part[nt][0] = zero[0] * __float_as_int(u.y);
        part[nt][1] = zero[0] * __float_as_int(u.w);
        part[nt][2] = ZERO ? zero[1] * __float_as_int(u.y) : part[nt][0];
        part[nt][3] = ZERO ? zero[1] * __float_as_int(u.w) : part[nt][1];
      }
#pragma unroll
      for (int w = 0; w < kWords; ++w) {
        const int at = (j % GPB) * kWords + w;
        const uint32_t a0 = q[0][w] & 0x0F0F0F0Fu, a1 = q[1][w] & 0x0F0F0F0Fu;
        const uint32_t a2 = (q[0][w] >> 4) & 0x0F0F0F0Fu, a3 = (q[1][w] >> 4) & 0x0F0F0F0Fu;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const uint4 b = xb[nt][at >> 1];
          mma(part[nt], a0, a1, a2, a3, at & 1 ? b.z : b.x, at & 1 ? b.w : b.y);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        // at most 15 * 128 * 256 in magnitude: exact in fp32
        acc[nt][0] += __int2float_rn(part[nt][0]) * (s[0] * unit[nt].x);
        acc[nt][1] += __int2float_rn(part[nt][1]) * (s[0] * unit[nt].y);
        acc[nt][2] += __int2float_rn(part[nt][2]) * (s[1] * unit[nt].x);
        acc[nt][3] += __int2float_rn(part[nt][3]) * (s[1] * unit[nt].y);
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
        const float gate = total_of(tile, tok, e), up = total_of(tile, tok, 8 + e);
        h = gate / (1.0f + expf(-gate)) * up * a.alpha[b];
      }
      a.h[static_cast<int64_t>(token) * a.rows + neuron] = h;
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

template <int NT, int GPB, bool GATEUP, bool ZERO>
cudaError_t launch(const W4Args& a, int cluster, cudaStream_t st) {
  auto kernel = w4_kernel<NT, GPB, GATEUP, ZERO>;
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

template <int GPB, bool GATEUP, bool ZERO>
cudaError_t launch_nt(const W4Args& a, int cluster, cudaStream_t st) {
  switch ((a.c.cols() + 7) / 8) {
    case 1: return launch<1, GPB, GATEUP, ZERO>(a, cluster, st);
    case 2: return launch<2, GPB, GATEUP, ZERO>(a, cluster, st);
    case 3: return launch<3, GPB, GATEUP, ZERO>(a, cluster, st);
    default: return cudaErrorInvalidValue;
  }
}

template <int GPB, bool GATEUP>
cudaError_t launch_zero(const W4Args& a, int cluster, cudaStream_t st) {
  return a.m[0].zero != nullptr || a.m[1].zero != nullptr ? launch_nt<GPB, GATEUP, true>(a, cluster, st)
                                                          : launch_nt<GPB, GATEUP, false>(a, cluster, st);
}

}  // namespace w4
}  // namespace mlpmoe
