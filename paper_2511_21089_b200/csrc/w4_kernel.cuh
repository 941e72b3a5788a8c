// The layer on 4-bit weights for a few tokens (mlpmoe_w4_forward): one kernel template for both products.
//     gate|up:  h[j, t] = alpha_b silu(sum_k Wg[j, k] x[k, t]) * (sum_k Wu[j, k] x[k, t])
//     down:     y[m, t] = residual + c_t sum_j Wd[m, j] h[j, t]
// with W[r, k] = (code - zero) * scale, one scale and zero per row and group of K.
//
// Bound by HBM: the codes are read once.  Between the copy and the result an SM issues only a few operations per code, and
// that is what limits such a kernel, so the products are taken on whole numbers (mma.sync, u8 x s8 in s32, exact): a
// word of eight codes becomes two operand registers with two ANDs and a shift, where a bf16 product needs eleven
// operations (120 instructions in all against 210 per 16 x 128 block of codes).  The activations are held as fixed
// point inside each group of K: x = (d0 + 256 d1 + 65536 d2) * unit with digits of 8 bits and unit a power of two;
// every digit is a column of the product, so up to eight columns (two tokens of three digits) cost what one does.
// Three digits (an fp32 y) are off by at most 2^-23 of the group's largest |x|, which is what an fp32 sum loses; two (y
// rounded to bf16, 2^-8) by 2^-15.  sum (code - zero) x = sum code x - zero sum x exactly, the second sum being
// the group's own; scale and unit are applied to the group's whole-number sum in fp32.
// mma.sync and not tcgen05: a scale per group of K means reading the accumulators back after every 32 to 128 columns of
// K, and for a few tokens converting the codes to an operand that tensor memory takes costs more than these products.
// Measured (4096 x 14336, group 128): one token 29.9 us, eight on a selection of 8 of 32 branches 46.4; the codes alone take
// 14.3 us of a copy.  Of the 29.9 about 12 are fixed: two launches, filling the rings, the digits, the sums' exchange between
// warps and blocks; the loop runs at 70 % of the issue slots.  Five ring stages instead of four bring nothing.
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
constexpr int kWideSmemMax = kSmemMax - 4096;   // the tiled kernels have more of those

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
// Stages of a warp's ring: about 100 KB under way in an SM; a fifth stage measured the same.
__host__ __device__ constexpr int stages(int nt) { return nt == 1 ? 4 : 3; }

// Dynamic shared memory, in bytes from its start.
struct Smem {
  int x, unit, sums, list, tiles, branch, total;
};
template <int NT, int GPB>
__host__ __device__ inline Smem smem_of(const W4Args& a) {
  Smem s;
  s.x = kWarps * stages(NT) * stage_bytes<GPB>();                       // digits: [entry][2][8 NT][4] pairs of eights
  s.unit = s.x + a.entries * NT * 8 * 128;                                // their (unit, - sum of digits): [entry][GPB][8 NT]
  s.sums = s.unit + a.entries * GPB * NT * 8 * 8;                         // parts of the sums: [warp + tile][column][16 rows]
  s.list = s.sums + (kWarps - 1 + a.tiles_per_block) * NT * 8 * kColPitch * 4;
  s.tiles = s.list + a.entries * 4;                                       // the block's K-blocks; its tiles: place, first and last warp
  s.branch = s.tiles + a.tiles_per_block * 12;                            // first neurons, running counts, then [tokens][B] computed or not
  s.total = s.branch + (a.dense ? 0 : (2 * (a.B + 1) * 4 + a.c.tokens * a.B));
  return s;
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
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

__device__ __forceinline__ float4 ld_cluster_f32x4(const float* p, uint32_t rank) {
  float4 v;
  const uint32_t addr = ptx::map_to_cta(ptx::smem_u32(p), rank);
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}

// The last b with first[b] <= value, first ascending.
__device__ __forceinline__ int find_branch(const int* first, int B, int value) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (first[mid] <= value) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Eight consecutive activations of one token from element `at`, as they stand in memory, and as fp32.
struct Raw {
  uint4 lo, hi;
};
__device__ __forceinline__ Raw load_raw(const void* x, int kind, int64_t at) {
  Raw r;
  r.lo = r.hi = make_uint4(0u, 0u, 0u, 0u);
  if (kind == MLPMOE_FP32) {
    const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(x) + at);
    r.lo = p[0];
    r.hi = p[1];
  } else if (kind == MLPMOE_BF16) {
    r.lo = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(x) + at);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(x) + at);
    r.lo.x = w.x;
    r.lo.y = w.y;
  }
  return r;
}
__device__ __forceinline__ void to_f32(const Raw& r, int kind, float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    v[0] = __uint_as_float(r.lo.x), v[1] = __uint_as_float(r.lo.y), v[2] = __uint_as_float(r.lo.z), v[3] = __uint_as_float(r.lo.w);
    v[4] = __uint_as_float(r.hi.x), v[5] = __uint_as_float(r.hi.y), v[6] = __uint_as_float(r.hi.z), v[7] = __uint_as_float(r.hi.w);
  } else if (kind == MLPMOE_BF16) {
    v[0] = __uint_as_float(r.lo.x << 16), v[1] = __uint_as_float(r.lo.x & 0xFFFF0000u), v[2] = __uint_as_float(r.lo.y << 16),
    v[3] = __uint_as_float(r.lo.y & 0xFFFF0000u), v[4] = __uint_as_float(r.lo.z << 16), v[5] = __uint_as_float(r.lo.z & 0xFFFF0000u),
    v[6] = __uint_as_float(r.lo.w << 16), v[7] = __uint_as_float(r.lo.w & 0xFFFF0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += 2) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2(static_cast<__nv_fp8x2_storage_t>((e < 4 ? r.lo.x : r.lo.y) >> (8 * (e & 3))), __NV_E4M3);
      const float2 f = __half22float2(__half2(h));
      v[e] = f.x, v[e + 1] = f.y;
    }
  }
}

__device__ __forceinline__ bool is_finite(float v) { return fabsf(v) <= 3.402823466e38f; }

// The largest magnitude; a NaN wins.
__device__ __forceinline__ float larger(float a, float b) {
  float top;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(top) : "f"(fabsf(a)), "f"(fabsf(b)));
  return top;
}
__device__ __forceinline__ float largest(const float (&v)[8]) {
  float top = larger(v[0], v[1]);
#pragma unroll
  for (int e = 2; e < 8; e += 2) {
    const float next = top;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(top) : "f"(next), "f"(fabsf(v[e])), "f"(fabsf(v[e + 1])));
  }
  return top;
}
// Eight activations as whole numbers of a unit, the power of two that puts the group's largest magnitude `top` between
// 2^22 / 1.004 and 8355711 (three digits of at most 127; two: 2^14 / 1.004 and 32639), so that x / unit is exact before it
// is rounded.  m: the number plus 0x808080, exclusive-or 0x808080, whose bytes are its digits -128 .. 127, lowest first.
// A group all below 2^-100 counts as 0 (its unit would leave the range of fp32).  The unit of a group with an infinity or a NaN is
// NaN and makes the token's sums NaN, whatever the digits are.
__device__ __forceinline__ void to_fixed(const float (&v)[8], float top, int pieces, float* unit, uint32_t (&m)[8]) {
  const int exponent = (__float_as_int(top * 1.00396f) >> 23) + (pieces == 3 ? 1 - 23 : 1 - 15);
  const bool some = top >= 7.8886091e-31f;
  const float inv = some ? __int_as_float((254 - exponent) << 23) : 0.0f;
  *unit = fmaf(top, 0.0f, some ? __int_as_float(exponent << 23) : 0.0f);
  if (pieces == 3) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = (static_cast<uint32_t>(__float2int_rn(v[e] * inv)) + 0x00808080u) ^ 0x00808080u;
  } else {                              // below 2^22: the sum with 1.5 * 2^23 has the rounded number in its low bits
#pragma unroll
    for (int e = 0; e < 8; ++e) m[e] = (__float_as_uint(fmaf(v[e], inv, 12582912.0f)) - 0x4B400000u + 0x00808080u) ^ 0x00808080u;
  }
}
// Digits p of the even and of the odd four.
__device__ __forceinline__ uint2 digit_of(const uint32_t (&m)[8], int p) {
  const uint32_t pick = p | (p + 4) << 4;
  return make_uint2(__byte_perm(__byte_perm(m[0], m[2], pick), __byte_perm(m[4], m[6], pick), 0x5410),
                    __byte_perm(__byte_perm(m[1], m[3], pick), __byte_perm(m[5], m[7], pick), 0x5410));
}
__device__ __forceinline__ int sum_of_eight(uint2 d) {
  return __dp4a(static_cast<int>(d.x), 0x01010101, __dp4a(static_cast<int>(d.y), 0x01010101, 0));
}

// grid: (shares of the row tiles, cluster along K, chunks of tokens)
template <int NT, int GPB, bool GATEUP, bool ZERO>
__global__ void __launch_bounds__(kThreads, 1) w4_kernel(const __grid_constant__ W4Args a) {
  constexpr int kStages = stages(NT), kStage = stage_bytes<GPB>(), kWords = 4 / GPB;
  constexpr int kLanes = 16 / GPB;      // threads that hold one group of a token's activations, eight each
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_scan[kWarps];
  __shared__ float s_coef[24];
  const Smem L = smem_of<NT, GPB>(a);
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int chunk = blockIdx.z, rank = blockIdx.y, cluster = gridDim.y;
  const int tokens = a.c.tokens, cols = a.c.cols();
  int* s_list = reinterpret_cast<int*>(smem + L.list);
  int* s_tiles = reinterpret_cast<int*>(smem + L.tiles);
  int* s_first = s_tiles + a.tiles_per_block;      // first and last warp with a part of the tile
  int* s_last = s_first + a.tiles_per_block;
  int* s_off = reinterpret_cast<int*>(smem + L.branch);
  int* s_run = s_off + a.B + 1;
  uint8_t* s_on = reinterpret_cast<uint8_t*>(s_run + a.B + 1);
  // ---- this block's K-blocks and tiles
  const int k_share = (a.kblocks + cluster - 1) / cluster;
  int n_entries = max(0, min(k_share, a.kblocks - rank * k_share));
  int n_tiles = min(a.tiles_per_block, a.tiles - static_cast<int>(blockIdx.x) * a.tiles_per_block);
  if (GATEUP || a.dense)
    for (int i = threadIdx.x; i < a.entries; i += kThreads) s_list[i] = rank * k_share + max(0, min(i, n_entries - 1));
  if (!GATEUP || a.dense)
    for (int i = threadIdx.x; i < n_tiles; i += kThreads) s_tiles[i] = blockIdx.x * a.tiles_per_block + i;
  // gate|up waits for everything before it on the stream; by the time all its blocks have passed here only gate|up
  // itself is outstanding, so the down kernel, which then may start, reads weights and selection without a wait.
  if (GATEUP) ptx::griddep_wait();
  if (GATEUP && a.status != nullptr && threadIdx.x == 0 && blockIdx.x == 0 && rank == 0 && chunk == 0) *a.status = kStatusOk;
  ptx::griddep_launch_dependents();
  if (!a.dense) {
    // what the chunk's tokens compute: [token][branch], and the branches of all of them
    for (int b = threadIdx.x; b <= a.B; b += kThreads) {
      s_off[b] = a.off[b];
      s_run[b] = b < a.B && a.alpha[b] != 0.0f;      // for now: available
    }
    const uint8_t* select = a.select != nullptr ? a.select + static_cast<int64_t>(chunk) * tokens * a.B : nullptr;
    const int n_pairs = min(tokens, a.n - chunk * tokens) * a.B;
    for (int i = threadIdx.x; i < tokens * a.B; i += kThreads) s_on[i] = i < n_pairs && (select == nullptr || select[i] != 0);
    __syncthreads();
    for (int i = threadIdx.x; i < tokens * a.B; i += kThreads) s_on[i] &= s_run[i % a.B];
    __syncthreads();
    if (!GATEUP && a.select != nullptr) {
      // c_t: the quotient and the root in double, rounded once, as the routed forward does
      for (int tok = warp; tok < tokens; tok += kWarps) {
        int k = 0, n_avail = 0;
        for (int b = lane; b < a.B; b += 32) {
          k += s_on[tok * a.B + b];
          n_avail += s_run[b];
        }
        k = __reduce_add_sync(0xFFFFFFFFu, k);
        n_avail = __reduce_add_sync(0xFFFFFFFFu, n_avail);
        if (lane == 0) s_coef[tok] = k == 0 ? 0.0f : (a.compensate ? static_cast<float>(sqrt(static_cast<double>(n_avail) / static_cast<double>(k))) : 1.0f);
      }
    }
    // running count of what is live: gate|up counts tiles branch by branch, down K-blocks with a live neuron
    int live = 0;
    if (GATEUP) {
      if (threadIdx.x < a.B) {
        for (int tok = 0; tok < tokens; ++tok) live |= s_on[tok * a.B + threadIdx.x];
        live *= (s_off[threadIdx.x + 1] - s_off[threadIdx.x]) / 8;
      }
    } else if (threadIdx.x < a.kblocks) {
      for (int b = find_branch(s_off, a.B, threadIdx.x * 128); b < a.B && s_off[b] < (static_cast<int>(threadIdx.x) + 1) * 128; ++b)
        for (int tok = 0; tok < tokens; ++tok) live |= s_on[tok * a.B + b];
    }
    int sum = live;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xFFFFFFFFu, sum, o);
      if (lane >= o) sum += u;
    }
    if (lane == 31) s_scan[warp] = sum;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kWarps; ++w) {
      if (w < warp) sum += s_scan[w];
      total += s_scan[w];
    }
    const int shares = GATEUP ? static_cast<int>(gridDim.x) : cluster, mine = GATEUP ? static_cast<int>(blockIdx.x) : rank;
    const int share = (total + shares - 1) / shares, first = mine * share;
    (GATEUP ? n_tiles : n_entries) = max(0, min(share, total - first));
    if (GATEUP) {
      if (threadIdx.x < a.B) s_run[threadIdx.x] = sum - live;      // live tiles before the branch
    } else if (live && sum - 1 >= first && sum - 1 < first + n_entries) {
      s_list[sum - 1 - first] = threadIdx.x;
    }
    __syncthreads();
    if (GATEUP) {
      for (int i = threadIdx.x; i < n_tiles; i += kThreads) {
        // the last branch with at most `first + i` live tiles before it: a branch without any shares its count with the next
        const int b = find_branch(s_run, a.B, first + i);
        s_tiles[i] = s_off[b] / 8 + first + i - s_run[b];
      }
    } else if (threadIdx.x < a.entries && static_cast<int>(threadIdx.x) >= n_entries && n_entries > 0) {
      s_list[threadIdx.x] = s_list[n_entries - 1];
    }
  }
  __syncthreads();

  // ---- this warp's run of steps (tile, two K-blocks)
  const int steps = (n_entries + 1) / 2;
  const int per_warp = (n_tiles * steps + kWarps - 1) / kWarps;
  const int run_begin = min(n_tiles * steps, warp * per_warp);
  const int count = min(n_tiles * steps, run_begin + per_warp) - run_begin;
  const int tile_begin = steps > 0 ? run_begin / steps : 0, step_begin = run_begin - tile_begin * steps;

  // ---- copies of one stage: of codes, eight lanes take the 64 bytes of a row in both K-blocks (a whole line where they
  // are neighbours), four rows at a time; scales and zeros by the first lanes
  const uint32_t ring = ptx::smem_u32(smem) + warp * kStages * kStage;
  const int c_row = lane >> 3, c_block = (lane >> 2) & 1;
  uint32_t q_dst[2];                    // rows c_row and c_row + 4 of a half
#pragma unroll
  for (int r = 0; r < 2; ++r) q_dst[r] = ring + c_block * 1024 + (c_row + 4 * r) * 64 + (t ^ (((c_row + 4 * r) >> 1) & 3)) * 16;
  const int s_block = (lane / (2 * GPB)) & 1, s_half = (lane / GPB) & 1, s_group = lane % GPB;   // lanes below 4 GPB
  const bool s_lane = lane < 4 * GPB;
  const uint8_t* const z_base = ZERO && s_lane ? (s_half ? a.m[1].zero : a.m[0].zero) : nullptr;
  const __nv_bfloat16* const s_base = s_half ? a.m[1].scale : a.m[0].scale;
  const uint32_t last_byte = static_cast<uint32_t>(a.m[0].pitch) - 16, last_group = static_cast<uint32_t>(a.m[0].n_groups) - 1;
  const uint32_t rows16 = static_cast<uint32_t>(a.m[0].rows16);
  // Rows past the last, K-blocks past the last and columns past K are read from the nearest valid place: their results
  // are not used, or their digits and units are 0.
  const uint8_t* q_src[2][2];           // [half][row]
  uint32_t s_row = 0;
  int i_tile = tile_begin, i_step = step_begin, i_left = count;
  if (ZERO && s_lane && z_base == nullptr) {         // a half without stored zeros beside one with them: 8 in every slot, for good
    for (int i = 0; i < kStages; ++i)
      *reinterpret_cast<uint2*>(smem + (warp * kStages + i) * kStage + 2048 + 4 * GPB * 16 + lane * 8) = make_uint2(0x08080808u, 0x08080808u);
  }
  bool open = true;
  auto issue = [&](int slot) {
    if (i_left > 0) {
      if (open) {                       // the first step of a tile
        const int tile = s_tiles[i_tile];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const int row = c_row + 4 * r + (GATEUP ? tile * 8 : min(tile * 16 + 8 * h, a.rows - 8));
            q_src[h][r] = a.m[h].q + row * a.m[h].pitch;
          }
        s_row = static_cast<uint32_t>(GATEUP ? tile * 8 : min(tile * 16 + 8 * s_half, a.rows - 8));
      }
      const uint2 kb = *reinterpret_cast<const uint2*>(s_list + 2 * i_step);
      const uint32_t byte = min((c_block == 0 ? kb.x : kb.y) * 64 + t * 16, last_byte);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) cp_async16(q_dst[r] + slot * kStage + h * 512, q_src[h][r] + byte);
      if (s_lane) {
        const uint32_t at = min((s_block == 0 ? kb.x : kb.y) * GPB + s_group, last_group) * rows16 + s_row;
        cp_async16(ring + slot * kStage + 2048 + lane * 16, s_base + at);
        if (ZERO && z_base != nullptr) cp_async8(ring + slot * kStage + 2048 + 4 * GPB * 16 + lane * 8, z_base + at);
      }
      --i_left;
      open = ++i_step == steps;
      if (open) {
        i_step = 0;
        ++i_tile;
      }
    }
    cp_async_commit();
  };

  // ---- the activations of this block's K-blocks as digits: a thread takes eight k of one token, the group's kLanes
  // threads are neighbours; four such loads are under way at a time
  uint2* s_x = reinterpret_cast<uint2*>(smem + L.x);
  float2* s_unit = reinterpret_cast<float2*>(smem + L.unit);
  const int even_entries = 2 * steps, units_per_token = even_entries * 16;
  const int kind = GATEUP ? a.x_kind : MLPMOE_FP32;
  // unit i of token tok; units_per_token is a multiple of 32, so a warp stays inside a token and is whole
  constexpr int kBatch = NT == 1 ? 4 : 2;          // what the registers hold
  Raw raw[kBatch];
  int toks[kBatch], is[kBatch], tok_next = 0, i_next = threadIdx.x;
  auto load_activations = [&]() {
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      while (tok_next < tokens && i_next >= units_per_token) i_next -= units_per_token, ++tok_next;
      toks[u] = tok_next;
      is[u] = i_next;
      i_next += kThreads;
      raw[u].lo = raw[u].hi = make_uint4(0u, 0u, 0u, 0u);
      if (toks[u] < tokens) {
        const int entry = is[u] >> 4, k = s_list[entry] * 128 + (is[u] & 15) * 8, token = chunk * tokens + toks[u];
        bool in = entry < n_entries && k < a.K && token < a.n;
        // what the token does not compute is 0, and gate|up may have left it unwritten
        if (!GATEUP && in && !a.dense) in = s_on[toks[u] * a.B + find_branch(s_off, a.B, k)] != 0;
        if (in) raw[u] = load_raw(a.x, kind, token * a.x_stride + k);
      }
    }
  };
  auto stage_activations = [&]() {
    for (int i = threadIdx.x; i < even_entries * GPB * NT * 8; i += kThreads)
      if (i % (NT * 8) >= cols) s_unit[i] = make_float2(0.0f, 0.0f);
    if (!GATEUP) {
      ptx::griddep_wait();              // h is complete
      load_activations();
    }
    while (toks[0] < tokens) {
#pragma unroll
      for (int u = 0; u < kBatch; ++u) {
        if (toks[u] >= tokens) break;
        const int k8 = is[u] & 15, entry = is[u] >> 4;
        float v[8];
        to_f32(raw[u], kind, v);
        float top = largest(v);
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) top = larger(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        float unit;
        uint32_t m[8];
        to_fixed(v, top, a.c.pieces, &unit, m);
        const int j = k8 / kLanes, word = unit_word<GPB>(k8);
        if (GATEUP && a.x_scale != nullptr && k8 % kLanes == 0 && s_list[entry] * 128 + k8 * 8 < a.K && chunk * tokens + toks[u] < a.n) {
          const int xg = a.x_groups == 1 ? 0 : (s_list[entry] * GPB + j) >> a.x_shift;
          unit *= a.x_scale[static_cast<int64_t>(chunk * tokens + toks[u]) * a.x_groups + xg];
        }
        uint2* out = s_x + (((entry * 2 + (word >> 1)) * (NT * 8) + toks[u]) * 4 + unit_lane<GPB>(k8)) * 2 + (word & 1);
        float2* units = s_unit + (entry * GPB + j) * (NT * 8) + toks[u];
        const uint2 d0 = digit_of(m, 0), d1 = digit_of(m, 1);
        // a sum over 128 digits fits in 16 bits: two digits' sums in one word
        int sums01 = sum_of_eight(d0) + (sum_of_eight(d1) << 16);
#pragma unroll
        for (int o = 1; o < kLanes; o *= 2) sums01 += __shfl_xor_sync(0xFFFFFFFFu, sums01, o);
        const int sum0 = static_cast<int16_t>(sums01), sum1 = (sums01 - sum0) >> 16;
        out[0] = d0;
        out[tokens * 8] = d1;
        if (k8 % kLanes == 0) {
          units[0] = make_float2(unit, __int_as_float(-sum0));
          units[tokens] = make_float2(unit * 256.0f, __int_as_float(-sum1));
        }
        if (a.c.pieces == 3) {
          const uint2 d2 = digit_of(m, 2);
          int sum2 = sum_of_eight(d2);
#pragma unroll
          for (int o = 1; o < kLanes; o *= 2) sum2 += __shfl_xor_sync(0xFFFFFFFFu, sum2, o);
          out[2 * tokens * 8] = d2;
          if (k8 % kLanes == 0) units[2 * tokens] = make_float2(unit * 65536.0f, __int_as_float(-sum2));
        }
      }
      load_activations();
    }
    __syncthreads();
  };
  if (GATEUP) load_activations();       // on their way before the weights

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

  // turns below 0 fill the ring, and the activations are staged while the first copies are under way: one copy of the
  // code of `issue`, since a block runs it cold
  int slot = 0, c_tile = tile_begin, c_step = step_begin;
  bool from_start = step_begin == 0;    // the run holds the current tile's first step
#pragma unroll 1
  for (int i = 1 - kStages; i < count; ++i) {
    if (i >= 0) cp_async_wait<kStages - 2>();
    __syncwarp();                       // the stage is in shared memory for all lanes, and the slot before it has been read by all
    const uint8_t* st = smem + (warp * kStages + slot) * kStage;
    issue(i < 0 ? i + kStages - 1 : (slot == 0 ? kStages - 1 : slot - 1));
    if (i < 0) {
      if (i == -1) stage_activations();
      continue;
    }
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
      // - zero * sum of digits first, then the codes' products; on top of the bits of 12582912 = 1.5 * 2^23, so that the bits
      // of the result (at most 15 * 128 * 128 in magnitude) are those of 12582912 + result in fp32
      const float4* up = reinterpret_cast<const float4*>(s_unit + ((2 * c_step) * GPB + j) * (NT * 8)) + t;
      int part[NT][4];
      float2 unit[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const float4 u = up[nt * 4];
        unit[nt] = make_float2(u.x, u.z);
        part[nt][0] = zero[0] * __float_as_int(u.y) + 0x4B400000;
        part[nt][1] = zero[0] * __float_as_int(u.w) + 0x4B400000;
        part[nt][2] = ZERO ? zero[1] * __float_as_int(u.y) + 0x4B400000 : part[nt][0];
        part[nt][3] = ZERO ? zero[1] * __float_as_int(u.w) + 0x4B400000 : part[nt][1];
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
      if (!GATEUP && !a.dense && !(is_finite(s[0]) && is_finite(s[1]))) {
        // perhaps a branch's that some token does not compute: nothing of it enters where the activations are 0
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float u = i & 1 ? unit[nt].y : unit[nt].x;
            if (u != 0.0f) acc[nt][i] += (__int_as_float(part[nt][i]) - 12582912.0f) * (s[i / 2] * u);
          }
      } else {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          acc[nt][0] += (__int_as_float(part[nt][0]) - 12582912.0f) * (s[0] * unit[nt].x);
          acc[nt][1] += (__int_as_float(part[nt][1]) - 12582912.0f) * (s[0] * unit[nt].y);
          acc[nt][2] += (__int_as_float(part[nt][2]) - 12582912.0f) * (s[1] * unit[nt].x);
          acc[nt][3] += (__int_as_float(part[nt][3]) - 12582912.0f) * (s[1] * unit[nt].y);
        }
      }
    }
    slot = slot + 1 == kStages ? 0 : slot + 1;
    if (++c_step == steps || i + 1 == count) {      // the run leaves this tile: its part of the tile's sums
      if (lane == 0 && from_start) s_first[c_tile] = warp;
      if (lane == 0 && c_step == steps) s_last[c_tile] = warp;
      from_start = true;
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

  // ---- a warp takes a tile, its half-warps a token each: the parts of the warps that worked on the tile, in order, and
  // the digits of the token
  const int row = lane & 15, half = lane >> 4;
  float* own = reinterpret_cast<float*>(smem);       // of a cluster: this block's sums, over the ring
  auto sum_of = [&](int w0, int w1, int tile, int tok) {
    float v = 0.0f;
    for (int w = w0; w <= w1; ++w) {
      const float* p = sums + (w + tile) * (NT * 8 * kColPitch) + row;
      for (int c = tok; c < cols; c += tokens) v += p[c * kColPitch];
    }
    return v;
  };
  if (cluster > 1) {
    for (int tile = warp; tile < n_tiles; tile += kWarps) {
      const int w0 = steps > 0 ? s_first[tile] : 0, w1 = steps > 0 ? s_last[tile] : -1;
      for (int tok = half; tok < tokens; tok += 2) own[(tile * tokens + tok) * 16 + row] = sum_of(w0, w1, tile, tok);
    }
    __syncthreads();
    ptx::cluster_sync_all();
  }
  for (int tile = rank * kWarps + warp; tile < n_tiles; tile += cluster * kWarps) {
    const int w0 = steps > 0 ? s_first[tile] : 0, w1 = steps > 0 ? s_last[tile] : -1;
    const int place = s_tiles[tile];
    const int b = GATEUP ? find_branch(a.off, a.B, place * 8) : 0;
    for (int tok0 = half; tok0 < tokens + half; tok0 += 8) {                // whole warps; four tokens' loads under way together
      float v[4], up[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int tok = tok0 + 2 * u;
        v[u] = 0.0f;
        if (tok < tokens) {
          if (cluster == 1) {
            v[u] = sum_of(w0, w1, tile, tok);
          } else {
            float part[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) part[r] = r < cluster ? ld_cluster_f32(own + (tile * tokens + tok) * 16 + row, r) : 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) v[u] += part[r];
          }
        }
      }
      if (GATEUP) {
#pragma unroll
        for (int u = 0; u < 4; ++u) up[u] = __shfl_down_sync(0xFFFFFFFFu, v[u], 8);      // rows 8..15 are the up rows of rows 0..7
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int tok = tok0 + 2 * u, token = chunk * tokens + tok;
        if (tok >= tokens || token >= a.n) break;
        if (GATEUP) {
          if (row >= 8) break;
          const bool on = a.dense || s_on[tok * a.B + b] != 0;
          a.h[static_cast<int64_t>(token) * a.rows + place * 8 + row] = on ? v[u] / (1.0f + expf(-v[u])) * up[u] * a.alpha[b] : 0.0f;
        } else {
          const int m = place * 16 + row;
          if (m >= a.rows) break;
          if (a.select != nullptr) v[u] *= s_coef[tok];
          const int64_t at = static_cast<int64_t>(token) * a.rows + m;
          if (a.residual != nullptr) v[u] += a.residual[at];
          if (a.y_bf16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v[u]);
          else static_cast<float*>(a.y)[at] = v[u];
        }
      }
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
  // the same for every call: the limit is the kernel's, and another thread's call may come between here and the launch
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMax);
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
