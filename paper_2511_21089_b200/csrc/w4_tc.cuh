// The layer on 4-bit weights for batches large enough for the 5th-generation tensor cores (y in bf16).
//
// The codes become fp16 whole numbers code - zero (exact) in tensor memory, where tcgen05.mma takes its first operand
// from; the activations come as its second, 128-byte-swizzled in shared memory: fp16 times a unit, a power of two of the token
// (x) or of the token and 128 columns (the intermediate activation, whose row is not known as a whole when it is
// written) that brings the largest to 2^14..2^15.  What is below 2^-28 of the largest loses bits; the rest is rounded to
// 2^-11 (not at all for x in bf16), where y is rounded to 2^-8.  The products of one group of K (32, 64 or 128 columns)
// accumulate in tensor memory too.  Two accumulators alternate: while the tensor core fills one, the epilogue warps read
// the other back and add it, times the row's scale, to their fp32 sums in registers.
//
// What bounds these kernels up to 64 tokens is the conversion of the codes (1.1 instructions a code of the 3.5 that a block's
// warps issue, at 2.2 a cycle), not the copy (floor of the Llama-shaped layer 14.5 us) nor the MMAs: before the last step below
// 128 columns of K took 1450 cycles of which the MMAs run 580 (gate|up), 1100 and 290 (down).  Measured there, 64 tokens,
// group 128 with zeros: 53 us (each alone, with cold caches: columns 6, gate|up 33, down 27).  On the way: the operand in shared
// memory (64 KB written and read for each 128 columns of K), waits that read the timer at once, and MMAs issued under
// `lane == 0` 99 us; the operand in tensor memory, the rest as it was 94; codes through a ring of copies instead of registers
// 82; scales through a ring too 70; waits that read the timer late 58; copies issued by three warps 56; an operand stage for
// each matrix and paired sums 53.  Tried without gain: stages of half a block of K, reading the next codes while tensor
// memory takes the last.  Down with more than 64 tokens a chunk spills 72 to 116 bytes a thread.
//
// A block: 128 neurons (128 gate rows and 128 up rows) or 128 rows of W_down.  Warps 0..7 epilogue (tensor memory lanes
// 32 (warp % 4).., columns NE (warp / 4)..), 8..15 codes to fp16 (the same lanes), 16 issues the MMAs, 17 copies the
// codes, 18 scales and zeros, 19 the activations.
#pragma once
#include "w4_wide.cuh"

namespace mlpmoe {
namespace w4 {

constexpr int kTcThreads = 20 * 32;

template <int NE, int GPB, bool GATEUP>
struct TcCfg {
  static constexpr int kMats = GATEUP ? 2 : 1;
  static constexpr int kCols = GATEUP ? NE : 2 * NE;             // columns of an MMA
  // Tensor memory: two accumulators of 2 NE columns, then the first operand's stages, each 64 columns: a block of K of one
  // matrix, two values a column.
  static constexpr int kOperands = 4 * NE, kFit = (512 - kOperands) / 64 / kMats, kStages = kFit < 4 ? kFit : 4;      // of each matrix
  static constexpr int kB = kCols * 256;
  // Shared memory: stages of one block of K, each the activations, the codes, scales and zeros of 128 rows and the units.
  static constexpr int kCodes = kB, kScales = kCodes + kMats * 8192, kZeros = kScales + kMats * GPB * 256, kUnits = kZeros + kMats * GPB * 128;
  static constexpr int kStage = (kUnits + (GATEUP ? 0 : kCols * 4) + 1023) / 1024 * 1024;
  static constexpr int kMost = (232448 - 6144) / kStage, kRing = kMost < 8 ? kMost : 8;
  static constexpr int kSums = 2 * NE * 128 * 4;                 // [column][row], over the stages at the end
  static constexpr int kBars = kRing * kStage > kSums ? kRing * kStage : kSums;
  static constexpr int kSmem = kBars + 512 + 1024;               // barriers, slack for 1024-byte alignment
};

// Eight codes -> four fp16 pairs code - zero, pairs (e, e + 4) of eight consecutive columns, by the widely used conversion of small
// whole numbers to floats through the mantissa: the code slides into that of 1024.0, as it is or times 16, which a multiplication by 1/16 takes back: one shift for two pairs.  All of it is exact.
// bias = -(1024 + zero) and -(64 + zero), twice each.
struct Bias {
  __half2 one, sixteen;
};
__device__ __forceinline__ Bias bias_of(uint32_t zero) {
  const uint32_t bits = 0xE400E400u + zero * 0x00010001u;
  const __half2 one = *reinterpret_cast<const __half2*>(&bits);
  return {one, __hadd2(one, __floats2half2_rn(960.0f, 960.0f))};
}
__device__ __forceinline__ void unpack_f16(uint32_t w, const Bias& bias, uint32_t* p) {
  const __half2 sixteenth = __floats2half2_rn(0.0625f, 0.0625f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t from = i < 2 ? w : w >> 8;
    uint32_t u;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(from), "r"(i % 2 ? 0x00F000F0u : 0x000F000Fu), "r"(0x64006400u));
    const __half2 v = *reinterpret_cast<const __half2*>(&u), o = i % 2 ? __hfma2(v, sixteenth, bias.sixteen) : __hadd2(v, bias.one);
    p[i] = *reinterpret_cast<const uint32_t*>(&o);
  }
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi));
  return v;
}
__device__ __forceinline__ uint64_t mul2(uint64_t x, uint64_t y) {
  uint64_t v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(x), "l"(y));
  return v;
}
__device__ __forceinline__ uint64_t fma2(uint64_t x, uint64_t y, uint64_t z) {
  uint64_t v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(x), "l"(y), "l"(z));
  return v;
}

// Sums of a row whose scale is not finite, perhaps of a branch that some tokens do not compute: nothing of it enters those whose
// product with the activations is 0.
template <int N>
__device__ __forceinline__ void add_where_not_zero(uint64_t* acc, const uint32_t (&r)[N], float s, const float* unit) {
#pragma unroll
  for (int k = 0; k < N; k += 2) {
    const float2 u = *reinterpret_cast<const float2*>(unit + k);
    const float v0 = __uint_as_float(r[k]), v1 = __uint_as_float(r[k + 1]);
    acc[k / 2] = fma2(pair(v0, v1), pair(v0 != 0.0f ? s * u.x : 0.0f, v1 != 0.0f ? s * u.y : 0.0f), acc[k / 2]);
  }
}

// The unit for values of at most `top`, and its reciprocal.  Infinities and NaN pass through.
__device__ __forceinline__ float unit_of(float top, float* inverse) {
  const int e = min(max(static_cast<int>(__float_as_uint(top) >> 23), 32), 255);      // biased exponent; 2^-95 and below share a unit
  const bool one = e == 255;
  *inverse = one ? 1.0f : __uint_as_float(static_cast<uint32_t>(268 - e) << 23);        // 2^(14 - (e - 127))
  return one ? 1.0f : __uint_as_float(static_cast<uint32_t>(e - 14) << 23);
}

// Eight k's as part of row c of an image's half.
__device__ __forceinline__ void store_column(uint8_t* half, int c, int k8, const float* v, float inverse) {
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const __half2 pair = __floats2half2_rn(v[e] * inverse, v[e + 4] * inverse);
    o[e] = *reinterpret_cast<const uint32_t*>(&pair);
  }
  *reinterpret_cast<uint4*>(half + c * 128 + (((k8 & 7) ^ (c & 7)) * 16)) = make_uint4(o[0], o[1], o[2], o[3]);
}

// x as the MMAs' second operand: per chunk and K-block, two halves of 64 columns of K, each `cols` rows of 128 bytes under the
// 128-byte swizzle; a row is a token.  A block takes one token, a thread eight k at a time; the second reading is from the
// caches.
static __global__ void __launch_bounds__(256) w4_columns_kernel(const __grid_constant__ W4ColumnsArgs a) {
  __shared__ float s_top[8];
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t token = blockIdx.x;
  if (a.status != nullptr && token == 0 && threadIdx.x == 0) *a.status = kStatusOk;
  auto load = [&](int u, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    if (u * 8 < a.K) {
      to_f32(load_raw(a.x, a.kind, token * a.stride + u * 8), a.kind, v);
      if (a.x_scale != nullptr) {
        const float s = a.x_scale[token * a.x_groups + (a.x_groups == 1 ? 0 : u * 8 / a.x_group)];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= s;
      }
    }
  };
  float top = 0.0f;
  for (int u = threadIdx.x; u * 8 < a.K; u += 256) {
    float v[8];
    load(u, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  if (threadIdx.x % 32 == 0) s_top[threadIdx.x / 32] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) top = fmaxf(top, s_top[w]);
  float inverse;
  const float unit = unit_of(top, &inverse);
  if (threadIdx.x == 0) a.unit[token] = unit;
  const int chunk = static_cast<int>(token / a.tokens), c = static_cast<int>(token % a.tokens);
  for (int u = threadIdx.x; u < a.kblocks * 16; u += 256) {
    float v[8];
    load(u, v);
    store_column(a.image + ((static_cast<int64_t>(chunk) * a.kblocks + u / 16) * 2 + (u >> 3 & 1)) * (a.cols * 128), c, u & 15, v, inverse);
  }
}

// What a block writes, from the [column][row] sums of all CL blocks of its cluster.  A thread takes eight rows of one token.
template <int CL, int NE, bool GATEUP>
__device__ __forceinline__ void tc_outputs(const W4TcArgs& a, const float* sums, const float* factor) {
  const int chunk = blockIdx.z, rank = blockIdx.y, n_here = min(a.tokens, a.n - chunk * a.tokens);
  auto total_of = [&](int col, int r, float* v) {
    const float* at = sums + col * 128 + r;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    constexpr int kAtOnce = CL < 4 ? CL : 4;
#pragma unroll
    for (int k0 = 0; k0 < CL; k0 += kAtOnce) {
      float4 part[kAtOnce][2];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q) part[k][q] = CL == 1 ? reinterpret_cast<const float4*>(at)[q] : ld_cluster_f32x4(at + 4 * q, k0 + k);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          v[4 * q] += part[k][q].x;
          v[4 * q + 1] += part[k][q].y;
          v[4 * q + 2] += part[k][q].z;
          v[4 * q + 3] += part[k][q].w;
        }
    }
  };
  for (int i = rank * kTcThreads + threadIdx.x; i < n_here * 16; i += CL * kTcThreads) {
    const int tok = i >> 4, k8 = i & 15, row = blockIdx.x * 128 + 8 * k8, token = chunk * a.tokens + tok;
    float v[8];
    if (GATEUP) {
      bool on = row < a.rows;
      const int b = find_branch(a.off, a.B, row);             // the eight rows are one branch's: its width is a multiple of 16
      const float alpha = a.alpha[b];
      on = on && alpha != 0.0f && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
      if (on) {
        float up[8];
        const float unit = factor[tok];
        total_of(tok, 8 * k8, v);
        total_of(NE + tok, 8 * k8, up);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float gate = v[e] * unit;
          // __expf is off by 2 + 1.2 |gate| units in the last place, the quotient by 2; with expf and the exact quotient these
          // lines took a quarter of what the block spends behind its last product
          v[e] = __fdividef(gate, 1.0f + __expf(-gate)) * (up[e] * unit) * alpha;
        }
      }
      // these 128 rows are one block of the down product's K; a token's 16 threads are one half of a warp
      float top = 0.0f, inverse;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFu << (threadIdx.x & 16), top, o));
      const float unit = unit_of(top, &inverse);
      const int64_t block = static_cast<int64_t>(token / a.h_tokens) * gridDim.x + blockIdx.x;
      const int c = token % a.h_tokens;
      store_column(a.h + (block * 2 + (k8 >> 3)) * (a.h_cols * 128), c, k8, v, inverse);
      if (k8 == 0) a.h_unit[block * a.h_cols + c] = unit;
    } else if (row < a.rows) {
      total_of(tok, 8 * k8, v);
      const int64_t at = static_cast<int64_t>(token) * a.rows + row;
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (a.select != nullptr) v[e] *= factor[tok];
        if (a.residual != nullptr) v[e] += a.residual[at + e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 pair = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        o[e] = *reinterpret_cast<const uint32_t*>(&pair);
      }
      *reinterpret_cast<uint4*>(a.y + at) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// grid: (blocks of 128 rows, cluster along K, chunks)
// MASKED: down where a token may leave out branches; their scales need not be finite.
template <int NE, int GPB, bool GATEUP, bool ZERO, bool MASKED>
__global__ void __launch_bounds__(kTcThreads, 1) w4_tc_kernel(const __grid_constant__ W4TcArgs a) {
  using C = TcCfg<NE, GPB, GATEUP>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int s_list[kW4MaxDim / 128];
  __shared__ int s_n;
  __shared__ float s_factor[128];                 // per token: gate|up x's unit, down the selection's factor
  __shared__ uint8_t s_live[kW4MaxBranches];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* full_a = reinterpret_cast<uint64_t*>(smem + C::kBars);
  uint64_t* empty_a = full_a + C::kMats * C::kStages;
  uint64_t* full = empty_a + C::kMats * C::kStages;
  uint64_t* empty = full + C::kRing;
  uint64_t* d_full = empty + C::kRing;
  uint64_t* d_empty = d_full + 2;
  uint64_t* drained = d_empty + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drained + 1);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int chunk = blockIdx.z, rank = blockIdx.y, cluster = gridDim.y;
  const int row0 = blockIdx.x * 128;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kMats * C::kStages; ++s) {
      ptx::mbar_init(&full_a[s], 8 / C::kMats + a.extra_arrivals);
      ptx::mbar_init(&empty_a[s], 1);
    }
    for (int s = 0; s < C::kRing; ++s) {
      ptx::mbar_init(&full[s], 3);
      ptx::mbar_init(&empty[s], 17);              // eight warps of either kind, and the MMAs
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&d_full[b], 1);
      ptx::mbar_init(&d_empty[b], 8);
    }
    ptx::mbar_init(drained, 1);
    *abort_flag = 0;
    ptx::fence_barrier_init();
  }
  // 61,440 of an SM's 65,536 registers are this block's: no second block that takes tensor memory fits beside it, so the
  // allocation waits for nobody who waits for this cluster.
  if (warp == 16) {
    ptx::tmem_alloc(tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  const int n_entries = list_kblocks<GATEUP>(a.kblocks, cluster, rank, a.dense, a.select, chunk, a.tokens, a.n, a.B, a.off, a.alpha, s_list,
                                             s_live, &s_n);
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  // the kernel before this one passed its own wait before this one could start: weights and selection may be read
  ptx::griddep_launch_dependents();

  if (warp < 8) {
    // ------------------------------------------------------------- sums of the groups
    if (!GATEUP && a.select != nullptr && threadIdx.x < 128 && chunk * a.tokens + static_cast<int>(threadIdx.x) < min(a.n, (chunk + 1) * a.tokens))
      s_factor[threadIdx.x] = token_factor(a.select + (static_cast<int64_t>(chunk) * a.tokens + threadIdx.x) * a.B, a.alpha, a.B, a.compensate);
    const int quad = warp % 4, half = warp / 4;
    const int steps = n_entries * GPB;
    const int at_scale = C::kScales + (GATEUP ? half * GPB * 256 : 0) + (quad * 32 + lane) * 2, at_unit = C::kUnits + half * NE * 4;
    int stage = 0;
    uint32_t phase = 0;
    uint64_t acc[NE / 2];                         // pairs of fp32
#pragma unroll
    for (int i = 0; i < NE / 2; ++i) acc[i] = 0;
    const uint32_t taddr = tmem + static_cast<uint32_t>(half * NE) + (static_cast<uint32_t>(quad * 32) << 16);
    for (int step = 0; step < steps; ++step) {
      bool ok = step % GPB != 0 || ptx::mbar_wait_bounded(&full[stage], phase, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const uint8_t* in = smem + stage * C::kStage;
      const float s = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(in + at_scale + step % GPB * 256));
      const bool odd = MASKED && !is_finite(s), some_odd = MASKED && NE == 64 && __any_sync(0xFFFFFFFFu, odd);
      const int b = step & 1;
      ok = ptx::mbar_wait_bounded(&d_full[b], (step >> 1) & 1, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      ptx::tc_fence_after();
      if (some_odd) {                             // for the warp, before the loop: 64 columns leave no registers for a branch in it
#pragma unroll
        for (int i = 0; i < NE; i += 8) {
          uint32_t r[8];
          ptx::tmem_ld_32x8(taddr + b * 2 * NE + i, r);
          ptx::tmem_ld_wait();
          add_where_not_zero(acc + i / 2, r, s, reinterpret_cast<const float*>(in + at_unit) + i);
        }
      }
      constexpr int kPart = NE == 64 ? (GATEUP ? 16 : 8) : 32;   // what the registers hold beside the sums
#pragma unroll
      for (int i = 0; i < NE; i += kPart) {
        if (some_odd) break;
        uint32_t r[kPart];
        if constexpr (kPart == 32) ptx::tmem_ld_32x32(taddr + b * 2 * NE + i, r);
        else if constexpr (kPart == 16) ptx::tmem_ld_32x16(taddr + b * 2 * NE + i, r);
        else ptx::tmem_ld_32x8(taddr + b * 2 * NE + i, r);
        ptx::tmem_ld_wait();
        if (NE == 32 && odd) {
          add_where_not_zero(acc + i / 2, r, s, reinterpret_cast<const float*>(in + at_unit) + i);
          continue;
        }
#pragma unroll
        for (int k = 0; k < kPart; k += 4) {
          uint64_t s0 = pair(s, s), s1 = s0;
          if constexpr (!GATEUP) {                // a scale (8 bits) times a power of two is exact
            const float4 u = *reinterpret_cast<const float4*>(in + at_unit + (i + k) * 4);
            s0 = mul2(s0, pair(u.x, u.y));
            s1 = mul2(s1, pair(u.z, u.w));
          }
          acc[(i + k) / 2] = fma2(pair(__uint_as_float(r[k]), __uint_as_float(r[k + 1])), s0, acc[(i + k) / 2]);
          acc[(i + k) / 2 + 1] = fma2(pair(__uint_as_float(r[k + 2]), __uint_as_float(r[k + 3])), s1, acc[(i + k) / 2 + 1]);
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&d_empty[b]);
      if (step % GPB == GPB - 1) {
        if (lane == 0) ptx::mbar_arrive(&empty[stage]);
        if (++stage == C::kRing) stage = 0, phase ^= 1u;
      }
    }
    __syncwarp();
    // every MMA of the block is complete once the last accumulator was, and no copy is under way: once the eight warps have
    // read the last scales the stages are free
    asm volatile("bar.sync 1, 256;" ::: "memory");
    float* sums = reinterpret_cast<float*>(smem) + half * NE * 128 + quad * 32 + lane;      // [column][row]
#pragma unroll
    for (int i = 0; i < NE; i += 2) {
      sums[i * 128] = __uint_as_float(static_cast<uint32_t>(acc[i / 2]));
      sums[(i + 1) * 128] = __uint_as_float(static_cast<uint32_t>(acc[i / 2] >> 32));
    }
  } else if (warp < 16) {
    // ------------------------------------------------------------- codes to fp16
    // gate|up: a warp takes 32 rows of one matrix; down: of half of the columns.  32 columns (16 bytes) at a time.
    constexpr int kChunks = 4 / (3 - C::kMats), kZeros = GPB * kChunks > 4 ? GPB * kChunks / 4 : 1;      // groups that the warp's columns touch
    const int quad = warp % 4, part = (warp - 8) / 4, chunk0 = GATEUP ? 0 : 2 * part, r = quad * 32 + lane;
    const bool has_zero = ZERO && a.m[GATEUP ? part : 0].zero != nullptr;
    const int at_codes = C::kCodes + (GATEUP ? part * 8192 : 0) + r * 64;
    const int at_zero = C::kZeros + (GATEUP ? part * GPB * 128 : chunk0 * GPB / 4 * 128) + r;
    const uint32_t to = tmem + C::kOperands + (GATEUP ? part * C::kStages * 64 : part * 32) + (static_cast<uint32_t>(quad * 32) << 16);
    uint64_t* full_mine = full_a + (GATEUP ? part * C::kStages : 0);
    uint64_t* empty_mine = empty_a + (GATEUP ? part * C::kStages : 0);
    int stage = 0, slot = 0;
    uint32_t phase = 0, slot_phase = 0;
    bool ok = true;
    for (int e = 0; ok && e < n_entries; ++e) {
      ok = ptx::mbar_wait_bounded(&full[slot], slot_phase, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      const uint8_t* in = smem + slot * C::kStage;
      uint4 c[kChunks];
#pragma unroll
      for (int i = 0; i < kChunks; ++i) c[i] = *reinterpret_cast<const uint4*>(in + at_codes + (((chunk0 + i) ^ (r >> 1 & 3)) * 16));
      Bias bias[kZeros];
#pragma unroll
      for (int j = 0; j < kZeros; ++j) bias[j] = bias_of(has_zero ? in[at_zero + j * 128] : 8u);
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&empty[slot]);
      if (++slot == C::kRing) slot = 0, slot_phase ^= 1u;
      ok = ptx::mbar_wait_bounded(&empty_mine[stage], phase ^ 1u, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      ptx::tc_fence_after();
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const uint32_t w[4] = {c[i].x, c[i].y, c[i].z, c[i].w};
        uint32_t p[16];
#pragma unroll
        for (int k = 0; k < 4; ++k) unpack_f16(w[k], bias[i * kZeros / kChunks], p + 4 * k);
        ptx::tmem_st_32x16(to + stage * 64 + i * 16, p);
      }
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&full_mine[stage]);
      if (++stage == C::kStages) stage = 0, phase ^= 1u;
    }
  } else if (warp == 16) {
    // ------------------------------------------------------------- MMAs
    if (ptx::elect_one()) {
      constexpr uint32_t idesc = ptx::make_idesc_f16_f32(128, C::kCols);
      constexpr int kSteps = 8 / GPB;             // of 16 columns, in a group
      int stage = 0, slot = 0, d = 0;
      uint32_t phase = 0, d_phase = 0;
      bool ok = true;
      for (int e = 0; ok && e < n_entries; ++e) {
        const uint32_t sb = ptx::smem_u32(smem + slot * C::kStage);
#pragma unroll
        for (int j = 0; j < GPB; ++j) {
          ok = ptx::mbar_wait_bounded(&d_empty[d], d_phase ^ 1u, abort_flag, a.wait_limit_ns);
#pragma unroll
          for (int mat = 0; mat < C::kMats; ++mat) {
            // the warps that made the operand have seen the stage's copies complete
            if (j == 0) ok = ok && ptx::mbar_wait_bounded(&full_a[mat * C::kStages + stage], phase, abort_flag, a.wait_limit_ns);
            if (!ok) break;
            ptx::tc_fence_after();
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
              // 16 columns of K: eight columns of tensor memory; in the swizzled 128-byte row +32 bytes = +2 in the descriptor's
              // address field
              const int ks = j * kSteps + k;
              const uint64_t db = ptx::make_desc_sw128_kmajor(sb + (ks >> 2) * (C::kCols * 128)) + 2 * (ks & 3);
              ptx::umma_f16_ts(tmem + d * 2 * NE + mat * C::kCols, tmem + C::kOperands + (mat * C::kStages + stage) * 64 + ks * 8, db, idesc,
                               k != 0 ? 1u : 0u);
            }
            if (j == GPB - 1) ptx::umma_commit(&empty_a[mat * C::kStages + stage]);
          }
          if (!ok) break;
          ptx::umma_commit(&d_full[d]);
          if (++d == 2) d = 0, d_phase ^= 1u;
        }
        if (!ok) break;
        ptx::umma_commit(&empty[slot]);
        if (++slot == C::kRing) slot = 0;
        if (++stage == C::kStages) stage = 0, phase ^= 1u;
      }
      if (!ok) {                                  // gave up: the MMAs under way still use tensor and shared memory
        ptx::umma_commit(drained);
        uint32_t polls = 0;
        while (!ptx::mbar_try_wait(drained, 0) && ++polls < 1000000u) {}
      }
    }
  } else {
    // ------------------------------------------------------------- copies
    // Warp 17 the codes, a lane for each matrix; 18 the scales, then the zeros, a lane for each matrix and group; 19 the
    // activations and (down) their units.
    const uint8_t* src = nullptr;
    int64_t pitch = 0;
    int mul = 1, add = 0, last = 1 << 30, to = 0;
    uint32_t bytes = 0;
    if (warp == 17) {
      bytes = lane < C::kMats ? 8192 : 0;
      to = C::kCodes + lane * 8192;
    } else if (warp == 18) {
      const bool is_zero = lane >= C::kMats * GPB;
      const int at = lane - (is_zero ? C::kMats * GPB : 0), mat = at / GPB % C::kMats, size = is_zero ? 1 : 2;
      const W4Mat& m = a.m[mat];
      if (at < C::kMats * GPB && (!is_zero || (ZERO && m.zero != nullptr))) {
        src = (is_zero ? m.zero : reinterpret_cast<const uint8_t*>(m.scale)) + row0 * size;
        bytes = static_cast<uint32_t>(min(m.rows16 - row0, static_cast<int64_t>(128))) * size;
      }
      pitch = m.rows16 * size;
      mul = GPB;
      add = at % GPB;
      last = static_cast<int>(m.n_groups) - 1;
      to = (is_zero ? C::kZeros : C::kScales) + at * 128 * size;
    } else if (lane == 0) {
      src = a.image;
      pitch = bytes = C::kB;
      add = chunk * a.kblocks;
    } else if (!GATEUP && lane == 1) {
      src = reinterpret_cast<const uint8_t*>(a.unit);
      pitch = bytes = C::kCols * 4;
      add = chunk * a.kblocks;
      to = C::kUnits;
    }
    const uint32_t all = __reduce_add_sync(0xFFFFFFFFu, bytes);
    if (warp == 19) ptx::griddep_wait();          // the activations are complete
    int stage = 0, issued = 0;
    uint32_t phase = 1;
    bool ok = true;
    for (int e = 0; e < n_entries; ++e) {
      ok = ptx::mbar_wait_bounded(&empty[stage], phase, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      if (lane == 0) ptx::mbar_expect_tx(&full[stage], all);
      __syncwarp();
      if (bytes != 0) {
        uint8_t* dst = smem + stage * C::kStage + to;
        if (warp == 17) ptx::tma_load_2d(dst, &a.codes[lane], s_list[e] * 64, row0, &full[stage]);
        else ptx::bulk_load_1d(dst, src + min(s_list[e] * mul + add, last) * pitch, bytes, &full[stage]);
      }
      ++issued;
      if (++stage == C::kRing) stage = 0, phase ^= 1u;
    }
    if (GATEUP && warp == 19)
      for (int t = lane; t < 64 && chunk * a.tokens + t < min(a.n, (chunk + 1) * a.tokens); t += 32) s_factor[t] = a.unit[chunk * a.tokens + t];
    // No copy of this warp's is under way when the block goes on.  Where another warp gave up earlier a stage stays
    // incomplete, and a copy of its own has landed long before the polls are used up.
    for (int e = max(issued - C::kRing, 0); e < issued; ++e) {
      uint32_t polls = 0;
      while (!ptx::mbar_try_wait(&full[e % C::kRing], (e / C::kRing) & 1) && ++polls < 20000u) {}
    }
  }

  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, 512);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, kStatusTimeout);
  if (cluster > 1) ptx::cluster_sync_all();

  if (cluster == 1) tc_outputs<1, NE, GATEUP>(a, reinterpret_cast<const float*>(smem), s_factor);
  else if (cluster == 2) tc_outputs<2, NE, GATEUP>(a, reinterpret_cast<const float*>(smem), s_factor);
  else if (cluster == 4) tc_outputs<4, NE, GATEUP>(a, reinterpret_cast<const float*>(smem), s_factor);
  else tc_outputs<8, NE, GATEUP>(a, reinterpret_cast<const float*>(smem), s_factor);
  if (cluster > 1) {
    __syncthreads();
    ptx::cluster_sync_all();                      // no block leaves while another reads its sums
  }
}

template <int NE, int GPB, bool GATEUP, bool ZERO, bool MASKED>
cudaError_t launch_tc(const W4TcArgs& a, int cluster, cudaStream_t st) {
  auto kernel = w4_tc_kernel<NE, GPB, GATEUP, ZERO, MASKED>;
  const int smem = TcCfg<NE, GPB, GATEUP>::kSmem;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.rows + 127) / 128), static_cast<unsigned>(cluster),
                     static_cast<unsigned>((a.n + a.tokens - 1) / a.tokens));
  cfg.blockDim = dim3(kTcThreads);
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

template <int NE, int GPB, bool GATEUP, bool ZERO>
cudaError_t launch_tc_masked(const W4TcArgs& a, int cluster, cudaStream_t st) {
  // the test of every scale costs up to 3 us of 98 (4096 x 14336, 128 tokens), so calls without a selection go without it
  return GATEUP || a.dense ? launch_tc<NE, GPB, GATEUP, ZERO, false>(a, cluster, st) : launch_tc<NE, GPB, GATEUP, ZERO, !GATEUP>(a, cluster, st);
}

template <int GPB, bool GATEUP>
cudaError_t launch_tc_any(const W4TcArgs& a, int cluster, cudaStream_t st) {
  const bool zero = a.m[0].zero != nullptr || a.m[1].zero != nullptr;
  if (a.ne == 32) return zero ? launch_tc_masked<32, GPB, GATEUP, true>(a, cluster, st) : launch_tc_masked<32, GPB, GATEUP, false>(a, cluster, st);
  return zero ? launch_tc_masked<64, GPB, GATEUP, true>(a, cluster, st) : launch_tc_masked<64, GPB, GATEUP, false>(a, cluster, st);
}

}  // namespace w4
}  // namespace mlpmoe
