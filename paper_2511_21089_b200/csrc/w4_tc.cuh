// The layer on 4-bit weights for batches large enough for the 5th-generation tensor cores (y in bf16).
//
// The codes become bf16 whole numbers code - zero (exact) in shared memory, in the 128-byte-swizzled K-major form that
// tcgen05.mma reads, the activations come prepared in the same form (w4_columns_kernel: one bf16 piece of x, or two
// pieces where x or the intermediate activation has more bits; 2^-16 of the value is left out, y is rounded to 2^-8),
// and the products of one group of K (32, 64 or 128 columns) accumulate in tensor memory.  Two accumulators alternate:
// while the tensor core fills one, the epilogue warps read the other back and add it, times the row's scale, to their fp32
// sums in registers.
// What it spends per 128 columns of K, 128 neurons and 64 tokens: 64 KB written and 96 KB read in shared memory, about
// 1300 cycles of an SM, and 660 of issue, where mma.sync (w4_wide.cuh) needs 5000.
//
// A block: 128 neurons (128 gate rows and 128 up rows) or 128 rows of W_down.  Warps 0..7 epilogue (tensor memory lanes
// 32 (warp % 4).., columns NE (warp / 4)..), 8..15 codes to bf16, 16 issues the MMAs, 17 fetches the activations.
#pragma once
#include "w4_wide.cuh"

namespace mlpmoe {
namespace w4 {

constexpr int kTcThreads = 18 * 32;
constexpr int kTcTile = 128 * 128 * 2;            // one matrix's operand of a stage: 128 rows x 128 columns of bf16

template <int NE, bool GATEUP>
struct TcCfg {
  static constexpr int kMats = GATEUP ? 2 : 1;
  static constexpr int kCols = GATEUP ? NE : 2 * NE;             // columns of an MMA
  static constexpr int kStages = GATEUP ? 2 : 3;
  static constexpr int kB = kCols * 256;
  static constexpr int kStage = kMats * kTcTile + kB;
  static constexpr int kBars = kStages * kStage;
  static constexpr int kSmem = kBars + 256 + 1024;               // barriers, slack for 1024-byte alignment
  static constexpr int kTmem = 4 * NE;                           // two accumulators of 2 NE columns
};

// Eight codes -> four bf16 pairs code - zero, pairs (e, e + 4) of eight consecutive columns; bias = (128 + zero) twice.  The
// code slides into the mantissa of 128.0; the difference is exact.
__device__ __forceinline__ uint4 unpack_bf16(uint32_t w, uint32_t bias) {
  uint32_t p[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(u) : "r"(w >> (4 * i)), "r"(0x000F000Fu), "r"(0x43004300u));
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&bias));
    p[i] = *reinterpret_cast<const uint32_t*>(&v);
  }
  return make_uint4(p[0], p[1], p[2], p[3]);
}

// Activations as the MMAs' second operand: per chunk and K-block, two halves of 64 columns of K, each `cols` rows of 128 bytes
// under the 128-byte swizzle; row p tokens + tok holds piece p of token tok.  A thread takes eight k of one token.
static __global__ void __launch_bounds__(256) w4_columns_kernel(const __grid_constant__ W4ColumnsArgs a) {
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (a.status != nullptr && i == 0) *a.status = kStatusOk;
  const int units = a.kblocks * 16, u = static_cast<int>(i % units), k8 = u & 15;
  const int64_t token = i / units;
  if (token >= a.n) return;
  float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
  if (u * 8 < a.K) {
    to_f32(load_raw(a.x, a.kind, token * a.stride + u * 8), a.kind, v);
    if (a.x_scale != nullptr) {
      const float s = a.x_scale[token * a.x_groups + (a.x_groups == 1 ? 0 : u * 8 / a.x_group)];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] *= s;
    }
  }
  const int chunk = static_cast<int>(token / a.tokens);
  uint8_t* half = a.image + ((static_cast<int64_t>(chunk) * a.kblocks + u / 16) * 2 + (k8 >> 3)) * (a.cols * 128);
  for (int p = 0; p < a.pieces; ++p) {
    const int c = p * a.tokens + static_cast<int>(token % a.tokens);
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 pair = __floats2bfloat162_rn(v[e], v[e + 4]);
      v[e] -= __low2float(pair);
      v[e + 4] -= __high2float(pair);
      o[e] = *reinterpret_cast<const uint32_t*>(&pair);
    }
    *reinterpret_cast<uint4*>(half + c * 128 + (((k8 & 7) ^ (c & 7)) * 16)) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// grid: (blocks of 128 rows, cluster along K, chunks)
template <int NE, int GPB, bool GATEUP, bool ZERO>
__global__ void __launch_bounds__(kTcThreads, 1) w4_tc_kernel(const __grid_constant__ W4TcArgs a) {
  using C = TcCfg<NE, GATEUP>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int s_list[kW4MaxDim / 128];
  __shared__ int s_n;
  __shared__ uint8_t s_live[kW4MaxBranches];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint64_t* full_a = reinterpret_cast<uint64_t*>(smem + C::kBars);
  uint64_t* full_b = full_a + C::kStages;
  uint64_t* empty = full_b + C::kStages;
  uint64_t* d_full = empty + C::kStages;
  uint64_t* d_empty = d_full + 2;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(d_empty + 2);
  volatile uint32_t* abort_flag = tmem_slot + 1;
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int chunk = blockIdx.z, rank = blockIdx.y, cluster = gridDim.y;
  const int row0 = blockIdx.x * 128;

  if (threadIdx.x == 0) {
    for (int s = 0; s < C::kStages; ++s) {
      ptx::mbar_init(&full_a[s], 256 + a.extra_arrivals);
      ptx::mbar_init(&full_b[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int b = 0; b < 2; ++b) {
      ptx::mbar_init(&d_full[b], 1);
      ptx::mbar_init(&d_empty[b], 8);
    }
    *abort_flag = 0;
    ptx::fence_barrier_init();
  }
  if (warp == 16) {
    ptx::tmem_alloc(tmem_slot, C::kTmem);
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
    const int quad = warp % 4, half = warp / 4, row = row0 + quad * 32 + lane;
    const W4Mat& m = a.m[GATEUP ? half : 0];
    const __nv_bfloat16* scale = m.scale + min(row, a.rows - 1);
    const int64_t rows16 = m.rows16;
    const int last_group = static_cast<int>(m.n_groups) - 1, steps = n_entries * GPB;
    auto load_scale = [&](int step) {
      return step < steps ? __bfloat162float(scale[min(s_list[step / GPB] * GPB + step % GPB, last_group) * rows16]) : 0.0f;
    };
    float acc[NE];
#pragma unroll
    for (int i = 0; i < NE; ++i) acc[i] = 0.0f;
    float s_next = load_scale(0);
    const uint32_t taddr = tmem + static_cast<uint32_t>(half * NE) + (static_cast<uint32_t>(quad * 32) << 16);
    for (int step = 0; step < steps; ++step) {
      const float s = s_next;
      s_next = load_scale(step + 1);
      const int b = step & 1;
      bool ok = ptx::mbar_wait_bounded(&d_full[b], (step >> 1) & 1, abort_flag, a.wait_limit_ns);
      ok = __all_sync(0xFFFFFFFFu, ok);
      if (!ok) break;
      ptx::tc_fence_after();
      constexpr int kPart = NE == 64 ? 16 : 32;   // what the registers hold beside the sums
#pragma unroll
      for (int i = 0; i < NE; i += kPart) {
        uint32_t r[kPart];
        if constexpr (kPart == 32) ptx::tmem_ld_32x32(taddr + b * 2 * NE + i, r);
        else ptx::tmem_ld_32x16(taddr + b * 2 * NE + i, r);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < kPart; ++k) acc[i + k] += __uint_as_float(r[k]) * s;
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&d_empty[b]);
    }
    __syncwarp();
    // every MMA of the block is complete once the last accumulator was: the stages are free
    float* sums = reinterpret_cast<float*>(smem) + half * NE * 128 + quad * 32 + lane;      // [column][row]
#pragma unroll
    for (int i = 0; i < NE; ++i) sums[i * 128] = acc[i];
  } else if (warp < 16) {
    // ------------------------------------------------------------- codes to bf16
    constexpr int kItems = 2 * C::kMats;          // 16 bytes of codes each: rows t / 4 + 64 i, columns 32 (t % 4)..
    const int t = threadIdx.x - 256, c = t & 3;
    const uint8_t* src[kItems];
    const uint8_t* zsrc[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const W4Mat& m = i < 2 ? a.m[0] : a.m[1];
      const int row = min(row0 + (((t >> 2) + 64 * i) & 127), a.rows - 1);
      src[i] = m.q + row * m.pitch;
      zsrc[i] = ZERO && m.zero != nullptr ? m.zero + row : nullptr;
    }
    const uint32_t last_byte = static_cast<uint32_t>(a.m[0].pitch) - 16;
    const int last_group = static_cast<int>(a.m[0].n_groups) - 1, group = c * GPB / 4;
    const int64_t rows16 = a.m[0].rows16;
    uint4 code[2][kItems];
    uint32_t zero[2][kItems];
    auto fetch = [&](int e, int u) {
      if (e >= n_entries) return;
      const int kb = s_list[e];
#pragma unroll
      for (int i = 0; i < kItems; ++i) {
        code[u][i] = *reinterpret_cast<const uint4*>(src[i] + min(static_cast<uint32_t>(kb) * 64 + c * 16, last_byte));
        if (ZERO) zero[u][i] = zsrc[i] != nullptr ? zsrc[i][min(kb * GPB + group, last_group) * rows16] : 8u;
      }
    };
    fetch(0, 0);
    fetch(1, 1);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int e = 0; ok && e < n_entries; e += 2) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (e + u >= n_entries) break;
        ok = ptx::mbar_wait_bounded(&empty[stage], phase ^ 1u, abort_flag, a.wait_limit_ns);
        ok = __all_sync(0xFFFFFFFFu, ok);
        if (!ok) break;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
          const int r = (t >> 2) + 64 * (i & 1);  // row of its matrix's operand
          uint8_t* to = smem + stage * C::kStage + (i >> 1) * kTcTile + (c >> 1) * (kTcTile / 2) + r * 128;
          const uint32_t bias = ZERO ? 0x43004300u + zero[u][i] * 0x00010001u : 0x43084308u;
          // the lanes of the second half of K store their words in another order, so that eight lanes meet eight banks
          const uint4 q = code[u][i];
          const uint32_t w[4] = {c & 2 ? q.z : q.x, c & 2 ? q.w : q.y, c & 2 ? q.x : q.z, c & 2 ? q.y : q.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j = (c & 1) * 4 + (k ^ (c & 2));          // 16-byte unit of the 128-byte row
            *reinterpret_cast<uint4*>(to + ((j ^ (r & 7)) * 16)) = unpack_bf16(w[k], bias);
          }
        }
        ptx::fence_proxy_async_smem();
        ptx::mbar_arrive(&full_a[stage]);
        fetch(e + u + 2, u);
        if (++stage == C::kStages) stage = 0, phase ^= 1u;
      }
    }
  } else if (warp == 16) {
    // ------------------------------------------------------------- MMAs
    if (lane == 0) {
      constexpr uint32_t idesc = ptx::make_idesc_bf16_f32(128, C::kCols);
      constexpr int kSteps = 8 / GPB;             // of 16 columns, in a group
      int stage = 0, d = 0;
      uint32_t phase = 0, d_phase = 0;
      bool ok = true;
      for (int e = 0; ok && e < n_entries; ++e) {
        ok = ptx::mbar_wait_bounded(&full_a[stage], phase, abort_flag, a.wait_limit_ns) &&
             ptx::mbar_wait_bounded(&full_b[stage], phase, abort_flag, a.wait_limit_ns);
        if (!ok) break;
        const uint32_t sa = ptx::smem_u32(smem + stage * C::kStage), sb = sa + C::kMats * kTcTile;
        for (int j = 0; j < GPB; ++j) {
          ok = ptx::mbar_wait_bounded(&d_empty[d], d_phase ^ 1u, abort_flag, a.wait_limit_ns);
          if (!ok) break;
          ptx::tc_fence_after();
#pragma unroll
          for (int mat = 0; mat < C::kMats; ++mat) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
              // 16 columns further inside the swizzled 128-byte row = +32 bytes = +2 in the descriptor's address field
              const int ks = j * kSteps + k;
              const uint64_t da = ptx::make_desc_sw128_kmajor(sa + mat * kTcTile + (ks >> 2) * (kTcTile / 2)) + 2 * (ks & 3);
              const uint64_t db = ptx::make_desc_sw128_kmajor(sb + (ks >> 2) * (C::kCols * 128)) + 2 * (ks & 3);
              ptx::umma_bf16(tmem + d * 2 * NE + mat * C::kCols, da, db, idesc, k != 0 ? 1u : 0u);
            }
          }
          ptx::umma_commit(&d_full[d]);
          if (++d == 2) d = 0, d_phase ^= 1u;
        }
        if (!ok) break;
        ptx::umma_commit(&empty[stage]);
        if (++stage == C::kStages) stage = 0, phase ^= 1u;
      }
    }
  } else if (lane == 0) {
    // ------------------------------------------------------------- activations
    ptx::griddep_wait();                          // they are complete
    int stage = 0, issued = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int e = 0; ok && e < n_entries; ++e) {
      ok = ptx::mbar_wait_bounded(&empty[stage], phase ^ 1u, abort_flag, a.wait_limit_ns);
      if (!ok) break;
      ++issued;
      ptx::mbar_expect_tx(&full_b[stage], C::kB);
      ptx::bulk_load_1d(smem + stage * C::kStage + C::kMats * kTcTile,
                        a.image + (static_cast<int64_t>(chunk) * a.kblocks + s_list[e]) * C::kB, C::kB, &full_b[stage]);
      if (++stage == C::kStages) stage = 0, phase ^= 1u;
    }
    // leave only when the MMAs have released every stage and no copy is under way
    for (int i = 0; ok && i < C::kStages; ++i) {
      ok = ptx::mbar_wait_bounded(&empty[stage], phase ^ 1u, abort_flag, a.wait_limit_ns);
      if (++stage == C::kStages) stage = 0, phase ^= 1u;
    }
    // gave up: the copies still on their way into this block's shared memory need nobody else to arrive
    for (int e = issued > C::kStages ? issued - C::kStages : 0; !ok && e < issued; ++e) {
      uint32_t polls = 0;
      while (!ptx::mbar_try_wait(&full_b[e % C::kStages], (e / C::kStages) & 1) && ++polls < 1000000u) {}
    }
  }

  __syncwarp();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 16) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(tmem, C::kTmem);
  }
  if (threadIdx.x == 0 && *abort_flag) atomicExch(a.status, kStatusTimeout);
  if (cluster > 1) ptx::cluster_sync_all();

  // ---- [column][row] sums of all blocks of the cluster; a token's pieces are columns tok, tokens + tok
  const float* sums = reinterpret_cast<const float*>(smem);
  auto total_of = [&](int col0, int tok, int r) {
    float part[2][8], v = 0.0f;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        part[p][k] = 0.0f;
        if (p < a.pieces && k < cluster) {
          const float* at = sums + (col0 + p * a.tokens + tok) * 128 + r;
          part[p][k] = cluster == 1 ? *at : ld_cluster_f32(at, k);
        }
      }
#pragma unroll
    for (int k = 0; k < 8; ++k) v += part[0][k] + part[1][k];
    return v;
  };
  const int n_here = min(a.tokens, a.n - chunk * a.tokens);
  for (int i = rank * kTcThreads + threadIdx.x; i < n_here * 128; i += cluster * kTcThreads) {
    const int tok = i >> 7, r = i & 127, row = row0 + r, token = chunk * a.tokens + tok;
    if (row >= a.rows) continue;
    if (GATEUP) {
      const int b = find_branch(a.off, a.B, row);
      const bool on = a.alpha[b] != 0.0f && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
      float h = 0.0f;
      if (on) {
        const float gate = total_of(0, tok, r), up = total_of(NE, tok, r);
        h = gate / (1.0f + expf(-gate)) * up * a.alpha[b];
      }
      a.h[static_cast<int64_t>(token) * a.rows + row] = h;
    } else {
      float v = total_of(0, tok, r);
      if (a.select != nullptr) v *= token_factor(a.select + static_cast<int64_t>(token) * a.B, a.alpha, a.B, a.compensate);
      const int64_t at = static_cast<int64_t>(token) * a.rows + row;
      if (a.residual != nullptr) v += a.residual[at];
      a.y[at] = __float2bfloat16_rn(v);
    }
  }
  if (cluster > 1) {
    __syncthreads();
    ptx::cluster_sync_all();                      // no block leaves while another reads its sums
  }
}

template <int NE, int GPB, bool GATEUP, bool ZERO>
cudaError_t launch_tc(const W4TcArgs& a, int cluster, cudaStream_t st) {
  auto kernel = w4_tc_kernel<NE, GPB, GATEUP, ZERO>;
  const int smem = TcCfg<NE, GATEUP>::kSmem;
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

template <int GPB, bool GATEUP>
cudaError_t launch_tc_any(const W4TcArgs& a, int cluster, cudaStream_t st) {
  const bool zero = a.m[0].zero != nullptr || a.m[1].zero != nullptr;
  if (a.ne == 32) return zero ? launch_tc<32, GPB, GATEUP, true>(a, cluster, st) : launch_tc<32, GPB, GATEUP, false>(a, cluster, st);
  return zero ? launch_tc<64, GPB, GATEUP, true>(a, cluster, st) : launch_tc<64, GPB, GATEUP, false>(a, cluster, st);
}

}  // namespace w4
}  // namespace mlpmoe
