// The layer on 4-bit weights for more tokens than fit beside all of K in shared memory: the same arithmetic as in
// w4_kernel.cuh (whole-number products of the codes with the activations' digits), tiled like a matrix product.
//
// A block holds 32 `row_groups` rows and streams K in blocks of 128: the codes of its rows and the digits of all the
// chunk's tokens, prepared by w4_digits_kernel in the order the tensor core wants them, through a ring of stages that the
// whole block fills with cp.async (one barrier per K-block).  A warp takes 32 rows and a share of the columns, so that an
// activation read from shared memory serves two row tiles; without that the reads of shared memory, not the tensor
// core, set the time (160 against 128 cycles of an SM per 16 rows x 128 K x 64 tokens).
// Two digits of one token are neighbouring columns and so sit in one lane: c0 + 256 c1 is still exact in 32 bits, and scale
// and unit are applied once per token ("slot": two digits; an fp32 y takes two slots per token, the second
// with the third digit alone).
// Measured (4096 x 14336, group 128, y bf16): 64 tokens 129 us, 16 tokens 66, 9 tokens 52; y fp32 (twice the slots)
// 236, 95 and 78; bound by the issue of mma.sync and of the reads that feed it (two digits are two columns per token).
#pragma once
#include "w4_kernel.cuh"

namespace mlpmoe {
namespace w4 {

// This block's K-blocks into s_list, in order: its share of all of them or, for a product over the intermediate activations
// with a selection, of those with a neuron that a token of the chunk computes.  Returns how many; ends with a barrier.
template <bool ALL>
__device__ __forceinline__ int list_kblocks(int kblocks, int cluster, int rank, int dense, const uint8_t* select, int chunk, int tokens, int n,
                                            int B, const int32_t* off, const float* alpha, int* s_list, uint8_t* s_live, int* s_n) {
  const int threads = blockDim.x, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  if (ALL || dense) {
    const int share = (kblocks + cluster - 1) / cluster, count = max(0, min(share, kblocks - rank * share));
    for (int i = threadIdx.x; i < count; i += threads) s_list[i] = rank * share + i;
    __syncthreads();
    return count;
  }
  const int n_here = min(tokens, n - chunk * tokens);
  for (int b = threadIdx.x; b < B; b += threads) s_live[b] = select == nullptr && alpha[b] != 0.0f;
  __syncthreads();
  if (select != nullptr) {
    const uint8_t* sel = select + static_cast<int64_t>(chunk) * tokens * B;
    for (int i = threadIdx.x; i < n_here * B; i += threads)
      if (sel[i] != 0 && alpha[i % B] != 0.0f) s_live[i % B] = 1;
  }
  __syncthreads();
  if (warp == 0) {
    int total = 0;
    for (int pass = 0; pass < 2; ++pass) {        // count, then list this block's share
      const int per = (total + cluster - 1) / cluster, first = rank * per;
      int running = 0;
      for (int base = 0; base < kblocks; base += 32) {
        const int kb = base + lane;
        bool live = false;
        if (kb < kblocks)
          for (int b = find_branch(off, B, kb * 128); b < B && off[b] < (kb + 1) * 128; ++b) live = live || s_live[b] != 0;
        const unsigned who = __ballot_sync(0xFFFFFFFFu, live);
        const int at = running + __popc(who & ((1u << lane) - 1u)) - first;
        if (pass == 1 && live && at >= 0 && at < per) s_list[at] = kb;
        running += __popc(who);
      }
      if (pass == 0) total = running;
      else if (lane == 0) *s_n = max(0, min(per, total - first));
    }
  }
  __syncthreads();
  return *s_n;
}

// c_t: the quotient and the root in double, rounded once, as the routed forward does.
__device__ __forceinline__ float token_factor(const uint8_t* select, const float* alpha, int B, int compensate) {
  int k = 0, n_avail = 0;
  for (int b = 0; b < B; ++b) {
    const bool avail = alpha[b] != 0.0f;
    n_avail += avail ? 1 : 0;
    k += avail && select[b] != 0 ? 1 : 0;
  }
  if (k == 0) return 0.0f;
  return compensate ? static_cast<float>(sqrt(static_cast<double>(n_avail) / static_cast<double>(k))) : 1.0f;
}

// A thread takes eight k of one token; the 16 / GPB threads of a group are neighbours.
template <int GPB>
__global__ void __launch_bounds__(256) w4_digits_kernel(const __grid_constant__ W4DigitsArgs a) {
  constexpr int kLanes = 16 / GPB;
  ptx::griddep_wait();
  ptx::griddep_launch_dependents();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (a.status != nullptr && i == 0) *a.status = kStatusOk;
  const int units = a.kblocks * 16, u = static_cast<int>(i % units), k8 = u & 15;
  const int64_t token = i / units;
  Raw raw;
  raw.lo = raw.hi = make_uint4(0u, 0u, 0u, 0u);
  if (token < a.n && u * 8 < a.K) raw = load_raw(a.x, a.kind, token * a.stride + u * 8);
  float v[8], unit;
  to_f32(raw, a.kind, v);
  float top = largest(v);
#pragma unroll
  for (int o = 1; o < kLanes; o *= 2) top = larger(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
  const int pieces = a.slots_per_token + 1;
  uint32_t m[8];
  to_fixed(v, top, pieces, &unit, m);
  const uint2 d0 = digit_of(m, 0), d1 = digit_of(m, 1), d2 = digit_of(m, 2);
  int sum01 = sum_of_eight(d0) + 256 * sum_of_eight(d1), sum2 = sum_of_eight(d2);
#pragma unroll
  for (int o = 1; o < kLanes; o *= 2) {
    sum01 += __shfl_xor_sync(0xFFFFFFFFu, sum01, o);
    sum2 += __shfl_xor_sync(0xFFFFFFFFu, sum2, o);
  }
  if (token >= a.n) return;
  const int chunk = static_cast<int>(token / a.tokens), slot = static_cast<int>(token % a.tokens) * a.slots_per_token;
  const int64_t block = static_cast<int64_t>(chunk) * a.kblocks + u / 16;
  const int word = unit_word<GPB>(k8), j = k8 / kLanes;
  auto place = [&](int s, int digit) {
    return reinterpret_cast<uint2*>(a.digits + ((block * a.slot_tiles + s / 4) * 2 + (word >> 1)) * 512 +
                                    ((2 * (s % 4) + digit) * 4 + unit_lane<GPB>(k8)) * 16 + (word & 1) * 8);
  };
  *place(slot, 0) = d0;
  *place(slot, 1) = d1;
  if (pieces == 3) {
    *place(slot + 1, 0) = d2;
    *place(slot + 1, 1) = make_uint2(0u, 0u);
  }
  if (k8 % kLanes == 0) {
    if (a.x_scale != nullptr && u * 8 < a.K) {
      const int xg = a.x_groups == 1 ? 0 : (u / 16 * GPB + j) >> a.x_shift;
      unit *= a.x_scale[token * a.x_groups + xg];
    }
    float2* out = a.units + (block * GPB + j) * 4 * a.slot_tiles + slot;
    out[0] = make_float2(unit, __int_as_float(-sum01));
    if (pieces == 3) out[1] = make_float2(unit * 65536.0f, __int_as_float(-sum2));
  }
}

// grid: (row blocks, cluster along K, chunks)
template <int NTW, int GPB, bool GATEUP, bool ZERO>
__global__ void __launch_bounds__(512, 1) w4_wide_kernel(const __grid_constant__ W4WideArgs a) {
  constexpr int kWords = 4 / GPB;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int s_list[kW4MaxDim / 128];
  __shared__ int s_n;
  __shared__ uint8_t s_live[kW4MaxBranches];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const int rg = warp % a.row_groups, cg = warp / a.row_groups;
  const int chunk = blockIdx.z, rank = blockIdx.y, cluster = gridDim.y;
  const int block_rows = 32 * a.row_groups;
  const int tile0 = (blockIdx.x * a.row_groups + rg) * 2;
  const int st0 = cg * NTW;                       // first slot tile of the warp
  const int threads = blockDim.x;

  const int n_entries = list_kblocks<GATEUP>(a.kblocks, cluster, rank, a.dense, a.select, chunk, a.tokens, a.n, a.B, a.off, a.alpha, s_list,
                                             s_live, &s_n);
  // the kernel before this one writes the digits, and passed its own wait before this one could start: weights may be read
  ptx::griddep_launch_dependents();
  __syncthreads();

  // ---- copies of one stage
  const int stage = w4_wide_stage_bytes(a.row_groups, a.slot_tiles, GPB);
  const uint32_t ring = ptx::smem_u32(smem);
  const int o_scale = block_rows * 64, o_zero = o_scale + block_rows * GPB * 2, o_x = o_zero + block_rows * GPB, o_unit = o_x + a.slot_tiles * 1024;
  const uint32_t last_byte = static_cast<uint32_t>(a.m[0].pitch) - 16, last_group = static_cast<uint32_t>(a.m[0].n_groups) - 1;
  const uint32_t rows16 = static_cast<uint32_t>(a.m[0].rows16);
  if (ZERO) {                                     // a matrix without stored zeros beside one with them: 8, for good
    for (int i = threadIdx.x; i < block_rows / 8 * GPB; i += threads) {
      const int piece = i / GPB;                  // 8-row half: tile piece / 2, half piece % 2
      if ((piece & 1 ? a.m[1].zero : a.m[0].zero) == nullptr)
        for (int s = 0; s < kW4WideStages; ++s)
          *reinterpret_cast<uint2*>(smem + s * stage + o_zero + i * 8) = make_uint2(0x08080808u, 0x08080808u);
    }
  }
  // first row (of its matrix) of half `half` of local tile `lt`; rows past the last are read from the last eight
  auto half_row = [&](int lt, int half) {
    const int tile = blockIdx.x * a.row_groups * 2 + lt;
    return GATEUP ? min(tile * 8, a.rows - 8) : min(tile * 16 + 8 * half, a.rows - 8);
  };
  // codes: 128 row_groups pieces of 16 bytes and 32 row_groups col_groups threads, four, two or one each; a thread's rows
  // never change.  One column group occurs with 1 or 3 tiles only.
  constexpr int kTurns = NTW == 1 || NTW == 3 ? 4 : 2;
  const uint8_t* q_src[kTurns];
  uint32_t q_dst[kTurns];
#pragma unroll
  for (int m = 0; m < kTurns; ++m) {
    const int i = threadIdx.x + m * threads, r = i >> 2, c = i & 3, half = (r >> 3) & 1;
    const bool in = i < block_rows * 4;
    q_src[m] = in ? (half == 0 ? a.m[0].q : a.m[1].q) + (half_row(r >> 4, half) + (r & 7)) * a.m[0].pitch : nullptr;
    q_dst[m] = ring + r * 64 + (c ^ ((r >> 1) & 3)) * 16;
  }
  const uint32_t q_col = (threadIdx.x & 3) * 16;
  // scales and zeros: 4 row_groups GPB pieces (an 8-row half and a group each), one per thread
  const int s_piece = threadIdx.x / GPB, s_half = s_piece & 1;
  const bool s_in = threadIdx.x < block_rows / 8 * GPB;
  const __nv_bfloat16* const s_src = (s_half == 0 ? a.m[0].scale : a.m[1].scale) + (s_in ? half_row(s_piece >> 1, s_half) : 0);
  const uint8_t* const z_base = s_half == 0 ? a.m[0].zero : a.m[1].zero;
  const uint8_t* const z_src = ZERO && s_in && z_base != nullptr ? z_base + half_row(s_piece >> 1, s_half) : nullptr;
  auto copy_weights = [&](int entry, int slot) {
    const uint32_t kb = s_list[entry], to = slot * stage, byte = min(kb * 64 + q_col, last_byte);
#pragma unroll
    for (int m = 0; m < kTurns; ++m)
      if (q_src[m] != nullptr) cp_async16(q_dst[m] + to, q_src[m] + byte);
    if (s_in) {
      const uint32_t at = min(kb * GPB + threadIdx.x % GPB, last_group) * rows16;
      cp_async16(ring + to + o_scale + threadIdx.x * 16, s_src + at);
      if (z_src != nullptr) cp_async8(ring + to + o_zero + threadIdx.x * 8, z_src + at);
    }
  };
  auto copy_digits = [&](int entry, int slot) {
    const int64_t at = static_cast<int64_t>(chunk) * a.kblocks + s_list[entry];
    const uint32_t to = ring + slot * stage;
    const uint8_t* x = a.digits + at * a.slot_tiles * 1024;
    for (int i = threadIdx.x * 16; i < a.slot_tiles * 1024; i += threads * 16) cp_async16(to + o_x + i, x + i);
    const uint8_t* u = reinterpret_cast<const uint8_t*>(a.units + at * GPB * 4 * a.slot_tiles);
    for (int i = threadIdx.x * 16; i < a.slot_tiles * GPB * 32; i += threads * 16) cp_async16(to + o_unit + i, u + i);
  };
  for (int i = 0; i < kW4WideStages - 1; ++i)
    if (i < n_entries) copy_weights(i, i);
  ptx::griddep_wait();                            // the digits are complete
  for (int i = 0; i < kW4WideStages - 1; ++i) {
    if (i < n_entries) copy_digits(i, i);
    cp_async_commit();
  }

  float acc[2][NTW][2];                           // [row tile][slot tile][row g, row g + 8] of slot 4 (st0 + nt) + t
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) acc[rt][nt][0] = acc[rt][nt][1] = 0.0f;

  int slot = 0;
#pragma unroll 1
  for (int i = 0; i < n_entries; ++i) {
    cp_async_wait<kW4WideStages - 2>();
    __syncthreads();                              // the stage is complete, and every warp has left the one before it
    {
      const int next = i + kW4WideStages - 1, into = slot == 0 ? kW4WideStages - 1 : slot - 1;
      if (next < n_entries) {
        copy_weights(next, into);
        copy_digits(next, into);
      }
      cp_async_commit();
    }
    const uint8_t* st = smem + slot * stage;
#pragma unroll
    for (int j = 0; j < GPB; ++j) {
      uint32_t op[2][kWords][4];                  // [row tile][word]: even and odd codes of rows g and g + 8
      float s[2][2];
      int zero[2][2];
#pragma unroll
      for (int rt = 0; rt < 2; ++rt) {
        uint32_t q[2][kWords];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = (rg * 2 + rt) * 16 + h * 8 + g, sw = (g >> 1) & 3;
          const uint8_t* row = st + r * 64;
          if (GPB == 1) {
            const uint4 v = *reinterpret_cast<const uint4*>(row + ((t ^ sw) * 16));
            q[h][0] = v.x, q[h][1 % kWords] = v.y, q[h][2 % kWords] = v.z, q[h][3 % kWords] = v.w;
          } else if (GPB == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + (((2 * j + (t >> 1)) ^ sw) * 16) + (t & 1) * 8);
            q[h][0] = v.x, q[h][1 % kWords] = v.y;
          } else {
            q[h][0] = *reinterpret_cast<const uint32_t*>(row + ((j ^ sw) * 16) + t * 4);
          }
          const int piece = ((rg * 2 + rt) * 2 + h) * GPB + j;
          s[rt][h] = __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(st + o_scale + piece * 16 + g * 2));
          zero[rt][h] = ZERO ? st[o_zero + piece * 8 + g] : 8;
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          op[rt][w][0] = q[0][w] & 0x0F0F0F0Fu;
          op[rt][w][1] = q[1][w] & 0x0F0F0F0Fu;
          op[rt][w][2] = (q[0][w] >> 4) & 0x0F0F0F0Fu;
          op[rt][w][3] = (q[1][w] >> 4) & 0x0F0F0F0Fu;
        }
      }
      const uint4* xs = reinterpret_cast<const uint4*>(st + o_x + st0 * 1024) + lane;
      const float2* us = reinterpret_cast<const float2*>(st + o_unit) + (j * 4 * a.slot_tiles + 4 * st0 + t);
#pragma unroll
      for (int nt = 0; nt < NTW; ++nt) {
        const uint4* xp = xs + nt * 64;
        const float2 unit = us[4 * nt];
        uint4 b[2];
        if (GPB < 4 || j < 2) b[0] = xp[0];
        if (GPB == 1 || (GPB == 2 && j == 1) || (GPB == 4 && j >= 2)) b[1] = xp[32];
#pragma unroll
        for (int rt = 0; rt < 2; ++rt) {
          int part[4] = {zero[rt][0] * __float_as_int(unit.y), 0, zero[rt][1] * __float_as_int(unit.y), 0};
#pragma unroll
          for (int w = 0; w < kWords; ++w) {
            const int at = j * kWords + w;
            const uint4 v = b[at >> 1];
            mma(part, op[rt][w][0], op[rt][w][1], op[rt][w][2], op[rt][w][3], at & 1 ? v.z : v.x, at & 1 ? v.w : v.y);
          }
          // at most 15 * 128 * (128 + 256 * 127): exact in 32 bits, rounded once to fp32
          // a branch that the token does not compute: its activations are 0, its scales may be anything
          if (GATEUP || a.dense || unit.x != 0.0f) {
            acc[rt][nt][0] += __int2float_rn(part[0] + 256 * part[1]) * (s[rt][0] * unit.x);
            acc[rt][nt][1] += __int2float_rn(part[2] + 256 * part[3]) * (s[rt][1] * unit.x);
          }
        }
      }
    }
    slot = slot + 1 == kW4WideStages ? 0 : slot + 1;
  }
  cp_async_wait<0>();
  // the second slot of a token (the third digit) belongs to the neighbouring lane
  if (a.slots_per_token == 2) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt)
#pragma unroll
      for (int nt = 0; nt < NTW; ++nt)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[rt][nt][h] += __shfl_xor_sync(0xFFFFFFFFu, acc[rt][nt][h], 1);
  }
  auto token_of = [&](int nt) {                   // of this lane, or -1 where it holds none
    const int s = 4 * (st0 + nt) + t, tok = s / a.slots_per_token, token = chunk * a.tokens + tok;
    return tok < a.tokens && token < a.n && (a.slots_per_token == 1 || (t & 1) == 0) ? token : -1;
  };
  if (GATEUP) {
#pragma unroll
    for (int rt = 0; rt < 2; ++rt) {
      const int neuron = (tile0 + rt) * 8 + g;
      if (neuron >= a.rows) continue;
      const int b = find_branch(a.off, a.B, neuron);
      const float alpha = a.alpha[b];
#pragma unroll
      for (int nt = 0; nt < NTW; ++nt) {
        const int token = token_of(nt);
        if (token < 0) continue;
        const float gate = acc[rt][nt][0], up = acc[rt][nt][1];
        const bool on = alpha != 0.0f && (a.select == nullptr || a.select[static_cast<int64_t>(token) * a.B + b] != 0);
        a.h[static_cast<int64_t>(token) * a.rows + neuron] = on ? gate / (1.0f + expf(-gate)) * up * alpha : 0.0f;
      }
    }
    return;
  }
  auto finish = [&](int token, int m, float v) {
    if (a.select != nullptr) v *= token_factor(a.select + static_cast<int64_t>(token) * a.B, a.alpha, a.B, a.compensate);
    const int64_t at = static_cast<int64_t>(token) * a.rows + m;
    if (a.residual != nullptr) v += a.residual[at];
    if (a.y_bf16) static_cast<__nv_bfloat16*>(a.y)[at] = __float2bfloat16_rn(v);
    else static_cast<float*>(a.y)[at] = v;
  };
  // the block's sums go through shared memory, [token][row], so that y is written along its rows
  float* own = reinterpret_cast<float*>(smem);
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < 2; ++rt)
#pragma unroll
    for (int nt = 0; nt < NTW; ++nt) {
      const int token = token_of(nt);
      if (token < 0) continue;
      float* p = own + (token - chunk * a.tokens) * (block_rows + 4) + (rg * 2 + rt) * 16 + g;
      p[0] = acc[rt][nt][0];
      p[8] = acc[rt][nt][1];
    }
  __syncthreads();
  if (cluster > 1) ptx::cluster_sync_all();
  const int n_here = min(a.tokens, a.n - chunk * a.tokens), row0 = blockIdx.x * block_rows;
  for (int i = rank * threads + threadIdx.x; i < n_here * block_rows; i += cluster * threads) {
    const int tok = i / block_rows, r = i % block_rows;
    if (row0 + r >= a.rows) continue;
    const float* p = own + tok * (block_rows + 4) + r;
    float v = 0.0f;
    if (cluster == 1) {
      v = *p;
    } else {
      float part[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) part[k] = k < cluster ? ld_cluster_f32(p, k) : 0.0f;
#pragma unroll
      for (int k = 0; k < 8; ++k) v += part[k];
    }
    finish(chunk * a.tokens + tok, row0 + r, v);
  }
  if (cluster > 1) {
    __syncthreads();
    ptx::cluster_sync_all();                      // no block leaves while another reads its sums
  }
}

template <int NTW, int GPB, bool GATEUP, bool ZERO>
cudaError_t launch_wide(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st) {
  auto kernel = w4_wide_kernel<NTW, GPB, GATEUP, ZERO>;
  int smem = kW4WideStages * w4_wide_stage_bytes(a.row_groups, a.slot_tiles, GPB);
  const int own = GATEUP ? 0 : a.tokens * (32 * a.row_groups + 4) * 4;
  if (own > smem) smem = own;
  if (smem > kWideSmemMax) return cudaErrorInvalidValue;
  // the same for every call: the limit is the kernel's, and another thread's call may come between here and the launch
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWideSmemMax);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>((a.tiles + 2 * a.row_groups - 1) / (2 * a.row_groups)), static_cast<unsigned>(cluster),
                     static_cast<unsigned>(chunks));
  cfg.blockDim = dim3(static_cast<unsigned>(32 * a.row_groups * a.col_groups));
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
cudaError_t launch_wide_tiles(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st) {
  switch (a.slot_tiles / a.col_groups) {
    case 1: return launch_wide<1, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    case 2: return launch_wide<2, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    case 3: return launch_wide<3, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    case 4: return launch_wide<4, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    case 6: return launch_wide<6, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    case 8: return launch_wide<8, GPB, GATEUP, ZERO>(a, cluster, chunks, st);
    default: return cudaErrorInvalidValue;
  }
}

template <int GPB, bool GATEUP>
cudaError_t launch_wide_zero(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st) {
  return a.m[0].zero != nullptr || a.m[1].zero != nullptr ? launch_wide_tiles<GPB, GATEUP, true>(a, cluster, chunks, st)
                                                          : launch_wide_tiles<GPB, GATEUP, false>(a, cluster, chunks, st);
}

template <int GPB>
cudaError_t launch_digits(const W4DigitsArgs& a, cudaStream_t st) {
  const int64_t threads = static_cast<int64_t>(a.n) * a.kblocks * 16;
  return launch_pdl(w4_digits_kernel<GPB>, dim3(static_cast<unsigned>((threads + 255) / 256)), dim3(256), 0, st, a);
}

}  // namespace w4
}  // namespace mlpmoe
