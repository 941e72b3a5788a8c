// Rows in memory to registers and back, eight consecutive elements a thread, and sums over a row's threads: shared by the norms
// and by the kernels that move and sum rows.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "../../include/mlpmoe.h"
#include "internal.h"

namespace mlpmoe {

__device__ __forceinline__ float bf16_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t u) { return __uint_as_float(u & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// Eight consecutive elements from column col, as they stand in memory (fp32: the whole of a and b; bf16: a), zeros past the
// row's end.  VEC: the row starts on 16 bytes and d % 8 == 0, so a chunk is whole.
struct Chunk {
  uint4 a, b;
};
template <bool VEC>
__device__ __forceinline__ Chunk load_chunk(const void* row, int kind, int col, int d) {
  Chunk c;
  c.a = c.b = make_uint4(0u, 0u, 0u, 0u);
  if (col >= d) return c;
  if (kind == MLPMOE_FP32) {
    const uint32_t* p = static_cast<const uint32_t*>(row) + col;
    if (VEC) {
      c.a = reinterpret_cast<const uint4*>(p)[0];
      c.b = reinterpret_cast<const uint4*>(p)[1];
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = col + i < d ? p[i] : 0u;
      c.a = make_uint4(w[0], w[1], w[2], w[3]);
      c.b = make_uint4(w[4], w[5], w[6], w[7]);
    }
  } else {
    const uint16_t* p = static_cast<const uint16_t*>(row) + col;
    if (VEC) {
      c.a = *reinterpret_cast<const uint4*>(p);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = col + i < d ? p[i] : 0u;
      c.a = make_uint4(w[0] | (w[1] << 16), w[2] | (w[3] << 16), w[4] | (w[5] << 16), w[6] | (w[7] << 16));
    }
  }
  return c;
}
__device__ __forceinline__ void to_f32(const Chunk& c, int kind, float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    v[0] = __uint_as_float(c.a.x), v[1] = __uint_as_float(c.a.y), v[2] = __uint_as_float(c.a.z), v[3] = __uint_as_float(c.a.w);
    v[4] = __uint_as_float(c.b.x), v[5] = __uint_as_float(c.b.y), v[6] = __uint_as_float(c.b.z), v[7] = __uint_as_float(c.b.w);
  } else {
    v[0] = bf16_lo(c.a.x), v[1] = bf16_hi(c.a.x), v[2] = bf16_lo(c.a.y), v[3] = bf16_hi(c.a.y);
    v[4] = bf16_lo(c.a.z), v[5] = bf16_hi(c.a.z), v[6] = bf16_lo(c.a.w), v[7] = bf16_hi(c.a.w);
  }
}

template <bool VEC>
__device__ __forceinline__ void store8(void* row, int kind, int col, int d, const float (&v)[8]) {
  if (kind == MLPMOE_FP32) {
    float* p = static_cast<float*>(row) + col;
    if (VEC) {
      __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = v[i];
    }
  } else if (kind == MLPMOE_BF16) {
    __nv_bfloat16* p = static_cast<__nv_bfloat16*>(row) + col;
    if (VEC) {
      *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = __float2bfloat16_rn(v[i]);
    }
  } else {
    uint8_t* p = static_cast<uint8_t*>(row) + col;
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __nv_cvt_float2_to_fp8x2(make_float2(v[2 * i], v[2 * i + 1]), __NV_SATFINITE, __NV_E4M3);
    if (VEC) {
      *reinterpret_cast<uint2*>(p) = make_uint2(c[0] | (c[1] << 16), c[2] | (c[3] << 16));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (col + i < d) p[i] = static_cast<uint8_t>(c[i / 2] >> (8 * (i & 1)));
    }
  }
}

// The same for kernels that may deal a row's columns to its threads as they like: chunk i of thread `tid` of T.  VEC: eight neighbours,
// (i T + tid) 8 + e.  Else, where they would be loaded one at a time, columns (8 i + e) T + tid: a warp's loads are neighbours.
template <bool VEC, int T>
__device__ __forceinline__ int column(int i, int tid, int e) { return VEC ? (i * T + tid) * 8 + e : (8 * i + e) * T + tid; }
// The 2 or 4 bytes at p, or 0: one predicated load whose result nothing touches yet.  (From C++ two bytes are widened where they are
// loaded, which waits for each: 16000 x 901 bf16 rows and their gradient 163 us.)
template <int BYTES>
__device__ __forceinline__ uint32_t load_if(const void* p, bool is) {
  uint32_t w;
  if (BYTES == 4) {
    asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\nmov.u32 %0, 0;\n@q ld.global.u32 %0, [%1];\n}\n" : "=r"(w) : "l"(p), "r"(static_cast<int>(is)) : "memory");
  } else {
    asm volatile("{\n.reg .pred q;\nsetp.ne.s32 q, %2, 0;\nmov.u32 %0, 0;\n@q ld.global.u16 %0, [%1];\n}\n" : "=r"(w) : "l"(p), "r"(static_cast<int>(is)) : "memory");
  }
  return w;
}
template <bool VEC, int T>
__device__ __forceinline__ Chunk load_columns(const void* row, int kind, int i, int tid, int d) {
  if (VEC) {
    return load_chunk<true>(row, kind, column<VEC, T>(i, tid, 0), d);
  } else {
    uint32_t w[8];                    // a word each, bf16 too
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int col = column<VEC, T>(i, tid, e);
      w[e] = kind == MLPMOE_FP32 ? load_if<4>(static_cast<const uint32_t*>(row) + col, col < d) : load_if<2>(static_cast<const uint16_t*>(row) + col, col < d);
    }
    return Chunk{make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7])};
  }
}
template <bool VEC>
__device__ __forceinline__ void columns_f32(const Chunk& c, int kind, float (&v)[8]) {
  if (VEC || kind == MLPMOE_FP32) {
    to_f32(c, kind, v);
  } else {
    v[0] = bf16_lo(c.a.x), v[1] = bf16_lo(c.a.y), v[2] = bf16_lo(c.a.z), v[3] = bf16_lo(c.a.w);
    v[4] = bf16_lo(c.b.x), v[5] = bf16_lo(c.b.y), v[6] = bf16_lo(c.b.z), v[7] = bf16_lo(c.b.w);
  }
}
template <bool VEC, int T>
__device__ __forceinline__ void store_columns(void* row, int kind, int i, int tid, int d, const float (&v)[8]) {
  if (VEC) {
    if (column<VEC, T>(i, tid, 0) < d) store8<true>(row, kind, column<VEC, T>(i, tid, 0), d, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int col = column<VEC, T>(i, tid, e);
      if (col >= d) continue;
      if (kind == MLPMOE_FP32) {
        static_cast<float*>(row)[col] = v[e];
      } else {
        static_cast<__nv_bfloat16*>(row)[col] = __float2bfloat16_rn(v[e]);
      }
    }
  }
}

// Sum (or maximum) over the T threads of a row, the same bits in all of them.  T = 32: the row's warp; else the block.
template <int T, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float u = __shfl_xor_sync(0xFFFFFFFFu, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  if (T > 32) {
    if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < T / 32; ++i) v = MAX ? fmaxf(v, red[i]) : v + red[i];
    __syncthreads();
  }
  return v;
}

// Sums of V values (V <= 4) over the 32 lanes of a warp: V == 1 in every lane, else value k in the lanes of the k-th half (V == 2) or
// quarter.  The first steps exchange values, so that four sums cost 6 exchanges and not 20.
template <int V>
__device__ __forceinline__ float warp_sums(const float (&v)[V]) {
  const int lane = threadIdx.x % 32;
  float x;
  if (V == 1) {
    x = v[0];
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 16);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
  } else if (V == 2) {
    x = (lane & 16 ? v[V - 1] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, lane & 16 ? v[0] : v[V - 1], 16);
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 8);
  } else {
    const float v3 = V == 4 ? v[V - 1] : 0.0f;
    const float a = (lane & 16 ? v[2 % V] : v[0]) + __shfl_xor_sync(0xFFFFFFFFu, lane & 16 ? v[0] : v[2 % V], 16);
    const float b = (lane & 16 ? v3 : v[1 % V]) + __shfl_xor_sync(0xFFFFFFFFu, lane & 16 ? v[1 % V] : v3, 16);
    x = (lane & 8 ? b : a) + __shfl_xor_sync(0xFFFFFFFFu, lane & 8 ? a : b, 8);
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  return x;
}
constexpr int __host__ __device__ lanes_of(int values) { return values == 1 ? 32 : (values == 2 ? 16 : 8); }      // lanes of a value there

// Sums of V values over the T threads of a row (T = 32: a warp, else the block), the same bits in all of them.  `red`: two sets, used
// in turn, so that one barrier a call will do.
template <int T, int V>
__device__ __forceinline__ void row_sums(float (&v)[V], float (*red)[T / 32][4], int& turn) {
  constexpr int L = lanes_of(V);
  const int lane = threadIdx.x % 32;
  float x = warp_sums<V>(v);
  if (T > 32) {
    float(*r)[4] = red[turn];
    turn ^= 1;
    if (lane % L == 0 && lane / L < V) r[threadIdx.x / 32][lane / L] = x;
    __syncthreads();
    x = 0.0f;
#pragma unroll
    for (int i = 0; i < T / 32; i += L)
      if (i + lane % L < T / 32) x += r[i + lane % L][lane / L];
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
  }
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = V == 1 ? x : __shfl_sync(0xFFFFFFFFu, x, k * L);
}

// Bytes of an element of a kind (MLPMOE_BF16, MLPMOE_FP32, MLPMOE_E4M3).
__host__ __device__ constexpr int bytes_of(int kind) { return kind == MLPMOE_FP32 ? 4 : (kind == MLPMOE_BF16 ? 2 : 1); }

inline bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace mlpmoe
