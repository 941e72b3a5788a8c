// Entry point of the layer on 4-bit weights (mlpmoe_w4_forward): checks, the split of the work, and the kernel that
// lays the activations out and reads the selection.  Three launches: prepare, gate|up, down; the second and third
// begin with their copies of the weights while the kernel before them runs.
#include <cuda_fp8.h>
#include <string.h>

#include "../../include/mlpmoe.h"
#include "w4_kernel.cuh"

namespace mlpmoe {
namespace {

constexpr int kPrepThreads = 256;

struct PrepArgs {
  const void* x;
  int64_t stride;
  int kind, gpb, d, n;
  W4Cols c;
  int kblocks;
  uint4* frag;
  // the down product's columns: units past the last neuron are cleared
  W4Cols hc;
  int h_kblocks, h_unit0;
  uint4* h_frag;
  int unit_blocks, pad_blocks;      // blocks for x and for those units; one more reads the selection
  // selection
  const uint8_t* select;
  int B, compensate;
  uint8_t* active;
  float* coef;
  int32_t* list;
  int32_t off[kW4MaxBranches + 1];
  float alpha[kW4MaxBranches];
};

__device__ __forceinline__ int unit_at_gpb(int gpb, int col, int k8) {
  return gpb == 1 ? w4::unit_at<1>(col, k8) : (gpb == 2 ? w4::unit_at<2>(col, k8) : w4::unit_at<4>(col, k8));
}

// Eight consecutive activations as `pieces` units of eight bf16 in the order of unit_pos.
__device__ void prepare_unit(const PrepArgs& a, int64_t i) {
  const int units = a.kblocks * 16;
  const int u = static_cast<int>(i % units), token = static_cast<int>(i / units);
  const int chunk = token / a.c.tokens, tok = token % a.c.tokens;
  uint4* out = a.frag + (static_cast<int64_t>(chunk) * a.kblocks + u / 16) * (a.c.nt * 128);
  float v[8];
  const bool in = u * 8 < a.d;
  const int64_t at = token * a.stride + u * 8;
  if (!in) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.0f;
  } else if (a.kind == MLPMOE_FP32) {
    const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(a.x) + at);
    const float4 lo = p[0], hi = p[1];
    v[0] = lo.x, v[1] = lo.y, v[2] = lo.z, v[3] = lo.w, v[4] = hi.x, v[5] = hi.y, v[6] = hi.z, v[7] = hi.w;
  } else if (a.kind == MLPMOE_BF16) {
    const uint4 w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.x) + at);
    v[0] = __uint_as_float(w.x << 16), v[1] = __uint_as_float(w.x & 0xFFFF0000u), v[2] = __uint_as_float(w.y << 16),
    v[3] = __uint_as_float(w.y & 0xFFFF0000u), v[4] = __uint_as_float(w.z << 16), v[5] = __uint_as_float(w.z & 0xFFFF0000u),
    v[6] = __uint_as_float(w.w << 16), v[7] = __uint_as_float(w.w & 0xFFFF0000u);
  } else {
    const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.x) + at);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const __half_raw h = __nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>((e < 4 ? w.x : w.y) >> (8 * (e & 3))), __NV_E4M3);
      v[e] = __half2float(__half(h));
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
    out[unit_at_gpb(a.gpb, p * a.c.tokens + tok, u % 16)] = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Which branches some token computes, every token's factor, and the K-blocks of the down product with a computed branch.
__device__ void prepare_selection(const PrepArgs& a) {
  __shared__ int s_active[kW4MaxBranches];
  __shared__ int s_warp[kPrepThreads / 32];
  __shared__ int s_total;
  int n_avail = 0;
  for (int b = 0; b < a.B; ++b) n_avail += a.alpha[b] != 0.0f ? 1 : 0;
  for (int b = threadIdx.x; b < a.B; b += kPrepThreads) s_active[b] = a.select == nullptr && a.alpha[b] != 0.0f;
  __syncthreads();
  if (a.select != nullptr) {
    for (int i = threadIdx.x; i < a.n * a.B; i += kPrepThreads)
      if (a.select[i] != 0 && a.alpha[i % a.B] != 0.0f) s_active[i % a.B] = 1;
    for (int t = threadIdx.x; t < a.n; t += kPrepThreads) {
      int k = 0;
      for (int b = 0; b < a.B; ++b) k += a.select[t * a.B + b] != 0 && a.alpha[b] != 0.0f ? 1 : 0;
      // the quotient and the root in double, rounded once, as the routed forward does
      float c = 0.0f;
      if (k > 0) c = a.compensate ? static_cast<float>(sqrt(static_cast<double>(n_avail) / static_cast<double>(k))) : 1.0f;
      a.coef[t] = c;
    }
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.B; b += kPrepThreads) a.active[b] = static_cast<uint8_t>(s_active[b]);
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  int running = 0;
  for (int base = 0; base < a.h_kblocks; base += kPrepThreads) {
    const int kb = base + threadIdx.x;
    bool live = false;
    if (kb < a.h_kblocks)
      for (int b = 0; b < a.B; ++b) live = live || (s_active[b] && a.off[b] < (kb + 1) * 128 && a.off[b + 1] > kb * 128);
    const unsigned ballot = __ballot_sync(0xFFFFFFFFu, live);
    if (lane == 0) s_warp[warp] = __popc(ballot);
    __syncthreads();
    int before = running;
    for (int w = 0; w < warp; ++w) before += s_warp[w];
    if (live) a.list[before + __popc(ballot & ((1u << lane) - 1u))] = kb;
    if (threadIdx.x == kPrepThreads - 1) s_total = before + __popc(ballot);
    __syncthreads();
    running = s_total;
    __syncthreads();
  }
  if (threadIdx.x == 0) a.list[a.h_kblocks] = running;
}

__global__ void __launch_bounds__(kPrepThreads) w4_prepare_kernel(const __grid_constant__ PrepArgs a) {
  ptx::griddep_launch_dependents();
  const int block = blockIdx.x;
  if (block < a.unit_blocks) {
    const int64_t i = static_cast<int64_t>(block) * kPrepThreads + threadIdx.x;
    if (i < static_cast<int64_t>(a.n) * a.kblocks * 16) prepare_unit(a, i);
  } else if (block < a.unit_blocks + a.pad_blocks) {
    const int64_t i = static_cast<int64_t>(block - a.unit_blocks) * kPrepThreads + threadIdx.x;
    const int pad = a.h_kblocks * 16 - a.h_unit0;
    if (i >= static_cast<int64_t>(a.n) * pad) return;
    const int u = a.h_unit0 + static_cast<int>(i % pad), token = static_cast<int>(i / pad);
    uint4* out = a.h_frag + (static_cast<int64_t>(token / a.hc.tokens) * a.h_kblocks + u / 16) * (a.hc.nt * 128);
    for (int p = 0; p < a.hc.pieces; ++p)
      out[unit_at_gpb(a.gpb, p * a.hc.tokens + token % a.hc.tokens, u % 16)] = make_uint4(0u, 0u, 0u, 0u);
  } else {
    prepare_selection(a);
  }
}

// Tokens of up to 64 columns share a pass over the weights; equal chunks, and the fewest tiles of eight columns.
W4Cols columns(int64_t n, int pieces) {
  W4Cols c;
  c.pieces = pieces;
  const int64_t most = 64 / pieces;
  c.chunks = static_cast<int>((n + most - 1) / most);
  c.tokens = static_cast<int>((n + c.chunks - 1) / c.chunks);
  c.nt = (c.tokens * pieces + 7) / 8;
  if (c.nt == 5) c.nt = 6;
  if (c.nt == 7) c.nt = 8;
  return c;
}

inline int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
inline int64_t frag_bytes(const W4Cols& c, int64_t kblocks) { return up256(static_cast<int64_t>(c.chunks) * kblocks * c.nt * 2048); }
inline bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Offsets of a workspace; x_bytes and h_bytes are the fragments' sizes.
struct Layout {
  int64_t active, coef, list, x, h, total;
};
Layout layout_of(int64_t n, int64_t h_kblocks, int64_t x_bytes, int64_t h_bytes) {
  Layout l;
  l.active = 0;
  l.coef = up256(kW4MaxBranches);
  l.list = l.coef + up256(4 * n);
  l.x = l.list + up256(4 * (h_kblocks + 1));
  l.h = l.x + x_bytes;
  l.total = l.h + h_bytes;
  return l;
}

mlpmoe_status_t check_matrix(const mlpmoe_w4_matrix_t& m) {
  return !m.q || !m.scale || !on(m.q, 16) || !on(m.scale, 16) || !on(m.zero, 16) ? MLPMOE_ERR_INVALID_ARG : MLPMOE_OK;
}

mlpmoe_status_t check_layer(const mlpmoe_w4_layer_t* l) {
  if (!l || !l->d_b || l->d_model <= 0 || l->d_inter <= 0 || l->B <= 0) return MLPMOE_ERR_INVALID_ARG;
  if (l->B > kW4MaxBranches || l->d_model % 8 != 0 || l->d_model > kW4MaxDim || l->d_inter > kW4MaxDim) return MLPMOE_ERR_UNSUPPORTED;
  if (l->group != 32 && l->group != 64 && l->group != 128) return MLPMOE_ERR_UNSUPPORTED;
  int64_t sum = 0;
  for (int b = 0; b < l->B; ++b) {
    if (l->d_b[b] <= 0 || l->d_b[b] % 16 != 0 || l->d_b[b] > l->d_inter) return MLPMOE_ERR_BAD_PARTITION;
    sum += l->d_b[b];
  }
  if (sum != l->d_inter) return MLPMOE_ERR_BAD_PARTITION;
  for (const mlpmoe_w4_matrix_t* m : {&l->gate, &l->up, &l->down})
    if (check_matrix(*m) != MLPMOE_OK) return MLPMOE_ERR_INVALID_ARG;
  return MLPMOE_OK;
}

W4Mat matrix(const mlpmoe_w4_matrix_t& m, int64_t rows, int64_t cols, int group) {
  W4Mat r;
  r.q = m.q;
  r.scale = static_cast<const __nv_bfloat16*>(m.scale);
  r.zero = m.zero;
  r.pitch = w4_pitch(cols);
  r.rows16 = w4_rows16(rows);
  r.n_groups = (cols + group - 1) / group;
  return r;
}

// Warps of a block along the rows: as many as still leave two blocks for every SM (the other warps share K), so that
// the blocks in flight keep the memory busy.
int warps_along_rows(int tiles, int chunks) {
  int wr = kW4Warps;
  while (wr > 1 && static_cast<int64_t>((tiles + wr - 1) / wr) * chunks < 296) wr /= 2;
  return wr;
}

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" {

mlpmoe_status_t mlpmoe_w4_workspace(const mlpmoe_w4_layer_t* layer, int64_t n_tokens, int64_t* bytes) {
  if (!bytes) return MLPMOE_ERR_INVALID_ARG;
  const mlpmoe_status_t rc = check_layer(layer);
  if (rc != MLPMOE_OK) return rc;
  if (n_tokens < 0) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens > kW4MaxTokens) return MLPMOE_ERR_UNSUPPORTED;
  const int64_t xk = (layer->d_model + 127) / 128, hk = (layer->d_inter + 127) / 128;
  int64_t xb = 0, hb = 0;
  if (n_tokens > 0) {
    for (int p = 1; p <= 3; ++p) {
      const W4Cols c = columns(n_tokens, p);
      const int64_t x = frag_bytes(c, xk), h = frag_bytes(c, hk);
      xb = x > xb ? x : xb;
      hb = h > hb ? h : hb;
    }
  }
  *bytes = layout_of(n_tokens, hk, xb, hb).total;
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_w4_forward(const mlpmoe_w4_layer_t* layer, const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride,
                                  const float* x_scale, int64_t x_group, const uint8_t* select, int32_t compensate,
                                  const float* residual, void* y, mlpmoe_dtype_t y_dtype, int64_t n_tokens, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  int64_t need = 0;
  const mlpmoe_status_t rc = mlpmoe_w4_workspace(layer, n_tokens, &need);
  if (rc != MLPMOE_OK) return rc;
  const int64_t d = layer->d_model, I = layer->d_inter;
  if (x_dtype != MLPMOE_BF16 && x_dtype != MLPMOE_FP32 && x_dtype != MLPMOE_E4M3) return MLPMOE_ERR_INVALID_ARG;
  if (y_dtype != MLPMOE_BF16 && y_dtype != MLPMOE_FP32) return MLPMOE_ERR_INVALID_ARG;
  if (x_stride == 0) x_stride = d;
  if (x_stride < d || x_stride % 8 != 0) return MLPMOE_ERR_INVALID_ARG;
  const bool scaled = x_dtype == MLPMOE_E4M3;
  if (scaled && x_group != 0) {
    if (x_group != 32 && x_group != 64 && x_group != 128) return MLPMOE_ERR_INVALID_ARG;
    if (x_group < layer->group) return MLPMOE_ERR_UNSUPPORTED;
  }
  if (n_tokens == 0) return MLPMOE_OK;
  if (!x || !y || !on(x, 16) || !on(y, 16) || !on(residual, 16) || (scaled && (!x_scale || !on(x_scale, 4)))) return MLPMOE_ERR_INVALID_ARG;
  if (residual && residual == y && y_dtype != MLPMOE_FP32) return MLPMOE_ERR_INVALID_ARG;
  if (!workspace || workspace_bytes < need || !on(workspace, 256)) return MLPMOE_ERR_INVALID_ARG;

  const int group = layer->group, gpb = 128 / group, n = static_cast<int>(n_tokens);
  bool dense = select == nullptr;
  for (int b = 0; b < layer->B; ++b) dense = dense && (!layer->alpha || layer->alpha[b] != 0.0f);
  const int xk = static_cast<int>((d + 127) / 128), hk = static_cast<int>((I + 127) / 128);
  const W4Cols xc = columns(n, x_dtype == MLPMOE_FP32 ? 3 : 1), hc = columns(n, y_dtype == MLPMOE_FP32 ? 3 : 2);
  const Layout l = layout_of(n, hk, frag_bytes(xc, xk), frag_bytes(hc, hk));
  char* ws = static_cast<char*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  PrepArgs p = {};
  p.x = x;
  p.stride = x_stride;
  p.kind = x_dtype;
  p.gpb = gpb;
  p.d = static_cast<int>(d);
  p.n = n;
  p.c = xc;
  p.kblocks = xk;
  p.frag = reinterpret_cast<uint4*>(ws + l.x);
  p.hc = hc;
  p.h_kblocks = hk;
  p.h_unit0 = static_cast<int>(I / 8);
  p.h_frag = reinterpret_cast<uint4*>(ws + l.h);
  p.unit_blocks = static_cast<int>((static_cast<int64_t>(n) * xk * 16 + kPrepThreads - 1) / kPrepThreads);
  p.pad_blocks = static_cast<int>((static_cast<int64_t>(n) * (hk * 16 - p.h_unit0) + kPrepThreads - 1) / kPrepThreads);
  p.select = select;
  p.B = layer->B;
  p.compensate = compensate ? 1 : 0;
  p.active = reinterpret_cast<uint8_t*>(ws + l.active);
  p.coef = reinterpret_cast<float*>(ws + l.coef);
  p.list = reinterpret_cast<int32_t*>(ws + l.list);
  for (int b = 0; b < layer->B; ++b) {
    p.off[b + 1] = p.off[b] + static_cast<int32_t>(layer->d_b[b]);
    p.alpha[b] = layer->alpha ? layer->alpha[b] : 1.0f;
  }

  W4Args u = {};
  u.m[0] = matrix(layer->gate, I, d, group);
  u.m[1] = matrix(layer->up, I, d, group);
  u.rows = static_cast<int>(I);
  u.tiles = static_cast<int>(I / 8);
  u.kblocks = xk;
  u.n = n;
  u.c = xc;
  u.frag = p.frag;
  if (scaled) {
    u.x_scale = x_scale;
    u.x_groups = x_group == 0 ? 1 : static_cast<int>((d + x_group - 1) / x_group);
    for (int64_t g = group; x_group != 0 && g < x_group; g *= 2) ++u.x_shift;
  }
  u.select = select;
  u.active = p.active;
  u.B = layer->B;
  u.hc = hc;
  u.h_kblocks = hk;
  u.h_frag = reinterpret_cast<__nv_bfloat16*>(ws + l.h);
  u.dense = dense ? 1 : 0;
  memcpy(u.off, p.off, sizeof(u.off));
  memcpy(u.alpha, p.alpha, sizeof(u.alpha));
  u.wr = warps_along_rows(u.tiles, xc.chunks);
  u.wk = kW4Warps / u.wr;

  W4Args w = {};
  w.m[0] = w.m[1] = matrix(layer->down, d, I, group);
  w.rows = static_cast<int>(d);
  w.tiles = static_cast<int>((d + 15) / 16);
  w.kblocks = hk;
  w.n = n;
  w.c = hc;
  w.frag = p.h_frag;
  w.list = dense ? nullptr : p.list;
  w.B = layer->B;
  w.dense = u.dense;
  w.coef = select ? p.coef : nullptr;
  w.residual = residual;
  w.y = y;
  w.y_bf16 = y_dtype == MLPMOE_BF16 ? 1 : 0;
  w.d = d;
  w.wr = warps_along_rows(w.tiles, hc.chunks);
  w.wk = kW4Warps / w.wr;
  // few rows: the blocks of a cluster share K, as long as every warp keeps two blocks of it
  int cluster = 1;
  while (cluster < 8 && static_cast<int64_t>((w.tiles + w.wr - 1) / w.wr) * hc.chunks * cluster < 222 && hk >= 4 * cluster * w.wk) cluster *= 2;

  // an ordinary launch: it begins when everything before it on the stream is complete, which the early copies of the
  // weights in the next two rely on
  w4_prepare_kernel<<<static_cast<unsigned>(p.unit_blocks + p.pad_blocks + (dense ? 0 : 1)), kPrepThreads, 0, st>>>(p);
  if (cudaGetLastError() != cudaSuccess) return MLPMOE_ERR_CUDA;
  cudaError_t e = group == 32 ? launch_w4_gateup_32(u, st) : (group == 64 ? launch_w4_gateup_64(u, st) : launch_w4_gateup_128(u, st));
  if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  e = group == 32 ? launch_w4_down_32(w, cluster, st) : (group == 64 ? launch_w4_down_64(w, cluster, st) : launch_w4_down_128(w, cluster, st));
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
