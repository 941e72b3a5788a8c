// Entry point of the layer on 4-bit weights (mlpmoe_w4_forward): checks and the split of the work.  Two launches, gate|up
// and down; the second begins with its copies of the weights while the first runs.
#include <string.h>

#include "../../include/mlpmoe.h"
#include "w4_kernel.cuh"

namespace mlpmoe {

// How a product is split.  Clusters of 1, 2, 4 or 8 blocks share K (148, 74, 33 or 15 of them are resident at once with
// this much shared memory, as the occupancy query reports); the row tiles are cut into equal shares, one per cluster,
// or two or more turns of them where the sums of a share would not fit; and a chunk has as many tokens as fit, up to
// 24 columns.  Of the splits that fit, the one that moves the fewest bytes through the busiest SM is taken, a
// cluster's exchange counted like 32 KB: the weights of its steps, the activations, the sums.
int w4_plan(W4Args* a, int pieces, int group) {
  static const int kResident[4] = {148, 74, 33, 15};
  const int gpb = 128 / group;
  const int64_t stage = 2048 + 96 * gpb;
  int best = 0;
  int64_t best_cost = INT64_MAX;
  W4Args pick = *a;
  for (int i = 0; i < 4; ++i) {
    const int cluster = 1 << i;
    if (cluster > 1 && a->kblocks < 4 * cluster) break;
    const int entries = ((a->kblocks + cluster - 1) / cluster + 1) / 2 * 2;
    bool found = false;
    for (int turns = 1; turns <= 64 && !found; ++turns) {
      const int slots = kResident[i] * turns;
      const int per = (a->tiles + slots - 1) / slots;
      int tokens = 24 / pieces < a->n ? 24 / pieces : a->n;
      for (; tokens > 0; --tokens) {
        const int cols = pieces * tokens, nt = (cols + 7) / 8;
        const int64_t ring = w4::kWarps * w4::stages(nt) * stage;
        const int64_t x = static_cast<int64_t>(entries) * nt * 1024, units = static_cast<int64_t>(entries) * gpb * nt * 64;
        const int64_t sums = static_cast<int64_t>(w4::kWarps - 1 + per) * nt * 8 * w4::kColPitch * 4;
        const int64_t own = static_cast<int64_t>(per) * tokens * 64;
        if (ring + x + units + sums + entries * 4 + per * 12 + (a->dense ? 0 : 8 * (a->B + 1) + tokens * a->B) > w4::kSmemMax || own > ring + x) continue;
        const int chunks = (a->n + tokens - 1) / tokens;
        const int even = (a->n + chunks - 1) / chunks;
        const int64_t blocks = static_cast<int64_t>((a->tiles + per - 1) / per) * chunks;
        const int64_t waves = (blocks + kResident[i] - 1) / kResident[i];
        const int64_t steps = (static_cast<int64_t>(per) * (entries / 2) + w4::kWarps - 1) / w4::kWarps;
        const int64_t cost = waves * (steps * w4::kWarps * stage + static_cast<int64_t>(entries) * even * 512 +
                                      static_cast<int64_t>(per) * even * 128 + (cluster > 1 ? 32768 : 0));
        if (cost < best_cost) {
          best_cost = cost;
          best = cluster;
          pick.tiles_per_block = per;
          pick.entries = entries;
          pick.c.pieces = pieces;
          pick.c.tokens = even;
          pick.c.chunks = chunks;
        }
        found = true;
        break;
      }
    }
  }
  *a = pick;
  return best;
}

namespace {

inline bool on(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

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
    if (!m->q || !m->scale || !on(m->q, 16) || !on(m->scale, 16) || !on(m->zero, 16)) return MLPMOE_ERR_INVALID_ARG;
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

inline int64_t h_bytes(const mlpmoe_w4_layer_t* l, int64_t n) { return (n * l->d_inter * 4 + 255) / 256 * 256; }

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
  *bytes = h_bytes(layer, n_tokens);
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_w4_forward(const mlpmoe_w4_layer_t* layer, const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride,
                                  const float* x_scale, int64_t x_group, const uint8_t* select, int32_t compensate,
                                  const float* residual, void* y, mlpmoe_dtype_t y_dtype, int64_t n_tokens, void* workspace,
                                  int64_t workspace_bytes, void* stream) {
  const mlpmoe_status_t rc = check_layer(layer);
  if (rc != MLPMOE_OK) return rc;
  if (n_tokens < 0) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens > kW4MaxTokens) return MLPMOE_ERR_UNSUPPORTED;
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

  if (!workspace || workspace_bytes < h_bytes(layer, n_tokens) || !on(workspace, 256)) return MLPMOE_ERR_INVALID_ARG;

  const int group = layer->group, n = static_cast<int>(n_tokens), digits = y_dtype == MLPMOE_FP32 ? 3 : 2;
  W4Args u = {};
  u.m[0] = matrix(layer->gate, I, d, group);
  u.m[1] = matrix(layer->up, I, d, group);
  u.rows = static_cast<int>(I);
  u.tiles = static_cast<int>(I / 8);
  u.K = static_cast<int>(d);
  u.kblocks = static_cast<int>((d + 127) / 128);
  u.n = n;
  if (scaled) {
    u.x_scale = x_scale;
    u.x_groups = x_group == 0 ? 1 : static_cast<int>((d + x_group - 1) / x_group);
    for (int64_t g = group; x_group != 0 && g < x_group; g *= 2) ++u.x_shift;
  }
  u.B = layer->B;
  u.select = select;
  u.dense = select == nullptr;
  for (int b = 0; b < layer->B; ++b) {
    u.off[b + 1] = u.off[b] + static_cast<int32_t>(layer->d_b[b]);
    u.alpha[b] = layer->alpha ? layer->alpha[b] : 1.0f;
    if (u.alpha[b] == 0.0f) u.dense = 0;
  }
  const int u_cluster = w4_plan(&u, digits, group);
  u.x = x;
  u.x_kind = x_dtype;
  u.x_stride = x_stride;
  u.h = static_cast<float*>(workspace);

  W4Args w = {};
  w.m[0] = w.m[1] = matrix(layer->down, d, I, group);
  w.rows = static_cast<int>(d);
  w.tiles = static_cast<int>((d + 15) / 16);
  w.K = static_cast<int>(I);
  w.kblocks = static_cast<int>((I + 127) / 128);
  w.n = n;
  w.B = u.B;
  w.dense = u.dense;
  const int w_cluster = w4_plan(&w, digits, group);
  if (u_cluster == 0 || w_cluster == 0) return MLPMOE_ERR_UNSUPPORTED;
  w.x = workspace;
  w.x_kind = MLPMOE_FP32;
  w.x_stride = I;
  w.select = select;
  memcpy(w.off, u.off, sizeof(u.off));
  memcpy(w.alpha, u.alpha, sizeof(u.alpha));
  w.compensate = compensate ? 1 : 0;
  w.residual = residual;
  w.y = y;
  w.y_bf16 = y_dtype == MLPMOE_BF16 ? 1 : 0;

  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = group == 32 ? launch_w4_gateup_32(u, u_cluster, st)
                              : (group == 64 ? launch_w4_gateup_64(u, u_cluster, st) : launch_w4_gateup_128(u, u_cluster, st));
  if (e != cudaSuccess) return MLPMOE_ERR_CUDA;
  e = group == 32 ? launch_w4_down_32(w, w_cluster, st) : (group == 64 ? launch_w4_down_64(w, w_cluster, st) : launch_w4_down_128(w, w_cluster, st));
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
