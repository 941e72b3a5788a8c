// Entry point of the layer on 4-bit weights (mlpmoe_w4_forward): checks, which kernels run, and the split of the work.  Two
// launches for a few tokens, gate|up and down; the second begins with its copies of the weights while the first runs.  Four for
// more (the activations of each product are prepared first), three on the tensor cores' kernels.
#include <string.h>

#include <atomic>

#include "../../include/mlpmoe.h"
#include "w4_kernel.cuh"

namespace mlpmoe {

// Clusters of 1, 2, 4 and 8 blocks of one SM each that are resident at once (what the occupancy query reports).
static constexpr int kResident[4] = {148, 74, 33, 15};

// How a product is split.  Clusters of 1, 2, 4 or 8 blocks share K; the row tiles are cut into equal shares, one per cluster,
// or two or more turns of them where the sums of a share would not fit; and a chunk has as many tokens as fit, up to
// 24 columns.  Of the splits that fit, the one that moves the fewest bytes through the busiest SM is taken, a
// cluster's exchange counted like 32 KB: the weights of its steps, the activations, the sums.
int w4_plan(W4Args* a, int pieces, int group) {
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

// From how many tokens on the tiled kernels are used.  The streaming kernels read the weights once per 24 columns at most, twelve
// tokens of two digits or eight of three.  4096 x 14336, y bf16, streaming / tiled: 8 tokens 44 / 55 us, 9 tokens 71 / 52.
constexpr int kWideFrom = 9;

// Tiles of eight columns for `slots` slots: 1, 2, 3, 4, 6, 8, 12 or 16, which divide among the warps of a block.
int wide_tiles(int slots) {
  int tiles = (slots + 3) / 4;
  if (tiles > 12) return 16;
  if (tiles > 8) return 12;
  if (tiles > 4) return tiles + (tiles & 1);
  return tiles;
}

// How a product of many tokens is split: fills the chunk, the warps of a block and entries; returns the cluster.  Of the
// splits that fit, the one with the least time by the counts of an SM's cycles per K-block: tensor core, reads of
// shared memory, instructions, memory.
int wide_plan(W4WideArgs* a, int pieces, int group, bool may_share_k) {
  const int gpb = 128 / group;
  a->slots_per_token = pieces - 1;
  const int most = kW4WideSlots / a->slots_per_token, chunks = (a->n + most - 1) / most;
  a->tokens = (a->n + chunks - 1) / chunks;
  a->slot_tiles = wide_tiles(a->tokens * a->slots_per_token);
  const int tiles = a->slot_tiles;
  int best = 0;
  int64_t best_cost = INT64_MAX;
  W4WideArgs pick = *a;
  for (int i = 0; i < (may_share_k ? 4 : 1); ++i) {
    const int cluster = 1 << i, entries = (a->kblocks + cluster - 1) / cluster;
    if (cluster > 1 && a->kblocks < 4 * cluster) break;
    for (int rg = 1; rg <= 8; ++rg) {
      const int cg_most = 16 / rg < tiles ? 16 / rg : tiles;
      const int64_t blocks = static_cast<int64_t>((a->tiles + 2 * rg - 1) / (2 * rg)) * chunks;
      const int64_t waves = (blocks + kResident[i] - 1) / kResident[i];
      for (int cg = 4; cg >= 1; cg /= 2) {
        if (cg > cg_most) continue;
        if (tiles % cg != 0 || (cg == 1 && tiles % 2 == 0)) continue;
        const int nt = tiles / cg;
        if (nt > 8) break;
        const int64_t warps = rg * cg;
        int64_t cycles = 16 * rg * tiles;                                                        // mma: 4 per tile pair and 16 rows, 2 each
        const int64_t reads = warps * (9 * nt + 20), issue = warps * (120 + 40 * nt) / 4, memory = 100 * rg + 45 * tiles;
        if (reads > cycles) cycles = reads;
        if (issue > cycles) cycles = issue;
        if (memory > cycles) cycles = memory;
        const int64_t own = static_cast<int64_t>(a->tokens) * (32 * rg + 4) * 4;
        if (kW4WideStages * w4_wide_stage_bytes(rg, tiles, gpb) > w4::kWideSmemMax || own > w4::kWideSmemMax) continue;
        const int64_t cost = waves * (entries * (cycles + 200) + 4000 + (cluster > 1 ? 4000 : 0));
        if (cost < best_cost) {
          best_cost = cost;
          best = cluster;
          pick.row_groups = rg;
          pick.col_groups = cg;
          pick.entries = entries;
        }
      }
    }
  }
  *a = pick;
  return best;
}

inline int chunks_of(const W4WideArgs& a) { return (a.n + a.tokens - 1) / a.tokens; }
inline int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }
// Digits and units of a product's activations.
inline int64_t digit_bytes(int64_t n, int pieces, int64_t kblocks, int gpb, int64_t* units) {
  const int spt = pieces - 1, most = kW4WideSlots / spt;
  const int64_t chunks = (n + most - 1) / most, tokens = (n + chunks - 1) / chunks, tiles = wide_tiles(static_cast<int>(tokens * spt));
  *units = up256(chunks * kblocks * gpb * tiles * 32);
  return up256(chunks * kblocks * tiles * 1024);
}

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

// From how many codes times tokens on the kernels of the 5th-generation tensor cores are used (y bf16, which is what their fp16
// operand is precise enough for), instead of the tiled kernels.  Measured, tiled / tensor, in us: 4096 x 14336, 9 tokens 52 / 47,
// 16 tokens 66 / 48, 64 tokens 129 / 53; 2048 x 8192, 16 tokens 26.5 / 27.0, 24 tokens 36 / 28; 896 x 4864, 32 tokens
// 20.5 / 21.1, 64 tokens 27.6 / 24.3; 512 x 2048, 64 tokens 17 / 22.  With fewer rows than their tile's 128 most of it is padding.
constexpr int64_t kTcWork = int64_t(768) << 20;

// Limits of the bounded waits of the tensor cores' kernels; changed by the test hook only.
std::atomic<uint64_t> g_wait_limit_ns{1000000000ull};
std::atomic<uint32_t> g_extra_arrivals{0};

// The streaming kernels' split of both products.
struct StreamPlan {
  W4Args u, w;                  // gate|up, down
  int u_cluster, w_cluster;     // 0: no split
};
void plan_stream(const mlpmoe_w4_layer_t* l, int n, int digits, bool dense, StreamPlan* p) {
  const int64_t d = l->d_model, I = l->d_inter;
  p->u = W4Args{};
  p->u.rows = static_cast<int>(I);
  p->u.tiles = static_cast<int>(I / 8);
  p->u.K = static_cast<int>(d);
  p->u.kblocks = static_cast<int>((d + 127) / 128);
  p->u.n = n;
  p->u.B = l->B;
  p->u.dense = dense;
  p->w = W4Args{};
  p->w.rows = static_cast<int>(d);
  p->w.tiles = static_cast<int>((d + 15) / 16);
  p->w.K = static_cast<int>(I);
  p->w.kblocks = static_cast<int>((I + 127) / 128);
  p->w.n = n;
  p->w.B = l->B;
  p->w.dense = dense;
  p->u_cluster = w4_plan(&p->u, digits, l->group);
  p->w_cluster = p->u_cluster == 0 ? 0 : w4_plan(&p->w, digits, l->group);
}

inline int digits_of(mlpmoe_dtype_t y_dtype) { return y_dtype == MLPMOE_FP32 ? 3 : 2; }

// A few tokens stream, unless a block's share of a row's activations does not fit beside the rings even where eight blocks share K
// (group 32: from about 49,000 columns on; group 64: both dimensions near 65,536); the tiled kernels stream K.  Fills the plan where
// the answer is STREAM.
enum Path { STREAM, WIDE, TENSOR };
Path path_of(const mlpmoe_w4_layer_t* l, int64_t n, mlpmoe_dtype_t y_dtype, bool dense, StreamPlan* plan) {
  if (n < kWideFrom) {
    if (n == 0) return STREAM;
    plan_stream(l, static_cast<int>(n), digits_of(y_dtype), dense, plan);
    return plan->w_cluster != 0 ? STREAM : WIDE;
  }
  if (y_dtype != MLPMOE_BF16 || l->d_model < 128 || l->d_inter < 128) return WIDE;
  return n * (3 * l->d_model * l->d_inter) >= kTcWork ? TENSOR : WIDE;
}

// A chunk of the tensor cores' products: tokens, and the columns of an epilogue warp, 32 or 64.  gate|up has one such set of columns
// for each matrix, down two.
struct TcChunk {
  int tokens, chunks, ne;
};
TcChunk tc_chunk(int64_t n, int sets) {
  TcChunk c;
  const int64_t most = 64 * sets;
  c.chunks = static_cast<int>((n + most - 1) / most);
  c.tokens = static_cast<int>((n + c.chunks - 1) / c.chunks);
  c.ne = c.tokens <= 32 * sets ? 32 : 64;
  return c;
}
inline TcChunk tc_up_chunk(int64_t n) { return tc_chunk(n, 1); }
inline TcChunk tc_down_chunk(int64_t n) { return tc_chunk(n, 2); }

// Workspace: a status word, the intermediate activations in fp32 (the tensor cores' kernels have them only as an image), then the
// activations of both products as the tiled kernels (digits, units) or the tensor cores' kernels (images) read them.
struct Layout {
  int64_t h, x, x_units, y, y_units, total;
};
Layout layout_of(const mlpmoe_w4_layer_t* l, int64_t n, Path path, int digits) {
  Layout w;
  const int gpb = 128 / l->group;
  const int64_t xk = (l->d_model + 127) / 128, hk = (l->d_inter + 127) / 128;
  int64_t xb = 0, xu = 0, hb = 0, hu = 0;
  if (path == WIDE) {
    xb = digit_bytes(n, digits, xk, gpb, &xu);
    hb = digit_bytes(n, digits, hk, gpb, &hu);
  } else if (path == TENSOR) {
    const TcChunk u = tc_up_chunk(n), d = tc_down_chunk(n);
    xb = u.chunks * xk * u.ne * 256;
    xu = up256(n * 4);
    hb = d.chunks * hk * d.ne * 512;
    hu = d.chunks * hk * d.ne * 8;
  }
  w.h = 256;
  w.x = w.h + (path == TENSOR ? 0 : up256(n * l->d_inter * 4));
  w.x_units = w.x + xb;
  w.y = w.x_units + xu;
  w.y_units = w.y + hb;
  w.total = w.y_units + hu;
  return w;
}

#define BY_GROUP(call, group, ...) \
  ((group) == 32 ? launch_w4_##call##_32(__VA_ARGS__) : ((group) == 64 ? launch_w4_##call##_64(__VA_ARGS__) : launch_w4_##call##_128(__VA_ARGS__)))

// Digits of x, gate|up, digits of h, down.
mlpmoe_status_t forward_wide(const mlpmoe_w4_layer_t* layer, const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride, const float* x_scale,
                             int64_t x_group, const uint8_t* select, int32_t compensate, const float* residual, void* y,
                             mlpmoe_dtype_t y_dtype, int n, void* workspace, void* stream) {
  const int64_t d = layer->d_model, I = layer->d_inter;
  const int group = layer->group, pieces = y_dtype == MLPMOE_FP32 ? 3 : 2;
  const Layout l = layout_of(layer, n, WIDE, pieces);
  char* ws = static_cast<char*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  W4WideArgs u = {};
  u.m[0] = matrix(layer->gate, I, d, group);
  u.m[1] = matrix(layer->up, I, d, group);
  u.rows = static_cast<int>(I);
  u.tiles = u.rows / 8;
  u.kblocks = static_cast<int>((d + 127) / 128);
  u.n = n;
  u.B = layer->B;
  u.select = select;
  u.dense = select == nullptr;
  for (int b = 0; b < layer->B; ++b) {
    u.off[b + 1] = u.off[b] + static_cast<int32_t>(layer->d_b[b]);
    u.alpha[b] = layer->alpha ? layer->alpha[b] : 1.0f;
    if (u.alpha[b] == 0.0f) u.dense = 0;
  }
  W4WideArgs w = u;
  w.m[0] = w.m[1] = matrix(layer->down, d, I, group);
  w.rows = static_cast<int>(d);
  w.tiles = (w.rows + 15) / 16;
  w.kblocks = static_cast<int>((I + 127) / 128);
  const int u_cluster = wide_plan(&u, pieces, group, false), w_cluster = wide_plan(&w, pieces, group, true);
  if (u_cluster == 0 || w_cluster == 0) return MLPMOE_ERR_UNSUPPORTED;
  u.digits = reinterpret_cast<uint8_t*>(ws + l.x);
  u.units = reinterpret_cast<float2*>(ws + l.x_units);
  u.h = reinterpret_cast<float*>(ws + l.h);
  w.digits = reinterpret_cast<uint8_t*>(ws + l.y);
  w.units = reinterpret_cast<float2*>(ws + l.y_units);
  w.compensate = compensate ? 1 : 0;
  w.residual = residual;
  w.y = y;
  w.y_bf16 = y_dtype == MLPMOE_BF16 ? 1 : 0;

  W4DigitsArgs p = {};
  p.x = x;
  p.kind = x_dtype;
  p.stride = x_stride;
  if (x_dtype == MLPMOE_E4M3) {
    p.x_scale = x_scale;
    p.x_groups = x_group == 0 ? 1 : static_cast<int>((d + x_group - 1) / x_group);
    for (int64_t g = group; x_group != 0 && g < x_group; g *= 2) ++p.x_shift;
  }
  p.K = static_cast<int>(d);
  p.kblocks = u.kblocks;
  p.n = n;
  p.tokens = u.tokens;
  p.slots_per_token = u.slots_per_token;
  p.slot_tiles = u.slot_tiles;
  p.digits = const_cast<uint8_t*>(u.digits);
  p.units = const_cast<float2*>(u.units);
  p.status = reinterpret_cast<uint32_t*>(ws);
  W4DigitsArgs q = p;
  q.status = nullptr;
  q.x = ws + l.h;
  q.kind = MLPMOE_FP32;
  q.stride = I;
  q.x_scale = nullptr;
  q.K = static_cast<int>(I);
  q.kblocks = w.kblocks;
  q.digits = const_cast<uint8_t*>(w.digits);
  q.units = const_cast<float2*>(w.units);

  pdl_overlap_enabled() = true;
  if (BY_GROUP(digits, group, p, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  if (BY_GROUP(wide_gateup, group, u, chunks_of(u), st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  if (BY_GROUP(digits, group, q, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  return BY_GROUP(wide_down, group, w, w_cluster, chunks_of(w), st) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

// The cluster along K of a product: 1, 2, 4 or 8 blocks, whichever takes the fewest turns of K-blocks (a turn is what one
// block per SM does at a time; six K-blocks' time for the start and the end, six more for the exchange).  4096 x 14336: gate|up
// 112 blocks alone, down clusters of four, 28 K-blocks to a block; alone its 32 blocks would have 112 each.
int tc_cluster(int64_t blocks, int64_t kblocks) {
  int best = 1;
  int64_t best_cost = INT64_MAX;
  for (int i = 0; i < 4; ++i) {
    const int64_t cluster = 1 << i, entries = (kblocks + cluster - 1) / cluster, waves = (blocks + kResident[i] - 1) / kResident[i];
    if (cluster > 1 && kblocks < 2 * cluster) break;
    const int64_t cost = waves * (entries + 6 + (cluster > 1 ? 6 : 0));
    if (cost < best_cost) best_cost = cost, best = static_cast<int>(cluster);
  }
  return best;
}

// Codes as boxes of 128 rows x 64 bytes.
bool code_map(CUtensorMap* map, const W4Mat& m, int64_t rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    const bool ok = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
    return ok ? reinterpret_cast<Encode>(p) : nullptr;
  }();
  const cuuint64_t dim[2] = {static_cast<cuuint64_t>(m.pitch), static_cast<cuuint64_t>(rows)}, stride[1] = {static_cast<cuuint64_t>(m.pitch)};
  const cuuint32_t box[2] = {64, 128}, one[2] = {1, 1};
  return encode != nullptr && encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(m.q), dim, stride, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                     CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Columns of x, gate|up, down.
mlpmoe_status_t forward_tc(const mlpmoe_w4_layer_t* layer, const void* x, mlpmoe_dtype_t x_dtype, int64_t x_stride, const float* x_scale,
                           int64_t x_group, const uint8_t* select, int32_t compensate, const float* residual, void* y, int n,
                           void* workspace, void* stream) {
  const int64_t d = layer->d_model, I = layer->d_inter;
  const int group = layer->group;
  const Layout l = layout_of(layer, n, TENSOR, 2);
  const TcChunk uc = tc_up_chunk(n), wc = tc_down_chunk(n);
  char* ws = static_cast<char*>(workspace);
  cudaStream_t st = static_cast<cudaStream_t>(stream);

  W4TcArgs u = {};
  u.m[0] = matrix(layer->gate, I, d, group);
  u.m[1] = matrix(layer->up, I, d, group);
  u.rows = static_cast<int>(I);
  u.kblocks = static_cast<int>((d + 127) / 128);
  u.n = n;
  u.tokens = uc.tokens;
  u.ne = uc.ne;
  u.image = reinterpret_cast<uint8_t*>(ws + l.x);
  u.unit = reinterpret_cast<float*>(ws + l.x_units);
  u.B = layer->B;
  u.select = select;
  u.dense = select == nullptr;
  for (int b = 0; b < layer->B; ++b) {
    u.off[b + 1] = u.off[b] + static_cast<int32_t>(layer->d_b[b]);
    u.alpha[b] = layer->alpha ? layer->alpha[b] : 1.0f;
    if (u.alpha[b] == 0.0f) u.dense = 0;
  }
  u.h = reinterpret_cast<uint8_t*>(ws + l.y);
  u.h_unit = reinterpret_cast<float*>(ws + l.y_units);
  u.h_tokens = wc.tokens;
  u.h_cols = 2 * wc.ne;
  u.status = reinterpret_cast<uint32_t*>(ws);
  u.wait_limit_ns = g_wait_limit_ns.load();
  u.extra_arrivals = g_extra_arrivals.load();
  W4TcArgs w = u;
  w.m[0] = w.m[1] = matrix(layer->down, d, I, group);
  w.rows = static_cast<int>(d);
  w.kblocks = static_cast<int>((I + 127) / 128);
  w.tokens = wc.tokens;
  w.ne = wc.ne;
  w.image = u.h;
  w.unit = u.h_unit;
  w.compensate = compensate ? 1 : 0;
  w.residual = residual;
  w.y = static_cast<__nv_bfloat16*>(y);
  if (!code_map(&u.codes[0], u.m[0], I) || !code_map(&u.codes[1], u.m[1], I) || !code_map(&w.codes[0], w.m[0], d)) return MLPMOE_ERR_CUDA;

  W4ColumnsArgs p = {};
  p.x = x;
  p.kind = x_dtype;
  p.stride = x_stride;
  if (x_dtype == MLPMOE_E4M3) {
    p.x_scale = x_scale;
    p.x_group = static_cast<int>(x_group);
    p.x_groups = x_group == 0 ? 1 : static_cast<int>((d + x_group - 1) / x_group);
  }
  p.K = static_cast<int>(d);
  p.kblocks = u.kblocks;
  p.n = n;
  p.tokens = u.tokens;
  p.cols = u.ne;
  p.image = const_cast<uint8_t*>(u.image);
  p.unit = const_cast<float*>(u.unit);
  p.status = u.status;
  pdl_overlap_enabled() = true;
  if (launch_w4_columns(p, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  if (BY_GROUP(tc_gateup, group, u, tc_cluster((I + 127) / 128 * uc.chunks, u.kblocks), st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  return BY_GROUP(tc_down, group, w, tc_cluster((d + 127) / 128 * wc.chunks, w.kblocks), st) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
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
  // the most that a call with any types, with or without a selection, needs
  *bytes = 0;
  for (const mlpmoe_dtype_t y_dtype : {MLPMOE_FP32, MLPMOE_BF16}) {
    for (const bool dense : {false, true}) {
      StreamPlan plan;
      const int64_t total = layout_of(layer, n_tokens, path_of(layer, n_tokens, y_dtype, dense, &plan), digits_of(y_dtype)).total;
      if (total > *bytes) *bytes = total;
    }
  }
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_w4_get_status(const void* workspace, void* stream) {
  if (!workspace || !on(workspace, 256)) return MLPMOE_ERR_INVALID_ARG;
  uint32_t word = 0;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (cudaMemcpyAsync(&word, workspace, sizeof(word), cudaMemcpyDeviceToHost, st) != cudaSuccess || cudaStreamSynchronize(st) != cudaSuccess)
    return MLPMOE_ERR_CUDA;
  return word == kStatusOk ? MLPMOE_OK : MLPMOE_ERR_DEVICE_TIMEOUT;
}

mlpmoe_status_t mlpmoe_w4_debug_set_wait(uint64_t limit_ns, uint32_t extra_arrivals) {
  g_wait_limit_ns = limit_ns ? limit_ns : 1000000000ull;
  g_extra_arrivals = extra_arrivals;
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

  bool dense = select == nullptr;
  for (int b = 0; b < layer->B && layer->alpha != nullptr; ++b) dense = dense && layer->alpha[b] != 0.0f;
  StreamPlan plan;
  const Path path = path_of(layer, n_tokens, y_dtype, dense, &plan);
  const Layout l = layout_of(layer, n_tokens, path, digits_of(y_dtype));
  if (!workspace || workspace_bytes < l.total || !on(workspace, 256)) return MLPMOE_ERR_INVALID_ARG;

  const int group = layer->group, n = static_cast<int>(n_tokens);
  if (path == TENSOR) return forward_tc(layer, x, x_dtype, x_stride, x_scale, x_group, select, compensate, residual, y, n, workspace, stream);
  if (path == WIDE)
    return forward_wide(layer, x, x_dtype, x_stride, x_scale, x_group, select, compensate, residual, y, y_dtype, n, workspace, stream);
  W4Args& u = plan.u;
  u.m[0] = matrix(layer->gate, I, d, group);
  u.m[1] = matrix(layer->up, I, d, group);
  if (scaled) {
    u.x_scale = x_scale;
    u.x_groups = x_group == 0 ? 1 : static_cast<int>((d + x_group - 1) / x_group);
    for (int64_t g = group; x_group != 0 && g < x_group; g *= 2) ++u.x_shift;
  }
  u.select = select;
  for (int b = 0; b < layer->B; ++b) {
    u.off[b + 1] = u.off[b] + static_cast<int32_t>(layer->d_b[b]);
    u.alpha[b] = layer->alpha ? layer->alpha[b] : 1.0f;
  }
  u.x = x;
  u.x_kind = x_dtype;
  u.x_stride = x_stride;
  u.h = reinterpret_cast<float*>(static_cast<char*>(workspace) + l.h);
  u.status = static_cast<uint32_t*>(workspace);

  W4Args& w = plan.w;
  w.m[0] = w.m[1] = matrix(layer->down, d, I, group);
  w.x = u.h;
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
  if (BY_GROUP(gateup, group, u, plan.u_cluster, st) != cudaSuccess) return MLPMOE_ERR_CUDA;
  return BY_GROUP(down, group, w, plan.w_cluster, st) == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
