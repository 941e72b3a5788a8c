// Stored form of 4-bit weights and the launch interface of the layer's kernels on them.
#pragma once
#include "internal.h"

namespace mlpmoe {

constexpr int64_t kW4MaxDim = int64_t(1) << 16;   // rows and columns of a matrix
constexpr int64_t kW4MaxTokens = 65536;
constexpr int kW4MaxBranches = 256;

__host__ __device__ inline int64_t w4_pitch(int64_t cols) { return (cols + 31) / 32 * 16; }     // bytes of a row of codes
__host__ __device__ inline int64_t w4_rows16(int64_t rows) { return (rows + 15) / 16 * 16; }    // elements of a row of scales

// The columns of a product: a token is `pieces` columns (digits of its activations); the tokens are cut into `chunks` of
// `tokens` each, and column c of a chunk is digit c / tokens of its token c % tokens.
struct W4Cols {
  int pieces, tokens, chunks;
  __host__ __device__ int cols() const { return pieces * tokens; }
};

struct W4Mat {
  const uint8_t* q;
  const __nv_bfloat16* scale;
  const uint8_t* zero;      // null: 8
  int64_t pitch;            // bytes
  int64_t rows16;
  int64_t n_groups;
};

struct W4Args {
  W4Mat m[2];               // matrices of the two 8-row halves of a tile: gate and up, or W_down twice
  int rows;                 // rows of each
  int tiles;                // 16-row tiles: eight neurons (gate, up), or sixteen rows of W_down
  int tiles_per_block;
  uint32_t* status;         // cleared where given
  int K, kblocks;           // columns, and ceil(K / 128)
  int entries;              // K-blocks of a block of the cluster at most, rounded up to an even number
  int n;                    // tokens
  W4Cols c;
  // the branches: neurons of branch b are off[b] .. off[b + 1]
  int B, dense;             // dense: every branch is computed for every token, nothing of the selection is read
  const uint8_t* select;    // [n x B] or null
  // activations: the layer's input (gate|up), or the intermediate activations (down)
  const void* x;
  int x_kind;
  int64_t x_stride;
  const float* x_scale;     // [n x x_groups] or null
  int x_groups, x_shift;    // group of x_scale of weight group g: g >> x_shift (x_groups = 1: 0)
  float* h;                 // gate|up: intermediate activations [n x rows]
  // down
  int compensate;
  const float* residual;
  void* y;
  int y_bf16;
  int32_t off[kW4MaxBranches + 1];
  float alpha[kW4MaxBranches];
};

// The same products for more tokens (w4_wide.cuh).
struct W4WideArgs {
  W4Mat m[2];
  int rows, tiles;              // as W4Args; a warp takes two tiles
  int row_groups, col_groups;   // warps of a block: 32 rows each along the rows, slot_tiles / col_groups tiles (1, 2, 3, 4, 6 or 8) along the columns
  int kblocks, entries;         // K-blocks in all, and of a block of the cluster at most
  int n, tokens, slots_per_token, slot_tiles;   // a chunk: tokens * slots_per_token slots, four to a tile of eight columns
  const uint8_t* digits;        // [chunk][kblock][slot_tile][2][32 lanes][16 bytes]
  const float2* units;          // [chunk][kblock][GPB][4 slot_tiles]: (unit, - sum of x in units)
  int B, dense;
  const uint8_t* select;
  float* h;                     // gate|up
  int compensate;               // down
  const float* residual;
  void* y;
  int y_bf16;
  int32_t off[kW4MaxBranches + 1];
  float alpha[kW4MaxBranches];
};

constexpr int kW4WideStages = 4;
constexpr int kW4WideSlots = 64;      // of a chunk, at most
// A stage: codes, scales and zeros of 32 row_groups rows, digits and units of the slots.
__host__ __device__ inline int w4_wide_stage_bytes(int row_groups, int slot_tiles, int gpb) {
  return 32 * row_groups * (64 + 3 * gpb) + slot_tiles * (1024 + gpb * 32);
}

// Activations [n x K] to digits in the order w4_wide_kernel reads them.
struct W4DigitsArgs {
  const void* x;
  int kind;
  int64_t stride;
  const float* x_scale;
  int x_groups, x_shift;
  int K, kblocks, n, tokens, slots_per_token, slot_tiles;
  uint8_t* digits;
  float2* units;
  uint32_t* status;             // cleared where given
};

// The same products on the 5th-generation tensor cores (w4_tc.cuh).
struct W4TcArgs {
  alignas(64) CUtensorMap codes[2];             // boxes of 128 rows x 64 bytes, 64-byte swizzle
  W4Mat m[2];
  int rows, kblocks;
  int n, tokens, ne;            // a chunk's tokens; columns of an epilogue warp, 32 or 64
  const uint8_t* image;         // activations as w4_columns_kernel lays them out
  const float* unit;            // gate|up: [token]; down: [chunk][K-block][column]
  int B, dense;
  const uint8_t* select;
  uint8_t* h;                   // gate|up: the intermediate activations as the down product's image and units, h_tokens a chunk
  float* h_unit;
  int h_tokens, h_cols;
  int compensate;               // down
  const float* residual;
  __nv_bfloat16* y;
  uint32_t* status;
  uint64_t wait_limit_ns;
  uint32_t extra_arrivals;
  int32_t off[kW4MaxBranches + 1];
  float alpha[kW4MaxBranches];
};
struct W4ColumnsArgs {
  const void* x;
  int kind;
  int64_t stride;
  const float* x_scale;
  int x_groups, x_group;
  int K, kblocks, n, tokens, cols;
  uint8_t* image;
  float* unit;
  uint32_t* status;             // cleared where given
};
cudaError_t launch_w4_columns(const W4ColumnsArgs& a, cudaStream_t st);

// One launch per group width (w4_g32.cu, w4_g64.cu, w4_g128.cu); `cluster` = blocks that share K.
#define MLPMOE_W4_LAUNCHES(G)                                                                     \
  cudaError_t launch_w4_gateup_##G(const W4Args& a, int cluster, cudaStream_t st);                \
  cudaError_t launch_w4_down_##G(const W4Args& a, int cluster, cudaStream_t st);                  \
  cudaError_t launch_w4_wide_gateup_##G(const W4WideArgs& a, int chunks, cudaStream_t st);        \
  cudaError_t launch_w4_wide_down_##G(const W4WideArgs& a, int cluster, int chunks, cudaStream_t st); \
  cudaError_t launch_w4_digits_##G(const W4DigitsArgs& a, cudaStream_t st);                       \
  cudaError_t launch_w4_tc_gateup_##G(const W4TcArgs& a, int cluster, cudaStream_t st);           \
  cudaError_t launch_w4_tc_down_##G(const W4TcArgs& a, int cluster, cudaStream_t st);
MLPMOE_W4_LAUNCHES(32)
MLPMOE_W4_LAUNCHES(64)
MLPMOE_W4_LAUNCHES(128)
#undef MLPMOE_W4_LAUNCHES

// Split of one product: fills a->tiles_per_block, entries and c, returns the cluster.  Host only.
int w4_plan(W4Args* a, int pieces, int group);

}  // namespace mlpmoe
