// Stored form of 4-bit weights and the launch interface of the layer's kernels on them.
#pragma once
#include "internal.h"

namespace mlpmoe {

constexpr int64_t kW4MaxDim = int64_t(1) << 20;   // rows and columns: keeps every index inside a row, a block list or a grid in 32 bits
constexpr int64_t kW4MaxTokens = 65536;
constexpr int kW4MaxBranches = 256;
constexpr int kW4Warps = 8;                       // warps of a block

inline int64_t w4_pitch(int64_t cols) { return (cols + 31) / 32 * 16; }     // bytes of a row of codes
inline int64_t w4_rows16(int64_t rows) { return (rows + 15) / 16 * 16; }    // elements of a row of scales

// The columns of a product: every token is `pieces` columns (bf16 pieces whose sum is the activation); the tokens are
// cut into `chunks` of `tokens` each, column c of a chunk is piece c / tokens of token c % tokens, and a chunk's columns
// are padded to `nt` tiles of eight.
struct W4Cols {
  int pieces, tokens, chunks, nt;
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
  int kblocks;              // ceil(K / 128)
  int wr, wk;               // warps of a block along the rows and along K; wr * wk = kW4Warps
  int n;                    // tokens
  W4Cols c;
  const uint4* frag;        // activations in fragment order: [chunk][kblock][nt][4][32] units of 8 bf16
  const int32_t* list;      // K-blocks to read (null: all); list[kblocks] = how many
  // gate|up
  const float* x_scale;     // [n x x_groups] (null: 1)
  int x_groups, x_shift;    // group of a column of scale groups g: g >> x_shift; x_groups = 1: applied to the sums
  const uint8_t* select;    // [n x B] or null
  const uint8_t* active;    // [B]: a branch that some token computes
  int B;
  W4Cols hc;                // columns of the down product
  int h_kblocks;
  __nv_bfloat16* h_frag;
  int dense;                // every branch computed by every token: nothing of the selection is read
  // down
  const float* coef;        // [n] (null: 1)
  const float* residual;
  void* y;
  int y_bf16;
  int64_t d;
  int32_t off[kW4MaxBranches + 1];   // gate|up: first neuron of each branch
  float alpha[kW4MaxBranches];
};

// One launch per group width (w4_g32.cu, w4_g64.cu, w4_g128.cu); `clusters` = blocks of a cluster along K (down only).
cudaError_t launch_w4_gateup_32(const W4Args& a, cudaStream_t st);
cudaError_t launch_w4_gateup_64(const W4Args& a, cudaStream_t st);
cudaError_t launch_w4_gateup_128(const W4Args& a, cudaStream_t st);
cudaError_t launch_w4_down_32(const W4Args& a, int cluster, cudaStream_t st);
cudaError_t launch_w4_down_64(const W4Args& a, int cluster, cudaStream_t st);
cudaError_t launch_w4_down_128(const W4Args& a, int cluster, cudaStream_t st);

}  // namespace mlpmoe
