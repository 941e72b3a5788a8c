// Tokens sorted by branch and back (mlpmoe_sort_tokens, mlpmoe_dispatch, mlpmoe_combine, mlpmoe_combine_backward):
//     rows of branch b = the tokens that select b, ascending;   x_rows[r] = x[token of r];
//     y[t] = residual[t] + sum_j w[t, j] y_rows[row_j of t];    d y_rows[row_j] = w[t, j] dy[t],  d w[t, j] = <dy[t], y_rows[row_j]>.
// Moving and summing rows is bound by memory: each kernel works from the token's side, so that what is shared by a token's rows (x, dy,
// y) crosses memory once and the rows themselves once.  8192 tokens x 4096 bf16, 8 of 32 branches: rows out 605 MB in 97 us (and 8 for the
// order), sum with an fp32 residual 806 MB in 122, gradient 1142 MB in 174: 6.2 to 6.6 TB/s.  The same rows in e4m3 with their order: 58 us with a scale
// a row, 66 with one per 32 columns (81 and 80 % of a copy, the order's 8 among them).  Rows that start anywhere go at 60 to 74 %
// of a copy in bf16 (two bytes a load), as fast as others in fp32.  No block waits for one outside of its cluster and nothing floating is added atomically.
#include <cooperative_groups.h>

#include "../../include/mlpmoe.h"
#include "internal.h"
#include "ptx.cuh"
#include "row_io.cuh"

namespace mlpmoe {
namespace {

constexpr int kMaxB = 256;
constexpr int kNone = 2;             // no residual, beside MLPMOE_BF16 (0) and MLPMOE_FP32 (1)
constexpr int kMaxAlign = 1024;

// ------------------------------------------------------------------------------------------------ the sorted order
// The selection as a matrix of bits, in squares of 32 tokens x 32 branches: a lane reads its token's row, and the square
// transposed holds, for each branch, which of the 32 tokens are in it.  First kernel: the transposed bits and their counts
// per tile of tokens.  Second: each tile adds up the tiles before it, and every set bit's place is its branch's start plus
// the bits before it.  A small batch is one tile, or one cluster's, and takes one launch.  Large batches are far above what their bytes take (masks in turn, beyond the
// L2 cache: 131072 x 32 25 us of 2.6, 131072 x 128 with 16 each 55 of 6.5): two or three launches whose blocks wait for one round trip after the other (the scan's loads
// follow its stores), tiles with fewer groups than a block has warps, and a row's token written four bytes at a time.
constexpr int kSortThreads = 512;
constexpr int kSortTiles = 592;           // tiles aimed at: four blocks per SM (131072 tokens x 32 branches: 23 us; one block per SM: 49)
constexpr int kSortScanCounts = 16384;    // every tile adds up every tile's counts; from here on a kernel of its own does so once
constexpr int kSortTileBits = 4096;       // words of 32 bits of one tile: 32 KB of shared memory with the places

struct SortArgs {
  const uint8_t* select;
  uint32_t* mask;          // [groups of 32 tokens][B32]: bit i: token i of the group is in the branch
  int32_t* tile_counts;    // [tiles][B32]; after the scan: of the tiles before
  int32_t* totals;         // [B32], the scan's
  int32_t* offsets;
  int32_t* counts;
  int32_t* row_token;
  int32_t* token_row;
  int32_t* token_branch;
  int64_t n, rows;
  int B, B32, slots, align, tile_groups, tiles, groups, wide, scanned, mode;
};

// Row lane, bit j -> row j, bit lane.
__device__ __forceinline__ uint32_t transpose32(uint32_t v, int lane) {
  uint32_t m = 0x0000FFFFu;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    const uint32_t u = __shfl_xor_sync(0xFFFFFFFFu, v, s);
    v = (lane & s) ? (v & ~m) | ((u >> s) & m) : (v & m) | ((u & m) << s);
    m ^= m << (s >> 1);
  }
  return v;
}

// One bit for each byte of x that is not zero.
__device__ __forceinline__ uint32_t nonzero4(uint32_t x) {
  const uint32_t t = (((x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | x) & 0x80808080u;
  return ((t >> 7) * 0x01020408u) >> 24 & 15u;
}

// Branches b0 .. b0 + 31 of the row at p.
__device__ __forceinline__ uint32_t row_bits(const uint8_t* p, int b0, int B, int wide) {
  uint32_t m = 0;
  if (wide == 16) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (b0 + 16 * h >= B) break;
      const uint4 v = *reinterpret_cast<const uint4*>(p + b0 + 16 * h);
      m |= (nonzero4(v.x) | nonzero4(v.y) << 4 | nonzero4(v.z) << 8 | nonzero4(v.w) << 12) << (16 * h);
    }
  } else if (wide == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (b0 + 4 * i < B) m |= nonzero4(*reinterpret_cast<const uint32_t*>(p + b0 + 4 * i)) << (4 * i);
  } else {
#pragma unroll 8
    for (int i = 0; i < 32; ++i)
      if (b0 + i < B && p[b0 + i] != 0) m |= 1u << i;
  }
  return m;
}

// The transposed bits of a group of 32 tokens, branch by branch, to out[B32]; a token's branches past its first `slots` are dropped.
template <typename F>
__device__ __forceinline__ void group_bits(const SortArgs& a, int64_t group, int lane, F&& out) {
  const int64_t t = group * 32 + lane;
  const uint8_t* p = a.select + t * a.B;
  int room = a.slots;
  for (int b0 = 0; b0 < a.B32; b0 += 32) {
    uint32_t m = t < a.n ? row_bits(p, b0, a.B, a.wide) : 0u;
    while (__popc(m) > room) m &= ~(0x80000000u >> __clz(m));
    room -= __popc(m);
    out(b0 + lane, transpose32(m, lane));
  }
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const __grid_constant__ SortArgs a) {
  __shared__ int32_t cnt[kMaxB];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  for (int b = threadIdx.x; b < a.B32; b += kSortThreads) cnt[b] = 0;
  __syncthreads();
  const int lane = threadIdx.x % 32;
  for (int i = threadIdx.x / 32; i < a.tile_groups; i += kSortThreads / 32) {
    const int64_t g = static_cast<int64_t>(blockIdx.x) * a.tile_groups + i;
    if (g >= a.groups) break;
    group_bits(a, g, lane, [&](int b, uint32_t m) {
      a.mask[g * a.B32 + b] = m;
      atomicAdd(&cnt[b], __popc(m));
    });
  }
  __syncthreads();
  for (int b = threadIdx.x; b < a.B32; b += kSortThreads) a.tile_counts[static_cast<int64_t>(blockIdx.x) * a.B32 + b] = cnt[b];
}

// Sums of the tiles before each tile, for very many tiles: a block to 32 branches, a warp to a stretch of the tiles.
__global__ void __launch_bounds__(1024) sort_scan_kernel(const __grid_constant__ SortArgs a) {
  __shared__ int32_t part[32][33];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % 32, w = threadIdx.x / 32, b = blockIdx.x * 32 + lane;
  const int per = (a.tiles + 31) / 32, lo = w * per, hi = min(a.tiles, lo + per);
  int32_t sum = 0;
  for (int i = lo; i < hi; ++i) sum += a.tile_counts[static_cast<int64_t>(i) * a.B32 + b];
  part[w][lane] = sum;
  __syncthreads();
  int32_t run = 0;
  for (int i = 0; i < w; ++i) run += part[i][lane];
  for (int i = lo; i < hi; ++i) {
    int32_t* p = a.tile_counts + static_cast<int64_t>(i) * a.B32 + b;
    const int32_t c = *p;
    *p = run;
    run += c;
  }
  if (w == 31) a.totals[b] = run;
}

// How a batch is dealt: one tile, a tile to each block of one cluster, whose blocks read one another's counts from shared memory, or any
// number of tiles, whose bits and counts another kernel has left in memory.
enum SortMode { ONE, CLUSTER, MANY };
constexpr int kSortCluster = 8;

template <SortMode MODE>
__device__ __forceinline__ void sort_place(const SortArgs& a) {
  __shared__ uint32_t mask[kSortTileBits];
  __shared__ int32_t place[kSortTileBits];     // where the group's first token of the branch goes; before that scratch of the sums
  __shared__ int32_t first[kMaxB + 1], total[kMaxB], before[kMaxB], own[MODE == CLUSTER ? kMaxB : 1], warp_sum[kMaxB / 32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, tile = blockIdx.x;
  const int64_t g0 = static_cast<int64_t>(tile) * a.tile_groups;
  const int n_groups = static_cast<int>(max(int64_t{0}, min(static_cast<int64_t>(a.tile_groups), a.groups - g0)));
  if (MODE != MANY) {
    for (int i = warp; i < n_groups; i += kSortThreads / 32) group_bits(a, g0 + i, lane, [&](int b, uint32_t m) { mask[i * a.B32 + b] = m; });
    __syncthreads();
    if (tid < a.B32) {
      int32_t sum = 0;
#pragma unroll 4
      for (int i = 0; i < n_groups; ++i) sum += __popc(mask[i * a.B32 + tid]);
      before[tid] = 0;
      (MODE == ONE ? total : own)[tid] = sum;
    }
    if (MODE == CLUSTER) {
      const auto cluster = cooperative_groups::this_cluster();
      cluster.sync();
      if (tid < a.B32) {
        int32_t sum = 0, sum_before = 0;
#pragma unroll
        for (int r = 0; r < kSortCluster; ++r) {
          const int32_t c = *cluster.map_shared_rank(&own[tid], r);
          sum += c;
          sum_before += r < tile ? c : 0;
        }
        before[tid] = sum_before;
        total[tid] = sum;
      }
    }
  } else {
    for (int i = tid; i < n_groups * a.B32; i += kSortThreads) mask[i] = a.mask[g0 * a.B32 + i];
    if (a.scanned) {
      if (tid < a.B32) {
        before[tid] = a.tile_counts[static_cast<int64_t>(tile) * a.B32 + tid];
        total[tid] = a.totals[tid];
      }
    } else {
      const int parts = kSortThreads / a.B32, b = tid % a.B32, part = tid / a.B32;
      if (part < parts) {
        int32_t sum = 0, sum_before = 0;
#pragma unroll 8
        for (int i = part; i < a.tiles; i += parts) {
          const int32_t c = a.tile_counts[static_cast<int64_t>(i) * a.B32 + b];
          sum += c;
          sum_before += i < tile ? c : 0;
        }
        place[part * a.B32 + b] = sum;
        place[(parts + part) * a.B32 + b] = sum_before;
      }
      __syncthreads();
      if (tid < a.B32) {
        int32_t sum = 0, sum_before = 0;
        for (int i = 0; i < parts; ++i) {
          sum += place[i * a.B32 + tid];
          sum_before += place[(parts + i) * a.B32 + tid];
        }
        before[tid] = sum_before;
        total[tid] = sum;
      }
    }
  }
  __syncthreads();
  // branch starts: a scan of the counts rounded up to the alignment
  const int32_t padded = tid < a.B32 ? (total[tid] + a.align - 1) / a.align * a.align : 0;
  int32_t incl = padded;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int32_t u = __shfl_up_sync(0xFFFFFFFFu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31 && warp < kMaxB / 32) warp_sum[warp] = incl;
  __syncthreads();
  if (tid < a.B32) {
    int32_t start = incl - padded;
    for (int i = 0; i < warp; ++i) start += warp_sum[i];
    first[tid] = start;
    if (tid == a.B32 - 1) first[a.B32] = start + padded;
    if (tile == 0 && tid < a.B) {
      a.offsets[tid] = start;
      a.counts[tid] = total[tid];
      if (tid == a.B - 1) a.offsets[a.B] = start + padded;
    }
  }
  __syncthreads();
  // the rows between a branch's end and the next start belong to no token
  if (a.align > 1)
    for (int b = tile * (kSortThreads / 32) + warp; b < a.B; b += gridDim.x * (kSortThreads / 32))
      for (int32_t r = first[b] + total[b] + lane; r < first[b + 1]; r += 32)
        if (r < a.rows) a.row_token[r] = -1;
  if (tid < a.B32) {
    int32_t run = first[tid] + before[tid];
    for (int i = 0; i < n_groups; ++i) {
      place[i * a.B32 + tid] = run;
      run += __popc(mask[i * a.B32 + tid]);
    }
  }
  __syncthreads();
  const uint32_t lower = (1u << lane) - 1u;
  for (int i = warp; i < n_groups; i += kSortThreads / 32) {
    const int64_t t = (g0 + i) * 32 + lane;
    int32_t* rows = a.token_row + t * a.slots;
    int32_t* branches = a.token_branch + t * a.slots;
    int slot = 0;
    for (int b0 = 0; b0 < a.B32; b0 += 32) {
      uint32_t m = transpose32(mask[i * a.B32 + b0 + lane], lane);
      while (m != 0) {
        const int b = b0 + __ffs(m) - 1;
        m &= m - 1;
        const int32_t r = place[i * a.B32 + b] + __popc(mask[i * a.B32 + b] & lower);
        if (r < a.rows) a.row_token[r] = static_cast<int32_t>(t);
        rows[slot] = r;
        if (a.token_branch != nullptr) branches[slot] = b;
        ++slot;
      }
    }
    if (t < a.n)
      for (; slot < a.slots; ++slot) {
        rows[slot] = -1;
        if (a.token_branch != nullptr) branches[slot] = -1;
      }
  }
  if (MODE == CLUSTER) cooperative_groups::this_cluster().sync();      // nobody leaves while its counts are read
}

__global__ void __launch_bounds__(kSortThreads) sort_one_kernel(const __grid_constant__ SortArgs a) { sort_place<ONE>(a); }
__global__ void __cluster_dims__(kSortCluster, 1, 1) __launch_bounds__(kSortThreads) sort_cluster_kernel(const __grid_constant__ SortArgs a) { sort_place<CLUSTER>(a); }
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const __grid_constant__ SortArgs a) { sort_place<MANY>(a); }

// Tiles of a batch.  Up to 128 tokens one block (32 branches: 2.6 us; 256 tokens 5.2), up to 1024, or 2048 from 128 branches on, one
// cluster (256 x 32 3.8 us and 1024 x 32 4.5 where two launches take 4.8 and 5.1; 2048 x 32 6.3 and 5.4), else tiles of two groups or
// more, four where there are many branches (8192 x 128: 9.9 us, two: 14.6), up to kSortTiles of them.
void sort_plan(int64_t n, int32_t B, SortArgs* a) {
  a->n = n;
  a->B = B;
  a->B32 = (B + 31) / 32 * 32;
  a->groups = static_cast<int>((n + 31) / 32);
  const int most = kSortTileBits / a->B32 < 32 ? kSortTileBits / a->B32 : 32, least = a->groups <= 4 || a->B32 >= 128 ? 4 : 2;
  int g = (a->groups + kSortTiles - 1) / kSortTiles;
  if (g < least) g = least;
  if (g > most) g = most;
  a->mode = a->groups <= g && a->groups <= 4 ? ONE : MANY;
  if (a->mode == MANY && a->groups <= (a->B32 >= 128 ? 64 : 32)) {
    a->mode = CLUSTER;
    g = (a->groups + kSortCluster - 1) / kSortCluster;
  }
  a->tile_groups = g;
  a->tiles = a->mode == ONE ? 1 : (a->mode == CLUSTER ? kSortCluster : (a->groups + g - 1) / g);
  a->scanned = static_cast<int64_t>(a->tiles) * a->B32 > kSortScanCounts;
}

int64_t round16(int64_t v) { return (v + 15) / 16 * 16; }
int64_t sort_mask_bytes(const SortArgs& a) { return a.mode != MANY ? 0 : round16(static_cast<int64_t>(a.groups) * a.B32 * 4); }
// (for as many tiles as any smaller batch has, too: a workspace serves every batch up to its own)
int64_t sort_bytes(const SortArgs& a) {
  if (a.mode != MANY) return 16;
  const int64_t aimed = a.groups < kSortTiles ? a.groups : kSortTiles, tiles = a.tiles > aimed ? a.tiles : aimed;
  return sort_mask_bytes(a) + round16((tiles + 1) * a.B32 * 4);
}

// ------------------------------------------------------------------------------------------------ rows to their branches
constexpr int kMoveThreads = 256;
// Units of a lane: a warp moves 2 KB of a row, or 16 units a lane where they are short.
__host__ __device__ constexpr int units_of(int bytes) { return bytes >= 4 ? 64 / bytes : 16; }

struct DispatchArgs {
  const uint8_t* x;
  const float* x_scale;
  const int32_t* offsets;
  const int32_t* counts;
  const int32_t* token_row;
  uint8_t* rows;
  float* row_scale;
  int64_t n, x_stride, rows_stride, units;    // strides in bytes; units of a row
  int64_t n_rows, token_blocks;
  int B, slots, scales, parts;            // parts: warps of a row; scales: scales of a row
};

// What a lane moves at a time: the widest unit that all rows start on and consist of.
template <int BYTES>
struct Unit {
  using type = uint4;
};
template <>
struct Unit<8> {
  using type = uint2;
};
template <>
struct Unit<4> {
  using type = uint32_t;
};
template <>
struct Unit<2> {
  using type = uint16_t;
};
template <>
struct Unit<1> {
  using type = uint8_t;
};

// One warp to a token's part of a row: the part is read once and written to each of the token's rows.  Behind the tokens, one
// warp to each row that aligning can have left between two branches: cleared, so that products over a branch's whole tiles see zeros.
template <int BYTES>
__global__ void __launch_bounds__(kMoveThreads) dispatch_kernel(const __grid_constant__ DispatchArgs a) {
  using E = typename Unit<BYTES>::type;
  constexpr int kVecs = units_of(BYTES);
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % 32;
  if (blockIdx.x >= a.token_blocks) {
    const int64_t u = (blockIdx.x - a.token_blocks) * (kMoveThreads / 32) + threadIdx.x / 32;
    const int64_t b = u % a.B, i = u / a.B;
    const int64_t r = static_cast<int64_t>(a.offsets[b]) + a.counts[b] + i;
    if (r >= a.offsets[b + 1] || r >= a.n_rows || r < 0) return;
    E* p = reinterpret_cast<E*>(a.rows + r * a.rows_stride);
    for (int64_t c = lane; c < a.units; c += 32) p[c] = E{};
    for (int s = lane; s < a.scales; s += 32) a.row_scale[r * a.scales + s] = 0.0f;
    return;
  }
  const int64_t u = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + threadIdx.x / 32;
  const int64_t t = u / a.parts;
  const int part = static_cast<int>(u - t * a.parts);
  if (t >= a.n) return;
  const int64_t c0 = static_cast<int64_t>(part) * (32 * kVecs) + lane;
  const E* x = reinterpret_cast<const E*>(a.x + t * a.x_stride);
  E v[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i)
    if (c0 + i * 32 < a.units) v[i] = x[c0 + i * 32];
  for (int j0 = 0; j0 < a.slots; j0 += 32) {
    const int32_t mine = j0 + lane < a.slots ? a.token_row[t * a.slots + j0 + lane] : -1;
    uint32_t live = __ballot_sync(0xFFFFFFFFu, static_cast<uint32_t>(mine) < static_cast<uint64_t>(a.n_rows));
    while (live != 0) {
      const int64_t r = __shfl_sync(0xFFFFFFFFu, mine, __ffs(live) - 1);
      live &= live - 1;
      E* p = reinterpret_cast<E*>(a.rows + r * a.rows_stride);
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
        if (c0 + i * 32 < a.units) p[c0 + i * 32] = v[i];
      if (part == 0)
        for (int s = lane; s < a.scales; s += 32) a.row_scale[r * a.scales + s] = a.x_scale[t * a.scales + s];
    }
  }
}

// ------------------------------------------------------------------------------------------------ rows summed to their tokens
struct CombineArgs {
  const void* rows;
  const int32_t* token_row;
  const float* weight;
  const void* residual;
  void* y;
  int64_t rows_stride, residual_stride, y_stride, n, n_rows;
  int slots, d, parts;
};

// One warp to 256 columns of a token: the sum stays in registers, and the loads of eight rows (four of fp32) are in flight at once.
// 8192 x 4096 bf16, 8 rows a token: 806 MB in 122 us; four rows of 256 columns 137, of 512 124; two of 512 163, of 1024 154.
template <int RK, int SK, int YK, bool VEC>
__global__ void __launch_bounds__(kMoveThreads, 4) combine_kernel(const __grid_constant__ CombineArgs a) {
  constexpr int kRows = VEC && RK == MLPMOE_BF16 ? 8 : 4;
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % 32;
  const int64_t u = static_cast<int64_t>(blockIdx.x) * (kMoveThreads / 32) + threadIdx.x / 32;
  const int64_t t = u / a.parts;
  if (t >= a.n) return;
  const int part = static_cast<int>(u - t * a.parts);
  float acc[8] = {};
  Chunk res;
  if (SK != kNone) res = load_columns<VEC, 32>(static_cast<const char*>(a.residual) + t * a.residual_stride * bytes_of(SK), SK, part, lane, a.d);
  for (int j0 = 0; j0 < a.slots; j0 += 32) {
    int32_t mine = j0 + lane < a.slots ? a.token_row[t * a.slots + j0 + lane] : -1;
    if (static_cast<uint32_t>(mine) >= static_cast<uint64_t>(a.n_rows)) mine = -1;
    const float w_mine = mine < 0 ? 0.0f : (a.weight != nullptr ? a.weight[t * a.slots + j0 + lane] : 1.0f);
    uint32_t live = __ballot_sync(0xFFFFFFFFu, mine >= 0);
    while (live != 0) {
      Chunk v[kRows];
      float w[kRows];
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int src = live != 0 ? __ffs(live) - 1 : 0;
        const int64_t r = __shfl_sync(0xFFFFFFFFu, mine, src);
        w[k] = __shfl_sync(0xFFFFFFFFu, w_mine, src);
        v[k] = load_columns<VEC, 32>(static_cast<const char*>(a.rows) + r * a.rows_stride * bytes_of(RK), RK, part, lane, live != 0 ? a.d : 0);
        if (live == 0) w[k] = 0.0f;
        live &= live - 1;
      }
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        float f[8];
        columns_f32<VEC>(v[k], RK, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fmaf(w[k], f[e], acc[e]);
      }
    }
  }
  if (SK != kNone) {
    float f[8];
    columns_f32<VEC>(res, SK, f);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += f[e];
  }
  store_columns<VEC, 32>(static_cast<char*>(a.y) + t * a.y_stride * bytes_of(YK), YK, part, lane, a.d, acc);
}

template <int RK, int SK, int YK, bool VEC>
cudaError_t launch_combine(CombineArgs a, cudaStream_t st) {
  a.parts = (a.d + 255) / 256;
  const int64_t blocks = (a.n * a.parts + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
  return launch_pdl(combine_kernel<RK, SK, YK, VEC>, dim3(static_cast<unsigned>(blocks)), dim3(kMoveThreads), 0, st, a);
}
template <int RK, int SK>
cudaError_t launch_combine_to(const CombineArgs& a, int y_kind, bool vec, cudaStream_t st) {
  if (y_kind == MLPMOE_FP32) return vec ? launch_combine<RK, SK, MLPMOE_FP32, true>(a, st) : launch_combine<RK, SK, MLPMOE_FP32, false>(a, st);
  return vec ? launch_combine<RK, SK, MLPMOE_BF16, true>(a, st) : launch_combine<RK, SK, MLPMOE_BF16, false>(a, st);
}
template <int RK>
cudaError_t launch_combine_from(const CombineArgs& a, int res_kind, int y_kind, bool vec, cudaStream_t st) {
  if (res_kind == MLPMOE_FP32) return launch_combine_to<RK, MLPMOE_FP32>(a, y_kind, vec, st);
  if (res_kind == MLPMOE_BF16) return launch_combine_to<RK, MLPMOE_BF16>(a, y_kind, vec, st);
  return launch_combine_to<RK, kNone>(a, y_kind, vec, st);
}

// ------------------------------------------------------------------------------------------------ its gradient
struct CombineGradArgs {
  const void* grad_y;
  const void* rows;
  const int32_t* token_row;
  const float* weight;
  const int32_t* offsets;
  const int32_t* counts;
  void* grad_rows;
  float* grad_weight;
  int64_t grad_y_stride, rows_stride, grad_rows_stride, n, n_rows, token_blocks;
  int slots, d, B;
};

// Above 8192 columns one row is under way at a time, for want of registers: 4096 x 12288, 4 rows a token, 66 % of a copy in bf16 and 83 % in fp32; 2048 x 20000 69
// and 74 %, 1024 x 32768 70 and 59 % (4096 x 8192: 92 and 88 %).
// T threads to a token (T = 32: a warp of a block of four): grad_y stays in registers, each of the token's rows is read for its
// product with it and receives w * grad_y.  Four rows' loads are in flight at once and their products are reduced together (8192 x 4096,
// 8 rows a token: 174 us; one row after the other 210).  A row is read before it is written, by the same thread, so both may be one buffer.
template <int GK, int RK, bool VEC, int T, int NCH>
__global__ void __launch_bounds__(T == 32 ? 128 : T, T == 32 ? 8 : (T < 1024 ? 1024 / T : 1)) combine_backward_kernel(const __grid_constant__ CombineGradArgs a) {
  constexpr int kGradRows = NCH == 4 ? 1 : (NCH == 2 && !VEC ? 2 : 4);       // rows of a token under way at a time: as many as there are registers for
  __shared__ float red[T / 32][32];
  ptx::griddep_launch_dependents();
  ptx::griddep_wait();
  const int lane = threadIdx.x % 32;
  if (blockIdx.x >= a.token_blocks) {      // the rows between a branch's end and the next start: no gradient
    constexpr int kWarps = (T == 32 ? 128 : T) / 32;
    const int64_t u = (blockIdx.x - a.token_blocks) * kWarps + threadIdx.x / 32;
    const int64_t b = u % a.B, i = u / a.B;
    const int64_t r = static_cast<int64_t>(a.offsets[b]) + a.counts[b] + i;
    if (r >= a.offsets[b + 1] || r >= a.n_rows || r < 0) return;
    char* p = static_cast<char*>(a.grad_rows) + r * a.grad_rows_stride * bytes_of(RK);
    const float zero[8] = {};
    for (int i = 0; i * 256 < a.d; ++i) store_columns<VEC, 32>(p, RK, i, lane, a.d, zero);
    return;
  }
  const int tid = T == 32 ? lane : threadIdx.x;
  const int64_t t = T == 32 ? static_cast<int64_t>(blockIdx.x) * 4 + threadIdx.x / 32 : blockIdx.x;
  if (t >= a.n) return;                    // T == 32 only: whole warps leave, no block barrier follows
  float g[NCH][8];
  {
    const char* p = static_cast<const char*>(a.grad_y) + t * a.grad_y_stride * bytes_of(GK);
    Chunk c[NCH];
#pragma unroll
    for (int i = 0; i < NCH; ++i) c[i] = load_columns<VEC, T>(p, GK, i, tid, a.d);
#pragma unroll
    for (int i = 0; i < NCH; ++i) columns_f32<VEC>(c[i], GK, g[i]);
  }
  for (int j0 = 0; j0 < a.slots; j0 += 32) {
    int32_t mine = j0 + lane < a.slots ? a.token_row[t * a.slots + j0 + lane] : -1;
    if (static_cast<uint32_t>(mine) >= static_cast<uint64_t>(a.n_rows)) mine = -1;
    const float w_mine = mine < 0 ? 0.0f : (a.weight != nullptr ? a.weight[t * a.slots + j0 + lane] : 1.0f);
    uint32_t live = __ballot_sync(0xFFFFFFFFu, mine >= 0);
    float dot_mine = 0.0f;
    while (live != 0) {
      int src[kGradRows];
      int64_t r[kGradRows];
      float w[kGradRows];
      uint32_t next = live;
#pragma unroll
      for (int k = 0; k < kGradRows; ++k) {
        src[k] = next != 0 ? __ffs(next) - 1 : -1;
        next &= next - 1;
        r[k] = __shfl_sync(0xFFFFFFFFu, mine, src[k] & 31);
        w[k] = __shfl_sync(0xFFFFFFFFu, w_mine, src[k] & 31);
      }
      live = next;
      if (a.grad_weight != nullptr) {
        Chunk c[kGradRows][NCH];
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
          const char* p = static_cast<const char*>(a.rows) + r[k] * a.rows_stride * bytes_of(RK);
#pragma unroll
          for (int i = 0; i < NCH; ++i) c[k][i] = load_columns<VEC, T>(p, RK, i, tid, src[k] >= 0 ? a.d : 0);
        }
        float dot[kGradRows];
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
          dot[k] = 0.0f;
#pragma unroll
          for (int i = 0; i < NCH; ++i) {
            float f[8];
            columns_f32<VEC>(c[k][i], RK, f);
#pragma unroll
            for (int e = 0; e < 8; ++e) dot[k] = fmaf(g[i][e], f[e], dot[k]);
          }
        }
        const float sum = warp_sums<kGradRows>(dot);
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
          const float of_k = __shfl_sync(0xFFFFFFFFu, sum, k * lanes_of(kGradRows));
          if (lane == src[k]) dot_mine = of_k;
        }
      }
      if (a.grad_rows != nullptr) {
#pragma unroll
        for (int k = 0; k < kGradRows; ++k) {
          if (src[k] < 0) continue;
          char* p = static_cast<char*>(a.grad_rows) + r[k] * a.grad_rows_stride * bytes_of(RK);
#pragma unroll
          for (int i = 0; i < NCH; ++i) {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = w[k] * g[i][e];
            store_columns<VEC, T>(p, RK, i, tid, a.d, f);
          }
        }
      }
    }
    if (a.grad_weight == nullptr) continue;
    if (T > 32) {
      red[threadIdx.x / 32][lane] = dot_mine;
      __syncthreads();
      if (threadIdx.x < 32) {
        dot_mine = red[0][lane];
#pragma unroll
        for (int i = 1; i < T / 32; ++i) dot_mine += red[i][lane];
      }
      __syncthreads();
    }
    if ((T == 32 || threadIdx.x < 32) && j0 + lane < a.slots) a.grad_weight[t * a.slots + j0 + lane] = dot_mine;
  }
}

template <int GK, int RK, bool VEC, int T, int NCH>
cudaError_t launch_grad(CombineGradArgs a, int64_t pad_rows, cudaStream_t st) {
  constexpr int kThreads = T == 32 ? 128 : T;
  a.token_blocks = T == 32 ? (a.n + 3) / 4 : a.n;
  const int64_t blocks = a.token_blocks + (pad_rows + kThreads / 32 - 1) / (kThreads / 32);
  return launch_pdl(combine_backward_kernel<GK, RK, VEC, T, NCH>, dim3(static_cast<unsigned>(blocks)), dim3(kThreads), 0, st, a);
}
template <int GK, int RK, bool VEC>
cudaError_t launch_grad_shape(const CombineGradArgs& a, int64_t pad_rows, cudaStream_t st) {
  if (a.d <= 256) return launch_grad<GK, RK, VEC, 32, 1>(a, pad_rows, st);
  if (a.d <= 1024) return launch_grad<GK, RK, VEC, 128, 1>(a, pad_rows, st);
  if (a.d <= 4096) return launch_grad<GK, RK, VEC, 256, 2>(a, pad_rows, st);
  if (a.d <= 8192) return launch_grad<GK, RK, VEC, 512, 2>(a, pad_rows, st);
  return launch_grad<GK, RK, VEC, 1024, 4>(a, pad_rows, st);
}
template <int GK>
cudaError_t launch_grad_from(const CombineGradArgs& a, int rows_kind, bool vec, int64_t pad_rows, cudaStream_t st) {
  if (rows_kind == MLPMOE_FP32)
    return vec ? launch_grad_shape<GK, MLPMOE_FP32, true>(a, pad_rows, st) : launch_grad_shape<GK, MLPMOE_FP32, false>(a, pad_rows, st);
  return vec ? launch_grad_shape<GK, MLPMOE_BF16, true>(a, pad_rows, st) : launch_grad_shape<GK, MLPMOE_BF16, false>(a, pad_rows, st);
}

inline bool plain_kind(mlpmoe_dtype_t t) { return t == MLPMOE_FP32 || t == MLPMOE_BF16; }

// Rows that aligning can have left between branches, at most.
inline int64_t pad_rows_of(int32_t B, int32_t align) { return static_cast<int64_t>(B) * (align - 1); }

}  // namespace
}  // namespace mlpmoe

using namespace mlpmoe;

extern "C" {

mlpmoe_status_t mlpmoe_sort_rows(int64_t n_tokens, int32_t B, int32_t slots, int32_t align, int64_t* rows) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || B <= 0 || slots <= 0 || align <= 0 || !rows) return MLPMOE_ERR_INVALID_ARG;
  if (B > kMaxB || align > kMaxAlign) return MLPMOE_ERR_UNSUPPORTED;
  const int64_t pairs = n_tokens * (slots < B ? slots : B);
  const int64_t most = pairs + (pairs < B ? pairs : B) * (align - 1);
  if (most > INT32_MAX) return MLPMOE_ERR_UNSUPPORTED;
  *rows = most;
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_sort_workspace(int64_t n_tokens, int32_t B, int64_t* bytes) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || B <= 0 || !bytes) return MLPMOE_ERR_INVALID_ARG;
  if (B > kMaxB) return MLPMOE_ERR_UNSUPPORTED;
  SortArgs a = {};
  sort_plan(n_tokens, B, &a);
  *bytes = sort_bytes(a);
  return MLPMOE_OK;
}

mlpmoe_status_t mlpmoe_sort_tokens(const uint8_t* select, int64_t n_tokens, int32_t B, int32_t slots, int32_t align, int32_t* offsets,
                                   int32_t* counts, int32_t* row_token, int64_t rows, int32_t* token_row, int32_t* token_branch,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
  int64_t most = 0;
  const mlpmoe_status_t rc = mlpmoe_sort_rows(n_tokens, B, slots, align, &most);
  if (rc != MLPMOE_OK) return rc;
  if (rows < most || rows > INT32_MAX || !offsets || !counts || !on(offsets, 4) || !on(counts, 4)) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens > 0 && (!select || !row_token || !token_row)) return MLPMOE_ERR_INVALID_ARG;
  if (!on(row_token, 4) || !on(token_row, 4) || !on(token_branch, 4)) return MLPMOE_ERR_INVALID_ARG;
  SortArgs a = {};
  sort_plan(n_tokens, B, &a);
  if (!workspace || workspace_bytes < sort_bytes(a) || !on(workspace, 16)) return MLPMOE_ERR_INVALID_ARG;
  a.select = select;
  a.mask = static_cast<uint32_t*>(workspace);
  a.tile_counts = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(workspace) + sort_mask_bytes(a));
  a.totals = a.tile_counts + static_cast<int64_t>(a.tiles) * a.B32;
  a.offsets = offsets;
  a.counts = counts;
  a.row_token = row_token;
  a.token_row = token_row;
  a.token_branch = token_branch;
  a.rows = rows;
  a.slots = slots;
  a.align = align;
  a.wide = B % 16 == 0 && on(select, 16) ? 16 : (B % 4 == 0 && on(select, 4) ? 4 : 1);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  pdl_overlap_enabled() = true;
  cudaError_t e;
  if (a.mode == ONE) {
    e = launch_pdl(sort_one_kernel, dim3(1), dim3(kSortThreads), 0, st, a);
  } else if (a.mode == CLUSTER) {
    e = launch_pdl(sort_cluster_kernel, dim3(kSortCluster), dim3(kSortThreads), 0, st, a);
  } else {
    e = launch_pdl(sort_count_kernel, dim3(static_cast<unsigned>(a.tiles)), dim3(kSortThreads), 0, st, a);
    if (e == cudaSuccess && a.scanned) e = launch_pdl(sort_scan_kernel, dim3(static_cast<unsigned>(a.B32 / 32)), dim3(1024), 0, st, a);
    if (e == cudaSuccess) e = launch_pdl(sort_place_kernel, dim3(static_cast<unsigned>(a.tiles)), dim3(kSortThreads), 0, st, a);
  }
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

mlpmoe_status_t mlpmoe_dispatch(const void* x, mlpmoe_dtype_t dtype, int64_t x_stride, const float* x_scale, int64_t group,
                                int64_t n_tokens, int64_t d_model, int32_t B, int32_t slots, int32_t align, const int32_t* offsets,
                                const int32_t* counts, const int32_t* token_row, void* rows, int64_t rows_stride, float* row_scale,
                                int64_t n_rows, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0 || d_model > INT32_MAX / 8 || slots <= 0 || align <= 0 || B <= 0 || n_rows < 0 ||
      n_rows > INT32_MAX)
    return MLPMOE_ERR_INVALID_ARG;
  if (B > kMaxB || align > kMaxAlign) return MLPMOE_ERR_UNSUPPORTED;
  if (dtype != MLPMOE_FP32 && dtype != MLPMOE_BF16 && dtype != MLPMOE_E4M3) return MLPMOE_ERR_INVALID_ARG;
  if (dtype == MLPMOE_E4M3 && group != 0 && group != 32 && group != 64 && group != 128) return MLPMOE_ERR_INVALID_ARG;
  if (x_stride == 0) x_stride = d_model;
  if (rows_stride == 0) rows_stride = d_model;
  if (x_stride < d_model || rows_stride < d_model) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens == 0) return MLPMOE_OK;
  const int es = bytes_of(dtype);
  if (!x || !token_row || !rows || !on(x, es) || !on(rows, es) || !on(token_row, 4)) return MLPMOE_ERR_INVALID_ARG;
  if (dtype == MLPMOE_E4M3 && (!x_scale || !row_scale || !on(x_scale, 4) || !on(row_scale, 4))) return MLPMOE_ERR_INVALID_ARG;
  if (align > 1 && (!offsets || !counts || !on(offsets, 4) || !on(counts, 4))) return MLPMOE_ERR_INVALID_ARG;
  DispatchArgs a = {};
  a.x = static_cast<const uint8_t*>(x);
  a.x_scale = x_scale;
  a.offsets = offsets;
  a.counts = counts;
  a.token_row = token_row;
  a.rows = static_cast<uint8_t*>(rows);
  a.row_scale = row_scale;
  a.n = n_tokens;
  a.x_stride = x_stride * es;
  a.rows_stride = rows_stride * es;
  const uintptr_t all = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(rows) | static_cast<uintptr_t>(a.x_stride | a.rows_stride | d_model * es);
  const int unit = static_cast<int>((all | 16) & -(all | 16));
  a.units = d_model * es / unit;
  a.n_rows = n_rows;
  a.B = B;
  a.slots = slots;
  a.scales = dtype == MLPMOE_E4M3 ? static_cast<int>(group == 0 ? 1 : (d_model + group - 1) / group) : 0;
  const int64_t part = 32 * units_of(unit);
  a.parts = static_cast<int>((a.units + part - 1) / part);
  a.token_blocks = (n_tokens * a.parts + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
  const int64_t blocks = a.token_blocks + (pad_rows_of(B, align) + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
  if (blocks > INT32_MAX) return MLPMOE_ERR_UNSUPPORTED;
  const dim3 grid(static_cast<unsigned>(blocks)), block(kMoveThreads);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  pdl_overlap_enabled() = true;
  cudaError_t e;
  switch (unit) {
    case 16: e = launch_pdl(dispatch_kernel<16>, grid, block, 0, st, a); break;
    case 8: e = launch_pdl(dispatch_kernel<8>, grid, block, 0, st, a); break;
    case 4: e = launch_pdl(dispatch_kernel<4>, grid, block, 0, st, a); break;
    case 2: e = launch_pdl(dispatch_kernel<2>, grid, block, 0, st, a); break;
    default: e = launch_pdl(dispatch_kernel<1>, grid, block, 0, st, a); break;
  }
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

mlpmoe_status_t mlpmoe_combine(const void* rows, mlpmoe_dtype_t rows_dtype, int64_t rows_stride, int64_t n_rows, const int32_t* token_row,
                               const float* weight, int32_t slots, const void* residual, mlpmoe_dtype_t residual_dtype,
                               int64_t residual_stride, void* y, mlpmoe_dtype_t y_dtype, int64_t y_stride, int64_t n_tokens,
                               int64_t d_model, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0 || d_model > INT32_MAX / 8 || slots <= 0 || n_rows < 0 || n_rows > INT32_MAX)
    return MLPMOE_ERR_INVALID_ARG;
  if (!plain_kind(rows_dtype) || !plain_kind(y_dtype) || (residual && !plain_kind(residual_dtype))) return MLPMOE_ERR_INVALID_ARG;
  if (rows_stride == 0) rows_stride = d_model;
  if (residual_stride == 0) residual_stride = d_model;
  if (y_stride == 0) y_stride = d_model;
  if (rows_stride < d_model || (residual && residual_stride < d_model) || y_stride < d_model) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens == 0) return MLPMOE_OK;
  if ((n_rows > 0 && !rows) || !token_row || !y || !on(rows, bytes_of(rows_dtype)) || !on(y, bytes_of(y_dtype)) || !on(token_row, 4) ||
      !on(weight, 4) || (residual && !on(residual, bytes_of(residual_dtype))))
    return MLPMOE_ERR_INVALID_ARG;
  if (residual == y && (residual_dtype != y_dtype || (residual_stride != y_stride && n_tokens > 1))) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens * ((d_model + 255) / 256) / (kMoveThreads / 32) >= INT32_MAX) return MLPMOE_ERR_UNSUPPORTED;      // blocks of a launch
  const bool vec = d_model % 8 == 0 && rows_stride % 8 == 0 && on(rows, 16) && y_stride % 8 == 0 && on(y, 16) &&
                   (!residual || (residual_stride % 8 == 0 && on(residual, 16)));
  CombineArgs a = {};
  a.rows = rows;
  a.token_row = token_row;
  a.weight = weight;
  a.residual = residual;
  a.y = y;
  a.rows_stride = rows_stride;
  a.residual_stride = residual ? residual_stride : 0;
  a.y_stride = y_stride;
  a.n = n_tokens;
  a.n_rows = n_rows;
  a.slots = slots;
  a.d = static_cast<int>(d_model);
  pdl_overlap_enabled() = true;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int res_kind = residual ? static_cast<int>(residual_dtype) : kNone;
  const cudaError_t e = rows_dtype == MLPMOE_FP32 ? launch_combine_from<MLPMOE_FP32>(a, res_kind, y_dtype, vec, st)
                                                  : launch_combine_from<MLPMOE_BF16>(a, res_kind, y_dtype, vec, st);
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

mlpmoe_status_t mlpmoe_combine_backward(const void* grad_y, mlpmoe_dtype_t grad_y_dtype, int64_t grad_y_stride, const void* rows,
                                        mlpmoe_dtype_t rows_dtype, int64_t rows_stride, int64_t n_rows, const int32_t* token_row,
                                        const float* weight, int32_t slots, int32_t B, int32_t align, const int32_t* offsets,
                                        const int32_t* counts, void* grad_rows, int64_t grad_rows_stride, float* grad_weight,
                                        int64_t n_tokens, int64_t d_model, void* stream) {
  if (n_tokens < 0 || n_tokens > INT32_MAX || d_model <= 0 || slots <= 0 || B <= 0 || align <= 0 || n_rows < 0 || n_rows > INT32_MAX)
    return MLPMOE_ERR_INVALID_ARG;
  if (!plain_kind(grad_y_dtype) || !plain_kind(rows_dtype)) return MLPMOE_ERR_INVALID_ARG;
  if (d_model > 32768 || B > kMaxB || align > kMaxAlign || n_tokens > INT32_MAX - kMaxB * kMaxAlign) return MLPMOE_ERR_UNSUPPORTED;
  if (grad_y_stride == 0) grad_y_stride = d_model;
  if (rows_stride == 0) rows_stride = d_model;
  if (grad_rows_stride == 0) grad_rows_stride = d_model;
  if (grad_y_stride < d_model || rows_stride < d_model || grad_rows_stride < d_model) return MLPMOE_ERR_INVALID_ARG;
  if (n_tokens == 0) return MLPMOE_OK;
  if (!grad_y || !token_row || (!grad_rows && !grad_weight) || (grad_weight && n_rows > 0 && !rows)) return MLPMOE_ERR_INVALID_ARG;
  if (!on(grad_y, bytes_of(grad_y_dtype)) || !on(rows, bytes_of(rows_dtype)) || !on(grad_rows, bytes_of(rows_dtype)) || !on(token_row, 4) ||
      !on(weight, 4) || !on(grad_weight, 4))
    return MLPMOE_ERR_INVALID_ARG;
  if (grad_rows && align > 1 && (!offsets || !counts || !on(offsets, 4) || !on(counts, 4))) return MLPMOE_ERR_INVALID_ARG;
  if (grad_rows && grad_rows == rows && grad_rows_stride != rows_stride) return MLPMOE_ERR_INVALID_ARG;
  const bool vec = d_model % 8 == 0 && grad_y_stride % 8 == 0 && on(grad_y, 16) && (!grad_weight || (rows_stride % 8 == 0 && on(rows, 16))) &&
                   (!grad_rows || (grad_rows_stride % 8 == 0 && on(grad_rows, 16)));
  CombineGradArgs a = {};
  a.grad_y = grad_y;
  a.rows = rows;
  a.token_row = token_row;
  a.weight = weight;
  a.offsets = offsets;
  a.counts = counts;
  a.grad_rows = grad_rows;
  a.grad_weight = grad_weight;
  a.grad_y_stride = grad_y_stride;
  a.rows_stride = rows_stride;
  a.grad_rows_stride = grad_rows_stride;
  a.n = n_tokens;
  a.n_rows = n_rows;
  a.slots = slots;
  a.d = static_cast<int>(d_model);
  a.B = B;
  const int64_t pad_rows = grad_rows ? pad_rows_of(B, align) : 0;
  pdl_overlap_enabled() = true;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const cudaError_t e = grad_y_dtype == MLPMOE_FP32 ? launch_grad_from<MLPMOE_FP32>(a, rows_dtype, vec, pad_rows, st)
                                                    : launch_grad_from<MLPMOE_BF16>(a, rows_dtype, vec, pad_rows, st);
  return e == cudaSuccess ? MLPMOE_OK : MLPMOE_ERR_CUDA;
}

}  // extern "C"
