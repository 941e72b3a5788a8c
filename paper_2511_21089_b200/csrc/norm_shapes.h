// How the norms' gradient deals rows to threads and blocks: host arithmetic alone, so that it can be compiled and checked without CUDA.
#pragma once
#include <cstdint>

namespace mlpmoe {

constexpr int kSms = 148;
constexpr int64_t kOnePassD = 8192;      // longer rows do not leave room for their columns' sums in registers
constexpr int kSplitRows = 64;           // slices of the rows there, for the sums over tokens

// Threads of a row (eight columns each), quads of a thread and blocks per SM, by the row's length: threads without columns cost as much as
// the others (12264 x 4104: 139 us with 640 threads, 180 with 1024).  Blocks: one for each row (up to 256 columns each eight rows) up to 148 of them, then 148
// until each has four, then one for each four, up to what the SMs hold at once, so that few sums are left to join.
struct Shape {
  int threads, quads, ctas;
};
constexpr Shape kShapes[] = {{32, 2, 3}, {64, 2, 16}, {96, 2, 10}, {128, 2, 8}, {192, 2, 5}, {256, 2, 4}, {320, 2, 3}, {512, 2, 2}, {640, 2, 1}, {1024, 2, 1}};
constexpr int kLastShape = static_cast<int>(sizeof(kShapes) / sizeof(kShapes[0])) - 1;
static_assert(kShapes[kLastShape].threads * 8 == kOnePassD, "the last shape takes the longest row of one pass");

// The first shape whose threads have the row's columns, eight each; rows above kOnePassD, which none has, give the last.
constexpr int shape_of(int64_t d) {
  int s = 0;
  while (s < kLastShape && kShapes[s].threads * 8 < d) ++s;
  return s;
}

// Blocks whose sums over tokens are joined: those of the one pass, above kOnePassD the slices of the rows.
constexpr int blocks_of(int64_t n, int64_t d) {
  if (d > kOnePassD) return static_cast<int>(n < kSplitRows ? n : kSplitRows);
  const int64_t need = d <= 256 ? (n + 7) / 8 : n, most = static_cast<int64_t>(kSms) * kShapes[shape_of(d)].ctas;
  const int64_t few = (need + 3) / 4 > kSms ? (need + 3) / 4 : kSms;
  const int64_t blocks = need < few ? need : few;
  return static_cast<int>(blocks < most ? blocks : most);
}

}  // namespace mlpmoe
