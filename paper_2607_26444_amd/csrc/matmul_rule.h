// Which kernel and which size of tile computes a call of moe_expert_matmul: host
// arithmetic on its sizes alone.  matmul.hip launches what it says.
#pragma once

#include "layer.h"

namespace moe {

constexpr int kTile = 256;
constexpr int kTileThreads = 512;

// Tiles of one launch of a streaming way, one workgroup to each: HIP's limit of 2^32
// threads, whole rounds of 256.  More rows than that have narrow outputs and are left
// to the tile kernels, whose workgroups stay and number their tiles in 32 bits (600
// million rows, 16 x 8).
constexpr int64_t kMaxGroups = (1ll << 32) / kTileThreads - 256;
constexpr int64_t kMaxTiles = INT32_MAX - 512;

// Row tiles of `size` that the windows can have: each window with rows adds at
// most one that is not full.
inline int64_t row_tiles(const MatmulArgs& a, int size) {
  if (!a.offset) return (a.rows + size - 1) / size;
  return a.rows / size + (a.rows < a.E ? a.rows : a.E);
}

// Row tiles of `size` if the rows are spread about evenly.
inline double even_tiles(const MatmulArgs& a, int size) {
  const double windows = (double)(a.rows < a.E ? a.rows : a.E), n = (double)a.rows / windows / size;
  return windows * (a.E == 1 ? __builtin_ceil(n) : n > 0.8 ? n + 0.5 : 1.0);
}

// One way to compute a call, and what its workgroups took on MI355X: `start`
// microseconds beside the stages, a stage `alone` on a compute unit or `shared`
// with a second workgroup, and the rate of the weights from memory.
struct Way {
  int rows, channels, depth;                           // of a workgroup; depth of a stage
  int resident;                                        // workgroups on the GPU at once
  double start, alone, shared;                         // us
  double rate;                                         // bytes / us
};
enum WayName { kTile256, kTile128, kWide, kHalf, kHalfTwo, kNarrow, kFewRows, kOneRow, kWays };
constexpr Way kWay[kWays] = {
    {256, 256, 128, 256, 9.0, 1.60, 1.60, 4.85e6},     // matmul_tile_kernel<256>
    {128, 256, 128, 256, 6.0, 1.05, 1.05, 4.85e6},     // matmul_tile_kernel<128>
    {64, 128, 128, 512, 3.0, 0.72, 1.15, 5.9e6},       // matmul_stream_kernel<64, 8, 1, 3>
    {64, 64, 256, 256, 3.0, 0.65, 0.65, 4.5e6},        // <64, 4, 2, 3>
    {64, 64, 256, 512, 3.0, 0.95, 1.00, 4.5e6},        // <64, 4, 2, 2>
    {64, 32, 512, 256, 3.0, 0.68, 0.68, 4.5e6},        // <64, 2, 4, 3>
    {16, 32, 512, 512, 3.0, 0.65, 0.80, 4.5e6},        // <16, 2, 4, 3>
    {16, 16, 1024, 512, 3.0, 0.80, 1.00, 4.5e6},       // <16, 1, 8, 2>
};

// Output channels of the call, those of a way's tile, and its tiles of all windows.
inline int out_channels(const MatmulArgs& a) { return a.swiglu ? a.N / 2 : a.N; }
inline int tile_channels(const MatmulArgs& a, const Way& w) {
  return a.swiglu ? w.channels / 2 : w.channels;
}
inline int pieces_of(const MatmulArgs& a, const Way& w) {
  const int per = tile_channels(a, w);
  return (out_channels(a) + per - 1) / per;
}
inline int64_t tiles_of(const MatmulArgs& a, const Way& w) {
  return row_tiles(a, w.rows) * pieces_of(a, w);
}

// Whether a way can be launched for the call.
inline bool way_fits(const MatmulArgs& a, int n) {
  return tiles_of(a, kWay[n]) <= (n == kTile256 || n == kTile128 ? kMaxTiles : kMaxGroups);
}

// Microseconds of a call: its rounds of workgroups, the last one counted for the
// larger part also where it is not full, and the reading of the weights, which partly
// hides behind them.  Measured where two ways are near each other, us:
//   rows, experts, K x N                   256   128    64 x 128  64 x 64 (three, two stages)
//   13483, 3, 5952 x 4752, swiglu          357   402    858       946   881
//   2048, 1, 4096 x 4096                    58    37     76        94    66
//   4096, 32, 7168 x 4096, swiglu          275   212    316       389   359
//   4662, 96, 2064 x 1416                  105    88     84       100    95
//   512, 1, 4096 x 4096                     46    35     24        26    19
//   256, 1, 4096 x 4096                     42    29     23        15    17
// and of few rows             64 x 128  64 x 64  64 x 32  16 x 32  16 x 16
//   64, 1, 7168 x 4096               28       17       13       16       18
//   64, 8, 2048 x 1024               11      8.6      7.3      5.6      6.2
//   1, 1, 7168 x 4096                26       16        -       12        9
inline double way_time(const MatmulArgs& a, const Way& w) {
  const double groups = even_tiles(a, w.rows) * pieces_of(a, w);
  const double full = groups / w.resident;
  const double rounds = full < 1.0 ? 1.0 : full + 0.75 * (__builtin_ceil(full) - full);
  const int stages = (a.K + w.depth - 1) / w.depth;
  const double work = rounds * (w.start + stages * (groups <= 256.0 ? w.alone : w.shared));
  const double read = (double)(a.rows < a.E ? a.rows : a.E) * a.N * a.K / w.rate;
  return __builtin_sqrt(work * work + read * read);
}

// The way that takes least of those that can be launched; kWays if none can be.
inline int choose_way(const MatmulArgs& a) {
  int best = kWays;
  double least = 0.0;
  for (int n = 0; n < kWays; ++n) {
    if (!way_fits(a, n)) continue;
    const double t = way_time(a, kWay[n]);
    if (best == kWays || t < least) {
      least = t;
      best = n;
    }
  }
  return best;
}

}  // namespace moe
