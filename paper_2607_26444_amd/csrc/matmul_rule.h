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
// hides behind them.  The model is there to order the ways; its times are mostly long, by
// up to a half where rounds and reading hide more of each other.  Measured / model, us,
// rows drawn to the experts evenly:
//   rows, experts, K x N               256      128      64 x 128  64 x 64 three, two stages
//   512, 32, 7168 x 4096, swiglu     183/276  158/233  157/209  168/269  163/243
//   2048, 32, the same               187/276  165/233  203/257  235/329  239/280
//   4096, 32, the same               217/276  219/274  315/373  393/473  361/374
//   4200, 32, the same               219/276  250/311  338/421  406/489  371/395
//   8192, 32, the same               331/354  314/378  555/627  683/791  598/596
//   8192, 32, 2048 x 7168            184/223  177/226  296/350  446/527  352/366
//   13483, 3, 5952 x 4752, swiglu    345/401  379/442  854/909  946/1168 883/858
//   2048, 1, 4096 x 4096              55/60    35/40    73/80    89/107   66/76
//   4662, 96, 2064 x 1416             90/117   79/89    73/79    93/101   84/85
//   512, 1, 4096 x 4096               47/60    34/40    23/26    25/27    20/19
//   256, 1, 4096 x 4096               42/60    30/40    22/26    13/14    16/19
// and of few rows                   64 x 128  64 x 64  64 x 32  16 x 32  16 x 16
//   64, 1, 7168 x 4096                27/44    16/22    13/14    15/16    15/21
//   64, 8, 2048 x 1024                10/15   6.2/9.0  6.0/6.8  4.1/6.7  4.9/6.2
//   1, 1, 7168 x 4096                 25/44    14/22    11/14    10/14   5.2/11
// The way chosen is the best of each line or within 6% of it, but for 64 rows over 8
// experts (4.9 for 4.1).
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
