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
inline int64_t row_tiles(const MatmulShape& a, int size) {
  if (!a.offset) return (a.rows + size - 1) / size;
  return a.rows / size + (a.rows < a.E ? a.rows : a.E);
}

// Row tiles of `size` if the rows are spread about evenly.
inline double even_tiles(const MatmulShape& a, int size) {
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
inline int out_channels(const MatmulShape& a) { return a.swiglu ? a.N / 2 : a.N; }
inline int tile_channels(const MatmulShape& a, const Way& w) {
  return a.swiglu ? w.channels / 2 : w.channels;
}
inline int pieces_of(const MatmulShape& a, const Way& w) {
  const int per = tile_channels(a, w);
  return (out_channels(a) + per - 1) / per;
}
inline int64_t tiles_of(const MatmulShape& a, const Way& w) {
  return row_tiles(a, w.rows) * pieces_of(a, w);
}

// Whether way `n`, with the sizes that its table has, can be launched for the call.
inline bool way_fits(const MatmulShape& a, const Way* ways, int n) {
  return tiles_of(a, ways[n]) <= (n == kTile256 || n == kTile128 ? kMaxTiles : kMaxGroups);
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
inline double way_time(const MatmulShape& a, const Way& w) {
  const double groups = even_tiles(a, w.rows) * pieces_of(a, w);
  const double full = groups / w.resident;
  const double rounds = full < 1.0 ? 1.0 : full + 0.75 * (__builtin_ceil(full) - full);
  const int stages = (a.K + w.depth - 1) / w.depth;
  const double work = rounds * (w.start + stages * (groups <= 256.0 ? w.alone : w.shared));
  const double read = (double)(a.rows < a.E ? a.rows : a.E) * a.N * a.K / w.rate;
  return __builtin_sqrt(work * work + read * read);
}

// The way of a table that takes least of those that can be launched; kWays if none can be.
inline int quickest_way(const MatmulShape& a, const Way* ways) {
  int best = kWays;
  double least = 0.0;
  for (int n = 0; n < kWays; ++n) {
    if (!way_fits(a, ways, n)) continue;
    const double t = way_time(a, ways[n]);
    if (best == kWays || t < least) {
      least = t;
      best = n;
    }
  }
  return best;
}
inline int choose_way(const MatmulShape& a) { return quickest_way(a, kWay); }

// The same for the products on 4-bit floats, depths in bytes of codes.  The rates are those that
// fit beside the rounds' times, not the memory's: most of the reading hides.  Measured / model, us,
// rows drawn to the experts evenly:
//   rows, experts, K x N               256      128      64 x 128  64 x 64 three, two stages
//   512, 32, 7168 x 4096, swiglu     100/120   89/97     82/85   101/107   93/95
//   512, 32, 2048 x 7168              63/88    59/65     49/54    72/84    56/62
//   2048, 32, 7168 x 4096, swiglu    110/120   98/97    133/121  182/156  152/136
//   4096, 32, the same               134/120  155/129   205/196  286/256  231/220
//   8192, 32, the same               230/175  212/201   340/349  507/459  382/393
//   8192, 32, 2048 x 7168            137/130  130/138   194/212  346/373  239/271
//   16384, 32, the same              191/198  222/242   355/396  647/704  454/508
//   13483, 3, 5952 x 4752, swiglu    225/237  265/270   523/534  727/713  601/606
//   32768, 16, 7168 x 4096, swiglu   477/504  596/649  1136/1268 1878/1652 1350/1412
//   2048, 1, 4096 x 4096              40/36    28/24     46/47    68/69    48/55
//   4662, 96, 2080 x 1416             61/68    55/49     50/42    74/60    54/49
//   512, 1, 4096 x 4096               37/36    26/24     16/14    20/17    15/14
//   24000, 64, 1024 x 512             19/15    22/20     27/31    53/59    34/40
// and of few rows                   64 x 128  64 x 64  64 x 32  16 x 32  16 x 16
//   8, 32, 7168 x 4096, swiglu        22/24    24/27    33/36    22/23    32/33
//   256, 1, 4096 x 4096               15/14   11.2/9.6  14/13    21/27    29/40
//   64, 1, 7168 x 4096, swiglu        21/23    14/14    11/10    11/9.6   14/13
//   64, 8, 2048 x 1024               7.3/8.7  5.8/6.4  5.6/5.5  4.5/4.4  4.7/4.4
//   1, 1, 7168 x 4096                 16/23    10/14   8.2/10   7.5/7.7  5.9/5.9
// The way chosen is the best of each line or within 3% of it, but for 8192 rows over 32
// experts (230 for 212, 137 for 130), where it depends on how many windows pass 256 rows: the model
// knows their sum alone.  For the same reason fixed windows are taken as if they were full: 512
// rows in 32 windows of 16 take what packed ones do (81 us, 7168 x 4096 with swiglu; 49, 2048 x
// 7168), in windows of 32 91 and 52, of 64 92 and 60, of 128 to 512 102 and 63.
constexpr Way kMxWay[kWays] = {
    {256, 256, 128, 256, 8.2, 1.73, 1.73, 11.5e6},     // matmul_mx_tile_kernel<256>
    {128, 256, 128, 256, 5.7, 1.17, 1.17, 8.0e6},      // matmul_mx_tile_kernel<128>
    {64, 128, 128, 512, 3.1, 0.70, 1.27, 13.5e6},      // matmul_mx_stream_kernel<64, 8, 1, 3>
    {64, 64, 256, 256, 3.2, 0.80, 0.68, 14.0e6},       // <64, 4, 2, 3>
    {64, 64, 256, 512, 3.2, 0.95, 1.32, 12.5e6},       // <64, 4, 2, 2>
    {64, 32, 512, 256, 3.5, 0.92, 0.70, 10.0e6},       // <64, 2, 4, 3>
    {16, 32, 512, 512, 2.9, 0.66, 0.94, 9.2e6},        // <16, 2, 4, 3>
    {16, 16, 1024, 512, 3.4, 0.48, 0.77, 6.0e6},       // <16, 1, 8, 2>
};
static_assert(kTile * 2ll * MOE_MAX_MX_CHANNELS < 1ll << 31, "a tile's stores have 31-bit offsets");
inline int choose_mx_way(const MatmulShape& a) { return quickest_way(a, kMxWay); }

// Whether a streaming way keeps the weights of a call on 4-bit floats out of the caches: those that
// one tile of a window reads and that the caches would not keep, 512 rows, 32 experts, 7168 x 4096
// 89 -> 83 us.  Windows of several tiles read them again (4662 rows over 96 experts 50 -> 63, 2048
// rows 31 -> 33), and rows that are no whole lines share lines between stages (512 rows, 32
// experts, 7136 x 4096 108 -> 122).
inline bool weights_read_once(const MatmulShape& a) {
  return a.rows <= 16 * (int64_t)a.E && a.K % 128 == 0 &&
         (int64_t)a.E * a.N * a.K >= (int64_t)128 << 20;
}

}  // namespace moe
