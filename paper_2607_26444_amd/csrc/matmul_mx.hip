// The experts' products on microscaled 4-bit floats:
//   v[r,n] = sum_k a[r,k] w[e,n,k] with the values that codes and scales stand for,
//   y = bf16(v), or with swiglu y[r,i] = bf16(silu(v[r,i]) v[r,N/2+i]).
// Scaled matrix instructions multiply 16 x 16 x 128 codes, a scale byte for each 32 of them,
// and add in float32; the result is rounded to bf16 once.  The kernels are those of the 8-bit
// products (tiles of 256 or 128 rows x 256 channels where arithmetic bounds the call, 64
// rows or fewer x 128 channels or fewer where reading the weights does): a fragment is 16
// bytes to a lane as theirs is, and holds twice the depth.
//
// Which of a row's blocks meet in one instruction is free as long as both operands agree: of a
// stage's eight chunks of 16 bytes (a block of 32 codes each) lane quarter q takes the chunks 2 q
// and 2 q + 1, one to an instruction, so that their two scales are neighbouring bytes which
// a lane reads at once and the instructions select.  In LDS chunk 2 q + h of row r is at place
// (q + 4 h) ^ (r & 7), which no two of the lanes that read together share (2 q + h ^ (r & 7):
// 46 M cycles of bank conflicts beside 104 M of reads).

#include <type_traits>

#include "matmul_tile.h"

namespace moe {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// The chunk of its row that a lane loads to its place.
__device__ __forceinline__ int chunk_of(int lane) {
  const int place = (lane & 7) ^ (lane / 8);
  return (place & 3) * 2 + place / 4;
}

constexpr int kStageScales = kDepth / 16;   // scale bytes of a row and stage

// Both operands are 4-bit floats (format 4), 16 bytes to a lane; SW, SA: the byte of the scale
// words that holds the scale.
template <int SW, int SA>
__device__ __forceinline__ f32x4 multiply_mx(i32x4 w, i32x4 a, f32x4 c, int sw, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
      i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0}, c, 4, 4,
      SW, sw, SA, sa);
}

// A lane's two scales of a row and stage, from LDS.
__device__ __forceinline__ uint32_t two_scales(const uint8_t* p) {
  return *reinterpret_cast<const uint16_t*>(p);
}

// Ones in the bytes of a lane's two scales that lie within the depth, in both halves: what
// lies behind it is no scale, and 255 among it would be NaN.  k: the stage's first byte.
__device__ __forceinline__ uint32_t depth_mask(int k, int quarter, int K) {
  const int at = k + quarter * 32;
  return (at < K ? 0x00FF00FFu : 0u) | (at + 16 < K ? 0xFF00FF00u : 0u);
}

__device__ __forceinline__ void load_scales_to_lds(Rsrc r, uint32_t offset, lds_u8* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 4, (int)offset, 0, 0, 0);
}

// LDS of the kernel of tiles of HEIGHT rows: stages of rows, weights and their scales, and the
// windows.
template <int HEIGHT>
struct MxTileLds {
  static constexpr int kStages = HEIGHT == 256 ? 2 : 3;
  static constexpr int kRowBytes = HEIGHT * kDepth;
  static constexpr int kRowScaleAt = kRowBytes + kTile * kDepth;
  static constexpr int kScaleAt = kRowScaleAt + HEIGHT * kStageScales;   // of the weights
  static constexpr int kStageBytes = kScaleAt + kTile * kStageScales;
  static constexpr int kWindowAt = kStages * kStageBytes;
  static constexpr int kWindows = HEIGHT == 256 ? MOE_MAX_EXPERTS : kMxTile128Experts;
  static constexpr int kBytes = kWindowAt + 3 * kWindows * 4;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
};

// What a wavefront loads of a tile.
template <int HEIGHT>
struct MxTileLoads {
  using Lds = MxTileLds<HEIGHT>;
  Rsrc ra, rw, rsa, rsw;
  uint32_t ao, wo;             // of instruction 0
  uint32_t sao, swo;
  int a_step, w_step;          // from one instruction to the next
  int K, chunk, wave, word;
  uint8_t* s_tile;

  __device__ __forceinline__ MxTileLoads(const MatmulMxArgs& a, const Tile& t, int tid, uint8_t* lds)
      : K(a.K), s_tile(lds) {
    const int lane = tid & (kWave - 1);
    wave = uniform(tid / kWave);
    // instruction j of a wavefront fills LDS rows (j * 8 + wave) * 8 + lane / 8
    const int lr = lane / 8, half = a.N / 2, c0 = t.piece * (a.swiglu ? kTile / 2 : kTile);
    chunk = chunk_of(lane);
    const int r = wave * 8 + lr;
    ao = (uint32_t)r * (uint32_t)a.a_pitch + chunk * 16;
    wo = (uint32_t)channel_of(r, a.swiglu) * (uint32_t)K + chunk * 16;
    a_step = 64 * a.a_pitch;
    w_step = (a.swiglu ? 32 : 64) * K;
    const int channels = (a.swiglu ? half : a.N) - c0, most = a.swiglu ? kTile / 2 : kTile;
    const int held = channels < most ? channels : most;
    const int64_t first = (int64_t)t.expert * a.N + c0;
    ra = buffer_of(a.a + t.row * a.a_pitch, (t.rows - 1) * a.a_pitch + K);
    rw = buffer_of(a.w + (first + (a.swiglu && (wave & 2) ? half : 0)) * K, held * K);
    // scales: two words of a row by two lanes.  Of the weights a wavefront has the rows of the
    // LDS tiles wave & 1 and (wave & 1) + 2 of a block of 64, which with swiglu are all gate
    // or all up channels.
    const int pitch = mx_scale_bytes(2 * K);
    word = (lane & 1) * 4;
    const int n = wave / 2 * 64 + (lane / 32) * 32 + (wave & 1) * 16 + (lane / 2 & 15);
    swo = (uint32_t)channel_of(n, a.swiglu) * (uint32_t)pitch + word;
    sao = (uint32_t)(wave * (HEIGHT / 8) + lane / 2) * (uint32_t)a.a_scale_pitch + word;
    rsa = buffer_of(a.a_scales + t.row * a.a_scale_pitch, (t.rows - 1) * a.a_scale_pitch + pitch);
    rsw = buffer_of(a.w_scales + (first + (a.swiglu && (wave & 1) ? half : 0)) * pitch, held * pitch);
  }

  // A stage into LDS; past the depth and past the tile's rows and channels:
  // zeros.  ROW_LOADS: as many 64 rows as the tile multiplies.
  template <int ROW_LOADS = HEIGHT / 64>
  __device__ __forceinline__ void stage(int k0, uint32_t buf, int lane) const {
    const bool in = k0 + chunk * 16 < K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < ROW_LOADS)
        load_to_lds(ra, in ? ao + (k0 + j * a_step) : kOutside,
                    (lds_u8*)(s_tile + buf + (j * 8 + wave) * 1024));
      load_to_lds(rw, in ? wo + (k0 + j * w_step) : kOutside,
                  (lds_u8*)(s_tile + buf + Lds::kRowBytes + (j * 8 + wave) * 1024));
    }
    // a word of scales covers 64 bytes of codes
    const bool some = k0 + word * 16 < K;
    const uint32_t at = (uint32_t)k0 / 16;
    if (HEIGHT == 256 || lane < HEIGHT / 4)
      load_scales_to_lds(rsa, some ? sao + at : kOutside,
                         (lds_u8*)(s_tile + buf + Lds::kRowScaleAt + wave * HEIGHT));
    load_scales_to_lds(rsw, some ? swo + at : kOutside,
                       (lds_u8*)(s_tile + buf + Lds::kScaleAt + wave * kTile));
  }
};

// One tile whose wavefronts take MT x 16 rows each: 8 for a full tile, 4 or 2
// for the last rows of a window.  Its first stages have been asked for; those of
// `next` are before its own outputs are computed and stored.
template <int HEIGHT, int MT>
__device__ __forceinline__ void multiply_mx_tile(const MatmulMxArgs& a, const Tile& t,
                                                 const Tile& next, int tid, uint8_t* s_tile) {
  using Lds = MxTileLds<HEIGHT>;
  constexpr int NT = 4;
  constexpr int kLoads = MT / 2 + 4 + 2;               // of a wavefront and stage
  const int lane = tid & (kWave - 1), wave = uniform(tid / kWave);
  const MxTileLoads<HEIGHT> loads(a, t, tid, s_tile);

  const int wm = wave / 4, wn = wave % 4;              // 2 x 4 wavefronts
  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = row * kDepth + ((quarter ^ (row & 7)) * 16);
  const uint32_t at_a = wm * (MT * 16 * kDepth) + place;
  const uint32_t at_w = Lds::kRowBytes + wn * (64 * kDepth) + place;
  const uint32_t mine = row * kStageScales + quarter * 2;
  const uint32_t at_sa = Lds::kRowScaleAt + wm * (MT * 16 * kStageScales) + mine;
  const uint32_t at_sw = Lds::kScaleAt + wn * (64 * kStageScales) + mine;
  f32x4 acc[MT][NT] = {};

  i32x4 av[2][MT], wv[2][NT];
  auto read = [&](int h, uint32_t buf) {               // half a stage into registers
    const uint8_t* pw = s_tile + (at_w ^ (h * 64)) + buf;
    const uint8_t* pa = s_tile + (at_a ^ (h * 64)) + buf;
#pragma unroll
    for (int j = 0; j < NT; ++j) wv[h][j] = *(const i32x4*)(pw + j * 16 * kDepth);
#pragma unroll
    for (int i = 0; i < MT; ++i) av[h][i] = *(const i32x4*)(pa + i * 16 * kDepth);
  };
  uint32_t sa[MT / 2], sw[NT / 2];                     // two tiles' scales to a word
  auto read_scales = [&](uint32_t buf) {
    const uint8_t* pw = s_tile + at_sw + buf;
    const uint8_t* pa = s_tile + at_sa + buf;
    // tiles j and j + 2 lie in one wavefront's part
#pragma unroll
    for (int j = 0; j < NT / 2; ++j)
      sw[j] = two_scales(pw + j * 32 * kStageScales) |
              two_scales(pw + (j * 32 + 16) * kStageScales) << 16;
#pragma unroll
    for (int i = 0; i < MT / 2; ++i)
      sa[i] = two_scales(pa + i * 32 * kStageScales) |
              two_scales(pa + (i * 32 + 16) * kStageScales) << 16;
  };
  auto multiply = [&](auto half, int i0, int i1) {
    constexpr int h = half.value;
#pragma unroll
    for (int i = i0; i < i1; ++i) {
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int s = (int)sw[j & 1], r = (int)sa[i / 2];   // channel tiles j and j + 2 share a word
        if (j < 2 && i % 2 == 0) acc[i][j] = multiply_mx<h, h>(wv[h][j], av[h][i], acc[i][j], s, r);
        if (j < 2 && i % 2 == 1) acc[i][j] = multiply_mx<h, h + 2>(wv[h][j], av[h][i], acc[i][j], s, r);
        if (j >= 2 && i % 2 == 0) acc[i][j] = multiply_mx<h + 2, h>(wv[h][j], av[h][i], acc[i][j], s, r);
        if (j >= 2 && i % 2 == 1) acc[i][j] = multiply_mx<h + 2, h + 2>(wv[h][j], av[h][i], acc[i][j], s, r);
      }
    }
  };
  constexpr std::integral_constant<int, 0> kFirst;
  constexpr std::integral_constant<int, 1> kSecond;

  // Stage s is in LDS at s % kStages.  Within a turn the wavefronts meet once: by
  // then each has read the last of stage s into registers, and its loads of
  // stage s + 1, asked for kStages - 1 turns ago, have arrived.  Half of the matrix
  // instructions of a register set stand on either side of the barrier.
  meet<0>();                                           // the first stages are there
  uint32_t buf = 0;
  read(0, 0);
  for (int k0 = 0; k0 < a.K; k0 += kDepth) {
    read_scales(buf);
    if (k0 + kDepth > a.K) {
      const uint32_t mask = depth_mask(k0, quarter, a.K);
#pragma unroll
      for (int j = 0; j < NT / 2; ++j) sw[j] &= mask;
#pragma unroll
      for (int i = 0; i < MT / 2; ++i) sa[i] &= mask;
    }
    read(1, buf);
    multiply(kFirst, 0, MT / 2);
    interleave<kIssueLdsRead, MT + NT, 1>();
    meet<(Lds::kStages - 2) * kLoads>();
    loads.template stage<MT / 2>(k0 + Lds::kStages * kDepth, buf, lane);
    multiply(kFirst, MT / 2, MT);
    if constexpr (Lds::kStages == 2) buf = Lds::kStageBytes - buf;
    else buf = buf + Lds::kStageBytes == Lds::kWindowAt ? 0 : buf + Lds::kStageBytes;
    __builtin_amdgcn_sched_barrier(0);
    read(0, buf);
    multiply(kSecond, 0, MT);
    interleave<kIssueLdsRead, MT + NT, MT / 4 + 1 < 2 ? 1 : 2>();
    // the reads stay in this turn
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  meet<0>();                                           // loads past the end have landed

  if (next.rows) {
    const MxTileLoads<HEIGHT> first(a, next, tid, s_tile);
#pragma unroll
    for (int n = 0; n < Lds::kStages; ++n) first.stage(n * kDepth, n * Lds::kStageBytes, lane);
  }

  const int out = a.swiglu ? a.N / 2 : a.N;
  const int c0 = t.piece * (a.swiglu ? kTile / 2 : kTile) +
                 (a.swiglu ? wn * 32 + quarter * 8 : wn * 64 + quarter * 16);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = wm * (MT * 16) + i * 16 + row;
    if (r >= t.rows) continue;
    uint16_t* y = a.y + (t.row + r) * out;
    float v[8];
    if (a.swiglu) {
      if (c0 >= out) continue;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int j = q / 4 * 2;
        v[q] = silu(acc[i][j][q & 3]) * acc[i][j + 1][q & 3];
      }
      st16(y + c0, pack8(v));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (c0 + h * 8 >= out) continue;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = acc[i][h * 2 + q / 4][q & 3];
        st16(y + c0 + h * 8, pack8(v));
      }
    }
  }
}

// A workgroup to each compute unit takes the tiles blockIdx.x, + 256, ... of
// an order in which the 32 tiles that an XCD's compute units hold together are
// neighbours.
template <int HEIGHT>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void matmul_mx_tile_kernel(MatmulMxArgs a, int pieces, int group) {
  using Lds = MxTileLds<HEIGHT>;
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[Lds::kBytes];
  int* s_end = reinterpret_cast<int*>(s_tile + Lds::kWindowAt);  // row tiles to a window's end
  int* s_start = s_end + Lds::kWindows;
  int* s_rows = s_start + Lds::kWindows;
  const int lane = threadIdx.x & (kWave - 1);
  if (threadIdx.x < kWave) {
    const int first = a.offset ? uniform((int)ld4(a.offset)) : 0;
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      int s = 0, m = (int)a.rows;
      if (a.offset) window_of(a, e0 + lane < a.E ? e0 + lane : a.E - 1, first, s, m);
      if (e0 + lane >= a.E) m = 0;
      const int end = before + scan_add((m + HEIGHT - 1) / HEIGHT);
      s_end[e0 + lane] = end;                          // E is at most kWindows, whole 64s
      s_start[e0 + lane] = s;
      s_rows[e0 + lane] = m;
      before = __builtin_amdgcn_readlane(end, kWave - 1);
    }
  }
  __syncthreads();
  auto tile_at = [&](int n) -> Tile {
    const int id = n * 256 + (blockIdx.x & 7) * 32 + blockIdx.x / 8;
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      const uint64_t hit = __ballot((int64_t)s_end[e0 + lane] * pieces > id);
      if (!hit) continue;
      const int e = e0 + __builtin_ctzll(hit);
      const int before = e ? uniform(s_end[e - 1]) : 0;
      return tile_of(e, uniform(s_start[e]), uniform(s_rows[e]), id - before * pieces, HEIGHT,
                     pieces, group);
    }
    return {0, 0, 0, 0};
  };

  Tile t = tile_at(0);
  if (t.rows == 0) return;                             // the whole workgroup
  int tid = threadIdx.x;
  {
    const MxTileLoads<HEIGHT> first(a, t, tid, s_tile);
#pragma unroll
    for (int n = 0; n < Lds::kStages; ++n) first.stage(n * kDepth, n * Lds::kStageBytes, lane);
  }
  for (int n = 1;; ++n) {
    const Tile next = tile_at(n);
    // what follows from the thread's number is worked out anew for each tile:
    // kept over the loop it would not fit the registers
    asm volatile("" : "+v"(tid));
    if (HEIGHT > 128 && t.rows > 128)
      multiply_mx_tile<HEIGHT, HEIGHT / 32>(a, t, next, tid, s_tile);
    else if (t.rows > 64) multiply_mx_tile<HEIGHT, 4>(a, t, next, tid, s_tile);
    else multiply_mx_tile<HEIGHT, 2>(a, t, next, tid, s_tile);
    if (next.rows == 0) return;
    t = next;
  }
}

// Few rows: ROWS rows of a window x 16 WC channels, bound by reading the
// weights.  Eight wavefronts, WC along the channels and WK along the depth; a
// stage is 128 WK bytes of the depth, STAGES - 1 stages are on their way while one is
// multiplied.  A wavefront loads its own weights (8 + 8 channels: with swiglu
// gate and up channels, so that a lane and its partner 32 further on hold both
// halves) and an eighth of the rows.  The sums of the WK wavefronts meet in LDS.
//
// Scales come as pieces of 16 bytes of a row, whose lines cost more than their bytes: 8 bytes of
// each row a stage, word by word, took 22 of 100 us (512 rows, 32 experts, 7168 x 4096 with
// swiglu).  A row's pieces hold the stage, with WK = 1 two stages.
template <int ROWS, int WC, int WK, int STAGES>
struct MxStreamLds {
  static constexpr int kBatch = WK == 1 ? 2 : 1;       // stages whose scales come together
  static constexpr int kRowScales = kBatch * WK * kStageScales, kPieces = kRowScales / 16;
  static constexpr int kScaleRows = WC * 16 + ROWS;    // the channels, then the rows
  static constexpr int kScaleBytes = kScaleRows * kRowScales;
  static constexpr int kPerWave = kScaleRows * kPieces / 8;
  static_assert(kPerWave * 8 == kScaleRows * kPieces && kPerWave <= kWave, "one instruction");
  static constexpr int kRowBytes = ROWS * kDepth * WK;
  static constexpr int kCodes = kRowBytes + 16 * 1024;
  static constexpr int kStage = kCodes + (kBatch == 1 ? kScaleBytes : 0);
  static constexpr int kBatchAt = STAGES * kStage;     // two batches, where they are no part of stages
  // what a tail's scales are read past the last row's
  static constexpr int kBytes = kBatchAt + (kBatch == 1 ? 0 : 2 * kScaleBytes) + 64;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
};

template <int ROWS, int WC, int WK, int STAGES>
__global__ __launch_bounds__(kTileThreads)
void matmul_mx_stream_kernel(MatmulMxArgs a, int pieces) {
  using Lds = MxStreamLds<ROWS, WC, WK, STAGES>;
  static_assert(WC * WK == 8, "eight wavefronts");
  constexpr int MT = ROWS / 16;
  constexpr int kRowBytes = Lds::kRowBytes, kStage = Lds::kStage;
  constexpr int kRowLoads = WK * ROWS / 64;            // of a wavefront and stage
  static_assert(kRowLoads * 64 == WK * ROWS, "whole load instructions");
  // a batch of two stages is asked for before the codes of its first one, so that no
  // count of loads on their way has to know of it
  constexpr int kLoads = 2 + kRowLoads + (Lds::kBatch == 1 ? 1 : 0);
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[Lds::kBytes];
  static_assert(STAGES * kStage >= 8 * MT * kWave * 16, "sums meet there");
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  // 32 neighbouring tiles (mostly one window's, which share rows) to an XCD
  const int b = blockIdx.x;
  const Tile t = find_tile(a, b / 256 * 256 + b % 8 * 32 + b / 8 % 32, ROWS, pieces);
  if (t.rows == 0) return;                             // the whole workgroup
  const int half = a.N / 2, out = a.swiglu ? half : a.N;
  const int wc = wave % WC, wk = wave / WC;
  const int step = a.swiglu ? 8 : 16;                  // output channels of a wavefront
  const int c0 = t.piece * WC * step + wc * step;

  const int lr = lane / 8, chunk = chunk_of(lane);
  const Rsrc ra = buffer_of(a.a + t.row * a.a_pitch, (t.rows - 1) * a.a_pitch + a.K);
  const uint8_t* wbase = a.w + ((int64_t)t.expert * a.N + c0) * a.K;
  const int c1 = a.swiglu ? c0 : c0 + 8;               // channels come in whole eights
  const Rsrc rw0 = buffer_of(wbase, c0 < out ? 8 * a.K : 0);
  const Rsrc rw1 = buffer_of(wbase + (int64_t)(a.swiglu ? half : 8) * a.K, c1 < out ? 8 * a.K : 0);
  const uint32_t wo = (uint32_t)lr * (uint32_t)a.K + wk * kDepth + chunk * 16;

  // A lane's piece of the scales, by address: that of a row or channel that is not there
  // is another's (its outputs are not stored).  A row's last piece ends with it: scales
  // are read as much further on.  Rows of less than a piece come word by word.
  const int scale_bytes = mx_scale_bytes(2 * a.K);
  const bool words = scale_bytes < 16;
  const int last_piece = words ? 0 : scale_bytes - 16;
  const int piece = (wave * Lds::kPerWave + lane) % Lds::kPieces * 16;
  const uint8_t* scales;
  {
    const int n = (wave * Lds::kPerWave + lane) / Lds::kPieces;
    if (n < WC * 16) {
      int c = t.piece * WC * step + n / 16 * step + (n & 7) + ((n & 8) && !a.swiglu ? 8 : 0);
      c = c < out ? c : out - 1;
      if ((n & 8) && a.swiglu) c += half;
      scales = a.w_scales + ((int64_t)t.expert * a.N + c) * scale_bytes;
    } else {
      const int r = n - WC * 16;
      scales = a.a_scales + (t.row + (r < t.rows ? r : t.rows - 1)) * a.a_scale_pitch;
    }
  }
  auto scales_at = [&](int k0, uint32_t at) -> uint32_t {   // of the stage at `at`
    return Lds::kBatch == 1 ? at + Lds::kCodes
                            : Lds::kBatchAt + (k0 / (2 * kDepth) & 1) * Lds::kScaleBytes;
  };
  if (words) {                                         // the only scales there are
    if (lane < Lds::kPerWave) {
      u32x4 v = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (piece + i * 4 < scale_bytes) v[i] = ld4(scales + piece + i * 4);
      *reinterpret_cast<u32x4*>(s_mem + scales_at(0, 0) + (wave * Lds::kPerWave + lane) * 16) = v;
    }
    scales = a.w;                                      // later stages read 16 bytes of no use
  }
  auto load_scales = [&](int k0, uint32_t at) {
    if (lane >= Lds::kPerWave || (words && k0 == 0)) return;
    const int want = (Lds::kBatch == 1 ? k0 / 16 : k0 / (2 * kDepth) * 16) + piece;
    const uint8_t* from = scales + (want < last_piece ? want : last_piece);
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) uint32_t*)(uintptr_t)from,
        (__attribute__((address_space(3))) uint32_t*)(lds_u8*)(s_mem + scales_at(k0, at) +
                                                               wave * Lds::kPerWave * 16),
        16, 0, 0);
  };
  auto load = [&](int k0, uint32_t at) {               // past the depth: zeros
    if (Lds::kBatch == 1 || !(k0 & kDepth)) load_scales(k0, at);
    const uint32_t w = (uint32_t)k0 + wk * kDepth + chunk * 16 < (uint32_t)a.K ? wo + k0 : kOutside;
    uint8_t* to = s_mem + at + kRowBytes + wave * 2048;
    load_to_lds(rw0, w, (lds_u8*)to);
    load_to_lds(rw1, w, (lds_u8*)(to + 1024));
#pragma unroll
    for (int g = 0; g < kRowLoads; ++g) {              // eight rows of a 128 of the depth
      const int n = g * 8 + wave, r = n % (ROWS / 8) * 8 + lr;
      const uint32_t k = (uint32_t)k0 + n / (ROWS / 8) * kDepth + chunk * 16;
      load_to_lds(ra, k < (uint32_t)a.K ? (uint32_t)r * (uint32_t)a.a_pitch + k : kOutside,
                  (lds_u8*)(s_mem + at + n * 1024));
    }
  };
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) load(s * kDepth * WK, s * kStage);

  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = row * kDepth + ((quarter ^ (row & 7)) * 16);
  const uint32_t mine = row * Lds::kRowScales + quarter * 2;
  f32x4 acc[MT] = {};
  auto multiply = [&](auto row_tiles) {
    constexpr int M = row_tiles.value;
    uint32_t at = 0, fill = (STAGES - 1) * kStage;     // stage to read, stage to fill
    for (int k0 = 0; k0 < a.K; k0 += kDepth * WK) {
      meet<(STAGES - 2) * kLoads>();                   // this stage is there, the last is read
      load(k0 + (STAGES - 1) * kDepth * WK, fill);
      i32x4 wv[2], av[2][M];
      const int k = k0 + wk * kDepth;                  // the wavefront's part of the stage
      const uint32_t mask = depth_mask(k, quarter, a.K);
      // its scales in their piece, and how far that lies before the place it was meant for
      const int first = k / 256 * 16;
      const int behind = words || first < last_piece ? 0 : first - last_piece;
      const uint32_t ps = scales_at(k0, at) + (Lds::kBatch == 1 ? k / 16 - k0 / 16 : k / 16 - first) +
                          (behind < 16 ? behind : 16) + mine;
      const int sw = (int)(two_scales(s_mem + ps + wc * 16 * Lds::kRowScales) & mask);
      int sa[M];
#pragma unroll
      for (int i = 0; i < M; ++i)
        sa[i] = (int)(two_scales(s_mem + ps + (WC + i) * 16 * Lds::kRowScales) & mask);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t p = at + (place ^ (h * 64));
        wv[h] = *(const i32x4*)(s_mem + kRowBytes + wave * 2048 + p);
#pragma unroll
        for (int i = 0; i < M; ++i)
          av[h][i] = *(const i32x4*)(s_mem + wk * (ROWS * kDepth) + i * 16 * kDepth + p);
      }
#pragma unroll
      for (int i = 0; i < M; ++i) {
        acc[i] = multiply_mx<0, 0>(wv[0], av[0][i], acc[i], sw, sa[i]);
        acc[i] = multiply_mx<1, 1>(wv[1], av[1][i], acc[i], sw, sa[i]);
      }
      at = at + kStage == STAGES * kStage ? 0 : at + kStage;
      fill = fill + kStage == STAGES * kStage ? 0 : fill + kStage;
    }
  };
  const int mt = (t.rows + 15) / 16;
  if (ROWS == 16 || mt == 1) multiply(std::integral_constant<int, 1>());
  else if (mt == 2) multiply(std::integral_constant<int, ROWS == 16 ? 1 : 2>());
  else multiply(std::integral_constant<int, MT>());
  meet<0>();                                           // loads past the end have landed

  f32x4* s_acc = reinterpret_cast<f32x4*>(s_mem);      // [wavefront][row tile][lane]
#pragma unroll
  for (int i = 0; i < MT; ++i) s_acc[(wave * MT + i) * kWave + lane] = acc[i];
  __syncthreads();
  // tile (w, i): channels of wavefront column w, rows 16 i..; a lane's four
  // sums are channels quarter * 4 .. + 3 of row `row`
  for (int n = wave; n < WC * mt; n += 8) {
    const int w = n % WC, i = n / WC;
    const int r = i * 16 + row;
    f32x4 sum = s_acc[(w * MT + i) * kWave + lane];
#pragma unroll
    for (int g = 1; g < WK; ++g) sum += s_acc[((g * WC + w) * MT + i) * kWave + lane];
    const int lc = w * step + (quarter * 4) % step, c = t.piece * WC * step + lc;
    const bool in = r < t.rows && c < out;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = sum[q];
      if (a.swiglu) v[q] = silu(v[q]) * __shfl_xor(v[q], 32, kWave);   // gate lanes, up lanes
    }
    if (in && !(a.swiglu && quarter > 1))
      st4x2(a.y + (t.row + r) * out + c, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

template <int HEIGHT, int WAY>
hipError_t launch_tile(const MatmulMxArgs& a, int group, hipStream_t stream) {
  constexpr Way w = kMxWay[WAY];
  static_assert(w.rows == HEIGHT && w.channels == kTile, "the rule's tile");
  hipLaunchKernelGGL((matmul_mx_tile_kernel<HEIGHT>), dim3(256), dim3(kTileThreads), 0, stream, a,
                     pieces_of(a, w), group);
  return hipGetLastError();
}

template <int ROWS, int WC, int WK, int STAGES, int WAY>
hipError_t launch_stream(const MatmulMxArgs& a, hipStream_t stream) {
  constexpr Way w = kMxWay[WAY];
  static_assert(w.rows == ROWS && w.channels == 16 * WC && w.depth == kDepth * WK,
                "the rule's tile");
  const int64_t groups = (tiles_of(a, w) + 255) / 256 * 256;
  hipLaunchKernelGGL((matmul_mx_stream_kernel<ROWS, WC, WK, STAGES>), dim3((unsigned)groups),
                     dim3(kTileThreads), 0, stream, a, pieces_of(a, w));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul_mx(const MatmulMxArgs& a, hipStream_t stream) {
  switch (choose_mx_way(a)) {
    case kTile256: return launch_tile<256, kTile256>(a, 6, stream);
    case kTile128: return launch_tile<128, kTile128>(a, 6, stream);
    case kWide: return launch_stream<64, 8, 1, 3, kWide>(a, stream);
    case kHalf: return launch_stream<64, 4, 2, 3, kHalf>(a, stream);
    case kHalfTwo: return launch_stream<64, 4, 2, 2, kHalfTwo>(a, stream);
    case kNarrow: return launch_stream<64, 2, 4, 3, kNarrow>(a, stream);
    case kFewRows: return launch_stream<16, 2, 4, 3, kFewRows>(a, stream);
    case kOneRow: return launch_stream<16, 1, 8, 2, kOneRow>(a, stream);
    default: return hipErrorInvalidConfiguration;
  }
}

}  // namespace moe
