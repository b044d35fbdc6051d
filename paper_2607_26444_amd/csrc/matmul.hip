// The experts' products on 8-bit integers:
//   v[r,n] = (sum_k a[r,k] w[e,n,k]) a_scale[r] w_scale[e,n], y = bf16(v), or with
//   swiglu y[r,i] = bf16(silu(v[r,i]) v[r,N/2+i]).
// int32 sums by matrix instructions, exact in any order, scaled and rounded to
// bf16 once.  Two kernels: tiles of 256 or 128 rows x 256 channels where
// arithmetic bounds the call, 64 rows or fewer x 128 channels or fewer where reading
// the weights does.
// Windows are on the GPU, so a launch covers every tile that they can have;
// workgroups find theirs by a scan of the counts.

#include <type_traits>

#include "matmul_tile.h"

namespace moe {
namespace {

// Tiles of 256 or 128 rows x 256 channels through LDS: eight wavefronts, each half
// the rows x 64 channels; stages of 128 of the depth go from memory into LDS by
// the loads themselves, one stage ahead of the matrix instructions, two with 128 rows.
// A wavefront of 128 rows reads 12 fragments for 32 matrix instructions of 16 x 16 x
// 64, half a stage ahead.  Tiles of 128 rows are for calls that make few of 256: a tile
// alone waits for memory 1.6 us a stage with 256 rows and one stage ahead, 1.05 us with
// 128 and two (32 experts of 128 rows, 7168 x 4096 with swiglu 225 and 184 us; 2048 x 4096
// x 4096 55 and 35).  With one stage ahead tiles of 128 rows took a quarter longer.
//
// Bound by the matrix instructions and the clock that the card's power leaves them.  Of
// four calls one after another the clock falls from 1.95 to 1.34 GHz and the matrix
// instructions are busy 59 to 70% of the cycles (operands of zeros run 8% faster); between a
// layer's other kernels 54% at 1.96 GHz.
// 32768 rows, 16 experts, 7168 x 4096 with swiglu: 805 to 847 us by card, 2270 to
// 2390 TOP/s; 16384 x 8192 x 8192: 807 to 842 us, 2610 to 2725 TOP/s; 32 experts of 980
// to 1080 rows, 7168 x 4096: 835 us.  Beside it 32 x 32 x 32 instructions 1012 us (16 x
// 16 x 64 then: 934), stages of half the depth with the wavefronts in two phases
// 920 (850), a second barrier +4%, touching the lines of later stages beforehand +2
// to 10%.

// LDS of the kernel of tiles of HEIGHT rows: stages of rows and weights, the scales
// of this tile and the next, and the windows.
template <int HEIGHT>
struct TileLds {
  static constexpr int kStages = HEIGHT == 256 ? 2 : 3;
  static constexpr int kRowBytes = HEIGHT * kDepth, kStageBytes = kRowBytes + kTile * kDepth;
  static constexpr int kScaleAt = kStages * kStageBytes;
  static constexpr int kWindowAt = kScaleAt + 2 * 2 * kTile * 4;
  static constexpr int kBytes = kWindowAt + 3 * MOE_MAX_EXPERTS * 4;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
};

// What a wavefront loads of a tile.
template <int HEIGHT>
struct TileLoads {
  using Lds = TileLds<HEIGHT>;
  Rsrc ra, rw;
  uint32_t ao, wo;             // of instruction 0
  int a_step, w_step;          // from one instruction to the next
  int K, chunk, wave;
  uint8_t* s_tile;

  __device__ __forceinline__ TileLoads(const MatmulArgs& a, const Tile& t, int tid, uint8_t* lds)
      : K(a.K), s_tile(lds) {
    const int lane = tid & (kWave - 1);
    wave = uniform(tid / kWave);
    // instruction j of a wavefront fills LDS rows (j * 8 + wave) * 8 + lane / 8
    const int lr = lane / 8, half = a.N / 2, c0 = t.piece * (a.swiglu ? kTile / 2 : kTile);
    chunk = (lane & 7) ^ lr;
    const int r = wave * 8 + lr;
    ao = (uint32_t)r * (uint32_t)K + chunk * 16;
    wo = (uint32_t)channel_of(r, a.swiglu) * (uint32_t)K + chunk * 16;
    a_step = 64 * K;
    w_step = (a.swiglu ? 32 : 64) * K;
    const int channels = (a.swiglu ? half : a.N) - c0, most = a.swiglu ? kTile / 2 : kTile;
    const bool up = a.swiglu && (wave & 2);            // this wavefront's rows are of odd tiles
    ra = buffer_of(a.a + t.row * K, t.rows * K);
    rw = buffer_of(a.w + ((int64_t)t.expert * a.N + c0 + (up ? half : 0)) * K,
                   (channels < most ? channels : most) * K);
  }

  // A stage into LDS; past the depth and past the tile's rows and channels:
  // zeros.  ROW_LOADS: as many 64 rows as the tile multiplies.
  template <int ROW_LOADS = HEIGHT / 64>
  __device__ __forceinline__ void stage(int k0, uint32_t buf) const {
    const bool in = k0 + chunk * 16 < K;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (j < ROW_LOADS)
        load_to_lds(ra, in ? ao + (k0 + j * a_step) : kOutside,
                    (lds_u8*)(s_tile + buf + (j * 8 + wave) * 1024));
      load_to_lds(rw, in ? wo + (k0 + j * w_step) : kOutside,
                  (lds_u8*)(s_tile + buf + Lds::kRowBytes + (j * 8 + wave) * 1024));
    }
  }
};

// A thread's scale of the tile: a row's, or a channel's in the order of LDS.
__device__ __forceinline__ float tile_scale(const MatmulArgs& a, const Tile& t, int tid) {
  const int n = tid & 255;
  if (tid < 256) return n < t.rows ? a.a_scales[(t.row + n) * a.a_scale_pitch] : 0.0f;
  const int out = a.swiglu ? a.N / 2 : a.N;
  const int c = t.piece * (a.swiglu ? kTile / 2 : kTile) + channel_of(n, a.swiglu);
  const bool up = a.swiglu && (n & 16);
  return c < out ? a.w_scales[(int64_t)t.expert * a.N + c + (up ? out : 0)] : 0.0f;
}

// One tile whose wavefronts take MT x 16 rows each: 8 for a full tile, 4 or 2
// for the last rows of a window (as long as reading the weights, but half or
// a quarter of the products).  Its first stages have been asked for; those of
// `next` are before its own outputs are computed and stored.
template <int HEIGHT, int MT>
__device__ __forceinline__ void multiply_tile(const MatmulArgs& a, const Tile& t, const Tile& next,
                                              int tid, uint8_t* s_tile, int slot, float& scale) {
  using Lds = TileLds<HEIGHT>;
  constexpr int NT = 4;
  constexpr int kLoads = MT / 2 + 4;                   // of a wavefront and stage
  float* s_scale = reinterpret_cast<float*>(s_tile + Lds::kScaleAt) + slot * 2 * kTile;
  const int lane = tid & (kWave - 1), wave = uniform(tid / kWave);
  const TileLoads<HEIGHT> loads(a, t, tid, s_tile);
  s_scale[tid] = scale;

  const int wm = wave / 4, wn = wave % 4;              // 2 x 4 wavefronts
  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = row * kDepth + ((quarter ^ (row & 7)) * 16);
  const uint32_t at_a = wm * (MT * 16 * kDepth) + place;
  const uint32_t at_w = Lds::kRowBytes + wn * (64 * kDepth) + place;
  i32x4 acc[MT][NT] = {};

  i32x4 av[2][MT], wv[2][NT];
  auto read = [&](int h, uint32_t buf) {               // half a stage into registers
    const uint8_t* pw = s_tile + (at_w ^ (h * 64)) + buf;
    const uint8_t* pa = s_tile + (at_a ^ (h * 64)) + buf;
#pragma unroll
    for (int j = 0; j < NT; ++j) wv[h][j] = *(const i32x4*)(pw + j * 16 * kDepth);
#pragma unroll
    for (int i = 0; i < MT; ++i) av[h][i] = *(const i32x4*)(pa + i * 16 * kDepth);
  };
  auto multiply = [&](int h, int i0, int i1) {
#pragma unroll
    for (int i = i0; i < i1; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[h][j], av[h][i], acc[i][j], 0, 0, 0);
  };

  // Stage s is in LDS at s % kStages.  Within a turn the wavefronts meet once: by
  // then each has read the last of stage s into registers, and its loads of
  // stage s + 1, asked for kStages - 1 turns ago, have arrived.  Half of the matrix
  // instructions of a register set stand on either side of the barrier.
  meet<0>();                                           // the first stages are there
  uint32_t buf = 0;
  read(0, 0);
  for (int k0 = 0; k0 < a.K; k0 += kDepth) {
    read(1, buf);
    multiply(0, 0, MT / 2);
    interleave<kIssueLdsRead, MT + NT, 1>();
    meet<(Lds::kStages - 2) * kLoads>();
    loads.template stage<MT / 2>(k0 + Lds::kStages * kDepth, buf);
    multiply(0, MT / 2, MT);
    if constexpr (Lds::kStages == 2) buf ^= Lds::kStageBytes;
    else buf = buf + Lds::kStageBytes == Lds::kScaleAt ? 0 : buf + Lds::kStageBytes;
    __builtin_amdgcn_sched_barrier(0);
    read(0, buf);
    multiply(1, 0, MT);
    interleave<kIssueLdsRead, MT + NT, MT / 4 + 1 < 2 ? 1 : 2>();
    // the reads stay in this turn
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  meet<0>();                                           // loads past the end have landed

  if (next.rows) {
    scale = tile_scale(a, next, tid);
    const TileLoads<HEIGHT> first(a, next, tid, s_tile);
#pragma unroll
    for (int n = 0; n < Lds::kStages; ++n) first.stage(n * kDepth, n * Lds::kStageBytes);
  }

  const int out = a.swiglu ? a.N / 2 : a.N;
  const int c0 = t.piece * (a.swiglu ? kTile / 2 : kTile) +
                 (a.swiglu ? wn * 32 + quarter * 8 : wn * 64 + quarter * 16);
  f32x4 sw[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j)
    sw[j] = *(const f32x4*)(s_scale + 256 + wn * 64 + j * 16 + quarter * 4);
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int r = wm * (MT * 16) + i * 16 + row;
    if (r >= t.rows) continue;
    const float sa = s_scale[r];
    uint16_t* y = a.y + (t.row + r) * out;
    float v[8];
    if (a.swiglu) {
      if (c0 >= out) continue;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int j = q / 4 * 2;
        v[q] = silu((float)acc[i][j][q & 3] * (sa * sw[j][q & 3])) *
               ((float)acc[i][j + 1][q & 3] * (sa * sw[j + 1][q & 3]));
      }
      st16(y + c0, pack8(v));
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (c0 + h * 8 >= out) continue;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int j = h * 2 + q / 4;
          v[q] = (float)acc[i][j][q & 3] * (sa * sw[j][q & 3]);
        }
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
void matmul_tile_kernel(MatmulArgs a, int pieces, int group) {
  using Lds = TileLds<HEIGHT>;
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[Lds::kBytes];
  int* s_end = reinterpret_cast<int*>(s_tile + Lds::kWindowAt);  // row tiles to a window's end
  int* s_start = s_end + MOE_MAX_EXPERTS;
  int* s_rows = s_start + MOE_MAX_EXPERTS;
  const int lane = threadIdx.x & (kWave - 1);
  if (threadIdx.x < kWave) {
    const int first = a.offset ? uniform((int)ld4(a.offset)) : 0;
    int before = 0;
    for (int e0 = 0; e0 < a.E; e0 += kWave) {
      int s = 0, m = (int)a.rows;
      if (a.offset) window_of(a, e0 + lane < a.E ? e0 + lane : a.E - 1, first, s, m);
      if (e0 + lane >= a.E) m = 0;
      const int end = before + scan_add(m / HEIGHT + (m % HEIGHT > 0));   // m may be 2^31 - 1
      s_end[e0 + lane] = end;                          // E is at most 16 times 64
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
  float scale = tile_scale(a, t, tid);
  {
    const TileLoads<HEIGHT> first(a, t, tid, s_tile);
#pragma unroll
    for (int n = 0; n < Lds::kStages; ++n) first.stage(n * kDepth, n * Lds::kStageBytes);
  }
  for (int n = 1;; ++n) {
    const Tile next = tile_at(n);
    // what follows from the thread's number is worked out anew for each tile:
    // kept over the loop it would not fit the registers
    asm volatile("" : "+v"(tid));
    if (HEIGHT > 128 && t.rows > 128)
      multiply_tile<HEIGHT, HEIGHT / 32>(a, t, next, tid, s_tile, n & 1, scale);
    else if (t.rows > 64) multiply_tile<HEIGHT, 4>(a, t, next, tid, s_tile, n & 1, scale);
    else multiply_tile<HEIGHT, 2>(a, t, next, tid, s_tile, n & 1, scale);
    if (next.rows == 0) return;
    t = next;
  }
}

// Few rows: ROWS rows of a window x 16 WC channels, bound by reading the
// weights: 512 rows, 32 experts, 7168 x 4096 with swiglu (946 MB) 149 us, 6.3 TB/s; without
// LDS between, whole rows of weights a wavefront, 262 us (half lines fetched twice).
// Two stages where there is room for three: 174 us.  4662 rows, 96 experts, 2064 x
// 1416 (304 MB): 82 us, the workgroups' beginnings and ends and a last round that
// fills a quarter of the GPU.  Eight wavefronts, WC along the channels and WK along the depth; a
// stage is 128 WK of the depth, STAGES - 1 stages are on their way while one is
// multiplied.  A wavefront loads its own weights (8 + 8 channels: with swiglu
// gate and up channels, so that a lane and its partner 32 further on hold both
// halves) and an eighth of the rows.  The sums of the WK wavefronts meet in
// LDS.
template <int ROWS, int WC, int WK, int STAGES>
__global__ __launch_bounds__(kTileThreads)
void matmul_stream_kernel(MatmulArgs a, int pieces) {
  static_assert(WC * WK == 8, "eight wavefronts");
  constexpr int MT = ROWS / 16;
  constexpr int kRowBytes = ROWS * kDepth * WK, kStage = kRowBytes + 16 * 1024;
  constexpr int kRowLoads = WK * ROWS / 64;            // of a wavefront and stage
  constexpr int kLoads = 2 + kRowLoads;
  static_assert(kRowLoads * 64 == WK * ROWS, "whole load instructions");
  // the stages, then the scales of the rows and of the channels (gate | up)
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[STAGES * kStage + (ROWS + 16 * WC) * 4];
  static_assert(STAGES * kStage >= 8 * MT * kWave * 16, "sums meet there");
  float* s_scale = reinterpret_cast<float*>(s_mem + STAGES * kStage);
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  // 32 neighbouring tiles (mostly one window's, which share rows) to an XCD
  const int b = blockIdx.x;
  const Tile t = find_tile(a, b / 256 * 256 + b % 8 * 32 + b / 8 % 32, ROWS, pieces);
  if (t.rows == 0) return;                             // the whole workgroup
  const int half = a.N / 2, out = a.swiglu ? half : a.N;
  const int wc = wave % WC, wk = wave / WC;
  const int step = a.swiglu ? 8 : 16;                  // output channels of a wavefront
  const int c0 = t.piece * WC * step + wc * step;

  const int lr = lane / 8, chunk = (lane & 7) ^ lr;
  const Rsrc ra = buffer_of(a.a + t.row * a.K, t.rows * a.K);
  const uint8_t* wbase = a.w + ((int64_t)t.expert * a.N + c0) * a.K;
  const int c1 = a.swiglu ? c0 : c0 + 8;               // channels come in whole eights
  const Rsrc rw0 = buffer_of(wbase, c0 < out ? 8 * a.K : 0);
  const Rsrc rw1 = buffer_of(wbase + (int64_t)(a.swiglu ? half : 8) * a.K, c1 < out ? 8 * a.K : 0);
  const uint32_t wo = (uint32_t)lr * (uint32_t)a.K + wk * kDepth + chunk * 16;
  auto load = [&](int k0, uint32_t at) {               // past the depth: zeros
    const uint32_t w = (uint32_t)k0 + wk * kDepth + chunk * 16 < (uint32_t)a.K ? wo + k0 : kOutside;
    uint8_t* to = s_mem + at + kRowBytes + wave * 2048;
    load_to_lds(rw0, w, (lds_u8*)to);
    load_to_lds(rw1, w, (lds_u8*)(to + 1024));
#pragma unroll
    for (int g = 0; g < kRowLoads; ++g) {              // eight rows of a 128 of the depth
      const int n = g * 8 + wave, r = n % (ROWS / 8) * 8 + lr;
      const uint32_t k = (uint32_t)k0 + n / (ROWS / 8) * kDepth + chunk * 16;
      load_to_lds(ra, k < (uint32_t)a.K ? (uint32_t)r * (uint32_t)a.K + k : kOutside,
                  (lds_u8*)(s_mem + at + n * 1024));
    }
  };
  float scale = 0.0f;
  if ((int)threadIdx.x < ROWS) {
    if ((int)threadIdx.x < t.rows) scale = a.a_scales[(t.row + threadIdx.x) * a.a_scale_pitch];
  } else if (threadIdx.x < ROWS + 16 * WC) {
    const int n = threadIdx.x - ROWS, c = t.piece * WC * step + n % (WC * step);
    if (c < out) scale = a.w_scales[(int64_t)t.expert * a.N + c + (n < WC * step ? 0 : half)];
  }
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) load(s * kDepth * WK, s * kStage);
  if (threadIdx.x < ROWS + 16 * WC) s_scale[threadIdx.x] = scale;

  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = row * kDepth + ((quarter ^ (row & 7)) * 16);
  i32x4 acc[MT] = {};
  auto multiply = [&](auto row_tiles) {
    constexpr int M = row_tiles.value;
    uint32_t at = 0, fill = (STAGES - 1) * kStage;     // stage to read, stage to fill
    for (int k0 = 0; k0 < a.K; k0 += kDepth * WK) {
      meet<(STAGES - 2) * kLoads>();                   // this stage is there, the last is read
      load(k0 + (STAGES - 1) * kDepth * WK, fill);
      i32x4 wv[2], av[2][M];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t p = at + (place ^ (h * 64));
        wv[h] = *(const i32x4*)(s_mem + kRowBytes + wave * 2048 + p);
#pragma unroll
        for (int i = 0; i < M; ++i)
          av[h][i] = *(const i32x4*)(s_mem + wk * (ROWS * kDepth) + i * 16 * kDepth + p);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < M; ++i)
          acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[h], av[h][i], acc[i], 0, 0, 0);
      at = at + kStage == STAGES * kStage ? 0 : at + kStage;
      fill = fill + kStage == STAGES * kStage ? 0 : fill + kStage;
    }
  };
  const int mt = (t.rows + 15) / 16;
  if (ROWS == 16 || mt == 1) multiply(std::integral_constant<int, 1>());
  else if (mt == 2) multiply(std::integral_constant<int, ROWS == 16 ? 1 : 2>());
  else multiply(std::integral_constant<int, MT>());
  meet<0>();                                           // loads past the end have landed

  i32x4* s_acc = reinterpret_cast<i32x4*>(s_mem);      // [wavefront][row tile][lane]
#pragma unroll
  for (int i = 0; i < MT; ++i) s_acc[(wave * MT + i) * kWave + lane] = acc[i];
  __syncthreads();
  // tile (w, i): channels of wavefront column w, rows 16 i..; a lane's four
  // sums are channels quarter * 4 .. + 3 of row `row`
  for (int n = wave; n < WC * mt; n += 8) {
    const int w = n % WC, i = n / WC;
    const int r = i * 16 + row;
    i32x4 sum = s_acc[(w * MT + i) * kWave + lane];
#pragma unroll
    for (int g = 1; g < WK; ++g) sum += s_acc[((g * WC + w) * MT + i) * kWave + lane];
    const int lc = w * step + (quarter * 4) % step, c = t.piece * WC * step + lc;
    const bool in = r < t.rows && c < out;
    const float sa = s_scale[r];
    const float* sw = s_scale + ROWS + lc + (a.swiglu && quarter > 1 ? WC * step : 0);
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = (float)sum[q] * (sa * sw[q]);
      if (a.swiglu) v[q] = silu(v[q]) * __shfl_xor(v[q], 32, kWave);   // gate lanes, up lanes
    }
    if (in && !(a.swiglu && quarter > 1))
      st4x2(a.y + (t.row + r) * out + c, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  }
}

template <int HEIGHT, int WAY>
hipError_t launch_tile(const MatmulArgs& a, int group, hipStream_t stream) {
  constexpr Way w = kWay[WAY];
  static_assert(w.rows == HEIGHT && w.channels == kTile, "the rule's tile");
  hipLaunchKernelGGL((matmul_tile_kernel<HEIGHT>), dim3(256), dim3(kTileThreads), 0, stream, a,
                     pieces_of(a, w), group);
  return hipGetLastError();
}

template <int ROWS, int WC, int WK, int STAGES, int WAY>
hipError_t launch_stream(const MatmulArgs& a, hipStream_t stream) {
  constexpr Way w = kWay[WAY];
  static_assert(w.rows == ROWS && w.channels == 16 * WC && w.depth == kDepth * WK,
                "the rule's tile");
  const int64_t groups = (tiles_of(a, w) + 255) / 256 * 256;
  hipLaunchKernelGGL((matmul_stream_kernel<ROWS, WC, WK, STAGES>), dim3((unsigned)groups),
                     dim3(kTileThreads), 0, stream, a, pieces_of(a, w));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul(const MatmulArgs& a, hipStream_t stream) {
  switch (choose_way(a)) {
    // six row tiles together: of 2, 4, 5, 6 and 8 the best or near it (32768 x
    // 2048 x 7168 over 32 experts 528 / 522 / 512 / 510 / 509 us, 16384 x 8192 x 8192
    // 846 / 832 / 815 / 811 / 835); of 128 rows six or twelve make no difference
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
