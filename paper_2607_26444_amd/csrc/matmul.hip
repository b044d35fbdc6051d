// The experts' products on 8-bit integers.
//
// A workgroup takes ROWS rows of one expert's window and CHANNELS of its channels; its
// four wavefronts take every fourth piece of the depth and add their int32
// sums in LDS (integer sums: exact in any order).  The operands go from
// memory into the matrix instructions' registers: weights are read once by one
// workgroup, rows again by each workgroup along the channels, from the caches.

#include "layer.h"

namespace moe {
namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kOutside = 0x7FFFFFF0u;   // past every buffer's range: reads zeros

// One window of rows: expert and first row of tile `tile` of `size` rows, and
// the rows left from there; rows 0: no such tile.
struct Tile {
  int expert;
  int64_t row;
  int rows;
};

__device__ __forceinline__ Tile find_tile(const MatmulArgs& a, int64_t tile, int size) {
  if (!a.offset) {
    const int64_t row = tile * size, left = a.rows - row;
    return {0, row, left < 0 ? 0 : left < size ? (int)left : size};
  }
  const int lane = threadIdx.x & (kWave - 1);
  const int first = (int)ld4(a.offset);
  int64_t before = 0;
  for (int e0 = 0; e0 < a.E; e0 += kWave) {
    const int e = e0 + lane;
    int64_t start = 0, n = 0;
    if (e < a.E) {
      const int o = (int)ld4(a.offset + e);
      start = (int64_t)o - first;
      n = a.count ? (int64_t)(int)ld4(a.count + e) : (int64_t)(int)ld4(a.offset + e + 1) - o;
      if (start < 0 || start > a.rows) n = 0;
      if (n > a.rows - start) n = a.rows - start;
      if (n < 0) n = 0;
    }
    const int tiles = (int)((n + size - 1) / size);
    int sum = tiles;                                   // inclusive over the lanes
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
      const int o = __shfl_up(sum, d, kWave);
      if (lane >= d) sum += o;
    }
    const uint64_t hit = __ballot(before + sum > tile);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      const int64_t at = tile - before - (__shfl(sum, l, kWave) - __shfl(tiles, l, kWave));
      const int64_t s = __shfl(start, l, kWave), m = __shfl(n, l, kWave);
      const int64_t left = m - at * size;
      return {e0 + l, s + at * size, left < size ? (int)left : size};
    }
    before += __shfl(sum, kWave - 1, kWave);
  }
  return {0, 0, 0};
}

__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

// MT x 16 rows, NT x 16 channels.  With swiglu the channel tiles alternate
// between gate and up, so that a lane holds both halves of its outputs.
template <int MT, int NT>
__global__ __launch_bounds__(kBlock) void matmul_split_kernel(MatmulArgs a, int64_t tiles,
                                                                int pieces) {
  __shared__ i32x4 s_acc[kWavesPerBlock][MT * NT][kWave];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int row = lane & 15, piece = lane / 16;
  const int half = a.N / 2;
  for (int64_t id = blockIdx.x; id < tiles * pieces; id += gridDim.x) {
  const Tile t = find_tile(a, id / pieces, MT * 16);
  if (t.rows == 0) continue;                           // the whole workgroup
  const int c0 = (int)(id % pieces) * (a.swiglu ? NT * 8 : NT * 16);   // first (gate) channel

  // A matrix instruction takes 64 of the depth, 16 bytes per lane.  Lanes read
  // 32 neighbouring bytes for two of them, so that four lanes cover a line of
  // a row; both operands are permuted alike.
  const Rsrc ra = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(a.a + t.row * a.K), (short)0, t.rows * a.K, kRsrcWord3);
  uint32_t ao[MT], wo[NT];
#pragma unroll
  for (int i = 0; i < MT; ++i) ao[i] = (uint32_t)(i * 16 + row) * (uint32_t)a.K + piece * 32;
  const uint8_t* wbase = a.w + (int64_t)t.expert * a.N * a.K;
  Rsrc rw[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    int c = a.swiglu ? c0 + (j / 2) * 16 + (j & 1) * half : c0 + j * 16;
    int n = (a.swiglu ? (j & 1 ? a.N : half) : a.N) - c;       // channels that are there
    if (n < 0) c = 0, n = 0;
    rw[j] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(wbase + (int64_t)c * a.K),
                                              (short)0, (n < 16 ? n : 16) * a.K, kRsrcWord3);
    wo[j] = (uint32_t)row * (uint32_t)a.K + piece * 32;
  }

  i32x4 acc[MT][NT] = {};
  for (int k0 = wave * 128; k0 < a.K; k0 += kWavesPerBlock * 128) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = k0 + h * 16;
      const bool in = k + piece * 32 < a.K;            // past the depth: zeros
      i32x4 av[MT], wv[NT];
#pragma unroll
      for (int j = 0; j < NT; ++j)
        wv[j] = (i32x4)__builtin_amdgcn_raw_buffer_load_b128(rw[j], in ? wo[j] + k : kOutside, 0, 0);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        av[i] = (i32x4)__builtin_amdgcn_raw_buffer_load_b128(ra, in ? ao[i] + k : kOutside, 0, 0);
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[j], av[i], acc[i][j], 0, 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) s_acc[wave][i * NT + j][lane] = acc[i][j];
  __syncthreads();

  // A lane's four sums of a tile: channels piece * 4 .. + 3 of row `row`.
  const int step = a.swiglu ? 2 : 1;
  const int out = a.swiglu ? half : a.N;
  for (int i = wave * step; i < MT * NT; i += kWavesPerBlock * step) {
    const int m = i / NT, j = i % NT;
    const int r = m * 16 + row;
    const int c = c0 + (a.swiglu ? j / 2 : j) * 16 + piece * 4;
    if (r >= t.rows || c >= out) continue;
    const float sa = a.a_scales[(t.row + r) * a.a_scale_pitch];
    const float* sw = a.w_scales + (int64_t)t.expert * a.N + c;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      int sum = 0;
#pragma unroll
      for (int p = 0; p < kWavesPerBlock; ++p) sum += s_acc[p][i][lane][q];
      v[q] = (float)sum * (sa * sw[q]);
      if (a.swiglu) {
        int up = 0;
#pragma unroll
        for (int p = 0; p < kWavesPerBlock; ++p) up += s_acc[p][i + 1][lane][q];
        v[q] = silu(v[q]) * ((float)up * (sa * sw[half + q]));
      }
    }
    uint16_t* y = a.y + (t.row + r) * out + c;
    st4(y, pack_bf16x2(v[0], v[1]));
    st4(y + 2, pack_bf16x2(v[2], v[3]));
  }
  __syncthreads();                                     // s_acc is free again
  }
}

}  // namespace

hipError_t launch_matmul(const MatmulArgs& a, hipStream_t stream) {
  constexpr int MT = 2, NT = 4;
  const int64_t tiles = (a.rows + MT * 16 - 1) / (MT * 16) + (a.offset ? a.E : 0);
  const int per = a.swiglu ? NT * 8 : NT * 16, out = a.swiglu ? a.N / 2 : a.N;
  const int pieces = (out + per - 1) / per;
  const int64_t blocks = tiles * pieces < kMaxGrid ? tiles * pieces : kMaxGrid;
  hipLaunchKernelGGL((matmul_split_kernel<MT, NT>), dim3((unsigned)blocks), dim3(kBlock), 0,
                     stream, a, tiles, pieces);
  return hipGetLastError();
}

}  // namespace moe
