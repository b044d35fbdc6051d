// The experts' products on microscaled 4-bit floats:
//   v[r,n] = sum_k a[r,k] w[e,n,k] with the values that codes and scales stand for,
//   y = bf16(v), or with swiglu y[r,i] = bf16(silu(v[r,i]) v[r,N/2+i]).
// Scaled matrix instructions multiply 16 x 16 x 128 codes, a scale byte for each 32 of them,
// and add in float32; the result is rounded to bf16 once.

#include "matmul_tile.h"

namespace moe {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// Both operands are 4-bit floats (format 4), 16 bytes to a lane.
template <int A, int B>
__device__ __forceinline__ f32x4 multiply_mx(i32x4 w, i32x4 a, f32x4 c, int sw, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
      i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0}, c, 4, 4,
      A, sw, B, sa);
}

// 16 rows x 16 output channels to a wavefront, operands straight from memory.
__global__ __launch_bounds__(kBlock) void matmul_mx_kernel(MatmulMxArgs a, int pieces) {
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const Tile t = find_tile(a, blockIdx.x, 16, pieces);
  if (t.rows == 0) return;
  const int half = a.N / 2, out = a.swiglu ? half : a.N, values = a.K * 2;
  const int c0 = t.piece * 64 + wave * 16;
  const int row = lane & 15, quarter = lane / 16;
  const int channel = c0 + row, pitch = mx_scale_bytes(values);
  const bool has_row = row < t.rows, has_channel = channel < out;
  const uint8_t* pa = a.a + (t.row + row) * a.a_pitch;
  const uint8_t* sa = a.a_scales + (t.row + row) * a.a_scale_pitch;
  const int64_t w0 = (int64_t)t.expert * a.N + channel;
  f32x4 acc[2] = {};
  for (int k0 = 0; k0 < values; k0 += 128) {
    const int k = k0 + quarter * 32;
    const bool in = k < values;
    i32x4 x = {}, w[2] = {};
    int sx = 0, sw[2] = {};
    if (in && has_row) {
      x = __builtin_bit_cast(i32x4, ld16(pa + k / 2));
      sx = sa[k / 32];
    }
    for (int h = 0; h < (a.swiglu ? 2 : 1); ++h)
      if (in && has_channel) {
        const int64_t n = w0 + h * half;
        w[h] = __builtin_bit_cast(i32x4, ld16(a.w + n * a.K + k / 2));
        sw[h] = a.w_scales[n * pitch + k / 32];
      }
    acc[0] = multiply_mx<0, 0>(w[0], x, acc[0], sw[0], sx);
    if (a.swiglu) acc[1] = multiply_mx<0, 0>(w[1], x, acc[1], sw[1], sx);
  }
  // a lane's four sums are channels quarter * 4 .. + 3 of row `row`
  const int c = c0 + quarter * 4;
  if (!has_row || c >= out) return;
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = a.swiglu ? silu(acc[0][q]) * acc[1][q] : acc[0][q];
  st4x2(a.y + (t.row + row) * out + c, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
}

}  // namespace

hipError_t launch_matmul_mx(const MatmulMxArgs& a, hipStream_t stream) {
  const int out = a.swiglu ? a.N / 2 : a.N, pieces = (out + 63) / 64;
  const int64_t tiles = row_tiles(a, 16) * pieces;
  if (tiles >= (1ll << 32) / kBlock) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(matmul_mx_kernel, dim3((unsigned)tiles), dim3(kBlock), 0, stream, a, pieces);
  return hipGetLastError();
}

}  // namespace moe
