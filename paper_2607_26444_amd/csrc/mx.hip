// Quantisation of bf16 rows to microscaled 4-bit floats.
//
// Of 32 neighbouring values v with a = max |v|: scale 2^e with the e that puts a into
// [3.5, 7) units, code = v / 2^e to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their
// negatives, ties to the even code.  Below 7 units the largest value rounds to 6 at most, so
// that none is cut off by more than half a step; a power of two less for a in [7, 8), which
// cuts off up to 2 of 8 units, has a 3% larger error over normal values (0.115 of their root
// mean square for 0.112), one more from 6 on as well.
//
// Bound by memory: 16384 rows of 7168 48.8 us (6.1 TB/s), with values 79 (6.7 TB/s).  Rows of less
// than a wavefront's 512 values leave lanes idle: as many values in rows of 512 take 58 us, of 256
// 105, of 64 387.

#include "layer.h"

namespace moe {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Maximum over groups of four neighbouring lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
  x = umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));
  return umax(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));
}

// Scale byte of a block whose largest magnitude has the bf16 pattern `a`: the exponent, one
// more from 1.75 times a power of two on, less 2.  255 marks infinity or NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t a) {
  if (a >= 0x7F80u) return 255u;
  if (a == 0u) return 127u;
  const uint32_t e = (a + 0x20u) >> 7;
  return e > 2u ? e - 2u : 0u;
}

__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}

// A wavefront takes NV times 512 neighbouring values of a row, eight to a lane: four lanes
// have a block, sixteen a word of scales.
template <int NV>
__global__ __launch_bounds__(kBlock) void quantize_mx_kernel(MxQuantArgs a, int pieces) {
  const int lane = threadIdx.x & (kWave - 1);
  const int64_t units = a.rows * pieces;
  for (int64_t u = (int64_t)blockIdx.x * kWavesPerBlock + uniform(threadIdx.x / kWave); u < units;
       u += (int64_t)gridDim.x * kWavesPerBlock) {
    const int64_t r = u / pieces;
    const int at = (int)(u - r * pieces) * NV * kWave + lane;   // in vectors of eight
    if (a.row_src && (int32_t)ld4(a.row_src + r) < 0) continue;
    const uint8_t* row = a.x + r * a.x_pitch;
    u32x4 x[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * kWave;
      x[i] = v < a.H / 8 ? ld16_stream(row + (int64_t)v * 16) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * kWave;
      uint32_t top = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        top = umax(top, umax(x[i][j] & 0x7FFFu, x[i][j] >> 16 & 0x7FFFu));
      const bool in = v < a.H / 8;
      const uint32_t byte = scale_byte(quad_max(top));
      const float scale = scale_value(byte == 255u ? 127u : byte);
      const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
      uint32_t codes = 0u;
#define MOE_CODE(J)                                             \
  codes = (uint32_t)__builtin_amdgcn_cvt_scalef32_pk_fp4_bf16( \
      codes, __builtin_bit_cast(bf16x2, w[J]), scale, J);
      MOE_CODE(0) MOE_CODE(1) MOE_CODE(2) MOE_CODE(3)
#undef MOE_CODE
      // scales of 16 lanes' four blocks into one word; blocks past the row are 0
      uint32_t word = in ? byte << (lane >> 2 & 3) * 8 : 0u;
      word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x124, 0xf, 0xf, true);   // row_ror
      word |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)word, 0x128, 0xf, 0xf, true);
      if (!in) continue;
      st4(a.q + r * a.q_pitch + (int64_t)v * 4, codes);
      if ((lane & 15) == 0) st4(a.scales + r * a.scale_pitch + (v >> 4) * 4, word);
      if (a.values) {
        u32x4 y;
#define MOE_VALUE(J) \
  y[J] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, J));
        MOE_VALUE(0) MOE_VALUE(1) MOE_VALUE(2) MOE_VALUE(3)
#undef MOE_VALUE
        if (byte == 255u) y = u32x4{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};
        st16_stream(a.values + (r * a.H + (int64_t)v * 8) * 2, y);
      }
    }
  }
}

}  // namespace

hipError_t launch_quantize_mx(const MxQuantArgs& a, hipStream_t stream) {
  constexpr int NV = 2;
  const int pieces = (a.H / 8 + NV * kWave - 1) / (NV * kWave);
  const int64_t want = (a.rows * pieces + kWavesPerBlock - 1) / kWavesPerBlock;
  hipLaunchKernelGGL((quantize_mx_kernel<NV>), dim3((unsigned)(want < kMaxGrid ? want : kMaxGrid)),
                     dim3(kBlock), 0, stream, a, pieces);
  return hipGetLastError();
}

}  // namespace moe
