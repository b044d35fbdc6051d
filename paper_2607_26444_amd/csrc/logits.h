// Rows of router logits in the lanes of a wavefront: their loading, scores and
// reductions, and the lanes that a row takes.  For the routing (route.hip) and the
// balance loss (balance.hip).
//
// One token takes LANES (16 or 64) neighbouring lanes, each with VPL of its experts.
#pragma once

#include <math.h>

#include <type_traits>

#include "layer.h"

namespace moe {

// Float -> unsigned that orders alike; 0 is below every float (it marks an
// expert that cannot be chosen).  The sign of zero does not order.
__device__ __forceinline__ uint32_t order_key(float f) {
  const uint32_t u = __float_as_uint(f + 0.0f);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float bf16_at(const uint16_t* p) {
  const __attribute__((address_space(1))) uint16_t* g =
      (const __attribute__((address_space(1))) uint16_t*)(uintptr_t)p;
  return __uint_as_float((uint32_t)*g << 16);
}

__device__ __forceinline__ float logit_at(const void* logits, bool f32, int64_t i) {
  return f32 ? __uint_as_float(ld4(static_cast<const float*>(logits) + i))
             : bf16_at(static_cast<const uint16_t*>(logits) + i);
}

// A lane's VPL neighbouring logits, -inf past the last expert.  `vec`: each
// lane's piece is whole and aligned, so that it is read as vectors.
template <int VPL>
__device__ __forceinline__ void load_logits(const void* logits, bool f32, int64_t at, int e0,
                                            int E, bool vec, float (&x)[VPL]) {
#pragma unroll
  for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
  if constexpr (VPL >= 4) if (vec) {
    if (e0 >= E) return;
    if (f32) {
      const float* p = static_cast<const float*>(logits) + at + e0;
#pragma unroll
      for (int i = 0; i + 3 < VPL; i += 4) {
        const u32x4 v = ld16(p + i);
        x[i] = __uint_as_float(v.x);
        x[i + 1] = __uint_as_float(v.y);
        x[i + 2] = __uint_as_float(v.z);
        x[i + 3] = __uint_as_float(v.w);
      }
    } else {
      const uint16_t* p = static_cast<const uint16_t*>(logits) + at + e0;
      if constexpr (VPL >= 8) {
#pragma unroll
        for (int i = 0; i + 7 < VPL; i += 8) {
          const u32x4 v = ld16(p + i);
          const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            x[i + 2 * j] = bf16_lo(w[j]);
            x[i + 2 * j + 1] = bf16_hi(w[j]);
          }
        }
      } else {
        const u32x2 w = ld8(p);                       // VPL is 4
        x[0] = bf16_lo(w.x);
        x[1] = bf16_hi(w.x);
        x[2] = bf16_lo(w.y);
        x[3] = bf16_hi(w.y);
      }
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i)
    if (e0 + i < E) x[i] = logit_at(logits, f32, at + e0 + i);
}

// exp(x - m), 0 for an expert that is not eligible (-inf or NaN logit); m is
// the largest eligible logit, whose own term is 1 also where it is infinite.
__device__ __forceinline__ float exp_term(float x, float m) {
  if (!(x > -INFINITY)) return 0.0f;
  return x == m ? 1.0f : expf(x - m);
}

// 1 / x for x >= 1 as an exact division rounds it: one Newton step on the
// hardware's reciprocal (1 ulp) is the correctly rounded one for every
// significand; a quarter of a division's instructions.  Infinity gives 0.
__device__ __forceinline__ float reciprocal(float x) {
  const float r = __builtin_amdgcn_rcpf(x);
  const float y = __builtin_fmaf(__builtin_fmaf(-x, r, 1.0f), r, r);
  return x < 0x1p126f ? y : 1.0f / x;              // beyond: the result is subnormal
}

__device__ __forceinline__ float sigmoid(float x) { return reciprocal(1.0f + expf(-x)); }

// Largest of the lanes' values; -inf where there is none.  NaN is passed over.
template <int LANES, int VPL>
__device__ __forceinline__ float row_max(const float (&x)[VPL]) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < VPL; ++i) m = fmaxf(m, x[i]);
  const uint32_t key = reduce_max<LANES>(order_key(m));
  return __uint_as_float(key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u));
}

// Expert of a lane's i-th value in the gradient: fours of neighbours, dealt
// to the lanes in turn, so that 16 lanes read and write 64 neighbours at once (with
// a lane's values all neighbours, inputs in the cache: 16384 x 256 float32 9.1 us, so 5.8;
// 32768 x 128 bf16 7.2, so 5.8).
template <int LANES, int VPL>
__device__ __forceinline__ int dealt(int sub, int i) {
  return VPL >= 4 ? (i / 4 * LANES + sub) * 4 + (i & 3) : sub * VPL + i;
}

// Whether every lane's piece of VPL logits is whole and aligned to the vectors
// it is read (and written) in.
inline bool vector_rows(const void* p, const void* q, int64_t pitch, int E, int vpl, int f32) {
  const int size = f32 ? 4 : 2;
  const int bytes = vpl * size < 16 ? vpl * size : 16;
  return vpl >= 4 && E % vpl == 0 && pitch * size % bytes == 0 && E * size % bytes == 0 &&
         (uintptr_t)p % bytes == 0 && (uintptr_t)q % bytes == 0;
}

template <typename F>
hipError_t by_width(int E, int k, int groups, F&& launch) {
  // 16 lanes per token (four tokens per wavefront) up to 256 experts where
  // slots and groups fit them, else the whole wavefront
  if (E <= 256 && k <= 16 && groups <= 16) {
    if (E <= 16) return launch(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (E <= 32) return launch(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
    if (E <= 64) return launch(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
    if (E <= 128) return launch(std::integral_constant<int, 16>(), std::integral_constant<int, 8>());
    return launch(std::integral_constant<int, 16>(), std::integral_constant<int, 16>());
  }
  if (E <= 64) return launch(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
  if (E <= 128) return launch(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
  if (E <= 256) return launch(std::integral_constant<int, 64>(), std::integral_constant<int, 4>());
  if (E <= 512) return launch(std::integral_constant<int, 64>(), std::integral_constant<int, 8>());
  return launch(std::integral_constant<int, 64>(), std::integral_constant<int, 16>());
}

}  // namespace moe
