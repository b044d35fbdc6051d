// Routing: the k experts of each token with their weights, and the gradient
// of the weights with respect to the logits.
//
// One token takes LANES (16 or 64) neighbouring lanes of a wavefront, each with
// VPL neighbouring experts in registers; the k winners are found one after
// another as the largest key of the lanes, equal keys by the lowest index.
// Keys are the floats' bit patterns made to order as unsigned integers, so a
// maximum over lanes is one DPP instruction per step.

#include <math.h>

#include <type_traits>

#include "layer.h"

namespace moe {
namespace {

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
#pragma unroll
        for (int i = 0; i + 1 < VPL; i += 2) {
          const uint32_t w = ld4(p + i);
          x[i] = bf16_lo(w);
          x[i + 1] = bf16_hi(w);
        }
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

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + expf(-x)); }

// Largest of the lanes' values; -inf where there is none.  NaN is passed over.
template <int LANES, int VPL>
__device__ __forceinline__ float row_max(const float (&x)[VPL]) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < VPL; ++i) m = fmaxf(m, x[i]);
  const uint32_t key = reduce_max<LANES>(order_key(m));
  return __uint_as_float(key ^ ((uint32_t)((int32_t)~key >> 31) | 0x80000000u));
}

template <int HALF, int N>
__device__ __forceinline__ void add_upper(float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < HALF; ++i) v[i] += v[i + HALF];
}

// Sum of the token's terms: upper half onto lower half until one is left.
template <int LANES, int VPL>
__device__ __forceinline__ float fold(const float (&x)[VPL]) {
#pragma clang fp contract(off)
  float v[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) v[i] = reduce_sum<LANES>(x[i]);
  if constexpr (VPL >= 16) add_upper<8>(v);
  if constexpr (VPL >= 8) add_upper<4>(v);
  if constexpr (VPL >= 4) add_upper<2>(v);
  if constexpr (VPL >= 2) add_upper<1>(v);
  return v[0];
}

// LDS is used by one wavefront at a time and its accesses complete in order:
// only the compiler has to keep them so.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Route token t: lane `sub` of its LANES, `tok` its place in the wavefront, `mine`
// the token's keys in LDS.  Every lane of the wavefront takes part.
template <int LANES, int VPL>
__device__ __forceinline__ void route_token(const RouteArgs& a, int vec, int64_t t, int sub, int tok,
                                            float* mine) {
#pragma clang fp contract(off)
  const bool in = t < a.tokens;
  const bool live = in && (!a.token_mask || a.token_mask[t]);
  const int e0 = sub * VPL;
  float x[VPL];
  if (live) {
    load_logits<VPL>(a.logits, a.f32, t * a.pitch, e0, a.E, vec, x);
  } else {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
  }

  // scores, where they order the experts or weigh them as they are
  const bool by_score = a.bias || (a.groups > 1 && a.group_top > 1);
  float m = 0.0f, total = 1.0f;
  const bool plain = !a.sigmoid && !a.renorm;
  float s[VPL];
  if (by_score || plain) {
    if (a.sigmoid) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) s[i] = sigmoid(x[i]);
    } else {
      m = row_max<LANES, VPL>(x);
#pragma unroll
      for (int i = 0; i < VPL; ++i) s[i] = exp_term(x[i], m);
      total = fold<LANES, VPL>(s);
      if (!(total > 0.0f)) total = 1.0f;
    }
  }
  float kf[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    kf[i] = x[i];
    if (by_score) {
      float v = a.sigmoid ? s[i] : s[i] / total;
      if (a.bias && e0 + i < a.E) v += a.bias[e0 + i];
      kf[i] = x[i] > -INFINITY ? v : -INFINITY;
    }
    if (!(kf[i] > -INFINITY)) kf[i] = -INFINITY;   // NaN too
  }

  if (a.groups > 1) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) mine[e0 + i] = kf[i];
    wave_order();
    const int size = a.E / a.groups;
    float best = -INFINITY, second = -INFINITY;
    if (sub < a.groups) {
      for (int i = 0; i < size; ++i) {
        const float v = mine[sub * size + i];
        second = fmaxf(second, fminf(best, v));
        best = fmaxf(best, v);
      }
      if (a.group_top > 1 && second > -INFINITY) best += second;
    }
    wave_order();
    if (sub < a.groups) mine[sub] = best;
    wave_order();
    int rank = 0;
    for (int g = 0; g < a.groups; ++g) {
      const float v = mine[g];
      rank += v > best || (v == best && g < sub);
    }
    const uint64_t kept =
        __ballot(sub < a.groups && best > -INFINITY && rank < a.top_groups) >> (tok * LANES);
    int g = e0 / size, r = e0 - g * size;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      if (g >= a.groups || !((kept >> g) & 1)) kf[i] = -INFINITY;
      if (++r == size) {
        r = 0;
        ++g;
      }
    }
  }

  uint32_t key[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i) key[i] = kf[i] > -INFINITY ? order_key(kf[i]) : 0u;
  int won = -1;                                   // slot `sub`'s expert
  for (int j = 0; j < a.k; ++j) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) top = umax(top, key[i]);
    top = reduce_max<LANES>(top);
    uint32_t at = 0xFFFFu;
#pragma unroll
    for (int i = VPL - 1; i >= 0; --i) at = key[i] == top ? (uint32_t)(e0 + i) : at;
    at = reduce_min<LANES>(at);
#pragma unroll
    for (int i = 0; i < VPL; ++i) key[i] = at == (uint32_t)(e0 + i) ? 0u : key[i];
    if (sub == j && top) won = (int)at;
  }

  // weights: lane j of the token has slot j
  float w = 0.0f;
  const bool slot = in && sub < a.k;
  float xw = -INFINITY;
  if (won >= 0) xw = logit_at(a.logits, a.f32, t * a.pitch + won);
  if (a.sigmoid) {
    w = won >= 0 ? sigmoid(xw) : 0.0f;
  } else if (plain) {
    w = exp_term(xw, m) / total;
  } else {
    const float one[1] = {xw};
    w = exp_term(xw, row_max<LANES, 1>(one));
  }
  if (a.renorm) {
    const float sum = reduce_sum<LANES>(w);
    w = sum > 0.0f ? w / sum : 0.0f;
  }
  if (slot) {
    a.topk_idx[t * a.k + sub] = won;
    a.topk_w[t * a.k + sub] = w * a.scale;
  }
}

template <int LANES, int VPL>
__global__ __launch_bounds__(kBlock) void route_kernel(RouteArgs a, int vec) {
  constexpr int kTokens = kWave / LANES;         // of a wavefront
  __shared__ float s_key[kWavesPerBlock][kTokens][LANES * VPL];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWavesPerBlock + wave) * kTokens; t0 < a.tokens;
       t0 += (int64_t)gridDim.x * kWavesPerBlock * kTokens)
    route_token<LANES, VPL>(a, vec, t0 + tok, sub, tok, s_key[wave][tok]);
}

// The dense part of a softmax's gradient reaches every expert, the others only
// the chosen ones; either way a token's row is put together in LDS (one
// value per slot) and written whole.
template <int LANES, int VPL>
__device__ __forceinline__ void route_token_backward(const RouteGradArgs& a, int vec, int64_t t,
                                                     int sub, float* row) {
  const bool in = t < a.tokens;
  const int e0 = sub * VPL;
#pragma unroll
  for (int i = 0; i < VPL; ++i) row[e0 + i] = 0.0f;

  int e = -1;
  float g = 0.0f, xe = -INFINITY;
  if (in && sub < a.k) {
    e = a.topk_idx[t * a.k + sub];
    if ((uint32_t)e >= (uint32_t)a.E) e = -1;
    if (e >= 0) {
      g = a.grad_w[t * a.k + sub] * a.scale;
      xe = logit_at(a.logits, a.f32, t * a.pitch + e);
      if (!(xe > -INFINITY)) {                     // never chosen by moe_route
        g = 0.0f;
        xe = -INFINITY;
      }
    }
  }

  const bool dense = !a.sigmoid && !a.renorm;
  float x[VPL], m = 0.0f, inv = 0.0f, q, d;
  if (dense) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
    if (in) load_logits<VPL>(a.logits, a.f32, t * a.pitch, e0, a.E, vec, x);
    m = row_max<LANES, VPL>(x);
    float local = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      x[i] = exp_term(x[i], m);
      local += x[i];
    }
    const float total = reduce_sum<LANES>(local);
    inv = total > 0.0f ? 1.0f / total : 0.0f;
    q = exp_term(xe, m) * inv;
    d = g;
  } else if (a.sigmoid) {
    const float s = e >= 0 ? sigmoid(xe) : 0.0f;
    q = s;
    if (a.renorm) {
      const float sum = reduce_sum<LANES>(s);
      q = sum > 0.0f ? s / sum : 0.0f;
    }
    d = q * (1.0f - s);
  } else {
    const float one[1] = {xe};
    q = exp_term(xe, row_max<LANES, 1>(one));
    const float sum = reduce_sum<LANES>(q);
    q = sum > 0.0f ? q / sum : 0.0f;
    d = q;
  }
  const float dot = dense || a.renorm ? reduce_sum<LANES>(g * q) : 0.0f;
  wave_order();
  if (e >= 0) row[e] = dense ? d : d * (g - dot);
  wave_order();
  if (!in) return;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    if (dense) x[i] = x[i] * inv * (row[e0 + i] - dot);
    else x[i] = row[e0 + i];
  }
  const int64_t at = t * a.E + e0;
  if constexpr (VPL >= 4) if (vec) {
    if (e0 >= a.E) return;
    if (a.f32) {
      float* p = static_cast<float*>(a.grad_logits) + at;
#pragma unroll
      for (int i = 0; i + 3 < VPL; i += 4)
        st16(p + i, u32x4{__float_as_uint(x[i]), __float_as_uint(x[i + 1]),
                          __float_as_uint(x[i + 2]), __float_as_uint(x[i + 3])});
    } else {
      uint16_t* p = static_cast<uint16_t*>(a.grad_logits) + at;
#pragma unroll
      for (int i = 0; i + 1 < VPL; i += 2) st4(p + i, pack_bf16x2(x[i], x[i + 1]));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    if (e0 + i >= a.E) {
    } else if (a.f32) {
      static_cast<float*>(a.grad_logits)[at + i] = x[i];
    } else {
      static_cast<uint16_t*>(a.grad_logits)[at + i] = (uint16_t)pack_bf16x2(x[i], 0.0f);
    }
  }
}

template <int LANES, int VPL>
__global__ __launch_bounds__(kBlock) void route_backward_kernel(RouteGradArgs a, int vec) {
  constexpr int kTokens = kWave / LANES;         // of a wavefront
  __shared__ float s_row[kWavesPerBlock][kTokens][LANES * VPL];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWavesPerBlock + wave) * kTokens; t0 < a.tokens;
       t0 += (int64_t)gridDim.x * kWavesPerBlock * kTokens) {
    route_token_backward<LANES, VPL>(a, vec, t0 + tok, sub, s_row[wave][tok]);
    wave_order();
  }
}

// Whether every lane's piece of VPL logits is whole and aligned to the vectors
// it is read (and written) in.
bool vector_rows(const void* p, const void* q, int64_t pitch, int E, int vpl, int f32) {
  const int size = f32 ? 4 : 2;
  const int bytes = vpl * size < 16 ? vpl * size : 16;
  return vpl >= 4 && E % vpl == 0 && pitch * size % bytes == 0 && E * size % bytes == 0 &&
         (uintptr_t)p % bytes == 0 && (uintptr_t)q % bytes == 0;
}

template <typename F>
hipError_t by_width(int E, int k, int groups, int64_t tokens, F&& launch) {
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

unsigned route_blocks(int64_t tokens, int lanes) {
  const int64_t per = (int64_t)kWavesPerBlock * (kWave / lanes);
  const int64_t blocks = (tokens + per - 1) / per;
  return (unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t stream) {
  return by_width(a.E, a.k, a.groups, a.tokens, [&](auto lanes, auto vpl) {
    const int vec = vector_rows(a.logits, nullptr, a.pitch, a.E, vpl.value, a.f32);
    hipLaunchKernelGGL((route_kernel<lanes.value, vpl.value>),
                       dim3(route_blocks(a.tokens, lanes.value)), dim3(kBlock), 0, stream, a, vec);
    return hipGetLastError();
  });
}

hipError_t launch_route_backward(const RouteGradArgs& a, hipStream_t stream) {
  return by_width(a.E, a.k, 1, a.tokens, [&](auto lanes, auto vpl) {
    const int vec = vector_rows(a.logits, a.grad_logits, a.pitch, a.E, vpl.value, a.f32);
    hipLaunchKernelGGL((route_backward_kernel<lanes.value, vpl.value>),
                       dim3(route_blocks(a.tokens, lanes.value)), dim3(kBlock), 0, stream, a, vec);
    return hipGetLastError();
  });
}

}  // namespace moe
