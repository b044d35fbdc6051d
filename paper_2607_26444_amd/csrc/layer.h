// Launchers of the layer around the exchange: routing (route.hip), RMS norm
// and quantisation (norm.hip), the experts' products (matmul.hip).
// api_layer.hip validates arguments and calls them.
#pragma once

#include "moe_internal.h"

namespace moe {

// Workgroups of one launch; larger batches are strided over.
constexpr int64_t kMaxGrid = 1 << 20;

struct RouteArgs {
  const void* logits;
  int64_t pitch;        // elements
  int64_t tokens;
  int32_t f32;          // logits are float32, else bf16
  int32_t k;
  int32_t E;
  int32_t sigmoid;
  const float* bias;
  int32_t groups;
  int32_t top_groups;
  int32_t group_top;
  int32_t renorm;
  float scale;
  const uint8_t* token_mask;
  int32_t* topk_idx;
  float* topk_w;
};

hipError_t launch_route(const RouteArgs& a, hipStream_t stream);

struct RouteGradArgs {
  const void* logits;
  int64_t pitch;
  int64_t tokens;
  int32_t f32;
  int32_t k;
  int32_t E;
  int32_t sigmoid;
  int32_t renorm;
  float scale;
  const int32_t* topk_idx;
  const float* grad_w;
  void* grad_logits;
};

hipError_t launch_route_backward(const RouteGradArgs& a, hipStream_t stream);

// 8-bit output of a row kernel.
enum QuantKind : int32_t { kQuantNone = 0, kQuantFp8 = 1, kQuantInt8 = 2 };

struct NormArgs {
  const uint8_t* x;          // bf16
  int64_t x_pitch;           // bytes
  const uint8_t* residual;   // or null
  int64_t residual_pitch;    // bytes
  int32_t residual_f32;
  int32_t weight_f32;
  const uint8_t* weight;     // null: no norm (quantisation alone)
  float eps;
  int64_t rows;
  int32_t H;
  const int32_t* row_src;    // rows with a negative entry are skipped; or null
  uint8_t* sum_out;
  uint8_t* y;
  int32_t stream_y;          // y is larger than the caches keep
  QuantKind quant;
  uint8_t* q;
  float* q_scales;
  int32_t scale_cols;
  float* rstd;
};

hipError_t launch_norm(const NormArgs& a, hipStream_t stream);

struct NormGradArgs {
  const uint8_t* grad_y;     // bf16
  const uint8_t* h;
  int32_t h_f32;
  int32_t weight_f32;
  const float* rstd;
  const uint8_t* weight;
  const uint8_t* grad_sum;   // or null
  int64_t rows;
  int32_t H;
  uint8_t* grad_x;
  float* grad_weight;        // or null
  float* partial;            // [norm_grad_parts][H]
};

// Workgroups of the row pass, each with one row of partial weight gradients.
int norm_grad_parts(int64_t rows, int H);
hipError_t launch_norm_backward(const NormGradArgs& a, hipStream_t stream);

struct MatmulArgs {
  const uint8_t* a;
  const float* a_scales;
  int32_t a_scale_pitch;
  int32_t E;
  int64_t rows;
  const uint8_t* w;
  const float* w_scales;
  int32_t N;
  int32_t K;
  const int32_t* offset;     // null: one window of all rows
  const int32_t* count;      // null: offset[e + 1] - offset[e]
  int32_t swiglu;
  uint16_t* y;
};

hipError_t launch_matmul(const MatmulArgs& a, hipStream_t stream);

// ---------------------------------------------------------------- device
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(1))) u32x2 gu32x2;

// 8-byte accesses to global memory.
__device__ __forceinline__ u32x2 ld8(const void* p) { return *(const gu32x2*)(uintptr_t)p; }
__device__ __forceinline__ void st4x2(void* p, uint32_t lo, uint32_t hi) {
  *(gu32x2*)(uintptr_t)p = u32x2{lo, hi};
}

// Value of the lane N before, around the row of 16.
template <int N>
__device__ __forceinline__ uint32_t row_rotate(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x120 + N, 0xf, 0xf, true);
}
template <int N>
__device__ __forceinline__ float row_rotate(float x) {
  return __uint_as_float(row_rotate<N>(__float_as_uint(x)));
}

__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t umin(uint32_t a, uint32_t b) { return a < b ? a : b; }

// Both halves of the lanes' values, exchanged over 32 or 16 lanes: op(own,
// partner) is the same in both partners for a commutative op.
template <typename F>
__device__ __forceinline__ uint32_t across32(uint32_t x, F&& op) {
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return op((uint32_t)r[0], (uint32_t)r[1]);
}
template <typename F>
__device__ __forceinline__ uint32_t across16(uint32_t x, F&& op) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return op((uint32_t)r[0], (uint32_t)r[1]);
}

// Reduction over groups of LANES (16 or 64) neighbouring lanes by a
// commutative op, halves first; every lane gets the result.
template <int LANES, typename F>
__device__ __forceinline__ uint32_t reduce(uint32_t x, F&& op) {
  if (LANES == 64) {
    x = across32(x, op);
    x = across16(x, op);
  }
  x = op(x, row_rotate<8>(x));
  x = op(x, row_rotate<4>(x));
  x = op(x, row_rotate<2>(x));
  return op(x, row_rotate<1>(x));
}
template <int LANES>
__device__ __forceinline__ uint32_t reduce_max(uint32_t x) {
  return reduce<LANES>(x, umax);
}
template <int LANES>
__device__ __forceinline__ uint32_t reduce_min(uint32_t x) {
  return reduce<LANES>(x, umin);
}
__device__ __forceinline__ uint32_t fadd_bits(uint32_t a, uint32_t b) {
  return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
}
template <int LANES>
__device__ __forceinline__ float reduce_sum(float x) {
  return __uint_as_float(reduce<LANES>(__float_as_uint(x), fadd_bits));
}

}  // namespace moe
