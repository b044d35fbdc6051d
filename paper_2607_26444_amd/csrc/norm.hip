// RMS norm with the residual's addition and 8-bit output, quantisation of
// rows, and the norm's gradients.
//
// A row is held in registers by one workgroup (rows of up to 64 * NV vectors
// of 8 values: by one wavefront, four rows to a workgroup), read once and
// written once; every sum is float32.

#include <math.h>

#include <type_traits>

#include "layer.h"

namespace moe {
namespace {

constexpr float kFp8Max = 448.0f, kInt8Max = 127.0f;
constexpr float kAmaxMin = 0x1p-100f;   // keeps M / amax finite and amax / M normal

struct Vec8 {
  float f[8];
};

__device__ __forceinline__ Vec8 unpack8(const u32x4& v) {
  return Vec8{{bf16_lo(v.x), bf16_hi(v.x), bf16_lo(v.y), bf16_hi(v.y), bf16_lo(v.z), bf16_hi(v.z),
               bf16_lo(v.w), bf16_hi(v.w)}};
}

__device__ __forceinline__ Vec8 from_f32(const u32x4& a, const u32x4& b) {
  return Vec8{{__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z),
               __uint_as_float(a.w), __uint_as_float(b.x), __uint_as_float(b.y),
               __uint_as_float(b.z), __uint_as_float(b.w)}};
}

// Vector v (8 values) of a row of bf16 or float32.
__device__ __forceinline__ Vec8 load8(const uint8_t* row, int64_t v, bool f32) {
  if (f32) return from_f32(ld16(row + v * 32), ld16(row + v * 32 + 16));
  return unpack8(ld16(row + v * 16));
}

__device__ __forceinline__ void store8(uint8_t* row, int64_t v, bool f32, const Vec8& x) {
  if (f32) {
    st16(row + v * 32, u32x4{__float_as_uint(x.f[0]), __float_as_uint(x.f[1]),
                             __float_as_uint(x.f[2]), __float_as_uint(x.f[3])});
    st16(row + v * 32 + 16, u32x4{__float_as_uint(x.f[4]), __float_as_uint(x.f[5]),
                                  __float_as_uint(x.f[6]), __float_as_uint(x.f[7])});
  } else {
    st16(row + v * 16, pack8(x.f));
  }
}

__device__ __forceinline__ void st8(uint8_t* p, uint32_t lo, uint32_t hi) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  *(__attribute__((address_space(1))) u32x2*)(uintptr_t)p = u32x2{lo, hi};
}

// |x| as an unsigned that orders alike, with NaN above infinity, so that a
// maximum keeps it.
__device__ __forceinline__ uint32_t abs_key(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// max(amax, 2^-100), NaN kept.
__device__ __forceinline__ float usable_amax(float amax) {
  return amax < kAmaxMin ? kAmaxMin : amax;
}

__device__ __forceinline__ float scale_of(float amax, float most) {
  return amax == 0.0f ? 1.0f : usable_amax(amax) / most;
}

__device__ __forceinline__ uint32_t clamp_pair_fp8(float a, float b, uint32_t old, bool hi) {
  a = fminf(fmaxf(a, -kFp8Max), kFp8Max);
  b = fminf(fmaxf(b, -kFp8Max), kFp8Max);
  return hi ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, true)
            : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, false);
}

__device__ __forceinline__ uint32_t code_int8(float v) {
  return (uint32_t)(int32_t)rintf(fminf(fmaxf(v, -kInt8Max), kInt8Max)) & 0xFFu;
}

__device__ __forceinline__ void store_codes(uint8_t* q, int64_t v, bool fp8, const Vec8& y,
                                            float inv) {
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float a = y.f[4 * h] * inv, b = y.f[4 * h + 1] * inv, c = y.f[4 * h + 2] * inv,
                d = y.f[4 * h + 3] * inv;
    if (fp8)
      w[h] = clamp_pair_fp8(c, d, clamp_pair_fp8(a, b, 0, false), true);
    else
      w[h] = code_int8(a) | code_int8(b) << 8 | code_int8(c) << 16 | code_int8(d) << 24;
  }
  st8(q + v * 8, w[0], w[1]);
}

// Sum and maximum over the row's wavefronts: wavefront results meet in LDS.
// Every thread adds them in the same order.
__device__ __forceinline__ void row_reduce(float& sum, uint32_t& top, int waves, int wave,
                                           int lane, float* s_sum, uint32_t* s_top) {
  sum = reduce_sum<64>(sum);
  top = reduce_max<64>(top);
  if (waves == 1) return;
  if (lane == 0) {
    s_sum[wave] = sum;
    s_top[wave] = top;
  }
  __syncthreads();
  sum = 0.0f;
  top = 0u;
  for (int w = 0; w < waves; ++w) {
    sum += s_sum[w];
    top = umax(top, s_top[w]);
  }
}

// Row r: thread `at` of the row's `threads`.
template <int NV>
__device__ __forceinline__ void norm_row(const NormArgs& a, int64_t r, int at, int waves, int wave,
                                         int lane, float* s_sum, uint32_t* s_top) {
  const int threads = waves * kWave;
  const int nv = a.H / 8;
  const bool has_res = a.residual != nullptr;
  Vec8 h[NV], w[NV];
  const uint8_t* x = a.x + r * a.x_pitch;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = at + i * threads;
    h[i] = v < nv ? load8(x, v, false) : Vec8{};
  }
  if (has_res) {
    const uint8_t* res = a.residual + r * a.residual_pitch;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) {
        const Vec8 b = load8(res, v, a.residual_f32);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[i].f[j] += b.f[j];
      }
    }
  }
  if (a.weight) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      w[i] = v < nv ? load8(a.weight, v, a.weight_f32) : Vec8{};
    }
  }
  if (a.sum_out) {
    const int64_t row = r * (int64_t)a.H * (a.residual_f32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) store8(a.sum_out + row, v, a.residual_f32, h[i]);
    }
  }

  float sum = 0.0f, rstd = 1.0f;
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum = __builtin_fmaf(h[i].f[j], h[i].f[j], sum);
      if (a.weight) h[i].f[j] *= w[i].f[j];
      top = umax(top, abs_key(h[i].f[j]));
    }
  }
  if (a.weight || a.quant == kQuantInt8)
    row_reduce(sum, top, waves, wave, lane, s_sum, s_top);
  if (a.weight) {
    rstd = 1.0f / sqrtf(sum / (float)a.H + a.eps);
    if (a.rstd && at == 0) a.rstd[r] = rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i].f[j] *= rstd;
  }

  if (a.y) {
    uint8_t* y = a.y + r * (int64_t)a.H * 2;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) store8(y, v, false, h[i]);
    }
  }
  if (a.quant == kQuantInt8) {
    const float amax = __uint_as_float(top) * rstd;
    const float inv = kInt8Max / usable_amax(amax);
    uint8_t* q = a.q + r * (int64_t)a.H;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) store_codes(q, v, false, h[i], inv);
    }
    for (int c = at; c < a.scale_cols; c += threads)
      a.q_scales[r * a.scale_cols + c] = scale_of(amax, kInt8Max);
  } else if (a.quant == kQuantFp8) {
    uint8_t* q = a.q + r * (int64_t)a.H;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      uint32_t key = 0u;                          // 16 lanes hold a block of 128
#pragma unroll
      for (int j = 0; j < 8; ++j) key = umax(key, abs_key(h[i].f[j]));
      const float amax = __uint_as_float(reduce_max<16>(key));
      if (v < nv) {
        store_codes(q, v, true, h[i], kFp8Max / usable_amax(amax));
        if ((v & 15) == 0) a.q_scales[r * a.scale_cols + v / 16] = scale_of(amax, kFp8Max);
      }
    }
  }
}

// waves: wavefronts of a row; 1: each wavefront of the workgroup has its own row.
template <int NV>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, int waves) {
  __shared__ float s_sum[16];
  __shared__ uint32_t s_top[16];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int at = waves == 1 ? lane : (int)threadIdx.x;
  const int per = waves == 1 ? blockDim.x / kWave : 1;         // rows of a workgroup
  for (int64_t r = (int64_t)blockIdx.x * per + (waves == 1 ? wave : 0); r < a.rows;
       r += (int64_t)gridDim.x * per) {
    if (a.row_src && (int32_t)ld4(a.row_src + r) < 0) continue;   // whole wavefronts or workgroups
    norm_row<NV>(a, r, at, waves, wave, lane, s_sum, s_top);
    if (waves > 1 && r + (int64_t)gridDim.x < a.rows) __syncthreads();   // s_sum, s_top are free
  }
}

// Gradients.  A workgroup takes the rows blockIdx.x, + gridDim.x, ...; each
// thread keeps the weight gradient of its columns in registers and leaves it
// in the workgroup's row of `partial` at the end.
template <int NV>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormGradArgs a) {
  __shared__ float s_sum[2][16];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int threads = blockDim.x, waves = threads / kWave;
  const int nv = a.H / 8;
  const int hb = a.h_f32 ? 4 : 2;
  Vec8 w[NV], dw[NV] = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + i * threads;
    w[i] = v < nv ? load8(a.weight, v, a.weight_f32) : Vec8{};
  }
  int phase = 0;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const uint8_t* dy = a.grad_y + r * (int64_t)a.H * 2;
    const uint8_t* hr = a.h + r * (int64_t)a.H * hb;
    const float rstd = __uint_as_float(ld4(a.rstd + r));
    Vec8 u[NV], h[NV];
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = threadIdx.x + i * threads;
      u[i] = v < nv ? load8(dy, v, false) : Vec8{};
      h[i] = v < nv ? load8(hr, v, a.h_f32) : Vec8{};
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        dw[i].f[j] = __builtin_fmaf(u[i].f[j] * h[i].f[j], rstd, dw[i].f[j]);
        u[i].f[j] *= w[i].f[j];
        dot = __builtin_fmaf(u[i].f[j], h[i].f[j], dot);
      }
    }
    dot = reduce_sum<64>(dot);
    if (waves > 1) {
      if (lane == 0) s_sum[phase][wave] = dot;
      __syncthreads();                           // the other half is free again by now
      dot = 0.0f;
      for (int k = 0; k < waves; ++k) dot += s_sum[phase][k];
      phase ^= 1;
    }
    const float c = dot / (float)a.H * rstd * rstd;
    uint8_t* dx = a.grad_x + r * (int64_t)a.H * hb;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = threadIdx.x + i * threads;
      if (v >= nv) continue;
      Vec8 g = a.grad_sum ? load8(a.grad_sum + r * (int64_t)a.H * hb, v, a.h_f32) : Vec8{};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        g.f[j] = __builtin_fmaf(rstd, u[i].f[j] - h[i].f[j] * c, g.f[j]);
      store8(dx, v, a.h_f32, g);
    }
  }
  if (!a.grad_weight) return;
  uint8_t* part = reinterpret_cast<uint8_t*>(a.partial + (int64_t)blockIdx.x * a.H);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int v = threadIdx.x + i * threads;
    if (v < nv) store8(part, v, true, dw[i]);
  }
}

// Column sums of partial [parts][H]: 16 columns to a workgroup, 16 threads of
// a column add every 16th row, their sums meet in LDS.
__global__ __launch_bounds__(kBlock) void norm_weight_kernel(const float* partial, int parts, int H,
                                                             float* out) {
  __shared__ float s[16][17];
  const int col = blockIdx.x * 16 + (threadIdx.x & 15), row = threadIdx.x / 16;
  float sum = 0.0f;
  if (col < H)
    for (int p = row; p < parts; p += 16) sum += partial[(int64_t)p * H + col];
  s[row][threadIdx.x & 15] = sum;
  __syncthreads();
  if (row == 0 && col < H) {
    for (int p = 1; p < 16; ++p) sum += s[p][threadIdx.x];
    out[col] = sum;
  }
}

struct RowShape {
  int nv;      // vectors of a thread: 1 or 2
  int waves;   // wavefronts of a row
};

RowShape row_shape(int H) {
  const int vecs = H / 8;
  const int nv = vecs <= kWave ? 1 : 2;
  return {nv, (vecs + kWave * nv - 1) / (kWave * nv)};
}

template <typename F>
hipError_t by_vectors(int nv, F&& launch) {
  return nv == 1 ? launch(std::integral_constant<int, 1>())
                 : launch(std::integral_constant<int, 2>());
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const RowShape s = row_shape(a.H);
  const int64_t want = s.waves == 1 ? (a.rows + kWavesPerBlock - 1) / kWavesPerBlock : a.rows;
  const int64_t blocks = want < kMaxGrid ? want : kMaxGrid;
  const int threads = s.waves == 1 ? kBlock : s.waves * kWave;
  return by_vectors(s.nv, [&](auto nv) {
    hipLaunchKernelGGL((norm_kernel<nv.value>), dim3((unsigned)blocks), dim3(threads), 0, stream,
                       a, s.waves);
    return hipGetLastError();
  });
}

int norm_grad_parts(int64_t rows, int H) {
  const RowShape s = row_shape(H);
  const int64_t most = 256 * 16 / s.waves;      // 16 wavefronts resident on each compute unit
  return (int)(rows < most ? rows : most);
}

hipError_t launch_norm_backward(const NormGradArgs& a, hipStream_t stream) {
  const RowShape s = row_shape(a.H);
  const int parts = norm_grad_parts(a.rows, a.H);
  if (parts > 0) {
    const hipError_t err = by_vectors(s.nv, [&](auto nv) {
      hipLaunchKernelGGL((norm_backward_kernel<nv.value>), dim3((unsigned)parts),
                         dim3(s.waves * kWave), 0, stream, a);
      return hipGetLastError();
    });
    if (err != hipSuccess) return err;
  }
  if (a.grad_weight)
    hipLaunchKernelGGL(norm_weight_kernel, dim3((unsigned)((a.H + 15) / 16)), dim3(kBlock), 0,
                       stream, a.partial, parts, a.H, a.grad_weight);
  return hipGetLastError();
}

}  // namespace moe
