// RMS norm with the residual's addition and 8-bit output, quantisation of
// rows, and the norm's gradients.
//
//   h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps), y = h rstd weight
//   with u = grad_y weight, n = h rstd:
//   grad_x = rstd (u - n mean(u n)) + grad_sum, grad_weight = sum over rows of grad_y n
// A row is held in registers by one workgroup (rows of up to 64 * NV vectors
// of 8 values: by one wavefront, four rows to a workgroup), read once and
// written once; every sum is float32.  h is rounded only where it is stored: the norm
// and the 8-bit codes follow from the unrounded row.
//
// Bound by HBM.  16384 rows of 7168, bf16 residual, to fp8 (826 MB): 159 us, 5.2 TB/s.
// Gradients of 32768 x 4096 bf16 (1074 MB): 201 us, 5.4 TB/s.  A workgroup that
// ends after its row reads nothing while it reduces, so workgroups stay and ask for
// the next row first (227 -> 159 us and 222 -> 201).  Small batches are bound by the
// launch: 64 rows of 7168 6.1 us; the gradients take two launches, 777 x 2056 11 us.

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

template <bool STREAM>
__device__ __forceinline__ void put16(uint8_t* p, u32x4 v) {
  if (STREAM) st16_stream(p, v);
  else st16(p, v);
}

// Vector v (8 values) of a row of bf16 or float32.
template <bool STREAM = false>
__device__ __forceinline__ void store8(uint8_t* row, int64_t v, bool f32, const Vec8& x) {
  if (f32) {
    put16<STREAM>(row + v * 32, u32x4{__float_as_uint(x.f[0]), __float_as_uint(x.f[1]),
                                      __float_as_uint(x.f[2]), __float_as_uint(x.f[3])});
    put16<STREAM>(row + v * 32 + 16, u32x4{__float_as_uint(x.f[4]), __float_as_uint(x.f[5]),
                                           __float_as_uint(x.f[6]), __float_as_uint(x.f[7])});
  } else {
    put16<STREAM>(row + v * 16, pack8(x.f));
  }
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
  st4x2(q + v * 8, w[0], w[1]);
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

// How a row's second input (the residual, the weight) is there.
enum Form : int { kNone = 0, kBf16 = 1, kF32 = 2 };

// Vectors of a row as they come from memory.
template <int NV, Form F>
struct Raw {
  u32x4 v[NV * (F == kF32 ? 2 : F == kBf16 ? 1 : 0) + (F == kNone)];

  // Vectors at, at + threads, ... of the nv of a row; zeros past the end.
  __device__ __forceinline__ void load(const uint8_t* row, int at, int threads, int nv, bool stream) {
    if constexpr (F != kNone) {
      constexpr int kParts = F == kF32 ? 2 : 1;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const int64_t n = at + i * threads;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          const uint8_t* from = row + (n * kParts + p) * 16;
          v[i * kParts + p] = n >= nv ? u32x4{0, 0, 0, 0} : stream ? ld16_stream(from) : ld16(from);
        }
      }
    }
  }
  __device__ __forceinline__ Vec8 get(int i) const {
    if constexpr (F == kF32) return from_f32(v[2 * i], v[2 * i + 1]);
    else return unpack8(v[i]);
  }
};

// A row's work after its vectors h (x + residual) are in registers.
template <int NV, Form RES, Form WEIGHT>
__device__ __forceinline__ void finish_row(const NormArgs& a, int64_t r, int at, int waves, int wave,
                                           int lane, Vec8 (&h)[NV], const Raw<NV, WEIGHT>& weight,
                                           float* s_sum, uint32_t* s_top) {
  const int threads = waves * kWave;
  const int nv = a.H / 8;
  if (RES != kNone && a.sum_out) {
    uint8_t* out = a.sum_out + r * (int64_t)a.H * (RES == kF32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) store8<true>(out, v, RES == kF32, h[i]);
    }
  }

  // One reduction gives the sum of squares and the largest |h weight|, which is
  // max |v| / rstd to float32's rounding.
  float sum = 0.0f, amax = 0.0f;
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    Vec8 w;
    if constexpr (WEIGHT != kNone) w = weight.get(i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sum = __builtin_fmaf(h[i].f[j], h[i].f[j], sum);
      top = umax(top, abs_key(WEIGHT != kNone ? h[i].f[j] * w.f[j] : h[i].f[j]));
    }
  }
  if (WEIGHT != kNone || a.quant == kQuantInt8)
    row_reduce(sum, top, waves, wave, lane, s_sum, s_top);
  amax = __uint_as_float(top);
  if constexpr (WEIGHT != kNone) {
    const float rstd = 1.0f / sqrtf(sum / (float)a.H + a.eps);
    if (a.rstd && at == 0) a.rstd[r] = rstd;
    const bool normal = top - 0x00800000u < 0x7F000000u;   // neither 0, subnormal, infinite nor NaN
    amax *= rstd;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Vec8 w = weight.get(i);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i].f[j] = h[i].f[j] * rstd * w.f[j];
    }
    // h weight may lie outside the normal range where v does not: then the maximum of v
    // itself (the row's threads agree on that)
    if (!normal && a.quant == kQuantInt8) {
      top = 0u;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) top = umax(top, abs_key(h[i].f[j]));
      if (waves > 1) __syncthreads();            // the first results have been read
      row_reduce(sum, top, waves, wave, lane, s_sum, s_top);
      amax = __uint_as_float(top);
    }
  }

  if (WEIGHT != kNone && a.y) {
    uint8_t* y = a.y + r * (int64_t)a.H * 2;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v >= nv) continue;
      if (a.stream_y) store8<true>(y, v, false, h[i]);
      else store8(y, v, false, h[i]);
    }
  }
  if (a.quant == kQuantInt8) {
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

template <int NV, Form RES>
__device__ __forceinline__ void join(const Raw<NV, kBf16>& x, const Raw<NV, RES>& res,
                                     Vec8 (&h)[NV]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    h[i] = x.get(i);
    if constexpr (RES != kNone) {
      const Vec8 b = res.get(i);
#pragma unroll
      for (int j = 0; j < 8; ++j) h[i].f[j] += b.f[j];
    }
  }
}

// waves: wavefronts of a row; 1: each wavefront of the workgroup has its own row.
// The weights stay in registers over a workgroup's rows, and the next row's
// vectors are asked for before the present one is worked on.
template <int NV, Form RES, Form WEIGHT>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs a, int waves) {
  __shared__ float s_sum[2][16];
  __shared__ uint32_t s_top[2][16];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int at = waves == 1 ? lane : (int)threadIdx.x;
  const int per = waves == 1 ? blockDim.x / kWave : 1;         // rows of a workgroup
  const int64_t step = (int64_t)gridDim.x * per;
  const int threads = waves * kWave, nv = a.H / 8;
  int64_t r = (int64_t)blockIdx.x * per + (waves == 1 ? wave : 0);
  if (r >= a.rows) return;                                     // whole wavefronts or workgroups
  Raw<NV, kBf16> x;
  Raw<NV, RES> res;
  Raw<NV, WEIGHT> weight;
  x.load(a.x + r * a.x_pitch, at, threads, nv, true);
  res.load(a.residual + r * a.residual_pitch, at, threads, nv, true);
  weight.load(a.weight, at, threads, nv, false);
  int phase = 0;
  for (;;) {
    Vec8 h[NV];
    join(x, res, h);
    const int64_t next = r + step;
    const bool more = next < a.rows;
    if (more) {
      x.load(a.x + next * a.x_pitch, at, threads, nv, true);
      res.load(a.residual + next * a.residual_pitch, at, threads, nv, true);
    }
    finish_row<NV, RES, WEIGHT>(a, r, at, waves, wave, lane, h, weight, s_sum[phase], s_top[phase]);
    if (!more) break;
    r = next;
    phase ^= 1;                                  // the other half is free: all have met since
  }
}

// Quantisation alone: rows to skip are found before they are read.
template <int NV>
__global__ __launch_bounds__(1024) void quantize_kernel(NormArgs a, int waves) {
  __shared__ float s_sum[16];
  __shared__ uint32_t s_top[16];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int at = waves == 1 ? lane : (int)threadIdx.x;
  const int per = waves == 1 ? blockDim.x / kWave : 1;         // rows of a workgroup
  const int threads = waves * kWave, nv = a.H / 8;
  for (int64_t r = (int64_t)blockIdx.x * per + (waves == 1 ? wave : 0); r < a.rows;
       r += (int64_t)gridDim.x * per) {
    if (a.row_src && (int32_t)ld4(a.row_src + r) < 0) continue;   // whole wavefronts or workgroups
    Raw<NV, kBf16> x;
    Raw<NV, kNone> none;
    x.load(a.x + r * a.x_pitch, at, threads, nv, true);
    Vec8 h[NV];
    join(x, none, h);
    finish_row<NV, kNone, kNone>(a, r, at, waves, wave, lane, h, none, s_sum, s_top);
    if (waves > 1 && r + (int64_t)gridDim.x < a.rows) __syncthreads();   // s_sum, s_top are free
  }
}

// Gradients.  A workgroup takes the rows r, r + step, ... (waves = 1: each of
// its wavefronts) and asks for the next row before it works on the present
// one; each thread keeps the weight gradient of its columns in registers and
// the workgroup leaves it in its row of `partial` at the end.
template <int NV, Form FORM, Form WEIGHT, bool SUM>
__global__ __launch_bounds__(1024) void norm_backward_kernel(NormGradArgs a, int waves) {
  constexpr bool F = FORM == kF32, kLate = F && NV == 2;
  __shared__ float s_sum[2][16];
  __shared__ float s_dw[NV == 2 ? 1024 : 512][kWavesPerBlock];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int at = waves == 1 ? lane : (int)threadIdx.x;
  const int per = waves == 1 ? kWavesPerBlock : 1;             // rows of a workgroup
  const int64_t step = (int64_t)gridDim.x * per;
  const int threads = waves * kWave, nv = a.H / 8;
  const int64_t wide = (int64_t)a.H * (F ? 4 : 2);
  Raw<NV, WEIGHT> weight;
  Raw<NV, kBf16> dy;
  Raw<NV, FORM> hv;
  Raw<NV, SUM ? FORM : kNone> gs;
  Vec8 dw[NV] = {};
  weight.load(a.weight, at, threads, nv, false);
  int64_t r = (int64_t)blockIdx.x * per + (waves == 1 ? wave : 0);
  float rstd = 0.0f;
  auto fetch = [&](int64_t n) {
    dy.load(a.grad_y + n * a.H * 2, at, threads, nv, true);
    hv.load(a.h + n * wide, at, threads, nv, true);
    rstd = __uint_as_float(ld4(a.rstd + n));
  };
  if (r < a.rows) fetch(r);
  for (int phase = 0; r < a.rows; r += step, phase ^= 1) {
    Vec8 u[NV], h[NV];
    const float rs = rstd;
    float dot = 0.0f;
    // needed last; float32 rows lack the registers to have it early
    if (!kLate) gs.load(a.grad_sum + r * wide, at, threads, nv, true);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      u[i] = dy.get(i);
      h[i] = hv.get(i);
    }
    if (!kLate && r + step < a.rows) fetch(r + step);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const Vec8 w = weight.get(i);
#pragma unroll
      for (int j = 0; j < 8; ++j) {              // h rstd first: products stay inside float32
        h[i].f[j] *= rs;
        dw[i].f[j] = __builtin_fmaf(u[i].f[j], h[i].f[j], dw[i].f[j]);
        u[i].f[j] *= w.f[j];
        dot = __builtin_fmaf(u[i].f[j], h[i].f[j], dot);
      }
    }
    dot = reduce_sum<64>(dot);
    if (waves > 1) {
      if (lane == 0) s_sum[phase][wave] = dot;
      __syncthreads();                           // the other half is free again by now
      dot = 0.0f;
      for (int k = 0; k < waves; ++k) dot += s_sum[phase][k];
    }
    if (kLate) gs.load(a.grad_sum + r * wide, at, threads, nv, true);
    const float c = dot / (float)a.H;
    uint8_t* dx = a.grad_x + r * wide;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v >= nv) continue;
      Vec8 g = {};
      if constexpr (SUM) g = gs.get(i);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        g.f[j] = __builtin_fmaf(rs, u[i].f[j] - h[i].f[j] * c, g.f[j]);
      store8<true>(dx, v, F, g);
    }
    if (kLate && r + step < a.rows) fetch(r + step);
  }
  if (!a.grad_weight) return;
  uint8_t* part = reinterpret_cast<uint8_t*>(a.partial + (int64_t)blockIdx.x * a.H);
  if (waves > 1) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int v = at + i * threads;
      if (v < nv) store8(part, v, true, dw[i]);
    }
    return;
  }
  // the four wavefronts' columns meet in LDS
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int c = (at + i * kWave) * 8 + j;
      if (c < a.H) s_dw[c][wave] = dw[i].f[j];
    }
  __syncthreads();
  for (int c = threadIdx.x; c < a.H; c += kBlock)
    reinterpret_cast<float*>(part)[c] = ((s_dw[c][0] + s_dw[c][1]) + s_dw[c][2]) + s_dw[c][3];
}

// Column sums of partial [parts][H]: 32 columns (a line) to a workgroup, 128
// rows at a time, the 128 sums of a column added in LDS.  A fixed order, where
// atomic additions would give another sum each time.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float* partial, int parts, int H,
                                                           float* out) {
  __shared__ float s[128][33];
  const int quad = threadIdx.x & 7, row = threadIdx.x / 8;
  const int col = blockIdx.x * 32 + quad * 4;            // H % 8 == 0: whole fours
  float sum[4] = {};
  if (col < H) {
    for (int n0 = row; n0 < parts; n0 += 1024) {         // eight rows asked for together
      u32x4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int n = n0 + i * 128;
        v[i] = n < parts ? ld16(partial + (int64_t)n * H + col) : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        sum[0] += __uint_as_float(v[i].x);
        sum[1] += __uint_as_float(v[i].y);
        sum[2] += __uint_as_float(v[i].z);
        sum[3] += __uint_as_float(v[i].w);
      }
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) s[row][quad * 4 + j] = sum[j];
  __syncthreads();
  const int c = threadIdx.x & 31, part = threadIdx.x / 32;   // 32 parts of four rows
  float t = 0.0f;
#pragma unroll
  for (int j = 0; j < 4; ++j) t += s[part * 4 + j][c];
  __syncthreads();
  s[part][c] = t;
  __syncthreads();
  if (part == 0 && blockIdx.x * 32 + c < H) {
    t = 0.0f;
#pragma unroll
    for (int j = 0; j < 32; ++j) t += s[j][c];
    out[blockIdx.x * 32 + c] = t;
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

template <typename F>
hipError_t by_type(bool f32, F&& launch) {
  return f32 ? launch(std::integral_constant<Form, kF32>())
             : launch(std::integral_constant<Form, kBf16>());
}

// Workgroups of a persistent row kernel: 16 wavefronts to a compute unit.
// More, with the fewer registers that allows, read no faster (16384 rows of 7168
// to fp8, us at 16 / 21 / 28 wavefronts: 160 / 161 / 198).
int64_t row_groups(int64_t want, int threads) {
  const int groups = 16 / (threads / kWave);
  const int64_t resident = 256 * (int64_t)(groups > 1 ? groups : 1);
  return want < resident ? want : resident;
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  const RowShape s = row_shape(a.H);
  const int threads = s.waves == 1 ? kBlock : s.waves * kWave;
  const int64_t want = s.waves == 1 ? (a.rows + kWavesPerBlock - 1) / kWavesPerBlock : a.rows;
  if (!a.weight) {
    const int64_t blocks = want < kMaxGrid ? want : kMaxGrid;
    return by_vectors(s.nv, [&](auto nv) {
      hipLaunchKernelGGL((quantize_kernel<nv.value>), dim3((unsigned)blocks), dim3(threads), 0,
                         stream, a, s.waves);
      return hipGetLastError();
    });
  }
  const int64_t blocks = row_groups(want, threads);
  return by_vectors(s.nv, [&](auto nv) {
    return by_type(a.weight_f32, [&](auto weight) {
      const auto run = [&](auto res) {
        hipLaunchKernelGGL((norm_kernel<nv.value, res.value, weight.value>), dim3((unsigned)blocks),
                           dim3(threads), 0, stream, a, s.waves);
        return hipGetLastError();
      };
      return a.residual ? by_type(a.residual_f32, run)
                        : run(std::integral_constant<Form, kNone>());
    });
  });
}

// Workgroups of the gradients' row pass.  One row to each would leave as many
// partial rows to add: beyond a workgroup for each compute unit they take several
// rows, up to three (us, one / three rows: 1500 x 4096 17.0 / 14.5, 777 x 2056
// float32 12.5 / 10.5, 256 x 4096 8.1 / 9.3).
int norm_grad_parts(int64_t rows, int H) {
  const RowShape s = row_shape(H);
  const int threads = s.waves == 1 ? kBlock : s.waves * kWave;
  const int64_t groups = s.waves == 1 ? (rows + kWavesPerBlock - 1) / kWavesPerBlock : rows;
  const int64_t want = groups <= 256 ? groups : groups <= 768 ? 256 : groups / 3;
  return (int)row_groups(want, threads);
}

hipError_t launch_norm_backward(const NormGradArgs& a, hipStream_t stream) {
  const RowShape s = row_shape(a.H);
  const int threads = s.waves == 1 ? kBlock : s.waves * kWave;
  const int parts = norm_grad_parts(a.rows, a.H);
  if (parts > 0) {
    const hipError_t err = by_vectors(s.nv, [&](auto nv) {
      return by_type(a.h_f32, [&](auto form) {
        return by_type(a.weight_f32, [&](auto weight) {
          if (a.grad_sum)
            hipLaunchKernelGGL((norm_backward_kernel<nv.value, form.value, weight.value, true>),
                               dim3((unsigned)parts), dim3(threads), 0, stream, a, s.waves);
          else
            hipLaunchKernelGGL((norm_backward_kernel<nv.value, form.value, weight.value, false>),
                               dim3((unsigned)parts), dim3(threads), 0, stream, a, s.waves);
          return hipGetLastError();
        });
      });
    });
    if (err != hipSuccess) return err;
  }
  if (a.grad_weight)
    hipLaunchKernelGGL(norm_weight_kernel, dim3((unsigned)((a.H + 31) / 32)), dim3(1024), 0, stream,
                       a.partial, parts, a.H, a.grad_weight);
  return hipGetLastError();
}

}  // namespace moe
