// Balance loss of routed sequences, and its gradient.
//
// Of a sequence with n live tokens: s a token's scores (softmax or sigmoid),
//   p_te = s_te / sum_e s_te, P_e = sum_t p_te / n, f_e = E count_e / sum_e count_e
//   loss = sum_e f_e P_e
//   dx_te = grad_loss / n p_te (f_e - sum_i f_i p_ti), times 1 - s_te for sigmoid scores
// (the counts have no gradient).  All of it is float32; tokens are summed in an order that
// follows from the sizes alone, slots in whole numbers.
//
// A sequence is cut into parts, a workgroup each: a lane keeps the sums of its experts
// over the part's tokens, the slots are counted in LDS.  A second launch adds the parts: one
// workgroup a sequence, or where there is more to add 32 experts to a workgroup, the last of
// which adds the loss.  Sequences of one part need no second launch.
//
// The logits are read once, but exponentials, reciprocals and sums over lanes take longer than
// that (vector instructions are issued in 7.6 of the first kernel's 12.4 us), not the waiting for
// loads (two rounds of tokens asked for ahead instead of one were a seventh slower): 32768 x 256
// float32 in 8 sequences 13.5 us by sigmoid (2.5 TB/s), 12.9 by softmax scores; the gradient of
// 32768 x 128 bf16 with another added 10.0 (2.5 TB/s), of 32768 x 256 float32, sigmoid, 15.8 (4.2
// TB/s).  Small batches are bound by the launches: 128 x 16 4.9 us.

#include "logits.h"

namespace moe {
namespace {

// Neighbouring logits that a lane has of a row: 16 bytes where it has as many.
template <int VPL, bool F32>
constexpr int run_of() {
  return VPL < (F32 ? 4 : 8) ? VPL : F32 ? 4 : 8;
}

// Expert of a lane's i-th value: runs of neighbours, dealt to the lanes in turn.
template <int LANES, int VPL, bool F32>
__device__ __forceinline__ int expert_of(int sub, int i) {
  constexpr int N = run_of<VPL, F32>();
  return (i / N * LANES + sub) * N + i % N;
}

// A token's dealt logits; -inf where the token takes no part.
template <int LANES, int VPL, bool F32>
__device__ __forceinline__ void load_token(const void* logits, int64_t at, int sub, int E, int vec,
                                           bool take, float (&x)[VPL]) {
#pragma unroll
  for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
  if (!take) return;
  constexpr int N = run_of<VPL, F32>();
#pragma unroll
  for (int g = 0; g < VPL / N; ++g) {
    float v[N];
    load_logits<N>(logits, F32, at, expert_of<LANES, VPL, F32>(sub, g * N), E, vec, v);
#pragma unroll
    for (int j = 0; j < N; ++j) x[g * N + j] = v[j];
  }
}

// exp(x) for x of [-150, 88], within 3 units of 2^-24 of it (0 below -87.3): the hardware's
// exponential (1 unit in the last place) of t = x log2(e).  What rounds in t, and the constant's
// error, up to |x| units together were they left out, 1 + (x log2(e) - t) ln(2) makes good.
__device__ __forceinline__ float exp_near(float x) {
  constexpr float kLog2E = 1.44269502f, kLow = 1.92596299e-8f, kLn2 = 0.693147181f;
  const float t = x * kLog2E;
  const float r = __builtin_fmaf(x, kLow, __builtin_fmaf(x, kLog2E, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fmaf(e, r * kLn2, e);
}

// Scores in place of the logits, and the factor that makes shares of them: 0 where their sum
// is none, or lies below float32's normal range (sigmoid scores of very low logits).  Sigmoid
// scores of a token whose logits all lie below -27 are exp(x) to 2^-40 of them; such come divided
// by the largest, so that they are there also where each is below float32's range.
// Exponentials and reciprocals are as near as the routing's (expf, exactly rounded) in fewer
// instructions: their arguments are clamped to where nothing overflows.  A rounded argument and
// the bare reciprocal would save 0.4 us (softmax) and 1.2 us (sigmoid) of 32768 x 256 logits and
// cost up to 63 units of a share, for 6.  REST: also 1 - s.
template <int LANES, int VPL, bool SIGMOID, bool REST = false>
__device__ __forceinline__ float scores(float (&x)[VPL], float (&rest)[REST ? VPL : 1]) {
  if constexpr (SIGMOID) {
    float v[VPL], local = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const float e = exp_near(__builtin_amdgcn_fmed3f(-x[i], -150.0f, 87.0f)), d = 1.0f + e;
      const float r = __builtin_amdgcn_rcpf(d);
      v[i] = x[i] >= -87.0f ? __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r) : 0.0f;
      if constexpr (REST) rest[i] = e > 1.0f ? 1.0f - v[i] : e * v[i];   // also where s rounds to 1
      local += v[i];
    }
    float total = reduce_sum<LANES>(local);
    if (total < 0x1p-40f) {                            // the token's lanes together
      const float m = row_max<LANES, VPL>(x);
      if (m > -INFINITY) {
        local = 0.0f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
          v[i] = exp_near(__builtin_amdgcn_fmed3f(x[i] - m, -150.0f, 0.0f));
          if constexpr (REST) rest[i] = 1.0f;
          local += v[i];
        }
        total = reduce_sum<LANES>(local);
        // the sum of the scores, e^64 times as large, against 2^-126
        if (exp_near(__builtin_amdgcn_fmed3f(m + 64.0f, -150.0f, 88.0f)) * total < 7.32938e-11f)
          total = 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = v[i];
    return total > 0.0f ? 1.0f / total : 0.0f;
  } else {
    float m = row_max<LANES, VPL>(x);
    if (m == INFINITY) {                               // infinite ones share alike
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] = x[i] == m ? 0.0f : -INFINITY;
      m = 0.0f;
    }
    // -inf, NaN and what lies far below the largest come to the lower end, which gives 0
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = exp_near(__builtin_amdgcn_fmed3f(x[i] - m, -150.0f, 0.0f));
    float local = 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) local += x[i];
    const float total = reduce_sum<LANES>(local);
    return total > 0.0f ? 1.0f / total : 0.0f;         // 1 at least
  }
}

// Sum over the workgroup's threads, each thread's the same; `s`: a word a wavefront.
__device__ __forceinline__ float block_sum(float x, float* s) {
  x = reduce_sum<64>(x);
  __syncthreads();                                     // s is free
  if ((threadIdx.x & (kWave - 1)) == 0) s[threadIdx.x / kWave] = x;
  __syncthreads();
  float sum = 0.0f;
  for (int w = 0; w < (int)blockDim.x / kWave; ++w) sum += s[w];
  return sum;
}

// Words of a part in the workspace: sums of the experts' shares, slots.
__host__ __device__ inline int part_pitch(int E) { return (E + 31) / 32 * 32; }

constexpr int kMaxWaves = 16;

// A workgroup of up to 16 wavefronts has 4 (16 lanes a token) or 1 tokens a wavefront at once.
template <int LANES, int VPL, bool F32, bool SIGMOID>
__global__ __launch_bounds__(kMaxWaves * kWave) void balance_kernel(BalanceArgs a, int vec) {
  constexpr int kTokens = kWave / LANES;
  __shared__ float s_sum[kMaxWaves][LANES * VPL];
  __shared__ int s_count[LANES * VPL];
  __shared__ int s_live[kMaxWaves];
  __shared__ float s_word[kMaxWaves];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  const int threads = blockDim.x, waves = threads / kWave, step = waves * kTokens;
  const int64_t units = a.seqs * a.parts;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t seq = u / a.parts;
    const int part = (int)(u - seq * a.parts);
    const int64_t begin = seq * a.seq + part * a.per, last = seq * a.seq + a.seq;
    const int64_t end = begin + a.per < last ? begin + a.per : last;
    float x[VPL], next[VPL], none[1];
    auto fetch = [&](int64_t t0) {
      const int64_t t = t0 + tok;
      const bool take = t < end && (!a.token_mask || a.token_mask[t]);
      load_token<LANES, VPL, F32>(a.logits, t * a.pitch, sub, a.E, vec, take, next);
    };
    fetch(begin + wave * kTokens);
    for (int e = threadIdx.x; e < LANES * VPL; e += threads) s_count[e] = 0;
    __syncthreads();

    // slots
    const int slots = (int)(end - begin) * a.k;
    for (int i = threadIdx.x; i < slots; i += threads) {
      const int e = (int)ld4(a.topk_idx + begin * a.k + i);
      const bool live = !a.token_mask || a.token_mask[begin + i / a.k];
      if (live && (uint32_t)e < (uint32_t)a.E) atomicAdd(&s_count[e], 1);
    }
    int live = 0;
    if (a.token_mask) {
      for (int64_t t = begin + threadIdx.x; t - threadIdx.x < end; t += threads)
        live += __builtin_popcountll(__ballot(t < end && a.token_mask[t]));
    }
    if (lane == 0) s_live[wave] = live;

    // shares
    float sum[VPL] = {};
    for (int64_t t0 = begin + wave * kTokens; t0 < end; t0 += step) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] = next[i];
      if (t0 + step < end) fetch(t0 + step);
      const float inv = scores<LANES, VPL, SIGMOID>(x, none);
#pragma unroll
      for (int i = 0; i < VPL; ++i) sum[i] = __builtin_fmaf(x[i], inv, sum[i]);
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      if (LANES == 16) {
        uint32_t b = __float_as_uint(sum[i]);
        b = across32(b, fadd_bits);
        sum[i] = __uint_as_float(across16(b, fadd_bits));
      }
      if (tok == 0) s_sum[wave][expert_of<LANES, VPL, F32>(sub, i)] = sum[i];
    }
    __syncthreads();
    live = (int)(end - begin);
    if (a.token_mask) {
      live = 0;
      for (int w = 0; w < waves; ++w) live += s_live[w];
    }
    auto share_of = [&](int e) {
      float t = s_sum[0][e];
      for (int w = 1; w < waves; ++w) t += s_sum[w][e];
      return t;
    };

    if (a.parts > 1) {
      const int pitch = part_pitch(a.E);
      float* out = a.partial + u * 2 * pitch;
      int* counts = reinterpret_cast<int*>(out + pitch);
      for (int e = threadIdx.x; e < pitch; e += threads) {
        out[e] = e < a.E ? share_of(e) : 0.0f;
        counts[e] = e < a.E ? s_count[e] : 0;
      }
      if (threadIdx.x == 0) {
        a.part_live[u] = live;
        if (part == 0) a.tickets[seq] = 0u;            // the second launch counts from 0
      }
    } else {
      float total = 0.0f, dot = 0.0f;
      const float n = (float)(live > 0 ? live : 1);
      for (int e = threadIdx.x; e < a.E; e += threads) {
        const float mean = share_of(e) / n, count = (float)s_count[e];
        a.expert_count[seq * a.E + e] = s_count[e];
        if (a.mean_score) a.mean_score[seq * a.E + e] = mean;
        total += count;
        dot = __builtin_fmaf(count, mean, dot);
      }
      total = block_sum(total, s_word);
      dot = block_sum(dot, s_word);
      if (threadIdx.x == 0) {
        a.live_tokens[seq] = live;
        if (a.loss) a.loss[seq] = total > 0.0f ? dot * ((float)a.E / total) : 0.0f;
      }
    }
    __syncthreads();                                   // LDS is free
  }
}

// Sums over the parts of a sequence: 32 experts to a workgroup, 32 rows of parts at a
// time in fours of neighbours.  Each leaves its part of the loss, and the last of them adds
// those in their order.  There are two workgroups at least: up to 32 experts the 256 parts that
// a sequence can have are few sums, for the kernel below.
__global__ __launch_bounds__(kBlock) void balance_join_kernel(BalanceArgs a, int blocks) {
  __shared__ float s_sum[kWavesPerBlock][32];
  __shared__ int s_count[kWavesPerBlock][32];
  __shared__ int s_live[kWavesPerBlock];
  const int64_t seq = blockIdx.x / blocks;
  const int block = blockIdx.x - (int)seq * blocks;
  const int pitch = part_pitch(a.E);
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const int quad = threadIdx.x & 7, row = threadIdx.x / 8;
  const float* from = a.partial + seq * a.parts * 2 * pitch + block * 32 + quad * 4;
  float sum[4] = {};
  int count[4] = {}, live = 0;
  for (int p = threadIdx.x; p < a.parts; p += kBlock) live += a.part_live[seq * a.parts + p];
  for (int p0 = row; p0 < a.parts; p0 += 128) {        // four rows asked for together
    u32x4 v[4], c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t p = p0 + i * 32;
      v[i] = p < a.parts ? ld16(from + p * 2 * pitch) : u32x4{0, 0, 0, 0};
      c[i] = p < a.parts ? ld16(from + p * 2 * pitch + pitch) : u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      sum[0] += __uint_as_float(v[i].x);
      sum[1] += __uint_as_float(v[i].y);
      sum[2] += __uint_as_float(v[i].z);
      sum[3] += __uint_as_float(v[i].w);
      count[0] += (int)c[i].x;
      count[1] += (int)c[i].y;
      count[2] += (int)c[i].z;
      count[3] += (int)c[i].w;
    }
  }
  const auto add = [](uint32_t x, uint32_t y) { return x + y; };
#pragma unroll
  for (int j = 0; j < 4; ++j) {                        // over the wavefront's eight rows
    uint32_t b = across16(across32(__float_as_uint(sum[j]), fadd_bits), fadd_bits);
    b = fadd_bits(b, row_rotate<8>(b));
    uint32_t n = across16(across32((uint32_t)count[j], add), add);
    n += row_rotate<8>(n);
    if (lane < 8) {
      s_sum[wave][quad * 4 + j] = __uint_as_float(b);
      s_count[wave][quad * 4 + j] = (int)n;
    }
  }
  live = (int)reduce<64>((uint32_t)live, add);
  if (lane == 0) s_live[wave] = live;
  __syncthreads();
  if (wave > 0) return;                                // one wavefront from here on
  live = s_live[0] + s_live[1] + s_live[2] + s_live[3];
  const int e = block * 32 + lane;
  float total = 0.0f, dot = 0.0f;
  if (lane < 32 && e < a.E) {
    const float t = (((s_sum[0][lane] + s_sum[1][lane]) + s_sum[2][lane]) + s_sum[3][lane]) /
                    (float)(live > 0 ? live : 1);
    const int m = s_count[0][lane] + s_count[1][lane] + s_count[2][lane] + s_count[3][lane];
    a.expert_count[seq * a.E + e] = m;
    if (a.mean_score) a.mean_score[seq * a.E + e] = t;
    total = (float)m;
    dot = total * t;
  }
  total = reduce_sum<64>(total);
  dot = reduce_sum<64>(dot);
  if (lane != 0) return;
  if (block == 0) a.live_tokens[seq] = live;
  if (!a.loss) return;
  float* pieces = a.pieces + seq * blocks * 2;
  __hip_atomic_store(pieces + 2 * block, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __hip_atomic_store(pieces + 2 * block + 1, dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  if (__hip_atomic_fetch_add(a.tickets + seq, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) !=
      (uint32_t)blocks - 1u)
    return;
  total = dot = 0.0f;
  for (int b = 0; b < blocks; ++b) {
    total += __hip_atomic_load(pieces + 2 * b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    dot += __hip_atomic_load(pieces + 2 * b + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  a.loss[seq] = total > 0.0f ? dot * ((float)a.E / total) : 0.0f;
}

// The same by one workgroup a sequence, for few sums: nothing to wait for between workgroups.
constexpr int kJoinThreads = 1024;
__global__ __launch_bounds__(kJoinThreads) void balance_join_one_kernel(BalanceArgs a) {
  __shared__ __attribute__((aligned(16))) float s_sum[kJoinThreads * 4];
  __shared__ __attribute__((aligned(16))) int s_count[kJoinThreads * 4];
  __shared__ float s_word[kJoinThreads / kWave], s_dot[kJoinThreads / kWave];
  __shared__ int s_live;
  const int64_t seq = blockIdx.x;
  const int pitch = part_pitch(a.E), quads = pitch / 4, rows = kJoinThreads / quads;
  const int row = threadIdx.x / quads, quad = threadIdx.x - row * quads;
  const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
  const float* from = a.partial + seq * a.parts * 2 * pitch + quad * 4;
  float sum[4] = {};
  int count[4] = {};
  int live = 0;
  if (wave == 0) {
    for (int p = lane; p < a.parts; p += kWave) live += a.part_live[seq * a.parts + p];
  }
  for (int p0 = row; p0 < a.parts; p0 += 2 * rows) {
    u32x4 v[2] = {}, c[2] = {};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t p = p0 + i * rows;
      if (row < rows && p < a.parts) {
        v[i] = ld16(from + p * 2 * pitch);
        c[i] = ld16(from + p * 2 * pitch + pitch);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[j] += __uint_as_float(v[i][j]);
        count[j] += (int)c[i][j];
      }
  }
  if (row < rows) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s_sum[threadIdx.x * 4 + j] = sum[j];
      s_count[threadIdx.x * 4 + j] = count[j];
    }
  }
  if (wave == 0) {
    live = (int)reduce<64>((uint32_t)live, [](uint32_t x, uint32_t y) { return x + y; });
    if (lane == 0) s_live = live;
  }
  __syncthreads();
  live = s_live;
  float total = 0.0f, dot = 0.0f;
  const int e = threadIdx.x;
  if (e < a.E) {
    float t = 0.0f;
    int m = 0;
    for (int r = 0; r < rows; ++r) {
      t += s_sum[r * pitch + e];
      m += s_count[r * pitch + e];
    }
    t /= (float)(live > 0 ? live : 1);
    a.expert_count[seq * a.E + e] = m;
    if (a.mean_score) a.mean_score[seq * a.E + e] = t;
    total = (float)m;
    dot = total * t;
  }
  total = reduce_sum<64>(total);
  dot = reduce_sum<64>(dot);
  if (lane == 0) {
    s_word[wave] = total;
    s_dot[wave] = dot;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  a.live_tokens[seq] = live;
  if (!a.loss) return;
  for (int w = 1; w < (a.E + 63) / 64; ++w) {
    total += s_word[w];
    dot += s_dot[w];
  }
  a.loss[seq] = total > 0.0f ? dot * ((float)a.E / total) : 0.0f;
}

template <int LANES, int VPL, bool F32, bool SIGMOID>
__global__ __launch_bounds__(kBlock) void balance_backward_kernel(BalanceGradArgs a, int vec) {
  constexpr int kTokens = kWave / LANES, kStep = kWavesPerBlock * kTokens;
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  const int64_t units = a.seqs * a.parts;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t seq = u / a.parts;
    const int64_t begin = seq * a.seq + (u - seq * a.parts) * a.per, last = seq * a.seq + a.seq;
    const int64_t end = begin + a.per < last ? begin + a.per : last;

    float load[VPL], total = 0.0f;                     // f of the lane's experts
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const int e = expert_of<LANES, VPL, F32>(sub, i);
      load[i] = e < a.E ? (float)(int)ld4(a.expert_count + seq * a.E + e) : 0.0f;
      total += load[i];
    }
    total = reduce_sum<LANES>(total);
    const float scale = total > 0.0f ? (float)a.E / total : 0.0f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) load[i] *= scale;
    const int n = (int)ld4(a.live_tokens + seq);
    const float c = __uint_as_float(ld4(a.grad_loss + seq)) / (float)(n > 0 ? n : 1);

    float x[VPL], next[VPL];
    auto fetch = [&](int64_t t0) {
      const int64_t t = t0 + tok;
      const bool take = t < end && (!a.token_mask || a.token_mask[t]);
      load_token<LANES, VPL, F32>(a.logits, t * a.pitch, sub, a.E, vec, take, next);
    };
    fetch(begin + wave * kTokens);
    for (int64_t t0 = begin + wave * kTokens; t0 < end; t0 += kStep) {
      const int64_t t = t0 + tok;
      float rest[SIGMOID ? VPL : 1], add[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] = next[i];
      if (t0 + kStep < end) fetch(t0 + kStep);
      load_token<LANES, VPL, F32>(a.grad_sum, t * a.E, sub, a.E, vec, a.grad_sum && t < end, add);
      const float inv = scores<LANES, VPL, SIGMOID, SIGMOID>(x, rest);
      float dot = 0.0f;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        x[i] *= inv;
        dot = __builtin_fmaf(load[i], x[i], dot);
      }
      dot = reduce_sum<LANES>(dot);
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        // an expert without a share has no gradient
        const float d = x[i] > 0.0f ? c * x[i] * (load[i] - dot) * (SIGMOID ? rest[SIGMOID ? i : 0] : 1.0f) : 0.0f;
        x[i] = a.grad_sum ? add[i] + d : d;
      }
      if (t >= end) continue;
      if constexpr (VPL >= 4) if (vec) {
        constexpr int N = run_of<VPL, F32>();
#pragma unroll
        for (int i = 0; i < VPL; i += N) {
          const int e = expert_of<LANES, VPL, F32>(sub, i);
          if (e >= a.E) continue;
          if constexpr (F32) {
            st16(static_cast<float*>(a.grad_logits) + t * a.E + e,
                 u32x4{__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                       __float_as_uint(x[i + 3])});
          } else {
            uint16_t* to = static_cast<uint16_t*>(a.grad_logits) + t * a.E + e;
            if constexpr (N == 8)
              st16(to, u32x4{pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]),
                             pack_bf16x2(x[i + 4], x[i + 5]), pack_bf16x2(x[i + 6], x[i + 7])});
            else
              st4x2(to, pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]));
          }
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = expert_of<LANES, VPL, F32>(sub, i);
        if (e >= a.E) {
        } else if (F32) {
          static_cast<float*>(a.grad_logits)[t * a.E + e] = x[i];
        } else {
          static_cast<uint16_t*>(a.grad_logits)[t * a.E + e] = (uint16_t)pack_bf16x2(x[i], 0.0f);
        }
      }
    }
  }
}

// launch(lanes, values of a lane, whether float32, whether sigmoid)
template <typename F>
hipError_t by_form(int E, bool f32, bool sigmoid, F&& launch) {
  constexpr std::integral_constant<bool, true> yes;
  constexpr std::integral_constant<bool, false> no;
  return by_width(E, 1, 1, [&](auto lanes, auto vpl) {
    return f32 ? sigmoid ? launch(lanes, vpl, yes, yes) : launch(lanes, vpl, yes, no)
               : sigmoid ? launch(lanes, vpl, no, yes) : launch(lanes, vpl, no, no);
  });
}

unsigned unit_blocks(int64_t seqs, int parts) {
  const int64_t units = seqs * parts;
  return (unsigned)(units < kMaxGrid ? units : kMaxGrid);
}

}  // namespace

// Tokens that a workgroup of `waves` wavefronts has at once.
static int64_t tokens_at_once(int E, int waves) { return waves * (E <= 256 ? 4 : 1); }

// Values that a lane has of a token (by_width).
static int values_of_lane(int E) {
  int n = E <= 256 ? 1 : E <= 512 ? 8 : 16;
  while (E <= 256 && 16 * n < E) n *= 2;
  return n;
}

// A workgroup of 16 wavefronts for each compute unit: 32768 x 256 in 8 sequences 13.5 us, with
// twice or half as many 19.0 and 17.7; 16384 x 512 15.9, so 20.4 and 19.6.  A sequence of few rounds
// of tokens has one workgroup, which saves the second launch: us by one and by two launches
//   rounds            2             4             6             8
//   16 experts     5.0 / 8.8     5.8 / 8.9     6.6 / 9.0     7.3 / 8.8
//   64             6.2 / 8.5     7.7 / 9.0     9.3 / 9.1    10.7 / 8.8
//   256            9.8 / 10.6   14.3 / 10.6   18.8 / 10.8   23.1 / 10.8
//   512            7.4 / 9.4     9.9 / 9.5    12.4 / 9.6    15.1 / 9.8
//   1000           9.4 / 10.2   14.0 / 10.4   18.5 / 10.9   23.0 / 11.0
// where a round takes about as long as its values of a lane and two; up to 36 of that in one.
// More than 128 sequences have one each whatever their length: 128 of 256 x 256 13.3, 129 15.1,
// 255 16.9, 257, in two rounds, 28.9.
BalanceShape balance_shape(int64_t T, int E, int64_t seq) {
  BalanceShape s;
  s.seq = seq ? seq : T;
  s.seqs = seq ? T / seq : 1;
  const int64_t step = tokens_at_once(E, kMaxWaves);
  int64_t parts = (s.seq + step - 1) / step;
  const int64_t most = 256 / (s.seqs > 0 ? s.seqs : 1);
  parts = parts < most ? parts : most;
  if (s.seq <= 36 / (values_of_lane(E) + 2) * step || parts < 1) parts = 1;
  s.per = ((s.seq + parts - 1) / parts + step - 1) / step * step;
  s.parts = s.seq > 0 ? (int)((s.seq + s.per - 1) / s.per) : 1;
  const int64_t a_wave = step / kMaxWaves, longest = s.seq < s.per ? s.seq : s.per;
  const int64_t waves = (longest + a_wave - 1) / a_wave;
  s.waves = (int)(waves < 1 ? 1 : waves < kMaxWaves ? waves : kMaxWaves);
  s.blocks = (E + 31) / 32;
  s.live_at = s.parts > 1 ? (size_t)s.seqs * s.parts * 2 * part_pitch(E) * 4 : 0;
  s.ticket_at = s.live_at + (s.parts > 1 ? (size_t)s.seqs * s.parts * 4 : 0);
  s.piece_at = s.ticket_at + (s.parts > 1 ? (size_t)s.seqs * 4 : 0);
  s.bytes = s.piece_at + (s.parts > 1 ? (size_t)s.seqs * s.blocks * 8 : 0);
  return s;
}

// The gradient's parts leave nothing behind: about 768 workgroups of four wavefronts, each
// with up to eight rounds of tokens (us with one, two, four, eight rounds: 32768 x 128 bf16 13.0,
// 9.8, 8.8, 10.5 and by the rule's three 9.7; 16384 x 512 17.0, 14.5, 13.1, 13.8, by its six 13.4;
// 2048 x 384 4.3, 4.6, 6.2, 9.1).
void balance_grad_parts(BalanceGradArgs& a) {
  const int64_t step = tokens_at_once(a.E, kWavesPerBlock);
  const int64_t all = a.seqs * ((a.seq + step - 1) / step), rounds = (all + 767) / 768;
  a.per = step * (rounds < 8 ? rounds : 8);
  a.parts = (int)((a.seq + a.per - 1) / a.per);
}

hipError_t launch_balance(const BalanceArgs& a, const BalanceShape& shape, hipStream_t stream) {
  const hipError_t err = by_form(a.E, a.f32, a.sigmoid, [&](auto lanes, auto vpl, auto f32,
                                                            auto sigmoid) {
    constexpr int run = run_of<vpl.value, f32.value>();
    const int vec = vector_rows(a.logits, nullptr, a.pitch, a.E, run, f32.value);
    hipLaunchKernelGGL((balance_kernel<lanes.value, vpl.value, f32.value, sigmoid.value>),
                       dim3(unit_blocks(a.seqs, a.parts)), dim3(shape.waves * kWave), 0, stream, a,
                       vec);
    return hipGetLastError();
  });
  if (err != hipSuccess || a.parts == 1) return err;
  // Up to 8192 sums a sequence one workgroup joins them sooner (us by one and by several: 16
  // sequences of 16 parts of 256 experts 13.1 and 16.1, 8 of 32 13.2 and 14.7, one of 128 parts of
  // 64 10.0 and 9.9, of 256 parts of 64 11.1 and 10.7; 4 of 64 parts of 256 13.6 and 14.5, one of
  // 256 of them 18.4 and 14.7).
  if (a.parts * part_pitch(a.E) <= 8192) {
    hipLaunchKernelGGL(balance_join_one_kernel, dim3((unsigned)a.seqs), dim3(kJoinThreads), 0,
                       stream, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(balance_join_kernel, dim3((unsigned)(a.seqs * shape.blocks)), dim3(kBlock), 0,
                     stream, a, shape.blocks);
  return hipGetLastError();
}

hipError_t launch_balance_backward(const BalanceGradArgs& a, hipStream_t stream) {
  return by_form(a.E, a.f32, a.sigmoid, [&](auto lanes, auto vpl, auto f32, auto sigmoid) {
    constexpr int run = run_of<vpl.value, f32.value>();
    const int vec = vector_rows(a.logits, a.grad_logits, a.pitch, a.E, run, f32.value) &&
                    vector_rows(a.grad_sum, nullptr, a.E, a.E, run, f32.value);
    hipLaunchKernelGGL((balance_backward_kernel<lanes.value, vpl.value, f32.value, sigmoid.value>),
                       dim3(unit_blocks(a.seqs, a.parts)), dim3(kBlock), 0, stream, a, vec);
    return hipGetLastError();
  });
}

}  // namespace moe
