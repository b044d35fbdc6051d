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
// over the part's tokens, the slots are counted in LDS.  A second launch adds the parts, 32
// experts to a workgroup; the last workgroup of a sequence adds the loss.  Sequences of
// one part need no second launch.

#include "logits.h"

namespace moe {
namespace {

// A token's dealt logits; -inf where the token takes no part.
template <int LANES, int VPL>
__device__ __forceinline__ void load_token(const void* logits, bool f32, int64_t at, int sub, int E,
                                           int vec, bool take, float (&x)[VPL]) {
#pragma unroll
  for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
  if (!take) return;
  constexpr int N = VPL >= 4 ? 4 : VPL;
#pragma unroll
  for (int g = 0; g < VPL / N; ++g) {
    float v[N];
    load_logits<N>(logits, f32, at, dealt<LANES, VPL>(sub, g * N), E, vec, v);
#pragma unroll
    for (int j = 0; j < N; ++j) x[g * N + j] = v[j];
  }
}

// Scores in place of the logits, and the factor that makes shares of them: 0 where their sum
// is none, or lies below float32's normal range (sigmoid scores of very low logits).
template <int LANES, int VPL, bool SIGMOID>
__device__ __forceinline__ float scores(float (&x)[VPL]) {
  float local = 0.0f;
  if constexpr (SIGMOID) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = x[i] > -INFINITY ? sigmoid(x[i]) : 0.0f;
  } else {
    const float m = row_max<LANES, VPL>(x);
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = exp_term(x[i], m);
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) local += x[i];
  const float total = reduce_sum<LANES>(local);
  return total >= 0x1p-126f ? 1.0f / total : 0.0f;
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

template <int LANES, int VPL, bool SIGMOID>
__global__ __launch_bounds__(kBlock) void balance_kernel(BalanceArgs a, int vec) {
  constexpr int kTokens = kWave / LANES, kStep = kWavesPerBlock * kTokens;
  __shared__ float s_sum[kWavesPerBlock][LANES * VPL];
  __shared__ int s_count[LANES * VPL];
  __shared__ int s_live[kWavesPerBlock];
  __shared__ float s_word[kWavesPerBlock];
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  const int64_t units = a.seqs * a.parts;
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int64_t seq = u / a.parts;
    const int part = (int)(u - seq * a.parts);
    const int64_t begin = seq * a.seq + part * a.per, last = seq * a.seq + a.seq;
    const int64_t end = begin + a.per < last ? begin + a.per : last;
    for (int e = threadIdx.x; e < LANES * VPL; e += kBlock) s_count[e] = 0;
    __syncthreads();

    // slots
    const int slots = (int)(end - begin) * a.k;
    for (int i = threadIdx.x; i < slots; i += kBlock) {
      const int e = (int)ld4(a.topk_idx + begin * a.k + i);
      const bool live = !a.token_mask || a.token_mask[begin + i / a.k];
      if (live && (uint32_t)e < (uint32_t)a.E) atomicAdd(&s_count[e], 1);
    }
    int live = 0;
    if (a.token_mask) {
      for (int64_t t = begin + threadIdx.x; t - threadIdx.x < end; t += kBlock)
        live += __builtin_popcountll(__ballot(t < end && a.token_mask[t]));
    }
    if (lane == 0) s_live[wave] = live;

    // shares
    float sum[VPL] = {};
    float x[VPL], next[VPL];
    auto fetch = [&](int64_t t0) {
      const int64_t t = t0 + tok;
      const bool take = t < end && (!a.token_mask || a.token_mask[t]);
      load_token<LANES, VPL>(a.logits, a.f32, t * a.pitch, sub, a.E, vec, take, next);
    };
    fetch(begin + wave * kTokens);
    for (int64_t t0 = begin + wave * kTokens; t0 < end; t0 += kStep) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] = next[i];
      if (t0 + kStep < end) fetch(t0 + kStep);
      const float inv = scores<LANES, VPL, SIGMOID>(x);
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
      if (tok == 0) s_sum[wave][dealt<LANES, VPL>(sub, i)] = sum[i];
    }
    __syncthreads();
    live = a.token_mask ? s_live[0] + s_live[1] + s_live[2] + s_live[3] : (int)(end - begin);

    if (a.parts > 1) {
      const int pitch = part_pitch(a.E);
      float* out = a.partial + u * 2 * pitch;
      int* counts = reinterpret_cast<int*>(out + pitch);
      for (int e = threadIdx.x; e < pitch; e += kBlock) {
        out[e] = e < a.E ? ((s_sum[0][e] + s_sum[1][e]) + s_sum[2][e]) + s_sum[3][e] : 0.0f;
        counts[e] = e < a.E ? s_count[e] : 0;
      }
      if (threadIdx.x == 0) {
        a.part_live[u] = live;
        if (part == 0) a.tickets[seq] = 0u;            // the second launch counts from 0
      }
    } else {
      float total = 0.0f, dot = 0.0f;
      const float n = (float)(live > 0 ? live : 1);
      for (int e = threadIdx.x; e < a.E; e += kBlock) {
        const float share = ((s_sum[0][e] + s_sum[1][e]) + s_sum[2][e]) + s_sum[3][e];
        const float count = (float)s_count[e];
        a.expert_count[seq * a.E + e] = s_count[e];
        if (a.mean_score) a.mean_score[seq * a.E + e] = share / n;
        total += count;
        dot = __builtin_fmaf(count, share / n, dot);
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

// Sums over the parts of a sequence: 32 experts to a workgroup, 128 rows of parts at a
// time in fours of neighbours.  Each leaves its part of the loss, and the last of them adds
// those in their order.
__global__ __launch_bounds__(1024) void balance_join_kernel(BalanceArgs a, int blocks) {
  __shared__ float s_sum[128][33];
  __shared__ int s_count[128][33];
  __shared__ int s_live[16];
  __shared__ uint32_t s_order;
  const int64_t seq = blockIdx.x / blocks;
  const int block = blockIdx.x - (int)seq * blocks;
  const int pitch = part_pitch(a.E);
  const int quad = threadIdx.x & 7, row = threadIdx.x / 8;
  const float* from = a.partial + seq * a.parts * 2 * pitch + block * 32 + quad * 4;
  float sum[4] = {};
  int count[4] = {}, live = 0;
  for (int p = row; p < a.parts; p += 128) {
    const u32x4 v = ld16(from + (int64_t)p * 2 * pitch);
    const u32x4 c = ld16(from + (int64_t)p * 2 * pitch + pitch);
    sum[0] += __uint_as_float(v.x);
    sum[1] += __uint_as_float(v.y);
    sum[2] += __uint_as_float(v.z);
    sum[3] += __uint_as_float(v.w);
    count[0] += (int)c.x;
    count[1] += (int)c.y;
    count[2] += (int)c.z;
    count[3] += (int)c.w;
  }
  for (int p = threadIdx.x; p < a.parts; p += 1024) live += a.part_live[seq * a.parts + p];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s_sum[row][quad * 4 + j] = sum[j];
    s_count[row][quad * 4 + j] = count[j];
  }
  live = (int)reduce<64>((uint32_t)live, [](uint32_t x, uint32_t y) { return x + y; });
  if ((threadIdx.x & 63) == 0) s_live[threadIdx.x / 64] = live;
  __syncthreads();
  live = 0;
  for (int w = 0; w < 16; ++w) live += s_live[w];
  const int c = threadIdx.x & 31, part = threadIdx.x / 32;   // 32 parts of four rows
  float t = 0.0f;
  int m = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    t += s_sum[part * 4 + j][c];
    m += s_count[part * 4 + j][c];
  }
  __syncthreads();
  s_sum[part][c] = t;
  s_count[part][c] = m;
  __syncthreads();
  if (threadIdx.x < kWave) {                           // one wavefront from here on
    const int e = block * 32 + c;
    float total = 0.0f, dot = 0.0f;
    if (threadIdx.x < 32 && e < a.E) {
      t = 0.0f;
      m = 0;
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        t += s_sum[j][c];
        m += s_count[j][c];
      }
      t /= (float)(live > 0 ? live : 1);
      a.expert_count[seq * a.E + e] = m;
      if (a.mean_score) a.mean_score[seq * a.E + e] = t;
      total = (float)m;
      dot = total * t;
    }
    total = reduce_sum<64>(total);
    dot = reduce_sum<64>(dot);
    float* piece = a.pieces + (seq * blocks + block) * 2;
    if (threadIdx.x == 0) {
      if (block == 0) a.live_tokens[seq] = live;
      __hip_atomic_store(piece, total, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(piece + 1, dot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      s_order = __hip_atomic_fetch_add(a.tickets + seq, 1u, __ATOMIC_ACQ_REL,
                                       __HIP_MEMORY_SCOPE_AGENT);
    }
    if (threadIdx.x == 0 && a.loss && s_order == (uint32_t)blocks - 1u) {
      total = dot = 0.0f;
      piece = a.pieces + seq * blocks * 2;
      for (int b = 0; b < blocks; ++b) {
        total += __hip_atomic_load(piece + 2 * b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        dot += __hip_atomic_load(piece + 2 * b + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      a.loss[seq] = total > 0.0f ? dot * ((float)a.E / total) : 0.0f;
    }
  }
}

template <int LANES, int VPL, bool SIGMOID>
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
      const int e = dealt<LANES, VPL>(sub, i);
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
      load_token<LANES, VPL>(a.logits, a.f32, t * a.pitch, sub, a.E, vec, take, next);
    };
    fetch(begin + wave * kTokens);
    for (int64_t t0 = begin + wave * kTokens; t0 < end; t0 += kStep) {
      const int64_t t = t0 + tok;
      float rest[VPL], add[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        x[i] = next[i];
        if (SIGMOID) rest[i] = sigmoid(-x[i]);         // 1 - s, also where s rounds to 1
      }
      if (t0 + kStep < end) fetch(t0 + kStep);
      load_token<LANES, VPL>(a.grad_sum, a.f32, t * a.E, sub, a.E, vec, a.grad_sum && t < end, add);
      const float inv = scores<LANES, VPL, SIGMOID>(x);
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
        const float d = x[i] > 0.0f ? c * x[i] * (load[i] - dot) * (SIGMOID ? rest[i] : 1.0f) : 0.0f;
        x[i] = a.grad_sum ? add[i] + d : d;
      }
      if (t >= end) continue;
      if constexpr (VPL >= 4) if (vec) {
#pragma unroll
        for (int i = 0; i < VPL; i += 4) {
          const int e = dealt<LANES, VPL>(sub, i);
          if (e >= a.E) continue;
          if (a.f32)
            st16(static_cast<float*>(a.grad_logits) + t * a.E + e,
                 u32x4{__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                       __float_as_uint(x[i + 3])});
          else
            st4x2(static_cast<uint16_t*>(a.grad_logits) + t * a.E + e, pack_bf16x2(x[i], x[i + 1]),
                  pack_bf16x2(x[i + 2], x[i + 3]));
        }
        continue;
      }
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const int e = dealt<LANES, VPL>(sub, i);
        if (e >= a.E) {
        } else if (a.f32) {
          static_cast<float*>(a.grad_logits)[t * a.E + e] = x[i];
        } else {
          static_cast<uint16_t*>(a.grad_logits)[t * a.E + e] = (uint16_t)pack_bf16x2(x[i], 0.0f);
        }
      }
    }
  }
}

template <typename F>
hipError_t by_score(bool sigmoid, F&& launch) {
  return sigmoid ? launch(std::integral_constant<bool, true>())
                 : launch(std::integral_constant<bool, false>());
}

unsigned unit_blocks(int64_t seqs, int parts) {
  const int64_t units = seqs * parts;
  return (unsigned)(units < kMaxGrid ? units : kMaxGrid);
}

}  // namespace

BalanceShape balance_shape(int64_t T, int E, int64_t seq) {
  BalanceShape s;
  s.seq = seq ? seq : T;
  s.seqs = seq ? T / seq : 1;
  const int64_t step = E <= 256 ? 16 : 4;              // tokens that a workgroup has at once
  int64_t parts = (s.seq + 4 * step - 1) / (4 * step);
  const int64_t most = 1024 / (s.seqs > 0 ? s.seqs : 1);
  parts = parts < most ? parts : most;
  parts = parts > 1 ? parts : 1;
  s.per = ((s.seq + parts - 1) / parts + step - 1) / step * step;
  s.parts = s.seq > 0 ? (int)((s.seq + s.per - 1) / s.per) : 1;
  s.blocks = (E + 31) / 32;
  s.live_at = s.parts > 1 ? (size_t)s.seqs * s.parts * 2 * part_pitch(E) * 4 : 0;
  s.ticket_at = s.live_at + (s.parts > 1 ? (size_t)s.seqs * s.parts * 4 : 0);
  s.piece_at = s.ticket_at + (s.parts > 1 ? (size_t)s.seqs * 4 : 0);
  s.bytes = s.piece_at + (s.parts > 1 ? (size_t)s.seqs * s.blocks * 8 : 0);
  return s;
}

hipError_t launch_balance(const BalanceArgs& a, int blocks, hipStream_t stream) {
  const hipError_t err = by_width(a.E, 1, 1, [&](auto lanes, auto vpl) {
    return by_score(a.sigmoid, [&](auto sigmoid) {
      const int vec = vpl.value >= 4 && vector_rows(a.logits, nullptr, a.pitch, a.E, 4, a.f32);
      hipLaunchKernelGGL((balance_kernel<lanes.value, vpl.value, sigmoid.value>),
                         dim3(unit_blocks(a.seqs, a.parts)), dim3(kBlock), 0, stream, a, vec);
      return hipGetLastError();
    });
  });
  if (err != hipSuccess || a.parts == 1) return err;
  hipLaunchKernelGGL(balance_join_kernel, dim3((unsigned)(a.seqs * blocks)), dim3(1024), 0, stream, a,
                     blocks);
  return hipGetLastError();
}

hipError_t launch_balance_backward(const BalanceGradArgs& a, hipStream_t stream) {
  return by_width(a.E, 1, 1, [&](auto lanes, auto vpl) {
    return by_score(a.sigmoid, [&](auto sigmoid) {
      const int vec = vpl.value >= 4 &&
                      vector_rows(a.logits, a.grad_logits, a.pitch, a.E, 4, a.f32) &&
                      vector_rows(a.grad_sum, nullptr, a.E, a.E, 4, a.f32);
      hipLaunchKernelGGL((balance_backward_kernel<lanes.value, vpl.value, sigmoid.value>),
                         dim3(unit_blocks(a.seqs, a.parts)), dim3(kBlock), 0, stream, a, vec);
      return hipGetLastError();
    });
  });
}

}  // namespace moe
