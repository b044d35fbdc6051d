// Routing: the k experts of each token with their weights, and the gradient
// of the weights with respect to the logits.
//
// One token takes LANES (16 or 64) neighbouring lanes of a wavefront, each with
// VPL neighbouring experts in registers.  Keys are the floats' bit patterns made to
// order as unsigned integers, so a maximum over lanes is one DPP instruction
// per step; equal keys go to the lowest index.  With few experts to a lane the k
// winners are found one after another as the largest key left, with many by a
// threshold that hardly more than k keys pass.  The softmax's sum is needed only where
// weights are not renormalised or scores are the keys: renormalised weights
// are a softmax over the k winners' logits.  All of it is float32, the sum in a
// fixed order, so equal inputs give equal keys.
//
// A batch is read once and little is written, but neither bounds it.  Up to about
// 4096 tokens it is the launch and the chain of one token's steps: 3.5 to 5 us where
// logits are the keys, 7 to 8.5 with scores, a bias and groups.  Beyond that the
// instructions of a token: 16384 tokens, 256 float32 logits, 8 slots (17.8 MB) 6.5 us with
// logits as keys, 9.7 with sigmoid scores and a bias, 11.8 with 4 of 8 groups
// besides.  The gradient of 32768 x 128 bf16 softmax logits (18.9 MB): 7.3 us.

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

// The two highest of a group's keys, over the lanes that share it.
struct TopTwo {
  float best, second;
  __device__ __forceinline__ void add(float b, float s) {
    second = fmaxf(fminf(best, b), fmaxf(second, s));
    best = fmaxf(best, b);
  }
  template <int CTRL>
  __device__ __forceinline__ void from_lane() {       // DPP exchange between lanes
    const int b = __float_as_int(best), s = __float_as_int(second);
    add(__int_as_float(__builtin_amdgcn_update_dpp(b, b, CTRL, 0xf, 0xf, false)),
        __int_as_float(__builtin_amdgcn_update_dpp(s, s, CTRL, 0xf, 0xf, false)));
  }
};

// Half the sum of the two highest: it orders as the sum does, which may lie outside
// float32 (two biases of the lowest value), where a group with eligible experts would
// look like one without.
__device__ __forceinline__ float group_key(const TopTwo& g, int group_top) {
  if (group_top == 1) return g.best;
  return 0.5f * g.best + (g.second > -INFINITY ? 0.5f * g.second : 0.0f);
}

// Groups of whole lanes, a power of two of them, that fill the token's 16 lanes
// (256 experts in 8 groups: two lanes each): keys of the groups that do not
// take part become -inf, by exchanges between lanes.
template <int VPL>
__device__ __forceinline__ void keep_lane_groups(const RouteArgs& a, int sub, float (&kf)[VPL]) {
  const int lanes = 16 / a.groups;
  TopTwo g = {-INFINITY, -INFINITY};
#pragma unroll
  for (int i = 0; i < VPL; ++i) g.add(kf[i], -INFINITY);
  if (lanes > 1) g.from_lane<0xB1>();               // lane ^ 1
  if (lanes > 2) g.from_lane<0x4E>();               // lane ^ 2
  if (lanes > 4) g.from_lane<0x141>();              // the other four of eight
  if (lanes > 8) g.from_lane<0x140>();              // the other eight
  const float key = group_key(g, a.group_top);
  const uint32_t own = order_key(key);
  // lanes of better groups, and of equal ones before this; each counts as often
  // as a group has lanes
  int better = 0;
  const int shift = __builtin_ctz((unsigned)lanes), group = sub >> shift;
  auto look = [&](uint32_t other, int n) {
    const bool before = ((sub - n) & 15) >> shift < group;
    better += other >= own + (before ? 0u : 1u);
  };
#define MOE_LOOK(N) look(row_rotate<N>(own), N);
  MOE_LOOK(1) MOE_LOOK(2) MOE_LOOK(3) MOE_LOOK(4) MOE_LOOK(5) MOE_LOOK(6) MOE_LOOK(7) MOE_LOOK(8)
  MOE_LOOK(9) MOE_LOOK(10) MOE_LOOK(11) MOE_LOOK(12) MOE_LOOK(13) MOE_LOOK(14) MOE_LOOK(15)
#undef MOE_LOOK
  const bool keep = key > -INFINITY && better < a.top_groups * lanes;
#pragma unroll
  for (int i = 0; i < VPL; ++i) kf[i] = keep ? kf[i] : -INFINITY;
}

// The same for any groups; `mine`: the keys in LDS.  Of a whole wavefront up to 16
// lanes look over each group (7638 tokens, 512 bf16 logits in 4 groups, one slot, 9.7 us,
// by one lane 16.5; 16384, 512 scores with a bias in 8, 8 slots, 28.6 and 33.5), of 16 lanes
// one (16384 tokens, 160 logits in 8 groups 11 us, by two 14.0).
template <int LANES, int VPL>
__device__ __forceinline__ void keep_groups(const RouteArgs& a, int sub, int tok, float* mine,
                                            float (&kf)[VPL]) {
  const int e0 = sub * VPL, size = a.E / a.groups;
  const int most = 31 - __builtin_clz((unsigned)(LANES / a.groups));
  const int shift = LANES == 16 ? 0 : most < 4 ? most : 4;
  const int lanes = 1 << shift, group = sub >> shift, part = sub & (lanes - 1);
  TopTwo g = {-INFINITY, -INFINITY};
  if (group < a.groups) {
    const float* from = mine + group * size;
    int i = part;
    for (; i + 3 * lanes < size; i += 4 * lanes) {
      const float v[4] = {from[i], from[i + lanes], from[i + 2 * lanes], from[i + 3 * lanes]};
#pragma unroll
      for (int j = 0; j < 4; ++j) g.add(v[j], -INFINITY);
    }
    for (; i < size; i += lanes) g.add(from[i], -INFINITY);
  }
  if (lanes > 1) g.from_lane<0xB1>();               // as above
  if (lanes > 2) g.from_lane<0x4E>();
  if (lanes > 4) g.from_lane<0x141>();
  if (lanes > 8) g.from_lane<0x140>();
  const float key = group_key(g, a.group_top);
  wave_order();
  if (group < a.groups && part == 0) mine[group] = key;
  wave_order();
  int rank = 0;
  for (int n = 0; n < a.groups; ++n) {
    const float v = mine[n];
    rank += v > key || (v == key && n < group);
  }
  const uint64_t kept =
      __ballot(group < a.groups && key > -INFINITY && rank < a.top_groups) >> (tok * LANES);
  int n = e0 / size, r = e0 - n * size;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    if (n >= a.groups || !((kept >> (n << shift)) & 1)) kf[i] = -INFINITY;
    if (++r == size) {
      r = 0;
      ++n;
    }
  }
  wave_order();
}

// Slot `sub`'s expert, or -1: the k highest keys one after another.
template <int LANES, int VPL>
__device__ __forceinline__ int winners_in_turn(int k, int sub, uint32_t (&key)[VPL]) {
  const int e0 = sub * VPL;
  int won = -1;
  for (int j = 0; j < k; ++j) {
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
  return won;
}

constexpr int kCandidates = 64;

// Candidates of a token in LDS, in the order of their experts.
struct Candidates {
  uint32_t key[kCandidates];
  uint16_t expert[kCandidates];
  int16_t slot[MOE_MAX_K];
};

// The same by a threshold: the k-th highest of the lanes' own maxima.  The k
// winners are at least as high, few others are; they are collected in LDS and
// each counts those above it.  Returns false, for the whole wavefront, where a
// token has more than kCandidates (equal keys, few lanes left).
template <int LANES, int VPL, int PARTS>
__device__ __forceinline__ bool winners_by_threshold(int k, int sub, const uint32_t (&key)[VPL],
                                                     const uint32_t* mine, Candidates* c,
                                                     int& won) {
  const int e0 = sub * VPL;
  uint32_t least;
  if constexpr (LANES == 16) {
    // PARTS maxima of a lane: with groups left out half the lanes have none, and
    // half a lane's are needed for k high ones
    constexpr int PER = VPL / PARTS;
    uint32_t top[PARTS] = {};
    int above[PARTS] = {};
#pragma unroll
    for (int p = 0; p < PARTS; ++p)
#pragma unroll
      for (int i = 0; i < PER; ++i) top[p] = umax(top[p], key[p * PER + i]);
    auto look = [&](uint32_t other) {
#pragma unroll
      for (int p = 0; p < PARTS; ++p) above[p] += other > top[p];
    };
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      if (PARTS > 1) look(top[p]);
#define MOE_LOOK(N) look(row_rotate<N>(top[p]));
      MOE_LOOK(1) MOE_LOOK(2) MOE_LOOK(3) MOE_LOOK(4) MOE_LOOK(5) MOE_LOOK(6) MOE_LOOK(7)
      MOE_LOOK(8) MOE_LOOK(9) MOE_LOOK(10) MOE_LOOK(11) MOE_LOOK(12) MOE_LOOK(13) MOE_LOOK(14)
      MOE_LOOK(15)
#undef MOE_LOOK
    }
    least = ~0u;
#pragma unroll
    for (int p = 0; p < PARTS; ++p) least = above[p] < k ? umin(least, top[p]) : least;
  } else {
    uint32_t left = 0;
#pragma unroll
    for (int i = 0; i < VPL; ++i) left = umax(left, key[i]);
    least = ~0u;
    for (int seen = 0; seen < k;) {                   // the same in every lane
      const uint32_t m = reduce_max<LANES>(left);
      const bool is = left == m;
      least = m;
      if (m == 0) break;
      left = is ? 0u : left;
      seen += __builtin_popcountll(__ballot(is));
    }
  }
  least = reduce_min<LANES>(least);
  least = umax(least, 1u);                            // eligible ones only
  uint32_t mask = 0;
#pragma unroll
  for (int i = 0; i < VPL; ++i) mask |= key[i] >= least ? 1u << i : 0u;
  const int count = __builtin_popcount(mask);
  uint32_t end = (uint32_t)count;                     // inclusive over the token's lanes
  end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x111, 0xf, 0xf, true);
  end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x112, 0xf, 0xf, true);
  end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x114, 0xf, 0xf, true);
  end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x118, 0xf, 0xf, true);
  if (LANES == 64) {
    end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x142, 0xa, 0xf, false);
    end += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)end, 0x143, 0xc, 0xf, false);
  }
  const int n = (int)reduce_max<LANES>(end);
  if (__ballot(n > kCandidates)) return false;
  for (int p = (int)end - count; mask; ++p, mask &= mask - 1) {
    const int e = e0 + __builtin_ctz(mask);
    c->key[p] = mine[e];
    c->expert[p] = (uint16_t)e;
  }
  if (sub < 4 && n + sub < kCandidates) c->key[n + sub] = 0;   // read in fours below
  if (sub < k) c->slot[sub] = -1;
  wave_order();
  for (int p = sub; p < n; p += LANES) {
    const uint32_t own = c->key[p];
    int rank = 0;
    for (int q = 0; q < n; q += 4) {                  // equal keys: the earlier one first
      const u32x4 o = *reinterpret_cast<const u32x4*>(&c->key[q]);
      rank += o.x >= own + (q >= p);
      rank += o.y >= own + (q + 1 >= p);
      rank += o.z >= own + (q + 2 >= p);
      rank += o.w >= own + (q + 3 >= p);
    }
    if (rank < k) c->slot[rank] = (int16_t)c->expert[p];
  }
  wave_order();
  won = sub < k ? c->slot[sub] : -1;
  return true;
}

// What the experts are ordered by: the logits, scores (+ bias), or the logits
// with the softmax's sum taken for the weights.  Kernels of their own: what
// each needs beyond the others costs it microseconds.
enum Groups : int { kOneGroup = 0, kLaneGroups = 1, kAnyGroups = 2 };
enum Keys : int { kLogits = 0, kSigmoidKeys = 1, kSoftmaxKeys = 2, kSoftmaxSum = 3 };

// From eight experts to a lane on the threshold is the faster way (16384
// tokens, 256 experts, 8 slots 9.0 -> 6.6 us; 32768 tokens, 128 experts 9.5 -> 8.2;
// four to a lane: equal).  Up to two slots are found in turn.
constexpr bool by_threshold(int vpl) { return vpl >= 8; }

// Route token t: lane `sub` of its LANES, `tok` its place in the wavefront,
// `mine` and `c` its LDS.  Every lane of the wavefront takes part.
template <int LANES, int VPL, Keys KEYS, Groups GROUPS>
__device__ __forceinline__ void route_token(const RouteArgs& a, int vec, int64_t t, int sub,
                                            int tok, float* mine, Candidates* c) {
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

  // x becomes the keys
  float m = 0.0f, total = 1.0f;
  if constexpr (KEYS == kSigmoidKeys) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = x[i] > -INFINITY ? sigmoid(x[i]) : -INFINITY;
  }
  if constexpr (KEYS == kSoftmaxKeys || KEYS == kSoftmaxSum) {
    m = row_max<LANES, VPL>(x);
    float s[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) s[i] = exp_term(x[i], m);
    total = fold<LANES, VPL>(s);
    if (!(total > 0.0f)) total = 1.0f;
    if constexpr (KEYS == kSoftmaxKeys) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] = x[i] > -INFINITY ? s[i] / total : -INFINITY;
    }
  }
  if constexpr (KEYS == kSigmoidKeys || KEYS == kSoftmaxKeys) {
    if (a.bias) {
      float b[VPL];
      load_logits<VPL>(a.bias, true, 0, e0, a.E, vec && (uintptr_t)a.bias % 16 == 0, b);
#pragma unroll
      for (int i = 0; i < VPL; ++i) x[i] += b[i];
    }
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) x[i] = x[i] > -INFINITY ? x[i] : -INFINITY;   // NaN too

  constexpr bool kThreshold = by_threshold(VPL);
  uint32_t key[VPL];
  if constexpr (GROUPS == kLaneGroups) {
    keep_lane_groups<VPL>(a, sub, x);
  } else if constexpr (GROUPS == kAnyGroups) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) mine[e0 + i] = x[i];
    wave_order();
    keep_groups<LANES, VPL>(a, sub, tok, mine, x);
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) key[i] = x[i] > -INFINITY ? order_key(x[i]) : 0u;

  int won = -1;                                   // slot `sub`'s expert
  bool found = false;
  if constexpr (kThreshold) {
    if (a.k > 2) {
      uint32_t* keys = reinterpret_cast<uint32_t*>(mine);
#pragma unroll
      for (int i = 0; i < VPL; ++i) keys[e0 + i] = key[i];
      wave_order();
      found = winners_by_threshold<LANES, VPL, GROUPS == kOneGroup ? 1 : 2>(a.k, sub, key, keys, c,
                                                                            won);
    }
  }
  if (!found) won = winners_in_turn<LANES, VPL>(a.k, sub, key);

  // weights: lane j of the token has slot j
  float w = 0.0f;
  const bool slot = in && sub < a.k;
  float xw = -INFINITY;
  if (won >= 0) xw = logit_at(a.logits, a.f32, t * a.pitch + won);
  if (a.sigmoid) {
    w = won >= 0 ? sigmoid(xw) : 0.0f;
  } else if ((KEYS == kSoftmaxKeys || KEYS == kSoftmaxSum) && !a.renorm) {
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

template <int LANES, int VPL, Keys KEYS, Groups GROUPS>
__global__ __launch_bounds__(kBlock, GROUPS == kAnyGroups || VPL == 16 ? 2 : 4)
void route_kernel(RouteArgs a, int vec) {
  constexpr int kTokens = kWave / LANES;         // of a wavefront
  __shared__ __attribute__((aligned(16))) float s_key[kWavesPerBlock][kTokens][LANES * VPL];
  constexpr bool kThreshold = by_threshold(VPL);
  __shared__ __attribute__((aligned(16)))
  Candidates s_candidates[kThreshold ? kWavesPerBlock : 1][kThreshold ? kTokens : 1];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWavesPerBlock + wave) * kTokens; t0 < a.tokens;
       t0 += (int64_t)gridDim.x * kWavesPerBlock * kTokens)
    route_token<LANES, VPL, KEYS, GROUPS>(
        a, vec, t0 + tok, sub, tok, s_key[wave][tok],
        &s_candidates[kThreshold ? wave : 0][kThreshold ? tok : 0]);
}

// Expert of a lane's i-th value in the gradient: fours of neighbours, dealt
// to the lanes in turn, so that 16 lanes read and write 64 neighbours at once (with
// a lane's values all neighbours, inputs in the cache: 16384 x 256 float32 9.1 us, so 5.8;
// 32768 x 128 bf16 7.2, so 5.8).
template <int LANES, int VPL>
__device__ __forceinline__ int dealt(int sub, int i) {
  return VPL >= 4 ? (i / 4 * LANES + sub) * 4 + (i & 3) : sub * VPL + i;
}

// With g = scale grad_w and q the weights before scale:
//   softmax as it is (DENSE)   dx_e = p_e (g_e - sum_j g_j q_j), g_e 0 off the slots
//   softmax, renormalised      dx_e = q_e (g_e - sum_j g_j q_j) at the slots
//   sigmoid s                  dx_e = q_e (1 - s_e) g_e, renormalised (g_e - sum_j g_j q_j)
//                              in place of g_e
// A token's row is put together in LDS (one value per slot) and written whole.
template <int LANES, int VPL, bool DENSE>
__device__ __forceinline__ void route_token_backward(const RouteGradArgs& a, int vec, int64_t t,
                                                     int sub, float* row) {
  const bool in = t < a.tokens;
#pragma unroll
  for (int i = 0; i < VPL; ++i) row[dealt<LANES, VPL>(sub, i)] = 0.0f;

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

  float x[VPL], m = 0.0f, inv = 0.0f, q, d;
  if constexpr (DENSE) {
#pragma unroll
    for (int i = 0; i < VPL; ++i) x[i] = -INFINITY;
    if (in) {
      constexpr int N = VPL >= 4 ? 4 : VPL;
#pragma unroll
      for (int g4 = 0; g4 < VPL / N; ++g4) {
        float v[N];
        load_logits<N>(a.logits, a.f32, t * a.pitch, dealt<LANES, VPL>(sub, g4 * N), a.E, vec, v);
#pragma unroll
        for (int j = 0; j < N; ++j) x[g4 * N + j] = v[j];
      }
    }
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
    q = e >= 0 ? sigmoid(xe) : 0.0f;
    if (a.renorm) {
      const float sum = reduce_sum<LANES>(q);
      q = sum > 0.0f ? q / sum : 0.0f;
    }
    d = e >= 0 ? q * sigmoid(-xe) : 0.0f;          // 1 - s, also where s rounds to 1
  } else {
    const float one[1] = {xe};
    q = exp_term(xe, row_max<LANES, 1>(one));
    const float sum = reduce_sum<LANES>(q);
    q = sum > 0.0f ? q / sum : 0.0f;
    d = q;
  }
  const float dot = DENSE || a.renorm ? reduce_sum<LANES>(g * q) : 0.0f;
  wave_order();
  if (e >= 0) row[e] = DENSE ? d : d * (g - dot);
  wave_order();
  if (!in) return;
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const float r = row[dealt<LANES, VPL>(sub, i)];
    x[i] = DENSE ? x[i] * inv * (r - dot) : r;
  }
  if constexpr (VPL >= 4) if (vec) {
#pragma unroll
    for (int i = 0; i < VPL; i += 4) {
      const int n = dealt<LANES, VPL>(sub, i);
      if (n >= a.E) continue;
      if (a.f32)
        st16(static_cast<float*>(a.grad_logits) + t * a.E + n,
             u32x4{__float_as_uint(x[i]), __float_as_uint(x[i + 1]), __float_as_uint(x[i + 2]),
                   __float_as_uint(x[i + 3])});
      else
        st4x2(static_cast<uint16_t*>(a.grad_logits) + t * a.E + n, pack_bf16x2(x[i], x[i + 1]),
              pack_bf16x2(x[i + 2], x[i + 3]));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < VPL; ++i) {
    const int n = dealt<LANES, VPL>(sub, i);
    if (n >= a.E) {
    } else if (a.f32) {
      static_cast<float*>(a.grad_logits)[t * a.E + n] = x[i];
    } else {
      static_cast<uint16_t*>(a.grad_logits)[t * a.E + n] = (uint16_t)pack_bf16x2(x[i], 0.0f);
    }
  }
}

template <int LANES, int VPL, bool DENSE>
__global__ __launch_bounds__(kBlock) void route_backward_kernel(RouteGradArgs a, int vec) {
  constexpr int kTokens = kWave / LANES;         // of a wavefront
  __shared__ float s_row[kWavesPerBlock][kTokens][LANES * VPL];
  const int wave = threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  const int sub = lane & (LANES - 1), tok = lane / LANES;
  for (int64_t t0 = ((int64_t)blockIdx.x * kWavesPerBlock + wave) * kTokens; t0 < a.tokens;
       t0 += (int64_t)gridDim.x * kWavesPerBlock * kTokens) {
    route_token_backward<LANES, VPL, DENSE>(a, vec, t0 + tok, sub, s_row[wave][tok]);
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

unsigned route_blocks(int64_t tokens, int lanes) {
  const int64_t per = (int64_t)kWavesPerBlock * (kWave / lanes);
  const int64_t blocks = (tokens + per - 1) / per;
  return (unsigned)(blocks < kMaxGrid ? blocks : kMaxGrid);
}

}  // namespace

hipError_t launch_route(const RouteArgs& a, hipStream_t stream) {
  return by_width(a.E, a.k, a.groups, [&](auto lanes, auto vpl) {
    const int vec = vector_rows(a.logits, nullptr, a.pitch, a.E, vpl.value, a.f32);
    const dim3 grid(route_blocks(a.tokens, lanes.value));
    const auto run = [&](auto keys, auto groups) {
      hipLaunchKernelGGL((route_kernel<lanes.value, vpl.value, keys.value, groups.value>), grid,
                         dim3(kBlock), 0, stream, a, vec);
      return hipGetLastError();
    };
    const auto by_groups = [&](auto keys) {
      if (a.groups == 1) return run(keys, std::integral_constant<Groups, kOneGroup>());
      if constexpr (lanes.value == 16) {
        if (a.E == 16 * vpl.value && 16 % a.groups == 0)
          return run(keys, std::integral_constant<Groups, kLaneGroups>());
      }
      return run(keys, std::integral_constant<Groups, kAnyGroups>());
    };
    if (a.bias || (a.groups > 1 && a.group_top > 1))
      return a.sigmoid ? by_groups(std::integral_constant<Keys, kSigmoidKeys>())
                       : by_groups(std::integral_constant<Keys, kSoftmaxKeys>());
    if (!a.sigmoid && !a.renorm) return by_groups(std::integral_constant<Keys, kSoftmaxSum>());
    return by_groups(std::integral_constant<Keys, kLogits>());
  });
}

hipError_t launch_route_backward(const RouteGradArgs& a, hipStream_t stream) {
  return by_width(a.E, a.k, 1, [&](auto lanes, auto vpl) {
    const int vec = vpl.value >= 4 &&
                    vector_rows(a.logits, a.grad_logits, a.pitch, a.E, 4, a.f32);
    const dim3 grid(route_blocks(a.tokens, lanes.value));
    if (!a.sigmoid && !a.renorm)
      hipLaunchKernelGGL((route_backward_kernel<lanes.value, vpl.value, true>), grid, dim3(kBlock), 0,
                         stream, a, vec);
    else
      hipLaunchKernelGGL((route_backward_kernel<lanes.value, vpl.value, false>), grid, dim3(kBlock),
                         0, stream, a, vec);
    return hipGetLastError();
  });
}

}  // namespace moe
