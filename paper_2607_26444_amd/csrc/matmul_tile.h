// Device code that the experts' products share, whatever their codes are: tiles of the
// experts' windows, LDS stages, SwiGLU.
#pragma once

#include "matmul_rule.h"

namespace moe {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kOutside = 0x7FFFFFF0u;   // past every buffer's range: reads zeros

// A tile of an expert's window: rows of the window from `row` on (0: no such
// tile) and the piece of its channels.
struct Tile {
  int expert;
  int64_t row;
  int rows;
  int piece;
};

// Inclusive sum over the wavefront's lanes.
__device__ __forceinline__ int scan_add(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);   // row_shr:1
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);   // row_shr:2
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);   // row_shr:4
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);   // row_shr:8
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
  return x;
}

// Expert e's window: first row and rows, clipped to the rows there are.
__device__ __forceinline__ void window_of(const MatmulShape& a, int e, int first, int& start,
                                          int& rows) {
  const int all = (int)a.rows;
  const int o = (int)ld4(a.offset + e);
  const int64_t s = (int64_t)o - first;
  const int64_t m =
      a.count ? (int64_t)(int)ld4(a.count + e) : (int64_t)(int)ld4(a.offset + e + 1) - o;
  const bool in = s >= 0 && s <= all && m > 0;
  start = in ? (int)s : 0;
  rows = in ? (int)(m < all - s ? m : all - s) : 0;
}

// Tile `at` of a window of n rows from `start`: `group` row tiles of `size`
// rows together, all channel pieces of a group before the next, so that
// neighbouring tiles share rows or weights.
__device__ __forceinline__ Tile tile_of(int expert, int start, int n, int at, int size, int pieces,
                                        int group) {
  const int tiles = n / size + (n % size > 0);
  if (at >= tiles * pieces) return {0, 0, 0, 0};
  if (group > 1) {                                     // groups as even as they can be
    const int groups = (tiles + group - 1) / group;
    group = (tiles + groups - 1) / groups;
  }
  const int per = group * pieces;
  const int g = at / per, in = at % per;
  const int here = tiles - g * group < group ? tiles - g * group : group;   // tiles of this group
  const int tile = g * group + in % here;
  const int left = n - tile * size;
  return {expert, (int64_t)start + (int64_t)tile * size, left < size ? left : size, in / here};
}

// Tile `id`, windows in the order of the experts.
__device__ __forceinline__ Tile find_tile(const MatmulShape& a, int id, int size, int pieces) {
  if (!a.offset) return tile_of(0, 0, (int)a.rows, id, size, pieces, 1);
  const int lane = threadIdx.x & (kWave - 1);
  const int first = uniform((int)ld4(a.offset));
  int before = 0;
  for (int e0 = 0; e0 < a.E; e0 += kWave) {
    int s, m;
    window_of(a, e0 + lane < a.E ? e0 + lane : a.E - 1, first, s, m);
    if (e0 + lane >= a.E) m = 0;
    const int tiles = m / size + (m % size > 0);
    const int sum = before + scan_add(tiles);          // inclusive over the lanes
    const uint64_t hit = __ballot((int64_t)sum * pieces > id);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      return tile_of(e0 + l, __builtin_amdgcn_readlane(s, l), __builtin_amdgcn_readlane(m, l),
                     id - __builtin_amdgcn_readlane(sum - tiles, l) * pieces, size, pieces, 1);
    }
    before = __builtin_amdgcn_readlane(sum, kWave - 1);
  }
  return {0, 0, 0, 0};
}

// g / (1 + exp(-g)) by the hardware's exponential and reciprocal (1 ulp each;
// the argument's rounding adds |g| 2^-24): far inside the bf16 rounding that
// follows, and a tenth of the exact division's instructions.
__device__ __forceinline__ float silu(float g) {
  return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
}

// Buffer resource of `bytes` bytes from `base`, both the same in every lane.
__device__ __forceinline__ Rsrc buffer_of(const uint8_t* base, int bytes) {
  const uint64_t p = (uint64_t)base;
  const uint32_t lo = (uint32_t)uniform((int)(uint32_t)p), hi = (uint32_t)uniform((int)(p >> 32));
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<uint8_t*>(((uint64_t)hi << 32) | lo),
                                           (short)0, uniform(bytes), kRsrcWord3);
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;

// LDS rows are 128 bytes of the depth, as eight chunks of 16: chunk c of row r at
// place c ^ (r & 7), so that eight lanes that read one chunk of eight rows
// touch all banks: no bank conflicts are counted.
constexpr int kDepth = 128;

// One load instruction of a wavefront: eight rows of 128 bytes from memory into
// the 1 KiB of LDS at `to`.
__device__ __forceinline__ void load_to_lds(Rsrc r, uint32_t offset, lds_u8* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, (int)offset, 0, 0, 0);
}

// Waits until this wavefront's LDS reads are done and all but its last PENDING
// memory loads have arrived, then for the workgroup's other wavefronts.
template <int PENDING>
__device__ __forceinline__ void meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  // lgkmcnt(0), vmcnt(PENDING), in the instruction's bit fields
  __builtin_amdgcn_s_waitcnt(0x0070 | (PENDING & 15) | (PENDING >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// Instruction classes of the scheduler's groups.
constexpr int kIssueMatrix = 0x008, kIssueLdsRead = 0x100;

// Asks for COUNT instructions of a class, each followed by MATRIX matrix
// instructions.
template <int CLASS, int COUNT, int MATRIX>
__device__ __forceinline__ void interleave() {
#pragma unroll
  for (int i = 0; i < COUNT; ++i) {
    __builtin_amdgcn_sched_group_barrier(CLASS, 1, 0);
    __builtin_amdgcn_sched_group_barrier(kIssueMatrix, MATRIX, 0);
  }
}

// Channel (of the tile's) that an LDS row of weights holds.  A lane's sums of a
// wavefront's four 16-channel tiles are 16 neighbouring channels this way (with
// swiglu tiles 1 and 3 are the up channels of 0 and 2, and a lane has 8), so that
// its outputs are whole vectors and a row's are whole lines.
__device__ __forceinline__ int channel_of(int r, bool swiglu) {
  const int block = r / 64, tile = r / 16 & 3, d = r & 15;
  return swiglu ? block * 32 + d / 4 * 8 + tile / 2 * 4 + (d & 3)
                : block * 64 + d / 4 * 16 + tile * 4 + (d & 3);
}

}  // namespace moe
