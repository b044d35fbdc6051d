// The experts' products on microscaled 4-bit floats:
//   v[r,n] = sum_k a[r,k] w[e,n,k] with the values that codes and scales stand for,
//   y = bf16(v), or with swiglu y[r,i] = bf16(silu(v[r,i]) v[r,N/2+i]).
// Scaled matrix instructions multiply 16 x 16 x 128 codes, a scale byte for each 32 of them,
// and add in float32; the result is rounded to bf16 once.  The kernels are those of the 8-bit
// products (tiles of 256 or 128 rows x 256 channels where arithmetic bounds the call, 64
// rows or fewer x 128 channels or fewer where reading the weights does): a fragment is 16
// bytes to a lane as theirs is, and holds twice the depth.
//
// Which of a row's blocks meet in one instruction is free as long as both operands agree: of a
// stage's eight chunks of 16 bytes (a block of 32 codes each) lane quarter q takes the chunks 2 q
// and 2 q + 1, one to an instruction, so that their two scales are neighbouring bytes which
// a lane reads at once and the instructions select.  In LDS chunk c of row r is at place
// c' ^ (r & 7), c' its number with the two low bits exchanged: lanes that read together touch
// all banks (with c itself 46 M cycles of conflicts beside 104 M of reads), lanes that
// load together have half a line (an order that spread them over whole lines made twice the
// requests).

#include <type_traits>

#include "matmul_tile.h"

namespace moe {
namespace {

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// The chunk of its row that a lane loads to its place: four neighbouring lanes have half a
// line.
__device__ __forceinline__ int chunk_of(int lane) {
  const int place = (lane & 7) ^ (lane / 8);
  return (place & 4) | (place & 1) << 1 | (place >> 1 & 1);
}

// Place of a lane's first chunk in a row of LDS; its second one is two further, 32 bytes.
__device__ __forceinline__ uint32_t place_of(int row, int quarter) {
  return row * kDepth + (((quarter & 2) << 1 | (quarter & 1)) ^ (row & 7)) * 16;
}

constexpr int kStageScales = kDepth / 16;   // scale bytes of a row and stage

// Both operands are 4-bit floats (format 4), 16 bytes to a lane; SW, SA: the byte of the scale
// words that holds the scale.
template <int SW, int SA>
__device__ __forceinline__ f32x4 multiply_mx(i32x4 w, i32x4 a, f32x4 c, int sw, int sa) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
      i32x8{w[0], w[1], w[2], w[3], 0, 0, 0, 0}, i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0}, c, 4, 4,
      SW, sw, SA, sa);
}

// A lane's two scales of a row and stage, from LDS.
__device__ __forceinline__ uint32_t two_scales(const uint8_t* p) {
  return *reinterpret_cast<const uint16_t*>(p);
}

// Ones in the bytes of a lane's two scales that lie within the depth, in both halves: what
// lies behind it is no scale, and 255 among it would be NaN.  k: the stage's first byte.
__device__ __forceinline__ uint32_t depth_mask(int k, int quarter, int K) {
  const int at = k + quarter * 32;
  return (at < K ? 0x00FF00FFu : 0u) | (at + 16 < K ? 0xFF00FF00u : 0u);
}

// load_to_lds past the caches, for weights that are read once.
__device__ __forceinline__ void stream_to_lds(Rsrc r, uint32_t offset, lds_u8* to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, to, 16, (int)offset, 0, 0, kLoadNonTemporal);
}

// f(0) to f(N - 1), their arguments constants.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>());
    each<N, I + 1>(f);
  }
}

// Tiles of 256 or 128 rows x 256 channels through LDS: eight wavefronts, each half the rows x 64
// channels; stages of 128 bytes of the depth go from memory into LDS by the loads themselves.
//
// Scales.  A lane needs two bytes of every row and stage; a request for any of a row's bytes moves
// a whole line to the compute unit, so that taking them stage by stage made a third of all
// requests.  With tiles of 256 rows they come for four stages at once (32 bytes of a row), half
// of a wavefront's rows at a time; before every second stage each thread takes 16 bytes of its own
// row from there and puts them, by quarter and tile, where a lane finds its words of four tiles
// in one read.
//
// 32768 rows, 16 experts, 7168 x 4096 with swiglu 472 to 480 us by card (4.0 PFLOP/s).  What bounds
// it is that the two wavefronts of a SIMD are in the same phase of a stage and meet once in it, so
// that both wait at a time: the matrix units are busy 44% of the cycles within a layer, at 2.0 GHz
// (with all codes 0 7% less time), reads of LDS a fifth, and the loads would come in a third of a
// stage (a loop of them reaches 110 to 130 bytes a ns and compute unit, 70 from rows that lie
// across lines).  With the loads left out it takes 370, without those of the scales alone 445.  The
// two in opposite phases, or instructions of 32 x 32 x 64, have not been tried.
// Shallow products also have their stores: 32 experts, 2048 x 7168 349 to 359 us, without stores
// 274; not waiting for them in the next tile's first stage changes nothing.
// A window's last rows walk all of the depth again: 32 windows of 256 rows, 7168 x 4096, 152 us, of
// 257 236, of 384 236, of 512 253.
// On the way there: scales word by word and stage by stage 527; 16 bytes every second stage 495;
// stages of half the depth, four of them, 510; four wavefronts with 128 x 128 each 523; lines asked
// for earlier, to have them in the L2 cache, +4 to 8%; the windows' short last tiles behind all
// others +1 to 15%; outputs in whole 64 bytes to a store, stores past the caches, workgroups that
// start at four different times, wavefronts of raised priority 0 to +2%.

// Scales of a row and pair of stages.
constexpr int kPairScales = 2 * kStageScales;

// LDS of the kernel of tiles of HEIGHT rows: stages of rows and weights; the scales of two stages
// in the order of the lanes, and as they came; the workgroup's next tiles.
template <int HEIGHT>
struct MxTileLds {
  static constexpr int kStages = HEIGHT == 256 ? 2 : 3;
  static constexpr int kRowBytes = HEIGHT * kDepth;
  static constexpr int kStageBytes = kRowBytes + kTile * kDepth;
  static constexpr int kScaleAt = kStages * kStageBytes;
  static constexpr bool kFourStages = HEIGHT == 256;   // scales come for four stages, else for two
  // Loads of a full tile's stage that are asked for during the first units of the stage before it,
  // and not as soon as their place is free: 0 486 us, 4 482, 6 477, 8 484 at the size above.  8192
  // rows over 32 experts, where half of the windows have a short tile besides, lost 2% (225 ->
  // 230).
  static constexpr int kLate = HEIGHT == 256 ? 6 : 0;
  static constexpr int kRawAt = kScaleAt + kTileThreads * kPairScales;
  static constexpr int kListAt = kRawAt + (kFourStages ? kTileThreads * 2 * kPairScales : 0);
  static constexpr int kBytes = kListAt + kWave * 16;
  static_assert(3 * MOE_MAX_EXPERTS * 4 <= kScaleAt, "the windows lie there before the stages");
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
};

// What a wavefront loads of a tile.
template <int HEIGHT>
struct MxTileLoads {
  using Lds = MxTileLds<HEIGHT>;
  Rsrc ra, rw;
  uint32_t ao, wo;             // of instruction 0
  int a_step, w_step;          // from one instruction to the next
  const uint8_t* scales;       // of the thread's row or channel
  // of the wavefront's 64 rows, in two sets of 32 (tiles of 16 in turn): the second `other` further
  const uint8_t* set;
  int64_t other;
  int set_bytes, other_bytes;
  uint32_t so;
  int K, wave, scale_bytes, last_piece;
  const uint8_t* spare;        // 16 bytes that may be read
  uint8_t* s_tile;

  __device__ __forceinline__ MxTileLoads(const MatmulMxArgs& a, const Tile& t, int tid, uint8_t* lds)
      : K(a.K), s_tile(lds) {
    const int lane = tid & (kWave - 1);
    wave = uniform(tid / kWave);
    // instruction j of a wavefront fills LDS rows (j * 8 + wave) * 8 + lane / 8
    const int half = a.N / 2, c0 = t.piece * (a.swiglu ? kTile / 2 : kTile);
    const int r = wave * 8 + lane / 8;
    ao = (uint32_t)r * (uint32_t)a.a_pitch + chunk_of(lane) * 16;
    wo = (uint32_t)channel_of(r, a.swiglu) * (uint32_t)K + chunk_of(lane) * 16;
    a_step = 64 * a.a_pitch;
    w_step = (a.swiglu ? 32 : 64) * K;
    const int channels = (a.swiglu ? half : a.N) - c0, most = a.swiglu ? kTile / 2 : kTile;
    const int held = channels < most ? channels : most;
    const int64_t first = (int64_t)t.expert * a.N + c0;
    ra = buffer_of(a.a + t.row * a.a_pitch, (t.rows - 1) * a.a_pitch + K);
    rw = buffer_of(a.w + (first + (a.swiglu && (wave & 2) ? half : 0)) * K, held * K);

    scale_bytes = mx_scale_bytes(2 * K);
    last_piece = scale_bytes > kPairScales ? scale_bytes - kPairScales : 0;
    spare = a.w;
    const int in_set = (lane / 2 & 15) + (lane / 2 & 16) * 2;   // row of the set by two lanes
    if (wave < HEIGHT / 64) {
      const int64_t pitch = a.a_scale_pitch;
      set = a.a_scales + t.row * pitch;
      scales = set + (tid < t.rows ? tid : t.rows - 1) * pitch;
      other = 16 * pitch;
      set_bytes = (t.rows - 1) * a.a_scale_pitch + scale_bytes;
      other_bytes = t.rows > 16 ? set_bytes - 16 * a.a_scale_pitch : 0;
      so = (uint32_t)(wave * 64 + in_set) * (uint32_t)a.a_scale_pitch;
    } else {                                           // tiles 1 and 3: up channels, or 4 further
      const int n = tid - HEIGHT, c = channel_of(n, a.swiglu);
      set = a.w_scales + first * scale_bytes;
      scales = set + ((c < held ? c : held - 1) + (int64_t)(a.swiglu && (n & 16) ? half : 0)) *
                         scale_bytes;
      other = (int64_t)(a.swiglu ? half : 4) * scale_bytes;
      set_bytes = held * scale_bytes;
      other_bytes = a.swiglu ? set_bytes : set_bytes - 4 * scale_bytes;   // 8 are held at least
      so = (uint32_t)channel_of((wave - HEIGHT / 64) * 64 + in_set, a.swiglu) * (uint32_t)scale_bytes;
    }
    if (scale_bytes < kPairScales) set_bytes = other_bytes = 0;
  }

  // A stage behind the depth is out of every range: zeros.
  __device__ __forceinline__ int depth_of(int k0) const { return k0 < K ? k0 : 0x70000000; }

  // Load `n` of a stage: rows and weights in turn, ROW_LOADS + 4 in all (ROW_LOADS: as many 64
  // rows as the tile multiplies).  Past the tile's rows and channels: zeros.  Past the depth:
  // those or the next row's codes, whose scales are 0.
  template <int ROW_LOADS>
  __device__ __forceinline__ void part(int n, int k0, uint32_t buf) const {
    const bool is_row = n < 2 * ROW_LOADS && n % 2 == 0;
    const int j = n < 2 * ROW_LOADS ? n / 2 : n - ROW_LOADS;
    if (is_row)
      load_to_lds(ra, ao + (k0 + j * a_step), (lds_u8*)(s_tile + buf + (j * 8 + wave) * 1024));
    else
      load_to_lds(rw, wo + (k0 + j * w_step),
                  (lds_u8*)(s_tile + buf + Lds::kRowBytes + (j * 8 + wave) * 1024));
  }

  // First byte of a pair's 16 of a row; the last ones end with the row.
  __device__ __forceinline__ int piece_of(int pair) const {
    const int at = pair * kPairScales;
    return at < last_piece ? at : last_piece;
  }
  // The thread's scales of a pair.
  __device__ __forceinline__ u32x4 fetch(int pair) const {
    return ld16(scale_bytes < kPairScales ? spare : scales + piece_of(pair));
  }
  // Those of the first pair also where a row has less than 16 bytes.
  __device__ __forceinline__ u32x4 fetch_first() const {
    if (scale_bytes >= kPairScales) return ld16(scales);
    u32x4 v = {ld4(scales), 0, 0, 0};
    if (scale_bytes > 4) v.y = ld4(scales + 4);
    if (scale_bytes > 8) v.z = ld4(scales + 8);
    return v;
  }
  // The scales of a pair and the next one of a set of the wavefront's rows into LDS.
  __device__ __forceinline__ void ask(int which, int pair, int lane) const {
    const Rsrc r = buffer_of(set + (which ? other : 0), which ? other_bytes : set_bytes);
    load_to_lds(r, so + (lane & 1 ? piece_of(pair + 1) : piece_of(pair)),
                (lds_u8*)(s_tile + Lds::kRawAt + wave * 2048 + which * 1024));
  }
  // The thread's scales of a pair from there: set 0 was asked for at even pairs, set 1 at odd ones.
  __device__ __forceinline__ u32x4 asked(int pair, int tid) const {
    const int l = tid & 63;
    const uint32_t at = tid / 64 * 2048 + (l & 16) * 64 + ((l & 15) + (l & 32) / 2) * 32 + (l & 16);
    return *reinterpret_cast<const u32x4*>(s_tile + Lds::kRawAt + (at ^ (pair & 1) * 16));
  }
  // A pair's scales in their places in LDS: for each quarter the words (two scales of either stage)
  // of four neighbouring tiles of 16.  What lies behind the depth is 0.
  __device__ __forceinline__ void place(u32x4 v, int pair, int tid) const {
    uint32_t d[4] = {v.x, v.y, v.z, v.w};
    const int at = pair * kPairScales, ahead = at - last_piece;   // bytes before the first stage
    d[0] = ahead < 4 ? d[0] : ahead < 8 ? d[1] : ahead < 12 ? d[2] : d[3];
    d[1] = ahead < 4 ? d[1] : ahead < 8 ? d[2] : d[3];
    d[2] = ahead < 4 ? d[2] : d[3];
    int left = K / 16 - at;                            // scales there are
    left = left < 0 ? 0 : left > 16 ? 16 : left;
    const uint64_t low = left < 8 ? (1ull << left * 8) - 1 : ~0ull;
    const uint64_t high = left < 8 ? 0ull : left < 16 ? (1ull << (left - 8) * 8) - 1 : ~0ull;
    d[0] &= (uint32_t)low;
    d[1] &= (uint32_t)(low >> 32);
    d[2] &= (uint32_t)high;
    d[3] &= (uint32_t)(high >> 32);
    uint8_t* to = s_tile + Lds::kScaleAt + tid / 64 * 1024 + (tid & 15) * 16 + (tid / 16 & 3) * 4;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint32_t*>(to + q * 256) =
          __builtin_amdgcn_perm(d[2 + q / 2], d[q / 2], q & 1 ? 0x07060302u : 0x05040100u);
  }
};

// A tile's first stages and scales.
template <int HEIGHT>
__device__ __forceinline__ void begin_tile(const MatmulMxArgs& a, const Tile& t, int tid,
                                           uint8_t* s_tile) {
  using Lds = MxTileLds<HEIGHT>;
  const MxTileLoads<HEIGHT> loads(a, t, tid, s_tile);
  constexpr int kLoads = HEIGHT / 64 + 4;
  const int second = t.rows > HEIGHT / 2 ? kLoads - Lds::kLate : kLoads;
#pragma unroll
  for (int s = 0; s < Lds::kStages; ++s)
#pragma unroll
    for (int n = 0; n < kLoads; ++n)
      if (s != 1 || n < second)
        loads.template part<HEIGHT / 64>(n, loads.depth_of(s * kDepth), s * Lds::kStageBytes);
  if constexpr (Lds::kFourStages) {
    loads.ask(0, 0, tid & (kWave - 1));
    loads.ask(1, 1, tid & (kWave - 1));
  }
  loads.place(loads.fetch_first(), 0, tid);
}

// One tile whose wavefronts take MT x 16 rows each: 8 for a full tile, 4 or 2
// for the last rows of a window.  Its first stages have been asked for; those of
// `next` are before its own outputs are computed and stored.  stores: what the tile before
// left on its way after them.
template <int HEIGHT, int MT>
__device__ __forceinline__ void multiply_mx_tile(const MatmulMxArgs& a, const Tile& t,
                                                 const Tile& next, int tid, uint8_t* s_tile,
                                                 int stores) {
  using Lds = MxTileLds<HEIGHT>;
  constexpr int NT = 4;
  constexpr int kLoads = MT / 2 + 4;                   // of a wavefront and stage
  constexpr int kLate = MT * 32 == HEIGHT ? Lds::kLate : 0, kEarly = kLoads - kLate;
  const int lane = tid & (kWave - 1), wave = uniform(tid / kWave);
  const MxTileLoads<HEIGHT> loads(a, t, tid, s_tile);

  const int wm = wave / 4, wn = wave % 4;              // 2 x 4 wavefronts
  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = place_of(row, quarter);
  const uint32_t at_a = wm * (MT * 16 * kDepth) + place;
  const uint32_t at_w = Lds::kRowBytes + wn * (64 * kDepth) + place;
  const uint32_t mine = Lds::kScaleAt + quarter * 256 + row * 16;
  const uint32_t at_sa = wm * MT / 4 * 1024 + (MT == 2 ? wm * 8 : 0) + mine;
  const uint32_t at_sw = (HEIGHT / 64 + wn) * 1024 + mine;
  f32x4 acc[MT][NT] = {};

  // A stage is U units of 16 rows (the first halves of the chunks, then the second), NT
  // instructions each.  Unit u asks for the rows of unit u + D; from unit B on all of the
  // stage is in registers.
  constexpr int U = 2 * MT, D = U == 16 ? 4 : U == 8 ? 3 : 2, B = U - D + 1, kLeft = U - B;
  constexpr int R = U < 8 ? U : 8, kPlace = B / 2 + 1;
  i32x4 av[R], wv[2][NT];
  uint32_t sa[MT], sw[NT], sa_next[MT], sw_next[NT];   // scales of two stages
  auto read_a = [&](int u, uint32_t buf) {
    av[u % R] = *(const i32x4*)(s_tile + (at_a ^ (u / MT * 32)) + buf + u % MT * 16 * kDepth);
  };
  auto read_w = [&](int h, int j, uint32_t buf) {
    wv[h][j] = *(const i32x4*)(s_tile + (at_w ^ (h * 32)) + buf + j * 16 * kDepth);
  };
  auto read_scales = [&](uint32_t (&a4)[MT], uint32_t (&w4)[NT]) {
    const u32x4 w = *(const u32x4*)(s_tile + at_sw);
#pragma unroll
    for (int j = 0; j < NT; ++j) w4[j] = w[j];
    if constexpr (MT == 2) {
      const u32x2 v = *(const u32x2*)(s_tile + at_sa);
      a4[0] = v.x;
      a4[1] = v.y;
    } else {
#pragma unroll
      for (int c = 0; c < MT / 4; ++c) {
        const u32x4 v = *(const u32x4*)(s_tile + at_sa + c * 1024);
#pragma unroll
        for (int i = 0; i < 4; ++i) a4[4 * c + i] = v[i];
      }
    }
  };
  // The first stages are there; the stores after them may be on their way.
  if (stores >= 16) meet<16>();
  else if (stores >= 8) meet<8>();
  else if (stores >= 4) meet<4>();
  else if (stores >= 2) meet<2>();
  else meet<0>();
  uint32_t buf = 0;
#pragma unroll
  for (int u = 0; u < D; ++u) read_a(u, 0);
#pragma unroll
  for (int j = 0; j < NT; ++j) read_w(0, j, 0);
  read_scales(sa, sw);
  u32x4 row_scales = {};
  if constexpr (!Lds::kFourStages) row_scales = loads.fetch(1);
  // Stage s is in LDS at s % kStages.  Within a turn the wavefronts meet once: by then each has
  // asked for the last of stage s, and its loads of stage s + 1 have arrived; those of stage s + 2
  // follow then and, of full tiles, in the next turn.  The scales of the
  // next two stages are placed before that in every second turn, and read behind it.
  auto turn = [&](auto parity, int k0) {
    constexpr int p = parity.value;
    const int fill = loads.depth_of(k0 + Lds::kStages * kDepth);
    uint32_t next_buf = buf + Lds::kStageBytes == Lds::kScaleAt ? 0 : buf + Lds::kStageBytes;
    if constexpr (Lds::kStages == 2) next_buf = Lds::kStageBytes - buf;
    __builtin_amdgcn_sched_barrier(0);
    each<U>([&](auto unit) {
      constexpr int u = unit.value, h = u / MT, i = u % MT, x = u - B;
      if constexpr (u == B) meet<(Lds::kStages - 2) * kLoads>();
      if constexpr (u + D < U) read_a(u + D, buf);
      if constexpr (u < kLate)
        loads.template part<MT / 2>(kEarly + u, loads.depth_of(k0 + kDepth), next_buf);
      if constexpr (h == 0) {
#pragma unroll
        for (int j = i * NT / MT; j < (i + 1) * NT / MT; ++j) read_w(1, j, buf);
      }
      const int pair = k0 / (2 * kDepth);
      if constexpr (p == 1 && u == kPlace - 1 && Lds::kFourStages)
        row_scales = loads.asked(pair + 1, tid);
      if constexpr (p == 1 && u == kPlace) loads.place(row_scales, pair + 1, tid);
      if constexpr (p == 1 && u == B) {
        if constexpr (Lds::kFourStages) loads.ask(pair & 1, pair + 2, lane);
        else row_scales = loads.fetch(pair + 2);
      }
      if constexpr (u >= B) {
#pragma unroll
        for (int n = x * kEarly / kLeft; n < (x + 1) * kEarly / kLeft; ++n)
          loads.template part<MT / 2>(n, fill, buf);
#pragma unroll
        for (int j = x * NT / kLeft; j < (x + 1) * NT / kLeft; ++j) read_w(0, j, next_buf);
#pragma unroll
        for (int v = x * D / kLeft; v < (x + 1) * D / kLeft; ++v) read_a(v, next_buf);
        if constexpr (p == 1 && u == B) read_scales(sa_next, sw_next);
      }
#pragma unroll
      for (int j = 0; j < NT; ++j)
        acc[i][j] = multiply_mx<h + 2 * p, h + 2 * p>(wv[h][j], av[u % R], acc[i][j], (int)sw[j],
                                                      (int)sa[i]);
    });
    buf = next_buf;
    if constexpr (p == 1) {
#pragma unroll
      for (int i = 0; i < MT; ++i) sa[i] = sa_next[i];
#pragma unroll
      for (int j = 0; j < NT; ++j) sw[j] = sw_next[j];
    }
  };
  // No branch within two turns: one there cost as much as a tenth of the loop.
  int k0 = 0;
  for (; k0 + kDepth < a.K; k0 += 2 * kDepth) {
    turn(std::integral_constant<int, 0>(), k0);
    turn(std::integral_constant<int, 1>(), k0 + kDepth);
  }
  if (k0 < a.K) turn(std::integral_constant<int, 0>(), k0);
  meet<0>();                                           // loads past the end have landed

  if (next.rows) begin_tile<HEIGHT>(a, next, tid, s_tile);

  // Rows and channels that are not there lie outside the range, so that every wavefront makes
  // the same number of stores.
  const int out = a.swiglu ? a.N / 2 : a.N;
  const int c0 = t.piece * (a.swiglu ? kTile / 2 : kTile) +
                 (a.swiglu ? wn * 32 + quarter * 8 : wn * 64 + quarter * 16);
  const Rsrc ry = buffer_of(reinterpret_cast<uint8_t*>(a.y + t.row * out), t.rows * out * 2);
  const uint32_t to = (uint32_t)(wm * (MT * 16) + row) * (uint32_t)out * 2;
  const uint32_t at0 = c0 < out ? to + c0 * 2 : kOutside;
  const uint32_t at1 = c0 + 8 < out ? to + c0 * 2 + 16 : kOutside;
  if (a.swiglu) {
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int j = q / 4 * 2;
        v[q] = silu(acc[i][j][q & 3]) * acc[i][j + 1][q & 3];
      }
      __builtin_amdgcn_raw_buffer_store_b128(pack8(v), ry, (int)(at0 + i * 32 * out), 0, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = acc[i][h * 2 + q / 4][q & 3];
        __builtin_amdgcn_raw_buffer_store_b128(pack8(v), ry, (int)((h ? at1 : at0) + i * 32 * out), 0, 0);
      }
  }
}

// A workgroup to each compute unit takes the tiles blockIdx.x, + 256, ... of
// an order in which the 32 tiles that an XCD's compute units hold together are
// neighbours.
template <int HEIGHT>
__global__ __launch_bounds__(kTileThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void matmul_mx_tile_kernel(MatmulMxArgs a, int pieces, int group) {
  using Lds = MxTileLds<HEIGHT>;
  __shared__ __attribute__((aligned(1024))) uint8_t s_tile[Lds::kBytes];
  struct Entry {
    int expert, row, rows, piece;
  };
  Entry* s_list = reinterpret_cast<Entry*>(s_tile + Lds::kListAt);
  const int lane = threadIdx.x & (kWave - 1);
  // The workgroup's next 64 tiles, one to a lane.  The windows' row tiles to their ends, first
  // rows and rows lie where the stages will be.
  auto list_tiles = [&](int first_tile) {
    int* s_end = reinterpret_cast<int*>(s_tile);
    int* s_start = s_end + MOE_MAX_EXPERTS;
    int* s_rows = s_start + MOE_MAX_EXPERTS;
    __syncthreads();
    if (threadIdx.x < kWave) {
      const int first = a.offset ? uniform((int)ld4(a.offset)) : 0;
      int before = 0;
      for (int e0 = 0; e0 < a.E; e0 += kWave) {
        int s = 0, m = (int)a.rows;
        if (a.offset) window_of(a, e0 + lane < a.E ? e0 + lane : a.E - 1, first, s, m);
        if (e0 + lane >= a.E) m = 0;
        const int end = before + scan_add(m / HEIGHT + (m % HEIGHT > 0));
        s_end[e0 + lane] = end;                        // E is at most 16 times 64
        s_start[e0 + lane] = s;
        s_rows[e0 + lane] = m;
        before = __builtin_amdgcn_readlane(end, kWave - 1);
      }
      const int64_t id = (int64_t)(first_tile + lane) * 256 + (blockIdx.x & 7) * 32 + blockIdx.x / 8;
      Entry entry = {0, 0, 0, 0};
      if ((int64_t)before * pieces > id) {
        int low = 0, high = a.E - 1;                   // the first window that ends behind it
        while (low < high) {
          const int mid = (low + high) / 2;
          if ((int64_t)s_end[mid] * pieces > id) high = mid;
          else low = mid + 1;
        }
        const int64_t start = low ? (int64_t)s_end[low - 1] * pieces : 0;
        const Tile t = tile_of(low, s_start[low], s_rows[low], (int)(id - start), HEIGHT, pieces,
                               group);
        entry = {t.expert, (int)t.row, t.rows, t.piece};
      }
      s_list[lane] = entry;
    }
    __syncthreads();
  };
  auto tile_at = [&](int n) -> Tile {
    const Entry e = s_list[n];
    return {uniform(e.expert), (int64_t)uniform(e.row), uniform(e.rows), uniform(e.piece)};
  };

  int tid = threadIdx.x;
  for (int first_tile = 0;; first_tile += kWave) {
    list_tiles(first_tile);
    Tile t = tile_at(0);
    if (t.rows == 0) return;                           // the whole workgroup
    begin_tile<HEIGHT>(a, t, tid, s_tile);
    int stores = 0;
    for (int n = 1;; ++n) {
      Tile next = {0, 0, 0, 0};
      if (n < kWave) next = tile_at(n);
      // what follows from the thread's number is worked out anew for each tile:
      // kept over the loop it would not fit the registers
      asm volatile("" : "+v"(tid));
      const int mt = HEIGHT > 128 && t.rows > 128 ? HEIGHT / 32 : t.rows > 64 ? 4 : 2;
      if (HEIGHT > 128 && mt == HEIGHT / 32)
        multiply_mx_tile<HEIGHT, HEIGHT / 32>(a, t, next, tid, s_tile, stores);
      else if (mt == 4) multiply_mx_tile<HEIGHT, 4>(a, t, next, tid, s_tile, stores);
      else multiply_mx_tile<HEIGHT, 2>(a, t, next, tid, s_tile, stores);
      if (next.rows == 0) {
        if (n < kWave) return;
        break;
      }
      stores = a.swiglu ? mt : 2 * mt;
      t = next;
    }
  }
}

// Few rows: ROWS rows of a window x 16 WC channels, bound by reading the
// weights.  Eight wavefronts, WC along the channels and WK along the depth; a
// stage is 128 WK bytes of the depth, STAGES - 1 stages are on their way while one is
// multiplied.  A wavefront loads its own weights (8 + 8 channels: with swiglu
// gate and up channels, so that a lane and its partner 32 further on hold both
// halves) and an eighth of the rows.  The sums of the WK wavefronts meet in LDS.
//
// Scales come as pieces of 16 bytes of a row, whose lines cost more than their bytes: 8 bytes of
// each row a stage, word by word, took 22 of 100 us (512 rows, 32 experts, 7168 x 4096 with
// swiglu).  A row's pieces hold the stage, with WK = 1 two stages.
template <int ROWS, int WC, int WK, int STAGES>
struct MxStreamLds {
  static constexpr int kBatch = WK == 1 ? 2 : 1;       // stages whose scales come together
  static constexpr int kRowScales = kBatch * WK * kStageScales, kPieces = kRowScales / 16;
  static constexpr int kScaleRows = WC * 16 + ROWS;    // the channels, then the rows
  static constexpr int kScaleBytes = kScaleRows * kRowScales;
  static constexpr int kPerWave = kScaleRows * kPieces / 8;
  static_assert(kPerWave * 8 == kScaleRows * kPieces && kPerWave <= kWave, "one instruction");
  static constexpr int kRowBytes = ROWS * kDepth * WK;
  static constexpr int kCodes = kRowBytes + 16 * 1024;
  static constexpr int kStage = kCodes + (kBatch == 1 ? kScaleBytes : 0);
  static constexpr int kBatchAt = STAGES * kStage;     // two batches, where they are no part of stages
  // what a tail's scales are read past the last row's
  static constexpr int kBytes = kBatchAt + (kBatch == 1 ? 0 : 2 * kScaleBytes) + 64;
  static_assert(kBytes <= 160 * 1024, "LDS of a compute unit");
};

template <int ROWS, int WC, int WK, int STAGES>
__global__ __launch_bounds__(kTileThreads)
void matmul_mx_stream_kernel(MatmulMxArgs a, int pieces) {
  using Lds = MxStreamLds<ROWS, WC, WK, STAGES>;
  static_assert(WC * WK == 8, "eight wavefronts");
  constexpr int MT = ROWS / 16;
  constexpr int kRowBytes = Lds::kRowBytes, kStage = Lds::kStage;
  constexpr int kRowLoads = WK * ROWS / 64;            // of a wavefront and stage
  static_assert(kRowLoads * 64 == WK * ROWS, "whole load instructions");
  // a batch of two stages is asked for before the codes of its first one, so that no
  // count of loads on their way has to know of it
  constexpr int kLoads = 2 + kRowLoads + (Lds::kBatch == 1 ? 1 : 0);
  __shared__ __attribute__((aligned(1024))) uint8_t s_mem[Lds::kBytes];
  static_assert(STAGES * kStage >= 8 * MT * kWave * 16, "sums meet there");
  const int lane = threadIdx.x & (kWave - 1), wave = uniform(threadIdx.x / kWave);
  // 32 neighbouring tiles (mostly one window's, which share rows) to an XCD
  const int b = blockIdx.x;
  const Tile t = find_tile(a, b / 256 * 256 + b % 8 * 32 + b / 8 % 32, ROWS, pieces);
  if (t.rows == 0) return;                             // the whole workgroup
  const int half = a.N / 2, out = a.swiglu ? half : a.N;
  const int wc = wave % WC, wk = wave / WC;
  const int step = a.swiglu ? 8 : 16;                  // output channels of a wavefront
  const int c0 = t.piece * WC * step + wc * step;

  const int lr = lane / 8, chunk = chunk_of(lane);
  const Rsrc ra = buffer_of(a.a + t.row * a.a_pitch, (t.rows - 1) * a.a_pitch + a.K);
  const uint8_t* wbase = a.w + ((int64_t)t.expert * a.N + c0) * a.K;
  const int c1 = a.swiglu ? c0 : c0 + 8;               // channels come in whole eights
  const Rsrc rw0 = buffer_of(wbase, c0 < out ? 8 * a.K : 0);
  const Rsrc rw1 = buffer_of(wbase + (int64_t)(a.swiglu ? half : 8) * a.K, c1 < out ? 8 * a.K : 0);
  const uint32_t wo = (uint32_t)lr * (uint32_t)a.K + wk * kDepth + chunk * 16;

  // A lane's piece of the scales, by address: that of a row or channel that is not there
  // is another's (its outputs are not stored).  A row's last piece ends with it: scales
  // are read as much further on.  Rows of less than a piece come word by word.
  const int scale_bytes = mx_scale_bytes(2 * a.K);
  const bool words = scale_bytes < 16;
  const int last_piece = words ? 0 : scale_bytes - 16;
  const int piece = (wave * Lds::kPerWave + lane) % Lds::kPieces * 16;
  const uint8_t* scales;
  {
    const int n = (wave * Lds::kPerWave + lane) / Lds::kPieces;
    if (n < WC * 16) {
      int c = t.piece * WC * step + n / 16 * step + (n & 7) + ((n & 8) && !a.swiglu ? 8 : 0);
      c = c < out ? c : out - 1;
      if ((n & 8) && a.swiglu) c += half;
      scales = a.w_scales + ((int64_t)t.expert * a.N + c) * scale_bytes;
    } else {
      const int r = n - WC * 16;
      scales = a.a_scales + (t.row + (r < t.rows ? r : t.rows - 1)) * a.a_scale_pitch;
    }
  }
  auto scales_at = [&](int k0, uint32_t at) -> uint32_t {   // of the stage at `at`
    return Lds::kBatch == 1 ? at + Lds::kCodes
                            : Lds::kBatchAt + (k0 / (2 * kDepth) & 1) * Lds::kScaleBytes;
  };
  if (words) {                                         // the only scales there are
    if (lane < Lds::kPerWave) {
      u32x4 v = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (piece + i * 4 < scale_bytes) v[i] = ld4(scales + piece + i * 4);
      *reinterpret_cast<u32x4*>(s_mem + scales_at(0, 0) + (wave * Lds::kPerWave + lane) * 16) = v;
    }
    scales = a.w;                                      // later stages read 16 bytes of no use
  }
  auto load_scales = [&](int k0, uint32_t at) {
    if (lane >= Lds::kPerWave || (words && k0 == 0)) return;
    const int want = (Lds::kBatch == 1 ? k0 / 16 : k0 / (2 * kDepth) * 16) + piece;
    const uint8_t* from = scales + (want < last_piece ? want : last_piece);
    __builtin_amdgcn_global_load_lds(
        (const __attribute__((address_space(1))) uint32_t*)(uintptr_t)from,
        (__attribute__((address_space(3))) uint32_t*)(lds_u8*)(s_mem + scales_at(k0, at) +
                                                               wave * Lds::kPerWave * 16),
        16, 0, 0);
  };
  auto load = [&](int k0, uint32_t at) {               // past the depth: zeros
    if (Lds::kBatch == 1 || !(k0 & kDepth)) load_scales(k0, at);
    const uint32_t w = (uint32_t)k0 + wk * kDepth + chunk * 16 < (uint32_t)a.K ? wo + k0 : kOutside;
    uint8_t* to = s_mem + at + kRowBytes + wave * 2048;
    if (a.stream_w) {
      stream_to_lds(rw0, w, (lds_u8*)to);
      stream_to_lds(rw1, w, (lds_u8*)(to + 1024));
    } else {
      load_to_lds(rw0, w, (lds_u8*)to);
      load_to_lds(rw1, w, (lds_u8*)(to + 1024));
    }
#pragma unroll
    for (int g = 0; g < kRowLoads; ++g) {              // eight rows of a 128 of the depth
      const int n = g * 8 + wave, r = n % (ROWS / 8) * 8 + lr;
      const uint32_t k = (uint32_t)k0 + n / (ROWS / 8) * kDepth + chunk * 16;
      load_to_lds(ra, k < (uint32_t)a.K ? (uint32_t)r * (uint32_t)a.a_pitch + k : kOutside,
                  (lds_u8*)(s_mem + at + n * 1024));
    }
  };
#pragma unroll
  for (int s = 0; s + 1 < STAGES; ++s) load(s * kDepth * WK, s * kStage);

  const int row = lane & 15, quarter = lane / 16;
  const uint32_t place = place_of(row, quarter);
  const uint32_t mine = row * Lds::kRowScales + quarter * 2;
  f32x4 acc[MT] = {};
  auto multiply = [&](auto row_tiles) {
    constexpr int M = row_tiles.value;
    uint32_t at = 0, fill = (STAGES - 1) * kStage;     // stage to read, stage to fill
    for (int k0 = 0; k0 < a.K; k0 += kDepth * WK) {
      meet<(STAGES - 2) * kLoads>();                   // this stage is there, the last is read
      load(k0 + (STAGES - 1) * kDepth * WK, fill);
      i32x4 wv[2], av[2][M];
      const int k = k0 + wk * kDepth;                  // the wavefront's part of the stage
      const uint32_t mask = depth_mask(k, quarter, a.K);
      // its scales in their piece, and how far that lies before the place it was meant for
      const int first = k / 256 * 16;
      const int behind = words || first < last_piece ? 0 : first - last_piece;
      const uint32_t ps = scales_at(k0, at) + (Lds::kBatch == 1 ? k / 16 - k0 / 16 : k / 16 - first) +
                          (behind < 16 ? behind : 16) + mine;
      const int sw = (int)(two_scales(s_mem + ps + wc * 16 * Lds::kRowScales) & mask);
      int sa[M];
#pragma unroll
      for (int i = 0; i < M; ++i)
        sa[i] = (int)(two_scales(s_mem + ps + (WC + i) * 16 * Lds::kRowScales) & mask);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t p = at + (place ^ (h * 32));
        wv[h] = *(const i32x4*)(s_mem + kRowBytes + wave * 2048 + p);
#pragma unroll
        for (int i = 0; i < M; ++i)
          av[h][i] = *(const i32x4*)(s_mem + wk * (ROWS * kDepth) + i * 16 * kDepth + p);
      }
#pragma unroll
      for (int i = 0; i < M; ++i) {
        acc[i] = multiply_mx<0, 0>(wv[0], av[0][i], acc[i], sw, sa[i]);
        acc[i] = multiply_mx<1, 1>(wv[1], av[1][i], acc[i], sw, sa[i]);
      }
      at = at + kStage == STAGES * kStage ? 0 : at + kStage;
      fill = fill + kStage == STAGES * kStage ? 0 : fill + kStage;
    }
  };
  const int mt = (t.rows + 15) / 16;
  if (ROWS == 16 || mt == 1) multiply(std::integral_constant<int, 1>());
  else if (mt == 2) multiply(std::integral_constant<int, ROWS == 16 ? 1 : 2>());
  else multiply(std::integral_constant<int, MT>());
  meet<0>();                                           // loads past the end have landed

  // tile (w, i): channels of wavefront column w, rows 16 i..; a lane's four
  // sums are channels quarter * 4 .. + 3 of row `row`
  auto store = [&](int w, int i, f32x4 sum) {
    const int r = i * 16 + row;
    const int lc = w * step + (quarter * 4) % step, c = t.piece * WC * step + lc;
    const bool in = r < t.rows && c < out;
    float v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      v[q] = sum[q];
      if (a.swiglu) v[q] = silu(v[q]) * __shfl_xor(v[q], 32, kWave);   // gate lanes, up lanes
    }
    if (in && !(a.swiglu && quarter > 1))
      st4x2(a.y + (t.row + r) * out + c, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  };
  if constexpr (WK == 1) {
#pragma unroll
    for (int i = 0; i < MT; ++i)
      if (i < mt) store(wc, i, acc[i]);
  } else {
    f32x4* s_acc = reinterpret_cast<f32x4*>(s_mem);    // [wavefront][row tile][lane]
#pragma unroll
    for (int i = 0; i < MT; ++i) s_acc[(wave * MT + i) * kWave + lane] = acc[i];
    __syncthreads();
    for (int n = wave; n < WC * mt; n += 8) {
      const int w = n % WC, i = n / WC;
      f32x4 sum = s_acc[(w * MT + i) * kWave + lane];
#pragma unroll
      for (int g = 1; g < WK; ++g) sum += s_acc[((g * WC + w) * MT + i) * kWave + lane];
      store(w, i, sum);
    }
  }
}

template <int HEIGHT, int WAY>
hipError_t launch_tile(const MatmulMxArgs& a, int group, hipStream_t stream) {
  constexpr Way w = kMxWay[WAY];
  static_assert(w.rows == HEIGHT && w.channels == kTile, "the rule's tile");
  hipLaunchKernelGGL((matmul_mx_tile_kernel<HEIGHT>), dim3(256), dim3(kTileThreads), 0, stream, a,
                     pieces_of(a, w), group);
  return hipGetLastError();
}

template <int ROWS, int WC, int WK, int STAGES, int WAY>
hipError_t launch_stream(const MatmulMxArgs& a, hipStream_t stream) {
  constexpr Way w = kMxWay[WAY];
  static_assert(w.rows == ROWS && w.channels == 16 * WC && w.depth == kDepth * WK,
                "the rule's tile");
  const int64_t groups = (tiles_of(a, w) + 255) / 256 * 256;
  MatmulMxArgs m = a;
  m.stream_w = weights_read_once(a);
  hipLaunchKernelGGL((matmul_mx_stream_kernel<ROWS, WC, WK, STAGES>), dim3((unsigned)groups),
                     dim3(kTileThreads), 0, stream, m, pieces_of(a, w));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_matmul_mx(const MatmulMxArgs& a, hipStream_t stream) {
  switch (choose_mx_way(a)) {
    case kTile256: return launch_tile<256, kTile256>(a, 6, stream);
    case kTile128: return launch_tile<128, kTile128>(a, 6, stream);
    case kWide: return launch_stream<64, 8, 1, 3, kWide>(a, stream);
    case kHalf: return launch_stream<64, 4, 2, 3, kHalf>(a, stream);
    case kHalfTwo: return launch_stream<64, 4, 2, 2, kHalfTwo>(a, stream);
    case kNarrow: return launch_stream<64, 2, 4, 3, kNarrow>(a, stream);
    case kFewRows: return launch_stream<16, 2, 4, 3, kFewRows>(a, stream);
    case kOneRow: return launch_stream<16, 1, 8, 2, kOneRow>(a, stream);
    default: return hipErrorInvalidConfiguration;
  }
}

}  // namespace moe
