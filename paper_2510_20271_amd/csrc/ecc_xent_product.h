// The matrix products of the linear head's cross entropy on the matrix cores, summed in float32:
//   kLogits  C[v][i] = sum_k W[v][k] H[i][k]    logits of a tile, consumed where they are made: a maximum and a sum for each
//                                               row (forward), or their gradient dz (backward)
//   kHidden  C[k][i] = sum_v W[v][k] dZ[i][v]   gradient of hidden
//   kWeight  C[k][v] = sum_i H[i][k] dZ[i][v]   gradient of the weight
// The product is transposed against its result's layout: the accumulators of a 32 x 32 matrix instruction hold, in lane l,
// column l % 32 and rows 8 (r / 4) + 4 (l / 32) + r % 4, so a lane has a row's logits side by side (their maximum and sum need
// no exchange but one between two lanes) and four neighbours along a result's row (stores of 8 or 16 bytes).
//
// Elements are 16-bit or float32, each by the instruction of its type.  16-bit gradients dz have a second plane, what the first one's
// rounding left, so that the sums of them are off by no more than float32 sums are: that rounding (2^-9 of each dz for bfloat16) is as
// much as the result's own, and neither sum averages it out, over classes (hidden's gradient) or over rows, where one term is most of
// it.  It costs the two gradients' products twice the matrix instructions (8192 x 4096 x 131072 bfloat16 step: 48.0 ms, 31.0 with one
// plane).  float32 operands are multiplied as they are (two float16 planes of each, scaled by its largest value, stand for values down
// to 2^-39 of that one only: 4096 x 512 x 10007 step 1366 us so, 690 by planes that lost every row beside a class masked by -1e9).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ecc_types.h"

namespace ecc {

constexpr int kLogits = 0, kHidden = 1, kWeight = 2;
// of kLogits: what is made of them; kSums: nothing yet, their sums are split
constexpr int kBackward = 0, kForward = 1, kSums = 2;
// elements of a tile along the summed axis: 128 bytes
template <typename T> constexpr int kDepth = 128 / (int)sizeof(T);

// A matrix [planes][rows][ld] (dz: kPlanes, others one), rows of whole 16-byte chunks, 16-byte aligned; elements between a row's end and ld are 0.
struct Matrix {
  const void* p;
  int64_t rows, ld, plane;  // plane: elements from one plane to the next
};

struct ProductArgs {
  Matrix a, b;         // operands; summed along their rows' elements (kLogits: both; kHidden: b), else along their rows
  int64_t M, N, K;     // of C; K: elements summed along (rows of the operand that is summed along its rows)
  int tiles_m, tiles_n;
  int splits;          // the summed axis in so many runs of `steps` tiles, each with a result of its own
  int steps;           // tiles of the summed axis of a run; all: total
  int total;
  const unsigned long long* keep;  // kWeight: bit i of the rows that count (others read as zeros)
  // results
  float* sums;         // kHidden, kWeight, kSums: [splits][N][M], or null: straight to out
  int add;             //   added to what is there
  void* out;           // [N][M], times scale[0] 2^scale[1]
  const float* scale;
  // kLogits; kHidden: rows that are left out are zeros, whatever weights and scale hold
  const int64_t* labels;
  int64_t v0;          // the first class of this piece (M: its classes)
  float2* part;        // forward: [N][parts], parts part0 ..: the maximum, and the sum of exponentials but the label's
  int64_t parts, part0;
  float* picked;       // forward: the label's logit
  const double* stats;      // backward: [N][2], see XentArgs
  const float* row_scale;   // backward
  void* dz;            // backward: [planes][N][dz_ld]
  int64_t dz_ld, dz_plane;
  int64_t ignore;
};

template <typename T> struct Lanes;
template <> struct Lanes<bf16_t> {
  using V8 = __bf16 __attribute__((ext_vector_type(8)));
};
template <> struct Lanes<half_t> {
  using V8 = _Float16 __attribute__((ext_vector_type(8)));
};
template <> struct Lanes<float> {
  using V8 = float __attribute__((ext_vector_type(4)));  // (of a step of 8: half the lanes have the other four)
};
using Acc = float __attribute__((ext_vector_type(16)));
using Quad = short __attribute__((ext_vector_type(4)));
using LdsVoid = __attribute__((address_space(3))) void;

// matrix instructions of a step: float32's takes two elements along the summed axis, one of each half of the lanes
template <typename T> constexpr int kMmas = sizeof(T) == 4 ? 4 : 1;
__device__ __forceinline__ Acc mma(Lanes<bf16_t>::V8 a, Lanes<bf16_t>::V8 b, Acc c, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc mma(Lanes<half_t>::V8 a, Lanes<half_t>::V8 b, Acc c, int) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc mma(Lanes<float>::V8 a, Lanes<float>::V8 b, Acc c, int k) {
  return __builtin_amdgcn_mfma_f32_32x32x2f32(a[k], b[k], c, 0, 0, 0);
}

// planes of dz
template <typename T> constexpr int kPlanes = sizeof(T) == 2 ? 2 : 1;

constexpr int kFar = 0x7fffff00;       // an offset that no buffer holds: such a lane's 16 bytes read as zeros
constexpr int64_t kReach = 0x40000000;  // what a tile's offsets stay below

// One operand's tile in LDS, SIDE x kDepth<T>, and how a wave fetches and reads it.  Fetches go straight to LDS, 1 KB a wave
// instruction, to consecutive 16-byte chunks; which chunk of its row a lane fetches is permuted so that reading is free of bank
// conflicts.
// ALONG: the operand's rows run along the summed axis: rows of 128 bytes, two of which fill the banks, chunk c of row r at
// place c ^ (r / 2 & 7): 16 lanes read one chunk of 16 rows at a time.
// Otherwise the tile has kDepth rows of SIDE elements.  float32 is read element by element; 16-bit elements are read through
// the transposing LDS read: 16 lanes get 16 neighbouring
// elements of 4 rows, transposed.  Four rows and their 64 bytes fill the banks once: chunk c of row r at c ^ 4 (r & 3) (for
// rows of 128 bytes, of which two fill the banks, c ^ 4 (r / 2 & 1); rows of 64 bytes as they are).
// where an operand's next tile is, uniform over the block
template <typename T, bool ALONG>
struct Cursor {
  const char* at;
  int64_t left;  // bytes of the operand from there
  int64_t step;  // bytes to the next tile
  int64_t plane;
  __device__ __forceinline__ Cursor(const Matrix& m, int64_t origin, int64_t K, int k0) {
    const int64_t first = ALONG ? origin * m.ld : (int64_t)k0 * kDepth<T> * m.ld + origin;
    at = static_cast<const char*>(m.p) + first * (int64_t)sizeof(T);
    left = ((ALONG ? m.rows : K) * m.ld - first) * (int64_t)sizeof(T);
    step = ALONG ? 0 : (int64_t)128 * m.ld;
    plane = m.plane * (int64_t)sizeof(T);
  }
  __device__ __forceinline__ int reach() const { return (int)(left < 0 ? 0 : left < kReach ? left : kReach); }
  __device__ __forceinline__ void next() {
    at += step;
    left -= step;
  }
};

template <typename T, bool ALONG, int SIDE, int WAVES>
struct Tile {
  static constexpr int kBytes = SIDE * 128;
  static constexpr int kFetches = kBytes / 1024;
  static constexpr int kEach = kFetches / WAVES;
  static_assert(kFetches % WAVES == 0, "every wave fetches alike");
  static constexpr int kRow = ALONG ? 8 : SIDE * (int)sizeof(T) / 16;   // chunks of a row
  static constexpr int kReads = ALONG ? 1 : sizeof(T) == 4 ? 4 : 2;     // LDS instructions of an operand
  static constexpr int kPer = 16 / (int)sizeof(T);                      // elements of a chunk
  using V8 = typename Lanes<T>::V8;
  int offset[kEach];  // of this lane's chunk, in bytes from the tile's origin
  int mark[kEach];    // ALONG: the chunk's first element along the summed axis; otherwise its row

  __device__ __forceinline__ static int place(int row, int c) {
    if (ALONG) return c ^ (row >> 1 & 7);
    if (sizeof(T) == 4) return c;
    if (kRow >= 16) return c ^ ((row & 3) << 2);
    if (kRow == 8) return c ^ ((row >> 1 & 1) << 2);
    return c;
  }
  // origin: the tile's first row (ALONG) or column
  __device__ __forceinline__ void init(const Matrix& m, int64_t origin, int wave, int lane) {
#pragma unroll
    for (int f = 0; f < kEach; ++f) {
      const int at = (wave * kEach + f) * 64 + lane, row = at / kRow, c = place(row, at % kRow);
      offset[f] = (int)(row * m.ld * (int)sizeof(T)) + c * 16;
      mark[f] = ALONG ? c * kPer : row;
      if (!ALONG && origin + c * kPer >= m.ld) offset[f] = kFar;
    }
  }
  // A tile to LDS at `to`: the tile's origin is at `from`, which `left` bytes of the operand follow; k: its first element along
  // the summed axis (ALONG: `from` is the row's first element); keep: the rows that count (not ALONG)
  __device__ __forceinline__ void fetch(const char* from, int left, int ld, int k, unsigned char* to, int wave,
                                        unsigned long long keep) const {
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(from), 0, left, 0x00020000);
    const int end = ld - k;  // ALONG: elements of a row from here
#pragma unroll
    for (int f = 0; f < kEach; ++f) {
      int at = offset[f];
      if (ALONG) at = mark[f] < end ? at : kFar;
      else at = (keep >> mark[f]) & 1 ? at : kFar;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsVoid*)(to + (wave * kEach + f) * 1024), 16, at,
                                               ALONG ? __builtin_amdgcn_readfirstlane(k * (int)sizeof(T)) : 0, 0, 0);
    }
  }
  // operand of a matrix instruction: 32 rows / columns from `side`, a quarter of the tile's elements along the summed axis
  __device__ __forceinline__ static V8 read(const unsigned char* from, int side, int ks, int lane) {
    if (ALONG) {
      const int row = side + (lane & 31);
      return *reinterpret_cast<const V8*>(from + row * 128 + place(row, ks * 2 + (lane >> 5)) * 16);
    }
    if constexpr (sizeof(T) == 4) {
      V8 v;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        v[k] = *reinterpret_cast<const float*>(from + ((ks * 8 + (lane >> 5) * 4 + k) * SIDE + side + (lane & 31)) * 4);
      return v;
    }
    const int q = lane >> 4, i = lane & 15, row = ks * 16 + (q >> 1) * 8 + (i >> 2), col = side + (q & 1) * 16 + (i & 3) * 4;
    typedef __attribute__((address_space(3))) Quad LdsQuad;
    // (rows + 4: the same place)
    const unsigned char* at = from + row * (SIDE * 2) + place(row, col >> 3) * 16 + (i & 1) * 8;
    union { Quad q[2]; V8 v; } u;
    u.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad*)(at));
    u.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsQuad*)(at + 4 * SIDE * 2));
    return u.v;
  }
};

// The scheduler's order for a step: LDS reads of the next step's operands between this step's matrix instructions.
template <int MMAS, int READS>
__device__ __forceinline__ void interleave() {
  constexpr int each = (READS + MMAS - 1) / MMAS;
#pragma unroll
  for (int i = 0; i < MMAS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, each, 0);
  }
}

// Blocks in an order in which those that run at a time share operands: each of the eight dies takes a run of tiles, in bands of
// four tiles of M, M fastest.
__device__ __forceinline__ void tile_of(int block, int blocks, int tiles_m, int tiles_n, int& m, int& n, int& split) {
  const int each = blocks / 8, over = blocks % 8, die = block % 8;
  const int at = die * each + (die < over ? die : over) + block / 8;
  const int tiles = tiles_m * tiles_n;
  split = at / tiles;
  const int t = at - split * tiles, band = t / (4 * tiles_n), in = t - band * 4 * tiles_n;
  const int high = min(4, tiles_m - band * 4);
  n = in / high;
  m = band * 4 + in - n * high;
}

// A wave's results on their way to memory: 32 columns of C (rows of the result) of TM x 32 elements, turned in the wave's part of
// LDS so that stores run along the result's rows.  Chunk c of row n at c ^ n: writes and reads are spread over the banks.
template <typename E, int TM>
struct Turn {
  static constexpr int kRow = TM * 32 * sizeof(E), kChunks = kRow / 16, kBytes = 32 * kRow, kPer = 16 / sizeof(E);
  __device__ __forceinline__ static unsigned char* place(unsigned char* room, int n, int c) {
    return room + n * kRow + ((c ^ (n & (kChunks - 1))) << 4);
  }
  // four elements from column m (a multiple of 4) of row n
  __device__ __forceinline__ static void put(unsigned char* room, int n, int m, const E (&e)[4]) {
    unsigned char* at = place(room, n, m * (int)sizeof(E) / 16) + m * (int)sizeof(E) % 16;
    if constexpr (sizeof(E) == 4) {
      uint4 w;
      __builtin_memcpy(&w, e, 16);
      *reinterpret_cast<uint4*>(at) = w;
    } else {
      uint2 w;
      __builtin_memcpy(&w, e, 8);
      *reinterpret_cast<uint2*>(at) = w;
    }
  }
  // rows and columns that are there; out: element (0, 0), rows `ld` apart, of any alignment (142 x 1863 x 56007 in float16, gradient
  // of the weight: 290 us with stores of an element each for such rows, 167 so)
  __device__ __forceinline__ static void store(unsigned char* room, int lane, E* out, int64_t ld, int64_t rows, int64_t columns) {
#pragma unroll
    for (int k = 0; k < kChunks / 2; ++k) {
      const int at = k * 64 + lane, n = at / kChunks, c = at % kChunks;
      const uint4 w = *reinterpret_cast<const uint4*>(place(room, n, c));
      const int64_t left = columns - c * kPer;
      if (n >= rows || left <= 0) continue;
      E* to = out + n * ld + c * kPer;
      if (left >= kPer) {
        __builtin_memcpy(to, &w, 16);
      } else {
        E e[kPer];
        __builtin_memcpy(e, &w, 16);
#pragma unroll
        for (int i = 0; i < kPer; ++i)
          if (i < left) to[i] = e[i];
      }
    }
  }
};

// a distance between classes as far as a tile is concerned
__device__ __forceinline__ int near(int64_t d) { return (int)(d < -1 ? -1 : d > 1024 ? 1024 : d); }

// Waits until all but the last N fetches of this wave have landed and its LDS reads are done, then for the other waves.
template <int N>
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// BM x BN: a block's tile of C, WM x WN waves;  STAGES: tiles in LDS, all but one of them on their way (thin tiles are computed
// faster than one arrives)
template <typename T, int KIND, int MODE, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(const ProductArgs g) {
  extern __shared__ __align__(16) unsigned char smem[];
  constexpr int kWaves = WM * WN, TM = BM / WM / 32, TN = BN / WN / 32;
  using TA = Tile<T, KIND == kLogits, BM, kWaves>;
  using TB = Tile<T, KIND != kWeight, BN, kWaves>;
  constexpr int kStage = TA::kBytes + TB::kBytes;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int tm, tn, split;
  tile_of((int)blockIdx.x, (int)gridDim.x, g.tiles_m, g.tiles_n, tm, tn, split);
  const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
  constexpr int kTurns = KIND == kLogits ? 1 : kPlanes<T>;  // of a tile of the summed axis: one for each plane of dz
  const int k0 = split * g.steps, ktiles = min(g.steps, g.total - k0), turns = ktiles * kTurns;
  TA ta;
  TB tb;
  ta.init(g.a, m0, wave, lane);
  tb.init(g.b, n0, wave, lane);
  Acc acc[TM][TN] = {};
  // Where a wave has one accumulator there is room for a second: sums of eight tiles are added up there, so that a long sum is
  // rounded at a few of its steps only (one row against 131072 x 4096 in bfloat16: the loss 1.3e-6 off without).
  constexpr bool kTwoSums = TM * TN == 1;
  Acc total = {};

  // the next fetch: tile, plane, and the rows that count (read a turn ahead)
  Cursor<T, KIND == kLogits> ca(g.a, m0, g.K, k0);
  Cursor<T, KIND != kWeight> cb(g.b, n0, g.K, k0);
  int lk = k0, lj = 0;
  const auto* rows = (const __attribute__((address_space(4))) unsigned long long*)g.keep;  // (scalar reads)
  const auto rows_at = [&](int k) { return rows[k * kDepth<T> / 64] >> (k * kDepth<T> % 64); };
  unsigned long long keep = KIND == kWeight ? rows_at(lk) : ~0ull;
  const auto fetch = [&](int turn) {
    const int64_t plane = kTurns > 1 && lj == 1 ? cb.plane : 0;
    unsigned char* to = smem + turn % STAGES * kStage;
    const bool any = turn < turns;  // (behind the last tile nothing is read: zeros go where no one looks)
    ta.fetch(ca.at, any ? ca.reach() : 0, (int)g.a.ld, lk * kDepth<T>, to, wave, keep);
    tb.fetch(cb.at + plane, any ? cb.reach() : 0, (int)g.b.ld, lk * kDepth<T>, to + TA::kBytes, wave, ~0ull);
    if (kTurns == 1 || ++lj == kTurns) {
      lj = 0;
      ++lk;
      ca.next();
      cb.next();
      if (KIND == kWeight) keep = rows_at(min(lk, g.total - 1));
    }
  };
  const int am = (wave % WM) * (BM / WM), bn = (wave / WM) * (BN / WN);
  // (STAGES 1: for one turn)
#pragma unroll
  for (int t = 0; t < (STAGES > 1 ? STAGES - 1 : 1); ++t) fetch(t);
  for (int t = 0; t < turns; ++t) {
    wait_and_meet<STAGES < 3 ? 0 : (STAGES - 2) * (TA::kEach + TB::kEach)>();  // the tile is there, and the one before has been read
    const unsigned char* from = smem + t % STAGES * kStage;
    typename TA::V8 a[2][TM], b[2][TN];
    const auto read = [&](int ks) {
#pragma unroll
      for (int j = 0; j < TN; ++j) b[ks & 1][j] = TB::read(from + TA::kBytes, bn + j * 32, ks, lane);
#pragma unroll
      for (int i = 0; i < TM; ++i) a[ks & 1][i] = TA::read(from, am + i * 32, ks, lane);
    };
    read(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks + 1 < 4) read(ks + 1);
#pragma unroll
      for (int k = 0; k < kMmas<T>; ++k)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) acc[i][j] = mma(a[ks & 1][i], b[ks & 1][j], acc[i][j], k);
      interleave<TM * TN * kMmas<T>, TA::kReads * TM + TB::kReads * TN>();
      if (STAGES > 1 && ks == 0) fetch(t + STAGES - 1);
    }
    if (kTwoSums && STAGES > 1 && t % 8 == 7) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        total[r] += acc[0][0][r];
        acc[0][0][r] = 0.0f;
      }
    }
  }
  if (kTwoSums && STAGES > 1) {
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] += total[r];
  }
  wait_and_meet<0>();  // the last fetches have landed and the tiles are read: LDS is free

  const int rows0 = 4 * (lane >> 5);  // accumulator r is row 8 (r / 4) + rows0 + r % 4 of its 32
#pragma unroll
  for (int j = 0; j < TN; ++j) {
    const int64_t n = n0 + bn + j * 32 + (lane & 31);
    const bool in = n < g.N;
    if constexpr (KIND == kLogits && MODE == kForward) {
      const int want = near(in ? g.labels[n] - g.v0 - m0 - am - rows0 : -1), left = near(g.M - m0 - am - rows0);
      float top = -INFINITY, sum = 0.0f, picked = 0.0f;
      // a wave whose classes are all there and no row's label (almost all, with many classes): no comparisons
      const bool plain = left >= TM * 32 && __ballot(want >= 0 && want < TM * 32) == 0;
      if (plain) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = i * 32 + 8 * (r / 4) + r % 4;
            if (row < left) top = fmaxf(top, acc[i][j][r]);
            picked = row == want ? acc[i][j][r] : picked;
          }
      }
      top = fmaxf(top, __shfl_xor(top, 32));
      const float base = top == -INFINITY ? 0.0f : top;
      if (plain) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum += __expf(acc[i][j][r] - base);
      } else {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int row = i * 32 + 8 * (r / 4) + r % 4;
            if (row < left && row != want) sum += __expf(acc[i][j][r] - base);
          }
      }
      sum += __shfl_xor(sum, 32);
      if (want >= 0 && want < min(left, TM * 32) && !(want & 4)) g.picked[n] = picked;  // (a lane has rows 0 .. 3 of every 8)
      if (in && lane < 32) g.part[n * g.parts + g.part0 + (int64_t)tm * WM + wave % WM] = make_float2(top, sum);
    } else if constexpr (KIND == kLogits && MODE == kBackward) {
      const int64_t label = in ? g.labels[n] : -1;
      const int want = near(label - g.v0 - m0 - am - rows0), left = near(g.M - m0 - am - rows0);
      const bool counts = in && label != g.ignore;
      const double2 st = in ? reinterpret_cast<const double2*>(g.stats)[n] : make_double2(0.0, 0.0);
      const float lse = (float)st.x, rest = (float)(st.x - (double)lse), miss = (float)st.y, scale = in ? g.row_scale[n] : 0.0f;
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = i * 32 + 8 * (r / 4) + r % 4;
          const float p = row == want ? -miss : __expf((acc[i][j][r] - lse) - rest);
          acc[i][j][r] = counts && row < left ? p * scale : 0.0f;
        }
      using Out = Turn<T, TM>;
      unsigned char* room = smem + wave * Out::kBytes;
#pragma unroll
      for (int k = 0; k < kPlanes<T>; ++k) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            T e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {  // (and what is left for the next plane)
              float f = acc[i][j][q * 4 + r];
              e[r] = narrow<T>(f);
              if (kPlanes<T> > 1) f -= widen(e[r]);
              acc[i][j][q * 4 + r] = f;
            }
            Out::put(room, lane & 31, i * 32 + 8 * q + rows0, e);
          }
        const int64_t first = n0 + bn + j * 32;
        Out::store(room, lane, static_cast<T*>(g.dz) + k * g.dz_plane + first * g.dz_ld + m0 + am, g.dz_ld,
                   g.N - first, g.dz_ld - m0 - am);
      }
    } else {
      if (g.sums) {
        const bool four = g.M % 4 == 0;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int64_t m = m0 + am + i * 32 + 8 * q + rows0;
            if (!in || m >= g.M) continue;
            float* to = g.sums + ((int64_t)split * g.N + n) * g.M + m;
            if (four) {
              float4 w = make_float4(acc[i][j][q * 4], acc[i][j][q * 4 + 1], acc[i][j][q * 4 + 2], acc[i][j][q * 4 + 3]);
              if (g.add) {
                const float4 o = *reinterpret_cast<const float4*>(to);
                w.x += o.x; w.y += o.y; w.z += o.z; w.w += o.w;
              }
              *reinterpret_cast<float4*>(to) = w;
            } else {
#pragma unroll
              for (int r = 0; r < 4; ++r)
                if (m + r < g.M) to[r] = g.add ? to[r] + acc[i][j][q * 4 + r] : acc[i][j][q * 4 + r];
            }
          }
      } else {
        using Out = Turn<T, TM>;
        unsigned char* room = smem + wave * Out::kBytes;
        const float scale = g.scale[0];
        const int exponent = (int)g.scale[1];
        const bool counts = KIND != kHidden || (in && g.labels[n] != g.ignore);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            T e[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) e[r] = narrow<T>(counts ? ldexpf(acc[i][j][q * 4 + r] * scale, exponent) : 0.0f);
            Out::put(room, lane & 31, i * 32 + 8 * q + rows0, e);
          }
        const int64_t first = n0 + bn + j * 32;
        Out::store(room, lane, static_cast<T*>(g.out) + first * g.M + m0 + am, g.M, g.N - first, g.M - m0 - am);
      }
    }
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------------
// Tiles: 0: 256 x 256 (8 waves, a block a CU), 1: 128 x 128 (4 waves, two blocks), 2: 128 x 32, 3: 32 x 128, 4: 64 x 256,
// 5: 128 x 64
struct ProductPlan { int bm, bn, wm; };
constexpr ProductPlan kPlans[] = {{256, 256, 2}, {128, 128, 2}, {128, 32, 4}, {32, 128, 1}, {64, 256, 1}, {128, 64, 4}};

// g.a .. g.K, splits set; tiles, steps and total are filled in here
template <typename T>
hipError_t launch_product(int kind, int mode, int shape, ProductArgs g, hipStream_t st);

}  // namespace ecc
