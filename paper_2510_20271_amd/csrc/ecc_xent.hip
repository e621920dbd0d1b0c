// Softmax cross entropy of a linear head, in pieces of the classes:
//   z_iv = <h_i, W_v>,   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_{i,label},
//   dz_iv = (exp(z_iv - lse_i) - [v = label_i]) g_i,   dh = dz W,   dW = dz^T h.
// The logits are never kept: the forward pass leaves a maximum and a sum for each row and tile of classes, the backward pass
// forms dz of one piece of the classes at a time, in planes of the operands' type, for the two products that read it.
//
// Matrix products bound it (ecc_xent_product.h): rows x dim x classes multiply-adds forward; backward three times that in float32, five
// times in 16-bit types, whose dz has two planes.
#include "ecc_xent.h"

#include <algorithm>
#include <numeric>
#include <type_traits>

#include "ecc_xent_product.h"

namespace ecc {

// float16 holds dz as a multiple of 2^-14 of the largest upstream gradient: the probabilities of a large vocabulary are far below its
// least number otherwise.  (They are at most 1: 2^14 is in range.  Two planes are good to 2^-39 of the largest, half a step of
// float16's least numbers wherever that gradient times a column's sum of weights is below 2^14.)
constexpr float kHalfScale = 16384.0f;

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }
static int64_t up_to(int64_t n, int64_t k) { return (n + k - 1) / k * k; }

// ---- operands --------------------------------------------------------------------------------------------------------------
// One operand to be laid out as the products take them: [rows][ld], zeros behind a row's end.  blocks: 0 where the caller's own
// memory will do.
struct Lay {
  const void* from;
  void* to;
  int64_t rows, blocks;
};
// A thread lays out chunks of 8 elements: of row `row` from element k.  Rows start anywhere, so whole chunks are fetched at the
// alignment of an element (8 fetches of an element each: 72 us for 125 MB of float32, 47 so).
constexpr int kLayTurns = 4;
template <typename T>
struct Eight { T e[8]; };
template <typename T>
__device__ __forceinline__ Eight<T> eight_of(const Lay& l, int dim, int64_t row, int k) {
  const T* from = static_cast<const T*>(l.from) + row * dim + k;
  Eight<T> w;
  if (k + 8 <= dim) {
    __builtin_memcpy(&w, from, sizeof(w));
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w.e[i] = k + i < dim ? from[i] : (T)0;
  }
  return w;
}
template <typename T>
__device__ __forceinline__ void lay_chunks(const Lay& l, int dim, int ld, int64_t block) {
  using Bits = typename std::conditional<sizeof(T) == 4, unsigned, unsigned short>::type;
  const int64_t all = l.rows * ld, at = (block * kLayTurns * 256 + threadIdx.x) * 8;
  const int hop = 256 * 8 / ld, move = 256 * 8 - hop * ld;  // rows and elements from one turn to the next
  int64_t row = at / ld;
  int k = (int)(at - row * ld);
#pragma unroll
  for (int t = 0; t < kLayTurns; ++t) {
    const int64_t here = at + t * 256 * 8;
    if (here >= all) return;
    const Eight<Bits> w = eight_of<Bits>(l, dim, row, k);
    __builtin_memcpy(__builtin_assume_aligned(static_cast<Bits*>(l.to) + here, 16), &w, sizeof(w));
    row += hop;
    k += move;
    if (k >= ld) {
      k -= ld;
      ++row;
    }
  }
}

// ---- rows ------------------------------------------------------------------------------------------------------------------
// s: the sum of the exponentials under the maximum m, but the label's
__device__ __forceinline__ float xent_row(const XentArgs& a, int64_t row, float m, double s, const float* picked, float* each) {
  const int64_t label = a.labels[row];
  const bool has = label >= 0 && label < a.classes;
  // below the maximum, and the sum with the label's exponential; where that is most of it, log1p of the others' share keeps a small
  // loss's digits
  const double d = has ? (double)m - (double)picked[row] : 0.0, all = has ? s + exp(-d) : s;
  if (a.stats) {
    a.stats[row * 2] = (double)m + log(all);
    a.stats[row * 2 + 1] = s / all;
  }
  const double loss = d < 40.0 ? log1p(s * exp(d)) : d + log(all);
  return each[row] = label == a.ignore ? 0.0f : has ? (float)loss : NAN;
}
// A row's tiles joined by `team` lanes (a power of two).
__global__ __launch_bounds__(256) void xent_rows_kernel(XentArgs a, const float2* part, const float* picked, float* each,
                                                        int64_t parts, int team, int64_t row0) {
  const int64_t row = row0 + ((int64_t)blockIdx.x * 256 + threadIdx.x) / team;
  const int lane = threadIdx.x & (team - 1);
  const bool in = row < a.rows;  // (whole waves take part in the exchanges)
  const float2* p = part + (in ? row : 0) * parts;
  float m = -INFINITY;
  for (int64_t t = lane; t < parts; t += team) m = fmaxf(m, p[t].x);
  for (int o = team / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  double s = 0.0;
  for (int64_t t = lane; t < parts; t += team) s += (double)p[t].y * (p[t].x == m ? 1.0 : (double)__expf(p[t].x - m));
  for (int o = team / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (in && lane == 0) xent_row(a, row, m, s, picked, each);
}
// The same with a block for a row, where rows are few and tiles many (one row, 4096 tiles: 32 us by a wave, 6 by a block).
__global__ __launch_bounds__(1024) void xent_long_row_kernel(XentArgs a, const float2* part, const float* picked, float* each,
                                                             int64_t parts) {
  __shared__ float top[16];
  __shared__ double sum[16];
  const int64_t row = blockIdx.x;
  const float2* p = part + row * parts;
  float m = -INFINITY;
  for (int64_t t = threadIdx.x; t < parts; t += 1024) m = fmaxf(m, p[t].x);
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
  __syncthreads();
  for (int k = 0; k < 16; ++k) m = fmaxf(m, top[k]);
  double s = 0.0;
  for (int64_t t = threadIdx.x; t < parts; t += 1024) s += (double)p[t].y * (p[t].x == m ? 1.0 : (double)__expf(p[t].x - m));
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) sum[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  for (int k = 0; k < 16; ++k) s += sum[k];
  xent_row(a, row, m, s, picked, each);
}

// Logits whose sums were split (few tiles, long rows of features): a row's maximum and sum, as a tile's epilogue leaves them ...
__global__ __launch_bounds__(256) void xent_fold_kernel(XentArgs a, const float* sums, int splits, float2* part, float* picked,
                                                        int team) {
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / team;
  const int lane = threadIdx.x & (team - 1);
  const bool in = row < a.rows;
  const int64_t all = a.rows * a.classes, label = in ? a.labels[row] : -1;
  const float* z = sums + (in ? row : 0) * a.classes;
  float m = -INFINITY, s = 0.0f;
  for (int64_t v = lane; v < a.classes; v += team) {
    float x = 0.0f;
#pragma unroll 4
    for (int k = 0; k < splits; ++k) x += z[k * all + v];
    if (in && v == label) picked[row] = x;
    const float top = fmaxf(m, x), base = top == -INFINITY ? 0.0f : top;
    s = s * __expf(m - base) + (v == label ? 0.0f : __expf(x - base));
    m = top;
  }
  for (int o = team / 2; o > 0; o >>= 1) {
    const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o), top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    s = s * __expf(m - base) + s2 * __expf(m2 - base);
    m = top;
  }
  if (in && lane == 0) part[row] = make_float2(m, s);
}
// ... or their gradient, [planes][rows][ld], for `count` classes from v0
template <typename T>
__global__ __launch_bounds__(256) void xent_dz_kernel(XentArgs a, const float* sums, int splits, int64_t v0, int64_t count, int64_t ld,
                                                      const float* row_scale, T* dz) {
  const int64_t all = a.rows * ld, n = a.rows * count;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / ld, v = i - row * ld, label = a.labels[row];
    float f = 0.0f;
    if (v < count && label != a.ignore) {
      float x = sums[row * count + v];
      for (int k = 1; k < splits; ++k) x += sums[k * n + row * count + v];
      const double lse = a.stats[row * 2];
      const float high = (float)lse, low = (float)(lse - (double)high);
      f = (v0 + v == label ? -(float)a.stats[row * 2 + 1] : __expf((x - high) - low)) * row_scale[row];
    }
#pragma unroll
    for (int k = 0; k < kPlanes<T>; ++k) {
      const T e = narrow<T>(f);
      dz[k * all + i] = e;
      f -= widen(e);
    }
  }
}

// Sum of the rows' losses and their count, a run of rows a block; one block: the loss itself.
struct RowSum { double sum; long long count; };
constexpr int kSumThreads = 1024;

__device__ __forceinline__ void xent_finish(const XentArgs& a, double s, long long n) {
  if (a.counted) a.counted[0] = n;
  if (a.reduction != kEach) a.loss[0] = (float)(a.reduction == kMean ? s / (double)(n > 0 ? n : 1) : s);
}
__global__ __launch_bounds__(kSumThreads) void xent_sum_kernel(XentArgs a, const float* each, int64_t per, RowSum* out) {
  __shared__ double sum[kSumThreads];
  __shared__ long long count[kSumThreads];
  const int t = threadIdx.x;
  double s = 0.0;
  long long n = 0;
  const int64_t end = min(a.rows, (int64_t)(blockIdx.x + 1) * per);
#pragma unroll 4
  for (int64_t i = (int64_t)blockIdx.x * per + t; i < end; i += kSumThreads) {
    s += (double)each[i];
    n += a.labels[i] != a.ignore;
  }
  sum[t] = s;
  count[t] = n;
  __syncthreads();
  for (int o = kSumThreads / 2; o > 0; o >>= 1) {
    if (t < o) {
      sum[t] += sum[t + o];
      count[t] += count[t + o];
    }
    __syncthreads();
  }
  if (t != 0) return;
  if (gridDim.x == 1) xent_finish(a, sum[0], count[0]);
  else out[blockIdx.x] = {sum[0], count[0]};
}
// Everything behind the sums in one block, where there is little of it: the rows, then the loss.
__global__ __launch_bounds__(kSumThreads) void xent_short_kernel(XentArgs a, const float2* part, const float* picked, float* each,
                                                                 int64_t parts, int team) {
  __shared__ double sum[kSumThreads / 64];
  __shared__ long long count[kSumThreads / 64];
  const int lane = threadIdx.x & (team - 1), step = kSumThreads / team;
  double loss = 0.0;
  long long n = 0;
  for (int64_t r0 = 0; r0 < a.rows; r0 += step) {  // (block-uniform)
    const int64_t row = r0 + threadIdx.x / team;
    const bool in = row < a.rows;
    const float2* p = part + (in ? row : 0) * parts;
    float m = -INFINITY;
    for (int64_t t = lane; t < parts; t += team) m = fmaxf(m, p[t].x);
    for (int o = team / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    double s = 0.0;
    for (int64_t t = lane; t < parts; t += team) s += (double)p[t].y * (p[t].x == m ? 1.0 : (double)__expf(p[t].x - m));
    for (int o = team / 2; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (in && lane == 0) {
      loss += (double)xent_row(a, row, m, s, picked, each);
      n += a.labels[row] != a.ignore;
    }
  }
  for (int o = 32; o > 0; o >>= 1) {
    loss += __shfl_xor(loss, o);
    n += __shfl_xor(n, o);
  }
  if ((threadIdx.x & 63) == 0) {
    sum[threadIdx.x >> 6] = loss;
    count[threadIdx.x >> 6] = n;
  }
  __syncthreads();
  if (threadIdx.x != 0) return;
  loss = 0.0;
  n = 0;
  for (int k = 0; k < kSumThreads / 64; ++k) {
    loss += sum[k];
    n += count[k];
  }
  xent_finish(a, loss, n);
}
__global__ __launch_bounds__(64) void xent_total_kernel(XentArgs a, const RowSum* part, int blocks) {
  double s = 0.0;
  long long n = 0;
  for (int k = threadIdx.x; k < blocks; k += 64) {
    s += part[k].sum;
    n += part[k].count;
  }
  for (int o = 32; o > 0; o >>= 1) {
    s += __shfl_xor(s, o);
    n += __shfl_xor(n, o);
  }
  if (threadIdx.x == 0) xent_finish(a, s, n);
}

// the largest finite |upstream gradient| of the rows that count, in one block: only where float16 meets a gradient for each row
__global__ __launch_bounds__(kSumThreads) void xent_top_kernel(XentArgs a, float* top) {
  __shared__ float part[kSumThreads / 64];
  float m = 0.0f;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < a.rows; i += kSumThreads) {
    const float v = fabsf(a.up[i]);
    if (v < INFINITY && a.labels[i] != a.ignore) m = fmaxf(m, v);
  }
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int k = 0; k < kSumThreads / 64; ++k) m = fmaxf(m, part[k]);
  top[0] = m;
}

// What each row's dz is multiplied by, which rows count, and what the products are multiplied by.
struct Scales {
  const float* top;  // float16 with a gradient for each row: the largest of them
  float* row_scale;
  unsigned long long* keep;
  float* scale;      // [2]: of both gradients: a factor and an exponent, which would be subnormal as one number where they are not
  bool half;         // dz is held in float16
  int64_t blocks;    // 0: none wanted
};
__device__ __forceinline__ void scale_rows(const XentArgs& a, const Scales& c, int64_t block) {
  const int64_t i = block * 256 + threadIdx.x;
  float by = c.half ? kHalfScale : 1.0f;
  double back = 1.0 / (double)by;
  if (a.reduction == kEach) {
    if (c.half) {
      const float t = c.top[0] > 0.0f ? fmaxf(c.top[0], 0x1p-100f) : 1.0f;  // (kHalfScale / t stays finite)
      by /= t;
      back *= (double)t;
    }
  } else {
    back *= (double)a.up[0];
    if (a.reduction == kMean) back /= (double)(a.counted[0] > 0 ? a.counted[0] : 1);
  }
  bool counts = false;
  if (i < a.rows) {
    const int64_t label = a.labels[i];
    counts = label != a.ignore;
    float v = a.reduction == kEach ? a.up[i] * by : by;
    if (counts && (label < 0 || label >= a.classes)) v = NAN;
    c.row_scale[i] = v;
  }
  const unsigned long long bits = __ballot(counts);
  if ((threadIdx.x & 63) == 0 && i < a.rows) c.keep[i / 64] = bits;
  if (i == 0) {
    int e = 0;
    const bool finite = fabs(back) < (double)INFINITY;
    c.scale[0] = finite ? (float)frexp(back, &e) : (float)back;
    c.scale[1] = (float)e;
  }
}

// What comes before the products, in one launch: both operands laid out and the rows' scales, a run of blocks each.
template <typename T>
__global__ __launch_bounds__(256) void xent_prepare_kernel(XentArgs a, Lay h, Lay w, int ld, Scales c) {
  int64_t block = blockIdx.x;
  if (block < h.blocks) return lay_chunks<T>(h, a.dim, ld, block);
  block -= h.blocks;
  if (block < w.blocks) return lay_chunks<T>(w, a.dim, ld, block);
  scale_rows(a, c, block - w.blocks);
}

// out = narrow(scale[0] 2^scale[1] * sum of the splits), `team` threads to an element, added in a fixed order.  labels: of out's rows of `dim`
// elements, where those that are left out are zeros (hidden's gradient), or null
template <typename O>
__global__ __launch_bounds__(256) void xent_out_kernel(const float* sums, int splits, int64_t n, const float* scale, int team,
                                                       const int64_t* labels, int64_t ignore, int dim, O* out) {
  __shared__ float room[256];
  const int cols = 256 / team, col = threadIdx.x % cols, lane = threadIdx.x / cols;
  const float by = scale[0];
  const int exponent = (int)scale[1];
  for (int64_t i0 = (int64_t)blockIdx.x * cols; i0 < n; i0 += (int64_t)gridDim.x * cols) {  // (block-uniform)
    const int64_t i = i0 + col;
    float s = 0.0f;
    if (i < n) {
#pragma unroll 8
      for (int k = lane; k < splits; k += team) s += sums[k * n + i];
    }
    if (team > 1) {
      __syncthreads();
      room[threadIdx.x] = s;
      __syncthreads();
      for (int o = team / 2; o > 0; o >>= 1) {
        if (lane < o) room[threadIdx.x] = s = s + room[threadIdx.x + o * cols];
        __syncthreads();
      }
    }
    if (i < n && lane == 0) {
      const int64_t row = n <= UINT32_MAX ? (int64_t)((uint32_t)i / (uint32_t)dim) : i / dim;
      out[i] = narrow<O>(!labels || labels[row] != ignore ? ldexpf(s * by, exponent) : 0.0f);
    }
  }
}

// ---- plans -----------------------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = (int64_t)128 << 20;  // of two bytes of every dz (a plane of it), and of laid-out weights
constexpr int64_t kPieceFew = (int64_t)1 << 30;      // of laid-out weights where rows are few, and of any backward
constexpr int64_t kPieceMost = (int64_t)1 << 17;     // classes of a piece (offsets within a tile are 32 bits)
constexpr int64_t kSumsBytes = (int64_t)256 << 20;   // of the splits' results
constexpr int64_t kLaunchThreads = (int64_t)1 << 31; // of a launch (a grid may have less than 2^32)

static int ld_of(int dim) { return (int)up_to(dim, 8); }

// Tiles of 256 x 256 (`large`) where they fill the card (one block a CU) and the summed axis is eight turns or more; of 128 x 128
// otherwise, two blocks a CU, so that one's start and end run beside the other's products.  Thin products have thin tiles.
// (385475 x 18 x 599 in float16, one turn: logits 228 us by large tiles, 176 by the others.)  float32 logits by the smaller ones: a
// round of tiles is four times as long there as a 16-bit one, and the last one is seldom full (4096 x 512 x 10007: 383 us, 436 by
// large tiles; gradients, whose sums are split into whole rounds: of the weight 385 by large ones, 553).
static int shape_of(int64_t M, int64_t N, int64_t runs, int64_t turns, bool large) {
  if (N <= 32) return 2;
  if (M <= 32) return 3;
  if (N <= 64) return 5;
  if (M <= 64 && N > 128) return 4;
  const int64_t tiles = (M + 255) / 256 * ((N + 255) / 256);
  return large && M > 128 && N > 128 && turns >= 8 && tiles * runs >= 256 ? 0 : 1;
}
// The summed axis in runs, so that blocks fill the card: eight turns a run or more, results within kSumsBytes.
static int splits_of(int64_t M, int64_t N, int64_t K, int shape, int planes, int depth) {
  const ProductPlan& p = kPlans[shape];
  const int64_t blocks = (M + p.bm - 1) / p.bm * ((N + p.bn - 1) / p.bn), total = (K + depth - 1) / depth;
  const int64_t fill = shape == 0 ? 256 : 512;  // blocks that the card holds
  int64_t want = std::min(std::max<int64_t>(1, fill / blocks), std::max<int64_t>(1, total * planes / 8));
  want = std::max<int64_t>(1, std::min({want, total, kSumsBytes / (M * N * 4)}));
  const int64_t steps = (total + want - 1) / want;
  return (int)((total + steps - 1) / steps);
}

struct XentPlan {
  int64_t fwd_piece, piece, ld_dz;
  int fwd_shape, fwd_splits, shape, splits, hidden_shape, hidden_splits, weight_shape, weight_splits;
  int64_t parts;
  bool hidden_sums;
  size_t lay_h, lay_w, lay_w_fwd;                        // bytes of laid-out operands
  size_t part, picked, each, row_sums, sums_f;           // forward
  size_t dz, sums_z, sums_h, sums_w, row_scale, keep, scalars;  // backward
};

// Whether the products can read the caller's own memory: rows of whole 16-byte chunks, aligned.
static bool whole_chunks(int dim, int dtype) { return dim % (dtype == kF32 ? 4 : 8) == 0; }
static bool as_it_is(const XentArgs& a, const void* p, int dtype) {
  return whole_chunks(a.dim, dtype) && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

// own_h, own_w: of hidden and the weight; the other needs room for a copy (the weight: of a piece)
static XentPlan xent_plan(int64_t rows, int dim, int64_t classes, int dtype, bool own_h, bool own_w) {
  XentPlan p{};
  const int64_t size = dtype == kF32 ? 4 : 2;
  const int planes = dtype == kF32 ? kPlanes<float> : kPlanes<half_t>, depth = 128 / (int)size;
  const int64_t ld = ld_of(dim);
  // Pieces of at most `most` classes, equal ones.  Where the last piece is small anyway the others hold whole rounds of 256 large
  // tiles (2048 rows, 50021 classes: 32768 and 17253, 4 + 3 rounds of blocks; halves: 4 + 4).
  const auto pieces = [&](int64_t most) {
    most = std::max<int64_t>(256, most / 256 * 256);
    const int64_t count = (classes + most - 1) / most;
    if (count == 1) return classes;
    const int64_t tiles_n = (rows + 255) / 256, round = 256 / std::gcd<int64_t>(256, tiles_n) * 256;
    if (most / round * round * count >= classes) return most / round * round;
    return up_to((classes + count - 1) / count, 256);
  };
  const int64_t dim_turns = (dim + depth - 1) / depth;
  p.fwd_shape = shape_of(classes, rows, 1, dim_turns, size == 2);
  p.parts = (classes + kPlans[p.fwd_shape].bm - 1) / kPlans[p.fwd_shape].bm * kPlans[p.fwd_shape].wm;
  // (few rows: pieces of as many tiles as the card holds blocks, within kPieceFew; 38 x 2030 x 92507 in float32: products 485 us by
  // pieces of kPieceBytes, 266 so)
  const int64_t tiles = (rows + kPlans[p.fwd_shape].bn - 1) / kPlans[p.fwd_shape].bn;
  const int64_t full = std::min((512 + tiles - 1) / tiles * kPlans[p.fwd_shape].bm, kPieceFew / (ld * size));
  p.fwd_piece = pieces(std::min(kPieceMost * 8, std::max(full, kPieceBytes / (ld * size))));
  p.piece = pieces(std::min({kPieceMost, kPieceBytes / (rows * 2), own_w ? kPieceMost : kPieceFew / (ld * size)}));
  p.ld_dz = up_to(p.piece, 8);
  p.shape = shape_of(p.piece, rows, 1, dim_turns, size == 2);
  // logits by split sums: where their tiles leave compute units idle through a long sum
  const auto split = [&](int64_t M, int shape) {
    const int splits = dim_turns < 16 || M > 1024 ? 1 : splits_of(M, rows, dim, shape, 1, depth);
    return splits >= 4 ? splits : 1;
  };
  p.fwd_splits = classes <= p.fwd_piece ? split(classes, p.fwd_shape) : 1;
  p.splits = split(p.piece, p.shape);
  if (p.fwd_splits > 1) p.parts = 1;
  const int64_t long_k = std::max<int64_t>(1, p.piece / depth / 16), long_n = std::max<int64_t>(1, rows / depth / 16);
  p.hidden_shape = shape_of(dim, rows, long_k, p.piece / depth * planes, true);
  p.hidden_splits = splits_of(dim, rows, p.piece, p.hidden_shape, planes, depth);
  p.hidden_sums = p.hidden_splits > 1 || p.piece < classes;
  p.weight_shape = shape_of(dim, p.piece, long_n, rows / depth * planes, true);
  p.weight_splits = splits_of(dim, p.piece, rows, p.weight_shape, planes, depth);
  p.lay_h = own_h ? 0 : align256((size_t)rows * ld * size);
  p.lay_w = own_w ? 0 : align256((size_t)p.piece * ld * size);
  p.lay_w_fwd = own_w ? 0 : align256((size_t)p.fwd_piece * ld * size);
  p.part = align256((size_t)rows * p.parts * sizeof(float2));
  p.picked = p.each = align256((size_t)rows * 4);
  p.row_sums = align256(256 * sizeof(RowSum));
  p.sums_f = p.fwd_splits > 1 ? align256((size_t)p.fwd_splits * rows * classes * 4) : 0;
  p.sums_z = p.splits > 1 ? align256((size_t)p.splits * rows * p.piece * 4) : 0;
  p.dz = align256((size_t)rows * p.ld_dz * size * planes);
  p.sums_h = p.hidden_sums ? align256((size_t)p.hidden_splits * rows * dim * 4) : 0;
  p.sums_w = p.weight_splits > 1 ? align256((size_t)p.weight_splits * p.piece * dim * 4) : 0;
  p.row_scale = align256((size_t)rows * 4);
  p.keep = align256((size_t)(rows + 63) / 64 * 8);
  p.scalars = 256;
  return p;
}

static XentPlan xent_plan(const XentArgs& a, int dtype) {
  return xent_plan(a.rows, a.dim, a.classes, dtype, as_it_is(a, a.h, dtype), as_it_is(a, a.w, dtype));
}
static size_t bytes_of(const XentPlan& p, bool backward) {
  if (!backward) return p.lay_h + p.lay_w_fwd + p.part + p.picked + p.each + p.row_sums + p.sums_f;
  return p.lay_h + p.lay_w + p.dz + p.sums_z + p.sums_h + p.sums_w + p.row_scale + p.keep + p.scalars;
}
size_t xent_workspace_bytes(const XentArgs& a, int dtype, bool backward) { return bytes_of(xent_plan(a, dtype), backward); }
size_t xent_workspace_bytes(int64_t rows, int dim, int64_t classes, int dtype, bool backward, bool aligned) {
  const bool whole = whole_chunks(dim, dtype);
  if (aligned || !whole) return bytes_of(xent_plan(rows, dim, classes, dtype, whole, whole), backward);
  size_t most = 0;  // (any alignment)
  for (int own = 0; own < 4; ++own)
    most = std::max(most, bytes_of(xent_plan(rows, dim, classes, dtype, own & 1, own & 2), backward));
  return most;
}

struct Room {  // hands out a workspace
  char* at;
  void* take(size_t n) {
    void* p = at;
    at += n;
    return p;
  }
};

// An operand as the products see it, and what has to be laid out for that.
static Matrix laid(const void* from, int64_t rows, int dim, void* room, bool own, Lay* l) {
  const int ld = ld_of(dim);
  *l = {from, room, rows, own ? 0 : (rows * ld / 8 + 256 * kLayTurns - 1) / (256 * kLayTurns)};
  if (own) return {from, rows, dim, 0};
  return {room, rows, ld, rows * ld};
}
template <typename T>
static void prepare(const XentArgs& a, const Lay& h, const Lay& w, const Scales& c, hipStream_t st) {
  const int64_t blocks = h.blocks + w.blocks + c.blocks;
  if (blocks) hipLaunchKernelGGL(xent_prepare_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, st, a, h, w, ld_of(a.dim), c);
}

template <typename T>
static hipError_t xent_fwd(const XentArgs& a, int dtype, hipStream_t st) {
  const XentPlan p = xent_plan(a, dtype);
  Room room{static_cast<char*>(a.ws)};
  void *lay_h = room.take(p.lay_h), *lay_w = room.take(p.lay_w_fwd);
  float2* part = static_cast<float2*>(room.take(p.part));
  float* picked = static_cast<float*>(room.take(p.picked));
  float* each = static_cast<float*>(room.take(p.each));
  RowSum* row_sums = static_cast<RowSum*>(room.take(p.row_sums));
  float* sums = static_cast<float*>(room.take(p.sums_f));
  if (a.reduction == kEach) each = a.loss;
  const T *h = static_cast<const T*>(a.h), *w = static_cast<const T*>(a.w);
  ProductArgs g{};
  Lay lh, lw;
  g.b = laid(h, a.rows, a.dim, lay_h, as_it_is(a, h, dtype), &lh);
  g.N = a.rows;
  g.K = a.dim;
  g.splits = p.fwd_splits;
  g.sums = sums;
  g.labels = a.labels;
  g.part = part;
  g.parts = p.parts;
  g.picked = picked;
  const bool own = as_it_is(a, w, dtype);
  const ProductPlan& plan = kPlans[p.fwd_shape];
  // (all classes at once where nothing is laid out, but no more threads than a grid may have: whole tiles, of up to 512 each)
  const int64_t most = std::max<int64_t>(1, kLaunchThreads / 512 / ((a.rows + plan.bn - 1) / plan.bn)) * plan.bm;
  const int64_t piece = p.fwd_splits > 1 ? a.classes : std::min(own ? a.classes : p.fwd_piece, most);
  hipError_t e = hipSuccess;
  for (int64_t v0 = 0; v0 < a.classes && e == hipSuccess; v0 += piece) {
    const int64_t count = std::min(piece, a.classes - v0);
    g.a = laid(w + v0 * a.dim, count, a.dim, lay_w, own, &lw);
    prepare<T>(a, lh, lw, Scales{}, st);
    lh.blocks = 0;
    g.M = count;
    g.v0 = v0;
    g.part0 = v0 / plan.bm * plan.wm;
    e = launch_product<T>(kLogits, p.fwd_splits > 1 ? kSums : kForward, p.fwd_shape, g, st);
  }
  if (e != hipSuccess) return e;
  int team = 64;
  if (p.fwd_splits > 1) {
    while (team > 1 && team / 2 >= a.classes) team /= 2;
    hipLaunchKernelGGL(xent_fold_kernel, dim3((unsigned)((a.rows * team + 255) / 256)), dim3(256), 0, st, a, sums, p.fwd_splits,
                       part, picked, team);
    team = 64;
  }
  while (team > 1 && team / 2 >= p.parts) team /= 2;
  if (p.parts <= 512 && a.rows * (p.parts + 8) <= 16384) {
    hipLaunchKernelGGL(xent_short_kernel, dim3(1), dim3(kSumThreads), 0, st, a, part, picked, each, p.parts, team);
    return hipGetLastError();
  }
  if (a.rows < 512 && p.parts > 512) {
    hipLaunchKernelGGL(xent_long_row_kernel, dim3((unsigned)a.rows), dim3(1024), 0, st, a, part, picked, each, p.parts);
  } else {
    // (one lane of a team ends its row, in float64: no larger teams than fill the card)
    while (team > 1 && a.rows * (team / 2) >= 131072 && p.parts <= 4 * team) team /= 2;
    const int64_t step = kLaunchThreads / team;
    for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
      const unsigned blocks = (unsigned)((std::min(step, a.rows - r0) * team + 255) / 256);
      hipLaunchKernelGGL(xent_rows_kernel, dim3(blocks), dim3(256), 0, st, a, part, picked, each, p.parts, team, r0);
    }
  }
  if (a.reduction != kEach || a.counted) {
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(256, a.rows / 8192));
    const int64_t per = (a.rows + blocks - 1) / blocks;
    hipLaunchKernelGGL(xent_sum_kernel, dim3((unsigned)blocks), dim3(kSumThreads), 0, st, a, each, per, row_sums);
    if (blocks > 1) hipLaunchKernelGGL(xent_total_kernel, dim3(1), dim3(64), 0, st, a, row_sums, (int)blocks);
  }
  return hipGetLastError();
}

template <typename T>
static void xent_out(const float* sums, int splits, int64_t n, const float* scale, const int64_t* labels, int64_t ignore, int dim,
                     T* out, hipStream_t st) {
  const int team = splits >= 64 ? 16 : splits >= 16 ? 4 : 1;
  const unsigned blocks = (unsigned)std::min<int64_t>((n + 256 / team - 1) / (256 / team), 4096);
  hipLaunchKernelGGL(xent_out_kernel<T>, dim3(blocks), dim3(256), 0, st, sums, splits, n, scale, team, labels,
                     ignore, dim, out);
}

template <typename T>
static hipError_t xent_bwd(const XentArgs& a, int dtype, hipStream_t st) {
  const XentPlan p = xent_plan(a, dtype);
  Room room{static_cast<char*>(a.ws)};
  void *lay_h = room.take(p.lay_h), *lay_w = room.take(p.lay_w), *dz = room.take(p.dz);
  float* sums_z = static_cast<float*>(room.take(p.sums_z));
  float* sums_h = static_cast<float*>(room.take(p.sums_h));
  float* sums_w = static_cast<float*>(room.take(p.sums_w));
  float* row_scale = static_cast<float*>(room.take(p.row_scale));
  unsigned long long* keep = static_cast<unsigned long long*>(room.take(p.keep));
  float* scale = static_cast<float*>(room.take(p.scalars));
  const T *h = static_cast<const T*>(a.h), *w = static_cast<const T*>(a.w);
  const bool half = dtype == kF16;
  if (half && a.reduction == kEach)
    hipLaunchKernelGGL(xent_top_kernel, dim3(1), dim3(kSumThreads), 0, st, a, scale + 2);
  Scales scales{scale + 2, row_scale, keep, scale, half, (a.rows + 255) / 256};
  Lay lh, lw;
  const Matrix hm = laid(h, a.rows, a.dim, lay_h, as_it_is(a, h, dtype), &lh);
  const bool own = as_it_is(a, w, dtype);
  hipError_t e = hipSuccess;
  for (int64_t v0 = 0; v0 < a.classes; v0 += p.piece) {
    const int64_t count = std::min(p.piece, a.classes - v0), ld = up_to(count, 8);
    const Matrix wm = laid(w + v0 * a.dim, count, a.dim, lay_w, own, &lw);
    prepare<T>(a, lh, lw, scales, st);
    lh.blocks = scales.blocks = 0;
    const Matrix zm{dz, a.rows, ld, a.rows * ld};
    ProductArgs g{};
    // dz of the piece
    g.a = wm; g.b = hm; g.M = count; g.N = a.rows; g.K = a.dim; g.splits = p.splits; g.sums = sums_z; g.add = 0;
    g.labels = a.labels; g.ignore = a.ignore; g.v0 = v0; g.stats = a.stats; g.row_scale = row_scale;
    g.dz = dz; g.dz_ld = ld; g.dz_plane = a.rows * ld;
    e = launch_product<T>(kLogits, p.splits > 1 ? kSums : kBackward, p.shape, g, st);
    if (e != hipSuccess) return e;
    if (p.splits > 1) {
      const unsigned blocks = (unsigned)std::min<int64_t>((a.rows * ld + 255) / 256, 4096);
      hipLaunchKernelGGL(xent_dz_kernel<T>, dim3(blocks), dim3(256), 0, st, a, sums_z, p.splits, v0, count, ld, row_scale,
                         static_cast<T*>(dz));
    }
    if (a.dh) {
      g.a = wm; g.b = zm; g.M = a.dim; g.N = a.rows; g.K = count;
      g.splits = std::min(p.hidden_splits, splits_of(a.dim, a.rows, count, p.hidden_shape, kPlanes<T>, kDepth<T>));
      g.sums = p.hidden_sums ? sums_h : nullptr;
      g.add = v0 > 0;
      g.out = a.dh;
      g.scale = scale;
      if ((e = launch_product<T>(kHidden, 0, p.hidden_shape, g, st)) != hipSuccess) return e;
    }
    if (a.dw) {
      T* out = static_cast<T*>(a.dw) + v0 * a.dim;
      g.a = hm; g.b = zm; g.M = a.dim; g.N = count; g.K = a.rows; g.keep = keep;
      g.splits = p.weight_splits;
      g.sums = p.weight_splits > 1 ? sums_w : nullptr;
      g.add = 0;
      g.out = out;
      g.scale = scale;
      if ((e = launch_product<T>(kWeight, 0, p.weight_shape, g, st)) != hipSuccess) return e;
      if (g.sums) xent_out(sums_w, p.weight_splits, count * a.dim, scale, nullptr, 0, a.dim, out, st);
    }
  }
  if (a.dh && p.hidden_sums)
    xent_out(sums_h, p.hidden_splits, a.rows * a.dim, scale, a.labels, a.ignore, a.dim, static_cast<T*>(a.dh), st);
  return hipGetLastError();
}

hipError_t launch_xent_fwd(const XentArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? xent_fwd<float>(a, dtype, st) : dtype == kF16 ? xent_fwd<half_t>(a, dtype, st) : xent_fwd<bf16_t>(a, dtype, st);
}
hipError_t launch_xent_bwd(const XentArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? xent_bwd<float>(a, dtype, st) : dtype == kF16 ? xent_bwd<half_t>(a, dtype, st) : xent_bwd<bf16_t>(a, dtype, st);
}

}  // namespace ecc
