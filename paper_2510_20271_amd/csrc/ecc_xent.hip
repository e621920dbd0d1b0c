// Softmax cross entropy of a linear head, in pieces of the classes:
//   z_iv = <h_i, W_v>,   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_{i,label},
//   dz_iv = (exp(z_iv - lse_i) - [v = label_i]) g_i,   dh = dz W,   dW = dz^T h.
// The logits are never kept: the forward pass leaves a maximum and a sum for each row and piece, the backward pass forms
// dz of one piece at a time.
#include "ecc_xent.h"

#include <algorithm>

namespace ecc {

constexpr int kTile = 64, kDeep = 16;          // a block's tile of a product and its steps along the summed axis
constexpr int64_t kPieceBytes = (int64_t)64 << 20;

// acc[i][j] += sum_k a(m0 + ty 4 + i, k) b(k, n0 + tx 4 + j) for 16 x 16 threads; a and b give 0 outside
template <typename A, typename B>
__device__ __forceinline__ void tile_product(const A& a, const B& b, int64_t m0, int64_t n0, int64_t K, float (&acc)[4][4]) {
  __shared__ float as[kDeep][kTile + 1], bs[kDeep][kTile + 1];
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  for (int64_t k0 = 0; k0 < K; k0 += kDeep) {
    for (int e = tid; e < kDeep * kTile; e += 256) {
      const int k = e % kDeep, i = e / kDeep;
      as[k][i] = k0 + k < K ? a(m0 + i, k0 + k) : 0.0f;
      bs[k][i] = k0 + k < K ? b(k0 + k, n0 + i) : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kDeep; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(as[k][ty * 4 + i], bs[k][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
}

// (m, s) stands for s exp(m); a sum of exponentials under a running maximum
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  if (top == -INFINITY) return;
  s = s * __expf(m - top) + s2 * __expf(m2 - top);
  m = top;
}

// piece sums: part[row][tile] = (maximum, sum), and the label's logit
template <typename T>
__global__ __launch_bounds__(256) void xent_sums_kernel(XentArgs a, float2* part, float* picked, int64_t tiles) {
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  const T *h = static_cast<const T*>(a.h), *w = static_cast<const T*>(a.w);
  tile_product([&](int64_t m, int64_t k) { return m < a.rows ? widen(h[m * a.dim + k]) : 0.0f; },
               [&](int64_t k, int64_t n) { return n < a.classes ? widen(w[n * a.dim + k]) : 0.0f; }, m0, n0, a.dim, acc);
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + ty * 4 + i;
    float m = -INFINITY, s = 0.0f;
    const int64_t label = row < a.rows ? a.labels[row] : -1;
    for (int j = 0; j < 4; ++j) {
      const int64_t v = n0 + tx * 4 + j;
      if (v >= a.classes) continue;
      if (acc[i][j] != acc[i][j]) { m = INFINITY; s = NAN; }
      else join(m, s, acc[i][j], 1.0f);
      if (v == label && row < a.rows) picked[row] = acc[i][j];
    }
    for (int o = 8; o > 0; o >>= 1) {
      const float m2 = __shfl_xor(m, o), s2 = __shfl_xor(s, o);
      join(m, s, m2, s2);
    }
    if (tx == 0 && row < a.rows) part[row * tiles + blockIdx.x] = make_float2(m, s);
  }
}

// a row's pieces joined: lse and the row's loss
__global__ __launch_bounds__(64) void xent_rows_kernel(XentArgs a, const float2* part, const float* picked, float* each,
                                                       int64_t tiles) {
  const int64_t row = blockIdx.x;
  float m = -INFINITY;
  for (int64_t t = threadIdx.x; t < tiles; t += 64) m = fmaxf(m, part[row * tiles + t].x);
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  double s = 0.0;
  for (int64_t t = threadIdx.x; t < tiles; t += 64) {
    const float2 p = part[row * tiles + t];
    s += (double)p.y * (p.x == m ? 1.0 : (double)__expf(p.x - m));
  }
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if (threadIdx.x != 0) return;
  const double lse = (double)m + log(s);
  if (a.lse) a.lse[row] = (float)lse;
  const int64_t label = a.labels[row];
  each[row] = label == a.ignore ? 0.0f : label < 0 || label >= a.classes ? NAN : (float)(lse - (double)picked[row]);
}

__global__ __launch_bounds__(256) void xent_mean_kernel(XentArgs a, const float* each) {
  __shared__ double part[256];
  __shared__ int64_t cnt[256];
  double s = 0.0;
  int64_t n = 0;
  for (int64_t i = threadIdx.x; i < a.rows; i += 256) {
    s += (double)each[i];
    n += a.labels[i] != a.ignore;
  }
  part[threadIdx.x] = s;
  cnt[threadIdx.x] = n;
  __syncthreads();
  if (threadIdx.x != 0) return;
  for (int k = 1; k < 256; ++k) { s += part[k]; n += cnt[k]; }
  if (a.counted) a.counted[0] = n;
  if (a.reduction != kEach) a.loss[0] = (float)(a.reduction == kMean ? s / (double)(n > 0 ? n : 1) : s);
}

// dz of the classes v0 .. v0 + count
template <typename T>
__global__ __launch_bounds__(256) void xent_dz_kernel(XentArgs a, float* dz, int64_t v0, int64_t count) {
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = v0 + (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  const T *h = static_cast<const T*>(a.h), *w = static_cast<const T*>(a.w);
  tile_product([&](int64_t m, int64_t k) { return m < a.rows ? widen(h[m * a.dim + k]) : 0.0f; },
               [&](int64_t k, int64_t n) { return n < a.classes ? widen(w[n * a.dim + k]) : 0.0f; }, m0, n0, a.dim, acc);
  for (int i = 0; i < 4; ++i) {
    const int64_t row = m0 + ty * 4 + i;
    if (row >= a.rows) continue;
    const int64_t label = a.labels[row];
    float g = a.reduction == kEach ? a.up[row] : a.up[0];
    if (a.reduction == kMean) g /= (float)(a.counted[0] > 0 ? a.counted[0] : 1);
    if (label != a.ignore && (label < 0 || label >= a.classes)) g = NAN;
    for (int j = 0; j < 4; ++j) {
      const int64_t v = n0 + tx * 4 + j;
      if (v >= v0 + count) continue;
      const float p = __expf(acc[i][j] - a.lse[row]) - (v == label ? 1.0f : 0.0f);
      dz[row * count + (v - v0)] = label == a.ignore ? 0.0f : p * g;
    }
  }
}

// dh (+)= dz W of a piece, summed in float32 over the pieces
template <typename T>
__global__ __launch_bounds__(256) void xent_dh_kernel(XentArgs a, const float* dz, float* sum, int64_t v0, int64_t count) {
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  const T* w = static_cast<const T*>(a.w);
  tile_product([&](int64_t m, int64_t k) { return m < a.rows ? dz[m * count + k] : 0.0f; },
               [&](int64_t k, int64_t n) { return n < a.dim ? widen(w[(v0 + k) * a.dim + n]) : 0.0f; }, m0, n0, count, acc);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t row = m0 + ty * 4 + i, k = n0 + tx * 4 + j;
      if (row >= a.rows || k >= a.dim) continue;
      const float v = acc[i][j] + (v0 > 0 ? sum[row * a.dim + k] : 0.0f);
      sum[row * a.dim + k] = v;
      if (v0 + count >= a.classes) static_cast<T*>(a.dh)[row * a.dim + k] = narrow<T>(v);
    }
}

// dW of a piece.  Rows left out count for nothing, whatever their features hold.
template <typename T>
__global__ __launch_bounds__(256) void xent_dw_kernel(XentArgs a, const float* dz, int64_t v0, int64_t count) {
  const int64_t m0 = (int64_t)blockIdx.y * kTile, n0 = (int64_t)blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  float acc[4][4] = {};
  const T* h = static_cast<const T*>(a.h);
  tile_product([&](int64_t m, int64_t k) { return m < count ? dz[k * count + m] : 0.0f; },
               [&](int64_t k, int64_t n) { return n < a.dim && a.labels[k] != a.ignore ? widen(h[k * a.dim + n]) : 0.0f; },
               m0, n0, a.rows, acc);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const int64_t v = m0 + ty * 4 + i, k = n0 + tx * 4 + j;
      if (v < count && k < a.dim) static_cast<T*>(a.dw)[(v0 + v) * a.dim + k] = narrow<T>(acc[i][j]);
    }
}

static size_t align256(size_t n) { return (n + 255) / 256 * 256; }
static int64_t tiles_of(int64_t n) { return (n + kTile - 1) / kTile; }
static int64_t piece_of(int64_t rows, int64_t classes) {
  return std::min<int64_t>(classes, std::max<int64_t>(kTile, kPieceBytes / 4 / rows / kTile * kTile));
}

size_t xent_workspace_bytes(int64_t rows, int dim, int64_t classes, int, bool backward) {
  if (backward) return align256(rows * piece_of(rows, classes) * 4) + align256(rows * dim * 4);
  return align256(rows * tiles_of(classes) * sizeof(float2)) + 2 * align256(rows * 4);
}

template <typename T>
static hipError_t xent_fwd(const XentArgs& a, hipStream_t st) {
  const int64_t tiles = tiles_of(a.classes);
  char* ws = static_cast<char*>(a.ws);
  float2* part = reinterpret_cast<float2*>(ws);
  float* picked = reinterpret_cast<float*>(ws + align256(a.rows * tiles * sizeof(float2)));
  float* each = a.reduction == kEach ? a.loss : picked + align256(a.rows * 4) / 4;
  hipLaunchKernelGGL(xent_sums_kernel<T>, dim3((unsigned)tiles, (unsigned)tiles_of(a.rows)), dim3(256), 0, st, a, part,
                     picked, tiles);
  hipLaunchKernelGGL(xent_rows_kernel, dim3((unsigned)a.rows), dim3(64), 0, st, a, part, picked, each, tiles);
  hipLaunchKernelGGL(xent_mean_kernel, dim3(1), dim3(256), 0, st, a, each);
  return hipGetLastError();
}

template <typename T>
static hipError_t xent_bwd(const XentArgs& a, hipStream_t st) {
  const int64_t piece = piece_of(a.rows, a.classes);
  char* ws = static_cast<char*>(a.ws);
  float* dz = reinterpret_cast<float*>(ws);
  float* sum = reinterpret_cast<float*>(ws + align256(a.rows * piece * 4));
  for (int64_t v0 = 0; v0 < a.classes; v0 += piece) {
    const int64_t count = std::min(piece, a.classes - v0);
    const unsigned rt = (unsigned)tiles_of(a.rows), vt = (unsigned)tiles_of(count), dt = (unsigned)tiles_of(a.dim);
    hipLaunchKernelGGL(xent_dz_kernel<T>, dim3(vt, rt), dim3(256), 0, st, a, dz, v0, count);
    if (a.dh) hipLaunchKernelGGL(xent_dh_kernel<T>, dim3(dt, rt), dim3(256), 0, st, a, dz, sum, v0, count);
    if (a.dw) hipLaunchKernelGGL(xent_dw_kernel<T>, dim3(dt, vt), dim3(256), 0, st, a, dz, v0, count);
  }
  return hipGetLastError();
}

hipError_t launch_xent_fwd(const XentArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? xent_fwd<float>(a, st) : dtype == kF16 ? xent_fwd<half_t>(a, st) : xent_fwd<bf16_t>(a, st);
}
hipError_t launch_xent_bwd(const XentArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? xent_bwd<float>(a, st) : dtype == kF16 ? xent_bwd<half_t>(a, st) : xent_bwd<bf16_t>(a, st);
}

}  // namespace ecc
