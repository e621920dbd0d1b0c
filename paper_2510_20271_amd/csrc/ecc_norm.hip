// Group normalisation with an activation over channels-last features x [batch][points][C], G groups of Cg = C / G channels:
//   xhat = (x - mean) rstd over the points and channels of a group,   v = xhat w_c + b_c,   y = act(v)
// and its derivatives, with dv = dy act'(v) and m = points Cg:
//   db_c = sum dv,   dw_c = sum dv xhat,   dx = rstd (w_c dv - (1/m) sum_g w dv - (xhat / m) sum_g w dv xhat).
#include "ecc_norm.h"

namespace ecc {

constexpr int kNormBlock = 256;

__device__ __forceinline__ double block_sum(double v, double* part) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
  __syncthreads();
  if ((tid & 63) == 0) part[tid >> 6] = v;
  __syncthreads();
  double r = 0.0;
  for (int k = 0; k < kNormBlock / 64; ++k) r += part[k];
  return r;
}

// a block for each item and group: mean, squares about it, then the output
template <typename T>
__global__ __launch_bounds__(kNormBlock) void norm_fwd_kernel(NormArgs a) {
  __shared__ double part[kNormBlock / 64];
  const int64_t n = blockIdx.x / a.G;
  const int g = blockIdx.x % a.G, Cg = a.C / a.G;
  const T* x = static_cast<const T*>(a.x) + n * a.points * a.C;
  T* y = static_cast<T*>(a.y) + n * a.points * a.C;
  const int64_t m = a.points * Cg;
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < m; i += kNormBlock) s += (double)widen(x[i / Cg * a.C + g * Cg + i % Cg]);
  const double mean = block_sum(s, part) / (double)m;
  s = 0.0;
  for (int64_t i = threadIdx.x; i < m; i += kNormBlock) {
    const double d = (double)widen(x[i / Cg * a.C + g * Cg + i % Cg]) - mean;
    s += d * d;
  }
  const double rstd = 1.0 / sqrt(block_sum(s, part) / (double)m + (double)a.eps);
  if (a.stats && threadIdx.x == 0) {
    a.stats[(n * a.G + g) * 2] = mean;
    a.stats[(n * a.G + g) * 2 + 1] = rstd;
  }
  for (int64_t i = threadIdx.x; i < m; i += kNormBlock) {
    const int c = g * Cg + (int)(i % Cg);
    const int64_t at = i / Cg * a.C + c;
    const float xhat = (float)(((double)widen(x[at]) - mean) * rstd);
    y[at] = narrow<T>(activate(fmaf(xhat, a.w ? a.w[c] : 1.0f, a.b ? a.b[c] : 0.0f), a.act));
  }
}

template <typename T>
__device__ __forceinline__ void norm_terms(const NormArgs& a, int64_t n, int64_t at, int c, float& dv, float& xhat) {
  const double* st = a.stats + (n * a.G + c / (a.C / a.G)) * 2;
  const int64_t i = n * a.points * a.C + at;
  xhat = (float)(((double)widen(static_cast<const T*>(a.x)[i]) - st[0]) * st[1]);
  const float v = fmaf(xhat, a.w ? a.w[c] : 1.0f, a.b ? a.b[c] : 0.0f);
  dv = widen(static_cast<const T*>(a.dy)[i]) * slope(v, a.act);
}

// dx: a block for each item and group
template <typename T>
__global__ __launch_bounds__(kNormBlock) void norm_dx_kernel(NormArgs a) {
  __shared__ double part[kNormBlock / 64];
  const int64_t n = blockIdx.x / a.G;
  const int g = blockIdx.x % a.G, Cg = a.C / a.G;
  const int64_t m = a.points * Cg;
  double s1 = 0.0, s2 = 0.0;
  for (int64_t i = threadIdx.x; i < m; i += kNormBlock) {
    const int c = g * Cg + (int)(i % Cg);
    float dv, xhat;
    norm_terms<T>(a, n, i / Cg * a.C + c, c, dv, xhat);
    const double t = (double)dv * (a.w ? (double)a.w[c] : 1.0);
    s1 += t;
    s2 += t * (double)xhat;
  }
  const double m1 = block_sum(s1, part) / (double)m, m2 = block_sum(s2, part) / (double)m;
  const double rstd = a.stats[(n * a.G + g) * 2 + 1];
  for (int64_t i = threadIdx.x; i < m; i += kNormBlock) {
    const int c = g * Cg + (int)(i % Cg);
    const int64_t at = i / Cg * a.C + c;
    float dv, xhat;
    norm_terms<T>(a, n, at, c, dv, xhat);
    static_cast<T*>(a.dx)[n * a.points * a.C + at] =
        narrow<T>((float)(rstd * ((double)dv * (a.w ? (double)a.w[c] : 1.0) - m1 - (double)xhat * m2)));
  }
}

// dweight, dbias: a block for each channel
template <typename T>
__global__ __launch_bounds__(kNormBlock) void norm_dparam_kernel(NormArgs a) {
  __shared__ double part[kNormBlock / 64];
  const int c = blockIdx.x;
  double sw = 0.0, sb = 0.0;
  for (int64_t i = threadIdx.x; i < a.batch * a.points; i += kNormBlock) {
    float dv, xhat;
    norm_terms<T>(a, i / a.points, i % a.points * a.C + c, c, dv, xhat);
    sw += (double)dv * (double)xhat;
    sb += (double)dv;
  }
  sw = block_sum(sw, part);
  sb = block_sum(sb, part);
  if (threadIdx.x == 0) {
    if (a.dw) a.dw[c] = (float)sw;
    if (a.db) a.db[c] = (float)sb;
  }
}

size_t norm_workspace_bytes(int64_t, int64_t, int, int) { return 256; }

template <typename T>
static hipError_t norm_fwd(const NormArgs& a, hipStream_t st) {
  hipLaunchKernelGGL(norm_fwd_kernel<T>, dim3((unsigned)(a.batch * a.G)), dim3(kNormBlock), 0, st, a);
  return hipGetLastError();
}
template <typename T>
static hipError_t norm_bwd(const NormArgs& a, hipStream_t st) {
  if (a.dx) hipLaunchKernelGGL(norm_dx_kernel<T>, dim3((unsigned)(a.batch * a.G)), dim3(kNormBlock), 0, st, a);
  if (a.dw || a.db) hipLaunchKernelGGL(norm_dparam_kernel<T>, dim3((unsigned)a.C), dim3(kNormBlock), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_norm_fwd(const NormArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? norm_fwd<float>(a, st) : dtype == kF16 ? norm_fwd<half_t>(a, st) : norm_fwd<bf16_t>(a, st);
}
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, hipStream_t st) {
  return dtype == kF32 ? norm_bwd<float>(a, st) : dtype == kF16 ? norm_bwd<half_t>(a, st) : norm_bwd<bf16_t>(a, st);
}

}  // namespace ecc
