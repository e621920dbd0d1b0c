// Arguments and element functions of the normalisation kernels (ecc_norm.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ecc_types.h"

namespace ecc {

// activations, ECC_ACT_* of include/ecc.h
constexpr int kActNone = 0, kActRelu = 1, kActSilu = 2;

struct NormArgs {
  const void *x, *dy;   // [batch][points][C];  dy: backward only
  const float *w, *b;   // [C] or null (1 and 0)
  void *y, *dx;         // the outputs of the two directions (dx may be null)
  float *dw, *db;       // [C], either may be null
  double* stats;        // [batch][G][2]: mean and 1 / sqrt(var + eps); null in a forward pass that keeps none
  void* ws;
  int64_t batch, points;
  int C, G, act;
  float eps;
};

size_t norm_workspace_bytes(int64_t batch, int64_t points, int C, int G);
hipError_t launch_norm_fwd(const NormArgs& a, int dtype, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs& a, int dtype, hipStream_t st);

// 1 / (1 + exp(-v)) by the hardware's exp2 and reciprocal (an ulp each; for v below -88 the exponential is infinite and the
// gate 0, its limit)
__device__ __forceinline__ float gate_of(float v) { return __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

__device__ __forceinline__ float activate(float v, int act) {
  if (act == kActSilu) return v * gate_of(v);
  if (act == kActRelu) return v < 0.0f ? 0.0f : v;  // (a NaN stays one)
  return v;
}
__device__ __forceinline__ float slope(float v, int act) {
  if (act == kActSilu) {
    const float s = gate_of(v);
    return s * fmaf(v, 1.0f - s, 1.0f);
  }
  if (act == kActRelu) return v > 0.0f ? 1.0f : 0.0f;
  return 1.0f;
}

}  // namespace ecc
