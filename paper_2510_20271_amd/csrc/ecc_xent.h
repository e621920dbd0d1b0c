// Arguments of the kernels of the linear head's cross entropy (ecc_xent.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ecc_types.h"

namespace ecc {

// reductions, ECC_MEAN / ECC_SUM / ECC_EACH of include/ecc.h
constexpr int kMean = 0, kSum = 1, kEach = 2;

struct XentArgs {
  const void *h, *w;      // hidden [rows][dim], weight [classes][dim]
  const int64_t* labels;  // [rows]; `ignore`: the row is left out
  int64_t rows, classes;
  int dim, reduction;
  int64_t ignore;
  float* loss;            // forward out: [1] or [rows]
  // [rows][2], forward out (or null), backward in: log sum_v exp z_iv, and 1 - p_label without a difference of near numbers
  double* stats;
  int64_t* counted;       // [1], rows that are not left out: forward out (or null), backward in
  const float* up;        // backward: upstream gradient, [1] or [rows]
  void *dh, *dw;          // backward out, either may be null
  void* ws;
};

// what a call takes, and what any call of these sizes does (aligned: whose operands are 16-byte aligned)
size_t xent_workspace_bytes(const XentArgs& a, int dtype, bool backward);
size_t xent_workspace_bytes(int64_t rows, int dim, int64_t classes, int dtype, bool backward, bool aligned);
hipError_t launch_xent_fwd(const XentArgs& a, int dtype, hipStream_t st);
hipError_t launch_xent_bwd(const XentArgs& a, int dtype, hipStream_t st);

}  // namespace ecc
