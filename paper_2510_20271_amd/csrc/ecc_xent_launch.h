// Instances of the product kernels for one pair of element types (included by the ecc_xent_*.hip files).
#pragma once
#include "ecc_xent_product.h"

namespace ecc {

template <typename T, typename O, int BM, int BN, int WM, int WN, int STAGES>
static hipError_t product_shape(int kind, bool forward, const ProductArgs& g, hipStream_t st) {
  constexpr int kShared = STAGES * (BM + BN) * kDepth * 2;
  const dim3 grid((unsigned)(g.tiles_m * g.tiles_n * g.splits)), block(WM * WN * 64);
  const auto go = [&](auto kernel) -> hipError_t {
    if (kShared > 64 << 10) {
      const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kShared);
      if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, block, kShared, st, g);
    return hipGetLastError();
  };
  if (kind == kLogits) return forward ? go(product_kernel<T, O, kLogits, true, BM, BN, WM, WN, STAGES>)
                                      : go(product_kernel<T, O, kLogits, false, BM, BN, WM, WN, STAGES>);
  if (kind == kHidden) return go(product_kernel<T, O, kHidden, false, BM, BN, WM, WN, STAGES>);
  return go(product_kernel<T, O, kWeight, false, BM, BN, WM, WN, STAGES>);
}

template <typename T, typename O>
hipError_t launch_product(int kind, bool forward, int shape, ProductArgs g, hipStream_t st) {
  const ProductPlan& p = kPlans[shape];
  g.tiles_m = (int)((g.M + p.bm - 1) / p.bm);
  g.tiles_n = (int)((g.N + p.bn - 1) / p.bn);
  g.total = (int)((g.K + kDepth - 1) / kDepth);
  g.steps = (g.total + g.splits - 1) / g.splits;
  g.splits = (g.total + g.steps - 1) / g.steps;  // (no run is empty)
  const int turns = g.steps * (sizeof(O) == 4 ? 6 : 1);
  switch (shape) {
    case 0: return product_shape<T, O, 256, 256, 2, 4, 2>(kind, forward, g, st);
    case 1: return product_shape<T, O, 128, 128, 2, 2, 2>(kind, forward, g, st);
    // four tiles in LDS leave room for half the blocks: only where there are tiles to come (one tile of 64 elements, 524288 x 64 x
    // 21 in bfloat16: 20 us with two, 28 with four; six turns or more, 32 x 128 x 1000 in float32: 10.4 with two, 7.8 with four)
    case 2: return turns < 4 ? product_shape<T, O, 128, 32, 4, 1, 2>(kind, forward, g, st)
                             : product_shape<T, O, 128, 32, 4, 1, 4>(kind, forward, g, st);
    case 3: return turns < 4 ? product_shape<T, O, 32, 128, 1, 4, 2>(kind, forward, g, st)
                             : product_shape<T, O, 32, 128, 1, 4, 4>(kind, forward, g, st);
    default: return product_shape<T, O, 64, 256, 1, 4, 2>(kind, forward, g, st);
  }
}

}  // namespace ecc
