// Instances of the product kernels for one element type (included by the ecc_xent_*.hip files).
#pragma once
#include <atomic>

#include "ecc_xent_product.h"

namespace ecc {

template <auto KERNEL, int SHARED>
static hipError_t product_go(const ProductArgs& g, int threads, hipStream_t st) {
  if (SHARED > 64 << 10) {  // (told once for each kernel and device)
    static std::atomic<uint64_t> told{0};
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    const uint64_t bit = (uint64_t)1 << (device & 63);
    if (device > 63 || !(told.load(std::memory_order_relaxed) & bit)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, SHARED);
      if (e != hipSuccess) return e;
      told.fetch_or(bit, std::memory_order_relaxed);
    }
  }
  hipLaunchKernelGGL(KERNEL, dim3((unsigned)(g.tiles_m * g.tiles_n * g.splits)), dim3((unsigned)threads), SHARED, st, g);
  return hipGetLastError();
}

template <typename T, int BM, int BN, int WM, int WN, int STAGES>
static hipError_t product_shape(int kind, int mode, const ProductArgs& g, hipStream_t st) {
  constexpr int kShared = STAGES * (BM + BN) * 128, kThreads = WM * WN * 64;
  if (kind == kLogits && mode == kForward)
    return product_go<product_kernel<T, kLogits, kForward, BM, BN, WM, WN, STAGES>, kShared>(g, kThreads, st);
  if (kind == kLogits && mode == kSums)
    return product_go<product_kernel<T, kLogits, kSums, BM, BN, WM, WN, STAGES>, kShared>(g, kThreads, st);
  if (kind == kLogits)
    return product_go<product_kernel<T, kLogits, kBackward, BM, BN, WM, WN, STAGES>, kShared>(g, kThreads, st);
  if (kind == kHidden) return product_go<product_kernel<T, kHidden, 0, BM, BN, WM, WN, STAGES>, kShared>(g, kThreads, st);
  return product_go<product_kernel<T, kWeight, 0, BM, BN, WM, WN, STAGES>, kShared>(g, kThreads, st);
}

template <typename T>
hipError_t launch_product(int kind, int mode, int shape, ProductArgs g, hipStream_t st) {
  const ProductPlan& p = kPlans[shape];
  g.tiles_m = (int)((g.M + p.bm - 1) / p.bm);
  g.tiles_n = (int)((g.N + p.bn - 1) / p.bn);
  g.total = (int)((g.K + kDepth<T> - 1) / kDepth<T>);
  g.steps = (g.total + g.splits - 1) / g.splits;
  g.splits = (g.total + g.steps - 1) / g.steps;  // (no run is empty)
  const int turns = g.steps * (kind == kLogits ? 1 : kPlanes<T>);
  // One turn needs one tile in LDS, which leaves room for more blocks (385475 x 18 x 599 in float16: logits 176 us with two,
  // 145 with one); thin tiles are four ahead where there are turns to come (7 x 710 x 24651 in float16, 12 turns: logits 12.4 us with two,
  // 10.0 with four; 4 turns, 32 x 128 x 1000 in float32: 7.2 and 7.4).
  switch (shape) {
    case 0: return product_shape<T, 256, 256, 2, 4, 2>(kind, mode, g, st);
    case 1: return turns == 1 ? product_shape<T, 128, 128, 2, 2, 1>(kind, mode, g, st)
                              : product_shape<T, 128, 128, 2, 2, 2>(kind, mode, g, st);
    case 2: return turns == 1  ? product_shape<T, 128, 32, 4, 1, 1>(kind, mode, g, st)
                   : turns < 4 ? product_shape<T, 128, 32, 4, 1, 2>(kind, mode, g, st)
                               : product_shape<T, 128, 32, 4, 1, 4>(kind, mode, g, st);
    case 3: return turns == 1  ? product_shape<T, 32, 128, 1, 4, 1>(kind, mode, g, st)
                   : turns < 4 ? product_shape<T, 32, 128, 1, 4, 2>(kind, mode, g, st)
                               : product_shape<T, 32, 128, 1, 4, 4>(kind, mode, g, st);
    case 4: return turns == 1 ? product_shape<T, 64, 256, 1, 4, 1>(kind, mode, g, st)
                              : product_shape<T, 64, 256, 1, 4, 2>(kind, mode, g, st);
    default: return turns == 1 ? product_shape<T, 128, 64, 4, 1, 1>(kind, mode, g, st)
                               : product_shape<T, 128, 64, 4, 1, 3>(kind, mode, g, st);
  }
}

}  // namespace ecc
