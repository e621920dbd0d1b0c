// Products of the linear head's cross entropy for float32 (planes of float16).
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<half_t, float, kBoth>(int, int, int, ProductArgs, hipStream_t);
}
