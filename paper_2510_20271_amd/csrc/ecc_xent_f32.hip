// Products of the linear head's cross entropy for float32 (planes of bfloat16).
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<bf16_t, float, 3>(int, int, int, ProductArgs, hipStream_t);
}
