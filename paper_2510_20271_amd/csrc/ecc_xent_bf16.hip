// Products of the linear head's cross entropy for bfloat16.
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<bf16_t>(int, int, int, ProductArgs, hipStream_t);
}
