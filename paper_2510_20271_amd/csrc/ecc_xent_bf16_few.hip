// Products of the linear head's cross entropy for bfloat16 and few rows.
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<bf16_t, bf16_t, kTwo>(int, int, int, ProductArgs, hipStream_t);
}
