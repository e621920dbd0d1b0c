// Products of the linear head's cross entropy for float32 and few rows.
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<float, float, kOne>(int, int, int, ProductArgs, hipStream_t);
}
