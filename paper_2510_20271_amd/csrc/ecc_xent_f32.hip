// Products of the linear head's cross entropy for float32.
#include "ecc_xent_launch.h"

namespace ecc {
template hipError_t launch_product<float>(int, int, int, ProductArgs, hipStream_t);
}
