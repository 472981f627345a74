// The grouped products in bf16.
#include "product_launch.h"

namespace nimble {
template int launch_product<OfBf16, kMostGroups>(const ProductArgs&, const nimble_product_plan&, hipStream_t);
}
