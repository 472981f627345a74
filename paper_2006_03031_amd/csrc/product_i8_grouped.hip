// The grouped products in 8 bits.
#include "product_launch.h"

namespace nimble {
template int launch_product<OfInt8, kMostGroups>(const ProductArgs&, const nimble_product_plan&, hipStream_t);
}
