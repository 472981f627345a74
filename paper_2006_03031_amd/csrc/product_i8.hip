// Dense in 8 bits.
#include "product_launch.h"

namespace nimble {
template int launch_product<OfInt8, 0>(const ProductArgs&, const nimble_product_plan&, hipStream_t);
}
