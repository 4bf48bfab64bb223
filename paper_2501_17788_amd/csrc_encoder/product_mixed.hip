// Products whose operands lie along K and across K (gradients by a weight).
#include "product.h"

namespace warp {

hipError_t product_mixed(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    return product_any<kAlongK, kAcrossK>(g, element, tile, finish, s);
}

}  // namespace warp
