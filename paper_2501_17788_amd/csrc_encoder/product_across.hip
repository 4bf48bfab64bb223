// Products whose operands lie across K both (gradients by tokens: a weight's gradient).
#include "product.h"

namespace warp {

hipError_t product_across(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    return product_any<kAcrossK, kAcrossK>(g, element, tile, finish, s);
}

}  // namespace warp
