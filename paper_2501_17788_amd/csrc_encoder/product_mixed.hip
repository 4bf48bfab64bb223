// Products whose operands lie along K and across K (gradients by a weight).
#include "product.h"

namespace warp {

hipError_t product_mixed(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F32)
        return finish == kSum ? product_tiles<float, kAlongK, kAcrossK, kSum>(g, tile, s)
                              : product_tiles<float, kAlongK, kAcrossK, kStore>(g, tile, s);
    return product_any<kAlongK, kAcrossK>(g, element, tile, finish, s);
}

}  // namespace warp
