// Products whose operands lie along K both (tokens by a weight's rows).
#include "product.h"

namespace warp {

hipError_t product_along(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F32)
        return finish == kSum ? product_tiles<float, kAlongK, kAlongK, kSum>(g, tile, s)
                              : product_tiles<float, kAlongK, kAlongK, kStore>(g, tile, s);
    return product_any<kAlongK, kAlongK>(g, element, tile, finish, s);
}

}  // namespace warp
