// Logits of tokens over a vocabulary, never written: their statistics, or the loss's gradient for them.
#include "product.h"

namespace warp {

hipError_t product_softmax(const ProductArgs& g, int element, bool planes, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F32)
        return finish == kStats ? product_tiles<float, kAlongK, kAlongK, kStats>(g, tile, s)
                                : product_tiles<float, kAlongK, kAlongK, kGrad>(g, tile, s);
    if (finish == kStats)
        return element == WARP_F16 ? product_tiles<_Float16, kAlongK, kAlongK, kStats>(g, tile, s)
                                   : product_tiles<__bf16, kAlongK, kAlongK, kStats>(g, tile, s);
    if (planes) return product_tiles<__bf16, kAlongK, kAlongK, kGrad, kPlanes>(g, tile, s);
    return element == WARP_F16 ? product_tiles<_Float16, kAlongK, kAlongK, kGrad>(g, tile, s)
                               : product_tiles<__bf16, kAlongK, kAlongK, kGrad>(g, tile, s);
}

}  // namespace warp
