// Products whose operands lie across K both (gradients by tokens: a weight's gradient).
#include "product.h"

namespace warp {

hipError_t product_across(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F32)
        return finish == kSum ? product_tiles<float, kAcrossK, kAcrossK, kSum>(g, tile, s)
                              : product_tiles<float, kAcrossK, kAcrossK, kStore>(g, tile, s);
    return product_any<kAcrossK, kAcrossK>(g, element, tile, finish, s);
}

hipError_t product_bytes(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F16)
        return finish == kSum ? product_tiles<_Float16, kAcrossK, kAcrossK, kSum, kBytes>(g, tile, s)
                              : product_tiles<_Float16, kAcrossK, kAcrossK, kStore, kBytes>(g, tile, s);
    return finish == kSum ? product_tiles<__bf16, kAcrossK, kAcrossK, kSum, kBytes>(g, tile, s)
                          : product_tiles<__bf16, kAcrossK, kAcrossK, kStore, kBytes>(g, tile, s);
}

}  // namespace warp
