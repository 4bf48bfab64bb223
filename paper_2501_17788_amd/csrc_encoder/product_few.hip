// Products of few rows (a token, a query) by a weight: the weight's bytes and the launch are what counts.
#include "operands.h"

namespace warp {

namespace {

// A workgroup makes 16 columns of all rows (16 BM at most): its eight waves share the k range, 32 at a time and four such
// steps under way, straight from memory, and their sums meet in LDS in a fixed order. 1 x 1024 by 1024 takes 3.7 us, little
// more than an empty launch; tiles of 64 x 64 with the k range in parts took 8.3 with the launch that joined them.
constexpr int kFewWaves = 8;
template <typename E, int BM>
__global__ __launch_bounds__(64 * kFewWaves) void k_product_few(ProductArgs g) {
    typedef typename Eight<E>::type V;
    __shared__ float sums[kFewWaves][16 * BM][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, q = lane >> 4;
    const int64_t c0 = (int64_t)blockIdx.x * 16;
    const int rows = (int)g.m;
    const E* pb = (const E*)g.b + (c0 + li < g.n ? c0 + li : g.n - 1) * g.b_stride;
    const E* pa[BM];
#pragma unroll
    for (int i = 0; i < BM; ++i) pa[i] = (const E*)g.a + (int64_t)(16 * i + li < rows ? 16 * i + li : rows - 1) * g.a_stride;
    float4v acc[BM] = {};
    const int64_t by = 32 * kFewWaves;
    constexpr int U = 4;
    for (int64_t k = 32 * wave; k < g.k; k += U * by) {
        V a[U][BM], b[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t at = k + u * by + 8 * q;
            const bool in = at < g.k;  // pieces of 8: zeros beyond the range
            b[u] = V{};
            if (in) b[u] = *(const V*)(pb + at);
#pragma unroll
            for (int i = 0; i < BM; ++i) {
                a[u][i] = V{};
                if (in) a[u][i] = *(const V*)(pa[i] + at);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < BM; ++i) acc[i] = product_mfma(b[u], a[u][i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][16 * i + li][4 * q + e] = acc[i][e];
    __syncthreads();
    for (int t = threadIdx.x; t < 256 * BM; t += 64 * kFewWaves) {
        const int row = t >> 4, col = t & 15;
        if (row >= rows || c0 + col >= g.n) continue;
        float v[1] = {0.f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) v[0] += sums[w][row][col];
        if (g.bias) v[0] += load_float(g.bias, g.bias_type, c0 + col);
        store_floats<1>(g.out, g.out_type, row * g.out_stride + c0 + col, v, 1, false);
    }
}

template <typename E>
void few(const ProductArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)cover_of(g.n, 16)), block(64 * kFewWaves);
    if (g.m <= 16) hipLaunchKernelGGL((k_product_few<E, 1>), grid, block, 0, s, g);
    else hipLaunchKernelGGL((k_product_few<E, 2>), grid, block, 0, s, g);
}

}  // namespace

hipError_t product_few(const ProductArgs& g, int element, hipStream_t s) {
    (void)hipGetLastError();
    if (element == WARP_F16) few<_Float16>(g, s);
    else few<__bf16>(g, s);
    return hipGetLastError();
}

}  // namespace warp
