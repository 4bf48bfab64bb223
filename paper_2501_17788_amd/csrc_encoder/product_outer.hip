// float32 products over few k (a weight's or a table's gradient by few rows): what is written is what counts.
#include "operands.h"

namespace warp {

namespace {

// A lane makes four neighbouring columns of 16 rows, a workgroup 256 columns of 64 rows, eight k at a time: B's come from memory,
// A's from LDS, one number for all lanes. 4096 x 4096 over 1, 16 and 32 k takes 15, 21 and 29 us (4.5 to 2.3 TB/s written, with 32 as
// much work for the vector units); tiles of the matrix cores, whose steps of 64 k are mostly zeros in six products of planes, 95.
constexpr int kOuterRows = 64, kOuterStep = 8;
template <bool PLANES>
__global__ __launch_bounds__(256) void k_product_outer(OuterArgs g) {
    __shared__ __attribute__((aligned(16))) float a[kOuter][kOuterRows];
    const int lane = threadIdx.x & 63, r = threadIdx.x / 64 * 16;
    const int64_t m0 = (int64_t)blockIdx.y * kOuterRows, c = ((int64_t)blockIdx.x * kWave + lane) * 4;
    const int k = (int)(g.k_now ? *g.k_now : g.k), steps = (k + kOuterStep - 1) / kOuterStep;
    for (int i = threadIdx.x; i < steps * kOuterStep * kOuterRows; i += 256) {
        const int at = i / kOuterRows;
        const int64_t m = m0 + i % kOuterRows;
        float x = 0.f;
        if (at < k && m < g.m) {
            if constexpr (PLANES) {
                const uint16_t* p = (const uint16_t*)g.a + at * g.a_stride + m;
                x = as_f((uint32_t)p[2 * g.a_plane] << 16) + as_f((uint32_t)p[g.a_plane] << 16) + as_f((uint32_t)p[0] << 16);
            } else {
                x = ((const float*)g.a)[at * g.a_stride + m];
            }
        }
        a[at][i % kOuterRows] = x;
    }
    const float factor = g.factor ? *g.factor : 1.f;
    __syncthreads();
    if (g.sums && blockIdx.x == 0 && threadIdx.x < kOuterRows && m0 + threadIdx.x < g.m) {
        float sum = 0.f;
        for (int at = 0; at < k; ++at) sum += a[at][threadIdx.x];
        g.sums[m0 + threadIdx.x] = sum;
    }
    if (c >= g.n || m0 + r >= g.m) return;
    float4v acc[16] = {};
#pragma unroll 1
    for (int k0 = 0; k0 < k; k0 += kOuterStep) {
        float4v b[kOuterStep];
#pragma unroll
        for (int i = 0; i < kOuterStep; ++i) {
            const int64_t at = k0 + i;
            b[i] = float4v{};
            if (at >= k) continue;
            if constexpr (PLANES) {  // rows are padded to 64 columns, those of 8 bits to 128
                Vec<uint16_t, 4> x[3];
#pragma unroll
                for (int p = 0; p < 3; ++p) x[p] = load_vec<uint16_t, 4>((const uint16_t*)g.b + p * g.b_plane + at * g.b_stride + c);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    b[i][e] = as_f((uint32_t)x[2].e[e] << 16) + as_f((uint32_t)x[1].e[e] << 16) + as_f((uint32_t)x[0].e[e] << 16);
            } else {
                const auto x = load_vec<int8_t, 4>((const int8_t*)g.b + at * g.b_stride + c);
                const float scale = g.b_scale[at];
#pragma unroll
                for (int e = 0; e < 4; ++e) b[i][e] = (float)x.e[e] * scale;
            }
        }
#pragma unroll
        for (int i = 0; i < kOuterStep; ++i)
#pragma unroll
            for (int t = 0; t < 16; t += 4) {
                const float4v x = *(const float4v*)&a[k0 + i][r + t];
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[t + u] += x[u] * b[i];
            }
    }
#pragma unroll
    for (int t = 0; t < 16; ++t) {
        if (m0 + r + t >= g.m) return;
        const float v[4] = {acc[t][0] * factor, acc[t][1] * factor, acc[t][2] * factor, acc[t][3] * factor};
        store_floats<4>(g.out, WARP_F32, (m0 + r + t) * g.out_stride + c, v, g.n - c, true);
    }
}

}  // namespace

hipError_t product_outer(const OuterArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)cover_of(g.n, 256), (uint32_t)cover_of(g.m, kOuterRows)), block(256);
    (void)hipGetLastError();
    if (g.b_scale) hipLaunchKernelGGL(k_product_outer<false>, grid, block, 0, s, g);
    else hipLaunchKernelGGL(k_product_outer<true>, grid, block, 0, s, g);
    return hipGetLastError();
}

}  // namespace warp
