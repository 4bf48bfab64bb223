// Product of 8-bit token rows with 8-bit weight rows, a scale for each token and each output channel:
//   out[m][c] = (sum_j a[m][j] w[c][j]) w_scale[c] a_scale[m] + bias[c], sums exact in int32.
#include "encoder.h"

namespace warp {

namespace {

typedef int int4v __attribute__((ext_vector_type(4)));

struct LinearArgs {
    const int8_t* a;
    int64_t a_stride;
    const float* a_scale;
    int64_t rows;
    const int8_t* w;
    int64_t w_stride;
    const float* w_scale;
    int32_t n, k;  // k: padded to a multiple of kInt8Pad
    const float* bias;
    void* out;
    int64_t out_stride;
};

// Each wave multiplies 32 tokens by 32 channels straight from memory: v_mfma_i32_16x16x64_i8 takes 16 bytes of
// row lane % 16 from each lane, and lane / 16 picks the quarter of 64 columns.
template <typename T>
__global__ __launch_bounds__(256) void k_linear_direct(LinearArgs g) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, q = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * 64 + (wave & 1) * 32;
    const int64_t c0 = (int64_t)blockIdx.y * 64 + (wave >> 1) * 32;
    const int8_t *pa[2], *pw[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + 16 * i + li, c = c0 + 16 * i + li;
        pa[i] = g.a + (m < g.rows ? m : g.rows - 1) * g.a_stride + 16 * q;
        pw[i] = g.w + (c < g.n ? c : g.n - 1) * g.w_stride + 16 * q;
    }
    int4v acc[2][2] = {};
    for (int k = 0; k < g.k; k += 64) {
        int4v va[2], vw[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) va[i] = *(const int4v*)(pa[i] + k), vw[i] = *(const int4v*)(pw[i] + k);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(vw[j], va[i], acc[i][j], 0, 0, 0);
    }
    // lane (li, q) holds channels 4 q .. 4 q + 3 of block j for token li of block i
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + 16 * i + li;
        if (m >= g.rows) continue;
        const float sa = g.a_scale[m];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t c = c0 + 16 * j + 4 * q + r;
                if (c < g.n) {
                    const float b = g.bias ? g.bias[c] : 0.f;
                    ((T*)g.out)[m * g.out_stride + c] = (T)((float)acc[i][j][r] * g.w_scale[c] * sa + b);
                }
            }
    }
}

template <typename T>
void linear(const LinearArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)((g.rows + 63) / 64), (g.n + 63) / 64);
    hipLaunchKernelGGL(k_linear_direct<T>, grid, dim3(256), 0, s, g);
}

}  // namespace

}  // namespace warp

using namespace warp;

extern "C" int warp_linear_int8(const int8_t* a, int64_t a_stride, const float* a_scale, int64_t rows, const int8_t* w,
                                int64_t w_stride, const float* w_scale, int32_t n, int32_t k, const float* bias,
                                void* out, int64_t out_stride, int32_t out_dtype, void* hip_stream) {
    const char* what = "int8 linear";
    if (rows < 0) return fail(WARP_EINVAL, "%s: rows must be >= 0 (got %lld)", what, (long long)rows);
    if (n < 1 || k < 1) return fail(WARP_EINVAL, "%s: n and k must be >= 1 (got %d, %d)", what, n, k);
    if (k > 131071) return fail(WARP_ENOTSUP, "%s: k is at most 131071 (got %d)", what, k);
    if (rows > 1 << 24 || n > 1 << 21)
        return fail(WARP_ENOTSUP, "%s: at most 2^24 rows and 2^21 channels (got %lld, %d)", what, (long long)rows, n);
    if (!dtype_ok(out_dtype)) return fail(WARP_EINVAL, "%s: unknown dtype %d", what, out_dtype);
    if (!w || !w_scale || (rows && (!a || !a_scale || !out))) return fail(WARP_EINVAL, "%s: null pointer", what);
    const int32_t padded = (k + kInt8Pad - 1) / kInt8Pad * kInt8Pad;
    if (a_stride < padded || w_stride < padded || a_stride % 16 || w_stride % 16 || (uintptr_t)a % 16 ||
        (uintptr_t)w % 16)
        return fail(WARP_EINVAL, "%s: int8 rows need 16-byte alignment and strides that are multiples of 16 and at least "
                    "%d (got %lld, %lld)", what, padded, (long long)a_stride, (long long)w_stride);
    if ((uintptr_t)a_scale % 4 || (uintptr_t)w_scale % 4 || (uintptr_t)bias % 4 ||
        (uintptr_t)out % dtype_bytes(out_dtype))
        return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    if (rows > 1 && out_stride < n)
        return fail(WARP_EINVAL, "%s: a row stride of %lld is below %d columns", what, (long long)out_stride, n);
    const int rc = require_device();
    if (rc || !rows) return rc;
    const LinearArgs g{a, a_stride, a_scale, rows, w, w_stride, w_scale, n, padded, bias, out, out_stride};
    hipStream_t s = (hipStream_t)hip_stream;
    if (out_dtype == WARP_F32) WARP_LAUNCH(linear<float>(g, s));
    else if (out_dtype == WARP_F16) WARP_LAUNCH(linear<_Float16>(g, s));
    else WARP_LAUNCH(linear<__bf16>(g, s));
    return WARP_OK;
}
