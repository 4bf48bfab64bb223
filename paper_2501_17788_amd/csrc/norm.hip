// Layer norm of token rows, forward and backward, and rows in 8-bit integers.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), h = (x - mu) r, y = h w + b
//   c = dy w, dx = r (c - mean(c) - h mean(c h)), dw = sum over rows of dy h, db = sum of dy
//   int8: a = max |y|, q = rint(y * fl(127 / a)), scale = a * fl(1 / 127)
//
// Everything is computed in 32 bits; y, dx, dw and db are rounded once, to their own type. A row stays
// in registers between its loads and its stores, so each element is read once and written once, and
// the variance sums squared distances from the finished mean.
#include "encoder.h"

namespace warp {

namespace {

constexpr int kNormal = 0, kNormInt8 = 1, kInt8 = 2;  // what k_rows makes of a row

struct RowArgs {
    const void* x;
    int64_t x_stride, rows;
    int32_t cols;
    const void* weight;  // null: ones
    const void* bias;    // null: zeros
    int32_t params_f32;  // weight and bias are fp32; else of x's type
    float eps;
    void* y;             // kNormal
    int64_t y_stride;
    float* mean;         // null: not wanted
    float* rstd;
    int8_t* q;           // kNormInt8, kInt8
    int64_t q_stride;
    float* scale;
};

// Where a lane's vector j of a row lies. WAVES waves share a row of COLS columns; the row's last
// vector is moved back so that it ends with the row, and its first `skip` elements are left to its
// neighbour: it reads and writes them too (the same values) and leaves them out of sums.
struct Place {
    int at, skip;
    bool in;
};
template <int V, bool RAGGED>
__device__ __forceinline__ Place place(int j, int threads, int t, int cols) {
    const int c = (j * threads + t) * V;
    Place p{c, 0, c < cols};
    if (RAGGED && p.in && c + V > cols) {
        p.at = cols - V;
        p.skip = c - p.at;
    }
    return p;
}

template <typename T, int V>
__device__ __forceinline__ void load_params(const void* p, bool f32, int at, float (&out)[V]) {
    if (f32) {
        const auto v = load_vec<float, V>((const float*)p + at);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = v.e[i];
    } else {
        const auto v = load_vec<T, V>((const T*)p + at);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = (float)v.e[i];
    }
}

// Sum (or largest) over the WAVES waves of a row's workgroup; `part` has a slot for each wave.
template <int WAVES>
__device__ __forceinline__ float row_sum(float x, float* part) {
    x = wave_sum(x);
    if (WAVES == 1) return x;
    __syncthreads();  // the last reduction's slots have been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}
template <int WAVES>
__device__ __forceinline__ uint32_t row_max(uint32_t x, float* part) {
    x = wave_max(x);
    if (WAVES == 1) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = as_f(x);
    __syncthreads();
    uint32_t s = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s = max(s, as_u(part[w]));
    return s;
}

// One row by WAVES waves, NC vectors of V elements in each lane; a workgroup of max(4, WAVES) waves.
template <typename T, int V, int NC, int WAVES, bool RAGGED, int MODE>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void k_rows(RowArgs a) {
    __shared__ float part[WAVES];
    constexpr int kRows = WAVES < 4 ? 4 / WAVES : 1;  // rows of a workgroup
    constexpr int kThreads = WAVES * kWave;           // of a row
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int cols = a.cols;
    const float inv_n = 1.0f / (float)cols;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? threadIdx.x >> 6 : 0); row < a.rows;
         row += (int64_t)gridDim.x * kRows) {
        const T* x = (const T*)a.x + row * a.x_stride;
        float v[NC][V];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, kThreads, t, cols);
            if (p.in) {
                const auto r = load_vec<T, V>(x + p.at);
#pragma unroll
                for (int i = 0; i < V; ++i) v[j][i] = (float)r.e[i];
            }
        }
        if (MODE != kInt8) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                if (p.in) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (!RAGGED || i >= p.skip) s += v[j][i];
                }
            }
            const float mean = row_sum<WAVES>(s, part) * inv_n;
            s = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                if (p.in) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[j][i] -= mean;
                        if (!RAGGED || i >= p.skip) s += v[j][i] * v[j][i];
                    }
                }
            }
            const float rstd = 1.0f / sqrtf(row_sum<WAVES>(s, part) * inv_n + a.eps);
            if (t == 0 && a.mean) {
                a.mean[row] = mean;
                a.rstd[row] = rstd;
            }
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                if (p.in) {
#pragma unroll
                    for (int i = 0; i < V; ++i) v[j][i] *= rstd;
                    float w[V];
                    if (a.weight) {
                        load_params<T, V>(a.weight, a.params_f32, p.at, w);
#pragma unroll
                        for (int i = 0; i < V; ++i) v[j][i] *= w[i];
                    }
                    if (a.bias) {
                        load_params<T, V>(a.bias, a.params_f32, p.at, w);
#pragma unroll
                        for (int i = 0; i < V; ++i) v[j][i] += w[i];
                    }
                }
            }
        }
        if (MODE == kNormal) {
            T* y = (T*)a.y + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                if (p.in) {
                    Vec<T, V> r;
#pragma unroll
                    for (int i = 0; i < V; ++i) r.e[i] = (T)v[j][i];
                    store_vec<T, V>(y + p.at, r);
                }
            }
        } else {
            uint32_t m = 0;
#pragma unroll
            for (int j = 0; j < NC; ++j)
                if (place<V, RAGGED>(j, kThreads, t, cols).in) {
#pragma unroll
                    for (int i = 0; i < V; ++i) m = max(m, as_u(v[j][i]) & 0x7fffffffu);
                }
            const float top = as_f(row_max<WAVES>(m, part));
            // 127 / top is finite for a top of at least 2^-120; a row of smaller numbers is a row of zeros, and one
            // with an infinity or a NaN has zeros too and a scale that is no number, which its products then are
            const bool some = top >= 0x1p-120f && top < INFINITY;
            const float inv = some ? 127.0f / top : 0.f;
            int8_t* q = a.q + row * a.q_stride;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                if (p.in) {
                    Vec<int8_t, V> r;
#pragma unroll
                    for (int i = 0; i < V; ++i) r.e[i] = some ? (int8_t)(int)rintf(v[j][i] * inv) : (int8_t)0;
                    store_vec<int8_t, V>(q + p.at, r);
                }
            }
            const int padded = (cols + kInt8Pad - 1) / kInt8Pad * kInt8Pad;
            for (int c = cols + t; c < padded; c += kThreads) q[c] = 0;
            if (t == 0) a.scale[row] = top < INFINITY ? top * (1.0f / 127.0f) : NAN;
        }
    }
}

struct BackArgs {
    const void* dy;
    int64_t dy_stride;
    const void* x;
    int64_t x_stride, rows;
    int32_t cols;
    const void* weight;
    int32_t params_f32;
    const float* mean;
    const float* rstd;
    void* dx;
    int64_t dx_stride;
    float* parts;  // [gridDim.x][2][cols] sums of dy h and of dy over a workgroup's rows; null: not wanted
};

// dx, and each workgroup's share of dw and db. The weight and both sums of a lane's columns stay in registers
// over all rows of the workgroup; no atomics, so the sums' order is fixed by the sizes alone.
template <typename T, int V, int NC, int WAVES, bool RAGGED>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void k_rows_back(BackArgs a) {
    extern __shared__ float lds[];  // [2][cols] where waves have rows of their own; else [2 * WAVES]
    constexpr int kRows = WAVES < 4 ? 4 / WAVES : 1;
    constexpr int kThreads = WAVES * kWave;
    const int t = WAVES == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int wave = threadIdx.x >> 6;
    const int cols = a.cols;
    const float inv_n = 1.0f / (float)cols;
    float w[NC][V], dw[NC][V], db[NC][V];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const Place p = place<V, RAGGED>(j, kThreads, t, cols);
#pragma unroll
        for (int i = 0; i < V; ++i) w[j][i] = 1.f, dw[j][i] = 0.f, db[j][i] = 0.f;
        if (p.in && a.weight) load_params<T, V>(a.weight, a.params_f32, p.at, w[j]);
    }
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WAVES == 1 ? wave : 0); row < a.rows;
         row += (int64_t)gridDim.x * kRows) {
        const T* x = (const T*)a.x + row * a.x_stride;
        const T* dy = (const T*)a.dy + row * a.dy_stride;
        float h[NC][V], c[NC][V];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, kThreads, t, cols);
            if (p.in) {
                const auto rx = load_vec<T, V>(x + p.at);
                const auto rd = load_vec<T, V>(dy + p.at);
#pragma unroll
                for (int i = 0; i < V; ++i) h[j][i] = (float)rx.e[i], c[j][i] = (float)rd.e[i];
            }
        }
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, kThreads, t, cols);
            if (p.in) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    h[j][i] = (h[j][i] - mean) * rstd;
                    dw[j][i] += c[j][i] * h[j][i];
                    db[j][i] += c[j][i];
                    c[j][i] *= w[j][i];
                    if (!RAGGED || i >= p.skip) s1 += c[j][i], s2 += c[j][i] * h[j][i];
                }
            }
        }
        s1 = wave_sum(s1), s2 = wave_sum(s2);
        if (WAVES > 1) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[2 * wave] = s1, lds[2 * wave + 1] = s2;
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) s1 += lds[2 * k], s2 += lds[2 * k + 1];
        }
        s1 *= inv_n, s2 *= inv_n;
        T* dx = (T*)a.dx + row * a.dx_stride;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, kThreads, t, cols);
            if (p.in) {
                Vec<T, V> r;
#pragma unroll
                for (int i = 0; i < V; ++i) r.e[i] = (T)(rstd * (c[j][i] - s1 - h[j][i] * s2));
                store_vec<T, V>(dx + p.at, r);
            }
        }
    }
    if (!a.parts) return;
    float* out = a.parts + (int64_t)blockIdx.x * 2 * cols;
    if (WAVES == 1) {
        // the four waves' sums one after the other; a moved-back vector leaves its first elements out
        for (int k = 0; k < 4; ++k) {
            if (wave == k) {
#pragma unroll
                for (int j = 0; j < NC; ++j) {
                    const Place p = place<V, RAGGED>(j, kThreads, t, cols);
                    if (p.in) {
#pragma unroll
                        for (int i = 0; i < V; ++i)
                            if (!RAGGED || i >= p.skip) {
                                float& sw = lds[p.at + i];
                                float& sb = lds[cols + p.at + i];
                                sw = k == 0 ? dw[j][i] : sw + dw[j][i];
                                sb = k == 0 ? db[j][i] : sb + db[j][i];
                            }
                    }
                }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * cols; c += 256) out[c] = lds[c];
    } else {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, kThreads, t, cols);
            if (p.in) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    out[p.at + i] = dw[j][i];
                    out[cols + p.at + i] = db[j][i];
                }
            }
        }
    }
}

// dw and db: the workgroups' shares added up. A workgroup takes 64 of the 2 cols sums, 16 threads each.
__global__ __launch_bounds__(1024) void k_join_params(const float* parts, int32_t n_parts, int32_t cols, void* dw,
                                                      void* db, int32_t dtype) {
    __shared__ float lds[16][64];
    const int64_t n = 2 * (int64_t)cols;
    const int64_t c = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63);
    const int slice = threadIdx.x >> 6;
    float s = 0.f;
    if (c < n)
        for (int g = slice; g < n_parts; g += 16) s += parts[g * n + c];
    lds[slice][threadIdx.x & 63] = s;
    __syncthreads();
    if (slice || c >= n) return;
    for (int k = 1; k < 16; ++k) s += lds[k][threadIdx.x];
    void* out = c < cols ? dw : db;
    const int64_t at = c < cols ? c : c - cols;
    if (!out) return;
    if (dtype == WARP_F32) ((float*)out)[at] = s;
    else if (dtype == WARP_F16) ((_Float16*)out)[at] = (_Float16)s;
    else ((__bf16*)out)[at] = (__bf16)s;
}

constexpr int kMaxGrid = 2048;  // workgroups of the forward kernels: eight on each of 256 compute units

template <typename T, int V, int NC, int WAVES, int MODE>
void rows_launch(const RowArgs& a, hipStream_t s) {
    constexpr int kRows = WAVES < 4 ? 4 / WAVES : 1;
    const int64_t need = (a.rows + kRows - 1) / kRows;
    const dim3 grid((uint32_t)(need < kMaxGrid ? need : kMaxGrid)), block(WAVES < 4 ? 256 : WAVES * 64);
    if (a.cols % V) hipLaunchKernelGGL((k_rows<T, V, NC, WAVES, true, MODE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_rows<T, V, NC, WAVES, false, MODE>), grid, block, 0, s, a);
}

template <typename T, int MODE>
void rows_of(const RowArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int lane = (a.cols + kWave * V - 1) / (kWave * V);  // vectors a lane of one wave would hold
    if (a.cols < V) rows_launch<T, 1, 1, 1, MODE>(a, s);
    else if (lane <= 1) rows_launch<T, V, 1, 1, MODE>(a, s);
    else if (lane <= 2) rows_launch<T, V, 2, 1, MODE>(a, s);
    else if (lane <= 4) rows_launch<T, V, 4, 1, MODE>(a, s);
    else if (lane <= 8) rows_launch<T, V, 2, 4, MODE>(a, s);
    else if (lane <= 16) rows_launch<T, V, 4, 4, MODE>(a, s);
    else if (lane <= 32) rows_launch<T, V, 8, 4, MODE>(a, s);
    else rows_launch<float, 4, 4, 16, MODE>(a, s);  // only fp32 rows: kMaxCols is 32 vectors of 16-bit elements
}

template <int MODE>
void rows_any(int32_t dtype, const RowArgs& a, hipStream_t s) {
    if (dtype == WARP_F32) rows_of<float, MODE>(a, s);
    else if (dtype == WARP_F16) rows_of<_Float16, MODE>(a, s);
    else rows_of<__bf16, MODE>(a, s);
}

constexpr int kMaxCols = 16384;  // 16 waves of 64 lanes of 16 elements

int back_waves(int32_t cols) {
    const int per = kWave * 32;  // columns of a wave: 32 of each of five arrays in a lane's registers; 16 of 16 waves'
    return cols <= per ? 1 : cols <= 4 * per ? 4 : 16;
}

int back_grid(int64_t rows, int32_t cols) {
    const int waves = back_waves(cols);
    const int64_t need = waves == 1 ? (rows + 3) / 4 : rows;
    const int64_t most = waves == 16 ? 256 : 512;
    return (int)(need < most ? need : most);
}

template <typename T, int V, int NC, int WAVES>
void back_launch(const BackArgs& a, int grid, hipStream_t s) {
    const size_t lds = WAVES == 1 ? 2 * sizeof(float) * a.cols : 2 * sizeof(float) * WAVES;
    const dim3 block(WAVES < 4 ? 256 : WAVES * 64);
    if (a.cols % V) hipLaunchKernelGGL((k_rows_back<T, V, NC, WAVES, true>), dim3(grid), block, lds, s, a);
    else hipLaunchKernelGGL((k_rows_back<T, V, NC, WAVES, false>), dim3(grid), block, lds, s, a);
}

template <typename T>
void back_of(const BackArgs& a, int grid, int waves, hipStream_t s) {
    constexpr int V = 16 / sizeof(T), N = 32 / V;
    const int lane = (a.cols + kWave * V - 1) / (kWave * V);
    if (a.cols < V) back_launch<T, 1, 1, 1>(a, grid, s);
    else if (lane <= N / 4) back_launch<T, V, N / 4, 1>(a, grid, s);
    else if (lane <= N / 2) back_launch<T, V, N / 2, 1>(a, grid, s);
    else if (waves == 1) back_launch<T, V, N, 1>(a, grid, s);
    else if (waves == 4) back_launch<T, V, N, 4>(a, grid, s);
    else back_launch<T, V, N / 2, 16>(a, grid, s);
}

int check_rows(const char* what, const void* x, int64_t stride, int64_t rows, int32_t cols, int32_t dtype) {
    if (rows < 0) return fail(WARP_EINVAL, "%s: rows must be >= 0 (got %lld)", what, (long long)rows);
    if (cols < 1) return fail(WARP_EINVAL, "%s: cols must be >= 1 (got %d)", what, cols);
    if (cols > kMaxCols) return fail(WARP_ENOTSUP, "%s: at most %d columns (got %d)", what, kMaxCols, cols);
    if (!dtype_ok(dtype)) return fail(WARP_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (rows > INT32_MAX) return fail(WARP_ENOTSUP, "%s: at most 2^31-1 rows (got %lld)", what, (long long)rows);
    if (rows && !x) return fail(WARP_EINVAL, "%s: null pointer", what);
    if (rows > 1 && stride < cols)
        return fail(WARP_EINVAL, "%s: a row stride of %lld is below %d columns", what, (long long)stride, cols);
    if ((uintptr_t)x % dtype_bytes(dtype)) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    return WARP_OK;
}

int check_params(const char* what, const void* w, const void* b, int32_t dtype, int32_t param_dtype) {
    if (param_dtype != WARP_F32 && param_dtype != dtype)
        return fail(WARP_EINVAL, "%s: weight and bias are fp32 or of x's dtype (got dtype %d for %d)", what, param_dtype,
                    dtype);
    const int bytes = dtype_bytes(param_dtype);
    if ((uintptr_t)w % bytes || (uintptr_t)b % bytes) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    return WARP_OK;
}

int check_int8_rows(const char* what, int64_t rows, int32_t cols, const int8_t* q, int64_t q_stride,
                    const float* scale) {
    const int64_t padded = ((int64_t)cols + kInt8Pad - 1) / kInt8Pad * kInt8Pad;
    if (rows && (!q || !scale)) return fail(WARP_EINVAL, "%s: null pointer", what);
    if (q_stride < padded || q_stride % 16 || (uintptr_t)q % 16 || (uintptr_t)scale % 4)
        return fail(WARP_EINVAL, "%s: int8 rows need 16-byte alignment and a stride that is a multiple of 16 and at "
                    "least %lld (got %lld)", what, (long long)padded, (long long)q_stride);
    return WARP_OK;
}

}  // namespace

}  // namespace warp

using namespace warp;

extern "C" {

int warp_layer_norm(const void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t dtype, const void* weight,
                    const void* bias, int32_t param_dtype, float eps, void* y, int64_t y_stride, float* mean,
                    float* rstd, void* hip_stream) {
    const char* what = "layer norm";
    int rc = check_rows(what, x, x_stride, rows, cols, dtype);
    if (!rc) rc = check_rows(what, y, y_stride, rows, cols, dtype);
    if (!rc) rc = check_params(what, weight, bias, dtype, param_dtype);
    if (rc) return rc;
    if (!(eps >= 0.f)) return fail(WARP_EINVAL, "%s: eps must be >= 0", what);
    if (!mean != !rstd) return fail(WARP_EINVAL, "%s: mean and rstd come together", what);
    rc = require_device();
    if (rc || !rows) return rc;
    RowArgs a{x, x_stride, rows, cols, weight, bias, param_dtype == WARP_F32, eps, y, y_stride, mean, rstd, nullptr, 0,
              nullptr};
    WARP_LAUNCH(rows_any<kNormal>(dtype, a, (hipStream_t)hip_stream));
    return WARP_OK;
}

int warp_layer_norm_int8(const void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t dtype,
                         const void* weight, const void* bias, int32_t param_dtype, float eps, int8_t* q,
                         int64_t q_stride, float* scale, void* hip_stream) {
    const char* what = "layer norm to int8";
    int rc = check_rows(what, x, x_stride, rows, cols, dtype);
    if (!rc) rc = check_params(what, weight, bias, dtype, param_dtype);
    if (!rc) rc = check_int8_rows(what, rows, cols, q, q_stride, scale);
    if (rc) return rc;
    if (!(eps >= 0.f)) return fail(WARP_EINVAL, "%s: eps must be >= 0", what);
    rc = require_device();
    if (rc || !rows) return rc;
    RowArgs a{x, x_stride, rows, cols, weight, bias, param_dtype == WARP_F32, eps, nullptr, 0, nullptr, nullptr, q,
              q_stride, scale};
    WARP_LAUNCH(rows_any<kNormInt8>(dtype, a, (hipStream_t)hip_stream));
    return WARP_OK;
}

int warp_quantize_rows(const void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t dtype, int8_t* q,
                       int64_t q_stride, float* scale, void* hip_stream) {
    const char* what = "rows to int8";
    int rc = check_rows(what, x, x_stride, rows, cols, dtype);
    if (!rc) rc = check_int8_rows(what, rows, cols, q, q_stride, scale);
    if (!rc) rc = require_device();
    if (rc || !rows) return rc;
    RowArgs a{x, x_stride, rows, cols, nullptr, nullptr, 1, 0.f, nullptr, 0, nullptr, nullptr, q, q_stride, scale};
    WARP_LAUNCH(rows_any<kInt8>(dtype, a, (hipStream_t)hip_stream));
    return WARP_OK;
}

int warp_layer_norm_backward_scratch(int64_t rows, int32_t cols, int64_t* bytes) {
    if (!bytes || rows < 0 || cols < 1)
        return fail(WARP_EINVAL, "layer norm backward: bad sizes");
    *bytes = (int64_t)back_grid(rows, cols) * 2 * cols * (int64_t)sizeof(float);
    return WARP_OK;
}

int warp_layer_norm_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int64_t rows,
                             int32_t cols, int32_t dtype, const void* weight, int32_t param_dtype, const float* mean,
                             const float* rstd, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                             void* scratch, int64_t scratch_bytes, void* hip_stream) {
    const char* what = "layer norm backward";
    int rc = check_rows(what, dy, dy_stride, rows, cols, dtype);
    if (!rc) rc = check_rows(what, x, x_stride, rows, cols, dtype);
    if (!rc) rc = check_rows(what, dx, dx_stride, rows, cols, dtype);
    if (!rc) rc = check_params(what, weight, nullptr, dtype, param_dtype);
    if (!rc) rc = check_params(what, dweight, dbias, dtype, param_dtype);
    if (rc) return rc;
    if (rows && (!mean || !rstd)) return fail(WARP_EINVAL, "%s: null pointer", what);
    const bool sums = dweight || dbias;
    const int grid = back_grid(rows, cols);
    const int64_t need = (int64_t)grid * 2 * cols * (int64_t)sizeof(float);
    if (sums && need && (!scratch || scratch_bytes < need || (uintptr_t)scratch % 4))
        return fail(WARP_EINVAL, "%s: needs %lld bytes of scratch (got %lld)", what, (long long)need,
                    (long long)(scratch ? scratch_bytes : 0));
    rc = require_device();
    if (rc) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    BackArgs a{dy, dy_stride, x, x_stride, rows, cols, weight, param_dtype == WARP_F32, mean, rstd, dx, dx_stride,
               sums ? (float*)scratch : nullptr};
    const int waves = back_waves(cols);
    if (rows) {
        if (dtype == WARP_F32) WARP_LAUNCH(back_of<float>(a, grid, waves, s));
        else if (dtype == WARP_F16) WARP_LAUNCH(back_of<_Float16>(a, grid, waves, s));
        else WARP_LAUNCH(back_of<__bf16>(a, grid, waves, s));
    }
    if (sums)  // without rows: zeros
        WARP_LAUNCH(hipLaunchKernelGGL(k_join_params, dim3((2 * cols + 63) / 64), dim3(1024), 0, s,
                                       (const float*)scratch, rows ? grid : 0, cols, dweight, dbias, param_dtype));
    return WARP_OK;
}

}  // extern "C"
