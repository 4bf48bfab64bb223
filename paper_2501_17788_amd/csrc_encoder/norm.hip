// Layer norm of token rows, forward and backward, and rows in 8-bit integers.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), h = (x - mu) r, y = h w + b
//   c = dy w, dx = r (c - mean(c) - h mean(c h)), dw = sum over rows of dy h, db = sum of dy
//   int8: a = max |y|, q = rint(y * fl(127 / a)), scale = a * fl(1 / 127)
//
// Everything is computed in 32 bits; y, dx, dw and db are rounded once, to their own type. A row stays
// in registers between its loads and its stores, so each element is read once and written once, and
// the variance sums squared distances from the finished mean. Bound by memory; a large copy moves 5.1 to 5.6 TB/s.
// Called again and again on the same tensors, 131,072 rows of 1,024 bfloat16 take 85 us forward (6.3 TB/s) and 133 us
// backward with the sums (6.1 TB/s), 100,000 of 128 10 and 19 us. One after the other, their inputs not in the caches,
// the first size takes 101, 150 and, for the join of the sums, 5 us (5.3 TB/s; medians). 65,536 of 1,024 to int8 38 us
// (5.3 TB/s); 32 of 768 3.2 us forward.
#include "encoder.h"

namespace warp {

namespace {

constexpr int kNormal = 0, kNormInt8 = 1, kInt8 = 2;  // what k_rows makes of a row

// N words at any address
template <int N>
struct __attribute__((packed, aligned(1))) Words {
    uint32_t e[N];
};
template <>
struct Words<0> {
    uint32_t e[1];
};

// Whether a kernel's inputs pass the caches by: where all that it reads and writes exceeds the 256 MB of the last
// cache, inputs kept there only displace outputs. 131,072 rows of 1,024 bfloat16: forward 104 us without, 88 us with,
// backward 160 and 135 us; 30,000 of 2,048: backward 76 and 67 us, forward (245 MB) 41.8 and 42.2 us; 20,000 of 1,024:
// forward 14.6 and 17.2 us.
bool passes_by(int64_t rows, int32_t cols, int element_bytes) {
    return rows * cols * element_bytes > (int64_t)256 << 20;
}

struct RowArgs {
    const void* x;
    int64_t x_stride, rows;
    int32_t cols;
    const void* weight;  // null: ones
    const void* bias;    // null: zeros
    int32_t params_f32;  // weight and bias are fp32; else of x's type
    float eps;
    int32_t stream;      // x passes the caches by
    void* y;             // kNormal
    int64_t y_stride;
    float* mean;         // null: not wanted
    float* rstd;
    int8_t* q;           // kNormInt8, kInt8
    int64_t q_stride;
    float* scale;
};

// Where a lane's vector j of a row lies, of the `threads` lanes that share the row. The row's last
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

// Sum (or largest) over the LANES lanes of a row: a quarter of a wave, a wave, or a workgroup of several, whose `part`
// has a slot for each.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float* part) {
    if (LANES == 16) return quarter_sum(x);
    x = wave_sum(x);
    if (LANES == kWave) return x;
    __syncthreads();  // the last reduction's slots have been read
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / kWave; ++w) s += part[w];
    return s;
}
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t x, float* part) {
    if (LANES == 16) return quarter_max(x);
    x = wave_max(x);
    if (LANES == kWave) return x;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = as_f(x);
    __syncthreads();
    uint32_t s = 0;
#pragma unroll
    for (int w = 0; w < LANES / kWave; ++w) s = max(s, as_u(part[w]));
    return s;
}

// q = rint(v * inv) of four elements as the bytes of a word: adding 1.5 * 2^23 to the rounded product rounds it to
// the nearest even integer, whose two's complement is then in the sum's low bits.
__device__ __forceinline__ uint32_t four_bytes(const float* v, float inv) {
#pragma clang fp contract(off)
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = as_u(v[i] * inv + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u);
    return __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu) | lo;
}

// Rows by LANES lanes, NC vectors of V elements in each; a workgroup of 256 lanes or LANES, if more. A workgroup goes
// through several rows where there are many: the next row is loaded while one is worked on, and up to 32 columns a
// lane their weights and biases stay in registers (65,536 rows of 1,024 to int8: 71 us without both, 38 us with). Rows
// of at most 32 vectors take 16 lanes each (100,000 of 128 bfloat16: 23 us by whole waves, 10 us).
template <typename T, int V, int NC, int LANES, bool RAGGED, int MODE>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rows(RowArgs a) {
    __shared__ float part[16];
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;  // rows of a workgroup
    constexpr bool kKeep = NC * V <= 32 && MODE != kInt8;
    const int t = threadIdx.x % LANES;
    const int cols = a.cols;
    const float inv_n = 1.0f / (float)cols;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    Vec<T, V> next[NC];
    auto load = [&](int64_t r) {
        const T* x = (const T*)a.x + r * a.x_stride;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, LANES, t, cols);
            if (p.in) next[j] = a.stream ? stream_in<T, V>(x + p.at) : load_vec<T, V>(x + p.at);
        }
    };
    if (row < a.rows) load(row);
    float w[kKeep ? NC : 1][V], b[kKeep ? NC : 1][V];
    auto params = [&](int j, int k, const Place& p) {  // of vector j, into w[k] and b[k]
#pragma unroll
        for (int i = 0; i < V; ++i) w[k][i] = 1.f, b[k][i] = 0.f;
        if (p.in && a.weight) load_params<T, V>(a.weight, a.params_f32, p.at, w[k]);
        if (p.in && a.bias) load_params<T, V>(a.bias, a.params_f32, p.at, b[k]);
    };
    if (kKeep) {
#pragma unroll
        for (int j = 0; j < NC; ++j) params(j, j, place<V, RAGGED>(j, LANES, t, cols));
    }
    for (; row < a.rows; row += step) {
        float v[NC][V];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) v[j][i] = (float)next[j].e[i];
        if (row + step < a.rows) load(row + step);
        if (MODE != kInt8) {
            float s = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, LANES, t, cols);
                if (p.in) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
                        if (!RAGGED || i >= p.skip) s += v[j][i];
                }
            }
            const float mean = row_sum<LANES>(s, part) * inv_n;
            s = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, LANES, t, cols);
                if (p.in) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        v[j][i] -= mean;
                        if (!RAGGED || i >= p.skip) s += v[j][i] * v[j][i];
                    }
                }
            }
            const float rstd = 1.0f / sqrtf(row_sum<LANES>(s, part) * inv_n + a.eps);
            if (t == 0 && a.mean) {
                a.mean[row] = mean;
                a.rstd[row] = rstd;
            }
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int k = kKeep ? j : 0;
                if (!kKeep) params(j, k, place<V, RAGGED>(j, LANES, t, cols));
#pragma unroll
                for (int i = 0; i < V; ++i) v[j][i] = v[j][i] * rstd * w[k][i] + b[k][i];
            }
        }
        if (MODE == kNormal) {
            T* y = (T*)a.y + row * a.y_stride;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, LANES, t, cols);
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
                if (place<V, RAGGED>(j, LANES, t, cols).in) {
#pragma unroll
                    for (int i = 0; i < V; ++i) m = max(m, as_u(v[j][i]) & 0x7fffffffu);
                }
            const float top = as_f(row_max<LANES>(m, part));
            // 127 / top is finite for a top of at least 2^-120; a row of smaller numbers is a row of zeros, and one
            // with an infinity or a NaN has zeros too and a scale that is no number, which its products then are
            const bool some = top >= 0x1p-120f && top < INFINITY;
            const float inv = some ? 127.0f / top : 0.f;
            const uint32_t keep = some ? ~0u : 0u;
            int8_t* q = a.q + row * a.q_stride;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const Place p = place<V, RAGGED>(j, LANES, t, cols);
                if (p.in) {
                    if (V == 1) {
                        q[p.at] = some ? (int8_t)(int)rintf(v[j][0] * inv) : (int8_t)0;
                    } else {
                        Words<V / 4> r;
#pragma unroll
                        for (int i = 0; i < V / 4; ++i) r.e[i] = four_bytes(v[j] + 4 * i, inv) & keep;
                        *reinterpret_cast<Words<V / 4>*>(q + p.at) = r;
                    }
                }
            }
            const int padded = (cols + kInt8Pad - 1) / kInt8Pad * kInt8Pad;
            for (int c = cols + t; c < padded; c += LANES) q[c] = 0;
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
    int32_t stream;  // x and dy pass the caches by
    float* parts;    // [gridDim.x][2][cols] sums of dy h and of dy over a workgroup's rows; null: not wanted
};

// dx, and each workgroup's share of dw and db. The weight and both sums of a lane's columns stay in registers
// over all rows of the workgroup; no atomics, so the sums' order is fixed by the sizes alone. With the next row's loads
// under way and four waves on each SIMD instead of two, 131,072 rows of 1,024 went from 240 to 150 us.
template <typename T, int V, int NC, int LANES, bool RAGGED>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void k_rows_back(BackArgs a) {
    // two waves' sums of their columns where waves have rows of their own; else two sums of each wave
    __shared__ float lds[LANES <= kWave ? 2 * 2 * NC * V * kWave : 2 * 16];
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
    const int t = threadIdx.x % LANES;
    const int wave = threadIdx.x >> 6;
    const int cols = a.cols;
    const float inv_n = 1.0f / (float)cols;
    float w[NC][V], dw[NC][V], db[NC][V];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const Place p = place<V, RAGGED>(j, LANES, t, cols);
#pragma unroll
        for (int i = 0; i < V; ++i) w[j][i] = 1.f, dw[j][i] = 0.f, db[j][i] = 0.f;
        if (p.in && a.weight) load_params<T, V>(a.weight, a.params_f32, p.at, w[j]);
    }
    const int64_t step = (int64_t)gridDim.x * kRows;
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    Vec<T, V> next_x[NC], next_dy[NC];
    float next_mean = 0.f, next_rstd = 0.f;
    auto load = [&](int64_t r) {
        const T* x = (const T*)a.x + r * a.x_stride;
        const T* dy = (const T*)a.dy + r * a.dy_stride;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, LANES, t, cols);
            if (p.in) {
                next_x[j] = a.stream ? stream_in<T, V>(x + p.at) : load_vec<T, V>(x + p.at);
                next_dy[j] = a.stream ? stream_in<T, V>(dy + p.at) : load_vec<T, V>(dy + p.at);
            }
        }
        next_mean = a.mean[r], next_rstd = a.rstd[r];
    };
    if (row < a.rows) load(row);
    for (; row < a.rows; row += step) {
        float h[NC][V], c[NC][V];
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) h[j][i] = (float)next_x[j].e[i], c[j][i] = (float)next_dy[j].e[i];
        const float mean = next_mean, rstd = next_rstd;
        if (row + step < a.rows) load(row + step);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, LANES, t, cols);
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
        if (LANES == 16) s1 = quarter_sum(s1), s2 = quarter_sum(s2);
        else s1 = wave_sum(s1), s2 = wave_sum(s2);
        if (LANES > kWave) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0) lds[2 * wave] = s1, lds[2 * wave + 1] = s2;
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int k = 0; k < LANES / kWave; ++k) s1 += lds[2 * k], s2 += lds[2 * k + 1];
        }
        s1 *= inv_n, s2 *= inv_n;
        T* dx = (T*)a.dx + row * a.dx_stride;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const Place p = place<V, RAGGED>(j, LANES, t, cols);
            if (p.in) {
                Vec<T, V> r;
#pragma unroll
                for (int i = 0; i < V; ++i) r.e[i] = (T)(rstd * (c[j][i] - s1 - h[j][i] * s2));
                store_vec<T, V>(dx + p.at, r);
            }
        }
    }
    if (!a.parts) return;
    if (LANES == 16) {  // the sums of a wave's four rows meet in each of them
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int k = 16; k < kWave; k <<= 1) {
                    dw[j][i] += __shfl_xor(dw[j][i], k);
                    db[j][i] += __shfl_xor(db[j][i], k);
                }
    }
    if (LANES <= kWave) {
        // the four waves' sums meet in the first: two and two, then one and one
        constexpr int kHeld = 2 * NC * V;
#pragma unroll
        for (int half = 2; half; half >>= 1) {
            float* slot = lds + (wave & (half - 1)) * kHeld * kWave + (threadIdx.x & 63);
            __syncthreads();
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        slot[(2 * (j * V + i)) * kWave] = dw[j][i];
                        slot[(2 * (j * V + i) + 1) * kWave] = db[j][i];
                    }
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        dw[j][i] += slot[(2 * (j * V + i)) * kWave];
                        db[j][i] += slot[(2 * (j * V + i) + 1) * kWave];
                    }
            }
        }
        if (threadIdx.x >= LANES) return;
    }
    float* out = a.parts + (int64_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const Place p = place<V, RAGGED>(j, LANES, t, cols);
        if (p.in) {
            Vec<float, V> rw, rb;
#pragma unroll
            for (int i = 0; i < V; ++i) rw.e[i] = dw[j][i], rb.e[i] = db[j][i];
            store_vec<float, V>(out + p.at, rw);
            store_vec<float, V>(out + cols + p.at, rb);
        }
    }
}

constexpr int kMaxParts = 1024;  // workgroups of the backward kernel: 32 shares for each of 32 threads below

// dw and db: the workgroups' shares added up. A workgroup takes 32 of the 2 cols sums, 32 threads each.
__global__ __launch_bounds__(1024) void k_join_params(const float* parts, int32_t n_parts, int32_t cols, void* dw,
                                                      void* db, int32_t dtype) {
    __shared__ float lds[32][33];
    const int64_t n = 2 * (int64_t)cols;
    const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < n) {
        float v[32];  // all loads at once: the shares come from other XCDs' memory
#pragma unroll
        for (int k = 0; k < 32; ++k) v[k] = slice + 32 * k < n_parts ? parts[(slice + 32 * k) * n + c] : 0.f;
#pragma unroll
        for (int k = 0; k < 32; ++k) s += v[k];
    }
    lds[slice][lane] = s;
    __syncthreads();
    // 32 neighbouring lanes take one column's slices
    s = lds[lane][slice];
#pragma unroll
    for (int k = 16; k; k >>= 1) s += __shfl_xor(s, k);
    const int64_t out_c = (int64_t)blockIdx.x * 32 + slice;
    if (lane || out_c >= n) return;
    void* out = out_c < cols ? dw : db;
    const int64_t at = out_c < cols ? out_c : out_c - cols;
    if (!out) return;
    if (dtype == WARP_F32) ((float*)out)[at] = s;
    else if (dtype == WARP_F16) ((_Float16*)out)[at] = (_Float16)s;
    else ((__bf16*)out)[at] = (__bf16)s;
}

constexpr int kMaxGrid = 2048;  // workgroups of the forward kernels: eight on each of 256 compute units

template <typename T, int V, int NC, int LANES, int MODE>
void rows_launch(const RowArgs& a, hipStream_t s) {
    constexpr int kRows = LANES < 256 ? 256 / LANES : 1;
    const int64_t need = (a.rows + kRows - 1) / kRows;
    const dim3 grid((uint32_t)(need < kMaxGrid ? need : kMaxGrid)), block(LANES < 256 ? 256 : LANES);
    if (a.cols % V) hipLaunchKernelGGL((k_rows<T, V, NC, LANES, true, MODE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((k_rows<T, V, NC, LANES, false, MODE>), grid, block, 0, s, a);
}

template <typename T, int MODE>
void rows_of(const RowArgs& a, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const int vectors = (a.cols + V - 1) / V;  // of a row
    if (a.cols < V) rows_launch<T, 1, 1, 16, MODE>(a, s);
    else if (vectors <= 16) rows_launch<T, V, 1, 16, MODE>(a, s);
    else if (vectors <= 32) rows_launch<T, V, 2, 16, MODE>(a, s);
    else if (vectors <= 64) rows_launch<T, V, 1, 64, MODE>(a, s);
    else if (vectors <= 128) rows_launch<T, V, 2, 64, MODE>(a, s);
    else if (vectors <= 256) rows_launch<T, V, 4, 64, MODE>(a, s);
    else if (vectors <= 512) rows_launch<T, V, 2, 256, MODE>(a, s);
    else if (vectors <= 1024) rows_launch<T, V, 4, 256, MODE>(a, s);
    else if (vectors <= 2048) rows_launch<T, V, 4, 512, MODE>(a, s);
    else rows_launch<float, 4, 8, 512, MODE>(a, s);  // only fp32 rows: kMaxCols is 2048 vectors of 16-bit elements
}

template <int MODE>
void rows_any(int32_t dtype, const RowArgs& a, hipStream_t s) {
    if (dtype == WARP_F32) rows_of<float, MODE>(a, s);
    else if (dtype == WARP_F16) rows_of<_Float16, MODE>(a, s);
    else rows_of<__bf16, MODE>(a, s);
}

constexpr int kMaxCols = 16384;  // 512 lanes of 32 columns

// Lanes of a row in the backward kernel, which holds five arrays of a lane's columns: at most 32 columns a lane. (fp32
// rows above 8,192 columns spill a tenth to a fifth of their registers then, and still move 4.4 TB/s.)
int back_lanes(int32_t cols, int32_t dtype) {
    if (cols <= 32 * (16 / dtype_bytes(dtype))) return 16;
    return cols <= 32 * kWave ? kWave : cols <= 32 * 256 ? 256 : 512;
}

int back_grid(int64_t rows, int32_t cols, int32_t dtype) {
    const int lanes = back_lanes(cols, dtype), at_once = lanes < 256 ? 256 / lanes : 1;
    const int64_t need = (rows + at_once - 1) / at_once;
    const int64_t most = cols <= kWave * 16 ? kMaxParts : lanes == 512 ? 256 : 512;  // as many as fit the registers
    const int64_t some = need < 256 ? need : need / 4 < 256 ? 256 : need / 4;
    return (int)(some < most ? some : most);
}

template <typename T, int V, int NC, int LANES>
void back_launch(const BackArgs& a, int grid, hipStream_t s) {
    const dim3 block(LANES < 256 ? 256 : LANES);
    if (a.cols % V) hipLaunchKernelGGL((k_rows_back<T, V, NC, LANES, true>), dim3(grid), block, 0, s, a);
    else hipLaunchKernelGGL((k_rows_back<T, V, NC, LANES, false>), dim3(grid), block, 0, s, a);
}

template <typename T>
void back_of(const BackArgs& a, int grid, int lanes, hipStream_t s) {
    constexpr int V = 16 / sizeof(T), N = 32 / V;
    const int vectors = (a.cols + V - 1) / V;
    if (a.cols < V) back_launch<T, 1, 1, 16>(a, grid, s);
    else if (vectors <= 16) back_launch<T, V, 1, 16>(a, grid, s);
    else if (lanes == 16) back_launch<T, V, 2, 16>(a, grid, s);
    else if (lanes == kWave && vectors <= N / 4 * kWave) back_launch<T, V, N / 4, kWave>(a, grid, s);
    else if (lanes == kWave && vectors <= N / 2 * kWave) back_launch<T, V, N / 2, kWave>(a, grid, s);
    else if (lanes == kWave) back_launch<T, V, N, kWave>(a, grid, s);
    else if (lanes == 256) back_launch<T, V, N, 256>(a, grid, s);
    else back_launch<T, V, N, 512>(a, grid, s);
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
    RowArgs a{x, x_stride, rows, cols, weight, bias, param_dtype == WARP_F32, eps,
              passes_by(rows, cols, 2 * dtype_bytes(dtype)), y, y_stride, mean, rstd, nullptr, 0,
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
    RowArgs a{x, x_stride, rows, cols, weight, bias, param_dtype == WARP_F32, eps,
              passes_by(rows, cols, dtype_bytes(dtype) + 1), nullptr, 0, nullptr, nullptr, q,
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
    RowArgs a{x, x_stride, rows, cols, nullptr, nullptr, 1, 0.f, passes_by(rows, cols, dtype_bytes(dtype) + 1), nullptr,
              0, nullptr, nullptr, q, q_stride, scale};
    WARP_LAUNCH(rows_any<kInt8>(dtype, a, (hipStream_t)hip_stream));
    return WARP_OK;
}

int warp_layer_norm_backward_scratch(int64_t rows, int32_t cols, int32_t dtype, int64_t* bytes) {
    if (!bytes || rows < 0 || cols < 1 || !dtype_ok(dtype))
        return fail(WARP_EINVAL, "layer norm backward: bad sizes");
    *bytes = (int64_t)back_grid(rows, cols, dtype) * 2 * cols * (int64_t)sizeof(float);
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
    const int grid = back_grid(rows, cols, dtype);
    const int64_t need = (int64_t)grid * 2 * cols * (int64_t)sizeof(float);
    if (sums && need && (!scratch || scratch_bytes < need || (uintptr_t)scratch % 4))
        return fail(WARP_EINVAL, "%s: needs %lld bytes of scratch (got %lld)", what, (long long)need,
                    (long long)(scratch ? scratch_bytes : 0));
    rc = require_device();
    if (rc) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    BackArgs a{dy, dy_stride, x, x_stride, rows, cols, weight, param_dtype == WARP_F32, mean, rstd, dx, dx_stride,
               passes_by(rows, cols, 3 * dtype_bytes(dtype)), sums ? (float*)scratch : nullptr};
    const int lanes = back_lanes(cols, dtype);
    if (rows) {
        if (dtype == WARP_F32) WARP_LAUNCH(back_of<float>(a, grid, lanes, s));
        else if (dtype == WARP_F16) WARP_LAUNCH(back_of<_Float16>(a, grid, lanes, s));
        else WARP_LAUNCH(back_of<__bf16>(a, grid, lanes, s));
    }
    if (sums)  // without rows: zeros
        WARP_LAUNCH(hipLaunchKernelGGL(k_join_params, dim3((2 * cols + 31) / 32), dim3(1024), 0, s,
                                       (const float*)scratch, rows ? grid : 0, cols, dweight, dbias, param_dtype));
    return WARP_OK;
}

}  // extern "C"
