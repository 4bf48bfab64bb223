// Operands of the products made ready and parts of sums joined: kernels bound by memory. 32,768 rows of 4096 bf16: 8-bit rows
// unpacked in 65 us (6.2 TB/s), columns summed in 41 (6.6 TB/s). 16,384 x 1024 sums joined in 29 us (3.5 TB/s).
#include "operands.h"

namespace warp {

namespace {

// Workgroups of four waves, a wave a row at a time and 512 columns of it; rows by steps of the grid.
constexpr int kRowWaves = 4;
constexpr int64_t kMaxRowGroups = 32768;
dim3 row_grid(int64_t rows, int64_t width) {
    const int64_t groups = cover_of(rows, kRowWaves);
    return dim3((uint32_t)cover_of(width, 512), (uint32_t)(groups < kMaxRowGroups ? groups : kMaxRowGroups));
}

// One matrix for each blockIdx.z.
struct PackJobs {
    PackRows m[2];
};
template <typename T, int PLANES>
__global__ __launch_bounds__(64 * kRowWaves) void k_pack_rows(PackJobs jobs) {
    const PackRows& j = jobs.m[blockIdx.z];
    const int64_t width = packed_width(j.cols), plane = j.rows * width;
    const int64_t c = ((int64_t)blockIdx.x * kWave + (threadIdx.x & 63)) * 8;
    if (c >= width) return;
    const int64_t end = j.now ? *j.now : j.rows;
    for (int64_t r = (int64_t)blockIdx.y * kRowWaves + (threadIdx.x >> 6); r < end; r += (int64_t)gridDim.y * kRowWaves) {
        const T* p = (const T*)j.x + (j.list ? (int64_t)j.list[r] : r) * j.stride + c;
        float v[8];
        if (c + 8 <= j.cols) {
            const auto in = load_vec<T, 8>(p);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)in.e[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < j.cols ? (float)p[e] : 0.f;
        }
        store_packed<T, PLANES>(j.out, plane, r * width + c, v);
    }
}

template <typename E, int PLANES>
__global__ __launch_bounds__(64 * kRowWaves) void k_unpack_int8(const int8_t* q, int64_t q_stride, const float* scale,
                                                                int64_t rows, int64_t cols, uint16_t* out, int64_t width,
                                                                int64_t plane) {
    const int64_t c = ((int64_t)blockIdx.x * kWave + (threadIdx.x & 63)) * 8;
    if (c >= width) return;
    for (int64_t r = (int64_t)blockIdx.y * kRowWaves + (threadIdx.x >> 6); r < rows; r += (int64_t)gridDim.y * kRowWaves) {
        const auto in = load_vec<int8_t, 8>(q + r * q_stride + c);  // rows are padded to 128
        const float f = scale[r];
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? (float)in.e[e] * f : 0.f;
        store_packed<E, PLANES>(out, plane, r * width + c, v);
    }
}

// A wave 256 columns of one row. Few rows of many parts: the four waves of a workgroup share a row's parts.
template <bool SHARED>
__global__ __launch_bounds__(64 * kRowWaves) void k_join_parts(Join j) {
    __shared__ float4v joined[SHARED ? kRowWaves : 1][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * kWave + lane) * 4;
    const int64_t m = j.m_now ? *j.m_now : j.m, k = j.k_now ? *j.k_now : j.k;
    const int parts = j.parts ? j.parts : product_splits(m, j.n, product_steps(k, j.terms), j.tile, j.splits, j.jobs);
    const float factor = j.factor ? *j.factor : 1.f;
    float bias[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = j.bias && c + e < j.n ? load_float(j.bias, j.bias_type, c + e) : 0.f;
    const int64_t plane = m * j.part_stride;
    const int by = SHARED ? kRowWaves : 1;
    for (int64_t r = (int64_t)blockIdx.y * (kRowWaves / by) + (SHARED ? 0 : w); r < j.rows;
         r += (int64_t)gridDim.y * (kRowWaves / by)) {
        const int64_t from = j.place ? (int64_t)j.place[r] : r;
        float4v sum = {};
        if (from >= 0 && c < j.n) {
            const float* p = j.part + from * j.part_stride + c;
            int i = SHARED ? w : 0;
            for (; i + 7 * by < parts; i += 8 * by) {
                float4v x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = *(const float4v*)(p + (int64_t)(i + u * by) * plane);
#pragma unroll
                for (int u = 0; u < 8; ++u) sum += x[u];
            }
            for (; i < parts; i += by) sum += *(const float4v*)(p + (int64_t)i * plane);
        }
        if constexpr (SHARED) {
            __syncthreads();  // the last row's have been read
            joined[w][lane] = sum;
            __syncthreads();
            if (w) continue;
#pragma unroll
            for (int i = 1; i < kRowWaves; ++i) sum += joined[i][lane];
        }
        if (c >= j.n) continue;
        sum *= factor;
        if (from < -1) sum += __builtin_nanf("");
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = sum[e] + bias[e];
        store_floats<4>(j.out, j.out_type, r * j.out_stride + c, v, j.n - c, false);
    }
}

// Sums of eight neighbouring columns a lane over a chunk of rows, then of the chunks.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_column_parts(const T* x, int64_t stride, int64_t rows, int64_t cols, float* room) {
    __shared__ float joined[3][V][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int64_t c = ((int64_t)blockIdx.x * kWave + lane) * V;
    const bool in = c < cols;
    if (c + V > cols) c = cols - V;
    const int64_t each = cover_of(rows, gridDim.y), first = blockIdx.y * each;
    const int64_t end = first + each < rows ? first + each : rows;
    float sum[V] = {};
    constexpr int U = 4;
    for (int64_t r = first + w; r < end; r += 4 * U) {
        Vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (in && r + 4 * u < end) v[u] = load_vec<T, V>(x + (r + 4 * u) * stride + c);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (in && r + 4 * u < end)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += (float)v[u].e[e];
    }
    if (w) {
#pragma unroll
        for (int e = 0; e < V; ++e) joined[w - 1][e][lane] = sum[e];
    }
    __syncthreads();
    if (w || !in) return;
    Vec<float, V> out;
#pragma unroll
    for (int e = 0; e < V; ++e) out.e[e] = sum[e] + joined[0][e][lane] + joined[1][e][lane] + joined[2][e][lane];
    store_vec<float, V>(room + blockIdx.y * cols + c, out);
}

// 16 columns a workgroup, 64 parts of each side by side.
__global__ __launch_bounds__(1024) void k_join_columns(const float* room, int64_t chunks, int64_t cols, void* out,
                                                       int32_t type) {
    __shared__ float joined[64][17];
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t c = (int64_t)blockIdx.x * 16 + col;
    float sum = 0.f;
    if (c < cols) {
#pragma unroll 8
        for (int64_t i = part; i < chunks; i += 64) sum += room[i * cols + c];
    }
    joined[part][col] = sum;
    __syncthreads();
    if (part || c >= cols) return;
    float v[1] = {0.f};
#pragma unroll
    for (int i = 0; i < 64; ++i) v[0] += joined[i][col];
    store_floats<1>(out, type, c, v, 1, false);
}

template <typename T>
void column_parts(const void* x, int64_t stride, int64_t rows, int64_t cols, float* room, hipStream_t s) {
    const uint32_t chunks = (uint32_t)column_chunks(rows);
    if (cols < 8)
        hipLaunchKernelGGL((k_column_parts<T, 1>), dim3(1, chunks), dim3(256), 0, s, (const T*)x, stride, rows, cols, room);
    else
        hipLaunchKernelGGL((k_column_parts<T, 8>), dim3((uint32_t)cover_of(cols, 512), chunks), dim3(256), 0, s, (const T*)x,
                           stride, rows, cols, room);
}

}  // namespace

void split_planes(const float* x, int64_t n, uint16_t* planes) {
    for (int64_t i = 0; i < n; ++i) {
        uint16_t p[3];
        split_f32(x[i], p);
        for (int t = 0; t < 3; ++t) planes[t * n + i] = p[t];
    }
}

hipError_t pack_rows(const PackRows& a, const PackRows& b, int32_t dtype, hipStream_t s) {
    PackJobs jobs{{a.rows ? a : b, b}};
    const int count = !!a.rows + !!b.rows;
    if (!count) return hipSuccess;
    dim3 grid = row_grid(jobs.m[0].rows, packed_width(jobs.m[0].cols));
    if (count == 2) {
        const dim3 other = row_grid(b.rows, packed_width(b.cols));
        grid = dim3(grid.x > other.x ? grid.x : other.x, grid.y > other.y ? grid.y : other.y, 2);
    }
    const dim3 block(64 * kRowWaves);
    (void)hipGetLastError();
    if (jobs.m[0].whole) hipLaunchKernelGGL((k_pack_rows<float, 1>), grid, block, 0, s, jobs);
    else if (dtype == WARP_F32) hipLaunchKernelGGL((k_pack_rows<float, 3>), grid, block, 0, s, jobs);
    else if (dtype == WARP_F16) hipLaunchKernelGGL((k_pack_rows<_Float16, 1>), grid, block, 0, s, jobs);
    else hipLaunchKernelGGL((k_pack_rows<__bf16, 1>), grid, block, 0, s, jobs);
    return hipGetLastError();
}

hipError_t unpack_int8(const int8_t* q, int64_t q_stride, const float* scale, int64_t rows, int64_t cols, int32_t dtype,
                       uint16_t* out, hipStream_t s, bool whole) {
    if (!rows) return hipSuccess;
    const int64_t width = packed_width(cols), plane = rows * width;
    const dim3 grid = row_grid(rows, width), block(64 * kRowWaves);
    (void)hipGetLastError();
    if (whole)
        hipLaunchKernelGGL((k_unpack_int8<float, 1>), grid, block, 0, s, q, q_stride, scale, rows, cols, out, width, plane);
    else if (dtype == WARP_F32)
        hipLaunchKernelGGL((k_unpack_int8<__bf16, 3>), grid, block, 0, s, q, q_stride, scale, rows, cols, out, width, plane);
    else if (dtype == WARP_F16)
        hipLaunchKernelGGL((k_unpack_int8<_Float16, 1>), grid, block, 0, s, q, q_stride, scale, rows, cols, out, width, plane);
    else
        hipLaunchKernelGGL((k_unpack_int8<__bf16, 1>), grid, block, 0, s, q, q_stride, scale, rows, cols, out, width, plane);
    return hipGetLastError();
}

hipError_t join_parts(const Join& j, hipStream_t s) {
    if (!j.rows) return hipSuccess;
    const uint32_t x = (uint32_t)cover_of(j.n, 256);
    const int64_t groups = cover_of(j.rows, kRowWaves);
    (void)hipGetLastError();
    if (j.rows * x <= 2048)
        hipLaunchKernelGGL(k_join_parts<true>, dim3(x, (uint32_t)j.rows), dim3(64 * kRowWaves), 0, s, j);
    else
        hipLaunchKernelGGL(k_join_parts<false>, dim3(x, (uint32_t)(groups < kMaxRowGroups ? groups : kMaxRowGroups)),
                           dim3(64 * kRowWaves), 0, s, j);
    return hipGetLastError();
}

hipError_t column_sums(const void* x, int64_t stride, int64_t rows, int64_t cols, int32_t dtype, float* room, void* out,
                       int32_t out_type, hipStream_t s) {
    (void)hipGetLastError();
    if (rows) {
        if (dtype == WARP_F32) column_parts<float>(x, stride, rows, cols, room, s);
        else if (dtype == WARP_F16) column_parts<_Float16>(x, stride, rows, cols, room, s);
        else column_parts<__bf16>(x, stride, rows, cols, room, s);
    }
    return join_columns(room, rows ? column_chunks(rows) : 0, cols, out, out_type, s);
}

hipError_t join_columns(const float* room, int64_t chunks, int64_t cols, void* out, int32_t out_type, hipStream_t s) {
    (void)hipGetLastError();
    hipLaunchKernelGGL(k_join_columns, dim3((uint32_t)cover_of(cols, 16)), dim3(1024), 0, s, room, chunks, cols, out,
                       out_type);
    return hipGetLastError();
}

}  // namespace warp
