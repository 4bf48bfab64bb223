// Products of few rows (a token, a query, a small batch) by a matrix that is read once, as it is stored: its bytes and the
// launch are what counts.
#include "operands.h"

namespace warp {

namespace {

// A piece: 16 bytes of a row, W elements. A step is 4 W k: a piece for each of a wave's quarters. float32 goes through the matrix
// instructions for it, which are fast enough for few rows and need no planes.
template <typename T>
struct Piece {
    static constexpr int W = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(W)));
};
__device__ __forceinline__ float4v few_mfma(float4v a, float4v b, float4v c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
template <typename V>
__device__ __forceinline__ float4v few_mfma(V a, V b, float4v c) {
    return product_mfma(a, b, c);
}

// The piece at p, of which `left` elements count; zeros behind them.
template <typename T>
__device__ __forceinline__ typename Piece<T>::type load_piece(const T* p, int64_t left) {
    constexpr int W = Piece<T>::W;
    typename Piece<T>::type v = {};
    if (left >= W) {
        v = __builtin_bit_cast(typename Piece<T>::type, load_vec<T, W>(p));
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (e < left) v[e] = p[e];
    }
    return v;
}
// The same of a float32 in planes, whose rows are padded to whole pieces.
__device__ __forceinline__ float4v load_planes(const uint16_t* p, int64_t plane, int64_t left) {
    float4v v = {};
    if (left <= 0) return v;
    Vec<uint16_t, 4> x[3];
#pragma unroll
    for (int t = 0; t < 3; ++t) x[t] = load_vec<uint16_t, 4>(p + t * plane);
#pragma unroll
    for (int e = 0; e < 4; ++e)
        v[e] = as_f((uint32_t)x[2].e[e] << 16) + as_f((uint32_t)x[1].e[e] << 16) + as_f((uint32_t)x[0].e[e] << 16);
    return v;
}

// x[j] of lane 4 l + t to x[t] of lane 4 l + j: registers and neighbouring lanes change places, by pairs and pairs of pairs.
template <typename V>
__device__ __forceinline__ void quad_transpose(V (&x)[4]) {
    typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
    uint4v r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __builtin_bit_cast(uint4v, x[j]);
    const bool one = threadIdx.x & 1, two = threadIdx.x & 2;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t a[4];
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            const uint32_t up = dpp<kDppXor1, 0xf>(r[j][e]), down = dpp<kDppXor1, 0xf>(r[j + 1][e]);
            a[j] = one ? down : r[j][e];
            a[j + 1] = one ? r[j + 1][e] : up;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t up = dpp<kDppXor2, 0xf>(a[j]), down = dpp<kDppXor2, 0xf>(a[j + 2]);
            r[j][e] = two ? down : a[j];
            r[j + 2][e] = two ? a[j + 2] : up;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = __builtin_bit_cast(V, r[j]);
}

// Waves make 16 BM rows of 16 BN columns; some or all of a workgroup share the k range (or their part of it), and their sums meet in
// LDS in a fixed order. Operands go straight from memory to registers.
// Along K a lane needs one column's piece, but neighbouring lanes of a load should read neighbouring pieces: four loads take
// four rows' four pieces by fours of lanes, and quad_transpose hands them to the lanes of their rows. Across K a lane loads the pieces
// of W columns at each of W k, which are the W x W elements that it needs of W blocks (block j: every Wth column from the jth on).
// Bound by memory and the loads under way: 4096 x 4096 float32 along K 22 us (3.1 TB/s), across 15 (4.5); 32,128 rows of 768
// bf16 13 to 15 us (3.5); 1 x 1024 by 1024 3.6 us, little more than an empty launch. By tiles with the weight in planes the
// first took 50, with the launches that packed it.
template <Layout LB>
constexpr int few_waves() { return LB == kAlongK ? 8 : 4; }

template <typename T, bool PLANES, Layout LB, int BM, int BN, Finish F>
__global__ __launch_bounds__(64 * few_waves<LB>()) void k_product_few(ProductArgs g) {
    constexpr int W = Piece<T>::W, kStep = 4 * W, kWaves = few_waves<LB>(), kCols = 16 * BN;
    static_assert(LB == kAlongK || BN == W, "a lane's pieces across K are of W blocks");
    typedef typename Piece<T>::type V;
    __shared__ float sums[kWaves][16 * BM][kCols + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), li = lane & 15, q = lane >> 4;
    const int sharing = LB == kAlongK ? g.splits : kWaves, group = wave / sharing, mine = wave % sharing;
    const int64_t tile = (int64_t)blockIdx.x * (kWaves / sharing) + group;
    const int64_t c0 = tile * kCols, m0 = (int64_t)blockIdx.y * 16 * BM;
    const int64_t rows = g.m_now ? *g.m_now : g.m;
    if (F == kStats && blockIdx.x == 0) {
        const int64_t t = m0 + threadIdx.x;
        if (threadIdx.x < 16 * BM && t < rows) {
            const int64_t y = g.wide ? ((const int64_t*)g.targets)[t] : (int64_t)((const int32_t*)g.targets)[t];
            g.place[t] = y >= 0 && y < g.vocabulary ? (int32_t)t : y < 0 ? -1 : -2;
        }
    }
    if (m0 >= rows) return;
    const int64_t part = F == kSum ? blockIdx.z : 0, each = F == kSum ? cover_of(cover_of(g.k, kStep), gridDim.z) * kStep : g.k;
    const int64_t first = part * each, end = first + each < g.k ? first + each : g.k;

    float4v acc[BM][BN] = {};
    auto load_a = [&](int64_t row, int64_t at) {
        const int64_t m = m0 + row < rows ? m0 + row : rows - 1;
        if constexpr (PLANES) return load_planes((const uint16_t*)g.a + m * g.a_stride + at, g.a_plane, end - at);
        else return load_piece<T>((const T*)g.a + m * g.a_stride + at, end - at);
    };
    if constexpr (LB == kAlongK) {
        // four steps: the loads' lanes are four neighbouring pieces of a row
        const int row = lane >> 2 & 3, piece = 4 * q + (lane & 3);
        constexpr int U = BM + BN <= 2 ? 2 : 1;
        for (int64_t k = first + 4 * kStep * mine; k < end; k += U * 4 * kStep * sharing) {
            V a[U][BM][4], b[U][BN][4];
            const int under_way = k + 4 * kStep * sharing < end ? U : 1;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= under_way) break;
                const int64_t at = k + u * 4 * kStep * sharing + W * piece;
#pragma unroll
                for (int j = 0; j < BN; ++j)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const int64_t c = c0 + 16 * j + 4 * row + t;
                        b[u][j][t] = load_piece<T>((const T*)g.b + (c < g.n ? c : g.n - 1) * g.b_stride + at, end - at);
                    }
#pragma unroll
                for (int i = 0; i < BM; ++i)
#pragma unroll
                    for (int t = 0; t < 4; ++t) a[u][i][t] = load_a(16 * i + 4 * row + t, at);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (u >= under_way) break;
#pragma unroll
                for (int j = 0; j < BN; ++j) quad_transpose(b[u][j]);
#pragma unroll
                for (int i = 0; i < BM; ++i) quad_transpose(a[u][i]);
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int i = 0; i < BM; ++i)
#pragma unroll
                        for (int j = 0; j < BN; ++j) acc[i][j] = few_mfma(b[u][j][t], a[u][i][t], acc[i][j]);
            }
        }
    } else {
        const int64_t column = c0 + W * li;
        const T* pb = (const T*)g.b + (column < g.n ? column : 0);
        constexpr int U = W == 4 ? 2 : 1;  // loads of 128 bytes a lane
        const int64_t columns = g.n - column;
        for (int64_t k = first + kStep * wave; k < end; k += U * kStep * kWaves) {
            V a[U][BM], b[U][W];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t at = k + u * kStep * kWaves + W * q;
#pragma unroll
                for (int w = 0; w < W; ++w) b[u][w] = load_piece<T>(pb + (at + w) * g.b_stride, at + w < end ? columns : 0);
#pragma unroll
                for (int i = 0; i < BM; ++i) a[u][i] = load_a(16 * i + li, at);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int j = 0; j < W; ++j) {
                    V t;
#pragma unroll
                    for (int w = 0; w < W; ++w) t[w] = b[u][w][j];
#pragma unroll
                    for (int i = 0; i < BM; ++i) acc[i][j] = few_mfma(t, a[u][i], acc[i][j]);
                }
        }
    }
#pragma unroll
    for (int i = 0; i < BM; ++i)
#pragma unroll
        for (int j = 0; j < BN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sums[wave][16 * i + li][LB == kAlongK ? 16 * j + 4 * q + e : BN * (4 * q + e) + j] = acc[i][j][e];
    __syncthreads();
    if (c0 >= g.n) return;
    for (int t = 64 * mine + lane; t < 16 * BM * kCols; t += 64 * sharing) {
        const int row = t / kCols, col = t % kCols;  // a row's columns lie in one wave
        const int64_t m = m0 + row, c = c0 + col;
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x += w < sharing ? sums[group * sharing + w][row][col] : 0.f;
        const bool in = c < g.n;
        if constexpr (F == kStore) {
            if (m >= rows || !in) continue;
            const float v[1] = {g.bias ? x + load_float(g.bias, g.bias_type, c) : x};
            store_floats<1>(g.out, g.out_type, m * g.out_stride + c, v, 1, false);
        } else if constexpr (F == kSum) {
            if (m >= rows || !in) continue;
            float* p = g.part + (part * rows + m) * g.part_stride + c;
            *p = g.accumulate ? *p + x : x;
        } else if constexpr (F == kStats) {
            const int64_t at = m < rows ? m : rows - 1;
            const int64_t y = g.wide ? ((const int64_t*)g.targets)[at] : (int64_t)((const int32_t*)g.targets)[at];
            if (in && m < rows && y - g.n0 == c) g.of_target[m] = x * g.to_log2;
            if (!in || y - g.n0 == c) x = g.to_log2 < 0.f ? INFINITY : -INFINITY;  // what does not count
            float top = x * g.to_log2;
#pragma unroll
            for (int d = 1; d < kCols; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
            float sum = __builtin_amdgcn_exp2f(__builtin_fmaf(x, g.to_log2, top == -INFINITY ? 0.f : -top));
#pragma unroll
            for (int d = 1; d < kCols; d <<= 1) sum += __shfl_xor(sum, d);
            if (col == 0 && m < rows) g.stats[tile * g.stats_stride + m] = make_float2(top, sum);
        } else {
            if (m >= rows) continue;
            float d = __builtin_amdgcn_exp2f(__builtin_fmaf(x, g.to_log2, -g.lse[m])) * (g.weight[m] * g.grad_scale);
            if (g.target[m] - g.n0 == c) d = g.at_target[m] * g.grad_scale;
            if (!in) d = 0.f;
            if constexpr (sizeof(T) == 4) {
                uint16_t s[3];
                split_f32(d, s);
#pragma unroll
                for (int p = 0; p < 3; ++p) ((uint16_t*)g.grad)[p * g.grad_plane + m * g.grad_stride + c] = s[p];
            } else {
                ((T*)g.grad)[m * g.grad_stride + c] = (T)d;
            }
        }
    }
}

// Waves that share a k range of so many times four steps: as many as have the least to do each, the others are for other columns.
inline int few_sharing(int64_t steps) {
    int best = 8;
    for (const int s : {4, 2, 1})
        if (cover_of(steps, s) * s * 5 < cover_of(steps, best) * best * 4) best = s;
    return best;
}

template <typename T, bool PLANES, Layout LB, int BN, Finish F>
void few(ProductArgs g, int parts, hipStream_t s) {
    if (LB == kAlongK) g.splits = few_sharing(cover_of(g.k, 16 * Piece<T>::W));
    auto go = [&](auto blocks) {
        constexpr int BM = blocks.value;
        const int groups = LB == kAlongK ? few_waves<LB>() / g.splits : 1;
        const dim3 grid((uint32_t)cover_of(g.n, 16 * BN * groups), (uint32_t)cover_of(g.m, 16 * BM), (uint32_t)parts);
        hipLaunchKernelGGL((k_product_few<T, PLANES, LB, BM, BN, F>), grid, dim3(64 * few_waves<LB>()), 0, s, g);
    };
    if (g.m <= 16) go(std::integral_constant<int, 1>{});
    else go(std::integral_constant<int, 2>{});
}

template <typename T, bool PLANES, Finish F>
void along(const ProductArgs& g, hipStream_t s) {
    if (few_wide(g.n)) few<T, PLANES, kAlongK, 2, F>(g, 1, s);
    else few<T, PLANES, kAlongK, 1, F>(g, 1, s);
}

template <typename T>
hipError_t few_of(const ProductArgs& g, bool planes, Finish finish, int parts, hipStream_t s) {
    constexpr bool kPlanesOf = sizeof(T) == 4;
    (void)hipGetLastError();
    if (finish == kStore) along<T, false, kStore>(g, s);
    else if (finish == kStats) along<T, false, kStats>(g, s);
    else if (finish == kGrad) along<T, kPlanesOf, kGrad>(g, s);
    else if (planes) few<T, kPlanesOf, kAcrossK, Piece<T>::W, kSum>(g, parts, s);
    else few<T, false, kAcrossK, Piece<T>::W, kSum>(g, parts, s);
    return hipGetLastError();
}

}  // namespace

hipError_t product_few(const ProductArgs& g, int32_t dtype, bool planes, Finish finish, int parts, hipStream_t s) {
    if (!g.m) return hipSuccess;
    return dtype == WARP_F32   ? few_of<float>(g, planes, finish, parts, s)
           : dtype == WARP_F16 ? few_of<_Float16>(g, planes, finish, parts, s)
                               : few_of<__bf16>(g, planes, finish, parts, s);
}

}  // namespace warp
