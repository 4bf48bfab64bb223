// Product of 8-bit token rows with 8-bit weight rows, a scale for each token and each output channel:
//   out[m][c] = (sum_j a[m][j] w[c][j]) w_scale[c] a_scale[m] + bias[c], sums exact in int32.
#include "encoder.h"

namespace warp {

static inline int64_t cover(int64_t n, int64_t of) { return (n + of - 1) / of; }

// Which kernel, by measured times (us, in a graph, operands in the caches; tokens x channels x columns).
// Up to four 16 x 16 tiles a compute unit, a tile's columns are split among waves, in 16 x 16, 32 x 16 or 32 x 32 so
// that there are about as many tiles as compute units: 1 x 1024 x 1024 2.8 (32 x 32 3.7, tiles of 64 x 64 4.0), 64 x
// 1024 x 1024 3.3 (4.3), 128 x 1024 x 1024 3.9 (16 x 16 4.2, 32 x 32 4.7), 400 x 400 x 400 3.7 (64 x 64 4.2), 500 x 500
// x 900 4.8 (5.1). Tiles of 32 x 32 no longer gain where rows are long: 64 x 4096 x 4096 10.6 (64 x 64 9.3), 512 x 512
// x 2048 6.6 (6.0), 450 x 450 x 2000 6.7 (6.6). Where one side has no more than 16, tiles of 16 x 16 waste no rows and
// go as far: 1 x 10,000 x 4096 9.4 (32 x 32 12.0, 64 x 64 16.4), 16 x 10,000 x 4096 13.5 (14.9, 16.7), 1 x 16,000 x
// 2048 7.0 (7.6, 9.0), 10,000 x 16 x 4096 13.4 (14.9, 17.2); at 16 x 20,000 x 1000 64 x 64 tiles take 5.0 (8.1).
// Else by a model of the time of each kind of tile, in hundredths of a full round of 128 x 128 tiles, 512 at once: up
// to 256 of them, one on a compute unit, take 0.7, and a last round costs half of what it does not fill. 64 x 64 tiles
// have no such steps and lose by long rows; 256 x 256 tiles, 256 at once, gain by them.
//                         64 x 64  128 x 128  256 x 256
//   1771 x 1003 x 771         6.4        8.5       21.6
//   512 x 4096 x 4096        17.6       21.3       46.4
//   2048 x 2048 x 2048       15.6       12.1       26.7
//   10,000 x 800 x 800       13.8       15.0       16.8
//   65,536 x 128 x 1024      18.1       15.8       21.2
//   2000 x 4000 x 4000       51.6       35.1       51.3
//   16,384 x 1024 x 1024     28.3       21.5       22.3
//   20,000 x 1500 x 2000      102       79.7       92.6
//   8192 x 4096 x 4096        200        138        115
int linear_kernel(int64_t m, int64_t n, int64_t k) {
    constexpr int64_t kUnits = 256;
    const int64_t t16 = cover(m, 16) * cover(n, 16);
    if (t16 <= (m <= 16 || n <= 16 ? 4 : 1) * kUnits) return kSplit16x16;
    if (t16 <= 2 * kUnits) return kSplit32x16;
    if (t16 <= 4 * kUnits && k <= 1024) return kSplit32x32;
    const int64_t t64 = cover(m, 64) * cover(n, 64), t128 = cover(m, 128) * cover(n, 128);
    const int64_t t256 = cover(m, 256) * cover(n, 256);
    const int64_t time64 = 10 + (100 + k / 80) * t64 / 2048;
    const int64_t time128 =
        t128 <= kUnits ? 70 : t128 <= 2 * kUnits ? 100 : 50 * cover(t128, 2 * kUnits) + 25 * t128 / kUnits;
    const int64_t time256 = (150 + 120000 / k) * cover(t256, kUnits);
    if (time64 <= time128 && time64 <= time256) return kTile64;
    return time128 <= time256 ? kTile128 : kTile256;
}

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

// One K step of a tile: kInt8Pad = 128 bytes of each of its rows.
constexpr int kStep = kInt8Pad;
// Tiles of tokens that a band of neighbouring tiles spans. An XCD's 32 tiles at work are then 4 x 8: 12 strips of
// rows and not 33 stream through its L2 (of 8192 x 8192 by 8192: 470 us without bands, 434 us with).
constexpr int kBand = 4;

typedef const __attribute__((address_space(1))) void global_void;
typedef __attribute__((address_space(3))) void lds_void;

// A row's eight 16-byte pieces lie in LDS in an order of their own, piece ^ key, so that the rows that eight
// neighbouring lanes read one piece of lie in different banks. Token blocks read rows 0 .. 15 in order. A
// channel block j reads rows 4 j + i % 4 + 16 (i / 4), which gives a lane 16 neighbouring channels of a token.
__device__ __forceinline__ int token_key(int row) { return row & 7; }
template <int BN>
__device__ __forceinline__ int channel_key(int row) { return (row & 3) | (row / (4 * BN) & 1) << 2; }

// Waits for this wave's loads into LDS. A barrier alone orders no loads that pass no registers: without this wait it
// would be the compiler's choice whether other waves find the rows there behind the barrier.
__device__ __forceinline__ void landed() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// A workgroup makes a tile of TM tokens by TN channels with WM x WN waves. Each K step's rows are copied to LDS
// by loads that pass no registers, into one of two buffers, while the matrix cores work on the other. The two
// buffers are arrays of their own, so that the compiler sees that a read of one needs no wait for loads into
// the other. Results pass the caches by: 32,768 x 4096 by 4096 went from 502 to 450 us with that, 65,536 x 1024 by 128 from
// 20 to 16 us, also where the next kernel reads them (26 to 23.5 us with one that does), as the operands stay cached.
//
// Bound by power and by the loads behind the matrix cores: 8192 x 8192 by 8192 takes 418 us (2.6e15 operations a second)
// with random values and 364 us with zeros, the matrix cores busy 63% of cycles at 1.6 to 1.8 GHz. With results kept in
// the caches (437 and 376 us; 32,768 x 4096 by 4096 502 us) it took 370 us without its loads (and 426 us). No faster, of
// 502 us: products of 32 x 32 x 32 (609), quarter steps (520), order pinned by scheduling barriers (495 with operands
// and sums tied to registers by hand, 1450 and more where the compiler spills), tokens loaded two steps ahead (511),
// workgroups that stay for several tiles and load the next one's first rows before they store (495 to 500), waits by
// counts instead of a full one (537), tiles by four waves of 128 x 128 (710). Smaller tiles gain nothing from four
// buffers and waits by counts either, nor from waves that share a tile's columns (a compute unit's loads bound them).
template <typename T, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_tile(LinearArgs g) {
    constexpr int kWaves = WM * WN;
    constexpr int kBM = TM / WM / 16, kBN = TN / WN / 16;  // 16 x 16 blocks of a wave
    constexpr int kLoadM = TM / 8 / kWaves, kLoadN = TN / 8 / kWaves;  // loads of 8 rows by a wave
    static_assert(kLoadM * 8 * kWaves == TM && kLoadN * 8 * kWaves == TN, "whole loads");
    __shared__ __attribute__((aligned(16))) int8_t a0[TM * kStep];
    __shared__ __attribute__((aligned(16))) int8_t a1[TM * kStep];
    __shared__ __attribute__((aligned(16))) int8_t w0[TN * kStep];
    __shared__ __attribute__((aligned(16))) int8_t w1[TN * kStep];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, q = lane >> 4;
    const int wm = (wave / WN) * (TM / WM), wn = (wave % WN) * (TN / WN);
    // tiles of one XCD (every eighth workgroup) are neighbours: its L2 then serves their common rows
    const int tiles_n = (g.n + TN - 1) / TN;
    const int tiles = gridDim.x;
    const int xcd = blockIdx.x & 7, per = tiles >> 3, more = tiles & 7;
    const int tile = xcd * per + (xcd < more ? xcd : more) + (blockIdx.x >> 3);
    // and they go through bands of kBand tiles of tokens, channels slower than tokens
    const int tiles_m = tiles / tiles_n, band = tile / (kBand * tiles_n);
    const int wide = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
    const int in = tile - band * kBand * tiles_n;
    const int64_t m0 = (int64_t)(band * kBand + in % wide) * TM, c0 = (int64_t)(in / wide) * TN;

    // offsets of this lane's pieces from the tile's first rows; rows past the last are the last one again
    uint32_t oa[kLoadM], ow[kLoadN];
    const int last_m = (int)(g.rows - m0 < TM ? g.rows - m0 : TM) - 1;
    const int last_c = (int)(g.n - c0 < TN ? g.n - c0 : TN) - 1;
#pragma unroll
    for (int i = 0; i < kLoadM; ++i) {
        const int row = (wave * kLoadM + i) * 8 + (lane >> 3);
        oa[i] = (uint32_t)(row < last_m ? row : last_m) * (uint32_t)g.a_stride + 16 * ((lane & 7) ^ token_key(row));
    }
#pragma unroll
    for (int i = 0; i < kLoadN; ++i) {
        const int row = (wave * kLoadN + i) * 8 + (lane >> 3);
        ow[i] = (uint32_t)(row < last_c ? row : last_c) * (uint32_t)g.w_stride +
                16 * ((lane & 7) ^ channel_key<kBN>(row));
    }
    const int8_t* pa = g.a + m0 * g.a_stride;
    const int8_t* pw = g.w + c0 * g.w_stride;
    auto load = [&](int8_t* la, int8_t* lw) {
#pragma unroll
        for (int i = 0; i < kLoadM; ++i)
            __builtin_amdgcn_global_load_lds((global_void*)(pa + oa[i]), (lds_void*)(la + (wave * kLoadM + i) * 1024),
                                             16, 0, 0);
#pragma unroll
        for (int i = 0; i < kLoadN; ++i)
            __builtin_amdgcn_global_load_lds((global_void*)(pw + ow[i]), (lds_void*)(lw + (wave * kLoadN + i) * 1024),
                                             16, 0, 0);
        pa += kStep, pw += kStep;
    };
    // where this lane reads its pieces of a block: rows 16 i + li (channels: 4 j + ...) are at fixed distances, and
    // the second half of a step's columns is at the address with bit 6 turned
    const int row_a = wm + li, row_w = wn + (li & 3) + 4 * kBN * (li >> 2);
    const int at_a = row_a * kStep + 16 * (q ^ token_key(row_a));
    const int at_w = row_w * kStep + 16 * (q ^ channel_key<kBN>(row_w));
    struct Part {  // a wave's operands of half a step
        int4v a[kBM], w[kBN];
    } part[2];
    auto read = [&](Part& p, const int8_t* la, const int8_t* lw, int half) {
#pragma unroll
        for (int j = 0; j < kBN; ++j) p.w[j] = *(const int4v*)(lw + (at_w ^ (64 * half)) + 4 * j * kStep);
#pragma unroll
        for (int i = 0; i < kBM; ++i) p.a[i] = *(const int4v*)(la + (at_a ^ (64 * half)) + 16 * i * kStep);
    };
    int4v acc[kBM][kBN] = {};
    auto multiply = [&](const Part& p) {
#pragma unroll
        for (int i = 0; i < kBM; ++i)
#pragma unroll
            for (int j = 0; j < kBN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(p.w[j], p.a[i], acc[i][j], 0, 0, 0);
    };
    // The operands of each half step are read while the matrix cores work on the half step before it, so the first
    // half of a step overlaps the second half of the last one, across the barrier.
    const int steps = g.k / kStep;
    auto step = [&](int k, const int8_t* la, const int8_t* lw, int8_t* na, int8_t* nw) {
        landed();
        __syncthreads();  // this step's rows are there, and the other buffer has been read by all
        if (k + 1 < steps) load(na, nw);
        read(part[0], la, lw, 0);
        if (k) multiply(part[1]);
        read(part[1], la, lw, 1);
        multiply(part[0]);
    };
    load(a0, w0);
    step(0, a0, w0, a1, w1);
    int k = 1;
    for (; k + 1 < steps; k += 2) {
        step(k, a1, w1, a0, w0);
        step(k + 1, a0, w0, a1, w1);
    }
    if (k < steps) step(k, a1, w1, a0, w0);
    // D[row][col] of a block lies in lane col + 16 (row / 4), element row % 4: lane (li, q) holds channels
    // kOut q + 4 j + r, r = 0 .. 3, of token li of block i. The scales are on their way during the last products
    // (1771 x 771 by 1003 7.2 us without, 6.6 us with).
    constexpr int kOut = 4 * kBN;  // neighbouring channels of a lane
    const int64_t c = c0 + wn + kOut * q;
    constexpr bool kEarly = kBM * kBN <= 16;  // 256 x 256 tiles have no registers for it
    float sw[kOut], b[kOut], sa[kBM];
    auto load_scales = [&] {
        if (kEarly && c + kOut <= g.n) {
            const auto vw = load_vec<float, kOut>(g.w_scale + c);
            const auto vb = g.bias ? load_vec<float, kOut>(g.bias + c) : Vec<float, kOut>{};
#pragma unroll
            for (int e = 0; e < kOut; ++e) sw[e] = vw.e[e], b[e] = vb.e[e];
        } else {
#pragma unroll
            for (int e = 0; e < kOut; ++e) {
                sw[e] = c + e < g.n ? g.w_scale[c + e] : 0.f;
                b[e] = c + e < g.n && g.bias ? g.bias[c + e] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t m = m0 + wm + 16 * i + li;
            if (kEarly) sa[i] = g.a_scale[m < g.rows ? m : g.rows - 1];
        }
    };
    if (kEarly) load_scales();
    multiply(part[1]);
    if (!kEarly) load_scales();
#pragma unroll
    for (int i = 0; i < kBM; ++i) {
        const int64_t m = m0 + wm + 16 * i + li;
        if (m >= g.rows) continue;
        const float s = kEarly ? sa[i] : g.a_scale[m];
        T* out = (T*)g.out + m * g.out_stride + c;
        Vec<T, kOut> v;
#pragma unroll
        for (int e = 0; e < kOut; ++e) v.e[e] = (T)((float)acc[i][e >> 2][e & 3] * sw[e] * s + b[e]);
        if (c + kOut <= g.n) {
            stream_out<T, kOut>(out, v);
        } else {
#pragma unroll
            for (int e = 0; e < kOut; ++e)
                if (c + e < g.n) out[e] = v.e[e];
        }
    }
}

// Few tiles: a workgroup's eight waves share the columns of one tile of 16 BM tokens by 16 BN channels. Wave w takes
// the steps w, w + 8, ..., straight from memory, and the waves' sums meet in LDS (integer additions: their order does
// not matter).
constexpr int kSplit = 8;
template <typename T, int BM, int BN>
__global__ __launch_bounds__(64 * kSplit) void k_linear_split(LinearArgs g) {
    constexpr int TM = 16 * BM, TN = 16 * BN, kRow = TN + 4;  // a row's padding spreads rows over the banks
    __shared__ int sums[TM * kRow];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, li = lane & 15, q = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * TM, c0 = (int64_t)blockIdx.y * TN;
    for (int i = threadIdx.x; i < TM * kRow; i += 64 * kSplit) sums[i] = 0;
    const int8_t *pa[BM], *pw[BN];
#pragma unroll
    for (int i = 0; i < BM; ++i) {
        const int64_t m = m0 + 16 * i + li;
        pa[i] = g.a + (m < g.rows ? m : g.rows - 1) * g.a_stride + 16 * q + wave * kStep;
    }
#pragma unroll
    for (int j = 0; j < BN; ++j) {
        const int64_t c = c0 + 16 * j + li;
        pw[j] = g.w + (c < g.n ? c : g.n - 1) * g.w_stride + 16 * q + wave * kStep;
    }
    // a step's pieces are under way while the one before is multiplied
    struct Pieces {
        int4v a[2][BM], w[2][BN];
    } p0, p1;
    auto load = [&](Pieces& p) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int j = 0; j < BN; ++j) p.w[h][j] = *(const int4v*)(pw[j] + 64 * h);
#pragma unroll
            for (int i = 0; i < BM; ++i) p.a[h][i] = *(const int4v*)(pa[i] + 64 * h);
        }
#pragma unroll
        for (int i = 0; i < BM; ++i) pa[i] += kSplit * kStep;
#pragma unroll
        for (int j = 0; j < BN; ++j) pw[j] += kSplit * kStep;
    };
    int4v acc[BM][BN] = {};
    auto multiply = [&](const Pieces& p) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < BM; ++i)
#pragma unroll
                for (int j = 0; j < BN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(p.w[h][j], p.a[h][i], acc[i][j], 0, 0, 0);
    };
    int left = (g.k / kStep - wave + kSplit - 1) / kSplit;  // this wave's steps
    if (left > 0) load(p0);
    for (; left > 0; left -= 2) {
        if (left > 1) load(p1);
        multiply(p0);
        if (left > 2) load(p0);
        if (left > 1) multiply(p1);
    }
    __syncthreads();
    if (wave * kStep < g.k) {
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) atomicAdd(&sums[(16 * i + li) * kRow + 16 * j + 4 * q + r], acc[i][j][r]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < TM * TN; i += 64 * kSplit) {
        const int row = i / TN, col = i % TN;
        const int64_t m = m0 + row, c = c0 + col;
        if (m < g.rows && c < g.n)
            ((T*)g.out)[m * g.out_stride + c] =
                (T)((float)sums[row * kRow + col] * g.w_scale[c] * g.a_scale[m] + (g.bias ? g.bias[c] : 0.f));
    }
}

template <typename T, int BM, int BN>
void split(const LinearArgs& g, hipStream_t s) {
    const dim3 grid((uint32_t)((g.rows + 16 * BM - 1) / (16 * BM)), (g.n + 16 * BN - 1) / (16 * BN));
    hipLaunchKernelGGL((k_linear_split<T, BM, BN>), grid, dim3(64 * kSplit), 0, s, g);
}

template <typename T, int TM, int TN, int WM, int WN>
void tiles(const LinearArgs& g, hipStream_t s) {
    const int64_t n = ((g.rows + TM - 1) / TM) * ((g.n + TN - 1) / TN);
    hipLaunchKernelGGL((k_linear_tile<T, TM, TN, WM, WN>), dim3((uint32_t)n), dim3(64 * WM * WN), 0, s, g);
}

template <typename T>
void linear(const LinearArgs& g, hipStream_t s) {
    switch (linear_kernel(g.rows, g.n, g.k)) {
        case kSplit16x16: return split<T, 1, 1>(g, s);
        case kSplit32x16: return split<T, 2, 1>(g, s);
        case kSplit32x32: return split<T, 2, 2>(g, s);
        case kTile64: return tiles<T, 64, 64, 2, 2>(g, s);
        case kTile128: return tiles<T, 128, 128, 2, 4>(g, s);
        default: return tiles<T, 256, 256, 2, 4>(g, s);
    }
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
    if (a_stride > 1 << 23 || w_stride > 1 << 23)
        return fail(WARP_ENOTSUP, "%s: strides are at most 2^23 (got %lld, %lld)", what, (long long)a_stride,
                    (long long)w_stride);
    if ((uintptr_t)a_scale % 4 || (uintptr_t)w_scale % 4 || (uintptr_t)bias % 4 ||
        (uintptr_t)out % dtype_bytes(out_dtype))
        return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    if (rows > 1 && out_stride < n)
        return fail(WARP_EINVAL, "%s: a row stride of %lld is below %d columns", what, (long long)out_stride, n);
    if (cover(rows, 64) * cover(n, 64) >= 1 << 24)  // of 256 threads each: a grid has at most 2^32
        return fail(WARP_ENOTSUP, "%s: %lld rows by %d channels are more than 2^24 tiles of 64 x 64", what,
                    (long long)rows, n);
    const int rc = require_device();
    if (rc || !rows) return rc;
    const LinearArgs g{a, a_stride, a_scale, rows, w, w_stride, w_scale, n, padded, bias, out, out_stride};
    hipStream_t s = (hipStream_t)hip_stream;
    if (out_dtype == WARP_F32) WARP_LAUNCH(linear<float>(g, s));
    else if (out_dtype == WARP_F16) WARP_LAUNCH(linear<_Float16>(g, s));
    else WARP_LAUNCH(linear<__bf16>(g, s));
    return WARP_OK;
}
