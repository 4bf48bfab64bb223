// Products of matrices on the matrix cores, most of them of 16-bit elements, with what the callers do to a finished tile:
//   C[m][n] = sum_k A(m, k) B(n, k), sums in fp32.
// An operand's elements of one row lie together (kAlongK: tokens, weights as stored) or those of one k (kAcrossK: its
// transpose, as stored). Operands are 16-byte aligned, their strides multiples of 8 (float32: 4); along K a row's elements beyond k up
// to the next multiple of 8 are zeros; across K a row is readable up to the next multiple of 8.
//
// float32 operands come as three planes of bfloat16, high + middle + low = x to the last bit (split_f32), and a
// product as the six of nine products of planes that count: those left out are at most 2^-24 (1 + 2^-10) of |a b| together (2^-23
// beside the largest numbers), of either sign.
// (A matrix instruction for fp32 operands has a 16th of the rate; six products are 2.7 times as fast.) Where there are few
// rows, for which packing a whole weight would take longer than the product, they are multiplied as they are.
#pragma once

#include <type_traits>

#include "encoder.h"

namespace warp {

enum Layout { kAlongK, kAcrossK };
enum Finish {
    kStore,  // out = factor * C + bias
    kSum,    // part[split] (+)= C, in fp32
    kStats,  // softmax statistics of a tile's rows
    kGrad,   // the loss's gradient for the logits
};
enum Tile { kT64, kT128, kT256 };

struct ProductArgs {
    const void *a, *b;
    int64_t a_stride, b_stride;  // elements between rows as stored
    int64_t a_plane, b_plane;    // elements between the planes of a float32 operand
    int64_t m, n, k;
    const int32_t *m_now, *k_now;  // device counts that take the place of m and k where they are not null
    int32_t terms;                 // 1, or 6 products of planes
    int32_t splits, jobs;          // at most so many parts of the k range, to have about so many tiles at work
    // 8-bit rows in the place of b (across K): b_stride bytes apart, a scale for each
    const float* b_scale;
    float* sums;  // [split][tile column][m]: parts of the sums of A's columns over k; may be null
    void* all_sums;  // [m]: the sums themselves, of kStore products in tiles of 64; may be null
    int32_t sums_type;
    // kStore
    void* out;
    int64_t out_stride;
    int32_t out_type;
    const float* factor;
    const void* bias;  // only where B lies along K
    int32_t bias_type;
    // kSum
    float* part;
    int64_t part_stride;  // a part is as many rows as there are now
    bool accumulate;
    // kStats and kGrad: rows are tokens, columns n0, n0 + 1, ... of the vocabulary
    float to_log2;          // a logit in units of log 2 is to_log2 * C; not zero
    int64_t n0;
    const int32_t* target;  // a row's column
    float2* stats;          // [tile column][row]: largest logit of the others than the target, sum of their exponentials
    int64_t stats_stride;
    float* of_target;       // [row] the target's logit
    // instead of `target`, of few rows: the tokens' own targets, by which a row's place becomes its number, -1 or -2
    const void* targets;
    bool wide;
    int64_t vocabulary;
    int32_t* place;
    const float *lse, *weight, *at_target;  // [row] in units of log 2; of the row; value at the target
    void* grad;
    int64_t grad_stride, grad_plane;
    float grad_scale;
};

__host__ __device__ inline int64_t cover_of(int64_t n, int64_t of) { return (n + of - 1) / of; }

constexpr int kProductStep = 64;  // columns of a step: 128 bytes of a row

__host__ __device__ inline int64_t product_steps(int64_t k, int terms) { return cover_of(k, kProductStep) * terms; }

// Parts of the k range: so many that about `jobs` tiles are at work, of two steps at least.
__host__ __device__ inline int product_splits(int64_t m, int64_t n, int64_t steps, int tile, int splits, int jobs) {
    const int64_t tiles = cover_of(m, tile) * cover_of(n, tile);
    int64_t s = tiles ? jobs / tiles : 1;
    s = s < steps / 2 ? s : steps / 2;
    s = s < splits ? s : splits;
    return s < 1 ? 1 : (int)s;
}
inline int tile_size(Tile t) { return t == kT64 ? 64 : t == kT128 ? 128 : 256; }
// Tiles at work at once.
inline int tile_jobs(Tile t) { return t == kT64 ? 1024 : t == kT128 ? 512 : 256; }

// How a product is made: its tiles, and whether its k range is split.
struct ProductPlan {
    Tile tile;
    bool split;
    int64_t time;  // by the model below
};
// The faster one by a model of measured times, in ns. `jobs` tiles of `steps` steps take rounds of as many as are at work at
// once, the last one less where it leaves compute units to fewer. Their bytes take time too: operands from memory at 5 TB/s and
// again for each tile at 20 (unless the caches hold them), results at 5.5, less for short pieces of rows; a quarter of the
// shorter of both times is not hidden behind the longer. Parts are written and read once more, at 4 TB/s, by a launch of
// its own. Measured (us, 16-bit elements, operands in the caches; whole | in parts):
//                           64 x 64      128 x 128    256 x 256
//   1 x 1024 x 1024        7.0 | 6.5    10.5 | 7.2   23.5 | 9.1
//   1024 x 1024 x 1024     8.1 | 18     11.9 | 24    26.7 | 28
//   1024 x 1024 x 4096      33 | 25       42 | 27      87 | 43
//   8192 x 1024 x 1024      27            22           30
//   65,536 x 128 x 1024     31            25           31
//   2048 x 4096 x 4096      97            65           94
//   4096 x 4096 x 4096     192           129          111
//   128 x 1024 x 65,536    465 | 44      603 | 39    1403 | 54
//   4096 x 1024 x 65,536  1266           819 | 614   1533 | 490
inline int64_t product_time(Tile t, int64_t jobs, int64_t steps) {
    const int64_t at_once = tile_jobs(t), full = jobs / at_once, rest = jobs % at_once;
    if (t == kT64)
        return full * (650 * steps + 2200) + (!rest ? 0 : rest <= 256 ? 460 * steps + 1000 : rest <= 512 ? 500 * steps + 1500
                                                                                                         : 800 * steps + 2500);
    if (t == kT128) return full * (1000 * steps + 3500) + (!rest ? 0 : rest <= 256 ? 600 * steps + 3000 : 1000 * steps + 3500);
    return full * (1600 * steps + 9000) + (!rest ? 0 : rest <= 160 ? 1350 * steps + 6000 : 1600 * steps + 9000);
}
inline int64_t product_traffic(Tile t, int64_t m, int64_t n, int64_t steps) {
    const int64_t size = tile_size(t), a = m * steps * 128, b = n * steps * 128, cached = 4 << 20;
    const int64_t loads = a * (a > cached ? cover_of(n, size) : 1) + b * (b > cached ? cover_of(m, size) : 1);
    return (a + b) / 5000 + loads / 20000 + m * n * 2 * (96 + size) / size / 5500;
}
constexpr int kMaxSplits = 256;
inline ProductPlan plan_product(int64_t m, int64_t n, int64_t steps, bool may_split, Tile largest = kT256) {
    ProductPlan best{kT64, false, INT64_MAX};
    for (const Tile t : {kT64, kT128, kT256}) {
        if (t > largest) break;
        const int64_t tiles = cover_of(m, tile_size(t)) * cover_of(n, tile_size(t));
        if (t != largest && tiles >= 1 << 22) continue;  // a grid has at most 2^32 threads
        const int64_t traffic = product_traffic(t, m, n, steps);
        auto both = [&](int64_t time) { return time > traffic ? time + traffic / 4 : traffic + time / 4; };
        const int64_t whole = both(product_time(t, tiles, steps));
        if (whole < best.time) best = {t, false, whole};
        const int splits = may_split ? product_splits(m, n, steps, tile_size(t), kMaxSplits, tile_jobs(t)) : 1;
        if (splits < 2) continue;
        const int64_t parts = both(product_time(t, tiles * splits, cover_of(steps, splits))) + 5500 + m * n * splits / 500;
        if (parts < best.time) best = {t, true, parts};
    }
    return best;
}

// What a linear layer's products choose, for the tests, which have to reach each kernel: the tile, plus 4 where the k range
// is split; with `bytes` that of 8-bit rows as they are, -1 where they are unpacked.
int product_choice(int64_t m, int64_t n, int64_t k, int dtype, bool bytes);

// x = high + middle + low, each the bfloat16 that is nearest to what is left (ties away from zero): |middle| <= 2^-8 and |low| <= 2^-17 of
// x's power of two, on either side of zero. Cut off towards zero they would be twice and four times as large and all of x's sign, and what
// products leave out would be up to 2^-21 of them, always towards zero. Near the largest number the first is cut off: rounded up it is
// infinite. An infinity or a NaN stays in the first. Below 2^-110 what is finer than bfloat16's smallest number, 2^-133, is rounded away.
__host__ __device__ inline void split_f32(float x, uint16_t (&out)[3]) {
    uint32_t u;
    __builtin_memcpy(&u, &x, 4);
    const bool special = (u & 0x7f800000u) == 0x7f800000u;
    float rest = x;
    for (int i = 0; i < 3; ++i) {
        uint32_t v;
        __builtin_memcpy(&v, &rest, 4);
        const bool top = i == 0 && (v & 0x7fffffffu) >= 0x7f7f8000u;
        v = (top ? v : v + 0x8000u) & 0xffff0000u;
        if (special) v = i ? 0 : u & 0x7fffff ? 0x7fc00000u : u;
        out[i] = (uint16_t)(v >> 16);
        float part;
        __builtin_memcpy(&part, &v, 4);
        rest -= part;
    }
}
// The same for the tests: [3][n].
void split_planes(const float* x, int64_t n, uint16_t* planes);

// Launches: element is WARP_F16 or WARP_BF16 (also for planes), or WARP_F32 up to kT128.
hipError_t product_along(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s);   // A, B along K
hipError_t product_mixed(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s);   // B across K
hipError_t product_across(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s);  // both
// Operands as they are, of any alignment, A along K (with `planes` a float32 in planes). B along K: kStore, kStats or kGrad; across K:
// kSum in `parts` parts.
hipError_t product_few(const ProductArgs& g, int32_t dtype, bool planes, Finish finish, int parts, hipStream_t s);
hipError_t product_bytes(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s);  // b of 8 bits; to kT128
hipError_t product_softmax(const ProductArgs& g, int element, bool planes, Tile tile, Finish finish, hipStream_t s);

#ifdef __HIPCC__

typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

typedef const __attribute__((address_space(1))) void product_global;
typedef __attribute__((address_space(3))) void product_lds;
typedef __attribute__((address_space(3))) short4v product_lds4;

static __device__ __attribute__((aligned(16))) uint32_t g_zeros[4];  // where pieces beyond the k range are read

template <typename E>
struct Eight {
    typedef E type __attribute__((ext_vector_type(8)));
};
__device__ __forceinline__ float4v product_mfma(Eight<__bf16>::type a, Eight<__bf16>::type b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
template <>
struct Eight<float> {  // four of them
    typedef float4v type;
};
__device__ __forceinline__ float4v product_mfma(float4v a, float4v b, float4v c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ float4v product_mfma(Eight<_Float16>::type a, Eight<_Float16>::type b, float4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Waits for this wave's loads into LDS and for its reads of LDS, before a barrier behind which other waves read the ones
// and load over the others. A barrier alone orders neither: the compiler leaves reads under way across it, whose registers
// are needed only later, and where two kernels shared a compute unit, loads have come before such reads.
__device__ __forceinline__ void product_landed() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// Where the 16-byte pieces of a staged operand lie in LDS.
// Along K a row has eight pieces, in the order piece ^ key(row), so that the rows that neighbouring lanes read one
// piece of lie in different banks. Token blocks read rows 0 .. 15 in order; a channel block j reads rows
// 4 j + i % 4 + 4 B (i / 4), which gives a lane 4 B neighbouring columns of the result.
// Across K a k has T / 8 pieces, two for 16 columns, in the order pair ^ pair_key(k): the transposing reads of 16 lanes
// take 32 bytes of four k each, and lanes 16 apart take k 8 apart. A float32's k has T / 4 pieces, in the order piece ^
// float_key(k): 16 lanes read 16 neighbours of one k, lanes 16 apart take k four apart.
__device__ __forceinline__ int token_piece(int row) { return row & 7; }
template <int B>
__device__ __forceinline__ int channel_piece(int row) { return (row & 3) | (row / (4 * B) & 1) << 2; }
__device__ __forceinline__ int float_key(int k) { return (k >> 2 & 3) * 4; }
template <int T>
__device__ __forceinline__ int pair_key(int k) { return ((k & 3) | (k >> 3 & 3) << 2) & (T / 16 - 1); }

// One operand's part in a tile of T rows by 128 bytes of k, of S each, for one wave of WAVES.
template <Layout L, int T, int WAVES, bool CHANNELS, int B, int S>
struct Stage {
    static constexpr int kLoads = T / 8 / WAVES;  // of 1 KB
    static_assert(kLoads * 8 * WAVES == T, "whole loads");
    uint32_t off[kLoads];
    const uint8_t* at;  // the next step's first byte, of plane 0
    int64_t step_bytes;
    int lane, wave;

    __device__ __forceinline__ int key(int row) const { return CHANNELS ? channel_piece<B>(row) : token_piece(row); }
    // this lane's k within a step, in load i
    __device__ __forceinline__ int k_of(int i) const {
        const int unit = wave * kLoads + i;
        if (L == kAlongK) return 16 / S * ((lane & 7) ^ key(unit * 8 + (lane >> 3)));
        return (unit * 1024 + lane * 16) / (T * S);
    }
    __device__ __forceinline__ void start(const void* p, int64_t stride, int64_t first, int64_t rows, int lane_, int wave_) {
        lane = lane_, wave = wave_;
        if (L == kAlongK) {
            at = (const uint8_t*)p + first * stride * S;
            step_bytes = 128;
            const int last = (int)(rows - first < T ? rows - first : T) - 1;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int row = (wave * kLoads + i) * 8 + (lane >> 3);
                off[i] = (uint32_t)(row < last ? row : last) * (uint32_t)(stride * S) + S * k_of(i);
            }
        } else {
            constexpr int W = 16 / S;
            at = (const uint8_t*)p + first * S;
            step_bytes = stride * 128;
            const int64_t end = (rows - 1) / W * W - first;  // the last piece
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int k = k_of(i);
                const int piece = ((wave * kLoads + i) * 64 + lane) & (T / W - 1);
                const int64_t row = W * (piece ^ (S == 4 ? float_key(k) : pair_key<T>(k) << 1));
                off[i] = (uint32_t)k * (uint32_t)(stride * S) + (uint32_t)(row < end ? row : end) * S;
            }
        }
    }
    __device__ __forceinline__ void load(uint8_t* lds, int64_t plane) const {
        const uint8_t* from = at + 2 * plane;
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_global_load_lds((product_global*)(from + off[i]),
                                             (product_lds*)(lds + (wave * kLoads + i) * 1024), 16, 0, 0);
    }
    __device__ __forceinline__ void load_last(uint8_t* lds, int64_t plane, int left) const {  // zeros beyond `left` k
        const uint8_t* from = at + 2 * plane;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const uint8_t* p = k_of(i) < left ? from + off[i] : (const uint8_t*)g_zeros;
            __builtin_amdgcn_global_load_lds((product_global*)p, (product_lds*)(lds + (wave * kLoads + i) * 1024), 16,
                                             0, 0);
        }
    }
};

// The same for 8-bit rows across K, which pass registers: 16 bytes a thread, times their row's scale, rounded to E. Matrix instructions
// take no scale for each k, and what the rounding loses as a second operand would double the products: the weight's gradient
// is off by 0.23% of it in bf16 (0.17% is its own rounding), 0.028% in fp16 (0.021%).
template <typename E, int T>
struct ByteStage {
    const int8_t* at;
    const float* scale;
    int64_t step_bytes;
    int k, place;
    typedef int int4v __attribute__((ext_vector_type(4)));
    int4v data;
    float factor;
    __device__ __forceinline__ void start(const void* p, int64_t stride, const float* scales, int64_t first, int64_t step) {
        constexpr int kPairs = T / 16;
        k = threadIdx.x / kPairs;
        const int pair = threadIdx.x % kPairs;
        at = (const int8_t*)p + (step * kProductStep + k) * stride + first + 16 * pair;
        scale = scales + step * kProductStep + k;
        step_bytes = stride * kProductStep;
        place = k * T * 2 + (pair ^ pair_key<T>(k)) * 32;
    }
    __device__ __forceinline__ void load(int64_t left) {
        data = int4v{}, factor = 0.f;
        if (k < left) data = *(const int4v*)at, factor = *scale;
        at += step_bytes;
        scale += kProductStep;
    }
    __device__ __forceinline__ void put(uint8_t* lds) const {
        typename Eight<E>::type v[2];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e >> 3][e & 7] = (E)((float)(int8_t)(data[e >> 2] >> 8 * (e & 3)) * factor);
        *(typename Eight<E>::type*)(lds + place) = v[0];
        *(typename Eight<E>::type*)(lds + place + 16) = v[1];
    }
};

// Where a lane reads blocks of 16 rows of a staged operand: block i of B, half a step (32 k) at a time.
template <typename E, Layout L, int T, bool CHANNELS, int B>
struct Blocks {
    typedef typename Eight<E>::type V;
    int at;
    __device__ __forceinline__ void start(int first, int lane) {
        const int li = lane & 15, q = lane >> 4;
        if (L == kAlongK) {
            const int row = CHANNELS ? first + (li & 3) + 4 * B * (li >> 2) : first + li;
            at = row * 128 + 16 * (q ^ (CHANNELS ? channel_piece<B>(row) : token_piece(row)));
        } else if (sizeof(E) == 4) {
            at = 4 * q * T * 4 + ((first / 16) ^ q) * 64 + li * 4;
        } else {
            const int k = 8 * q + (li >> 2);
            at = k * T * 2 + ((first / 16) ^ pair_key<T>(k)) * 32 + (li & 3) * 8;
        }
    }
    __device__ __forceinline__ V read(const uint8_t* lds, int i, int half) const {
        if (L == kAlongK)
            return *(const V*)(lds + (at ^ (64 * half)) + (CHANNELS ? 4 : 16) * i * 128);
        if constexpr (L == kAcrossK && sizeof(E) == 4) {
            const uint8_t* p = lds + (at ^ (64 * i)) + half * 16 * T * 4;
            V v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *(const float*)(p + e * T * 4);
            return v;
        }
        int place = at;
        asm volatile("" : "+v"(place));  // kept from computing all blocks' addresses ahead, which takes registers
        const uint8_t* p = lds + (place ^ (32 * i)) + half * 32 * T * 2;
        const short4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((product_lds4*)p);
        const short4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((product_lds4*)(p + 4 * T * 2));
        typedef short short8v __attribute__((ext_vector_type(8)));
        const short8v both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(V, both);
    }
};

template <int W>
__device__ __forceinline__ void store_floats(void* out, int32_t type, int64_t at, const float (&v)[W], int64_t left,
                                             bool past_caches) {
    auto put = [&](auto t) {
        typedef decltype(t) T;
        T* p = (T*)out + at;
        Vec<T, W> r;
#pragma unroll
        for (int e = 0; e < W; ++e) r.e[e] = (T)v[e];
        if (left >= W) {
            if (past_caches) stream_out<T, W>(p, r);
            else store_vec<T, W>(p, r);
        } else {
#pragma unroll
            for (int e = 0; e < W; ++e)
                if (e < left) p[e] = r.e[e];
        }
    };
    if (type == WARP_F32) put(0.f);
    else if (type == WARP_F16) put((_Float16)0);
    else put((__bf16)0.f);
}

__device__ __forceinline__ float load_float(const void* p, int32_t type, int64_t at) {
    return type == WARP_F32 ? ((const float*)p)[at]
                            : type == WARP_F16 ? (float)((const _Float16*)p)[at] : (float)((const __bf16*)p)[at];
}

// From block j's columns 4 q + e in lane (li, q) to block q's (of two blocks: 4 (2 (q / 2) + j) + e of block q % 2).
template <int B>
__device__ __forceinline__ void neighbours(float4v (&x)[B]) {
    auto swap = [&](int a, int b, auto far) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t u = as_u(x[a][e]), v = as_u(x[b][e]);
            if constexpr (far.value) {
                const auto r = __builtin_amdgcn_permlane32_swap(u, v, false, false);
                x[a][e] = as_f(r[0]), x[b][e] = as_f(r[1]);
            } else {
                const auto r = __builtin_amdgcn_permlane16_swap(u, v, false, false);
                x[a][e] = as_f(r[0]), x[b][e] = as_f(r[1]);
            }
        }
    };
    if constexpr (B == 4) {
        swap(0, 2, std::true_type{});
        swap(1, 3, std::true_type{});
        swap(2, 3, std::false_type{});
    }
    swap(0, 1, std::false_type{});
}

// Tiles that neighbouring workgroups of an XCD work on span bands of four tiles of rows, so that its L2 serves what
// they have in common (bands of two and eight are as fast).
constexpr int kProductBand = 4;

enum Kind { kPlain, kPlanes, kBytes };  // G in planes of a float32; B of 8 bits

// One tile by four waves (64 x 64) or eight: a step's rows of A and B are loaded into one pair of buffers in LDS, past the
// registers, while the matrix cores work on the other. 256 x 256 has the fewest bytes from LDS and from memory for an
// operation, and one workgroup on a compute unit; the smaller tiles are for sizes that would leave compute units idle or
// round up too far (plan_product).
// Large products are bound by the matrix cores, busy 54 to 60% of the time at 1.9 to 2.0 GHz, and by what keeps them from
// work: a copy whose rows all came from the caches ran 3 to 5% faster, one without results 4% (k = 8192) to 16% (1024). No
// read of LDS has a bank conflict. bf16, us (and those of a library's product):
//                               both along K    B across K     both across K
//   8192 x 8192 by 8192           851  (767)     915  (873)      945  (991)
//   16,384 x 32,128 by 1024      1028  (942)    1056 (1085)     1090 (1185)
// Not faster: workgroups that stay for several tiles, the next one's first rows on their way (8192^3: 863); four waves of
// 128 x 128 each (1640 to 1790: accumulators are moved between registers); loads behind the reads, wave priorities and
// groups of instructions fixed by hints (spilled registers, 1.5 times slower and more). The products of 8-bit rows in tiles of 128 and
// in parts spill 16 registers.
template <typename E, Layout LA, Layout LB, int TM, int TN, int WM, int WN, Finish F, Kind KIND>
__global__ __launch_bounds__(64 * WM * WN, TM == 128 ? 4 : 2) void k_product(ProductArgs g) {
    constexpr int kWaves = WM * WN;
    constexpr int kBM = TM / WM / 16, kBN = TN / WN / 16;  // blocks of a wave
    constexpr bool kAllSums = F == kStore && TM == 64;
    constexpr bool kWide = LB == kAlongK;                  // a lane holds 4 kBN neighbouring columns, else 4 in each block
    __shared__ __attribute__((aligned(16))) uint8_t a0[TM * 128];
    __shared__ __attribute__((aligned(16))) uint8_t a1[TM * 128];
    __shared__ __attribute__((aligned(16))) uint8_t b0[TN * 128];
    __shared__ __attribute__((aligned(16))) uint8_t b1[TN * 128];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, q = lane >> 4;
    const int wm = (wave / WN) * (TM / WM), wn = (wave % WN) * (TN / WN);

    const int64_t rows = g.m_now ? *g.m_now : g.m;
    const int64_t k = g.k_now ? *g.k_now : g.k;
    constexpr int kStep = 128 / sizeof(E);
    const int64_t steps = cover_of(k, kStep) * g.terms;
    const int tiles_m = (int)cover_of(rows, TM), tiles_n = (int)cover_of(g.n, TN);
    const int splits = F == kSum ? product_splits(rows, g.n, steps, TM, g.splits, g.jobs) : 1;
    const int tiles = tiles_m * tiles_n, total = tiles * splits;
    // tiles of one XCD (every eighth workgroup) are neighbours
    const int xcd = blockIdx.x & 7, per = total >> 3, more = total & 7, in_xcd = blockIdx.x >> 3;
    if (in_xcd >= per + (xcd < more)) return;
    const int job = xcd * per + (xcd < more ? xcd : more) + in_xcd;
    const int split = job / tiles, tile = job % tiles;
    const int band = tile / (kProductBand * tiles_n), in = tile - band * kProductBand * tiles_n;
    const int wide = tiles_m - band * kProductBand < kProductBand ? tiles_m - band * kProductBand : kProductBand;
    const int tile_n = in / wide;
    const int64_t m0 = (int64_t)(band * kProductBand + in % wide) * TM, c0 = (int64_t)tile_n * TN;

    const int64_t each = cover_of(steps, splits);
    const int64_t first = split * each;
    const int count = (int)(steps - first < each ? (steps > first ? steps - first : 0) : each);

    Stage<LA, TM, kWaves, false, kBM, sizeof(E)> sa;
    Stage<LB, TN, kWaves, kWide, kBN, sizeof(E)> sb;
    sa.start(g.a, g.a_stride, m0, rows, lane, wave);
    // a step's 64 k go through all terms before the next ones: their planes are in the caches then
    int64_t kk = g.terms == 1 ? first : first / g.terms;
    int term = g.terms == 1 ? 0 : (int)(first % g.terms);
    ByteStage<E, TN> bytes;
    if constexpr (KIND == kBytes) {
        bytes.start(g.b, g.b_stride, g.b_scale, c0, first);
    } else {
        sb.start(g.b, g.b_stride, c0, g.n, lane, wave);
        sb.at += kk * sb.step_bytes;
    }
    sa.at += kk * sa.step_bytes;
    auto load = [&](uint8_t* la, uint8_t* lb) {
        // planes of the terms: (0,0) (0,1) (1,0) (1,1) (0,2) (2,0)
        const int64_t plane_a = (int64_t)(0x201100 >> 4 * term & 3) * g.a_plane, plane_b = (int64_t)(0x021010 >> 4 * term & 3) * g.b_plane;
        const int64_t left = k - kk * kStep;
        if constexpr (KIND == kBytes) bytes.load(left);
        if (left >= kStep) {
            sa.load(la, plane_a);
            if constexpr (KIND != kBytes) sb.load(lb, plane_b);
        } else {
            sa.load_last(la, plane_a, (int)left);
            if constexpr (KIND != kBytes) sb.load_last(lb, plane_b, (int)left);
        }
        if (++term < g.terms) return;
        term = 0;
        ++kk;
        sa.at += sa.step_bytes;
        if constexpr (KIND != kBytes) sb.at += sb.step_bytes;
    };

    Blocks<E, LA, TM, false, kBM> ra;
    Blocks<E, LB, TN, kWide, kBN> rb;
    ra.start(wm, lane);
    rb.start(wn, lane);
    typedef typename Eight<E>::type V;
    struct Part {  // a wave's operands of half a step
        V a[kBM], b[kBN];
    } part[2];
    auto read = [&](Part& p, const uint8_t* la, const uint8_t* lb, int half) {
#pragma unroll
        for (int j = 0; j < kBN; ++j) p.b[j] = rb.read(lb, j, half);
#pragma unroll
        for (int i = 0; i < kBM; ++i) p.a[i] = ra.read(la, i, half);
    };
    float4v acc[kBM][kBN] = {};
    auto multiply = [&](const Part& p) {
#pragma unroll
        for (int i = 0; i < kBM; ++i)
#pragma unroll
            for (int j = 0; j < kBN; ++j) acc[i][j] = product_mfma(p.b[j], p.a[i], acc[i][j]);
    };
    V ones;
#pragma unroll
    for (int e = 0; e < (int)(sizeof(V) / sizeof(E)); ++e) ones[e] = (E)1.f;
    float4v totals[kBM] = {};
    int turn = (int)(first % tiles_n);
    // The operands of each half step are read while the matrix cores work on the half step before it, across the
    // barrier between steps.
    auto step = [&](int s, const uint8_t* la, const uint8_t* lb, uint8_t* na, uint8_t* nb) {
        product_landed();
        __syncthreads();  // this step's rows are there, and the other buffer has been read by all
        if (s + 1 < count) load(na, nb);
        read(part[0], la, lb, 0);
        if (s) multiply(part[1]);
        read(part[1], la, lb, 1);
        multiply(part[0]);
        if constexpr (KIND == kBytes) {
            // sums of A's columns: products by ones, of steps that the workgroups of a row of tiles take in turn, or all by the
            // first one, which saves the launch that adds them (62 -> 59 us where that is one of six; tiles of 128, by which
            // it would take 57 instead of 42 for 3000 x 2048 by 2048, take turns)
            if ((kAllSums ? g.all_sums && tile_n == 0 : g.sums && turn == tile_n) && wave % WN == 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < kBM; ++i) totals[i] = product_mfma(ones, part[h].a[i], totals[i]);
            }
            turn = turn + 1 == tiles_n ? 0 : turn + 1;
            if (s + 1 < count) bytes.put(nb);
        }
    };
    if (count) {
        load(a0, b0);
        if constexpr (KIND == kBytes) bytes.put(b0);
        step(0, a0, b0, a1, b1);
        int s = 1;
        for (; s + 1 < count; s += 2) {
            step(s, a1, b1, a0, b0);
            step(s + 1, a0, b0, a1, b1);
        }
        if (s < count) step(s, a1, b1, a0, b0);
    }
    // What the tile's rows have is on its way during the last products: behind the first store it would be waited for row
    // by row.
    int64_t column_hit[kBM];
    float row_lse[kBM], row_weight[kBM];
    if constexpr (F == kStats || F == kGrad) {
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t at = m0 + wm + 16 * i + li, m = at < rows ? at : rows - 1;
            column_hit[i] = (int64_t)g.target[m] - g.n0 - (c0 + wn + 4 * kBN * q);
            if (at >= rows) column_hit[i] = -1;
            if constexpr (F == kGrad) row_lse[i] = g.lse[m], row_weight[i] = g.weight[m] * g.grad_scale;
        }
    }
    if (count) multiply(part[1]);

    // acc[i][j][e] is row m0 + wm + 16 i + li, column c0 + wn + 4 kBN q + 4 j + e of channels in their own order; else column
    // 16 j + 4 q + e of the wave's, which an exchange between lanes 16 and 32 apart turns into 4 kBN neighbours a lane.
    constexpr int kOut = 4 * kBN;
    if constexpr (!kWide) {
#pragma unroll
        for (int i = 0; i < kBM; ++i) neighbours<kBN>(acc[i]);
    }
    const int64_t c = c0 + wn + (kWide || kBN == 4 ? kOut * q : 16 * (q & 1) + 8 * (q >> 1));
    if constexpr (KIND == kBytes) {
        if ((kAllSums ? g.all_sums && tile_n == 0 : g.sums != nullptr) && wave % WN == 0 && q == 0) {
#pragma unroll
            for (int i = 0; i < kBM; ++i) {
                const int64_t m = m0 + wm + 16 * i + li;
                if (m >= rows) continue;
                const float v[1] = {totals[i][0]};
                if constexpr (kAllSums) store_floats<1>(g.all_sums, g.sums_type, m, v, 1, false);
                else g.sums[((int64_t)split * tiles_n + tile_n) * rows + m] = v[0];
            }
        }
    }
    if constexpr (F == kStore) {
        if (c >= g.n) return;
        const float factor = g.factor ? *g.factor : 1.f;
        float bias[kOut];
#pragma unroll
        for (int e = 0; e < kOut; ++e)
            bias[e] = kWide && g.bias && c + e < g.n ? load_float(g.bias, g.bias_type, c + e) : 0.f;
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t m = m0 + wm + 16 * i + li;
            if (m >= rows) continue;
            float v[kOut];
#pragma unroll
            for (int e = 0; e < kOut; ++e) v[e] = acc[i][e >> 2][e & 3] * factor + bias[e];
            store_floats<kOut>(g.out, g.out_type, m * g.out_stride + c, v, g.n - c, true);
        }
    } else if constexpr (F == kSum) {
        float* out = g.part + split * rows * g.part_stride;
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t m = m0 + wm + 16 * i + li;
            if (m >= rows) continue;
            // part_stride and part are multiples of 4 floats: whole vectors, the last one into the padding
#pragma unroll
            for (int j = 0; j < kBN; ++j) {
                if (c + 4 * j >= g.n) continue;
                float4v* p = (float4v*)(out + m * g.part_stride + c + 4 * j);
                *p = g.accumulate ? *p + acc[i][j] : acc[i][j];
            }
        }
    } else if constexpr (F == kStats) {
        // 16,384 tokens by 32,128 rows of 1024: 1011 us, a little less than with the logits written (1028)
        product_landed();
        __syncthreads();  // the staged operands have been read by all
        float2* shared = (float2*)a0;  // [WN][TM]
        const bool whole = c0 + TN <= g.n;  // of all lanes
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t m = m0 + wm + 16 * i + li;
            float x[kOut];
#pragma unroll
            for (int e = 0; e < kOut; ++e) x[e] = acc[i][e >> 2][e & 3];
            // what does not count is as far down as it goes
            const float down = g.to_log2 < 0.f ? INFINITY : -INFINITY;
            if (!whole) {
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (c + e >= g.n) x[e] = down;
            }
            const int64_t hit = column_hit[i];
            if (hit >= 0 && hit < kOut && c + hit < g.n) {
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (e == hit) g.of_target[m] = x[e] * g.to_log2, x[e] = down;
            }
            float top = x[0];
            if (g.to_log2 < 0.f) {
#pragma unroll
                for (int e = 1; e < kOut; ++e) top = fminf(top, x[e]);
            } else {
#pragma unroll
                for (int e = 1; e < kOut; ++e) top = fmaxf(top, x[e]);
            }
            top *= g.to_log2;
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < kOut; ++e) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], g.to_log2, -from));
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (q == 0) shared[(wave % WN) * TM + wm + 16 * i + li] = make_float2(top, sum);
        }
        __syncthreads();
        for (int r = threadIdx.x; r < TM; r += 64 * kWaves) {
            if (m0 + r >= rows) continue;
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < WN; ++w) top = fmaxf(top, shared[w * TM + r].x);
            const float from = top == -INFINITY ? 0.f : top;
#pragma unroll
            for (int w = 0; w < WN; ++w) {
                const float2 o = shared[w * TM + r];
                sum += o.y * __builtin_amdgcn_exp2f(o.x - from);
            }
            g.stats[tile_n * g.stats_stride + m0 + r] = make_float2(top, sum);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kBM; ++i) {
            const int64_t m = m0 + wm + 16 * i + li;
            if (m >= rows) continue;
            const int64_t hit = column_hit[i];
            float d[kOut];
#pragma unroll
            for (int e = 0; e < kOut; ++e)
                d[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][e >> 2][e & 3], g.to_log2, -row_lse[i])) * row_weight[i];
            if (hit >= 0 && hit < kOut) {
                const float at = g.at_target[m] * g.grad_scale;
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (e == hit) d[e] = at;
            }
            if (c0 + TN > g.n) {
#pragma unroll
                for (int e = 0; e < kOut; ++e)
                    if (c + e >= g.n) d[e] = 0.f;
            }
            if constexpr (KIND == kPlanes) {
                Vec<uint16_t, kOut> p[3];
#pragma unroll
                for (int e = 0; e < kOut; ++e) {
                    uint16_t s[3];
                    split_f32(d[e], s);
                    p[0].e[e] = s[0], p[1].e[e] = s[1], p[2].e[e] = s[2];
                }
#pragma unroll
                for (int t = 0; t < 3; ++t)
                    store_vec<uint16_t, kOut>((uint16_t*)g.grad + t * g.grad_plane + m * g.grad_stride + c, p[t]);
            } else {
                Vec<E, kOut> p;  // rounded as matrix instructions need it: what is lost would double both products of G
#pragma unroll
                for (int e = 0; e < kOut; ++e) p.e[e] = (E)d[e];
                store_vec<E, kOut>((E*)g.grad + m * g.grad_stride + c, p);
            }
        }
    }
}

// Workgroups for at most g.m rows.
template <typename E, Layout LA, Layout LB, Finish F, Kind KIND, int TM, int TN, int WM, int WN>
hipError_t product_launch(const ProductArgs& g, hipStream_t s) {
    const int64_t tiles = cover_of(g.m, TM) * cover_of(g.n, TN);
    // splits shrink as rows grow: at most `jobs` tiles, or one part of each
    const int64_t grid = F == kSum && tiles < g.jobs ? g.jobs : tiles;
    (void)hipGetLastError();
    if (tiles)
        hipLaunchKernelGGL((k_product<E, LA, LB, TM, TN, WM, WN, F, KIND>), dim3((uint32_t)grid), dim3(64 * WM * WN), 0,
                           s, g);
    return hipGetLastError();
}

template <typename E, Layout LA, Layout LB, Finish F, Kind KIND = kPlain>
hipError_t product_tiles(const ProductArgs& g, Tile tile, hipStream_t s) {
    switch (tile) {
        case kT64: return product_launch<E, LA, LB, F, KIND, 64, 64, 2, 2>(g, s);
        case kT128: return product_launch<E, LA, LB, F, KIND, 128, 128, 2, 4>(g, s);
        default:
            if constexpr (KIND == kBytes || sizeof(E) == 4) return hipErrorInvalidValue;
            else return product_launch<E, LA, LB, F, KIND, 256, 256, 2, 4>(g, s);
    }
}

template <Layout LA, Layout LB>
hipError_t product_any(const ProductArgs& g, int element, Tile tile, Finish finish, hipStream_t s) {
    if (element == WARP_F16)
        return finish == kSum ? product_tiles<_Float16, LA, LB, kSum>(g, tile, s)
                              : product_tiles<_Float16, LA, LB, kStore>(g, tile, s);
    return finish == kSum ? product_tiles<__bf16, LA, LB, kSum>(g, tile, s)
                          : product_tiles<__bf16, LA, LB, kStore>(g, tile, s);
}

#endif  // __HIPCC__

}  // namespace warp
