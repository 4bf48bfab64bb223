// What goes into the products of product.h and what comes out: operands made ready, parts of sums joined.
#pragma once

#include "product.h"

namespace warp {

// Space in the caller's scratch memory, 256-byte aligned; places are counted first and have addresses once there is a base.
struct Space {
    uint8_t* base = nullptr;
    int64_t used = 0;
    template <typename T>
    T* take(int64_t n) {
        const int64_t at = used;
        used += (n * (int64_t)sizeof(T) + 255) / 256 * 256;
        return base ? (T*)(base + at) : nullptr;
    }
};

// A matrix as the products read it.
struct Operand {
    const void* p = nullptr;
    int64_t stride = 0, plane = 0;
};

inline int planes_of(int32_t dtype) { return dtype == WARP_F32 ? 3 : 1; }
inline int terms_of(int32_t dtype) { return dtype == WARP_F32 ? 6 : 1; }
inline int element_of(int32_t dtype) { return dtype == WARP_F16 ? WARP_F16 : WARP_BF16; }
__host__ __device__ inline int64_t packed_width(int64_t cols) { return cover_of(cols, 64) * 64; }
inline int64_t packed_elements(int64_t rows, int64_t cols, int32_t dtype) {
    return planes_of(dtype) * rows * packed_width(cols);
}

// Whether the products can read a matrix where it lies: 16-bit elements, whole 16-byte pieces.
inline bool direct(const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype) {
    return dtype != WARP_F32 && (uintptr_t)p % 16 == 0 && cols % 8 == 0 && (rows <= 1 || (stride % 8 == 0 && stride <= 1 << 22));
}

// The same for float32 products without planes.
inline bool direct_f32(const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype) {
    return dtype == WARP_F32 && (uintptr_t)p % 16 == 0 && cols % 4 == 0 && (rows <= 1 || (stride % 4 == 0 && stride <= 1 << 21));
}
// Tiles of 128 load half as much, where there are enough of them.
inline Tile tile_f32(int64_t m, int64_t n) {
    return m <= 64 || cover_of(m, 128) * cover_of(n, 128) < 256 ? kT64 : kT128;
}

#ifdef __HIPCC__
// Eight elements of an operand.
template <typename E, int PLANES>
__device__ __forceinline__ void store_packed(uint16_t* out, int64_t plane, int64_t at, const float (&v)[8]) {
    if constexpr (PLANES == 3) {
        Vec<uint16_t, 8> p[3];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint16_t s[3];
            split_f32(v[e], s);
            p[0].e[e] = s[0], p[1].e[e] = s[1], p[2].e[e] = s[2];
        }
#pragma unroll
        for (int t = 0; t < 3; ++t) store_vec<uint16_t, 8>(out + t * plane + at, p[t]);
    } else {
        Vec<E, 8> p;
#pragma unroll
        for (int e = 0; e < 8; ++e) p.e[e] = (E)v[e];
        store_vec<E, 8>((E*)out + at, p);
    }
}
#endif

// Rows (those of `list`, if given, as many as *now) that become an operand of their own: padded with zeros to a multiple of
// 64 columns, float32 in planes. Two matrices in one launch; none where rows is 0.
struct PackRows {
    const void* x = nullptr;
    int64_t stride = 0, rows = 0, cols = 0;
    const int32_t *list = nullptr, *now = nullptr;
    uint16_t* out = nullptr;
    bool whole = false;  // float32 as it is
};
hipError_t pack_rows(const PackRows& a, const PackRows& b, int32_t dtype, hipStream_t s);
// The same of 8-bit rows: q * scale, rounded to `dtype` for its products (as ByteStage does).
hipError_t unpack_int8(const int8_t* q, int64_t q_stride, const float* scale, int64_t rows, int64_t cols, int32_t dtype,
                       uint16_t* out, hipStream_t s, bool whole = false);

// x as an operand: where it lies, or in `room`, for which `job` is then what has to be packed. `whole`: float32 without planes.
inline Operand operand_of(const void* x, int64_t stride, int64_t rows, int64_t cols, int32_t dtype, uint16_t* room,
                          PackRows* job, bool whole = false) {
    if (whole ? direct_f32(x, stride, rows, cols, dtype) : direct(x, stride, rows, cols, dtype)) return {x, rows <= 1 ? cols : stride, 0};
    *job = {x, stride, rows, cols, nullptr, nullptr, room, whole};
    return {room, packed_width(cols), rows * packed_width(cols)};
}

// out[r][c] = bias[c] + factor * sum of the parts of row `place[r]` (of r, without places; zero where that is negative, NaN where
// it is below -1): what kSum products of these sizes left.
struct Join {
    const float* part;
    int64_t part_stride;
    int64_t m, n, k;
    const int32_t *m_now, *k_now;
    int32_t terms, splits, jobs, tile;
    const float* factor;
    const int32_t* place;
    int64_t rows;
    void* out;
    int64_t out_stride;
    int32_t out_type;
    const void* bias;
    int32_t bias_type;
    int32_t parts = 0;  // where they were made by product_few
};
hipError_t join_parts(const Join& j, hipStream_t s);

// Products of few rows (product_few): whether those along K are made of 32 columns a wave or 16, and in how many parts those across K
// are made, to have 512 workgroups.
constexpr int kFewRows = 32;  // most that one load of the other operand serves
inline bool few_wide(int64_t n) { return n > 8192; }
inline int few_parts(int64_t m, int64_t n, int64_t k, int32_t dtype) {
    if (!m) return 1;
    const bool f32 = dtype == WARP_F32;
    const int64_t tiles = cover_of(m, m <= 16 ? 16 : 32) * cover_of(n, f32 ? 64 : 128);
    const int64_t most = cover_of(k, f32 ? 128 : 256), parts = 512 / tiles;
    return (int)(parts < 1 ? 1 : parts < most ? parts : most);
}

// float32 products over at most kOuter k, both operands across K: in planes, or A a float32 and B 8-bit rows with scales.
constexpr int kOuter = 64;
struct OuterArgs {
    const void *a, *b;
    int64_t a_stride, a_plane, b_stride, b_plane;
    const float* b_scale;
    int64_t m, n, k;
    const int32_t* k_now;
    const float* factor;
    float* out;
    int64_t out_stride;
    float* sums;  // of A's columns, or null
};
hipError_t product_outer(const OuterArgs& g, hipStream_t s);

// Floats that the parts of a kSum product need, whatever the present counts are.
inline int64_t part_floats(int64_t m, int64_t n, int64_t k, int terms, Tile tile, int splits, int jobs) {
    const int64_t t = tile_size(tile), stride = cover_of(n, 4) * 4;
    const int64_t most = product_splits(1, 1, product_steps(k, terms), (int)t, splits, jobs);
    // with fewer rows now there are more parts, of which about `jobs` tiles are at work
    const int64_t whole = m * stride, parts = most * whole, bounded = jobs * t * cover_of(stride, cover_of(n, t));
    const int64_t split = parts < bounded ? parts : bounded;
    return whole > split ? whole : split;
}

// out = sums of x's columns, in an order that the sizes fix; `room` for column_room floats.
inline int64_t column_chunks(int64_t rows) { return rows < 64 ? 1 : rows / 64 < 256 ? rows / 64 : 256; }
inline int64_t column_room(int64_t rows, int64_t cols) { return column_chunks(rows) * cols; }
hipError_t join_columns(const float* room, int64_t chunks, int64_t cols, void* out, int32_t out_type, hipStream_t s);
hipError_t column_sums(const void* x, int64_t stride, int64_t rows, int64_t cols, int32_t dtype, float* room, void* out,
                       int32_t out_type, hipStream_t s);

}  // namespace warp
