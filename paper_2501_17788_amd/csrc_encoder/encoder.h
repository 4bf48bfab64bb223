// Shared by the token encoder's kernels: element types, vectors of any element alignment, wave
// reductions, and the checks of their C entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "engine.h"  // fail, require_device
#include "warp.h"

namespace warp {

constexpr int kWave = 64;
constexpr int kInt8Pad = 128;  // int8 rows are padded with zeros to a multiple of this many columns

inline int dtype_bytes(int32_t dtype) { return dtype == WARP_F32 ? 4 : 2; }
inline bool dtype_ok(int32_t dtype) { return dtype == WARP_F32 || dtype == WARP_F16 || dtype == WARP_BF16; }

// The kernel that makes the int8 product of these sizes (k: padded), by its tiles. Visible for the tests, which have to
// reach each of them.
enum { kSplit16x16, kSplit32x16, kSplit32x32, kTile64, kTile128, kTile256 };
int linear_kernel(int64_t rows, int64_t n, int64_t k);

// A launch's own error, without taking one that an earlier call of the process left behind.
#define WARP_LAUNCH(...)                                                                             \
    do {                                                                                             \
        (void)hipGetLastError();                                                                     \
        __VA_ARGS__;                                                                                 \
        const hipError_t e_ = hipGetLastError();                                                     \
        if (e_ != hipSuccess) return fail(WARP_EDEVICE, "kernel launch failed: %s", hipGetErrorString(e_)); \
    } while (0)

// V elements at any address that suits one element: gfx950 loads and stores 16 bytes at once from
// any 4-byte (and, more slowly, any) address, so rows of odd width take the same instructions.
template <typename T, int V>
struct __attribute__((packed, aligned(sizeof(T)))) Vec {
    T e[V];
};

template <typename T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p) {
    return *reinterpret_cast<const Vec<T, V>*>(p);
}

template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& v) {
    *reinterpret_cast<Vec<T, V>*>(p) = v;
}

// The same for data that is not to stay in the caches.
template <int BYTES>
struct Raw {
    typedef uint32_t type __attribute__((ext_vector_type(BYTES / 4), aligned(1)));
};
template <>
struct Raw<2> {
    typedef uint16_t type __attribute__((aligned(1)));
};
template <typename T, int V>
__device__ __forceinline__ Vec<T, V> stream_in(const T* p) {
    return __builtin_bit_cast(Vec<T, V>, __builtin_nontemporal_load((const typename Raw<sizeof(T) * V>::type*)p));
}
template <typename T, int V>
__device__ __forceinline__ void stream_out(T* p, const Vec<T, V>& v) {
    typedef typename Raw<sizeof(T) * V>::type R;
    __builtin_nontemporal_store(__builtin_bit_cast(R, v), (R*)p);
}

// Sums over 16 lanes of a wave or all 64, returned to every lane: four steps inside 16 lanes, then
// those sums carried up to lane 63.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
constexpr int kDppXor1 = 0xB1, kDppXor2 = 0x4E, kDppHalfMirror = 0x141, kDppMirror = 0x140;
constexpr int kDppBcast15 = 0x142, kDppBcast31 = 0x143;

__device__ __forceinline__ float as_f(uint32_t u) { return __uint_as_float(u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __float_as_uint(f); }

__device__ __forceinline__ float quarter_sum(float x) {  // over 16 lanes
    x += as_f(dpp<kDppXor1, 0xf>(as_u(x)));
    x += as_f(dpp<kDppXor2, 0xf>(as_u(x)));
    x += as_f(dpp<kDppHalfMirror, 0xf>(as_u(x)));
    return x + as_f(dpp<kDppMirror, 0xf>(as_u(x)));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = quarter_sum(x);
    x += as_f(dpp<kDppBcast15, 0xa>(as_u(x)));
    x += as_f(dpp<kDppBcast31, 0xc>(as_u(x)));
    return as_f((uint32_t)__builtin_amdgcn_readlane((int)as_u(x), 63));
}

// The same for the largest of unsigned numbers (magnitudes of floats by their bits: a NaN is above
// infinity, which is above every number).
__device__ __forceinline__ uint32_t quarter_max(uint32_t x) {
    x = max(x, dpp<kDppXor1, 0xf>(x));
    x = max(x, dpp<kDppXor2, 0xf>(x));
    x = max(x, dpp<kDppHalfMirror, 0xf>(x));
    return max(x, dpp<kDppMirror, 0xf>(x));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    x = quarter_max(x);
    x = max(x, dpp<kDppBcast15, 0xa>(x));
    x = max(x, dpp<kDppBcast31, 0xc>(x));
    return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}

}  // namespace warp
