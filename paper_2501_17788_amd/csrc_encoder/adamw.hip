// One AdamW step over many tensors, with the moments in 32 or in 8 bits:
//   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// 8-bit moments. A block of 256 elements shares a scale S, its largest magnitude, and an element keeps a code c
// of m = S sign(c) (c / 127)^2 or v = S (c / 255)^4: neighbouring codes are 2 / c (m) and 4 / c (v) apart
// relative to their value, so values near the block's largest are kept to 1%, and v reaches down to 2e-10 of it.
// A code counts the cutoffs that the magnitude over S reaches. The new m and v are computed without fused
// multiply-adds, so that every step's codes follow from the formulas' 32-bit operations alone.
//
// A moment rests on its code until one step moves it by half the way to the next: 1 / c of an m, 2 / c of a v. A step
// without a gradient takes 1 - b1 of an m, so with b1 = 0.9 it rests up to code 9, and 1 - b2 of a v, so with b2 = 0.999
// it rests at every code, both while the block's largest stays. Growing gradients with noise are followed; constant ones
// that double are not, and falling ones are not. An element whose gradient vanishes goes on moving: with noise by 0.4,
// 3.3 and 72 lr in 2,400 steps after gradients of 1, 0.1 and 0.005 of its neighbours', by 11 and 108 lr after constant
// ones of 1 and 0.1; a gradient that has turned below 0.5% of the block's largest does not turn its m.
//
// Bound by memory: 96M parameters in 48 tensors, moments in 32 bits 441 us in fp32 (6.1 TB/s), moments in 8 bits 284 us
// in fp32 (5.4 TB/s) and 164 to 204 us in bfloat16 (5.8 to 4.7 TB/s, by the card). There the arithmetic, some 70
// operations an element, takes nearly as long: with the exact square root and division in the step it was the bound (240
// us).
#include <cmath>

#include "encoder.h"

namespace warp {

namespace {

constexpr int kMaxTensors = 104;    // of one launch: their records travel in the kernel's arguments (at most 4 KB)
constexpr int kBlock = 256;         // elements that share a scale; the kernel's threads too
constexpr int kPer = 8;             // elements of a thread
constexpr int kChunk = 256 * kPer;  // elements of a workgroup

struct StepArgs {
    warp_adamw_tensor t[kMaxTensors];
    uint32_t first[kMaxTensors + 1];  // chunks before each tensor's; first[n] = all
    int32_t n;
    void* m;
    void* v;
    float* m_scale;
    float* v_scale;
    const float* grad_scale;
    float b1, c1, b2, c2;   // c = 1 - b
    float decay, rate;      // 1 - lr wd, lr / (1 - b1^t)
    float root, eps;        // 1 / sqrt(1 - b2^t)
};

static_assert(sizeof(StepArgs) <= 4096, "the arguments of a launch");

// V elements of which `left` are there. NT: not kept in the caches. Gradients are not read again, and moments a step
// later; the parameters are, by the next forward pass. 96M fp32 parameters and gradients, 32-bit moments: 525 us
// without, 467 us with (on one card; 441 us on another).
template <typename T, int V, bool NT = true>
__device__ __forceinline__ void load_some(const T* p, int64_t left, float (&out)[V]) {
    if (left >= V) {
        const auto v = NT ? stream_in<T, V>(p) : load_vec<T, V>(p);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = (float)v.e[i];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = i < left ? (float)p[i] : 0.f;
    }
}
template <typename T, int V, bool NT = true>
__device__ __forceinline__ void store_some(T* p, int64_t left, const float (&in)[V]) {
    if (left >= V) {
        Vec<T, V> v;
#pragma unroll
        for (int i = 0; i < V; ++i) v.e[i] = (T)in[i];
        if (NT) stream_out<T, V>(p, v);
        else store_vec<T, V>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < left) p[i] = (T)in[i];
    }
}

// New moments of one element, from separately rounded products and sums.
__device__ __forceinline__ void moments(const StepArgs& a, float g, float& m, float& v) {
#pragma clang fp contract(off)
    m = m * a.b1 + g * a.c1;
    v = v * a.b2 + (g * g) * a.c2;
}
constexpr int kSubnormal = 0x80;  // a positive one, of the classes of v_cmp_class_f32
// The parameter after its step. The 8-bit kernel, which is bound by its arithmetic, takes the approximate square root
// and reciprocal (within 1 ulp each), except for a v below 2^-126, which that root takes for zero.
template <bool FAST>
__device__ __forceinline__ float moved(const StepArgs& a, float p, float m, float v) {
    if (FAST)
        return p * a.decay - a.rate * m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) * a.root + a.eps);
    return p * a.decay - a.rate * m / (sqrtf(v) * a.root + a.eps);
}

__device__ __forceinline__ float m_value(float c, float s) {
#pragma clang fp contract(off)
    const float t = c * (1.0f / 127.0f);
    return t * fabsf(t) * s;
}
__device__ __forceinline__ float v_value(float c, float s) {
#pragma clang fp contract(off)
    const float t = c * (1.0f / 255.0f);
    const float u = t * t;
    return (u * u) * s;
}
// The number of cutoffs that x = magnitude / S reaches. The approximate root is within 1e-4 codes, so rounding
// it a little down gives that number or one less, and one comparison with the next cutoff settles which.
__device__ __forceinline__ float m_code(float x) {
#pragma clang fp contract(off)
    const float c = floorf(__builtin_fmaf(__builtin_amdgcn_sqrtf(x), 127.0f, 0.499f));
    const float t = (c + 0.5f) * (1.0f / 127.0f);
    return c + (x >= t * t ? 1.0f : 0.0f);
}
__device__ __forceinline__ float v_code(float x) {
#pragma clang fp contract(off)
    const float c = floorf(__builtin_fmaf(__builtin_amdgcn_sqrtf(__builtin_amdgcn_sqrtf(x)), 255.0f, 0.499f));
    const float t = (c + 0.5f) * (1.0f / 255.0f);
    const float u = t * t;
    return c + (x >= u * u ? 1.0f : 0.0f);
}
// The low bytes of four whole numbers' two's complements: after the addition of 1.5 * 2^23 they are the sum's low bits.
__device__ __forceinline__ uint32_t four_bytes(const float* c) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = as_u(c[i] + 12582912.0f);
    return __builtin_amdgcn_perm(u[3], u[2], 0x04000c0cu) | __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u);
}

// Largest over the 32 lanes of a half wave.
__device__ __forceinline__ uint32_t half_max(uint32_t x) {
    x = quarter_max(x);
    return max(x, (uint32_t)__shfl_xor((int)x, 16));
}

// A workgroup takes one chunk of one tensor.
template <typename T, typename G, int BITS>
__global__ __launch_bounds__(256) void k_adamw(StepArgs a) {
    int lo = 0, hi = a.n;  // the last tensor whose chunks start at or before this one
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const int64_t base = (int64_t)(blockIdx.x - a.first[lo]) * kChunk;
    const int64_t n = a.t[lo].n, moment = a.t[lo].moment;
    T* param = (T*)a.t[lo].param;
    const G* grad = (const G*)a.t[lo].grad;
    const float gs = a.grad_scale ? *a.grad_scale : 1.0f;
    const int64_t padded = (n + kBlock - 1) / kBlock * kBlock;
    if (BITS == 32) {
        constexpr int V = 4, N = kPer / V;
        float p[N][V], g[N][V], m[N][V], v[N][V];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int64_t i = base + (j * 256 + threadIdx.x) * V;
            if (i < n) {
                load_some<T, V, false>(param + i, n - i, p[j]);
                load_some<G, V>(grad + i, n - i, g[j]);
                load_some<float, V>((const float*)a.m + moment + i, V, m[j]);  // whole: padded to 256
                load_some<float, V>((const float*)a.v + moment + i, V, v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int64_t i = base + (j * 256 + threadIdx.x) * V;
            if (i >= n) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                moments(a, g[j][e] * gs, m[j][e], v[j][e]);
                p[j][e] = moved<false>(a, p[j][e], m[j][e], v[j][e]);
            }
            store_some<T, V, false>(param + i, n - i, p[j]);
            store_some<float, V>((float*)a.m + moment + i, n - i, m[j]);
            store_some<float, V>((float*)a.v + moment + i, n - i, v[j]);
        }
    } else {
        constexpr int V = kPer;  // a block is 32 lanes of 8 elements
        const int64_t i = base + threadIdx.x * V;
        if (i >= padded) return;  // half waves at a time
        const int64_t s = (moment + i) / kBlock;
        float p[V], g[V], m[V], v[V];
        load_some<T, V, false>(param + i, n - i, p);
        load_some<G, V>(grad + i, n - i, g);
        uint32_t* cm = (uint32_t*)((int8_t*)a.m + moment + i);
        uint32_t* cv = (uint32_t*)((uint8_t*)a.v + moment + i);
        const auto om = stream_in<uint32_t, 2>(cm), ov = stream_in<uint32_t, 2>(cv);
        const float sm = a.m_scale[s], sv = a.v_scale[s];
        uint32_t top_m = 0, top_v = 0;
        bool low = false;  // some v is above zero and below 2^-126
#pragma unroll
        for (int e = 0; e < V; ++e) {
            m[e] = m_value((float)(int8_t)(om.e[e / 4] >> 8 * (e & 3)), sm);
            v[e] = v_value((float)(uint8_t)(ov.e[e / 4] >> 8 * (e & 3)), sv);
            moments(a, g[e] * gs, m[e], v[e]);
            p[e] = moved<true>(a, p[e], m[e], v[e]);
            top_m = max(top_m, as_u(m[e]) & 0x7fffffffu);
            top_v = max(top_v, as_u(v[e]));  // no number here is negative
            low |= __builtin_amdgcn_classf(v[e], kSubnormal);
        }
        if (low) {  // seldom: the parameters are read again rather than kept
            float was[V];
            load_some<T, V, false>(param + i, n - i, was);
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (__builtin_amdgcn_classf(v[e], kSubnormal)) p[e] = moved<false>(a, was[e], m[e], v[e]);
        }
        store_some<T, V, false>(param + i, n - i, p);
        const float nm = as_f(max(half_max(top_m), 0x00800000u));
        const float nv = as_f(max(half_max(top_v) & 0x7fffffffu, 0x00800000u));
        const float im = 1.0f / nm, iv = 1.0f / nv;
#pragma unroll
        for (int e = 0; e < V; ++e) {
            m[e] = copysignf(m_code(fabsf(m[e]) * im), m[e]);
            v[e] = fmaxf(v_code(v[e] * iv), v[e] > 0.f ? 1.0f : 0.0f);
        }
        stream_out<uint32_t, 2>(cm, {four_bytes(m), four_bytes(m + 4)});
        stream_out<uint32_t, 2>(cv, {four_bytes(v), four_bytes(v + 4)});
        if ((threadIdx.x & 31) == 0) a.m_scale[s] = nm, a.v_scale[s] = nv;
    }
}

__global__ __launch_bounds__(256) void k_moments(const int8_t* m, const float* m_scale, const uint8_t* v,
                                                 const float* v_scale, int64_t n, float* out_m, float* out_v) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += (int64_t)gridDim.x * 1024) {
        const auto cm = load_vec<int8_t, 4>(m + i);
        const auto cv = load_vec<uint8_t, 4>(v + i);
        const float sm = m_scale[i / kBlock], sv = v_scale[i / kBlock];
        Vec<float, 4> rm, rv;
#pragma unroll
        for (int e = 0; e < 4; ++e) rm.e[e] = m_value((float)cm.e[e], sm), rv.e[e] = v_value((float)cv.e[e], sv);
        store_vec<float, 4>(out_m + i, rm);
        store_vec<float, 4>(out_v + i, rv);
    }
}

template <typename T, typename G>
void step_launch(const StepArgs& a, int32_t bits, hipStream_t s) {
    const dim3 grid(a.first[a.n]);
    if (bits == 32) hipLaunchKernelGGL((k_adamw<T, G, 32>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_adamw<T, G, 8>), grid, dim3(256), 0, s, a);
}
template <typename T>
void step_grads(const StepArgs& a, int32_t grad_dtype, int32_t bits, hipStream_t s) {
    if (grad_dtype == WARP_F32) step_launch<T, float>(a, bits, s);
    else if (grad_dtype == WARP_F16) step_launch<T, _Float16>(a, bits, s);
    else step_launch<T, __bf16>(a, bits, s);
}
int step_any(const StepArgs& a, int32_t dtype, int32_t grad_dtype, int32_t bits, hipStream_t s) {
    if (dtype == WARP_F32) WARP_LAUNCH(step_grads<float>(a, grad_dtype, bits, s));
    else if (dtype == WARP_F16) WARP_LAUNCH(step_grads<_Float16>(a, grad_dtype, bits, s));
    else WARP_LAUNCH(step_grads<__bf16>(a, grad_dtype, bits, s));
    return WARP_OK;
}

}  // namespace

}  // namespace warp

using namespace warp;

extern "C" {

int warp_adamw_step(const warp_adamw_tensor* tensors, int32_t n_tensors, int32_t dtype, int32_t grad_dtype,
                    int32_t bits, void* m, float* m_scale, void* v, float* v_scale, double lr, double beta1,
                    double beta2, double eps, double weight_decay, int64_t step, const float* grad_scale,
                    void* hip_stream) {
    const char* what = "adamw step";
    if (n_tensors < 0 || (n_tensors && !tensors)) return fail(WARP_EINVAL, "%s: bad tensor list", what);
    if (!dtype_ok(dtype) || !dtype_ok(grad_dtype)) return fail(WARP_EINVAL, "%s: unknown dtype", what);
    if (bits != 8 && bits != 32) return fail(WARP_EINVAL, "%s: bits must be 8 or 32 (got %d)", what, bits);
    if (!(beta1 >= 0 && beta1 < 1 && beta2 >= 0 && beta2 < 1))
        return fail(WARP_EINVAL, "%s: betas must be in [0, 1) (got %g, %g)", what, beta1, beta2);
    if (!(lr >= 0 && eps >= 0 && weight_decay >= 0) || !std::isfinite(lr) || !std::isfinite(eps) ||
        !std::isfinite(weight_decay))
        return fail(WARP_EINVAL, "%s: lr, eps and weight_decay must be finite and >= 0", what);
    if (step < 1) return fail(WARP_EINVAL, "%s: step must be >= 1 (got %lld)", what, (long long)step);
    bool some = false;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const warp_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n > (int64_t)1 << 32)
            return fail(WARP_EINVAL, "%s: tensor %d has %lld elements (0 to 2^32)", what, i, (long long)t.n);
        if (t.moment < 0 || t.moment % kBlock)
            return fail(WARP_EINVAL, "%s: the moments of tensor %d start at %lld, no multiple of 256", what, i,
                        (long long)t.moment);
        if (!t.n || !t.grad) continue;
        some = true;
        if (!t.param) return fail(WARP_EINVAL, "%s: tensor %d is null", what, i);
        if ((uintptr_t)t.param % dtype_bytes(dtype) || (uintptr_t)t.grad % dtype_bytes(grad_dtype))
            return fail(WARP_EINVAL, "%s: tensor %d is misaligned", what, i);
    }
    if (some && (!m || !v || (bits == 8 && (!m_scale || !v_scale))))
        return fail(WARP_EINVAL, "%s: null moments", what);
    if ((uintptr_t)m % 16 || (uintptr_t)v % 16 || (uintptr_t)m_scale % 4 || (uintptr_t)v_scale % 4 ||
        (uintptr_t)grad_scale % 4)
        return fail(WARP_EINVAL, "%s: misaligned moments or gradient scale", what);
    int rc = require_device();
    if (rc) return rc;
    StepArgs a;
    a.n = 0;
    a.first[0] = 0;
    a.m = m, a.v = v, a.m_scale = m_scale, a.v_scale = v_scale, a.grad_scale = grad_scale;
    a.b1 = (float)beta1, a.c1 = (float)(1 - beta1), a.b2 = (float)beta2, a.c2 = (float)(1 - beta2);
    a.decay = (float)(1 - lr * weight_decay);
    a.rate = (float)(lr / (1 - std::pow(beta1, (double)step)));
    a.root = (float)(1 / std::sqrt(1 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const warp_adamw_tensor& t = tensors[i];
        if (t.n && t.grad) {
            a.t[a.n] = t;
            a.first[a.n + 1] = a.first[a.n] + (uint32_t)((t.n + kChunk - 1) / kChunk);
            ++a.n;
        }
        // a launch is full with kMaxTensors tensors or 2^22 chunks (a tensor of 2^32 elements has 2^21)
        if (a.n && (a.n == kMaxTensors || a.first[a.n] >= 1u << 22 || i + 1 == n_tensors)) {
            rc = step_any(a, dtype, grad_dtype, bits, (hipStream_t)hip_stream);
            if (rc) return rc;
            a.n = 0;
        }
    }
    return WARP_OK;
}

int warp_adamw_moments(const int8_t* m, const float* m_scale, const uint8_t* v, const float* v_scale, int64_t n,
                       float* out_m, float* out_v, void* hip_stream) {
    const char* what = "adamw moments";
    if (n < 0 || n % kBlock) return fail(WARP_EINVAL, "%s: n must be a multiple of 256 (got %lld)", what, (long long)n);
    if (n && (!m || !m_scale || !v || !v_scale || !out_m || !out_v)) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)m % 16 || (uintptr_t)v % 16 || (uintptr_t)m_scale % 4 || (uintptr_t)v_scale % 4 ||
        (uintptr_t)out_m % 16 || (uintptr_t)out_v % 16)
        return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    const int rc = require_device();
    if (rc || !n) return rc;
    const int64_t need = (n + 1023) / 1024;
    const dim3 grid((uint32_t)(need < 1 << 20 ? need : 1 << 20));
    WARP_LAUNCH(hipLaunchKernelGGL(k_moments, grid, dim3(256), 0, (hipStream_t)hip_stream, m, m_scale, v, v_scale, n,
                                   out_m, out_v));
    return WARP_OK;
}

}  // extern "C"
