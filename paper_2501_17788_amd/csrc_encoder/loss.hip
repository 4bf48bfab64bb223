// Softmax cross entropy of token rows h over a vocabulary, the rows E of a table, without keeping the logits:
//   l_tv = scale * h_t . E_v,  lse_t = log(sum_v exp(l_tv)),  loss_t = lse_t - l_ty   (y: the row's target)
//   G_tv = dloss_t * (exp(l_tv - lse_t) - [v = y]),  dh_t = scale * sum_v G_tv E_v,  dE_v = scale * sum_t G_tv h_t
// Rows without a target (a negative one) are left out before any product: the others are copied next to each other, and
// the products take their number from the device. The forward pass is one product whose tiles end in the largest logit
// and the sum of exponentials of their rows. The backward pass goes through the vocabulary in pieces: a product makes the
// piece's logits again and writes G in the inputs' type, two more make the piece's rows of dE from it and add to dh.
// 8 T V d operations, where 6 T V d would do if the logits had been kept: bound by the matrix cores. 16,384 tokens, 32,128
// rows of 1024, bf16: forward 1.03 ms, G 1.11, dE 0.98, dh 0.95, all else 0.05; with a target in 15% of the rows 0.77 ms
// together. Five tokens: 16 us, of which the table's 49 MB take 13 (3.8 TB/s).
//
// Precision. The target's exponential is left out of the sums, S the rest relative to it: loss = log(1 + S) keeps its
// digits where a token is sure, and so does the target's G, which is expm1(-loss). G is rounded to the inputs' type, as
// matrix instructions need it (float32: three bfloat16 planes, which hold all of it); with what that loses as a second operand
// dE and dh would take twice as long. Before that it is divided by the largest |dloss|, so that rows that count alike round 1 - p and
// not a multiple of it, and scaled to use float16's range; both come back as a factor of the sums. Against 64 bits the gradients of
// 16,384 tokens in bf16 are off by 0.19% (15% of them: 0.18), of which their own rounding is 0.17.
#include "operands.h"

namespace warp {

namespace {

constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kHalfScale = 32768.f;  // |G| <= 1 before it
constexpr int64_t kPieceBytes = 512ll << 20;  // of G, and of a packed table
constexpr int64_t kStatsBytes = 256ll << 20;

// ---------------------------------------------------------------------------- rows that have a target

struct SelectArgs {
    const void* targets;
    bool wide;
    int64_t tokens, vocabulary;
    const float* dloss;
    float scale, grad_scale;
    int32_t *list, *place, *target;  // [now] token and target; [tokens] row, -1: none, -2: target outside the vocabulary
    int32_t* now;
    float* factor;  // of the sums: largest |dloss| * scale / grad_scale; written without tokens too, whose dloss may be null
    float* largest;
};

// Up to 2^17 tokens: a workgroup for each 1024, which counts the rows before its own by itself (16,384 tokens 8 us; by one
// workgroup 13). The last one has seen all of them.
constexpr int64_t kSelectWide = 1 << 17;
__global__ __launch_bounds__(1024) void k_select_wide(SelectArgs g) {
    constexpr int U = 8;
    __shared__ int32_t waves[2][16];
    __shared__ uint32_t tops[16];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t base = (int64_t)blockIdx.x * 1024;
    const bool last = blockIdx.x == gridDim.x - 1;
    auto target = [&](int64_t t) { return g.wide ? ((const int64_t*)g.targets)[t] : (int64_t)((const int32_t*)g.targets)[t]; };
    int32_t mine = 0;  // of this thread's tokens before the workgroup's
    uint32_t top = 0;
    for (int64_t t0 = tid; t0 < base; t0 += 1024 * U) {
        int64_t y[U];
        uint32_t d[U] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) y[u] = t0 + 1024 * u < base ? target(t0 + 1024 * u) : -1;
        if (last && g.dloss) {
#pragma unroll
            for (int u = 0; u < U; ++u) d[u] = t0 + 1024 * u < base ? as_u(g.dloss[t0 + 1024 * u]) & 0x7fffffffu : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = y[u] >= 0 && y[u] < g.vocabulary;
            mine += in;
            if (in && d[u] < 0x7f800000u) top = max(top, d[u]);
        }
    }
    const int64_t t = base + tid;
    const int64_t y = t < g.tokens ? target(t) : -1;
    const bool in = y >= 0 && y < g.vocabulary;
    if (last && in && g.dloss) {
        const uint32_t d = as_u(g.dloss[t]) & 0x7fffffffu;
        if (d < 0x7f800000u) top = max(top, d);
    }
    const unsigned long long all = __ballot(in);
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) mine += __shfl_xor(mine, s);
    top = wave_max(top);
    if (lane == 0) waves[0][w] = mine, waves[1][w] = (int32_t)__popcll(all), tops[w] = top;
    __syncthreads();
    int32_t first = 0, count = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        first += waves[0][i] + (i < w ? waves[1][i] : 0);
        count += waves[0][i] + waves[1][i];
    }
    const int32_t row = first + (int32_t)__popcll(all & ((1ull << lane) - 1));
    if (t < g.tokens) g.place[t] = in ? row : y < 0 ? -1 : -2;
    if (in) g.list[row] = (int32_t)t, g.target[row] = (int32_t)y;
    if (!last || tid) return;
    *g.now = count;
    if (!g.factor) return;
    for (int i = 0; i < 16; ++i) top = max(top, tops[i]);
    const float largest = top ? as_f(top) : 1.f;
    *g.largest = largest;
    *g.factor = largest * g.scale / g.grad_scale;
}

// One workgroup: turns of eight times 1024 neighbouring tokens, whose loads and stores are in one piece a wave.
__global__ __launch_bounds__(1024) void k_select(SelectArgs g) {
    constexpr int N = 8;
    __shared__ __attribute__((aligned(8))) int32_t waves[N][16];
    __shared__ uint32_t tops[16];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    int32_t count = 0;
    uint32_t top = 0;
    for (int64_t base = 0; base < g.tokens; base += 1024 * N) {
        const int64_t t0 = base + tid;
        int64_t y[N];
        uint32_t d[N] = {};
        auto at = [&](int e) { return t0 + 1024 * e < g.tokens ? t0 + 1024 * e : g.tokens - 1; };
        if (g.wide) {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = ((const int64_t*)g.targets)[at(e)];
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) y[e] = ((const int32_t*)g.targets)[at(e)];
        }
        if (g.dloss) {
#pragma unroll
            for (int e = 0; e < N; ++e) d[e] = as_u(g.dloss[at(e)]) & 0x7fffffffu;
        }
        int32_t rank[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const bool in = t0 + 1024 * e < g.tokens && y[e] >= 0 && y[e] < g.vocabulary;
            const unsigned long long all = __ballot(in);
            rank[e] = in ? (int32_t)__popcll(all & ((1ull << lane) - 1)) : -1;
            if (lane == 0) waves[e][w] = (int32_t)__popcll(all);
            if (in && d[e] < 0x7f800000u) top = max(top, d[e]);
        }
        __syncthreads();
        // the turn's tokens before each wave of each 1024: 128 numbers, two a lane
        const int2 n = ((const int2*)waves)[lane];
        const int32_t mine = n.x + n.y;
        int32_t x = mine;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const int32_t v = __shfl_up(x, s);
            if (lane >= s) x += v;
        }
        const int32_t before = x - mine + (w & 1 ? n.x : 0);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int32_t first = count + __builtin_amdgcn_readlane(before, 8 * e + (w >> 1));
            const int64_t t = t0 + 1024 * e;
            if (t >= g.tokens) continue;
            g.place[t] = rank[e] >= 0 ? first + rank[e] : y[e] < 0 ? -1 : -2;
            if (rank[e] >= 0) {
                g.list[first + rank[e]] = (int32_t)t;
                g.target[first + rank[e]] = (int32_t)y[e];
            }
        }
        count += __builtin_amdgcn_readlane(x, 63);
        __syncthreads();  // before the next turn's counts
    }
    top = wave_max(top);
    if (lane == 0) tops[w] = top;
    __syncthreads();
    if (tid) return;
    *g.now = count;
    if (!g.factor) return;
    for (int i = 0; i < 16; ++i) top = max(top, tops[i]);
    const float largest = top ? as_f(top) : 1.f;
    *g.largest = largest;
    *g.factor = largest * g.scale / g.grad_scale;
}

void select(const SelectArgs& g, hipStream_t s) {
    if (g.tokens && g.tokens <= kSelectWide)
        hipLaunchKernelGGL(k_select_wide, dim3((uint32_t)cover_of(g.tokens, 1024)), dim3(1024), 0, s, g);
    else
        hipLaunchKernelGGL(k_select, dim3(1), dim3(1024), 0, s, g);
}

// Up to 64 tokens, in one launch: a workgroup for each, whose waves all look at all targets; it packs its own row, and the
// first one writes what k_select and k_rows write.
constexpr int kFewTokens = 64;
struct FewArgs {
    SelectArgs select;
    const void* hidden;
    int64_t hidden_stride, cols, width, plane;
    uint16_t* packed;
    const float *loss, *lse;  // of the forward pass, with dloss
    float *lse2, *weight, *at_target;
};
template <typename T, int PLANES>
__global__ __launch_bounds__(256) void k_take_few(FewArgs f) {
    const SelectArgs& g = f.select;
    const int lane = threadIdx.x & 63, me = (int)blockIdx.x;
    int64_t y = -1;
    if (lane < g.tokens) y = g.wide ? ((const int64_t*)g.targets)[lane] : (int64_t)((const int32_t*)g.targets)[lane];
    const bool in = y >= 0 && y < g.vocabulary;
    const unsigned long long all = __ballot(in);
    const int rank = (int)__popcll(all & ((1ull << lane) - 1));
    if (me == 0 && threadIdx.x < 64) {
        if (lane < g.tokens) g.place[lane] = in ? rank : y < 0 ? -1 : -2;
        if (in) g.list[rank] = lane, g.target[rank] = (int32_t)y;
        if (lane == 0) *g.now = (int32_t)__popcll(all);
        if (g.dloss) {
            const float d = in ? g.dloss[lane] : 0.f;
            const uint32_t u = as_u(d) & 0x7fffffffu, top = wave_max(u < 0x7f800000u ? u : 0u);
            const float largest = top ? as_f(top) : 1.f;
            if (lane == 0) *g.largest = largest, *g.factor = largest * g.scale / g.grad_scale;
            if (in) {
                const float weight = d / largest;
                f.lse2[rank] = f.lse[lane] * kLog2E;
                f.weight[rank] = weight;
                f.at_target[rank] = weight * expm1f(-f.loss[lane]);
            }
        }
    }
    if (!(all >> me & 1)) return;
    const int64_t row = __builtin_amdgcn_readlane(rank, me);
    const T* x = (const T*)f.hidden + me * f.hidden_stride;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < f.width; c += 8 * 256) {
        float v[8];
        if (c + 8 <= f.cols) {
            const auto r = load_vec<T, 8>(x + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = (float)r.e[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = c + e < f.cols ? (float)x[c + e] : 0.f;
        }
        store_packed<T, PLANES>(f.packed, f.plane, row * f.width + c, v);
    }
}
void take_few(const FewArgs& f, int32_t dtype, hipStream_t s) {
    const dim3 grid((uint32_t)f.select.tokens), block(256);
    if (dtype == WARP_F32) hipLaunchKernelGGL((k_take_few<float, 3>), grid, block, 0, s, f);
    else if (dtype == WARP_F16) hipLaunchKernelGGL((k_take_few<_Float16, 1>), grid, block, 0, s, f);
    else hipLaunchKernelGGL((k_take_few<__bf16, 1>), grid, block, 0, s, f);
}

// ---------------------------------------------------------------------------- forward

struct JoinStatsArgs {
    const float2* stats;  // [tile][stride]
    int64_t stride;
    int tiles;
    bool first, last;
    float2* running;  // [row] of the pieces before
    const float* of_target;
    const int32_t* place;
    int64_t tokens;
    float *loss, *lse;
};

__device__ __forceinline__ float2 join_stats(float2 a, float2 b) {
    const float top = fmaxf(a.x, b.x), from = top == -INFINITY ? 0.f : top;
    return make_float2(top, a.y * __builtin_amdgcn_exp2f(a.x - from) + b.y * __builtin_amdgcn_exp2f(b.x - from));
}

// Lane k's and lane k ^ d's.
__device__ __forceinline__ float2 join_lanes(float2 s, int d) {
    return join_stats(s, make_float2(__shfl_xor(s.x, d), __shfl_xor(s.y, d)));
}

// The row's loss from the others' sum, s.y * 2^s.x, and the target's term, 2^y.
__device__ __forceinline__ void store_loss(const JoinStatsArgs& g, int64_t t, int32_t row, float2 s) {
    if (row < 0) {
        if (g.last) g.loss[t] = g.lse[t] = row == -1 ? 0.f : __builtin_nanf("");
        return;
    }
    if (!g.last) {
        g.running[row] = s;
        return;
    }
    const float y = g.of_target[row];
    if (y >= s.x) {
        const float others = s.y * __builtin_amdgcn_exp2f(s.x - y), loss = log1pf(others);
        g.loss[t] = loss;
        g.lse[t] = y * kLn2 + loss;
    } else {
        const float all = logf(s.y + __builtin_amdgcn_exp2f(y - s.x));
        g.loss[t] = (s.x - y) * kLn2 + all;
        g.lse[t] = s.x * kLn2 + all;
    }
}

// 64 tokens a workgroup, whose 16 waves share the tiles; of few tokens one, whose lanes share them too.
template <bool FEW>
__global__ __launch_bounds__(1024) void k_join_stats(JoinStatsArgs g) {
    __shared__ float2 joined[16][FEW ? 1 : kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t t = FEW ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kWave + lane;
    const int32_t row = t < g.tokens ? g.place[t] : -1;
    float2 s = make_float2(-INFINITY, 0.f);
    if (row >= 0) {
        if ((FEW ? threadIdx.x : w) == 0 && !g.first) s = g.running[row];
        constexpr int U = FEW ? 1 : 4;
        const int from = FEW ? (int)threadIdx.x : w, by = FEW ? 1024 : 16;
        for (int i = from; i < g.tiles; i += by * U) {
            float2 x[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                x[u] = i + by * u < g.tiles ? g.stats[(i + by * u) * g.stride + row] : make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int u = 0; u < U; ++u) s = join_stats(s, x[u]);
        }
    }
    if constexpr (FEW) {
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s = join_lanes(s, d);
        if (lane == 0) joined[w][0] = s;
    } else {
        joined[w][lane] = s;
    }
    __syncthreads();
    if ((FEW ? threadIdx.x : w) || t >= g.tokens) return;
    if (row >= 0)
        for (int i = 1; i < 16; ++i) s = join_stats(s, joined[i][FEW ? 0 : lane]);
    store_loss(g, t, row, s);
}

// ---------------------------------------------------------------------------- backward

struct RowArgs {
    const int32_t *list, *now;
    const float *dloss, *loss, *lse, *largest;
    float *lse2, *weight, *at_target;
};
__global__ __launch_bounds__(256) void k_rows(RowArgs g) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= *g.now) return;
    const int32_t t = g.list[i];
    const float weight = g.dloss[t] / *g.largest;
    g.lse2[i] = g.lse[t] * kLog2E;
    g.weight[i] = weight;
    g.at_target[i] = weight * expm1f(-g.loss[t]);
}

// ---------------------------------------------------------------------------- sizes and scratch

int check_sizes(const char* what, int64_t tokens, int64_t vocabulary, int32_t cols, int32_t dtype) {
    if (tokens < 0) return fail(WARP_EINVAL, "%s: tokens must be >= 0 (got %lld)", what, (long long)tokens);
    if (vocabulary < 1) return fail(WARP_EINVAL, "%s: vocabulary must be >= 1 (got %lld)", what, (long long)vocabulary);
    if (cols < 1) return fail(WARP_EINVAL, "%s: cols must be >= 1 (got %d)", what, cols);
    if (tokens > 1 << 22 || vocabulary > 1 << 25 || cols > 1 << 14)
        return fail(WARP_ENOTSUP, "%s: at most 2^22 tokens, a vocabulary of 2^25 and 2^14 columns (got %lld, %lld, %d)", what,
                    (long long)tokens, (long long)vocabulary, cols);
    if (!dtype_ok(dtype)) return fail(WARP_EINVAL, "%s: unknown dtype %d", what, dtype);
    return WARP_OK;
}
int check_matrix(const char* what, const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype) {
    if (rows && !p) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)p % dtype_bytes(dtype)) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    if (rows > 1 && stride < cols)
        return fail(WARP_EINVAL, "%s: a row stride of %lld is below %lld columns", what, (long long)stride, (long long)cols);
    return WARP_OK;
}
int check_scratch(const char* what, const void* scratch, int64_t bytes, int64_t need) {
    if (!scratch || bytes < need || (uintptr_t)scratch % 16)
        return fail(WARP_EINVAL, "%s: needs %lld bytes of scratch, 16-byte aligned (got %lld)", what, (long long)need,
                    (long long)(scratch ? bytes : 0));
    return WARP_OK;
}
int check_rows(const char* what, const void* targets, int32_t target_bytes, int64_t tokens, float scale, const void* loss,
               const void* lse) {
    if (target_bytes != 4 && target_bytes != 8)
        return fail(WARP_EINVAL, "%s: targets of 4 or 8 bytes (got %d)", what, target_bytes);
    if (tokens && (!targets || !loss || !lse)) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)targets % target_bytes || (uintptr_t)loss % 4 || (uintptr_t)lse % 4)
        return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    if (!(scale - scale == 0.f)) return fail(WARP_EINVAL, "%s: scale must be finite", what);
    return WARP_OK;
}

// Not zero, by which what lies outside the vocabulary, minus infinity, could not be multiplied: the smallest number has no
// effect on logits below 2^100 either.
float to_log2(float scale) { return scale ? scale * kLog2E : 1.17549435e-38f; }

// Columns of a piece of the vocabulary: a multiple of 256 (the last piece is shorter).
int64_t piece_of(int64_t vocabulary, int64_t bytes_a_column, int64_t most_bytes) {
    int64_t p = most_bytes / bytes_a_column / 256 * 256;
    const int64_t all = cover_of(vocabulary, 256) * 256;
    p = p < 256 ? 256 : p > all ? all : p;
    p = p > 1 << 20 ? 1 << 20 : p;
    // pieces of one size
    return cover_of(cover_of(vocabulary, cover_of(vocabulary, p)), 256) * 256;
}

struct Sizes {
    int64_t tokens, vocabulary, cols, width;
    int32_t dtype;
    int planes;
    bool few;    // rows: the table is read where it lies
    bool packs;  // the table
    bool whole;  // float32 without planes
};
Sizes sizes_of(int64_t tokens, const void* table, int64_t stride, int64_t vocabulary, int32_t cols, int32_t dtype, bool back) {
    // us with the table where it lies | by tiles. 16 tokens in 16 bits: forward, 5000 rows of 4096 18 | 40, 32,128 of 768 19 | 18,
    // 100,001 of 1023 (packed for tiles) 135 | 146, 200,001 of 65 40 | 58; backward 43 | 64, 46 | 44, 516 | 403, 79 | 87. 32 tokens in
    // float32, forward 49 | 210, 41 | 88, 167 | 364, 91 | 104, both passes 201 | 504, 194 | 261, 748 | 1275, 286 | 296.
    const bool few = dtype == WARP_F32 ? tokens <= kFewRows
                                       : tokens <= kFewRows / 2 && (vocabulary <= 16384 || (cols % 8 && !back));
    // More float32 tokens as they are | in planes, both passes: 64 tokens 164 | 300, 120 | 192, 1144 | 1346, 249 | 522, 272 | 336
    // (tables of 768 x 32,128, 128 x 100,001, 1023, 4096 x 5000, 65 x 200,001), 100 tokens 276 | 335, 200 | 234, 1494 | 1656, 294 | 510,
    // 394 | 448; the forward pass of 200 121 | 123, 88 | 90, 711 | 468, 153 | 213, 161 | 163, of 400 224 | 164, 143 | 134, 1120 | 724,
    // 236 | 259, 249 | 226.
    const bool whole = !few && dtype == WARP_F32 && tokens <= (vocabulary <= 16384 ? 256 : 128);
    const bool packs = !few && !(whole ? direct_f32 : direct)(table, stride, vocabulary, cols, dtype);
    return {tokens, vocabulary, cols, packed_width(cols), dtype, planes_of(dtype), few, packs, whole};
}

struct Forward {
    Space space;
    int64_t piece;
    Tile tile;
    uint16_t *hidden, *table;
    int32_t *list, *place, *target, *now;
    float2 *stats, *running;
    float* of_target;
    Forward(void* base, const Sizes& z) {
        space.base = (uint8_t*)base;
        const int64_t tokens = z.tokens > 0 ? z.tokens : 1;
        const int64_t by_table = z.packs ? piece_of(z.vocabulary, z.width * 2 * z.planes, kPieceBytes) : 1 << 30;
        tile = plan_product(tokens, z.vocabulary, product_steps(z.cols, terms_of(z.dtype)), false).tile;
        if (z.whole) tile = tile_f32(tokens, z.vocabulary);
        const int64_t columns = z.few ? 16 : tile_size(tile);
        const int64_t by_stats = piece_of(z.vocabulary, cover_of(tokens * 8, columns), kStatsBytes);
        piece = by_table < by_stats ? by_table : by_stats;
        hidden = space.take<uint16_t>(packed_elements(tokens, z.cols, z.dtype));
        table = space.take<uint16_t>(z.packs ? packed_elements(piece, z.cols, z.dtype) : 0);
        list = space.take<int32_t>(tokens), place = space.take<int32_t>(tokens), target = space.take<int32_t>(tokens);
        now = space.take<int32_t>(1);
        stats = space.take<float2>(cover_of(piece, columns) * tokens), running = space.take<float2>(tokens);
        of_target = space.take<float>(tokens);
    }
};

struct Backward {
    Space space;
    int64_t piece;
    Tile logits, dh, de;
    bool de_split, outer;
    int dh_parts;  // of few rows
    uint16_t *hidden, *table, *grad;
    int32_t *list, *place, *target, *now;
    float *largest, *factor, *lse2, *weight, *at_target, *dh_part, *de_part;
    Backward(void* base, const Sizes& z) {
        space.base = (uint8_t*)base;
        const int64_t tokens = z.tokens > 0 ? z.tokens : 1;
        const int terms = terms_of(z.dtype);
        piece = piece_of(z.vocabulary, tokens * 2 * z.planes, kPieceBytes);
        if (z.packs) {
            const int64_t by_table = piece_of(z.vocabulary, z.width * 2 * z.planes, kPieceBytes);
            piece = by_table < piece ? by_table : piece;
        }
        const int64_t cols = z.vocabulary < piece ? z.vocabulary : piece;
        logits = plan_product(tokens, cols, product_steps(z.cols, terms), false).tile;
        dh = plan_product(tokens, z.cols, product_steps(cols, terms), true).tile;
        const ProductPlan e = plan_product(cols, z.cols, product_steps(tokens, terms), true);
        if (z.whole) logits = tile_f32(tokens, cols), dh = tile_f32(tokens, z.cols);
        outer = z.dtype == WARP_F32 && tokens <= kFewRows;
        de = z.whole ? tile_f32(cols, z.cols) : e.tile, de_split = !outer && !z.whole && e.split;
        hidden = space.take<uint16_t>(packed_elements(tokens, z.cols, z.dtype));
        table = space.take<uint16_t>(z.packs ? packed_elements(piece, z.cols, z.dtype) : 0);
        grad = space.take<uint16_t>(z.planes * tokens * piece);
        list = space.take<int32_t>(tokens), place = space.take<int32_t>(tokens), target = space.take<int32_t>(tokens);
        now = space.take<int32_t>(1);
        largest = space.take<float>(1), factor = space.take<float>(1);
        lse2 = space.take<float>(tokens), weight = space.take<float>(tokens), at_target = space.take<float>(tokens);
        dh_parts = z.few ? few_parts(tokens, z.cols, cols, z.dtype) : 0;
        dh_part = space.take<float>(z.few ? dh_parts * tokens * cover_of(z.cols, 4) * 4
                                          : part_floats(tokens, z.cols, z.whole ? 2 * cols : cols, z.whole ? 1 : terms, dh, kMaxSplits, tile_jobs(dh)));
        de_part = space.take<float>(
            de_split ? part_floats(cols, z.cols, tokens, terms, de, kMaxSplits, tile_jobs(de)) : 0);
    }
};

#define WARP_STEP(...)                                                                                       \
    do {                                                                                                     \
        const hipError_t e_ = (__VA_ARGS__);                                                                 \
        if (e_ != hipSuccess) return fail(WARP_EDEVICE, "%s: launch failed: %s", what, hipGetErrorString(e_)); \
    } while (0)

}  // namespace

}  // namespace warp

using namespace warp;

extern "C" {

int warp_cross_entropy_scratch(int64_t tokens, int32_t cols, int32_t dtype, const void* table, int64_t table_stride,
                               int64_t vocabulary, int64_t* bytes, int64_t* backward_bytes) {
    const char* what = "cross entropy";
    if (const int rc = check_sizes(what, tokens, vocabulary, cols, dtype)) return rc;
    auto sizes = [&](bool back) { return sizes_of(tokens, table, table_stride, vocabulary, cols, dtype, back); };
    if (bytes) *bytes = Forward(nullptr, sizes(false)).space.used;
    if (backward_bytes) *backward_bytes = Backward(nullptr, sizes(true)).space.used;
    return WARP_OK;
}

int warp_cross_entropy(const void* hidden, int64_t hidden_stride, int64_t tokens, int32_t cols, int32_t dtype,
                       const void* table, int64_t table_stride, int64_t vocabulary, const void* targets,
                       int32_t target_bytes, float scale, float* loss, float* lse, void* scratch, int64_t scratch_bytes,
                       void* hip_stream) {
    const char* what = "cross entropy";
    int rc = check_sizes(what, tokens, vocabulary, cols, dtype);
    if (!rc) rc = check_matrix(what, hidden, hidden_stride, tokens, cols, dtype);
    if (!rc) rc = check_matrix(what, table, table_stride, vocabulary, cols, dtype);
    if (!rc) rc = check_rows(what, targets, target_bytes, tokens, scale, loss, lse);
    if (rc) return rc;
    const Sizes z = sizes_of(tokens, table, table_stride, vocabulary, cols, dtype, false);
    const Forward f(scratch, z);
    rc = check_scratch(what, scratch, scratch_bytes, f.space.used);
    if (!rc) rc = require_device();
    if (rc || !tokens) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    const SelectArgs sel{targets, target_bytes == 8, tokens, vocabulary, nullptr, scale, 1.f, f.list, f.place, f.target,
                         f.now, nullptr, nullptr};
    const bool few = tokens <= kFewTokens;
    if (z.few) {  // all rows, the others' results unused
    } else if (few && !z.whole) {
        WARP_LAUNCH(take_few({sel, hidden, hidden_stride, cols, z.width, tokens * z.width, f.hidden, nullptr, nullptr, nullptr,
                              nullptr, nullptr}, dtype, s));
    } else {
        WARP_LAUNCH(select(sel, s));
        WARP_STEP(pack_rows({hidden, hidden_stride, tokens, cols, f.list, f.now, f.hidden, z.whole}, {}, dtype, s));
    }
    for (int64_t v0 = 0; v0 < vocabulary; v0 += f.piece) {
        const int64_t n = vocabulary - v0 < f.piece ? vocabulary - v0 : f.piece;
        const void* rows = (const uint8_t*)table + v0 * table_stride * dtype_bytes(dtype);
        hipError_t e = hipSuccess;
        Operand t{rows, vocabulary <= 1 ? cols : table_stride, 0};
        if (z.packs) {
            e = pack_rows({rows, table_stride, n, cols, nullptr, nullptr, f.table, z.whole}, {}, dtype, s);
            t = {f.table, z.width, n * z.width};
        }
        WARP_STEP(e);
        ProductArgs g{};
        g.a = f.hidden, g.a_stride = z.width, g.a_plane = tokens * z.width;
        g.b = t.p, g.b_stride = t.stride, g.b_plane = t.plane;
        g.m = tokens, g.n = n, g.k = cols, g.m_now = f.now, g.terms = terms_of(dtype);
        g.to_log2 = to_log2(scale), g.n0 = v0, g.target = f.target;
        g.stats = f.stats, g.stats_stride = tokens, g.of_target = f.of_target;
        if (z.few) {
            g.a = hidden, g.a_stride = tokens <= 1 ? cols : hidden_stride, g.m_now = nullptr;
            g.targets = targets, g.wide = target_bytes == 8, g.vocabulary = vocabulary, g.place = f.place;
        }
        if (z.whole) g.terms = 1;
        if (z.few) WARP_STEP(product_few(g, dtype, false, kStats, 1, s));
        else if (z.whole) WARP_STEP(product_softmax(g, WARP_F32, false, f.tile, kStats, s));
        else WARP_STEP(product_softmax(g, element_of(dtype), false, f.tile, kStats, s));
        const int64_t columns = !z.few ? tile_size(f.tile) : few_wide(n) ? 32 : 16;
        const JoinStatsArgs j{f.stats, tokens, (int)cover_of(n, columns), v0 == 0, v0 + n == vocabulary, f.running,
                              f.of_target, f.place, tokens, loss, lse};
        if (few) WARP_LAUNCH(hipLaunchKernelGGL(k_join_stats<true>, dim3((uint32_t)tokens), dim3(1024), 0, s, j));
        else WARP_LAUNCH(hipLaunchKernelGGL(k_join_stats<false>, dim3((uint32_t)cover_of(tokens, kWave)), dim3(1024), 0, s, j));
    }
    return WARP_OK;
}

int warp_cross_entropy_backward(const float* dloss, const void* hidden, int64_t hidden_stride, int64_t tokens, int32_t cols,
                                int32_t dtype, const void* table, int64_t table_stride, int64_t vocabulary,
                                const void* targets, int32_t target_bytes, float scale, const float* loss,
                                const float* lse, void* dhidden, int64_t dhidden_stride, void* dtable,
                                int64_t dtable_stride, void* scratch, int64_t scratch_bytes, void* hip_stream) {
    const char* what = "cross entropy backward";
    int rc = check_sizes(what, tokens, vocabulary, cols, dtype);
    if (!rc) rc = check_matrix(what, hidden, hidden_stride, tokens, cols, dtype);
    if (!rc) rc = check_matrix(what, table, table_stride, vocabulary, cols, dtype);
    if (!rc) rc = check_rows(what, targets, target_bytes, tokens, scale, loss, lse);
    if (!rc && dhidden) rc = check_matrix(what, dhidden, dhidden_stride, tokens, cols, dtype);
    if (!rc && dtable) rc = check_matrix(what, dtable, dtable_stride, vocabulary, cols, dtype);
    if (rc) return rc;
    if (tokens && !dloss) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)dloss % 4) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    const Sizes z = sizes_of(tokens, table, table_stride, vocabulary, cols, dtype, true);
    const Backward w(scratch, z);
    rc = check_scratch(what, scratch, scratch_bytes, w.space.used);
    if (!rc) rc = require_device();
    if (rc || (!dhidden && !dtable)) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    const int element = z.whole ? (int)WARP_F32 : element_of(dtype), terms = z.whole ? 1 : terms_of(dtype);
    const float grad_scale = dtype == WARP_F16 ? kHalfScale : 1.f;
    const SelectArgs sel{targets, target_bytes == 8, tokens, vocabulary, dloss, scale, grad_scale, w.list, w.place, w.target,
                         w.now, w.factor, w.largest};
    const bool few = tokens <= kFewTokens && !z.whole;
    if (tokens && few) {
        WARP_LAUNCH(take_few({sel, hidden, hidden_stride, cols, z.width, tokens * z.width, w.hidden, loss, lse, w.lse2, w.weight,
                              w.at_target}, dtype, s));
    } else {
        WARP_LAUNCH(select(sel, s));
    }
    if (!few) {
        WARP_STEP(pack_rows({hidden, hidden_stride, tokens, cols, w.list, w.now, w.hidden, z.whole}, {}, dtype, s));
        const RowArgs r{w.list, w.now, dloss, loss, lse, w.largest, w.lse2, w.weight, w.at_target};
        WARP_LAUNCH(hipLaunchKernelGGL(k_rows, dim3((uint32_t)cover_of(tokens, 256)), dim3(256), 0, s, r));
    }
    const Operand h{w.hidden, z.width, (tokens ? tokens : 1) * z.width};
    const int64_t part_stride = cover_of(cols, 4) * 4;
    Join dh{w.dh_part, part_stride, tokens, cols, 0, w.now, nullptr, terms, kMaxSplits, tile_jobs(w.dh), tile_size(w.dh),
            w.factor, w.place, tokens, dhidden, dhidden_stride, dtype, nullptr, 0, w.dh_parts};
    for (int64_t v0 = 0; v0 < vocabulary; v0 += w.piece) {
        const int64_t n = vocabulary - v0 < w.piece ? vocabulary - v0 : w.piece;
        const void* rows = (const uint8_t*)table + v0 * table_stride * dtype_bytes(dtype);
        Operand t{rows, vocabulary <= 1 ? cols : table_stride, 0};
        if (z.packs) {
            WARP_STEP(pack_rows({rows, table_stride, n, cols, nullptr, nullptr, w.table, z.whole}, {}, dtype, s));
            t = {w.table, z.width, n * z.width};
        }
        ProductArgs g{};
        g.a = h.p, g.a_stride = h.stride, g.a_plane = h.plane;
        g.b = t.p, g.b_stride = t.stride, g.b_plane = t.plane;
        g.m = tokens, g.n = n, g.k = cols, g.m_now = w.now, g.terms = terms;
        g.to_log2 = to_log2(scale), g.n0 = v0, g.target = w.target;
        g.lse = w.lse2, g.weight = w.weight, g.at_target = w.at_target;
        g.grad = w.grad, g.grad_stride = w.piece, g.grad_plane = tokens * w.piece, g.grad_scale = grad_scale;
        if (z.few) WARP_STEP(product_few(g, dtype, z.planes == 3, kGrad, 1, s));
        else WARP_STEP(product_softmax(g, element, z.planes == 3, w.logits, kGrad, s));
        void* rows_out = dtable ? (uint8_t*)dtable + v0 * dtable_stride * dtype_bytes(dtype) : nullptr;
        if (dtable && w.outer) {
            WARP_STEP(product_outer({w.grad, h.p, w.piece, g.grad_plane, h.stride, h.plane, nullptr, n, cols, tokens, w.now,
                                     w.factor, (float*)rows_out, dtable_stride, nullptr}, s));
        } else if (dtable) {
            ProductArgs e{};
            e.a = w.grad, e.a_stride = w.piece, e.a_plane = g.grad_plane;
            e.b = h.p, e.b_stride = h.stride, e.b_plane = h.plane;
            e.m = n, e.n = cols, e.k = tokens, e.k_now = w.now, e.terms = terms;
            e.out = rows_out, e.out_stride = dtable_stride, e.out_type = dtype, e.factor = w.factor;
            e.splits = kMaxSplits, e.jobs = tile_jobs(w.de), e.part = w.de_part, e.part_stride = part_stride;
            WARP_STEP(product_across(e, element, w.de, w.de_split ? kSum : kStore, s));
            if (w.de_split)
                WARP_STEP(join_parts({w.de_part, part_stride, n, cols, tokens, nullptr, w.now, terms, kMaxSplits, e.jobs,
                                      tile_size(w.de), w.factor, nullptr, n, e.out, e.out_stride, dtype, nullptr, 0}, s));
        }
        if (dhidden && tokens) {
            ProductArgs d{};
            d.a = w.grad, d.a_stride = w.piece, d.a_plane = g.grad_plane;
            d.b = t.p, d.b_stride = t.stride, d.b_plane = t.plane;
            d.m = tokens, d.n = cols, d.k = n, d.m_now = w.now, d.terms = terms;
            d.splits = kMaxSplits, d.jobs = tile_jobs(w.dh), d.part = w.dh_part, d.part_stride = part_stride;
            d.accumulate = v0 > 0;
            if (!v0) dh.k = z.whole ? 2 * n : n;  // the last piece, shorter, may have fewer parts: the others stay as they were
            if (z.few) WARP_STEP(product_few(d, dtype, z.planes == 3, kSum, w.dh_parts, s));
            else WARP_STEP(product_mixed(d, element, w.dh, kSum, s));
        }
    }
    if (dhidden) WARP_STEP(join_parts(dh, s));
    return WARP_OK;
}

}  // extern "C"
