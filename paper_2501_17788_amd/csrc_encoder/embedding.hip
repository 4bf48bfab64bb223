// Rows of a table by token, scaled, and the table's gradient:
//   out[t] = scale * table[id_t],   dtable[v] = scale * sum over t with id_t = v of dy[t]
// Both are bound by memory. The gradient's sums have a fixed order, without atomics on floats: tokens are sorted by
// id (stably, so that a row's tokens come in order) and summed in chunks of 32 sorted tokens, whatever rows these belong
// to. A row whose tokens lie in one chunk is written from there; one that goes on in another leaves a part in each, and
// those are added last, together with the zeros of the rows without tokens: the gradient is written once, and a
// common token's thousands are as many waves' work.
// A training step's 131,072 tokens (30% padding), 32,128 rows of 1024 bf16: lookup 67 us, 5.0 TB/s of the output and the table;
// gradient 120 us: sorting 32, chunks 73, the rest 15. Sorting by rows' own counts instead needs the counts' prefix sums and
// atomics that fix no order.
#include <type_traits>

#include "encoder.h"

namespace warp {

namespace {

inline int64_t cover(int64_t n, int64_t of) { return (n + of - 1) / of; }

__device__ __forceinline__ int64_t id_at(const void* ids, bool wide, int64_t t) {
    return wide ? ((const int64_t*)ids)[t] : (int64_t)((const int32_t*)ids)[t];
}

// A wave holds NV vectors of V elements of a row's column block, 64 V NV columns. A row's last vector is moved back to
// end with the row: its first elements are its neighbour's too, and get the same values.
template <int V>
struct Columns {
    int64_t at;
    bool in;
};
template <int V>
__device__ __forceinline__ Columns<V> column_of(int64_t block, int j, int nv, int lane, int64_t cols) {
    const int64_t c = ((block * nv + j) * kWave + lane) * V;
    return {c + V > cols ? cols - V : c, c < cols};
}

// ---------------------------------------------------------------------------- lookup

struct LookupArgs {
    const void* ids;
    bool wide;
    int64_t tokens, vocabulary;
    const void* table;
    int64_t table_stride;
    int64_t cols;
    float scale;
    void* out;
    int64_t out_stride;
    bool past_caches;
};

// One wave for R tokens and a block of 64 V NV columns, all its rows under way at once: a row's address has to wait for its
// id. 32 rows of 768 take 2.6 us, an empty launch's time.
template <typename T, int V, int NV, int R>
__global__ __launch_bounds__(256) void k_lookup(LookupArgs g) {
    const int lane = threadIdx.x & 63;
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * R;
    if (t0 >= g.tokens) return;
    Columns<V> c[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) c[j] = column_of<V>(blockIdx.y, j, NV, lane, g.cols);
    int64_t id[R];
#pragma unroll
    for (int r = 0; r < R; ++r) id[r] = id_at(g.ids, g.wide, t0 + r < g.tokens ? t0 + r : t0);
    Vec<T, V> x[R][NV];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool inside = id[r] >= 0 && id[r] < g.vocabulary;
        const T* row = (const T*)g.table + (inside ? id[r] : 0) * g.table_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j)
            if (c[j].in) x[r][j] = load_vec<T, V>(row + c[j].at);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (t0 + r >= g.tokens) return;
        const bool inside = id[r] >= 0 && id[r] < g.vocabulary;
        const float fill = id[r] < 0 ? 0.f : __builtin_nanf("");
        T* out = (T*)g.out + (t0 + r) * g.out_stride;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if (!c[j].in) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) x[r][j].e[e] = inside ? (T)((float)x[r][j].e[e] * g.scale) : (T)fill;
            if (g.past_caches) stream_out<T, V>(out + c[j].at, x[r][j]);
            else store_vec<T, V>(out + c[j].at, x[r][j]);
        }
    }
}

// ---------------------------------------------------------------------------- sorting tokens by id

// Stable radix sort by digits of at most 9 bits. At most 128 tiles of equal size; a tile's eight waves hold neighbouring
// parts of it. Bound by latency: a pass over 131,072 tokens takes 5 us for the counts and 11 for the places.
constexpr int kDigits = 512, kSortThreads = 512, kSortWaves = kSortThreads / kWave;
constexpr int kMaxTiles = 128, kTileUnit = 1024;
// So many tokens are sorted by one workgroup, in LDS: the whole gradient of 4096 into 9973 rows of 64 columns takes 28 us
// this way and 29 by tiles, of 8192 39 and 31, of 500 rows 2000 tokens 16 and 18.
constexpr int kSmall = 4096;

struct SortPlan {
    int64_t tokens;
    int64_t tile;  // tokens of a tile
    int tiles, bits, passes, digit_bits;
};
SortPlan sort_plan(int64_t tokens, int64_t vocabulary) {
    SortPlan p{};
    p.tokens = tokens;
    p.tile = cover(cover(tokens > 0 ? tokens : 1, kMaxTiles), kTileUnit) * kTileUnit;
    p.tiles = (int)cover(tokens, p.tile);
    while (p.bits < 40 && (vocabulary >> p.bits)) ++p.bits;  // keys up to `vocabulary`, which stands for no row
    p.passes = (int)cover(p.bits, 9);
    p.digit_bits = (int)cover(p.bits, p.passes);
    return p;
}

__device__ __forceinline__ uint32_t key_of(const void* ids, bool wide, int64_t t, int64_t vocabulary) {
    const int64_t id = id_at(ids, wide, t);
    return (uint32_t)(id < 0 || id >= vocabulary ? vocabulary : id);
}

__device__ __forceinline__ void clear_spans(int2* spans, int64_t vocabulary, int64_t thread, int64_t threads) {
    for (int64_t v = thread; v < vocabulary; v += threads) spans[v] = make_int2(0, 0);
}

// Sum of s over the workgroup's threads before this one.
__device__ __forceinline__ uint32_t sum_before(uint32_t s, uint32_t* waves) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t x = s;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) waves[w] = x;
    __syncthreads();
    uint32_t before = x - s;
    for (int i = 0; i < w; ++i) before += waves[i];
    __syncthreads();
    return before;
}

// Place of this lane's key among those of its wave with its digit, with next[digit] the first free place; lanes take
// turns in their order, and next moves on.
__device__ __forceinline__ uint32_t take_place(uint32_t digit, bool in, int digit_bits, uint32_t* next) {
    unsigned long long same = __ballot(in);
    for (int b = 0; b < digit_bits; ++b) {
        const unsigned long long ones = __ballot(digit >> b & 1u);
        same &= digit >> b & 1u ? ones : ~ones;
    }
    const int lane = threadIdx.x & 63;
    const uint32_t rank = (uint32_t)__popcll(same & ((1ull << lane) - 1));
    uint32_t place = 0;
    if (in) place = next[digit] + rank;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (in && rank == 0) next[digit] = place + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return place;
}

struct SortArgs {
    const void* ids;
    bool wide;
    int64_t tokens, vocabulary, tile;
    int tiles, shift, digit_bits;
    bool first;
    const uint32_t *keys, *places;
    uint32_t *keys_out, *places_out;
    uint32_t* counts;  // [tile][digit]
    int2* spans;
};

// Counts of a tile's digits; in the first pass the workgroups behind the tiles' clear the rows' spans.
__global__ __launch_bounds__(kSortThreads) void k_token_counts(SortArgs g) {
    __shared__ uint32_t count[kDigits];
    if ((int)blockIdx.x >= g.tiles) {
        clear_spans(g.spans, g.vocabulary, (int64_t)((int)blockIdx.x - g.tiles) * kSortThreads + threadIdx.x,
                    (int64_t)((int)gridDim.x - g.tiles) * kSortThreads);
        return;
    }
    count[threadIdx.x] = 0;
    __syncthreads();
    const int64_t start = (int64_t)blockIdx.x * g.tile;
    const uint32_t mask = (1u << g.digit_bits) - 1;
    for (int64_t i = threadIdx.x; i < g.tile && start + i < g.tokens; i += kSortThreads) {
        const uint32_t key = g.first ? key_of(g.ids, g.wide, start + i, g.vocabulary) : g.keys[start + i];
        atomicAdd(&count[key >> g.shift & mask], 1u);
    }
    __syncthreads();
    g.counts[(int64_t)blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

// Tokens to their places: a digit's first place in a tile is what all tiles have of smaller digits and the tiles before
// have of it. Every workgroup adds these up from the table of counts (at most 512 KB, in the L2s).
__global__ __launch_bounds__(kSortThreads) void k_token_places(SortArgs g) {
    __shared__ uint32_t next[kSortWaves][kDigits];
    __shared__ uint32_t waves[kSortWaves];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t start = (int64_t)blockIdx.x * g.tile;
    const int64_t part = g.tile / kSortWaves;  // a multiple of 64
    const uint32_t mask = (1u << g.digit_bits) - 1;
    auto key_at = [&](int64_t t) { return g.first ? key_of(g.ids, g.wide, t, g.vocabulary) : g.keys[t]; };
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) next[i][tid] = 0;
    __syncthreads();
    for (int64_t i = lane; i < part; i += 64) {
        const int64_t t = start + w * part + i;
        if (t < g.tokens) atomicAdd(&next[w][key_at(t) >> g.shift & mask], 1u);
    }
    uint32_t before = 0, all = 0;
#pragma unroll 16
    for (int t = 0; t < g.tiles; ++t) {
        const uint32_t c = g.counts[(int64_t)t * kDigits + tid];
        all += c;
        before += t < (int)blockIdx.x ? c : 0;
    }
    uint32_t place = sum_before(all, waves) + before;  // (its barriers also end the counting above)
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) {
        const uint32_t c = next[i][tid];
        next[i][tid] = place;
        place += c;
    }
    __syncthreads();
    for (int64_t i = lane; i < part; i += 64) {
        const int64_t t = start + w * part + i;
        const bool in = t < g.tokens;
        const uint32_t key = in ? key_at(t) : 0;
        const uint32_t to = take_place(key >> g.shift & mask, in, g.digit_bits, next[w]);
        if (in) {
            g.keys_out[to] = key;
            g.places_out[to] = g.first ? (uint32_t)t : g.places[t];
        }
    }
}

// Few tokens: workgroup 0 sorts them in LDS, in all passes, while the others clear the rows' spans.
__global__ __launch_bounds__(kSortThreads) void k_sort_few(SortArgs g, int passes) {
    if (blockIdx.x) {
        clear_spans(g.spans, g.vocabulary, (int64_t)(blockIdx.x - 1) * kSortThreads + threadIdx.x,
                    (int64_t)(gridDim.x - 1) * kSortThreads);
        return;
    }
    __shared__ uint32_t next[kSortWaves][kDigits];
    __shared__ uint32_t waves[kSortWaves];
    __shared__ uint32_t key[2][kSmall], place[2][kSmall];
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = (int)g.tokens;
    const int part = (n + kSortThreads - 1) / kSortThreads * 64;  // of a wave
    const uint32_t mask = (1u << g.digit_bits) - 1;
    for (int i = tid; i < n; i += kSortThreads) key[0][i] = key_of(g.ids, g.wide, i, g.vocabulary), place[0][i] = i;
    for (int p = 0; p < passes; ++p) {
        const int from = p & 1, shift = p * g.digit_bits;
#pragma unroll
        for (int i = 0; i < kSortWaves; ++i) next[i][tid] = 0;
        __syncthreads();
        for (int i = w * part + lane; i < (w + 1) * part; i += 64)
            if (i < n) atomicAdd(&next[w][key[from][i] >> shift & mask], 1u);
        __syncthreads();
        uint32_t all = 0;
#pragma unroll
        for (int i = 0; i < kSortWaves; ++i) all += next[i][tid];
        uint32_t at = sum_before(all, waves);
#pragma unroll
        for (int i = 0; i < kSortWaves; ++i) {
            const uint32_t c = next[i][tid];
            next[i][tid] = at;
            at += c;
        }
        __syncthreads();
        for (int i = w * part + lane; i < (w + 1) * part; i += 64) {
            const bool in = i < n;
            const uint32_t k = in ? key[from][i] : 0;
            const uint32_t to = take_place(k >> shift & mask, in, g.digit_bits, next[w]);
            if (in) key[from ^ 1][to] = k, place[from ^ 1][to] = place[from][i];
        }
        __syncthreads();
    }
    for (int i = tid; i < n; i += kSortThreads) g.keys_out[i] = key[passes & 1][i], g.places_out[i] = place[passes & 1][i];
}

// ---------------------------------------------------------------------------- sums

constexpr int kChunk = 32;  // sorted tokens of a chunk
constexpr int kFew = 8;     // parts that one wave adds

struct SumArgs {
    const void* dy;
    int64_t dy_stride;
    int64_t tokens, vocabulary, cols;
    const uint32_t *keys, *places;  // sorted
    int2* spans;                    // of each row, its sorted tokens [x, y)
    // [chunk][2][part_stride]: sums of the chunk's tokens of a row that came before, and of one that began there and goes on
    float* parts;
    int64_t part_stride;
    float scale;
    void* out;
    int64_t out_stride;
    int32_t blocks;  // of columns
    int64_t common;  // workgroups for rows of many parts
    bool past_caches;
};

// Rows of dy at places that the lanes hold, U from lane `from` on, all under way at once.
template <typename T, int V, int U>
struct Batch {
    Vec<T, V> x[U];
    __device__ __forceinline__ void load(const SumArgs& g, uint32_t places, int from, Columns<V> c) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t t = (uint32_t)__builtin_amdgcn_readlane((int)places, from + u);
            x[u] = load_vec<T, V>((const T*)g.dy + (int64_t)t * g.dy_stride + (c.in ? c.at : 0));
        }
    }
    // Waits for all of them at once: behind a store that not every wave makes, each use of a loaded value would wait for
    // all loads and stores under way.
    __device__ __forceinline__ void arrive() {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if constexpr (V == 1) {
                uint32_t v = 0;
                __builtin_memcpy(&v, &x[u], sizeof(x[u]));
                asm volatile("" : "+v"(v));
                __builtin_memcpy(&x[u], &v, sizeof(x[u]));
            } else {
                typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
                uint4v v = __builtin_bit_cast(uint4v, x[u]);
                asm volatile("" : "+v"(v));
                x[u] = __builtin_bit_cast(Vec<T, V>, v);
            }
        }
    }
};

template <typename T, int V>
__device__ __forceinline__ void store_sums(const float (&sum)[V], const SumArgs& g, int64_t row, Columns<V> c) {
    if (!c.in) return;
    Vec<T, V> r;
#pragma unroll
    for (int e = 0; e < V; ++e) r.e[e] = (T)(sum[e] * g.scale);
    T* out = (T*)g.out + row * g.out_stride + c.at;
    if (g.past_caches) stream_out<T, V>(out, r);
    else store_vec<T, V>(out, r);
}

// One wave a chunk and column block (those of a chunk are neighbours), half of its rows under way while the other half is
// added; and the chunk's part of the rows' spans. 91,721 rows of 2 KB, 190 MB read and 46 written: 39 us (6.0 TB/s) where the last-level
// cache holds dy, 73 in a training step and 85 (2.8 TB/s) where all of it comes from memory. That its rows lie scattered by
// sorting is not why: of ids in order, whose rows come as they lie, 83. A wave waits for its keys, then for each half of its rows, and
// ends with its chunk.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_sum_chunks(SumArgs g) {
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), chunk = wave / g.blocks, start = chunk * kChunk;
    const int block = (int)(wave % g.blocks);
    if (start >= g.tokens) return;
    const int64_t i = start + lane;
    const bool in = lane < kChunk && i < g.tokens;
    const uint32_t key = in ? g.keys[i] : ~0u;
    const uint32_t before = in && i ? g.keys[i - 1] : ~0u, behind = in && i + 1 < g.tokens ? g.keys[i + 1] : ~0u;
    const uint32_t places = in ? g.places[i] : 0;
    if (block == 0 && in && key < g.vocabulary) {
        if (key != before) g.spans[key].x = (int)i;
        if (key != behind) g.spans[key].y = (int)i + 1;
    }
    const int total = (int)__popcll(__ballot(in && key < g.vocabulary));  // the others come last
    if (!total) return;
    const unsigned long long ends = __ballot(in && key != behind);
    bool open = __builtin_amdgcn_readfirstlane((int)(key == before));  // the row's sum began in another chunk
    const Columns<V> c = column_of<V>(block, 0, 1, lane, g.cols);
    auto store_part = [&](const float (&sum)[V], int which) {
        if (!c.in) return;
        Vec<float, V> r;
#pragma unroll
        for (int e = 0; e < V; ++e) r.e[e] = sum[e];
        store_vec<float, V>(g.parts + (2 * chunk + which) * g.part_stride + c.at, r);
    };
    constexpr int U = 16;
    Batch<T, V, U> half[2];
    float sum[V] = {};
    half[0].load(g, places, 0, c);  // lanes behind the end hold a place too, whose row is not added
    auto add = [&](const Batch<T, V, U>& b, int at) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (at + u >= total) break;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += (float)b.x[u].e[e];
            if (!(ends >> (at + u) & 1)) continue;
            if (open) store_part(sum, 0);
            else store_sums<T, V>(sum, g, __builtin_amdgcn_readlane((int)key, at + u), c);
            open = false;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = 0.f;
        }
    };
    half[0].arrive();
    if (total > U) half[1].load(g, places, U, c);
    add(half[0], 0);
    if (total > U) {
        half[1].arrive();
        add(half[1], U);
    }
    if (!(ends >> (total - 1) & 1)) store_part(sum, open ? 0 : 1);
}

// Adds a row's parts, those of chunks first, first + 1, ... last: one a wave, every `by`th from `from` on.
template <int V>
__device__ __forceinline__ void add_parts(float (&sum)[V], const SumArgs& g, int first, int last, int from, int by, Columns<V> c) {
    auto add = [&](int i, auto count) {
        constexpr int U = count.value;
        Vec<float, V> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t chunk = i + by * u;
            if (c.in) x[u] = load_vec<float, V>(g.parts + (2 * chunk + (chunk == first)) * g.part_stride + c.at);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += x[u].e[e];
    };
    int i = first + from;
    for (; i + 3 * by <= last; i += 4 * by) add(i, std::integral_constant<int, 4>{});
    for (; i <= last; i += by) add(i, std::integral_constant<int, 1>{});
}

// The first `common` workgroups: one for each chunk; the second one of a row that has many stands for it, and the
// workgroup's waves share its parts. The others: kRows neighbouring rows a wave, those without tokens and those of few
// parts. 250,001 rows of 768 fp16, of which 8192 tokens reach few: 72 us, 5.3 TB/s of zeros.
constexpr int kRows = 4;
template <typename T, int V>
__global__ __launch_bounds__(256) void k_finish_rows(SumArgs g) {
    __shared__ float joined[3][V][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const Columns<V> c = column_of<V>(blockIdx.y, 0, 1, lane, g.cols);
    if ((int64_t)blockIdx.x >= g.common) {
        const int64_t row0 = (((int64_t)blockIdx.x - g.common) * 4 + w) * kRows;
        int2 span = make_int2(0, 0);
        if (lane < kRows && row0 + lane < g.vocabulary) span = g.spans[row0 + lane];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (row0 + r >= g.vocabulary) return;
            const int from = __builtin_amdgcn_readlane(span.x, r), to = __builtin_amdgcn_readlane(span.y, r);
            const int first = from / kChunk, last = (to - 1) / kChunk;
            if (from < to && (first == last || last - first >= kFew)) continue;
            float sum[V] = {};
            if (from < to) add_parts<V>(sum, g, first, last, 0, 1, c);
            store_sums<T, V>(sum, g, row0 + r, c);
        }
        return;
    }
    const int chunk = (int)blockIdx.x;
    const uint32_t row = g.keys[(int64_t)chunk * kChunk];
    if (row >= g.vocabulary) return;
    const int2 span = g.spans[row];
    const int first = span.x / kChunk, last = (span.y - 1) / kChunk;
    if (chunk != first + 1 || last - first < kFew) return;
    float sum[V] = {};
    add_parts<V>(sum, g, first, last, w, 4, c);
    if (w) {
#pragma unroll
        for (int e = 0; e < V; ++e) joined[w - 1][e][lane] = sum[e];
    }
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] += joined[0][e][lane] + joined[1][e][lane] + joined[2][e][lane];
    store_sums<T, V>(sum, g, row, c);
}

// ---------------------------------------------------------------------------- launches

// Vectors of 16 bytes, or single elements where a row is shorter.
template <typename F>
void by_width(int64_t cols, int wide, F f) {
    if (cols < wide) f(std::true_type{}, (int64_t)1);
    else f(std::false_type{}, cover(cols, (int64_t)wide * kWave));
}

// Results of more than the last-level cache holds pass it by.
constexpr int64_t kCached = 256ll << 20;

template <typename T>
void lookup(LookupArgs g, hipStream_t s) {
    constexpr int W = 16 / sizeof(T);
    g.past_caches = g.tokens * g.cols * (int64_t)sizeof(T) > kCached;
    by_width(g.cols, W, [&](auto narrow, int64_t blocks) {
        constexpr int V = narrow.value ? 1 : W;
        if (g.tokens < 4096)
            hipLaunchKernelGGL((k_lookup<T, V, 1, 1>), dim3((uint32_t)cover(g.tokens, 4), (uint32_t)blocks), dim3(256), 0, s,
                               g);
        else
            hipLaunchKernelGGL((k_lookup<T, V, 2, 4>), dim3((uint32_t)cover(g.tokens, 16), (uint32_t)cover(blocks, 2)),
                               dim3(256), 0, s, g);
    });
}

template <typename T>
void sums(SumArgs g, hipStream_t s) {
    constexpr int W = 16 / sizeof(T);
    g.blocks = 1;
    g.common = g.tokens > kFew * kChunk ? cover(g.tokens, kChunk) : 0;
    g.past_caches = g.vocabulary * g.cols * (int64_t)sizeof(T) > kCached;
    by_width(g.cols, W, [&](auto narrow, int64_t blocks) {
        constexpr int V = narrow.value ? 1 : W;
        g.blocks = (int32_t)blocks;
        if (g.tokens)
            hipLaunchKernelGGL((k_sum_chunks<T, V>), dim3((uint32_t)cover(cover(g.tokens, kChunk) * blocks, 4)), dim3(256), 0, s, g);
        hipLaunchKernelGGL((k_finish_rows<T, V>), dim3((uint32_t)(g.common + cover(g.vocabulary, 4 * kRows)), (uint32_t)blocks),
                           dim3(256), 0, s, g);
    });
}

struct BackwardScratch {
    int64_t keys[2], places[2], counts, spans, parts, bytes;
};
BackwardScratch backward_scratch(int64_t tokens, int64_t vocabulary, int64_t cols) {
    BackwardScratch b{};
    auto take = [&](int64_t bytes) {
        const int64_t at = b.bytes;
        b.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    for (int i = 0; i < 2; ++i) b.keys[i] = take(tokens * 4), b.places[i] = take(tokens * 4);
    b.counts = take((int64_t)kMaxTiles * kDigits * 4);
    b.spans = take(vocabulary * 8);
    b.parts = take(cover(tokens, kChunk) * 2 * cols * 4);
    return b;
}

int check_sizes(const char* what, int64_t tokens, int64_t vocabulary, int64_t cols) {
    if (tokens < 0) return fail(WARP_EINVAL, "%s: tokens must be >= 0 (got %lld)", what, (long long)tokens);
    if (vocabulary < 1) return fail(WARP_EINVAL, "%s: vocabulary must be >= 1 (got %lld)", what, (long long)vocabulary);
    if (cols < 1) return fail(WARP_EINVAL, "%s: cols must be >= 1 (got %lld)", what, (long long)cols);
    if (tokens > 1 << 25 || vocabulary > 1 << 25 || cols > 1 << 20 || tokens * cols > 1ll << 37 || vocabulary * cols > 1ll << 37)
        return fail(WARP_ENOTSUP, "%s: at most 2^25 tokens, 2^25 table rows, 2^20 columns and 2^37 elements (got %lld, %lld, "
                    "%lld)", what, (long long)tokens, (long long)vocabulary, (long long)cols);
    return WARP_OK;
}
int check_embedding(const char* what, const void* ids, int32_t id_bytes, int64_t tokens, int64_t vocabulary, int64_t cols,
                    int32_t dtype, float scale) {
    if (const int rc = check_sizes(what, tokens, vocabulary, cols)) return rc;
    if (id_bytes != 4 && id_bytes != 8) return fail(WARP_EINVAL, "%s: ids of 4 or 8 bytes (got %d)", what, id_bytes);
    if (!dtype_ok(dtype)) return fail(WARP_EINVAL, "%s: unknown dtype %d", what, dtype);
    if (!(scale - scale == 0.f)) return fail(WARP_EINVAL, "%s: scale must be finite", what);
    if (tokens && !ids) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)ids % id_bytes) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    return WARP_OK;
}
int check_matrix(const char* what, const void* p, int64_t stride, int64_t rows, int64_t cols, int32_t dtype) {
    if (rows && !p) return fail(WARP_EINVAL, "%s: null pointer", what);
    if ((uintptr_t)p % dtype_bytes(dtype)) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    if (rows > 1 && stride < cols)
        return fail(WARP_EINVAL, "%s: a row stride of %lld is below %lld columns", what, (long long)stride, (long long)cols);
    return WARP_OK;
}

}  // namespace

}  // namespace warp

using namespace warp;

extern "C" {

int warp_embedding(const void* ids, int32_t id_bytes, int64_t tokens, const void* table, int64_t table_stride,
                   int64_t vocabulary, int32_t cols, int32_t dtype, float scale, void* out, int64_t out_stride,
                   void* hip_stream) {
    const char* what = "embedding";
    int rc = check_embedding(what, ids, id_bytes, tokens, vocabulary, cols, dtype, scale);
    if (!rc) rc = check_matrix(what, table, table_stride, vocabulary, cols, dtype);
    if (!rc) rc = check_matrix(what, out, out_stride, tokens, cols, dtype);
    if (!rc) rc = require_device();
    if (rc || !tokens) return rc;
    const LookupArgs g{ids, id_bytes == 8, tokens, vocabulary, table, table_stride, cols, scale, out, out_stride, false};
    hipStream_t s = (hipStream_t)hip_stream;
    if (dtype == WARP_F32) WARP_LAUNCH(lookup<float>(g, s));
    else if (dtype == WARP_F16) WARP_LAUNCH(lookup<_Float16>(g, s));
    else WARP_LAUNCH(lookup<__bf16>(g, s));
    return WARP_OK;
}

int warp_embedding_backward_scratch(int64_t tokens, int64_t vocabulary, int32_t cols, int64_t* bytes) {
    const char* what = "embedding backward";
    if (!bytes) return fail(WARP_EINVAL, "%s: null pointer", what);
    if (const int rc = check_sizes(what, tokens, vocabulary, cols)) return rc;
    *bytes = backward_scratch(tokens, vocabulary, cols).bytes;
    return WARP_OK;
}

int warp_embedding_backward(const void* dy, int64_t dy_stride, const void* ids, int32_t id_bytes, int64_t tokens,
                            int64_t vocabulary, int32_t cols, int32_t dtype, float scale, void* dtable,
                            int64_t dtable_stride, void* scratch, int64_t scratch_bytes, void* hip_stream) {
    const char* what = "embedding backward";
    int rc = check_embedding(what, ids, id_bytes, tokens, vocabulary, cols, dtype, scale);
    if (!rc) rc = check_matrix(what, dy, dy_stride, tokens, cols, dtype);
    if (!rc) rc = check_matrix(what, dtable, dtable_stride, vocabulary, cols, dtype);
    if (rc) return rc;
    const BackwardScratch b = backward_scratch(tokens, vocabulary, cols);
    if (!scratch || scratch_bytes < b.bytes || (uintptr_t)scratch % 16)
        return fail(WARP_EINVAL, "%s: needs %lld bytes of scratch, 16-byte aligned (got %lld)", what, (long long)b.bytes,
                    (long long)(scratch ? scratch_bytes : 0));
    rc = require_device();
    if (rc) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    uint8_t* base = (uint8_t*)scratch;
    uint32_t *keys[2], *places[2];
    for (int i = 0; i < 2; ++i) keys[i] = (uint32_t*)(base + b.keys[i]), places[i] = (uint32_t*)(base + b.places[i]);
    const SortPlan p = sort_plan(tokens, vocabulary);
    SortArgs a{ids, id_bytes == 8, tokens, vocabulary, p.tile, p.tiles, 0, p.digit_bits, true, nullptr, nullptr, keys[0],
               places[0], (uint32_t*)(base + b.counts), (int2*)(base + b.spans)};
    int sorted = 0;
    const int clear = (int)(cover(vocabulary, 8 * kSortThreads) < 255 ? cover(vocabulary, 8 * kSortThreads) : 255);
    if (tokens <= kSmall) {
        WARP_LAUNCH(hipLaunchKernelGGL(k_sort_few, dim3(1 + clear), dim3(kSortThreads), 0, s, a, p.passes));
    } else {
        for (int i = 0; i < p.passes; ++i) {
            a.shift = i * p.digit_bits, a.first = i == 0;
            a.keys = keys[(i + 1) & 1], a.places = places[(i + 1) & 1];
            a.keys_out = keys[i & 1], a.places_out = places[i & 1];
            WARP_LAUNCH(hipLaunchKernelGGL(k_token_counts, dim3(p.tiles + (i ? 0 : clear)), dim3(kSortThreads), 0, s, a));
            WARP_LAUNCH(hipLaunchKernelGGL(k_token_places, dim3(p.tiles), dim3(kSortThreads), 0, s, a));
        }
        sorted = (p.passes - 1) & 1;
    }
    const SumArgs g{dy, dy_stride, tokens, vocabulary, cols, keys[sorted], places[sorted], a.spans,
                    (float*)(base + b.parts), cols, scale, dtable, dtable_stride, 0, 0, false};
    if (dtype == WARP_F32) WARP_LAUNCH(sums<float>(g, s));
    else if (dtype == WARP_F16) WARP_LAUNCH(sums<_Float16>(g, s));
    else WARP_LAUNCH(sums<__bf16>(g, s));
    return WARP_OK;
}

}  // extern "C"
