// A linear layer for training that keeps its input in 8-bit rows:
//   y = x W^T + b;  dx = dy W,  dW = dy^T (q * s),  db = sum of dy's rows
// Bound by the matrix cores where the sizes are large; every product reads its operands as they are stored. 32,768 x 4096 by
// 4096, bf16: y 0.94 ms, 8-bit rows 0.07, dx 0.94, dW 0.95 and 0.06 for its rows, db 0.05. 65,536 x 1024 by 128, bound by
// memory: y 27 us, 8-bit rows 32, dx 45 (3.4 TB/s, most of it written), dW and db 51.
#include "operands.h"

namespace warp {

namespace {

int check_sizes(const char* what, int64_t rows, int32_t cols, int32_t n, int32_t dtype) {
    if (rows < 0) return fail(WARP_EINVAL, "%s: rows must be >= 0 (got %lld)", what, (long long)rows);
    if (n < 1 || cols < 1) return fail(WARP_EINVAL, "%s: n and cols must be >= 1 (got %d, %d)", what, n, cols);
    if (rows > 1 << 24 || n > 1 << 20 || cols > 1 << 20 || (int64_t)n * cols > 1ll << 34 || rows * n > 1ll << 36 ||
        rows * cols > 1ll << 36)
        return fail(WARP_ENOTSUP, "%s: at most 2^24 rows, 2^20 columns and channels, and matrices of 2^36 elements (weights: "
                    "2^34; got %lld, %d, %d)", what, (long long)rows, cols, n);
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
    if (need && (!scratch || bytes < need || (uintptr_t)scratch % 16))
        return fail(WARP_EINVAL, "%s: needs %lld bytes of scratch, 16-byte aligned (got %lld)", what, (long long)need,
                    (long long)(scratch ? bytes : 0));
    return WARP_OK;
}

// A product whose k range may be split: in one launch, or in parts that are joined.
struct Product {
    Tile tile;
    bool split;
    int64_t floats, time;
    Product(int64_t m, int64_t n, int64_t k, int32_t dtype, Tile largest = kT256) {
        const ProductPlan p = plan_product(m, n, product_steps(k, terms_of(dtype)), true, largest);
        tile = p.tile, split = p.split, time = p.time;
        floats = split ? part_floats(m, n, k, terms_of(dtype), tile, kMaxSplits, tile_jobs(tile)) : 0;
    }
    Product(int64_t m, int64_t n, int64_t k) : tile(tile_f32(m, n)), time(0) {  // float32 without planes: steps of 32
        split = tile == kT64 && product_splits(m, n, cover_of(k, 32), 64, kMaxSplits, tile_jobs(tile)) > 1;
        floats = split ? part_floats(m, n, 2 * k, 1, tile, kMaxSplits, tile_jobs(tile)) : 0;
    }
};

// Most float32 rows that are multiplied as they are, without planes: the matrix instructions for them have a 16th of the
// rate, but nothing has to be packed. us, as they are | in planes, for 64, 256 and 384 rows: 4096 by 4096 29 | 63, 85 | 105,
// 118 | 136, 1024 by 1024 10 | 22, 25 | 28, 25 | 30, 771 by 3001 (copied to rows of whole pieces) 25 | 24, 32 | 33, 39 | 36; for 800
// rows 4096 by 4096 297 | 214. With gradients, 65, 200 and 384 rows: 4096 by 4096 144 | 232, 251 | 330, 363 | 406, 771 by 3001
// 75 | 73, 90 | 98, 115 | 116.
constexpr int kWholeRows = 384;

typedef hipError_t (*ProductCall)(const ProductArgs&, int, Tile, Finish, hipStream_t);

hipError_t run_product(ProductCall call, ProductArgs g, const Product& plan, float* part, int32_t dtype, hipStream_t s,
                       bool whole = false) {
    g.terms = whole ? 1 : terms_of(dtype);
    g.splits = kMaxSplits, g.jobs = tile_jobs(plan.tile);
    g.part = part, g.part_stride = cover_of(g.n, 4) * 4;
    const Finish finish = plan.split ? kSum : kStore;
    const hipError_t e = g.b_scale ? product_bytes(g, element_of(dtype), plan.tile, finish, s)
                                   : call(g, whole ? dtype : element_of(dtype), plan.tile, finish, s);
    if (e || !plan.split) return e;
    const Join j{part, g.part_stride, g.m, g.n, whole ? 2 * g.k : g.k, nullptr, nullptr, g.terms, g.splits, g.jobs, tile_size(plan.tile),
                 nullptr, nullptr, g.m, g.out, g.out_stride, g.out_type, g.bias, g.bias_type};
    return join_parts(j, s);
}

ProductArgs product_args(const Operand& a, const Operand& b, int64_t m, int64_t n, int64_t k, void* out, int64_t out_stride,
                         int32_t out_type) {
    ProductArgs g{};
    g.a = a.p, g.a_stride = a.stride, g.a_plane = a.plane;
    g.b = b.p, g.b_stride = b.stride, g.b_plane = b.plane;
    g.m = m, g.n = n, g.k = k;
    g.out = out, g.out_stride = out_stride, g.out_type = out_type;
    return g;
}

struct Forward {
    Space space;
    uint16_t *x, *w;
    float* part;
    Product y;
    bool few, whole;  // float32 without planes
    Forward(void* base, const void* x_, int64_t x_stride, int64_t rows, int64_t cols, int32_t dtype, const void* w_,
            int64_t w_stride, int64_t n)
        : y(rows, n, cols, dtype) {
        space.base = (uint8_t*)base;
        few = rows <= kFewRows;
        whole = !few && dtype == WARP_F32 && rows <= kWholeRows;
        if (few) y.floats = 0;
        if (whole) y = Product(rows, n, cols);
        auto room = [&](const void* p, int64_t stride, int64_t count) {
            if (few || (whole ? direct_f32 : direct)(p, stride, count, cols, dtype)) return (int64_t)0;
            return whole ? 2 * count * packed_width(cols) : packed_elements(count, cols, dtype);
        };
        x = space.take<uint16_t>(room(x_, x_stride, rows));
        w = space.take<uint16_t>(room(w_, w_stride, n));
        part = space.take<float>(y.floats);
    }
};

// Whether dweight's product takes the 8-bit rows as they are, and dbias with them, or has them unpacked and dy summed
// first. Its loads pass registers then, and tiles are 128 x 128 at most: an eighth more time for each; the other way
// reads and writes the rows and reads dy once more, with three launches. `direct`, `packed`: the products' times, ns.
// us for dweight and dbias, as they are | unpacked: 1 x 1024 by 1024 9.4 | 15.9, 1771 x 768 by 1000 19.4 | 30.9, 65,536 x 1024 by
// 128 45 | 96, by 512 112 | 172, by 1024 188 | 222, 16,384 x 1024 by 1024 67 | 72, 32,768 x 2048 by 2048 351 | 314, 4096 x 4096 by
// 4096 168 | 133, 32,768 x 4096 by 4096 1344 | 990.
inline bool takes_bytes(int64_t rows, int64_t n, int64_t cols, int32_t dtype, int64_t direct, int64_t packed) {
    return dtype != WARP_F32 && direct + direct / 8 + 5000 < packed + rows * cols * 3 / 5000 + rows * n * 2 / 5000 + 12000;
}

// dx of few rows by the weight where it lies, dweight of few float32 rows. us for both, dbias and the 8-bit rows, so | by tiles in
// planes: 16 x 4096 by 4096 40 | 157, 32 53 | 157, 64 76 | 168, 771 by 3001 30 | 45, 41 | 45, 38 | 44, 16 x 1024 by 1024 21 | 32.
inline bool few_dx(int64_t rows, int32_t dtype) { return rows <= (dtype == WARP_F32 ? 2 * kFewRows : kFewRows); }
inline bool takes_outer(int64_t rows, int64_t n, int64_t cols, int32_t dtype) {
    return dtype == WARP_F32 && rows && rows <= (n * cols < 1 << 23 ? kOuter / 2 : kOuter);
}

struct Backward {
    Space space;
    uint16_t *dy, *x, *w;
    float *part, *room;
    Product dx, dw;
    bool bytes, few, outer;  // dx of few rows, dweight over few
    bool whole;              // float32 without planes
    int64_t sums;     // parts of dbias; none where it comes with dweight
    int parts;        // of dx of few rows
    Backward(void* base, const void* dy_, int64_t dy_stride, int64_t rows, int64_t cols, int32_t dtype, const void* w_,
             int64_t w_stride, int64_t n)
        : dx(rows, cols, n, dtype), dw(n, cols, rows, dtype) {
        space.base = (uint8_t*)base;
        few = few_dx(rows, dtype);
        outer = takes_outer(rows, n, cols, dtype);
        whole = dtype == WARP_F32 && rows > kFewRows && rows <= kWholeRows;
        if (whole) dx = Product(rows, cols, n), dw = Product(n, cols, rows);
        auto room_of = [&](const void* p, int64_t stride, int64_t count, int64_t width) {
            if ((whole ? direct_f32 : direct)(p, stride, count, width, dtype)) return (int64_t)0;
            return whole ? 2 * count * packed_width(width) : packed_elements(count, width, dtype);
        };
        dy = space.take<uint16_t>(few && outer ? 0 : room_of(dy_, dy_stride, rows, n));
        parts = few ? few_parts(rows, cols, n, dtype) : 0;
        if (few) dx.floats = parts * rows * cover_of(cols, 4) * 4;
        w = space.take<uint16_t>(few ? 0 : room_of(w_, w_stride, n, cols));
        const Product direct_dw(n, cols, rows, dtype, kT128);
        bytes = takes_bytes(rows, n, cols, dtype, direct_dw.time, dw.time);
        sums = 0;
        if (bytes) {
            dw = direct_dw;
            if (dw.split)
                sums = product_splits(n, cols, product_steps(rows, 1), tile_size(dw.tile), kMaxSplits, tile_jobs(dw.tile));
            else
                sums = dw.tile == kT64 ? 0 : 1;
            sums *= cover_of(cols, tile_size(dw.tile));
        }
        x = space.take<uint16_t>(bytes || outer ? 0 : packed_elements(rows, cols, dtype));
        if (outer) dw.floats = 0;
        part = space.take<float>(dx.floats > dw.floats ? dx.floats : dw.floats);
        room = space.take<float>(sums * n > column_room(rows, n) ? sums * n : column_room(rows, n));
    }
};

#define WARP_STEP(...)                                                                                       \
    do {                                                                                                     \
        const hipError_t e_ = (__VA_ARGS__);                                                                 \
        if (e_ != hipSuccess) return fail(WARP_EDEVICE, "%s: launch failed: %s", what, hipGetErrorString(e_)); \
    } while (0)

}  // namespace

int product_choice(int64_t m, int64_t n, int64_t k, int dtype, bool bytes) {
    Product p(m, n, k, dtype);
    if (bytes) {
        const Product direct(m, n, k, dtype, kT128);
        if (!takes_bytes(k, m, n, dtype, direct.time, p.time)) return -1;
        p = direct;
    }
    return p.tile + 4 * p.split;
}

}  // namespace warp

using namespace warp;

extern "C" {

int warp_linear_scratch(const void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t dtype, const void* weight,
                        int64_t weight_stride, int32_t n, int64_t* bytes) {
    const char* what = "linear";
    if (!bytes) return fail(WARP_EINVAL, "%s: null pointer", what);
    if (const int rc = check_sizes(what, rows, cols, n, dtype)) return rc;
    *bytes = Forward(nullptr, x, x_stride, rows, cols, dtype, weight, weight_stride, n).space.used;
    return WARP_OK;
}

int warp_linear(const void* x, int64_t x_stride, int64_t rows, int32_t cols, int32_t dtype, const void* weight,
                int64_t weight_stride, int32_t n, const void* bias, int32_t bias_dtype, void* y, int64_t y_stride,
                void* scratch, int64_t scratch_bytes, void* hip_stream) {
    const char* what = "linear";
    int rc = check_sizes(what, rows, cols, n, dtype);
    if (!rc) rc = check_matrix(what, x, x_stride, rows, cols, dtype);
    if (!rc) rc = check_matrix(what, weight, weight_stride, n, cols, dtype);
    if (!rc) rc = check_matrix(what, y, y_stride, rows, n, dtype);
    if (rc) return rc;
    if (bias && bias_dtype != WARP_F32 && bias_dtype != dtype)
        return fail(WARP_EINVAL, "%s: bias must be float32 or of x's type", what);
    if (bias && (uintptr_t)bias % dtype_bytes(bias_dtype)) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    const Forward f(scratch, x, x_stride, rows, cols, dtype, weight, weight_stride, n);
    rc = check_scratch(what, scratch, scratch_bytes, f.space.used);
    if (!rc) rc = require_device();
    if (rc || !rows) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    if (f.few) {
        ProductArgs g = product_args({x, rows <= 1 ? cols : x_stride, 0}, {weight, n <= 1 ? cols : weight_stride, 0}, rows, n, cols, y,
                                     y_stride, dtype);
        g.bias = bias, g.bias_type = bias_dtype;
        WARP_STEP(product_few(g, dtype, false, kStore, 1, s));
        return WARP_OK;
    }
    PackRows pack_x, pack_w;
    const Operand a = operand_of(x, x_stride, rows, cols, dtype, f.x, &pack_x, f.whole);
    const Operand b = operand_of(weight, weight_stride, n, cols, dtype, f.w, &pack_w, f.whole);
    WARP_STEP(pack_rows(pack_x, pack_w, dtype, s));
    ProductArgs g = product_args(a, b, rows, n, cols, y, y_stride, dtype);
    g.bias = bias, g.bias_type = bias_dtype;
    WARP_STEP(run_product(product_along, g, f.y, f.part, dtype, s, f.whole));
    return WARP_OK;
}

int warp_linear_backward_scratch(const void* dy, int64_t dy_stride, int64_t rows, int32_t n, int32_t dtype, int32_t cols,
                                 const void* weight, int64_t weight_stride, int64_t* bytes) {
    const char* what = "linear backward";
    if (!bytes) return fail(WARP_EINVAL, "%s: null pointer", what);
    if (const int rc = check_sizes(what, rows, cols, n, dtype)) return rc;
    *bytes = Backward(nullptr, dy, dy_stride, rows, cols, dtype, weight, weight_stride, n).space.used;
    return WARP_OK;
}

int warp_linear_backward(const void* dy, int64_t dy_stride, int64_t rows, int32_t n, int32_t dtype, const int8_t* q,
                         int64_t q_stride, const float* q_scale, int32_t cols, const void* weight, int64_t weight_stride,
                         void* dx, int64_t dx_stride, void* dweight, int64_t dweight_stride, void* dbias, int32_t dbias_dtype,
                         void* scratch, int64_t scratch_bytes, void* hip_stream) {
    const char* what = "linear backward";
    int rc = check_sizes(what, rows, cols, n, dtype);
    if (!rc) rc = check_matrix(what, dy, dy_stride, rows, n, dtype);
    if (!rc) rc = check_matrix(what, weight, weight_stride, n, cols, dtype);
    if (!rc && dx) rc = check_matrix(what, dx, dx_stride, rows, cols, dtype);
    if (!rc && dweight) rc = check_matrix(what, dweight, dweight_stride, n, cols, dtype);
    if (rc) return rc;
    if (dweight && rows) {
        if (!q || !q_scale) return fail(WARP_EINVAL, "%s: null pointer", what);
        if (q_stride < (cols + kInt8Pad - 1) / kInt8Pad * kInt8Pad || q_stride % 16 || (uintptr_t)q % 16 ||
            (uintptr_t)q_scale % 4)
            return fail(WARP_EINVAL, "%s: int8 rows need 16-byte alignment and a stride that is a multiple of 16 and at least "
                        "%d (got %lld)", what, (cols + kInt8Pad - 1) / kInt8Pad * kInt8Pad, (long long)q_stride);
    }
    if (dbias && dbias_dtype != WARP_F32 && dbias_dtype != dtype)
        return fail(WARP_EINVAL, "%s: dbias must be float32 or of dy's type", what);
    if (dbias && (uintptr_t)dbias % dtype_bytes(dbias_dtype)) return fail(WARP_EINVAL, "%s: misaligned pointer", what);
    const Backward w(scratch, dy, dy_stride, rows, cols, dtype, weight, weight_stride, n);
    rc = check_scratch(what, scratch, scratch_bytes, w.space.used);
    if (!rc) rc = require_device();
    if (rc) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    PackRows pack_dy, pack_w;
    Operand d{}, t{};
    if (rows && ((dx && !w.few) || (dweight && !w.outer))) d = operand_of(dy, dy_stride, rows, n, dtype, w.dy, &pack_dy, w.whole);
    if (rows && dx && !w.few) t = operand_of(weight, weight_stride, n, cols, dtype, w.w, &pack_w, w.whole);
    WARP_STEP(pack_rows(pack_dy, pack_w, dtype, s));
    if (rows && dx && w.few) {
        ProductArgs g = product_args({dy, rows <= 1 ? n : dy_stride, 0}, {weight, n <= 1 ? cols : weight_stride, 0}, rows, cols, n, dx,
                                     dx_stride, dtype);
        g.part = w.part, g.part_stride = cover_of(cols, 4) * 4;
        WARP_STEP(product_few(g, dtype, false, kSum, w.parts, s));
        Join j{w.part, g.part_stride, rows, cols, n, nullptr, nullptr, 0, 0, 0, 0, nullptr, nullptr, rows, dx, dx_stride, dtype,
               nullptr, 0};
        j.parts = w.parts;
        WARP_STEP(join_parts(j, s));
    } else if (rows && dx) {
        WARP_STEP(run_product(product_mixed, product_args(d, t, rows, cols, n, dx, dx_stride, dtype), w.dx, w.part, dtype, s,
                              w.whole));
    }
    const bool bytes = dweight && w.bytes && rows;
    if (dweight && w.outer) {
        WARP_STEP(product_outer({dy, q, rows <= 1 ? n : dy_stride, 0, q_stride, 0, q_scale, n, cols, rows, nullptr, nullptr, (float*)dweight,
                                 dweight_stride, (float*)dbias}, s));
    } else if (bytes) {
        ProductArgs g = product_args(d, {q, q_stride, 0}, n, cols, rows, dweight, dweight_stride, dtype);
        g.b_scale = q_scale;
        if (dbias && w.sums) g.sums = w.room;
        else g.all_sums = dbias, g.sums_type = dbias_dtype;
        WARP_STEP(run_product(nullptr, g, w.dw, w.part, dtype, s));
        if (g.sums) WARP_STEP(join_columns(w.room, w.sums, n, dbias, dbias_dtype, s));
    } else if (dweight) {  // without rows: zeros
        WARP_STEP(unpack_int8(q, q_stride, q_scale, rows, cols, dtype, w.x, s, w.whole));
        const Operand x{w.x, packed_width(cols), rows * packed_width(cols)};
        WARP_STEP(run_product(product_across, product_args(d, x, n, cols, rows, dweight, dweight_stride, dtype), w.dw, w.part,
                              dtype, s, w.whole));
    }
    if (dbias && !bytes && !(dweight && w.outer)) WARP_STEP(column_sums(dy, dy_stride, rows, n, dtype, w.room, dbias, dbias_dtype, s));
    return WARP_OK;
}

}  // extern "C"
