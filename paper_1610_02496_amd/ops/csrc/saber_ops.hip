// Host side of the head's operators (include/saber_ops.h): checks of arguments, choice of a kernel's variant, launches.  Nothing here
// allocates, synchronises or keeps state between calls.
#include <cstdarg>
#include <cstdio>
#include <type_traits>

#include "../../../include/saber_ops.h"
#include "ops_norm.hpp"
#include "ops_xent.hpp"

using namespace saber_ops;

namespace {

thread_local char g_err[512] = "";
int fail(int code, const char *fmt, ...) {
    va_list ap; va_start(ap, fmt); vsnprintf(g_err, sizeof(g_err), fmt, ap); va_end(ap);
    return code;
}
#define OPS_HIP(expr)                                                                                       \
    do {                                                                                                    \
        hipError_t e_ = (expr);                                                                             \
        if (e_ != hipSuccess)                                                                               \
            return fail(e_ == hipErrorOutOfMemory ? SABER_ENOMEM : SABER_EDEVICE, "%s failed: %s", #expr, hipGetErrorString(e_)); \
    } while (0)

constexpr int64_t kMaxRows = (int64_t)1 << 31, kMaxCols = (int64_t)1 << 20, kMaxWords = (int64_t)1 << 31;
constexpr int kCus = 256;   // of gfx950: sizes of grids only
constexpr int64_t kXentRows = ((int64_t)1 << 26) - 16, kMaxTiles = (int64_t)1 << 24;   // (a launch has fewer than 2^32 threads)

size_t size_of(int type) { return type == SABER_F32 ? 4 : 2; }
bool is_type(int type) { return type == SABER_F32 || type == SABER_F16 || type == SABER_BF16; }
int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t parts_of(int64_t v, int64_t by) { return (v + by - 1) / by; }
bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// calls f(T{}) with the element type
template <class F>
int with_type(int type, F &&f) {
    if (type == SABER_F32) return f(f32{});
    if (type == SABER_F16) return f(f16{});
    return f(bf16{});
}

int check_rows(const char *who, int64_t rows, int64_t cols, int dtype) {
    if (!is_type(dtype)) return fail(SABER_EINVAL, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || cols < 1) return fail(SABER_EINVAL, "%s: %lld rows of %lld columns", who, (long long)rows, (long long)cols);
    if (rows >= kMaxRows || cols > kMaxCols) return fail(SABER_ERANGE, "%s: %lld rows of %lld columns (limits 2^31 - 1 and 2^20)", who, (long long)rows, (long long)cols);
    return SABER_OK;
}
int check_stride(const char *who, const char *what, int64_t stride, int64_t cols) {
    if (stride < cols) return fail(SABER_EINVAL, "%s: rows of %s lie %lld elements apart, fewer than their %lld columns", who, what, (long long)stride, (long long)cols);
    if (stride > (int64_t)1 << 40) return fail(SABER_ERANGE, "%s: stride of %s", who, what);
    return SABER_OK;
}
int check_pointer(const char *who, const char *what, const void *p, size_t align) {
    if (!p) return fail(SABER_EINVAL, "%s: %s is null", who, what);
    if (!aligned(p, align)) return fail(SABER_EINVAL, "%s: %s is not aligned to its elements", who, what);
    return SABER_OK;
}
#define OPS_TRY(expr) do { const int rc_ = (expr); if (rc_ != SABER_OK) return rc_; } while (0)

// ---- layer norm --------------------------------------------------------------------------------------------------------------

// Rows of up to 1,024 columns belong to a wavefront, up to 4,096 to a workgroup of 256, up to 8,192 to one of 512: a lane has 16
// elements of a row at most, so that the row after can be on its way.  Measured in us, forward and backward: 16,384 x 1024 in bf16 with
// the checkpoint, a wavefront 24 and 21, a workgroup 32 and 28; 65,536 x 2048 in f16, a workgroup 98 and 157, a wavefront (32 elements a
// lane) 92 and 163, more in all with the partial sums.  Wider ones are read again for every sum.
constexpr int64_t kNormCols = 8192;

template <class F>
int with_norm_shape(int64_t cols, F &&f) {
    using C1 = std::integral_constant<int, 1>; using C2 = std::integral_constant<int, 2>;
    using W = std::integral_constant<int, 64>; using G = std::integral_constant<int, 256>; using GG = std::integral_constant<int, 512>;
    if (cols <= 512) return f(W{}, C1{});
    if (cols <= 1024) return f(W{}, C2{});
    if (cols <= 2048) return f(G{}, C1{});
    if (cols <= 4096) return f(G{}, C2{});
    return f(GG{}, C2{});
}
int64_t rows_per_group(int64_t cols) { return cols <= 1024 ? 4 : 1; }
// workgroups of the backward pass, as many as the CUs hold at a time: each leaves a partial row of both sums
int64_t norm_parts(int64_t rows, int64_t cols) {
    if (cols > kNormCols) return rows < 256 ? (rows > 0 ? rows : 1) : 256;
    const int64_t groups = parts_of(rows > 0 ? rows : 1, rows_per_group(cols)), most = (cols <= 1024 ? 3 : cols <= 4096 ? 4 : 2) * kCus;
    return groups < most ? groups : most;
}

}  // namespace

extern "C" const char *saber_ops_last_error(void) { return g_err; }

extern "C" int saber_layer_norm_forward(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t rows, int64_t cols,
                                        int dtype, int wtype, float eps, void *y, float *mean, float *rstd, int8_t *q, float *scale,
                                        void *stream) {
    const char *who = "saber_layer_norm_forward";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    if (!is_type(wtype)) return fail(SABER_EINVAL, "%s: unknown type %d of weight and bias", who, wtype);
    OPS_TRY(check_stride(who, "x", x_stride, cols));
    if (!(eps >= 0.f)) return fail(SABER_EINVAL, "%s: eps must not be negative", who);
    if (!q != !scale) return fail(SABER_EINVAL, "%s: q and scale are given together", who);
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    OPS_TRY(check_pointer(who, "y", y, size_of(dtype)));
    OPS_TRY(check_pointer(who, "mean", mean, 4));
    OPS_TRY(check_pointer(who, "rstd", rstd, 4));
    if (weight) OPS_TRY(check_pointer(who, "weight", weight, size_of(wtype)));
    if (bias) OPS_TRY(check_pointer(who, "bias", bias, size_of(wtype)));
    if (scale) OPS_TRY(check_pointer(who, "scale", scale, 4));
    const NormForward a{x, x_stride, weight, bias, wtype, rows, cols, eps, y, mean, rstd, q, scale};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        if (cols > kNormCols) norm_forward_wide_kernel<T><<<(unsigned)(rows < 64 * kCus ? rows : 64 * kCus), 1024, 0, st>>>(a);
        else {
            const int64_t groups = parts_of(rows, rows_per_group(cols));
            const unsigned grid = (unsigned)(groups < 8 * kCus ? groups : 8 * kCus);
            OPS_TRY(with_norm_shape(cols, [&](auto tpr, auto nc) -> int {
                if (q) norm_forward_kernel<T, tpr.value, nc.value, true><<<grid, kNormThreads<tpr.value>, 0, st>>>(a);
                else norm_forward_kernel<T, tpr.value, nc.value, false><<<grid, kNormThreads<tpr.value>, 0, st>>>(a);
                return SABER_OK;
            }));
        }
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

extern "C" int saber_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t *bytes) {
    OPS_TRY(check_rows("saber_layer_norm_backward_workspace", rows, cols, SABER_F32));
    if (!bytes) return fail(SABER_EINVAL, "saber_layer_norm_backward_workspace: bytes is null");
    *bytes = norm_parts(rows, cols) * 2 * cols * 4;
    return SABER_OK;
}

extern "C" int saber_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const int8_t *q,
                                         const float *scale, const float *mean, const float *rstd, const void *weight, int64_t rows,
                                         int64_t cols, int dtype, int wtype, void *dx, void *dweight, void *dbias, void *workspace,
                                         int64_t workspace_bytes, void *stream) {
    const char *who = "saber_layer_norm_backward";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    if (!is_type(wtype)) return fail(SABER_EINVAL, "%s: unknown type %d of weight and bias", who, wtype);
    if (!q != !scale) return fail(SABER_EINVAL, "%s: q and scale are given together", who);
    if (x && q) return fail(SABER_EINVAL, "%s: either x or a checkpoint of it is given, not both", who);
    OPS_TRY(check_stride(who, "dy", dy_stride, cols));
    if (x) OPS_TRY(check_stride(who, "x", x_stride, cols));
    const bool sums = dweight || dbias;
    if (dweight) OPS_TRY(check_pointer(who, "dweight", dweight, size_of(wtype)));
    if (dbias) OPS_TRY(check_pointer(who, "dbias", dbias, size_of(wtype)));
    if (dx) OPS_TRY(check_pointer(who, "dx", dx, size_of(dtype)));
    if (weight) OPS_TRY(check_pointer(who, "weight", weight, size_of(wtype)));
    if (rows > 0) {
        OPS_TRY(check_pointer(who, "dy", dy, size_of(dtype)));
        if (q) OPS_TRY(check_pointer(who, "scale", scale, 4));
        else OPS_TRY(check_pointer(who, "x (or its checkpoint)", x, size_of(dtype)));
        OPS_TRY(check_pointer(who, "mean", mean, 4));
        OPS_TRY(check_pointer(who, "rstd", rstd, 4));
    }
    const int64_t parts = rows > 0 ? norm_parts(rows, cols) : 0;
    if (sums && parts) {
        OPS_TRY(check_pointer(who, "workspace", workspace, 16));
        if (workspace_bytes < parts * 2 * cols * 4) return fail(SABER_EINVAL, "%s: work space of %lld bytes, %lld are needed", who, (long long)workspace_bytes, (long long)(parts * 2 * cols * 4));
    }
    if (!sums && (!dx || rows == 0)) return SABER_OK;
    const NormBackward a{dy, dy_stride, x, x_stride, q, scale, mean, rstd, weight, wtype, rows, cols, dx,
                         sums ? static_cast<float *>(workspace) : nullptr, (int)parts};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    OPS_TRY(with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        if (rows == 0) return SABER_OK;
        if (cols > kNormCols) {
            if (dx) norm_backward_wide_kernel<T><<<(unsigned)(rows < 64 * kCus ? rows : 64 * kCus), 1024, 0, st>>>(a);
            if (sums) norm_columns_wide_kernel<T><<<dim3((unsigned)parts_of(cols, 2048), (unsigned)parts), 256, 0, st>>>(a);
        } else
            OPS_TRY(with_norm_shape(cols, [&](auto tpr, auto nc) -> int {
                if (q) norm_backward_kernel<T, tpr.value, nc.value, true><<<(unsigned)parts, kNormThreads<tpr.value>, 0, st>>>(a);
                else norm_backward_kernel<T, tpr.value, nc.value, false><<<(unsigned)parts, kNormThreads<tpr.value>, 0, st>>>(a);
                return SABER_OK;
            }));
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    }));
    if (sums) {   // (no rows: zeros)
        norm_weight_kernel<<<dim3((unsigned)parts_of(cols, 32), 2), 1024, 0, st>>>(static_cast<const float *>(workspace), (int)parts, cols, dweight, dbias, wtype);
        OPS_HIP(hipGetLastError());
    }
    return SABER_OK;
}

// ---- checkpoints in 8 bits ---------------------------------------------------------------------------------------------------

namespace {
struct Blocks { unsigned grid; int64_t step_rows, step_blocks; };
Blocks blocks_of(int64_t rows, int64_t cols) {
    const int64_t nb = parts_of(cols, kBlock), groups = parts_of(rows * nb, 16), grid = groups < 16 * kCus ? groups : 16 * kCus;
    return {(unsigned)grid, grid * 16 / nb, grid * 16 % nb};
}
}  // namespace

extern "C" int saber_checkpoint8_save(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int dtype, int8_t *q, float *scale,
                                      void *stream) {
    const char *who = "saber_checkpoint8_save";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    OPS_TRY(check_stride(who, "x", x_stride, cols));
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    OPS_TRY(check_pointer(who, "q", q, 1));
    OPS_TRY(check_pointer(who, "scale", scale, 4));
    const Blocks b = blocks_of(rows, cols);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        checkpoint8_save_kernel<T><<<b.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(static_cast<const T *>(x), x_stride, rows, cols, q, scale, b.step_rows, b.step_blocks);
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

extern "C" int saber_checkpoint8_restore(const int8_t *q, const float *scale, int64_t rows, int64_t cols, int dtype, void *x, void *stream) {
    const char *who = "saber_checkpoint8_restore";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_pointer(who, "q", q, 1));
    OPS_TRY(check_pointer(who, "scale", scale, 4));
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    const Blocks b = blocks_of(rows, cols);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        checkpoint8_restore_kernel<T><<<b.grid, 256, 0, static_cast<hipStream_t>(stream)>>>(q, scale, rows, cols, static_cast<T *>(x), b.step_rows, b.step_blocks);
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

// ---- softmax cross entropy with its projection -------------------------------------------------------------------------------

namespace {

// Up to 64 rows whose features fit LDS go through the kernel for few rows.  It reads the projection as it lies where the products would
// have it packed first (us of few rows and of products: 61 rows of 777 in f16, 30,011 words, 31 and 39; 1 row of 2048 in f32, 100,000
// words, 263 and 654), and shares out long rows of few words (9 rows in bf16, which the caches do not hold yet: 2048 columns of 1000 words
// 15.8 and 23.0, 1024 of 30,000 25.4 and 28.4).  Where a 16-bit projection lies well and is large it gains nothing (9 rows of 1024 and
// 100,000 words 82.6 and 83.4) or loses: 9 rows of 2048, 149 and 129; 60 rows of 64, 43 and 22.  The rule stays as simple as it is: what it
// loses there is a part of a call that reads the whole projection for a handful of rows.
constexpr int64_t kFewRows = 64;
constexpr int64_t kFewLds = 150 * 1024;
// 16-bit values of d, and of packed words, per piece: 256 MB of each, what the last-level cache holds.  A value of binary32 is three of d,
// two of the logits' words, five of the gradients' words.  (In binary32 fewer pieces are faster, a training step of 2,048 rows of 512
// columns and 60,000 words 2.42 ms in one and 2.67 in four, but d of all words is larger than the logits.)
constexpr int64_t kPieceValues = (int64_t)1 << 27;

struct Xent {
    const void *x; int64_t x_stride;
    const void *w; int64_t w_stride;
    int64_t rows, vocab, cols; int dtype;
    int planes;               // 3 for binary32
    bool pack_x, pack_w;
    int64_t cols_pad;         // columns of packed rows
};

// 16-bit rows that start at multiples of 16 bytes and are whole pieces of 8 elements go to LDS as they lie
bool direct(const void *p, int64_t stride, int64_t cols, int dtype) {
    return dtype != SABER_F32 && cols % 8 == 0 && stride % 8 == 0 && aligned(p, 16) && stride <= (int64_t)1 << 21;
}

int check_xent(const char *who, Xent &c) {
    OPS_TRY(check_rows(who, c.rows, c.cols, c.dtype));
    if (c.rows > kXentRows) return fail(SABER_ERANGE, "%s: %lld rows (limit 2^26 - 16)", who, (long long)c.rows);
    if (c.vocab < 1) return fail(SABER_EINVAL, "%s: a vocabulary of %lld words", who, (long long)c.vocab);
    if (c.vocab >= kMaxWords) return fail(SABER_ERANGE, "%s: a vocabulary of %lld words (limit 2^31 - 1)", who, (long long)c.vocab);
    OPS_TRY(check_stride(who, "x", c.x_stride, c.cols));
    OPS_TRY(check_stride(who, "weight", c.w_stride, c.cols));
    OPS_TRY(check_pointer(who, "weight", c.w, size_of(c.dtype)));
    if (c.rows) OPS_TRY(check_pointer(who, "x", c.x, size_of(c.dtype)));
    c.planes = c.dtype == SABER_F32 ? 3 : 1;
    c.pack_x = !direct(c.x, c.x_stride, c.cols, c.dtype);
    c.pack_w = !direct(c.w, c.w_stride, c.cols, c.dtype);
    c.cols_pad = up(c.cols, 8);
    return SABER_OK;
}

// The tile of a product of `steps` steps of 64 along k.  256 x 256 has twice the arithmetic per byte from LDS of 128 x 128 and four times
// that of 64 x 64, but takes a CU for itself; two of the second share one, four of the third, and then one's loads and stores go on beside
// the other's products.  Which ends first, in units of 0.1 us: rounds of workgroups times what a step and what a workgroup's two ends cost, and
// the first loads and last stores, which nothing hides.  Measured in us with 256, 128 and 64 in turn (bf16 but for the last; 250 x 5000
// in f32 has 12 steps), of products m x n by steps: 4096 x 32,768 by 16: 342, 362, -; 32,768 x 1024 by 64: 235, 287, -;
// 200 x 60,000 by 8: 33.7, 25.7, 35.4; 60,000 x 512 by 4: 37.6, 35.2, 49.6; 500 x 10,000 by 5: 28.3, 13.3, 14.8; 32 x 2000 by 8: 26.0,
// 11.5, 7.6; 250 x 5000 by 12: 41.4, 15.2, 10.9.
int tile_of(int64_t m, int64_t n, int64_t steps) {
    auto tiles = [&](int64_t t) { return parts_of(m, t) * parts_of(n, t); };
    const int64_t large = tiles(256), middle = tiles(128), small = tiles(64);
    const int64_t t256 = parts_of(large, kCus) * (18 * steps + 100) + 100;
    const int64_t t128 = middle <= kCus ? 8 * steps + 55 : parts_of(middle, 2 * kCus) * (11 * steps + 45) + 20;
    const int64_t t64 = small <= kCus ? 4 * steps + 35 : small <= 2 * kCus ? 6 * steps + 35 : parts_of(small, 4 * kCus) * (10 * steps + 20) + 35;
    return t64 < t128 && t64 < t256 ? 64 : t128 < t256 ? 128 : 256;
}

// Words of a piece, at most `most` (and 2^20: offsets within a tile are 32 bits), whole tiles.  Either all pieces are even, or all but
// the last fill the CUs with whole rounds of tiles: of d (words x rows), and of the weight's gradient (words x columns), whichever
// takes fewer rounds in all, the latter if they are alike.  (4,096 rows of 1,024 columns, 100,000 words, both passes: 36 rounds and 3.46 ms
// even, 32 and 3.30 ms the other way; 2,048 of 512 in binary32, 60,000 words: 12 rounds either way, 2.73 and 2.67 ms.)
int64_t piece_words(int64_t vocab, int64_t most, int64_t rows, int64_t cols) {
    if (most > (int64_t)1 << 20) most = (int64_t)1 << 20;
    most = most / 256 * 256;
    if (most < 256) most = 256;
    if (vocab <= most) return up(vocab, 8);
    const int64_t row_tiles = parts_of(rows, 256), col_tiles = parts_of(cols, 256);
    auto rounds = [&](int64_t words) {
        int64_t sum = 0;
        for (int64_t v0 = 0; v0 < vocab; v0 += words) {
            const int64_t tiles = parts_of(vocab - v0 < words ? vocab - v0 : words, 256);
            sum += parts_of(tiles * row_tiles, kCus) + parts_of(tiles * col_tiles, kCus);
        }
        return sum;
    };
    const int64_t even = up(parts_of(vocab, parts_of(vocab, most)), 256);
    const int64_t round = row_tiles <= kCus ? kCus / row_tiles * 256 : 256, filled = most / round * round;
    return filled > 0 && rounds(filled) <= rounds(even) ? filled : even;
}

int64_t few_lds(const Xent &c) { return c.rows * (up(c.cols, 32) * 2 + 16) * c.planes; }
bool few(const Xent &c) { return c.rows <= kFewRows && few_lds(c) <= kFewLds; }

struct Carve {   // a work space handed out piece by piece; base null: only counted
    char *base; int64_t at = 0;
    template <class T> T *take(int64_t n) {
        T *p = base ? reinterpret_cast<T *>(base + at) : nullptr;
        at += up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

struct ForwardSpace { float2 *partial; float *at; uint16_t *x, *w; int *x_powers, *w_powers; float *x_sums, *w_sums; int64_t piece, parts, rows_pad, few_grid; int tile, share_log; };
ForwardSpace forward_space(const Xent &c, Carve &s) {
    ForwardSpace f{};
    f.rows_pad = up(c.rows, 16);
    if (few(c)) {
        const int64_t tiles = parts_of(c.vocab, 16), each = 160 * 1024 / (few_lds(c) + 1024), most = kCus * (each > 4 ? 4 : each < 1 ? 1 : each);
        const int64_t batch = 32 * (c.planes == 3 ? kFewBatch<f32> : kFewBatch<bf16>);
        // few words: wavefronts share a tile's columns, as long as that leaves no CU with two workgroups (3 rows of 1912 in f32, 1000 words:
        // 58.9, 39.8, 28.1, 23.2 us with 1, 2, 4, 8 of them, both kernels; 16,400 words, where two would have to share a CU, 69.9 and 82.2)
        for (f.share_log = 0; 1 << f.share_log < kFewWaves && parts_of(tiles << (f.share_log + 1), kFewWaves) <= kCus && batch << f.share_log < c.cols;) ++f.share_log;
        const int64_t groups = parts_of(tiles << f.share_log, kFewWaves);
        f.few_grid = f.parts = groups < most ? groups : most;
    } else {
        const int64_t most = (kMaxTiles - 1) / parts_of(c.rows > 0 ? c.rows : 1, 64) * 64;   // words that one launch takes
        f.piece = c.pack_w ? piece_words(c.vocab, kPieceValues / (c.planes == 3 ? 2 : 1) / c.cols_pad, c.rows, c.cols) : c.vocab;
        if (f.piece > most) f.piece = most / 256 * 256;
        f.tile = tile_of(f.piece, c.rows, parts_of(c.cols, kStep) * (c.planes == 3 ? 3 : 1));
        f.parts = c.vocab / f.piece * parts_of(f.piece, f.tile) + parts_of(c.vocab % f.piece, f.tile);
        const int planes = c.planes == 3 ? 2 : 1;   // (the logits' form)
        if (c.pack_x) f.x = s.take<uint16_t>(c.rows * c.cols_pad * planes);
        if (c.pack_w) f.w = s.take<uint16_t>(f.piece * c.cols_pad * planes);
        if (planes == 2) {
            f.x_powers = s.take<int>(c.rows);
            f.w_powers = s.take<int>(f.piece);
            f.x_sums = s.take<float>(c.rows);
            f.w_sums = s.take<float>(f.piece);
        }
    }
    f.partial = s.take<float2>(f.parts * f.rows_pad);
    f.at = s.take<float>(f.rows_pad);
    return f;
}

struct BackwardSpace { GradScale *scale; uint32_t *most; int most_parts; uint16_t *x_plain, *x, *w, *d, *x_even, *w_even; int *x_powers, *w_powers; float *x_sums, *w_sums, *sums; int64_t piece, stride; int splits, dx_tile; };
BackwardSpace backward_space(const Xent &c, Carve &s) {
    BackwardSpace b{};
    const int64_t row = c.rows > 0 ? c.rows : 1, most_d = kPieceValues / c.planes / row, most_w = kPieceValues / (c.planes == 3 ? 5 : 1) / c.cols_pad;
    b.piece = piece_words(c.vocab, most_d < most_w ? most_d : most_w, row, c.cols);
    const int64_t steps = parts_of(b.piece, kStep) * (c.planes == 3 ? 6 : 1);
    // The features' gradient has few tiles and many steps, which are shared out until every CU has a workgroup: of the largest tiles
    // of which each still has 16 steps or more.
    b.dx_tile = 64;
    for (int tile : {256, 128}) {
        const int64_t tiles = parts_of(c.cols_pad, tile) * parts_of(row, tile);
        if (b.dx_tile == 64 && parts_of(kCus, tiles) <= steps / 16) b.dx_tile = tile;
    }
    while (b.dx_tile < 256 && parts_of(c.cols_pad, b.dx_tile) * parts_of(row, b.dx_tile) >= kMaxTiles) b.dx_tile *= 2;
    const int64_t tiles = parts_of(c.cols_pad, b.dx_tile) * parts_of(row, b.dx_tile);
    int64_t splits = kCus * (b.dx_tile == 256 ? 1 : 2) / tiles;
    if (splits > steps / 8) splits = steps / 8;
    if (splits < 1) splits = 1;
    b.splits = (int)splits;
    b.scale = s.take<GradScale>(1);
    if (c.dtype == SABER_F16) {
        b.most_parts = (int)(parts_of(row, 4) < kCus ? parts_of(row, 4) : kCus);
        b.most = s.take<uint32_t>(b.most_parts);
    }
    if (c.planes == 1 && c.pack_x) b.x_plain = s.take<uint16_t>(c.rows * c.cols_pad);
    b.x = s.take<uint16_t>(c.rows * c.cols_pad * c.planes);
    if (c.pack_w) b.w = s.take<uint16_t>(b.piece * c.cols_pad * c.planes);
    if (c.planes == 3) {   // the logits' form of both
        b.x_even = s.take<uint16_t>(c.rows * c.cols_pad * 2);
        b.w_even = s.take<uint16_t>(b.piece * c.cols_pad * 2);
        b.x_powers = s.take<int>(c.rows);
        b.w_powers = s.take<int>(b.piece);
        b.x_sums = s.take<float>(c.rows);
        b.w_sums = s.take<float>(b.piece);
    }
    b.stride = up(b.piece, 64) | 64;
    b.d = s.take<uint16_t>(c.rows * b.stride * c.planes);
    b.sums = s.take<float>(b.splits * c.rows * c.cols_pad);
    return b;
}

dim3 pack_grid(int64_t rows, const Xent &c) {
    const int64_t y = parts_of(rows, 4);
    return dim3((unsigned)parts_of(c.cols_pad, 512), (unsigned)(y < 32768 ? y : 32768));
}
template <class T>
int pack(const T *src, int64_t stride, int64_t rows, const Xent &c, uint16_t *dst, hipStream_t st) {
    pack_kernel<T><<<pack_grid(rows, c), 256, 0, st>>>(src, stride, rows, c.cols, dst, c.cols_pad);
    OPS_HIP(hipGetLastError());
    return SABER_OK;
}
int pack32(const Rows32 &x, const Rows32 &w, const Xent &c, hipStream_t st) {
    const int64_t groups = parts_of(x.rows + w.rows, 4);
    pack32_kernel<<<(unsigned)(groups < 16 * kCus ? groups : 16 * kCus), 256, 0, st>>>(x, w, c.cols, c.cols_pad);
    OPS_HIP(hipGetLastError());
    return SABER_OK;
}

template <class T, bool A_SLOW, bool B_SLOW, class E, class LeftOut = None>
int product(Operand a, Operand b, int64_t k, int segments, int splits, const E &e, hipStream_t st, int tile, const LeftOut &left_out = LeftOut{}) {
    Product p{a, b, (uint32_t)k, segments, 0, 0, splits};
    p.tiles_m = (int)parts_of(a.major, tile);
    p.tiles_n = (int)parts_of(b.major, tile);
    const int64_t grid = (int64_t)p.tiles_m * p.tiles_n * splits;
    if (grid >= kMaxTiles) return fail(SABER_ERANGE, "a product of %lld tiles", (long long)grid);
    if (tile == 256) product_kernel<T, A_SLOW, B_SLOW, 256, 256, 2, 2, E, LeftOut><<<(unsigned)grid, 256, 0, st>>>(p, e, left_out);
    else if (tile == 128) product_kernel<T, A_SLOW, B_SLOW, 128, 128, 2, 2, E, LeftOut><<<(unsigned)grid, 256, 0, st>>>(p, e, left_out);
    else product_kernel<T, A_SLOW, B_SLOW, 64, 64, 2, 2, E, LeftOut><<<(unsigned)grid, 256, 0, st>>>(p, e, left_out);
    OPS_HIP(hipGetLastError());
    if constexpr (std::is_same<LeftOut, Direct32>::value) {
        if (tile == 256) direct32_kernel<256, 256, 4, 2, E><<<(unsigned)grid, 512, 0, st>>>(p, e, left_out);
        else if (tile == 128) direct32_kernel<128, 128, 2, 2, E><<<(unsigned)grid, 256, 0, st>>>(p, e, left_out);
        else direct32_kernel<64, 64, 2, 2, E><<<(unsigned)grid, 256, 0, st>>>(p, e, left_out);
        OPS_HIP(hipGetLastError());
    }
    return SABER_OK;
}

// of the operands: of the gradients' products, of the logits'
template <class T> struct MatrixType { using type = T; using logits = T; };
template <> struct MatrixType<f32> { using type = bf16; using logits = f16; };

int check_targets(const char *who, const void *target, int target64) {
    return check_pointer(who, "target", target, target64 ? 8 : 4);
}

template <class T, int NT>
int launch_few(const Xent &c, const ForwardSpace &f, Targets t, hipStream_t st) {
    const int64_t least = kFewWaves * NT * (f.share_log ? 1024 : 128), lds = few_lds(c) > least ? few_lds(c) : least;   // the wavefronts' results at the end
    const auto kernel = score_few_kernel<T, NT>;
    if (lds > 64 * 1024) OPS_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    kernel<<<(unsigned)f.few_grid, kFewWaves * 64, (size_t)lds, st>>>(static_cast<const T *>(c.x), c.x_stride, static_cast<const T *>(c.w), c.w_stride, t, c.rows, c.vocab, c.cols, f.share_log, f.partial, f.rows_pad, f.at);
    OPS_HIP(hipGetLastError());
    return SABER_OK;
}

}  // namespace

extern "C" int saber_linear_xent_forward(const void *x, int64_t x_stride, const void *weight, int64_t w_stride, const void *target,
                                         int target64, int64_t rows, int64_t vocab, int64_t cols, int dtype, float *loss, float *lse,
                                         void *workspace, int64_t *workspace_bytes, void *stream) {
    const char *who = "saber_linear_xent_forward";
    Xent c{x, x_stride, weight, w_stride, rows, vocab, cols, dtype, 0, false, false, 0};
    OPS_TRY(check_xent(who, c));
    if (!workspace_bytes) return fail(SABER_EINVAL, "%s: workspace_bytes is null", who);
    Carve s{static_cast<char *>(workspace)};
    const ForwardSpace f = forward_space(c, s);
    if (!workspace) { *workspace_bytes = s.at; return SABER_OK; }
    if (!aligned(workspace, 256)) return fail(SABER_EINVAL, "%s: the work space is not aligned to 256 bytes", who);
    if (*workspace_bytes < s.at) return fail(SABER_EINVAL, "%s: work space of %lld bytes, %lld are needed", who, (long long)*workspace_bytes, (long long)s.at);
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_targets(who, target, target64));
    OPS_TRY(check_pointer(who, "loss", loss, 4));
    OPS_TRY(check_pointer(who, "lse", lse, 4));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const Targets t{target, target64};
    int64_t parts = 0;
    OPS_TRY(with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        using M = typename MatrixType<T>::logits;
        constexpr bool F32 = std::is_same<T, f32>::value;
        if (few(c)) {
            parts = f.parts;
            if (rows <= 16) return launch_few<T, 1>(c, f, t, st);
            if (rows <= 32) return launch_few<T, 2>(c, f, t, st);
            return launch_few<T, 4>(c, f, t, st);
        }
        const Targets none{nullptr, 0};
        const int64_t plane_x = rows * c.cols_pad, plane_w = f.piece * c.cols_pad;
        if constexpr (!F32)
            if (c.pack_x) OPS_TRY(pack(static_cast<const T *>(x), x_stride, rows, c, f.x, st));
        const Operand ox = c.pack_x ? Operand{f.x, c.cols_pad, plane_x, rows} : Operand{x, x_stride, 0, rows};
        for (int64_t v0 = 0; v0 < vocab; v0 += f.piece) {
            const int64_t words = vocab - v0 < f.piece ? vocab - v0 : f.piece;
            const T *w0 = static_cast<const T *>(weight) + v0 * w_stride;
            if constexpr (F32)
                OPS_TRY(pack32(Rows32{static_cast<const T *>(x), x_stride, v0 ? 0 : rows, nullptr, plane_x, f.x, f.x_powers, f.x_sums, none},
                               Rows32{w0, w_stride, words, nullptr, plane_w, f.w, f.w_powers, f.w_sums, none}, c, st));
            else if (c.pack_w) OPS_TRY(pack(w0, w_stride, words, c, f.w, st));
            const Operand ow = c.pack_w ? Operand{f.w, c.cols_pad, plane_w, words} : Operand{w0, w_stride, 0, words};
            const Powers powers{f.w_powers, f.x_powers};
            const ScoreEpilogue<F32> ep{f.partial, f.rows_pad, f.at, t, rows, words, v0, (int)parts, powers};
            if constexpr (F32) {
                const Direct32 direct{w0, w_stride, static_cast<const T *>(x), x_stride, f.w_sums, f.x_sums, powers};
                OPS_TRY((product<M, false, false>(ow, ox, cols, 3, 1, ep, st, f.tile, direct)));
            } else
                OPS_TRY((product<M, false, false>(ow, ox, cols, 1, 1, ep, st, f.tile)));
            parts += parts_of(words, f.tile);
        }
        return SABER_OK;
    }));
    score_join_kernel<<<(unsigned)parts_of(rows, 16), 1024, 0, st>>>(f.partial, f.rows_pad, (int)parts, f.at, t, rows, vocab, loss, lse);
    OPS_HIP(hipGetLastError());
    return SABER_OK;
}

extern "C" int saber_linear_xent_backward(const float *dloss, const void *x, int64_t x_stride, const void *weight, int64_t w_stride,
                                          const void *target, int target64, const float *lse, int64_t rows, int64_t vocab, int64_t cols,
                                          int dtype, void *dx, void *dweight, void *workspace, int64_t *workspace_bytes, void *stream) {
    const char *who = "saber_linear_xent_backward";
    Xent c{x, x_stride, weight, w_stride, rows, vocab, cols, dtype, 0, false, false, 0};
    OPS_TRY(check_xent(who, c));
    if (!workspace_bytes) return fail(SABER_EINVAL, "%s: workspace_bytes is null", who);
    Carve s{static_cast<char *>(workspace)};
    const BackwardSpace b = backward_space(c, s);
    if (parts_of(c.cols_pad, b.dx_tile) * parts_of(rows, b.dx_tile) * b.splits >= kMaxTiles)   // (features of 2^40 values)
        return fail(SABER_ERANGE, "%s: %lld rows of %lld columns", who, (long long)rows, (long long)cols);
    if (!workspace) { *workspace_bytes = s.at; return SABER_OK; }
    if (!aligned(workspace, 256)) return fail(SABER_EINVAL, "%s: the work space is not aligned to 256 bytes", who);
    if (*workspace_bytes < s.at) return fail(SABER_EINVAL, "%s: work space of %lld bytes, %lld are needed", who, (long long)*workspace_bytes, (long long)s.at);
    if (dx && rows) OPS_TRY(check_pointer(who, "dx", dx, size_of(dtype)));
    if (dweight) OPS_TRY(check_pointer(who, "dweight", dweight, size_of(dtype)));
    if (rows) {
        OPS_TRY(check_targets(who, target, target64));
        OPS_TRY(check_pointer(who, "dloss", dloss, 4));
        OPS_TRY(check_pointer(who, "lse", lse, 4));
    }
    if (!dweight && (!dx || !rows)) return SABER_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const Targets t{target, target64};
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        using M = typename MatrixType<T>::type;
        using L = typename MatrixType<T>::logits;
        constexpr bool F32 = std::is_same<T, f32>::value;
        constexpr int PLANES = F32 ? 3 : 1, SEGMENTS = F32 ? 6 : 1;
        const int64_t plane_x = rows * c.cols_pad, plane_w = b.piece * c.cols_pad, plane_d = rows * b.stride;
        if (rows == 0) {   // (a gradient of nothing: zeros)
            const int64_t n = vocab * cols, groups = parts_of(n, 2048);
            zeros_kernel<T><<<(unsigned)(groups < 16 * kCus ? groups : 16 * kCus), 256, 0, st>>>(static_cast<T *>(dweight), n);
            OPS_HIP(hipGetLastError());
            return SABER_OK;
        }
        const GradScale *scale = F32 ? nullptr : b.scale;   // (three planes keep all bits)
        if constexpr (!F32) {
            const T *from = static_cast<const T *>(x);
            if constexpr (std::is_same<T, f16>::value) {
                magnitude_kernel<T><<<b.most_parts, 256, 0, st>>>(from, x_stride, rows, cols, t, b.most);
                OPS_HIP(hipGetLastError());
            }
            grad_scale_kernel<<<1, 1024, 0, st>>>(dloss, t, rows, kGradTo<T>, b.most, b.most_parts, b.scale);
            OPS_HIP(hipGetLastError());
            pack_scaled_kernel<T><<<pack_grid(rows, c), 256, 0, st>>>(from, x_stride, rows, cols, b.x, c.cols_pad, t, dloss, scale);
            OPS_HIP(hipGetLastError());
            if (c.pack_x) OPS_TRY(pack(from, x_stride, rows, c, b.x_plain, st));
        }
        for (int64_t v0 = 0; v0 < vocab; v0 += b.piece) {
            const int64_t words = vocab - v0 < b.piece ? vocab - v0 : b.piece;
            const T *w0 = static_cast<const T *>(weight) + v0 * w_stride;
            T *dw = dweight ? static_cast<T *>(dweight) + v0 * cols : nullptr;
            if constexpr (F32)
                OPS_TRY(pack32(Rows32{static_cast<const T *>(x), x_stride, v0 ? 0 : rows, b.x, plane_x, b.x_even, b.x_powers, b.x_sums, t},
                               Rows32{w0, w_stride, words, b.w, plane_w, b.w_even, b.w_powers, b.w_sums, Targets{nullptr, 0}}, c, st));
            else if (c.pack_w) OPS_TRY(pack(w0, w_stride, words, c, b.w, st));
            const Operand ow = c.pack_w ? Operand{b.w, c.cols_pad, plane_w, words} : Operand{w0, w_stride, 0, words};
            const Operand ox = c.pack_x ? Operand{b.x_plain, c.cols_pad, 0, rows} : Operand{x, x_stride, 0, rows};
            const Powers powers{b.w_powers, b.x_powers};
            const GradEpilogue<M, PLANES> ep{reinterpret_cast<M *>(b.d), b.stride, plane_d, lse, dloss, scale, t, rows, words, v0, vocab, powers};
            const int tile = tile_of(words, rows, parts_of(cols, kStep) * (F32 ? 3 : 1));
            if constexpr (F32) {
                const Operand lw{b.w_even, c.cols_pad, plane_w, words}, lx{b.x_even, c.cols_pad, plane_x, rows};
                const Direct32 direct{w0, w_stride, static_cast<const T *>(x), x_stride, b.w_sums, b.x_sums, powers};
                OPS_TRY((product<L, false, false>(lw, lx, cols, 3, 1, ep, st, tile, direct)));
            } else
                OPS_TRY((product<L, false, false>(ow, ox, cols, 1, 1, ep, st, tile)));
            if (dx) {
                const SumEpilogue sum{b.sums, c.cols_pad, rows, c.cols_pad, v0 > 0};
                const Operand cw{ow.p, ow.stride, ow.plane, c.cols_pad}, od{b.d, b.stride, plane_d, rows};
                OPS_TRY((product<M, true, false>(cw, od, words, SEGMENTS, b.splits, sum, st, b.dx_tile)));
            }
            if (dweight) {
                const Operand cx{b.x, c.cols_pad, plane_x, c.cols_pad}, cd{b.d, b.stride, plane_d, up(words, 8)};
                const StoreEpilogue<T> store{dw, words, cols, scale};
                OPS_TRY((product<M, true, true>(cx, cd, rows, SEGMENTS, 1, store, st, tile_of(cols, words, parts_of(rows, kStep) * SEGMENTS))));
            }
        }
        if (dx) {
            sum_kernel<T><<<dim3((unsigned)parts_of(cols, 512), (unsigned)(rows < 16384 ? rows : 16384)), 256, 0, st>>>(b.sums, b.splits, rows, c.cols_pad, cols, t, dloss, scale, static_cast<T *>(dx));
            OPS_HIP(hipGetLastError());
        }
        return SABER_OK;
    });
}
