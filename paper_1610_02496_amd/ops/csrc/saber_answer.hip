// Host side of the operators of a head that answers (include/saber_ops.h): norm of the residual stream, rows in 8 bits and their
// product, words drawn from logits.  Checks of arguments, choice of a kernel's variant, launches; nothing here allocates, synchronises or
// keeps state between calls.
#include <type_traits>

#include "ops_host.hpp"
#include "ops_linear8.hpp"
#include "ops_rms.hpp"
#include "ops_sample.hpp"

using namespace saber_ops;

namespace {

// ---- root-mean-square norm ---------------------------------------------------------------------------------------------------

// Rows of up to 1,024 columns belong to a wavefront, up to 4,096 to a workgroup of 256, up to 8,192 to one of 512; wider ones are read again.  Rows of up
// to 2,048 belong to a wavefront as well (32 elements a lane), which needs no barrier, where the result is in 8 bits (rows in 8 bits of 65,536 x 2048 85 us
// with a wavefront, 140 with a workgroup, of 5000 10.3 and 13.4) and, where there are enough rows to keep the CUs busy with fewer of them:
//   forward from 24,000 rows on.  Times with a wavefront, relative to those with a workgroup, over ten widths and three pairs of types: 8192 rows 1.03 to
//     1.33, 16,384 0.93 to 1.17 (mean 1.02), 24,000 0.93 to 1.05 (0.99), 32,768 0.86 to 1.03, 65,536 0.81 to 1.00 (2048 columns in bf16, stream in binary32: 312
//     and 296 us);
//   backward from 40,000 rows of 1,600 columns on where the stream is in binary32.  The same, 1664 columns: 32,768 rows 1.01 to 1.02, 49,152 0.99, 65,536 0.97
//     to 0.98; 65,536 rows of 1030 1.10 to 1.28, of 1500 1.00 to 1.03, of 2048 0.94 to 0.95 (bf16 430 and 409 us).  With all in bf16 65,536 rows of 1500 take 1.29, of
//     1984 1.05, of 2047 1.06 and only those of 2048, where every lane has all its chunks, 0.94.
// 16,384 x 1024 in bf16 forward 21.5 us with a wavefront and 23.7, in 8 bits 21.5 and 42.5.
constexpr int64_t kRmsCols = 8192;
constexpr int64_t kForwardRows = 24000, kBackwardRows = 40000, kBackwardCols = 1600;

template <class F>
int with_rms_shape(int64_t cols, bool wavefront, F &&f) {
    using C1 = std::integral_constant<int, 1>; using C2 = std::integral_constant<int, 2>; using C4 = std::integral_constant<int, 4>;
    using W = std::integral_constant<int, 64>; using G = std::integral_constant<int, 256>; using GG = std::integral_constant<int, 512>;
    if (cols <= 512) return f(W{}, C1{});
    if (cols <= 1024) return f(W{}, C2{});
    if (cols <= 2048) return wavefront ? f(W{}, C4{}) : f(G{}, C1{});
    if (cols <= 4096) return f(G{}, C2{});
    return f(GG{}, C2{});
}
// workgroups for the rows that a workgroup has at a time: four if they belong to wavefronts
unsigned rms_grid(int64_t rows, int tpr) {
    const int64_t groups = parts_of(rows, tpr == 64 ? 4 : 1);
    return (unsigned)(groups < 8 * kCus ? groups : 8 * kCus);
}
unsigned wide_grid(int64_t rows) { return (unsigned)(rows < 64 * kCus ? rows : 64 * kCus); }
bool rms_backward_wavefront(int64_t rows, int64_t cols, int rtype) { return cols <= 1024 || (cols <= 2048 && cols >= kBackwardCols && rows >= kBackwardRows && rtype == SABER_F32); }
// workgroups of the backward pass, as many as the CUs hold at a time: each leaves a partial row
int64_t rms_parts(int64_t rows, int64_t cols, bool wavefront) {
    if (cols > kRmsCols) return rows < 256 ? (rows > 0 ? rows : 1) : 256;
    const int64_t groups = parts_of(rows > 0 ? rows : 1, wavefront ? 4 : 1);
    const int64_t most = (cols <= 1024 ? 3 : wavefront || cols > 4096 ? 2 : 4) * kCus;
    return groups < most ? groups : most;
}

// f(T{}, R{}): the type of the features, and of the stream, which is the same or binary32
template <class F>
int with_types(int dtype, int rtype, F &&f) {
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        if constexpr (!std::is_same<T, f32>::value)
            if (rtype == SABER_F32) return f(e, f32{});
        return f(e, e);
    });
}
int check_stream(const char *who, int dtype, int rtype, int wtype) {
    if (!is_type(wtype)) return fail(SABER_EINVAL, "%s: unknown type %d of weight", who, wtype);
    if (rtype != dtype && rtype != SABER_F32) return fail(SABER_EINVAL, "%s: the residual stream has the type of x or binary32, not type %d", who, rtype);
    return SABER_OK;
}
// rows of 8-bit values start at multiples of 16 bytes and go on with zeros to the next one
int check_rows8(const char *who, const char *what, const void *q, int64_t stride, int64_t cols) {
    OPS_TRY(check_stride(who, what, stride, cols));
    if (stride % 16) return fail(SABER_EINVAL, "%s: rows of %s lie %lld bytes apart, not a multiple of 16", who, what, (long long)stride);
    if (!q) return fail(SABER_EINVAL, "%s: %s is null", who, what);
    if (!aligned(q, 16)) return fail(SABER_EINVAL, "%s: %s is not aligned to 16 bytes", who, what);
    return SABER_OK;
}

}  // namespace

extern "C" int saber_rms_norm_forward(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const void *weight, int64_t rows,
                                      int64_t cols, int dtype, int rtype, int wtype, float eps, void *sum, void *y, float *rstd, int8_t *q,
                                      int64_t q_stride, float *scale, void *stream) {
    const char *who = "saber_rms_norm_forward";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    OPS_TRY(check_stream(who, dtype, rtype, wtype));
    OPS_TRY(check_stride(who, "x", x_stride, cols));
    if (residual) OPS_TRY(check_stride(who, "residual", residual_stride, cols));
    else if (rtype != dtype) return fail(SABER_EINVAL, "%s: a stream of another type without a residual", who);
    if (!(eps >= 0.f)) return fail(SABER_EINVAL, "%s: eps must not be negative", who);
    if (!q != !scale) return fail(SABER_EINVAL, "%s: q and scale are given together", who);
    if (rows == 0) return SABER_OK;
    if (!y == !q) return fail(SABER_EINVAL, "%s: either y or its form in 8 bits is wanted", who);
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    if (!residual != !sum) return fail(SABER_EINVAL, "%s: residual and sum are given together", who);
    if (residual) {
        OPS_TRY(check_pointer(who, "residual", residual, size_of(rtype)));
        OPS_TRY(check_pointer(who, "sum", sum, size_of(rtype)));
    }
    if (weight) OPS_TRY(check_pointer(who, "weight", weight, size_of(wtype)));
    if (y) OPS_TRY(check_pointer(who, "y", y, size_of(dtype)));
    if (rstd) OPS_TRY(check_pointer(who, "rstd", rstd, 4));
    if (q) {
        OPS_TRY(check_rows8(who, "q", q, q_stride, cols));
        OPS_TRY(check_pointer(who, "scale", scale, 4));
    }
    const RmsForward a{x, x_stride, residual, residual_stride, weight, wtype, rows, cols, eps, sum, y, rstd, q, q_stride, scale};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_types(dtype, rtype, [&](auto e, auto r) -> int {
        using T = decltype(e);
        using R = decltype(r);
        if (cols > kRmsCols) {
            if (q) rms_forward_wide_kernel<T, R, true><<<wide_grid(rows), 1024, 0, st>>>(a);
            else rms_forward_wide_kernel<T, R, false><<<wide_grid(rows), 1024, 0, st>>>(a);
        } else
            OPS_TRY(with_rms_shape(cols, q || rows >= kForwardRows, [&](auto tpr, auto nc) -> int {
                if (q) rms_forward_kernel<T, R, tpr.value, nc.value, true><<<rms_grid(rows, tpr.value), kRmsThreads<tpr.value>, 0, st>>>(a);
                else rms_forward_kernel<T, R, tpr.value, nc.value, false><<<rms_grid(rows, tpr.value), kRmsThreads<tpr.value>, 0, st>>>(a);
                return SABER_OK;
            }));
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

extern "C" int saber_rms_norm_backward_workspace(int64_t rows, int64_t cols, int64_t *bytes) {
    OPS_TRY(check_rows("saber_rms_norm_backward_workspace", rows, cols, SABER_F32));
    if (!bytes) return fail(SABER_EINVAL, "saber_rms_norm_backward_workspace: bytes is null");
    *bytes = rms_parts(rows, cols, cols <= 1024) * cols * 4;   // (wider rows that belong to a wavefront have fewer parts)
    return SABER_OK;
}

extern "C" int saber_rms_norm_backward(const void *dy, int64_t dy_stride, const void *dsum, int64_t dsum_stride, const void *s, int64_t s_stride,
                                       const float *rstd, const void *weight, int64_t rows, int64_t cols, int dtype, int rtype, int wtype, void *dx,
                                       void *dresidual, void *dweight, void *workspace, int64_t workspace_bytes, void *stream) {
    const char *who = "saber_rms_norm_backward";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    OPS_TRY(check_stream(who, dtype, rtype, wtype));
    OPS_TRY(check_stride(who, "dy", dy_stride, cols));
    OPS_TRY(check_stride(who, "s", s_stride, cols));
    if (dsum) OPS_TRY(check_stride(who, "dsum", dsum_stride, cols));
    if (dx) OPS_TRY(check_pointer(who, "dx", dx, size_of(dtype)));
    if (dresidual) OPS_TRY(check_pointer(who, "dresidual", dresidual, size_of(rtype)));
    if (dweight) OPS_TRY(check_pointer(who, "dweight", dweight, size_of(wtype)));
    if (weight) OPS_TRY(check_pointer(who, "weight", weight, size_of(wtype)));
    if (rows > 0) {
        OPS_TRY(check_pointer(who, "dy", dy, size_of(dtype)));
        OPS_TRY(check_pointer(who, "s", s, size_of(rtype)));
        if (dsum) OPS_TRY(check_pointer(who, "dsum", dsum, size_of(rtype)));
        OPS_TRY(check_pointer(who, "rstd", rstd, 4));
    }
    const bool wavefront = rms_backward_wavefront(rows, cols, rtype);
    const int64_t parts = rows > 0 ? rms_parts(rows, cols, wavefront) : 0;
    if (dweight && parts) {
        OPS_TRY(check_pointer(who, "workspace", workspace, 16));
        if (workspace_bytes < parts * cols * 4) return fail(SABER_EINVAL, "%s: work space of %lld bytes, %lld are needed", who, (long long)workspace_bytes, (long long)(parts * cols * 4));
    }
    if (!dweight && ((!dx && !dresidual) || rows == 0)) return SABER_OK;
    const RmsBackward a{dy, dy_stride, dsum, dsum_stride, s, s_stride, rstd, weight, wtype, rows, cols, dx, dresidual,
                        dweight ? static_cast<float *>(workspace) : nullptr, (int)parts};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows > 0)
        OPS_TRY(with_types(dtype, rtype, [&](auto e, auto r) -> int {
            using T = decltype(e);
            using R = decltype(r);
            if (cols > kRmsCols) {
                if (dx || dresidual) {
                    rms_backward_wide_kernel<T, R><<<wide_grid(rows), 1024, 0, st>>>(a);
                    OPS_HIP(hipGetLastError());
                }
                if (dweight) rms_columns_wide_kernel<T, R><<<dim3((unsigned)parts_of(cols, 2048), (unsigned)parts), 256, 0, st>>>(a);
            } else
                OPS_TRY(with_rms_shape(cols, wavefront, [&](auto tpr, auto nc) -> int {
                    rms_backward_kernel<T, R, tpr.value, nc.value><<<(unsigned)parts, kRmsThreads<tpr.value>, 0, st>>>(a);
                    return SABER_OK;
                }));
            OPS_HIP(hipGetLastError());
            return SABER_OK;
        }));
    if (dweight) {   // (no rows: zeros)
        rms_weight_kernel<<<(unsigned)parts_of(cols, 32), 1024, 0, st>>>(static_cast<const float *>(workspace), (int)parts, cols, dweight, wtype);
        OPS_HIP(hipGetLastError());
    }
    return SABER_OK;
}

// ---- rows in 8 bits and their product ----------------------------------------------------------------------------------------

extern "C" int saber_rows8_save(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int dtype, int8_t *q, int64_t q_stride, float *scale,
                                void *stream) {
    const char *who = "saber_rows8_save";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    OPS_TRY(check_stride(who, "x", x_stride, cols));
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    OPS_TRY(check_rows8(who, "q", q, q_stride, cols));
    OPS_TRY(check_pointer(who, "scale", scale, 4));
    const Rows8Save a{x, x_stride, rows, cols, q, q_stride, scale};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        if (cols > kRmsCols) rows8_save_wide_kernel<T><<<wide_grid(rows), 1024, 0, st>>>(a);
        else
            OPS_TRY(with_rms_shape(cols, true, [&](auto tpr, auto nc) -> int {
                rows8_save_kernel<T, tpr.value, nc.value><<<rms_grid(rows, tpr.value), kRmsThreads<tpr.value>, 0, st>>>(a);
                return SABER_OK;
            }));
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

extern "C" int saber_rows8_restore(const int8_t *q, int64_t q_stride, const float *scale, int64_t rows, int64_t cols, int dtype, void *x, void *stream) {
    const char *who = "saber_rows8_restore";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_rows8(who, "q", q, q_stride, cols));
    OPS_TRY(check_pointer(who, "scale", scale, 4));
    OPS_TRY(check_pointer(who, "x", x, size_of(dtype)));
    const int64_t chunks = parts_of(cols, 8), groups = parts_of(rows * chunks, 256), grid = groups < 16 * kCus ? groups : 16 * kCus;
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        rows8_restore_kernel<T><<<(unsigned)grid, 256, 0, static_cast<hipStream_t>(stream)>>>(q, q_stride, scale, rows, cols, static_cast<T *>(x), grid * 256 / chunks, grid * 256 % chunks);
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

namespace {

constexpr int64_t kMaxCols8 = ((int64_t)1 << 17) - 1;   // products of a sum in int32: each up to 2^14

// The tile of a product of `steps` steps of 128 columns: the rule of the 16-bit products, whose steps and ends take about as long.  Measured in
// us with 256, 128 and 64 in turn (bf16), runs of many calls: 8192 x 1000 x 141,000: 1597, 1694, 2579; 4096 x 1000 x 100,000: 570, 590, 938; 4096 x 777 x 30,011: 179, 165,
// 221; 300 x 777 x 30,011: 26.2, 20.9, 24.4; 61 x 777 x 30,011: 21.2, 9.6, 9.4; 1 x 1024 x 100,000: 41.7, 25.2, 20.9.
int tile8_of(int64_t m, int64_t n, int64_t steps) {
    auto tiles = [&](int64_t t) { return parts_of(m, t) * parts_of(n, t); };
    const int64_t large = tiles(256), middle = tiles(128), small = tiles(64);
    const int64_t t256 = parts_of(large, kCus) * (18 * steps + 100) + 100;
    const int64_t t128 = middle <= kCus ? 8 * steps + 55 : parts_of(middle, 2 * kCus) * (11 * steps + 45) + 20;
    const int64_t t64 = small <= kCus ? 4 * steps + 35 : small <= 2 * kCus ? 6 * steps + 35 : parts_of(small, 4 * kCus) * (10 * steps + 20) + 35;
    int tile = t64 < t128 && t64 < t256 ? 64 : t128 < t256 ? 128 : 256;
    while (tile < 256 && tiles(tile) >= kMaxTiles) tile *= 2;
    return tile;
}

}  // namespace

extern "C" int saber_linear8(const int8_t *x, int64_t x_stride, const float *x_scale, const int8_t *weight, int64_t w_stride, const float *w_scale,
                             int64_t rows, int64_t words, int64_t cols, int dtype, void *out, void *stream) {
    const char *who = "saber_linear8";
    OPS_TRY(check_rows(who, rows, cols, dtype));
    if (cols > kMaxCols8) return fail(SABER_ERANGE, "%s: %lld columns (limit 2^17 - 1)", who, (long long)cols);
    if (words < 1) return fail(SABER_EINVAL, "%s: a vocabulary of %lld words", who, (long long)words);
    if (words >= kMaxWords) return fail(SABER_ERANGE, "%s: a vocabulary of %lld words (limit 2^31 - 1)", who, (long long)words);
    OPS_TRY(check_rows8(who, "weight", weight, w_stride, cols));
    OPS_TRY(check_pointer(who, "w_scale", w_scale, 4));
    if (w_stride > (int64_t)1 << 21) return fail(SABER_ERANGE, "%s: stride of weight (limit 2^21)", who);
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_rows8(who, "x", x, x_stride, cols));
    if (x_stride > (int64_t)1 << 21) return fail(SABER_ERANGE, "%s: stride of x (limit 2^21)", who);
    OPS_TRY(check_pointer(who, "x_scale", x_scale, 4));
    OPS_TRY(check_pointer(who, "out", out, size_of(dtype)));
    const int tile = tile8_of(words, rows, parts_of(cols, 2 * kStep));
    // (two bytes are an element of the products' operands)
    Product p{{weight, w_stride / 2, 0, words}, {x, x_stride / 2, 0, rows}, (uint32_t)(up(cols, 16) / 2), 1, (int)parts_of(words, tile), (int)parts_of(rows, tile), 1};
    const int64_t grid = (int64_t)p.tiles_m * p.tiles_n;
    if (grid >= kMaxTiles) return fail(SABER_ERANGE, "%s: %lld rows of %lld words", who, (long long)rows, (long long)words);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        using E = Linear8Epilogue<T>;
        const E ep{static_cast<T *>(out), rows, words, x_scale, w_scale, words % 8 == 0 && aligned(out, 16)};
        if (tile == 256) product_kernel<Int8, false, false, 256, 256, 2, 2, E, None><<<(unsigned)grid, 256, 0, st>>>(p, ep, None{});
        else if (tile == 128) product_kernel<Int8, false, false, 128, 128, 2, 2, E, None><<<(unsigned)grid, 256, 0, st>>>(p, ep, None{});
        else product_kernel<Int8, false, false, 64, 64, 2, 2, E, None><<<(unsigned)grid, 256, 0, st>>>(p, ep, None{});
        OPS_HIP(hipGetLastError());
        return SABER_OK;
    });
}

// ---- words drawn from logits -------------------------------------------------------------------------------------------------

namespace {
constexpr int kFewTiles = 16, kManyTiles = 512;   // of 512 words or more
constexpr int64_t kMostRows = (int64_t)1 << 21;    // of a launch (of fewer than 2^32 threads)
// Threads of a workgroup: 256 for many short rows, of which a CU then holds four; 1,024 where there is a CU for every row and the row is long; else
// 512.  Measured in us with top_p 0.95, with 256, 512 and 1,024 in turn (256 where a row has no more tiles): bf16, 250 rows of 1000 20.2, 19.8, 21.7; 257 22.1,
// 23.2, 37.1; 1024 rows of 5000 33.7, 47.9, 77.8; with 512 and 1,024: 250 of 10,000 22.5, 22.8; of 20,000 26.8, 26.0; of 100,000 62.3, 52.3; 300 of 100,000 83.9,
// 97.5; 1024 156, 195; one row of 10,000 in binary32 21.2, 21.8; of 20,000 25.0, 24.1; of 100,000 56.8, 48.2; 2048 rows of 141,000 464, 574.
constexpr int64_t kFewWords = 20000;
}

extern "C" int saber_sample(const void *logits, int64_t stride, int64_t rows, int64_t words, int dtype, const float *u, const float *temperatures,
                            float temperature, const void *top_ks, int top_k64, int64_t top_k, const float *top_ps, float top_p, const float *min_ps,
                            float min_p, int64_t *word, float *p, void *stream) {
    const char *who = "saber_sample";
    if (!is_type(dtype)) return fail(SABER_EINVAL, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || words < 1) return fail(SABER_EINVAL, "%s: %lld rows of %lld words", who, (long long)rows, (long long)words);
    if (rows >= kMaxRows || words >= kMaxWords) return fail(SABER_ERANGE, "%s: %lld rows of %lld words (limits 2^31 - 1)", who, (long long)rows, (long long)words);
    OPS_TRY(check_stride(who, "logits", stride, words));
    if (!temperatures && !(temperature >= 0.f)) return fail(SABER_EINVAL, "%s: a temperature of %g", who, (double)temperature);
    if (!top_ks && top_k < 0) return fail(SABER_EINVAL, "%s: top_k must not be negative", who);
    if (!top_ps && !(top_p >= 0.f && top_p <= 1.f)) return fail(SABER_EINVAL, "%s: top_p must be within 0 and 1, not %g", who, (double)top_p);
    if (!min_ps && !(min_p >= 0.f && min_p <= 1.f)) return fail(SABER_EINVAL, "%s: min_p must be within 0 and 1, not %g", who, (double)min_p);
    if (rows == 0) return SABER_OK;
    OPS_TRY(check_pointer(who, "logits", logits, size_of(dtype)));
    OPS_TRY(check_pointer(who, "u", u, 4));
    if (temperatures) OPS_TRY(check_pointer(who, "temperatures", temperatures, 4));
    if (top_ks) OPS_TRY(check_pointer(who, "top_ks", top_ks, top_k64 ? 8 : 4));
    if (top_ps) OPS_TRY(check_pointer(who, "top_ps", top_ps, 4));
    if (min_ps) OPS_TRY(check_pointer(who, "min_ps", min_ps, 4));
    OPS_TRY(check_pointer(who, "word", word, 8));
    OPS_TRY(check_pointer(who, "p", p, 4));
    int bits = 0;
    while (((int64_t)1 << bits) < words) ++bits;
    Sample a{logits, stride, 0, words, u, temperatures, temperature, top_ks, top_k64, top_k, top_ps, top_p, min_ps, min_p, word, p, 0, bits < 17 ? 45 : 62 - bits};
    while (parts_of(words, (int64_t)512 << a.tile_log) > kManyTiles) ++a.tile_log;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return with_type(dtype, [&](auto e) -> int {
        using T = decltype(e);
        for (; a.first_row < rows; a.first_row += kMostRows) {
            const unsigned grid = (unsigned)(rows - a.first_row < kMostRows ? rows - a.first_row : kMostRows);
            if (rows > kCus && words <= 512 * kFewTiles) sample_kernel<T, 256, kFewTiles><<<grid, 256, 0, st>>>(a);
            else if (rows > kCus || words <= kFewWords) sample_kernel<T, 512, kManyTiles><<<grid, 512, 0, st>>>(a);
            else sample_kernel<T, 1024, kManyTiles><<<grid, 1024, 0, st>>>(a);
            OPS_HIP(hipGetLastError());
        }
        return SABER_OK;
    });
}
