// Host side of the operators: errors, checks of arguments, work spaces.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "../../../include/saber_ops.h"
#include "ops_common.hpp"

namespace saber_ops {

inline thread_local char g_err[512] = "";
inline int fail(int code, const char *fmt, ...) {
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
constexpr int64_t kMaxTiles = (int64_t)1 << 24;   // (a launch has fewer than 2^32 threads)

inline size_t size_of(int type) { return type == SABER_F32 ? 4 : 2; }
inline bool is_type(int type) { return type == SABER_F32 || type == SABER_F16 || type == SABER_BF16; }
inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t parts_of(int64_t v, int64_t by) { return (v + by - 1) / by; }
inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// calls f(T{}) with the element type
template <class F>
int with_type(int type, F &&f) {
    if (type == SABER_F32) return f(f32{});
    if (type == SABER_F16) return f(f16{});
    return f(bf16{});
}

inline int check_rows(const char *who, int64_t rows, int64_t cols, int dtype) {
    if (!is_type(dtype)) return fail(SABER_EINVAL, "%s: unknown element type %d", who, dtype);
    if (rows < 0 || cols < 1) return fail(SABER_EINVAL, "%s: %lld rows of %lld columns", who, (long long)rows, (long long)cols);
    if (rows >= kMaxRows || cols > kMaxCols) return fail(SABER_ERANGE, "%s: %lld rows of %lld columns (limits 2^31 - 1 and 2^20)", who, (long long)rows, (long long)cols);
    return SABER_OK;
}
inline int check_stride(const char *who, const char *what, int64_t stride, int64_t cols) {
    if (stride < cols) return fail(SABER_EINVAL, "%s: rows of %s lie %lld elements apart, fewer than their %lld columns", who, what, (long long)stride, (long long)cols);
    if (stride > (int64_t)1 << 40) return fail(SABER_ERANGE, "%s: stride of %s", who, what);
    return SABER_OK;
}
inline int check_pointer(const char *who, const char *what, const void *p, size_t align) {
    if (!p) return fail(SABER_EINVAL, "%s: %s is null", who, what);
    if (!aligned(p, align)) return fail(SABER_EINVAL, "%s: %s is not aligned to its elements", who, what);
    return SABER_OK;
}
#define OPS_TRY(expr) do { const int rc_ = (expr); if (rc_ != SABER_OK) return rc_; } while (0)

struct Carve {   // a work space handed out piece by piece; base null: only counted
    char *base; int64_t at = 0;
    template <class T> T *take(int64_t n) {
        T *p = base ? reinterpret_cast<T *>(base + at) : nullptr;
        at += up(n * (int64_t)sizeof(T), 256);
        return p;
    }
};

}  // namespace saber_ops
