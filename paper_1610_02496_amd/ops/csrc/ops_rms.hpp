// Root-mean-square norm of the residual stream (forward, backward), its output in 8 bits, and rows held in 8 bits.
//
//   s = x + residual, rounded to the stream's type;  r = 1/sqrt(1/H sum s^2 + eps),  h = s r,  y = h w
//   ds = r (g - h mean(g h)) + dsum  with g = dy w,   dw = sum over rows of dy h
//   in 8 bits: t = s w (binary32), c = max|t| / 127, q = round(t / c), ties to even; y is held as q c r
//
// The norm is of the sum as it is held, so that the backward pass, which reads that, has the gradient of what the forward pass
// computed.  r scales all of a row, so that the whole numbers q do not depend on it.  All sums are binary32.
//
// What bounds it: memory.  Every operand is read once and kept in registers, the next row's are asked for before this one's are worked on.  65,536 x 2048 in
// bf16 with the stream in binary32: forward 295 us (5.5 TB/s), backward 407 (5.3); 32,768 x 4096 in binary16 to 8 bits 176 to 190 (5 TB/s), back 66.
#pragma once
#include "ops_common.hpp"

namespace saber_ops {

struct RmsForward {
    const void *x; int64_t x_stride;
    const void *res; int64_t res_stride;    // or null: the norm is of x
    const void *weight; int wtype;
    int64_t rows, cols; float eps;
    void *sum, *y; float *rstd;             // sum: with res; rstd: or null
    int8_t *q; int64_t q_stride; float *scale;   // in place of y
};
struct RmsBackward {
    const void *dy; int64_t dy_stride;
    const void *dsum; int64_t dsum_stride;  // or null: nothing
    const void *s; int64_t s_stride;
    const float *rstd;
    const void *weight; int wtype;
    int64_t rows, cols;
    void *dx, *dres;                        // of the types of dy and of s; either may be null
    float *partial; int parts;              // [parts][cols]: sums of dy h over a workgroup's rows; null: not wanted
};
struct Rows8Save {
    const void *x; int64_t x_stride, rows, cols;
    int8_t *q; int64_t q_stride; float *scale;
};

template <class T>
__device__ __forceinline__ f32x8 rounded(f32x8 v) {
    if constexpr (sizeof(T) == 4) return v;
    else {
        typedef T V __attribute__((ext_vector_type(8)));
        return __builtin_convertvector(__builtin_convertvector(v, V), f32x8);
    }
}
__device__ __forceinline__ f32x8 zeros8() { return f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// largest magnitude of a chunk, as bits (NaN above infinity)
__device__ __forceinline__ uint32_t magnitude(f32x8 v) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    return top;
}
// A row's step: 127 of it are finite if the row is; not finite if it is not.
__device__ __forceinline__ float step_of(uint32_t top) {
    const float step = __uint_as_float(top) / 127.f;
    return top < 0x7f800000u ? fminf(step, 0x1.020406p+121f) : step;
}

// A sum and a largest value over the TPR threads of a row, the same in all of them.  One barrier: `slot` alternates from row to row, so that
// nobody writes what another still reads.
template <int TPR, bool TOP>
__device__ __forceinline__ void row_join(float &sum, uint32_t &top, float *lds, int slot) {
    sum = wave_sum(sum);
    if constexpr (TOP) top = wave_max(top);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        float *at = lds + slot * 2 * W;
        if ((threadIdx.x & 63) == 0) {
            at[threadIdx.x >> 6] = sum;
            if constexpr (TOP) at[W + (threadIdx.x >> 6)] = __uint_as_float(top);
        }
        __syncthreads();
        sum = 0.f;
        top = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            sum += at[i];
            if constexpr (TOP) top = max(top, __float_as_uint(at[W + i]));
        }
    }
}

// 1 / sqrt(ss / H + eps).  A sum of squares beyond binary32 is taken again of 2^-80 s, next to which eps is nothing; one below 2^-100, where
// squares are no normal numbers, of 2^90 s, unless eps is more than that.  (Without eps a row of zeros has the largest finite r, and stays zeros.)
__device__ __forceinline__ float rstd_of(float ss, float inv, float eps) { return 1.f / sqrtf(ss * inv + eps); }
__device__ __forceinline__ float scale_of_sum(float ss, float eps) { return !(ss < INFINITY) ? 0x1p-80f : ss < 0x1p-100f && eps < 0x1p-100f ? 0x1p90f : 0.f; }
__device__ __forceinline__ float rstd_of_scaled(float ss, float inv, float eps, float by) {
    if (by < 1.f) return by / sqrtf(ss * inv);
    return fminf(by / sqrtf(ss * inv + eps * by * by), 0x1.fffffep127f);
}

template <int TPR> constexpr int kRmsThreads = TPR > 256 ? TPR : 256;   // of a workgroup

// A row per wavefront (TPR = 64) or per workgroup; a lane holds NC chunks of eight columns of its row in registers, so that every
// operand is read once, and asks for the next row before it works on this one.
template <class T, class R, int TPR, int NC, bool HELD8>
__global__ __launch_bounds__(kRmsThreads<TPR>) void rms_forward_kernel(RmsForward a) {
    __shared__ float lds[5 * (TPR / 64)];
    constexpr int RPB = kRmsThreads<TPR> / TPR;
    const int t = threadIdx.x % TPR;
    const int64_t H = a.cols;
    f32x8 w[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int64_t c = (int64_t)(j * TPR + t) * 8;
        w[j] = load8_as(a.weight, a.wtype, c, H - c, 1.f);
    }
    const float inv = 1.f / (float)H;
    const int64_t step_rows = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Raw8<T> raw_x[NC];
    Raw8<R> raw_r[NC];
    auto ask = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            raw_x[j] = load_raw8(static_cast<const T *>(a.x) + r * a.x_stride + c, H - c);
            if (a.res) raw_r[j] = load_raw8(static_cast<const R *>(a.res) + r * a.res_stride + c, H - c);
        }
    };
    if (row < a.rows) ask(row);
    for (int slot = 0; row < a.rows; row += step_rows, slot ^= 1) {
        f32x8 v[NC];
        float ss = 0.f;
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            v[j] = widen(raw_x[j]);
            if (a.res) v[j] = rounded<R>(v[j] + widen(raw_r[j]));
        }
        if (row + step_rows < a.rows) ask(row + step_rows);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            if (a.res) store8(static_cast<R *>(a.sum) + row * H + c, H - c, v[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(v[j][i], v[j][i], ss);
            if constexpr (HELD8) top = max(top, magnitude(v[j] * w[j]));
        }
        row_join<TPR, HELD8>(ss, top, lds, slot);
        float rstd = rstd_of(ss, inv, a.eps);
        if (const float by = scale_of_sum(ss, a.eps); by != 0.f) {
            ss = 0.f;
#pragma unroll
            for (int j = 0; j < NC; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(v[j][i] * by, v[j][i] * by, ss);
            ss = row_sum<TPR>(ss, lds + 4 * (TPR / 64), 0);
            rstd = rstd_of_scaled(ss, inv, a.eps, by);
        }
        if constexpr (HELD8) {
            const float step = step_of(top);
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t c = (int64_t)(j * TPR + t) * 8;
                Bytes8 q;
                whole8<true>(v[j] * w[j], step, q);
                if (c < (H + 15) / 16 * 16) *reinterpret_cast<Bytes8 *>(a.q + row * a.q_stride + c) = q;   // (zeros past the row's end)
            }
            if (t == 0) a.scale[row] = step * rstd;
        } else {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t c = (int64_t)(j * TPR + t) * 8;
                store8(static_cast<T *>(a.y) + row * H + c, H - c, v[j] * rstd * w[j]);
            }
        }
        if (t == 0 && a.rstd) a.rstd[row] = rstd;
    }
}

// The same layout.  Every lane keeps the sums of dy h of its columns over the rows it sees; a workgroup's wavefronts add theirs in
// LDS and write one partial row, which rms_weight_kernel adds up in a fixed order (no atomics: the same result every time).
template <class T, class R, int TPR, int NC>
__global__ __launch_bounds__(kRmsThreads<TPR>) void rms_backward_kernel(RmsBackward a) {
    constexpr int RPB = kRmsThreads<TPR> / TPR;
    __shared__ float lds[4 * (TPR / 64)];
    __shared__ float sums[RPB > 1 ? 64 * NC * 8 : 1];
    const int t = threadIdx.x % TPR;
    const int64_t H = a.cols;
    f32x8 w[NC], dw[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int64_t c = (int64_t)(j * TPR + t) * 8;
        w[j] = load8_as(a.weight, a.wtype, c, H - c, 1.f);
        dw[j] = zeros8();
    }
    const float inv = 1.f / (float)H;
    const int64_t step_rows = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Raw8<T> raw_g[NC];
    Raw8<R> raw_s[NC], raw_d[NC];
    float raw_rstd = 0.f;
    auto ask = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            raw_g[j] = load_raw8(static_cast<const T *>(a.dy) + r * a.dy_stride + c, H - c);
            raw_s[j] = load_raw8(static_cast<const R *>(a.s) + r * a.s_stride + c, H - c);
            if (a.dsum) raw_d[j] = load_raw8(static_cast<const R *>(a.dsum) + r * a.dsum_stride + c, H - c);
        }
        raw_rstd = a.rstd[r];
    };
    if (row < a.rows) ask(row);
    for (int slot = 0; row < a.rows; row += step_rows, slot ^= 1) {
        f32x8 h[NC], g[NC], d[NC];
        const float rstd = raw_rstd;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            g[j] = widen(raw_g[j]);
            h[j] = widen(raw_s[j]);
            d[j] = a.dsum ? widen(raw_d[j]) : zeros8();
        }
        if (row + step_rows < a.rows) ask(row + step_rows);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {   // (past the row's end all are zeros)
                h[j][i] *= rstd;
                dw[j][i] = fmaf(g[j][i], h[j][i], dw[j][i]);
                g[j][i] *= w[j][i];
                s = fmaf(g[j][i], h[j][i], s);
            }
        if (!a.dx && !a.dres) continue;
        uint32_t none = 0;
        row_join<TPR, false>(s, none, lds, slot);
        s *= inv;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            f32x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(rstd, fmaf(-h[j][i], s, g[j][i]), d[j][i]);
            if (a.dx) store8(static_cast<T *>(a.dx) + row * H + c, H - c, o);
            if (a.dres) store8(static_cast<R *>(a.dres) + row * H + c, H - c, o);
        }
    }
    if (!a.partial) return;
    float *out = a.partial + (int64_t)blockIdx.x * H;
    if constexpr (RPB > 1) {
        for (int wv = 0; wv < RPB; ++wv) {
            __syncthreads();
            if ((int)(threadIdx.x / TPR) == wv) {
#pragma unroll
                for (int j = 0; j < NC; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int at = (j * 8 + i) * 64 + t;
                        sums[at] = wv ? sums[at] + dw[j][i] : dw[j][i];
                    }
            }
        }
        __syncthreads();
        for (int64_t c = threadIdx.x; c < H; c += kRmsThreads<TPR>) {
            const int chunk = (int)(c >> 3);
            out[c] = sums[((chunk / 64) * 8 + (int)(c & 7)) * 64 + chunk % 64];
        }
    } else {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            store8(out + c, H - c, dw[j]);
        }
    }
}

// dw of 32 columns per workgroup: 32 lanes across the columns, 32 groups that each take every 32nd partial row.
__global__ __launch_bounds__(1024) void rms_weight_kernel(const float *partial, int parts, int64_t cols, void *dweight, int wtype) {
    __shared__ float lds[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int grp = threadIdx.x / 32;
    float s = 0.f;
    if (c < cols) {
        const float *from = partial + c;
        int p = grp;
        for (; p + 7 * 32 < parts; p += 8 * 32) {   // eight on their way at a time
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from[(int64_t)(p + i * 32) * cols];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; p < parts; p += 32) s += from[(int64_t)p * cols];
    }
    lds[grp][threadIdx.x % 32] = s;
    __syncthreads();
    if (grp == 0 && c < cols) {
        for (int i = 1; i < 32; ++i) s += lds[i][threadIdx.x];
        store_as(dweight, wtype, c, s);
    }
}

// Rows too wide for registers: a workgroup of 1,024 goes over its row a second time, from the caches.  A thread reads again only what it
// wrote itself.
template <class T, class R, bool HELD8>
__global__ __launch_bounds__(1024) void rms_forward_wide_kernel(RmsForward a) {
    __shared__ float lds[5 * 16];
    const int64_t H = a.cols;
    const float inv = 1.f / (float)H;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, slot ^= 1) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        R *sum = static_cast<R *>(a.sum) + row * H;
        float ss = 0.f;
        uint32_t top = 0;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
            f32x8 v = load8(x + c, H - c);
            if (a.res) {
                v = rounded<R>(v + load8(static_cast<const R *>(a.res) + row * a.res_stride + c, H - c));
                store8(sum + c, H - c, v);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
            if constexpr (HELD8) top = max(top, magnitude(v * load8_as(a.weight, a.wtype, c, H - c, 1.f)));
        }
        row_join<1024, HELD8>(ss, top, lds, slot);
        auto again = [&](int64_t c) { return a.res ? load8(static_cast<const R *>(sum) + c, H - c) : load8(x + c, H - c); };
        float rstd = rstd_of(ss, inv, a.eps);
        if (const float by = scale_of_sum(ss, a.eps); by != 0.f) {
            ss = 0.f;
            for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
                const f32x8 v = again(c);
#pragma unroll
                for (int i = 0; i < 8; ++i) ss = fmaf(v[i] * by, v[i] * by, ss);
            }
            ss = row_sum<1024>(ss, lds + 4 * 16, 0);
            rstd = rstd_of_scaled(ss, inv, a.eps, by);
        }
        const float step = HELD8 ? step_of(top) : 0.f;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < (HELD8 ? (H + 15) / 16 * 16 : H); c += 8192) {
            const f32x8 v = again(c), w = load8_as(a.weight, a.wtype, c, H - c, 1.f);
            if constexpr (HELD8) {
                Bytes8 q;
                whole8<true>(v * w, step, q);
                *reinterpret_cast<Bytes8 *>(a.q + row * a.q_stride + c) = q;
            } else
                store8(static_cast<T *>(a.y) + row * H + c, H - c, v * rstd * w);
        }
        if (threadIdx.x == 0) {
            if (a.rstd) a.rstd[row] = rstd;
            if constexpr (HELD8) a.scale[row] = step * rstd;
        }
    }
}

template <class T, class R>
__global__ __launch_bounds__(1024) void rms_backward_wide_kernel(RmsBackward a) {
    __shared__ float lds[4 * 16];
    const int64_t H = a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, slot ^= 1) {
        const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
        const R *in = static_cast<const R *>(a.s) + row * a.s_stride;
        const float rstd = a.rstd[row];
        float s = 0.f;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
            const f32x8 g = load8(dy + c, H - c) * load8_as(a.weight, a.wtype, c, H - c, 1.f), h = load8(in + c, H - c) * rstd;
#pragma unroll
            for (int i = 0; i < 8; ++i) s = fmaf(g[i], h[i], s);
        }
        uint32_t none = 0;
        row_join<1024, false>(s, none, lds, slot);
        s /= (float)H;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
            const f32x8 g = load8(dy + c, H - c) * load8_as(a.weight, a.wtype, c, H - c, 1.f), h = load8(in + c, H - c) * rstd;
            f32x8 o = a.dsum ? load8(static_cast<const R *>(a.dsum) + row * a.dsum_stride + c, H - c) : zeros8();
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(rstd, fmaf(-h[i], s, g[i]), o[i]);
            if (a.dx) store8(static_cast<T *>(a.dx) + row * H + c, H - c, o);
            if (a.dres) store8(static_cast<R *>(a.dres) + row * H + c, H - c, o);
        }
    }
}

// Partial sums for such rows: a workgroup takes 2,048 columns (grid.x) of every parts-th row (grid.y).
template <class T, class R>
__global__ __launch_bounds__(256) void rms_columns_wide_kernel(RmsBackward a) {
    const int64_t H = a.cols, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (c >= H) return;
    f32x8 dw = zeros8();
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const f32x8 g = load8(static_cast<const T *>(a.dy) + row * a.dy_stride + c, H - c);
        const f32x8 h = load8(static_cast<const R *>(a.s) + row * a.s_stride + c, H - c) * a.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[i] = fmaf(g[i], h[i], dw[i]);
    }
    store8(a.partial + (int64_t)blockIdx.y * H + c, H - c, dw);
}

// ---- rows in 8 bits ----------------------------------------------------------------------------------------------------------

// A row per wavefront or workgroup, as above.
template <class T, int TPR, int NC>
__global__ __launch_bounds__(kRmsThreads<TPR>) void rows8_save_kernel(Rows8Save a) {
    __shared__ float lds[4 * (TPR / 64)];
    constexpr int RPB = kRmsThreads<TPR> / TPR;
    const int t = threadIdx.x % TPR;
    const int64_t H = a.cols;
    const int64_t step_rows = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Raw8<T> raw[NC];
    auto ask = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            raw[j] = load_raw8(static_cast<const T *>(a.x) + r * a.x_stride + c, H - c);
        }
    };
    if (row < a.rows) ask(row);
    for (int slot = 0; row < a.rows; row += step_rows, slot ^= 1) {
        f32x8 v[NC];
        uint32_t top = 0;
        float none = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            v[j] = widen(raw[j]);
            top = max(top, magnitude(v[j]));
        }
        if (row + step_rows < a.rows) ask(row + step_rows);
        row_join<TPR, true>(none, top, lds, slot);
        const float step = step_of(top);
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            Bytes8 q;
            whole8<true>(v[j], step, q);
            if (c < (H + 15) / 16 * 16) *reinterpret_cast<Bytes8 *>(a.q + row * a.q_stride + c) = q;
        }
        if (t == 0) a.scale[row] = step;
    }
}
template <class T>
__global__ __launch_bounds__(1024) void rows8_save_wide_kernel(Rows8Save a) {
    __shared__ float lds[4 * 16];
    const int64_t H = a.cols;
    int slot = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x, slot ^= 1) {
        const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
        uint32_t top = 0;
        float none = 0.f;
        for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) top = max(top, magnitude(load8(x + c, H - c)));
        row_join<1024, true>(none, top, lds, slot);
        const float step = step_of(top);
        for (int64_t c = (int64_t)threadIdx.x * 8; c < (H + 15) / 16 * 16; c += 8192) {
            Bytes8 q;
            whole8<true>(load8(x + c, H - c), step, q);
            *reinterpret_cast<Bytes8 *>(a.q + row * a.q_stride + c) = q;
        }
        if (threadIdx.x == 0) a.scale[row] = step;
    }
}

// eight values per lane, rows and chunks of a row in one stride without a division in the loop
template <class T>
__global__ __launch_bounds__(256) void rows8_restore_kernel(const int8_t *q, int64_t q_stride, const float *scale, int64_t rows, int64_t cols, T *x,
                                                            int64_t step_rows, int64_t step_chunks) {
    const int64_t chunks = (cols + 7) / 8, first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int64_t row = first / chunks, chunk = first - row * chunks;
    while (row < rows) {
        const int64_t c = chunk * 8;
        store8(x + row * cols + c, cols - c, widen_q(*reinterpret_cast<const Bytes8 *>(q + row * q_stride + c), scale[row]));
        row += step_rows; chunk += step_chunks;
        if (chunk >= chunks) { chunk -= chunks; ++row; }
    }
}

}  // namespace saber_ops
