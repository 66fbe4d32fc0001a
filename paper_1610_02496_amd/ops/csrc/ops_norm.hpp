// Layer norm (forward, backward, reduction of the weight's and bias's gradients) and 8-bit checkpoints.
//
//   m = 1/H sum x,  v = 1/H sum (x - m)^2,  r = 1/sqrt(v + eps),  h = (x - m) r,  y = h w + b
//   dx = r (g - mean(g) - h mean(g h)) with g = dy w,   dw = sum over rows of dy h,   db = sum over rows of dy
//
// All sums are binary32.  The variance is taken about the mean that the row has (second pass over registers), not as a
// difference of moments.
#pragma once
#include "ops_common.hpp"

namespace saber_ops {

struct NormForward {
    const void *x; int64_t x_stride;
    const void *weight, *bias; int wtype;
    int64_t rows, cols; float eps;
    void *y; float *mean, *rstd;
    int8_t *q; float *scale;      // checkpoint of x, or null
};
struct NormBackward {
    const void *dy; int64_t dy_stride;
    const void *x; int64_t x_stride;
    const int8_t *q; const float *scale;   // in place of x
    const float *mean, *rstd;
    const void *weight; int wtype;
    int64_t rows, cols;
    void *dx;
    float *partial; int parts;    // [parts][2][cols]: sums of dy h and of dy over a workgroup's rows; null: not wanted
};

// sum over the TPR threads of a row, the same value in all of them; `slot` alternates between calls so that one barrier is
// enough
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *lds, int slot) {
    v = wave_sum(v);
    if constexpr (TPR == 64) return v;
    else {
        constexpr int W = TPR / 64;
        if ((threadIdx.x & 63) == 0) lds[slot * W + (threadIdx.x >> 6)] = v;
        __syncthreads();
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) s += lds[slot * W + i];
        return s;
    }
}

// A row per wavefront (TPR = 64) or per workgroup (TPR = 256, 512); a lane holds NC chunks of eight columns of its row in registers, so
// that x is read once.  A workgroup goes over several rows, keeps weight and bias in registers, and asks for a row before it works on the one
// before.  Memory bounds it: 65,536 x 2048 in f16 (537 MB read and written) 98 us, 5.5 TB/s; 16,384 x 1024 in bf16 with the checkpoint
// (84 MB) 24 us, 3.5 TB/s.  A single row of 1000 takes 3.6 us.
template <int TPR> constexpr int kNormThreads = TPR > 256 ? TPR : 256;   // of a workgroup

template <class T, int TPR, int NC, bool SAVE8>
__global__ __launch_bounds__(kNormThreads<TPR>) void norm_forward_kernel(NormForward a) {
    __shared__ float lds[2 * (TPR / 64)];
    constexpr int RPB = kNormThreads<TPR> / TPR;
    const int t = threadIdx.x % TPR;
    const int64_t H = a.cols;
    f32x8 w[NC], b[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int64_t c = (int64_t)(j * TPR + t) * 8;
        w[j] = load8_as(a.weight, a.wtype, c, H - c, 1.f);
        b[j] = load8_as(a.bias, a.wtype, c, H - c, 0.f);
    }
    const float inv = 1.f / (float)H;
    const int64_t step_rows = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Raw8<T> raw[NC];   // of the row to come
    auto ask = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            raw[j] = load_raw8(static_cast<const T *>(a.x) + r * a.x_stride + c, H - c);
        }
    };
    if (row < a.rows) ask(row);
    for (; row < a.rows; row += step_rows) {
        f32x8 v[NC];
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) v[j] = widen(raw[j]);
        if (row + step_rows < a.rows) ask(row + step_rows);
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[j][i];
        if constexpr (SAVE8) {
            const int64_t nb = (H + kBlock - 1) / kBlock;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t c = (int64_t)(j * TPR + t) * 8;
                Bytes8 q;
                const float step = quantise8(v[j], q);
                if (c < H) {
                    store_q(a.q + row * H + c, H - c, q);
                    if ((t & 15) == 0) a.scale[row * nb + c / kBlock] = step;
                }
            }
        }
        const float mean = row_sum<TPR>(s, lds, 0) * inv;
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[j][i] -= mean;
                ss += c + i < H ? v[j][i] * v[j][i] : 0.f;
            }
        }
        const float rstd = 1.f / sqrtf(row_sum<TPR>(ss, lds, 1) * inv + a.eps);
        T *y = static_cast<T *>(a.y) + row * H;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            f32x8 o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = fmaf(v[j][i] * rstd, w[j][i], b[j][i]);
            store8(y + c, H - c, o);
        }
        if (t == 0) {
            a.mean[row] = mean;
            a.rstd[row] = rstd;
        }
    }
}

// The same layout.  Every lane keeps the sums of dy h and dy of its columns over the rows it sees; a workgroup's wavefronts add
// theirs in LDS and write one partial row, which norm_weight_kernel adds up in a fixed order (no atomics: the same result every time).
// Bound by memory: 65,536 x 2048 in f16 (805 MB) 157 us, 5.1 TB/s; 16,384 x 1024 in bf16 from the checkpoint (84 MB) 21 us, 4.0 TB/s.
template <class T, int TPR, int NC, bool IN8>
__global__ __launch_bounds__(kNormThreads<TPR>) void norm_backward_kernel(NormBackward a) {
    constexpr int RPB = kNormThreads<TPR> / TPR;
    __shared__ float lds[4 * (TPR / 64)];
    __shared__ float sums[RPB > 1 ? 64 * NC * 8 : 1];
    const int t = threadIdx.x % TPR;
    const int64_t H = a.cols;
    f32x8 w[NC], dw[NC], db[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
        const int64_t c = (int64_t)(j * TPR + t) * 8;
        w[j] = load8_as(a.weight, a.wtype, c, H - c, 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[j][i] = db[j][i] = 0.f;
    }
    const float inv = 1.f / (float)H;
    const int64_t nb = (H + kBlock - 1) / kBlock;
    const int64_t step_rows = (int64_t)gridDim.x * RPB;
    int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    Raw8<T> raw_g[NC], raw_x[IN8 ? 1 : NC];   // of the row to come
    Bytes8 raw_q[IN8 ? NC : 1];
    float raw_step[IN8 ? NC : 1], raw_mean = 0.f, raw_rstd = 0.f;
    auto ask = [&](int64_t r) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
            raw_g[j] = load_raw8(static_cast<const T *>(a.dy) + r * a.dy_stride + c, H - c);
            if constexpr (IN8) {
                raw_q[j] = load_raw_q(a.q + r * H + c, H - c);
                raw_step[j] = c < H ? a.scale[r * nb + c / kBlock] : 0.f;
            } else
                raw_x[j] = load_raw8(static_cast<const T *>(a.x) + r * a.x_stride + c, H - c);
        }
        raw_mean = a.mean[r]; raw_rstd = a.rstd[r];
    };
    if (row < a.rows) ask(row);
    for (; row < a.rows; row += step_rows) {
        f32x8 h[NC], g[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            g[j] = widen(raw_g[j]);
            if constexpr (IN8) h[j] = widen_q(raw_q[j], raw_step[j]);
            else h[j] = widen(raw_x[j]);
        }
        const float mean = raw_mean, rstd = raw_rstd;
        if (row + step_rows < a.rows) ask(row + step_rows);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const int64_t c = (int64_t)(j * TPR + t) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) {   // past the row's end: g = 0 already, h is made 0
                h[j][i] = c + i < H ? (h[j][i] - mean) * rstd : 0.f;
                dw[j][i] = fmaf(g[j][i], h[j][i], dw[j][i]);
                db[j][i] += g[j][i];
                g[j][i] *= w[j][i];
                s1 += g[j][i];
                s2 = fmaf(g[j][i], h[j][i], s2);
            }
        }
        if (a.dx) {
            if constexpr (TPR == 64) { s1 = wave_sum(s1) * inv; s2 = wave_sum(s2) * inv; }
            else {
                constexpr int W = TPR / 64;
                s1 = wave_sum(s1); s2 = wave_sum(s2);
                __syncthreads();   // the row before has been read
                if ((threadIdx.x & 63) == 0) { lds[threadIdx.x >> 6] = s1; lds[W + (threadIdx.x >> 6)] = s2; }
                __syncthreads();
                s1 = s2 = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) { s1 += lds[i]; s2 += lds[W + i]; }
                s1 *= inv; s2 *= inv;
            }
            T *dx = static_cast<T *>(a.dx) + row * H;
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t c = (int64_t)(j * TPR + t) * 8;
                f32x8 o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = rstd * (g[j][i] - s1 - h[j][i] * s2);
                store8(dx + c, H - c, o);
            }
        }
    }
    if (!a.partial) return;
    float *out = a.partial + (int64_t)blockIdx.x * 2 * H;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if constexpr (RPB > 1) {
            for (int wv = 0; wv < RPB; ++wv) {
                __syncthreads();
                if ((int)(threadIdx.x / TPR) == wv) {
#pragma unroll
                    for (int j = 0; j < NC; ++j)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int at = (j * 8 + i) * 64 + t;
                            const float v = k ? db[j][i] : dw[j][i];
                            sums[at] = wv ? sums[at] + v : v;
                        }
                }
            }
            __syncthreads();
            for (int64_t c = threadIdx.x; c < H; c += 256) {
                const int chunk = (int)(c >> 3);
                out[k * H + c] = sums[((chunk / 64) * 8 + (int)(c & 7)) * 64 + chunk % 64];
            }
        } else {
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                const int64_t c = (int64_t)(j * TPR + t) * 8;
                store8(out + k * H + c, H - c, k ? db[j] : dw[j]);
            }
        }
    }
}

// dw and db of 32 columns per workgroup: 32 lanes across the columns, 32 groups that each take every 32nd partial row.  4 to 5 us:
// latency.
__global__ __launch_bounds__(1024) void norm_weight_kernel(const float *partial, int parts, int64_t cols, void *dweight, void *dbias,
                                                           int wtype) {
    __shared__ float lds[32][33];
    const int64_t c = (int64_t)blockIdx.x * 32 + threadIdx.x % 32;
    const int grp = threadIdx.x / 32, k = blockIdx.y;
    void *to = k ? dbias : dweight;
    if (!to) return;
    float s = 0.f;
    if (c < cols) {
        const float *from = partial + k * cols + c;
        int p = grp;
        for (; p + 7 * 32 < parts; p += 8 * 32) {   // eight on their way at a time
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from[(int64_t)(p + i * 32) * 2 * cols];
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        for (; p < parts; p += 32) s += from[(int64_t)p * 2 * cols];
    }
    lds[grp][threadIdx.x % 32] = s;
    __syncthreads();
    if (grp == 0 && c < cols) {
        for (int i = 1; i < 32; ++i) s += lds[i][threadIdx.x];
        store_as(to, wtype, c, s);
    }
}

// Rows too wide for registers: a workgroup of 1,024 goes over its row once per sum, from the caches after the first time.
template <class T>
__device__ __forceinline__ void norm_forward_wide_row(const NormForward &a, int64_t row, float *lds) {
    const int64_t H = a.cols, nb = (H + kBlock - 1) / kBlock;
    const T *x = static_cast<const T *>(a.x) + row * a.x_stride;
    const int64_t wide = (H + 8191) / 8192 * 8192;   // all lanes stay in the loop: they share a block's step
    float s = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < wide; c += 8192) {
        f32x8 v;
        v = load8(x + c, H - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += v[i];
        if (a.q) {
            Bytes8 q;
            const float step = quantise8(v, q);
            if (c < H) {
                store_q(a.q + row * H + c, H - c, q);
                if ((threadIdx.x & 15) == 0) a.scale[row * nb + c / kBlock] = step;
            }
        }
    }
    const float mean = row_sum<1024>(s, lds, 0) / (float)H;
    float ss = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
        f32x8 v;
        v = load8(x + c, H - c);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = c + i < H ? fmaf(v[i] - mean, v[i] - mean, ss) : ss;
    }
    const float rstd = 1.f / sqrtf(row_sum<1024>(ss, lds, 1) / (float)H + a.eps);
    for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
        f32x8 v, w, b;
        v = load8(x + c, H - c);
        w = load8_as(a.weight, a.wtype, c, H - c, 1.f);
        b = load8_as(a.bias, a.wtype, c, H - c, 0.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf((v[i] - mean) * rstd, w[i], b[i]);
        store8(static_cast<T *>(a.y) + row * H + c, H - c, v);
    }
    if (threadIdx.x == 0) { a.mean[row] = mean; a.rstd[row] = rstd; }
}
template <class T>
__global__ __launch_bounds__(1024) void norm_forward_wide_kernel(NormForward a) {
    __shared__ float lds[32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) norm_forward_wide_row<T>(a, row, lds);
}

template <class T>
__device__ __forceinline__ f32x8 load_hat(const NormBackward &a, int64_t row, int64_t c, float mean, float rstd) {
    f32x8 h;
    const int64_t H = a.cols;
    if (a.q) h = load_q(a.q + row * H + c, H - c, a.scale[row * ((H + kBlock - 1) / kBlock) + c / kBlock]);
    else h = load8(static_cast<const T *>(a.x) + row * a.x_stride + c, H - c);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = c + i < H ? (h[i] - mean) * rstd : 0.f;
    return h;
}

template <class T>
__device__ __forceinline__ void norm_backward_wide_row(const NormBackward &a, int64_t row, float *lds) {
    const int64_t H = a.cols;
    const T *dy = static_cast<const T *>(a.dy) + row * a.dy_stride;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
        f32x8 g, h, w;
        g = load8(dy + c, H - c);
        h = load_hat<T>(a, row, c, mean, rstd);
        w = load8_as(a.weight, a.wtype, c, H - c, 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) { s1 += g[i] * w[i]; s2 = fmaf(g[i] * w[i], h[i], s2); }
    }
    s1 = row_sum<1024>(s1, lds, 0) / (float)H;
    s2 = row_sum<1024>(s2, lds, 1) / (float)H;
    for (int64_t c = (int64_t)threadIdx.x * 8; c < H; c += 8192) {
        f32x8 g, h, w;
        g = load8(dy + c, H - c);
        h = load_hat<T>(a, row, c, mean, rstd);
        w = load8_as(a.weight, a.wtype, c, H - c, 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = rstd * (g[i] * w[i] - s1 - h[i] * s2);
        store8(static_cast<T *>(a.dx) + row * H + c, H - c, g);
    }
}
template <class T>
__global__ __launch_bounds__(1024) void norm_backward_wide_kernel(NormBackward a) {
    __shared__ float lds[32];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) norm_backward_wide_row<T>(a, row, lds);
}

// Partial sums for such rows: a workgroup takes 2,048 columns (grid.x) of every parts-th row (grid.y).
template <class T>
__global__ __launch_bounds__(256) void norm_columns_wide_kernel(NormBackward a) {
    const int64_t H = a.cols, c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (c >= H) return;
    f32x8 dw, db;
#pragma unroll
    for (int i = 0; i < 8; ++i) dw[i] = db[i] = 0.f;
    for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
        f32x8 g, h;
        g = load8(static_cast<const T *>(a.dy) + row * a.dy_stride + c, H - c);
        h = load_hat<T>(a, row, c, a.mean[row], a.rstd[row]);
#pragma unroll
        for (int i = 0; i < 8; ++i) { dw[i] = fmaf(g[i], h[i], dw[i]); db[i] += g[i]; }
    }
    float *out = a.partial + (int64_t)blockIdx.y * 2 * H;
    store8(out + c, H - c, dw);
    store8(out + H + c, H - c, db);
}

// A block of 128 columns per 16 lanes.  A lane group steps through the blocks of all rows with a fixed stride, given as rows
// and blocks (no division in the loop).  Bound by memory: 32,768 x 4096 in bf16 (407 MB each way) saved in 84 to 98 us, restored in 65 us
// (6.2 TB/s).
template <class T>
__global__ __launch_bounds__(256) void checkpoint8_save_kernel(const T *x, int64_t x_stride, int64_t rows, int64_t cols, int8_t *q,
                                                               float *scale, int64_t step_rows, int64_t step_blocks) {
    const int64_t nb = (cols + kBlock - 1) / kBlock, first = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int lane = threadIdx.x & 15;
    int64_t row = first / nb, blk = first - row * nb;
    while (row < rows) {
        const int64_t c = blk * kBlock + lane * 8;
        f32x8 v;
        v = load8(x + row * x_stride + c, cols - c);
        Bytes8 b;
        const float step = quantise8(v, b);
        if (c < cols) store_q(q + row * cols + c, cols - c, b);
        if (lane == 0) scale[row * nb + blk] = step;
        row += step_rows; blk += step_blocks;
        if (blk >= nb) { blk -= nb; ++row; }
    }
}
template <class T>
__global__ __launch_bounds__(256) void checkpoint8_restore_kernel(const int8_t *q, const float *scale, int64_t rows, int64_t cols, T *x,
                                                                  int64_t step_rows, int64_t step_blocks) {
    const int64_t nb = (cols + kBlock - 1) / kBlock, first = (int64_t)blockIdx.x * 16 + threadIdx.x / 16;
    const int lane = threadIdx.x & 15;
    int64_t row = first / nb, blk = first - row * nb;
    while (row < rows) {
        const int64_t c = blk * kBlock + lane * 8;
        if (c < cols) {
            f32x8 v;
            v = load_q(q + row * cols + c, cols - c, scale[row * nb + blk]);
            store8(x + row * cols + c, cols - c, v);
        }
        row += step_rows; blk += step_blocks;
        if (blk >= nb) { blk -= nb; ++row; }
    }
}

}  // namespace saber_ops
