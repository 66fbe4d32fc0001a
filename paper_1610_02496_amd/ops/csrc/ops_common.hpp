// Element types, unaligned chunks of eight elements and wavefront sums of the head's operators (gfx950, wave64).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace saber_ops {

constexpr int kChunk = 8;     // elements a lane handles at a time: 16 bytes of a 16-bit type, 32 of binary32
constexpr int kBlock = 128;   // columns that share a scale of a checkpoint: the chunks of 16 lanes

using f32 = float;
using f16 = _Float16;
using bf16 = __bf16;

// 16 bytes at any alignment that the element type allows (global loads and stores of gfx950 take every address)
struct __attribute__((packed, aligned(1))) Bytes16 { uint32_t v[4]; };
struct __attribute__((packed, aligned(1))) Bytes8 { uint32_t v[2]; };

typedef float f32x8 __attribute__((ext_vector_type(8)));

// Eight elements from p, of which the first n exist (the others are zeros; n <= 0: none is read), in two halves: the bytes as they
// lie, which may be asked for early, and their values.
template <class T>
struct Raw8 { uint32_t v[sizeof(T) * 2]; };
template <class T>
__device__ __forceinline__ Raw8<T> load_raw8(const T *p, int64_t n) {
    struct __attribute__((packed, aligned(1))) Any { Raw8<T> r; };
    if (n >= 8) return reinterpret_cast<const Any *>(p)->r;
    constexpr int kDwords = sizeof(T) * 2;
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < kDwords; ++i) r.v[i] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (sizeof(T) == 4) r.v[i] = __builtin_bit_cast(uint32_t, p[i]);
            else r.v[i / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, p[i]) << (16 * (i & 1));
        }
    return r;
}
template <class T>
__device__ __forceinline__ f32x8 widen(const Raw8<T> &r) {
    typedef T V __attribute__((ext_vector_type(8)));
    return __builtin_convertvector(__builtin_bit_cast(V, r), f32x8);
}

template <class T>
__device__ __forceinline__ f32x8 load8(const T *p, int64_t n) { return widen(load_raw8(p, n)); }

// rounds to nearest even; the first n of eight elements
template <class T>
__device__ __forceinline__ void store8(T *p, int64_t n, f32x8 f) {
    if (n >= 8) {
        if constexpr (sizeof(T) == 2) {
            typedef T V __attribute__((ext_vector_type(8)));
            *reinterpret_cast<Bytes16 *>(p) = __builtin_bit_cast(Bytes16, __builtin_convertvector(f, V));
        } else {
            struct Two { Bytes16 lo, hi; };
            *reinterpret_cast<Two *>(p) = __builtin_bit_cast(Two, f);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (T)f[i];
    }
}

// a weight or a gradient of one: its type is known at run time, the same for the whole launch
enum : int { kF32 = 0, kF16 = 1, kBF16 = 2 };
__device__ __forceinline__ f32x8 load8_as(const void *p, int type, int64_t at, int64_t n, float fill) {
    if (!p) return f32x8{fill, fill, fill, fill, fill, fill, fill, fill};
    if (type == kF32) return load8(static_cast<const f32 *>(p) + at, n);
    if (type == kF16) return load8(static_cast<const f16 *>(p) + at, n);
    return load8(static_cast<const bf16 *>(p) + at, n);
}
__device__ __forceinline__ void store_as(void *p, int type, int64_t at, float v) {
    if (type == kF32) static_cast<f32 *>(p)[at] = v;
    else if (type == kF16) static_cast<f16 *>(p)[at] = (f16)v;
    else static_cast<bf16 *>(p)[at] = (bf16)v;
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}

// sum over each row of 16 lanes by rotations, then over the four rows by lane reads: the same value in every lane, always in
// the same order
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<0x128>(v);   // row_ror:8
    v += dpp<0x124>(v);
    v += dpp<0x122>(v);
    v += dpp<0x121>(v);
    const int b = __float_as_int(v);
    const float r0 = __int_as_float(__builtin_amdgcn_readlane(b, 0)), r1 = __int_as_float(__builtin_amdgcn_readlane(b, 16));
    const float r2 = __int_as_float(__builtin_amdgcn_readlane(b, 32)), r3 = __int_as_float(__builtin_amdgcn_readlane(b, 48));
    return (r0 + r1) + (r2 + r3);
}
// largest of the 16 lanes of a row, as unsigned bits: for magnitudes this is the order of the floats, with NaN above infinity
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    v = max(v, dpp<0x128>(v));
    v = max(v, dpp<0x124>(v));
    v = max(v, dpp<0x122>(v));
    v = max(v, dpp<0x121>(v));
    return v;
}

// the same over the whole wavefront
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = row_max(v);
    return max(max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16)),
               max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48)));
}

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

// Whole numbers round(x / step) of a chunk, ties to even, within -127 .. 127; zeros where the step is zero or not finite.
// The product with the inverse is off by 2^-22 * 127 at most, so it gives the whole number of the quotient unless that is as near as that to
// the middle of two: then, rarely, a division decides.  EXACT: one of 64 bits, so that the number is that of the quotient itself; else the
// quotient is rounded to binary32 before.  Adding 1.5 * 2^23 rounds to a whole number, which the sum's low byte then holds in two's
// complement.
template <bool EXACT>
__device__ __forceinline__ void whole8(f32x8 x, float step, Bytes8 &q) {
    constexpr float kWhole = 12582912.f;
    const float inverse = __builtin_amdgcn_rcpf(step);
    uint32_t v[8];
    bool near = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = fmaf(x[i], inverse, kWhole);
        near |= !(fabsf(fmaf(x[i], inverse, kWhole - t)) < 0.4999f);   // (what is not a number as well)
        v[i] = __float_as_uint(t);
    }
    if (near) {
        const bool sound = step > 0.f && step < INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float n = EXACT ? (float)rint((double)x[i] / (double)step) : rintf(x[i] / step);
            v[i] = __float_as_uint((sound ? fminf(fmaxf(n, -127.f), 127.f) : 0.f) + kWhole);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
        q.v[k] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(v[4 * k + 3], v[4 * k + 2], 0x0c0c0400), __builtin_amdgcn_perm(v[4 * k + 1], v[4 * k], 0x0c0c0400), 0x05040100);
}

// One lane's chunk of a block of 128 columns, in 8 bits: step c = max|x| / 127 of the block, whole numbers round(x / c), ties to
// even.  A block of zeros has step 0; a step ends where 127 of it are finite (kMostStep: the largest number of binary32, a mask's value
// perhaps, is restored one unit lower, not as infinity).  A NaN or an infinity makes the step not finite: the block is restored as NaN.
// All 16 lanes of the block call this together.
__device__ __forceinline__ float quantise8(f32x8 x, Bytes8 &q) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
    top = row_max(top);
    constexpr float kMostStep = 0x1.020406p+121f;
    float step = __uint_as_float(top) / 127.f;
    step = top < 0x7f800000u ? fminf(step, kMostStep) : step;
    whole8<false>(x, step, q);
    return step;
}
__device__ __forceinline__ void store_q(int8_t *p, int64_t n, const Bytes8 &q) {
    if (n >= 8) *reinterpret_cast<Bytes8 *>(p) = q;
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (int8_t)(q.v[i >> 2] >> (8 * (i & 3)));
    }
}
__device__ __forceinline__ Bytes8 load_raw_q(const int8_t *p, int64_t n) {
    if (n >= 8) return *reinterpret_cast<const Bytes8 *>(p);
    Bytes8 q = {{0, 0}};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) q.v[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
    return q;
}
__device__ __forceinline__ f32x8 widen_q(const Bytes8 &q, float step) {
    f32x8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (float)((int)(q.v[i >> 2] << (24 - 8 * (i & 3))) >> 24) * step;
    return f;
}
__device__ __forceinline__ f32x8 load_q(const int8_t *p, int64_t n, float step) { return widen_q(load_raw_q(p, n), step); }

}  // namespace saber_ops
