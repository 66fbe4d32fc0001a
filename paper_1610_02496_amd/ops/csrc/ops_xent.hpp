// Softmax cross entropy of a projection onto a large vocabulary, without the logits in memory, and its gradient.
//
//   l_nv = x_n . W_v,   lse_n = log sum_v exp l_nv,   loss_n = lse_n - l_n,t(n)
//   d_nv = g_n (exp(l_nv - lse_n) - [v = t(n)]),   dx_n = sum_v d_nv W_v,   dW_v = sum_n d_nv x_n
//
// Forward: every tile of logits leaves a maximum and a sum of exponentials per row; one small kernel joins them.  Backward: the
// logits are computed again, one piece of the vocabulary at a time; d of a piece, in the type of the features, is the operand of the
// two products that follow.
#pragma once
#include "ops_product.hpp"

namespace saber_ops {

constexpr float kLog2e = 1.44269504088896340736f;

struct Targets {
    const void *p; int wide;   // int64 if wide, else int32
    __device__ __forceinline__ int64_t at(int64_t n) const {
        return wide ? static_cast<const int64_t *>(p)[n] : (int64_t)static_cast<const int32_t *>(p)[n];
    }
};

// a running maximum and the sum of exponentials relative to it; an empty one is (-inf, 0)
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2) {
    const float top = fmaxf(m, m2);
    // (a NaN sum stays NaN; where a maximum is -inf its sum counts as it is: nothing, or NaN)
    const float a = m == top ? 1.f : expf(m - top), b = m2 == top ? 1.f : expf(m2 - top);
    s = s * a + s2 * b;
    m = top;
}

// exp(l - m) by the hardware's 2^x.  The difference is rounded before it is scaled, so logits of any size keep their precision; the
// scaling costs up to 2^-24 |l - m| log2(e) of each exponential.  Next to the rounding of the logits' own binary32 sums that is little:
// a loss is off by 1e-7 at most where it was by 1e-8, d by far less than the 2^-9 (2^-12) with which it is stored.  EXACT, for features of
// binary32: what the scaling's rounding left is put back, exp(d) = 2^h (1 + ln 2 (d log2 e - h)), to about an ulp (a call of expf, of
// whose range little is needed, took a third of the logits' kernel).  For 16-bit features that would cost 8 % of a score of 8192 rows of
// 1000 and 141,000 words (2.56 -> 2.76 ms).
template <bool EXACT>
struct Exp {
    float m;
    __device__ __forceinline__ explicit Exp(float top) : m(top) {}
    __device__ __forceinline__ float operator()(float l) const {
        const float d = l - m, h = d * kLog2e, p = __builtin_amdgcn_exp2f(h);
        if constexpr (!EXACT) return p;
        else {
            const float rest = fmaf(d, 1.92596299e-8f, fmaf(d, kLog2e, -h));   // log2(e) is kLog2e + 1.926e-8
            return h > -200.f ? fmaf(p, rest * 0.693147181f, p) : p;           // (below: 0, of an infinity as well)
        }
    }
};

// Values of two neighbouring tiles of sums, i and i + 1, of which lane group g = lane / 16 holds rows 4 g .. + 3: afterwards a lane has
// eight rows that follow each other, 8 (g / 2) .. + 7 of tile i + g % 2; `lo` and `hi` are their halves.
template <int N>
__device__ __forceinline__ void pair_rows(uint32_t (&lo)[N], uint32_t (&hi)[N]) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const auto p = __builtin_amdgcn_permlane16_swap(lo[i], hi[i], false, false);
        lo[i] = p[0];
        hi[i] = p[1];
    }
#endif
}
__device__ __forceinline__ int paired_row(int lane) { return 16 * (lane >> 4 & 1) + 8 * (lane >> 5); }

// the largest, the sum of a value over the four lane groups that hold the same column: the same in all of them
__device__ __forceinline__ float groups_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float groups_sum(float v) {
    v += __shfl_xor(v, 16);
    return v + __shfl_xor(v, 32);
}

// ---- epilogues of the logits' tiles (m: words, n: rows of features) ----------------------------------------------------------

// Rows of binary32 are multiplied after they were brought to one magnitude: the sums' powers of two, of the words and of the rows.
struct Powers { const int *words, *rows; };

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
#else
    return c;
#endif
}

// The logits' tiles of binary32 whose rows the two planes do not hold.  A value is held to 2^-23 of itself, but no better than to 2^-25
// after the row's power of two (the steps of binary16 end there), so a logit is off by up to 2^-25 (2^px sum|W| + 2^pw sum|x|) more than
// by its products' roundings: up to 2^-22 is left as it is, next to the rounding of a binary32 sum.  Rows whose values are all of one
// magnitude, as a norm gives them, stay a thousand times below that.  Beyond (a count of 10^6 next to features of 1; rows that hold an
// infinity or NaN, whose sum stands as infinite) the tile is computed from the operands themselves by products in binary32, right for all
// values, infinities included.  2,048 rows of 512 and 60,000 words, forward: 0.50 ms with planes, 1.43 ms where every tile is such a
// one (130 TFLOP/s in binary32).
struct Direct32 {
    const float *a; int64_t a_stride;    // words
    const float *b; int64_t b_stride;    // rows
    const float *a_sums, *b_sums;        // of magnitudes, per row; infinite where they are not finite
    Powers powers;

    template <int BM, int BN>
    __device__ __forceinline__ bool has(int64_t m0, int64_t n0, int64_t words, int64_t rows, int lane) const {
        uint32_t a_power = 0, b_power = 0, a_sum = 0, b_sum = 0;   // (sums as bits: magnitudes keep their order)
#pragma unroll
        for (int i = 0; i < BM; i += 64)
            if (m0 + i + lane < words) {
                a_power = max(a_power, (uint32_t)(powers.words[m0 + i + lane] + 512));
                a_sum = max(a_sum, __float_as_uint(a_sums[m0 + i + lane]));
            }
#pragma unroll
        for (int i = 0; i < BN; i += 64)
            if (n0 + i + lane < rows) {
                b_power = max(b_power, (uint32_t)(powers.rows[n0 + i + lane] + 512));
                b_sum = max(b_sum, __float_as_uint(b_sums[n0 + i + lane]));
            }
        a_power = wave_max(a_power); b_power = wave_max(b_power); a_sum = wave_max(a_sum); b_sum = wave_max(b_sum);
        const float off = ldexpf(__uint_as_float(a_sum), (int)b_power - 512) + ldexpf(__uint_as_float(b_sum), (int)a_power - 512);
        return !(off <= 8.f);
    }

    // Four values of k per lane group and turn, straight from memory, into sums of words from m on and of rows from n on.  A lane past the
    // last one takes the last one's values, which the epilogue does not use.
    template <int TM, int TN>
    __device__ __forceinline__ void run(f32x4 (&acc)[TM][TN], int64_t m, int64_t n, int64_t words, int64_t rows, int64_t cols, int lane) const {
        const float *pa[TM], *pb[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) pa[i] = a + last(m + i * 16 + (lane & 15), words) * a_stride + 4 * (lane >> 4);
#pragma unroll
        for (int j = 0; j < TN; ++j) pb[j] = b + last(n + j * 16 + (lane & 15), rows) * b_stride + 4 * (lane >> 4);
#pragma unroll 1
        for (int64_t k = 0; k < cols; k += 16) {
            const int64_t left = k + 16 <= cols ? 4 : cols - k - 4 * (lane >> 4);
            f32x4 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = load4(pa[i] + k, left);
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = load4(pb[j] + k, left);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) acc[i][j] = mfma4(fa[i][r], fb[j][r], acc[i][j]);
        }
    }

private:
    static __device__ __forceinline__ int64_t last(int64_t at, int64_t of) { return at < of ? at : of - 1; }
    // the first n of four elements, zeros for the others
    static __device__ __forceinline__ f32x4 load4(const float *p, int64_t n) {
        struct __attribute__((packed, aligned(4))) Four { f32x4 v; };
        if (n >= 4) return reinterpret_cast<const Four *>(p)->v;
        f32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < n ? p[i] : 0.f;
        return v;
    }
};

// Those tiles, in the numbering of the product that leaves them out; the others' workgroups end at once.
template <int BM, int BN, int WM, int WN, class Epilogue>
__global__ __launch_bounds__(WM * WN * 64) void direct32_kernel(Product p, Epilogue e, Direct32 tiles) {
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    __shared__ float2 lds[WM * BN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int split, tm, tn;
    tile_of_workgroup(p, blockIdx.x, split, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    if (!tiles.template has<BM, BN>(m0, n0, p.a.major, p.b.major, lane)) return;
    const int wm = (wave / WN) * TM * 16, wn = (wave % WN) * TN * 16;
    typename Epilogue::template State<TN> state;
    e.prepare(state, n0 + wn + (lane & 15));
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    tiles.run(acc, m0 + wm, n0 + wn, p.a.major, p.b.major, p.k, lane);
    e.template finish<BM, BN, WM, WN, false>(acc, state, m0, n0, wm, wn, lane, wave, split, tm, (void *)lds);
}

// A column's target relative to the tile, clipped to -1 and what a tile cannot hold.
__device__ __forceinline__ int within_tile(int64_t target, int64_t first_word) {
    const int64_t t = target - first_word;
    return t < 0 ? -1 : t > 4096 ? 4096 : (int)t;
}

// sums of this lane's words from `words` on, of which `left` exist
template <int TM, int TN>
__device__ __forceinline__ void scale_sums(f32x4 (&acc)[TM][TN], const int (&rows)[TN], const int *words, int left) {
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int w = i * 16 + r < left ? words[i * 16 + r] : 0;
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j][r] = __builtin_amdgcn_ldexpf(acc[i][j][r], w + rows[j]);
        }
}

template <bool EXACT>
struct ScoreEpilogue {
    float2 *partial; int64_t rows_pad;   // [tile of words][rows_pad]
    float *at;                           // logit of the target
    Targets target;
    int64_t rows, words, word0;          // rows; words of this piece and the first one's number
    int tile0;
    Powers powers;                       // EXACT

    template <int TN> struct State { int64_t target[TN]; int power[EXACT ? TN : 1]; };
    template <int TN>
    __device__ __forceinline__ void prepare(State<TN> &s, int64_t n) const {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            s.target[j] = n + j * 16 < rows ? target.at(n + j * 16) : -1;
            if constexpr (EXACT) s.power[j] = n + j * 16 < rows ? powers.rows[n + j * 16] : 0;
        }
    }
    template <int BM, int BN, int WM, int WN, bool SCALED = true, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &st, int64_t m0, int64_t n0, int wm, int wn, int lane, int wave,
                                           int, int tm, void *lds) const {
        float2 *join_lds = static_cast<float2 *>(lds);
        const int first = wm + 4 * (lane >> 4);
        const int left = (int)(words - m0 < BM ? words - m0 : BM) - first;   // words of this lane's rows that exist
        if constexpr (EXACT && SCALED) scale_sums(acc, st.power, powers.words + m0 + first, left);
        if (words - m0 < BM) {   // (the vocabulary's last tile alone)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (i * 16 + r >= left)
#pragma unroll
                        for (int j = 0; j < TN; ++j) acc[i][j][r] = -INFINITY;
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int col = wn + j * 16 + (lane & 15);
            const int t = within_tile(st.target[j], word0 + m0 + first);
            const bool here = t < left && t < TM * 16 && (t & 12) == 0;      // (t = -1 has all bits)
            if (__builtin_amdgcn_ballot_w64(here)) {
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (i * 16 + r == t && here) at[n0 + col] = acc[i][j][r];
            }
            float m = -INFINITY, s = 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) m = fmaxf(m, acc[i][j][r]);
            m = groups_max(m);
            const Exp<EXACT> power(m > -INFINITY ? m : 0.f);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) s += power(acc[i][j][r]);
            s = groups_sum(s);
            if (lane < 16) join_lds[(wave / WN) * BN + col] = make_float2(m, s);
        }
        __syncthreads();
        for (int col = threadIdx.x; col < BN; col += WM * WN * 64)
            if (n0 + col < rows) {
                float2 v = join_lds[col];
#pragma unroll
                for (int w = 1; w < WM; ++w) join(v.x, v.y, join_lds[w * BN + col].x, join_lds[w * BN + col].y);
                partial[(int64_t)(tile0 + tm) * rows_pad + n0 + col] = v;
            }
    }
};

// d of 16 bits is brought to one magnitude row by row, so that a row's products are as good whatever its dloss is next to the others':
// with `top` the largest |dloss| and dloss_n = m 2^j top, 1 <= |m| < 2, it is held as (p - [v = t]) m to.  What is missing stands outside of
// the products: dx_n is multiplied by 2^j top / to in binary32, and the product of the weight's gradient takes x_n 2^j in place of x_n (a
// power of two).  With one dloss for all rows (a mean) m is 1: neither the rounding of dloss itself nor, near a target, that of 1 - p then
// stands in every value (with dloss rounded along, the weight's gradient was up to 1.5 times as far from the exact one).
// to is 2^14 for binary16, of which |d| < 2 to neither overflows nor loses bits until it is 2^-28 of it; x then is multiplied by a power
// of two 2^u as well, which brings its largest value to 2^14 .. 2^15, so that x_n 2^j keeps its bits down to about 2^-28 of the largest.
template <class T> constexpr float kGradTo = std::is_same<T, f16>::value ? 0x1p14f : 1.f;
struct GradScale { float top, down; int up; };   // down: top / to / 2^u; up: u
// (m, j) of a dloss; one that is not finite stands for itself
__device__ __forceinline__ float split_dloss(float dloss, float top, int &j) {
    const float q = dloss / top;
    const bool odd = !(fabsf(q) < INFINITY) || q == 0.f;
    j = odd ? 0 : __builtin_amdgcn_frexp_expf(q) - 1;
    return odd ? q : 2.f * __builtin_amdgcn_frexp_mantf(q);
}

// d of the piece, [row][words of the piece], PLANES planes of 16 bits; words past the vocabulary are zeros
template <class T, int PLANES>
struct GradEpilogue {
    T *d; int64_t stride, plane;
    const float *lse, *dloss;
    const GradScale *scale;              // one plane
    Targets target;
    int64_t rows, words, word0, vocab;
    Powers powers;                       // three planes

    template <int TN> struct State { int64_t target[TN]; float top[TN], g[TN]; int power[PLANES == 3 ? TN : 1]; };
    template <int TN>
    __device__ __forceinline__ void prepare(State<TN> &s, int64_t n) const {
        float top = 1.f;
        if constexpr (PLANES == 1) top = scale->top;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const bool row = n + j * 16 < rows;
            s.target[j] = row ? target.at(n + j * 16) : -1;
            s.top[j] = row ? lse[n + j * 16] : 0.f;
            s.g[j] = row ? dloss[n + j * 16] : 0.f;
            if constexpr (PLANES == 1) {
                int power;
                s.g[j] = split_dloss(s.g[j], top, power) * kGradTo<T>;
            }
            if constexpr (PLANES == 3) s.power[j] = row ? powers.rows[n + j * 16] : 0;
        }
    }
    template <int BM, int BN, int WM, int WN, bool SCALED = true, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &st, int64_t m0, int64_t n0, int wm, int wn, int lane, int, int, int,
                                           void *) const {
        const int first = wm + 4 * (lane >> 4);
        const int left = (int)(words - m0 < BM ? words - m0 : BM) - first;
        const int out0 = wm + paired_row(lane), room = (int)(stride - m0 < BM ? stride - m0 : BM) - out0;
        const bool whole = words - m0 >= BM;                                 // all but the vocabulary's last tile
        if constexpr (PLANES == 3 && SCALED) scale_sums(acc, st.power, powers.words + m0 + first, left);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + (lane & 15);
            const int t = within_tile(st.target[j], word0 + m0 + first);
            const bool here = t < TM * 16 && (t & 12) == 0;
            const bool counted = st.target[j] >= 0;
            const Exp<PLANES == 3> power(counted ? (st.target[j] < vocab ? st.top[j] : NAN) : INFINITY);
            const float g = counted ? st.g[j] : 0.f;
            const bool any = __builtin_amdgcn_ballot_w64(here || !counted) != 0;
            T *to = d + n * stride + m0 + out0;
#pragma unroll
            for (int i = 0; i < TM; i += 2) {
                uint32_t out[2][PLANES][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float v[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = power(acc[i + h][j][r]);
                    if (any) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if ((i + h) * 16 + r == t) v[r] -= 1.f;
                            if (!counted) v[r] = 0.f;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v[r] *= g;
                        if (!whole && (i + h) * 16 + r >= left) v[r] = 0.f;
                    }
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) {
                        union { T t[4]; uint32_t u[2]; } o;
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            if constexpr (PLANES == 1) o.t[r] = (T)v[r];
                            else {   // the upper half of the bits, then of what is left
                                const uint32_t b = __float_as_uint(v[r]) & 0xffff0000u;
                                o.t[r] = __builtin_bit_cast(T, (uint16_t)(b >> 16));
                                const float rest = v[r] - __uint_as_float(b);
                                v[r] = (b & 0x7f800000u) == 0x7f800000u ? 0.f : rest;
                            }
                        }
                        out[h][q][0] = o.u[0];
                        out[h][q][1] = o.u[1];
                    }
                }
#pragma unroll
                for (int q = 0; q < PLANES; ++q) {
                    pair_rows(out[0][q], out[1][q]);
                    if (n < rows && i * 16 < room)   // (the stride is a multiple of 8)
                        *reinterpret_cast<u32x4 *>(to + i * 16 + q * plane) = u32x4{out[0][q][0], out[0][q][1], out[1][q][0], out[1][q][1]};
                }
            }
        }
    }
};

// ---- epilogues of the gradients' products (m: columns of features) -----------------------------------------------------------

// dx: [split][rows][stride] partial sums in binary32, over the pieces of the vocabulary
struct SumEpilogue {
    float *sums; int64_t stride, rows, cols;
    int add;

    template <int TN> struct State {};
    template <int TN> __device__ __forceinline__ void prepare(State<TN> &, int64_t) const {}
    template <int BM, int BN, int WM, int WN, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &, int64_t m0, int64_t n0, int wm, int wn, int lane, int, int split, int, void *) const {
        float *to = sums + split * rows * stride;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + (lane & 15);
#pragma unroll
            for (int i = 0; i < TM; i += 2) {
                uint32_t v[2][4];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r / 4][r % 4] = __float_as_uint(acc[i + r / 4][j][r % 4]);
                pair_rows(v[0], v[1]);
                const int64_t m = m0 + wm + i * 16 + paired_row(lane);
                if (n >= rows || m >= cols) continue;   // cols is a multiple of 8
                f32x8 *p = reinterpret_cast<f32x8 *>(to + n * stride + m), u;
#pragma unroll
                for (int r = 0; r < 8; ++r) u[r] = __uint_as_float(v[r / 4][r % 4]);
                *p = add ? *p + u : u;
            }
        }
    }
};

// dW: rows n (words) of cols columns in the type of W, any alignment
template <class T>
struct StoreEpilogue {
    T *out; int64_t rows, cols;
    const GradScale *scale;              // of d, or null

    template <int TN> struct State {};
    template <int TN> __device__ __forceinline__ void prepare(State<TN> &, int64_t) const {}
    template <int BM, int BN, int WM, int WN, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &, int64_t m0, int64_t n0, int wm, int wn, int lane, int, int, int, void *) const {
        const float down = scale ? scale->down : 1.f;
        const bool whole = cols % 8 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = n0 + wn + j * 16 + (lane & 15);
#pragma unroll
            for (int i = 0; i < TM; i += 2) {
                constexpr int DWORDS = sizeof(T);        // of four values
                union Four { T t[4]; uint32_t u[DWORDS]; } v[2];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r / 4].t[r % 4] = (T)(acc[i + r / 4][j][r % 4] * down);
                pair_rows(v[0].u, v[1].u);
                const int64_t m = m0 + wm + i * 16 + paired_row(lane);
                if (n >= rows || m >= cols) continue;
                T *to = out + n * cols + m;
                struct alignas(16) Eight { Four f[2]; };
                if (whole) *reinterpret_cast<Eight *>(to) = Eight{{v[0], v[1]}};
                else {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (m + r < cols) to[r] = v[r / 4].t[r % 4];
                }
            }
        }
    }
};

// ---- small kernels ---------------------------------------------------------------------------------------------------------

// The bits of eight values as operands of the matrix cores: one of 16 bits, or three of bfloat16 whose sum is the value of 32
// (cut off, so that it is exact; an infinity or NaN stays whole in the first).  SIGNED: the second and third plane of a value that leaves
// nothing for them hold its sign and 2^-126 in place of zero, so that times an infinity each plane gives the same infinity, none NaN
// (to a sum of products this adds 2^-125 of the other operand's at most).
template <class T, bool SIGNED = false>
__device__ __forceinline__ void planes_of(const Raw8<T> &r, u32x4 (&o)[sizeof(T) == 4 ? 3 : 1]) {
    if constexpr (sizeof(T) == 2) o[0] = u32x4{r.v[0], r.v[1], r.v[2], r.v[3]};
    else {
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.v[i]);
        float least[SIGNED ? 8 : 1];
        if constexpr (SIGNED)
#pragma unroll
            for (int i = 0; i < 8; ++i) least[i] = copysignf(fminf(fabsf(v[i]), 0x1p-126f), v[i]);
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            uint32_t h[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t all = __float_as_uint(v[i]), b = all & 0xffff0000u;
                const bool odd = (b & 0x7f800000u) == 0x7f800000u;
                // a NaN whose upper half would read as an infinity keeps a bit of it
                h[i] = odd && (all & 0x7fffffu) ? b | 0x400000u : b;
                v[i] = odd ? 0.f : v[i] - __uint_as_float(b);
                if constexpr (SIGNED) v[i] = fabsf(v[i]) < 0x1p-126f ? least[i] : v[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) o[q][i] = __builtin_amdgcn_perm(h[2 * i + 1], h[2 * i], 0x07060302);
        }
    }
}

// Rows of 16-bit elements as aligned rows, zeros up to their stride.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(const T *src, int64_t src_stride, int64_t rows, int64_t cols, uint16_t *dst, int64_t stride) {
    const int64_t c = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * 8;
    if (c >= stride) return;
    for (int64_t row = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.y * 4) {
        u32x4 o[1];
        planes_of<T>(load_raw8(src + row * src_stride + c, cols - c), o);
        *reinterpret_cast<u32x4 *>(dst + row * stride + c) = o[0];
    }
}

// Features for the product of the weight's gradient: the same, times 2^(j + u).  Rows without a target become zeros, so that nothing in
// them, NaN included, reaches a product.
template <class T>
__global__ __launch_bounds__(256) void pack_scaled_kernel(const T *src, int64_t src_stride, int64_t rows, int64_t cols, uint16_t *dst, int64_t stride,
                                                          Targets target, const float *dloss, const GradScale *scale) {
    const int64_t c = ((int64_t)blockIdx.x * 64 + (threadIdx.x & 63)) * 8;
    if (c >= stride) return;
    const float top = scale->top;
    const int up = scale->up;
    for (int64_t row = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.y * 4) {
        f32x8 v = load8(src + row * src_stride + c, target.at(row) < 0 ? 0 : cols - c);
        int j;
        split_dloss(dloss[row], top, j);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_ldexpf(v[i], j + up);
        store8(reinterpret_cast<T *>(dst) + row * stride + c, 8, v);
    }
}

// The same for binary32, a row per wavefront, with a second form for the logits: the row times the power of two that brings its largest
// finite value to 2^14 .. 2^15, in two planes of binary16 (x = x1 + x2 to 2^-23 of it, or to 2^-40 of the row's largest where that is
// more); the power that undoes it goes to `powers`, the sum of magnitudes to `sums`, from which a tile sees whether that is enough.  The
// planes may be left out.  One launch packs features and projection, one after the other.
struct Rows32 { const float *src; int64_t src_stride, rows; uint16_t *dst; int64_t plane; uint16_t *even; int *powers; float *sums; Targets mask; };
__global__ __launch_bounds__(256) void pack32_kernel(Rows32 x, Rows32 w, int64_t cols, int64_t stride) {
    const int lane = threadIdx.x & 63;
    for (int64_t at = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); at < x.rows + w.rows; at += (int64_t)gridDim.x * 4) {
        const bool first = at < x.rows;
        const int64_t row = first ? at : at - x.rows, plane = first ? x.plane : w.plane;
        uint16_t *const dst = first ? x.dst : w.dst, *const even = first ? x.even : w.even;
        const float *const from = first ? x.src + row * x.src_stride : w.src + row * w.src_stride;
        const int64_t have = first && x.mask.p && x.mask.at(row) < 0 ? 0 : cols;
        uint32_t top = 0;
        float sum = 0.f;
        for (int64_t c = lane * 8; c < stride; c += 512) {
            const Raw8<f32> r = load_raw8(from + c, have - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = r.v[i] & 0x7fffffffu;
                top = max(top, b < 0x7f800000u ? b : 0u);
                sum += __uint_as_float(b);
            }
        }
        top = wave_max(top);
        sum = wave_sum(sum);
        int e = 14 - ((int)(top >> 23) - 127);         // (kept within the normal numbers; a row of zeros has the smallest power)
        e = e > 126 ? 126 : e;
        const float up = __uint_as_float((uint32_t)(e + 127) << 23);
        if (lane == 0) {
            (first ? x.powers : w.powers)[row] = -e;
            (first ? x.sums : w.sums)[row] = sum < INFINITY ? sum : INFINITY;   // (of a NaN as well)
        }
        for (int64_t c = lane * 8; c < stride; c += 512) {
            const Raw8<f32> r = load_raw8(from + c, have - c);
            if (dst) {
                u32x4 o[3];
                planes_of<f32>(r, o);
#pragma unroll
                for (int q = 0; q < 3; ++q) *reinterpret_cast<u32x4 *>(dst + q * plane + row * stride + c) = o[q];
            }
            union { f16 t[8]; u32x4 u; } hi, lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = __uint_as_float(r.v[i]) * up;
                hi.t[i] = (f16)v;
                lo.t[i] = fabsf(v) < INFINITY ? (f16)(v - (float)hi.t[i]) : (f16)0.f;
            }
            *reinterpret_cast<u32x4 *>(even + row * stride + c) = hi.u;
            *reinterpret_cast<u32x4 *>(even + plane + row * stride + c) = lo.u;
        }
    }
}

// joins the partial sums of a row: 16 rows per workgroup, 64 groups of lanes over the parts
__global__ __launch_bounds__(1024) void score_join_kernel(const float2 *partial, int64_t rows_pad, int parts, const float *at, Targets target,
                                                          int64_t rows, int64_t vocab, float *loss, float *lse) {
    __shared__ float2 lds[64][17];
    const int64_t n = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15);
    const int grp = threadIdx.x >> 4;
    float m = -INFINITY, s = 0.f;
    if (n < rows)
        for (int p = grp; p < parts; p += 8 * 64) {   // eight on their way at a time
            float2 v[8];
            float top = m;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = p + i * 64 < parts ? partial[(int64_t)(p + i * 64) * rows_pad + n] : make_float2(-INFINITY, 0.f);
                top = fmaxf(top, v[i].x);
            }
            s *= m == top ? 1.f : expf(m - top);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i].y * (v[i].x == top ? 1.f : expf(v[i].x - top));
            m = top;
        }
    lds[grp][threadIdx.x & 15] = make_float2(m, s);
    for (int half = 32; half; half >>= 1) {
        __syncthreads();
        if (grp < half) {
            const float2 v = lds[grp + half][threadIdx.x & 15];
            join(m, s, v.x, v.y);
            lds[grp][threadIdx.x & 15] = make_float2(m, s);
        }
    }
    if (grp == 0 && n < rows) {
        const float l = m + logf(s);
        const int64_t t = target.at(n);
        lse[n] = l;
        loss[n] = t < 0 ? 0.f : t < vocab ? l - at[n] : NAN;
    }
}

// largest finite magnitude of the rows with a target, one per workgroup
template <class T>
__global__ __launch_bounds__(256) void magnitude_kernel(const T *src, int64_t src_stride, int64_t rows, int64_t cols, Targets target, uint32_t *most) {
    __shared__ uint32_t lds[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t top = 0;
    for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < rows; row += (int64_t)gridDim.x * 4) {
        if (target.at(row) < 0) continue;
        for (int64_t c = lane * 8; c < cols; c += 512) {
            const f32x8 v = load8(src + row * src_stride + c, cols - c);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
                top = max(top, b < 0x7f800000u ? b : 0u);
            }
        }
    }
    top = wave_max(top);
    if (lane == 0) lds[wave] = top;
    __syncthreads();
    if (threadIdx.x == 0) most[blockIdx.x] = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
}

// what d is relative to: the largest finite |dloss| of the rows with a target (1 if there is none but zeros), and of `parts` magnitudes of
// features the largest (none: u = 0)
__global__ __launch_bounds__(1024) void grad_scale_kernel(const float *dloss, Targets target, int64_t rows, float to, const uint32_t *most, int parts,
                                                          GradScale *scale) {
    __shared__ uint32_t lds[2][16];
    uint32_t top = 0, size = 0;
    for (int64_t n = threadIdx.x; n < rows; n += 1024)
        if (target.at(n) >= 0) {
            const uint32_t b = __float_as_uint(dloss[n]) & 0x7fffffffu;
            top = max(top, b < 0x7f800000u ? b : 0u);
        }
    for (int i = threadIdx.x; i < parts; i += 1024) size = max(size, most[i]);
    top = wave_max(top);
    size = wave_max(size);
    if ((threadIdx.x & 63) == 0) { lds[0][threadIdx.x >> 6] = top; lds[1][threadIdx.x >> 6] = size; }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 16; ++i) { top = max(top, lds[0][i]); size = max(size, lds[1][i]); }
        const float g = top ? __uint_as_float(top) : 1.f;
        const int up = size ? 14 - ((int)(size >> 23) - 127) : 0;   // (binary16 has no magnitude below 2^-24)
        *scale = GradScale{g, __builtin_amdgcn_ldexpf(g / to, -up), up};
    }
}

// dx = sum of the splits' partial sums times what d is relative to, in a fixed order; zeros for a row without a target: every wavefront takes a quarter of the splits of 512 columns of a row, eight
// on their way at a time, and the quarters meet in LDS
template <class T>
__global__ __launch_bounds__(256) void sum_kernel(const float *sums, int splits, int64_t rows, int64_t stride, int64_t cols, Targets target,
                                                  const float *dloss, const GradScale *scale, T *dx) {
    __shared__ f32x8 lds[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * 8;
    const int k0 = splits * wave / 4, k1 = splits * (wave + 1) / 4;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        f32x8 v = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c < cols) {
            const float *from = sums + row * stride + c;   // (the stride is a multiple of 8)
            int k = k0;
            for (; k + 8 <= k1; k += 8) {
                f32x8 u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) u[i] = load8(from + (int64_t)(k + i) * rows * stride, 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) v += u[i];
            }
#pragma unroll 4
            for (; k < k1; ++k) v += load8(from + (int64_t)k * rows * stride, 8);
        }
        lds[wave][lane] = v;
        __syncthreads();
        if (wave == 0 && c < cols) {
            for (int i = 1; i < 4; ++i) v += lds[i][lane];
            float down = 1.f;
            if constexpr (sizeof(T) == 2) {
                int j;
                split_dloss(dloss[row], scale->top, j);
                down = __builtin_amdgcn_ldexpf(scale->top / kGradTo<T>, j);
            }
            if (target.at(row) < 0) v = f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            else v *= down;
            store8(dx + row * cols + c, cols - c, v);
        }
        __syncthreads();
    }
}

template <class T>
__global__ __launch_bounds__(256) void zeros_kernel(T *p, int64_t n) {
    for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 2048)
        store8(p + i, n - i, f32x8{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f});
}

// ---- few rows --------------------------------------------------------------------------------------------------------------

template <class T>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
#if defined(__HIP_DEVICE_COMPILE__)
    if constexpr (std::is_same<T, bf16>::value)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
#else
    return c;
#endif
}

// Up to 16 NT rows: W is read once from memory straight into the matrix cores' operand registers, 16 words by 32 columns at a time, any
// alignment, a batch ahead of its use; the rows' features stay in LDS.  Every wave keeps a running maximum and sum for its
// words; a workgroup leaves one partial result per row.  With few words 2^share_log waves (1, 2, 4, 8) take a tile's columns in turn, so that
// more of the weights are on their way at once; the first of them adds up what they found.  Bound by memory: one row of 1024 in bf16 and
// 100,000 words (205 MB) 42 us, 4.9 TB/s; 61 rows of 777 in f16 and 30,011 words (47 MB, no row aligned) 27 us, the loads' latency and number.
constexpr int kFewWaves = 8;
template <class T> constexpr int kFewBatch = sizeof(T) == 4 ? 4 : 8;   // fragments of 32 columns that a wavefront asks for at a time

template <class T, int NT>
__global__ __launch_bounds__(kFewWaves * 64) void score_few_kernel(const T *x, int64_t x_stride, const T *w, int64_t w_stride, Targets target,
                                                                   int64_t rows, int64_t vocab, int64_t cols, int share_log, float2 *partial,
                                                                   int64_t rows_pad, float *at) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int PLANES = F32 ? 3 : 1, BATCH = kFewBatch<T>;
    using M = typename std::conditional<F32, bf16, T>::type;
    extern __shared__ __attribute__((aligned(16))) char few_lds[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, grp = lane >> 4;
    const int pad = (int)((cols + 31) / 32 * 32), row_bytes = pad * 2 + 16, plane_bytes = (int)rows * row_bytes;
    const int64_t tiles = (vocab + 15) / 16;
    const int share = 1 << share_log, k_first = (wave & (share - 1)) * 32 * BATCH, k_step = share * 32 * BATCH;
    const int64_t next_tile = (int64_t)gridDim.x * kFewWaves >> share_log, first_tile = ((int64_t)blockIdx.x * kFewWaves + wave) >> share_log;
    int64_t tile = k_first < pad ? first_tile : tiles;
    int k = k_first;                     // first column of the batch to come
    Raw8<T> raw[BATCH];
    auto ask = [&] {
        const int64_t v = tile * 16 + (lane & 15);
        const T *from = w + (v < vocab ? v : vocab - 1) * w_stride + k + grp * 8;
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (k + 32 * u + 32 <= cols) raw[u] = load_raw8(from + 32 * u, 8);
            else raw[u] = load_raw8(from + 32 * u, cols - k - 32 * u - grp * 8);   // (none: zeros)
        }
    };
    if (tile < tiles) ask();
    // features: 16 bytes apart from a multiple of 128, so that eight rows lie in different banks
    for (int c = (threadIdx.x & 127) * 8; c < pad; c += 1024) {
        for (int n = threadIdx.x >> 7; n < rows; n += kFewWaves / 2 * BATCH) {
            Raw8<T> f[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int m = n + i * (kFewWaves / 2);
                f[i] = load_raw8(x + (int64_t)(m < rows ? m : n) * x_stride + c, cols - c);
            }
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int m = n + i * (kFewWaves / 2);
                u32x4 o[PLANES];
                planes_of<T, true>(f[i], o);
                if (m < rows)
#pragma unroll
                    for (int q = 0; q < PLANES; ++q) *reinterpret_cast<u32x4 *>(few_lds + q * plane_bytes + m * row_bytes + c * 2) = o[q];
            }
        }
    }
    __syncthreads();
    float m[NT], s[NT];
    int64_t t[NT];
    const char *mine[NT];   // a lane beyond the last row takes the last one: its column is never used
    f32x4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        m[j] = -INFINITY; s[j] = 0.f;
        const int64_t n = j * 16 + (lane & 15);
        t[j] = n < rows ? target.at(n) : -1;
        mine[j] = few_lds + (int)(n < rows ? n : rows - 1) * row_bytes + grp * 16;
        acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto fold = [&](int64_t v0) {   // 16 words' logits into the sums
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            float top = m[j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (v0 + r == t[j] && t[j] < vocab) at[j * 16 + (lane & 15)] = acc[j][r];
                if (v0 + r >= vocab) acc[j][r] = -INFINITY;
                top = fmaxf(top, acc[j][r]);
            }
            if (__builtin_amdgcn_ballot_w64(top > m[j])) s[j] *= m[j] == top ? 1.f : expf(m[j] - top);   // ever more rarely
            m[j] = top;
            const Exp<F32> power(top > -INFINITY ? top : 0.f);
#pragma unroll
            for (int r = 0; r < 4; ++r) s[j] += power(acc[j][r]);
            acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    while (tile < tiles) {
        const int64_t v0 = tile * 16 + 4 * grp;
        const int k_now = k;
        Raw8<T> now[BATCH];
#pragma unroll
        for (int u = 0; u < BATCH; ++u) now[u] = raw[u];
        k += k_step;
        const bool done = k >= pad;
        if (done) { k = k_first; tile += next_tile; }
        if (tile < tiles) ask();
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (k_now + 32 * u >= pad) break;
            u32x4 a[PLANES];
            planes_of<T>(now[u], a);
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                u32x4 b[PLANES];
#pragma unroll
                for (int q = 0; q < PLANES; ++q) b[q] = *reinterpret_cast<const u32x4 *>(mine[j] + q * plane_bytes + (k_now + 32 * u) * 2);
                if constexpr (!F32) acc[j] = mfma16<M>(a[0], b[0], acc[j]);
                else {
#pragma unroll
                    for (int q = 0; q < 6; ++q) acc[j] = mfma16<M>(a[(0x001012 >> (4 * q)) & 15], b[(0x010210 >> (4 * q)) & 15], acc[j]);
                }
            }
        }
        if (done && share == 1) fold(v0);
    }
    __syncthreads();   // the features have been read: LDS is free
    if (share > 1) {
        f32x4 *sums = reinterpret_cast<f32x4 *>(few_lds);
#pragma unroll
        for (int j = 0; j < NT; ++j) sums[(j * kFewWaves + wave) * 64 + lane] = acc[j];
        __syncthreads();
        if ((wave & (share - 1)) == 0) {
#pragma unroll
            for (int j = 0; j < NT; ++j)
                for (int i = 1; i < share; ++i) acc[j] += sums[(j * kFewWaves + wave + i) * 64 + lane];
            fold(first_tile * 16 + 4 * grp);
        }
        __syncthreads();
    }
    float2 *lds = reinterpret_cast<float2 *>(few_lds);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        join(m[j], s[j], __shfl_xor(m[j], 16), __shfl_xor(s[j], 16));
        join(m[j], s[j], __shfl_xor(m[j], 32), __shfl_xor(s[j], 32));
        if (lane < 16) lds[wave * NT * 16 + j * 16 + lane] = make_float2(m[j], s[j]);
    }
    __syncthreads();
    if (threadIdx.x < NT * 16 && threadIdx.x < rows) {
        float2 p = lds[threadIdx.x];
#pragma unroll
        for (int i = 1; i < kFewWaves; ++i) join(p.x, p.y, lds[i * NT * 16 + threadIdx.x].x, lds[i * NT * 16 + threadIdx.x].y);
        partial[(int64_t)blockIdx.x * rows_pad + threadIdx.x] = p;
    }
}

}  // namespace saber_ops
