// Logits from 8-bit integers: out_nv = (sum_k qx_nk qw_vk) sx_n sw_v, the sums in int32 (exact: at most 2^17 - 1 products of at most 2^14), then
// in binary32, rounded once to the type of the output.
#pragma once
#include "ops_product.hpp"

namespace saber_ops {

// Tiles of sums (m: words, n: rows of features) with their scales to [row][word], any alignment.
template <class T>
struct Linear8Epilogue {
    T *out; int64_t rows, words;
    const float *x_scale, *w_scale;

    template <int TN> struct State { float scale[TN]; };
    template <int TN>
    __device__ __forceinline__ void prepare(State<TN> &s, int64_t n) const {
#pragma unroll
        for (int j = 0; j < TN; ++j) s.scale[j] = n + j * 16 < rows ? x_scale[n + j * 16] : 0.f;
    }
    template <int BM, int BN, int WM, int WN, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &st, int64_t m0, int64_t n0, int wm, int wn, int lane, int, int, int, void *) const {
#pragma unroll
        for (int i = 0; i < TM; i += 2) {
            const int64_t m = m0 + wm + i * 16 + paired_row(lane);
            const f32x8 sw = load8(w_scale + m, words - m);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                uint32_t v[2][4];
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r / 4][r % 4] = __float_as_uint(acc[i + r / 4][j][r % 4]);
                pair_rows(v[0], v[1]);
                const int64_t n = n0 + wn + j * 16 + (lane & 15);
                if (n >= rows || m >= words) continue;
                f32x8 o;
#pragma unroll
                for (int r = 0; r < 8; ++r) o[r] = (float)(int)v[r / 4][r % 4] * st.scale[j] * sw[r];
                store8(out + n * words + m, words - m, o);
            }
        }
    }
};

}  // namespace saber_ops
