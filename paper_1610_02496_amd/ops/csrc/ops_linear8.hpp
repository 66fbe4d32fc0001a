// Logits from 8-bit integers: out_nv = (sum_k qx_nk qw_vk) sx_n sw_v, the sums in int32 (exact: at most 2^17 - 1 products of at most 2^14), then
// in binary32, rounded once to the type of the output.
//
// What bounds it: for few rows the weights' bytes (1 row of 1024 and 100,000 words 19 us, 5.3 TB/s); for many rows the matrix cores and, where the
// columns are as few as here, what a tile does before and after its steps.  8192 rows and 141,000 words in bf16, 60 calls in a row: 128 columns 0.98 ms, 512 1.21, 1000
// 1.54 (1.50 POPS), 2048 2.61 (1.82), 4096 4.05 (2.34), 8192 7.27 (2.60): a step of 128 columns is 0.08 to 0.1 ms, all that is not steps 0.9, of which the stores' bytes
// (2.3 GB) alone are 0.34.  The first calls after a rest take 1.76, as do calls whose inputs change (the clock, by the load of the matrix cores).
#pragma once
#include "ops_product.hpp"

namespace saber_ops {

// Tiles of sums (m: words, n: rows of features) with their scales to [row][word], any alignment.  A lane holds four words of a row and its
// neighbours hold other rows: stored from there, every 16 bytes are a request of their own.  So the tile goes through LDS, and neighbouring
// lanes store neighbouring words (8192 x 1000 x 141,000 in bf16: 2.23 -> 1.87 ms).  Past the caches where rows are whole pieces of 16 bytes, as
// nobody reads them soon and the operands stay (1.87 -> 1.60 ms); other rows end inside of what a cache has to put together (4096 x 777 x
// 30,011: 165 us through the caches, 176 past them).
template <class T>
struct Linear8Epilogue {
    T *out; int64_t rows, words;
    const float *x_scale, *w_scale;
    int past;            // the caches

    template <int TN> struct State { float scale[TN]; };
    template <int TN>
    __device__ __forceinline__ void prepare(State<TN> &s, int64_t n) const {
#pragma unroll
        for (int j = 0; j < TN; ++j) s.scale[j] = n + j * 16 < rows ? x_scale[n + j * 16] : 0.f;
    }
    template <int BM, int BN, int WM, int WN, int TM, int TN>
    __device__ __forceinline__ void finish(f32x4 (&acc)[TM][TN], const State<TN> &st, int64_t m0, int64_t n0, int wm, int wn, int lane, int wave, int, int, void *smem) const {
        typedef T T4 __attribute__((ext_vector_type(4)));
        typedef T T8 __attribute__((ext_vector_type(8)));
        constexpr int STRIDE = BM * (int)sizeof(T) + 16;                // bytes of a row in LDS: the rows of 16 lanes start at different banks
        constexpr int PARTS = BM == 256 && sizeof(T) == 4 ? 2 : 1;      // (all of such a tile does not fit)
        constexpr int JN = TN / PARTS, CHUNKS = BM / 8, AT_ONCE = 64 / CHUNKS;   // chunks of eight words in a row; rows that a wavefront stores at once
        char *const lds = static_cast<char *>(smem);
        const int chunk = lane % CHUNKS;
        const int64_t m = m0 + chunk * 8, room = words - m;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            if (p) __syncthreads();
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int at = wm + i * 16 + 4 * (lane >> 4);
                float sw[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) sw[r] = m0 + at + r < words ? w_scale[m0 + at + r] : 0.f;
#pragma unroll
                for (int j = 0; j < JN; ++j) {
                    T4 o;
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[r] = (T)((float)__float_as_int(acc[i][p * JN + j][r]) * st.scale[p * JN + j] * sw[r]);
                    *reinterpret_cast<T4 *>(lds + (wn / PARTS + j * 16 + (lane & 15)) * STRIDE + at * (int)sizeof(T)) = o;
                }
            }
            __syncthreads();
#pragma unroll 4
            for (int l = wave * AT_ONCE + lane / CHUNKS; l < BN / PARTS; l += WM * WN * AT_ONCE) {
                const int64_t n = n0 + l / (JN * 16) * (TN * 16) + p * JN * 16 + l % (JN * 16);   // (a wavefront's rows, part by part)
                if (n >= rows || room <= 0) continue;
                const T8 v = *reinterpret_cast<const T8 *>(lds + l * STRIDE + chunk * 8 * (int)sizeof(T));
                T *to = out + n * words + m;
                if (past) {
                    if constexpr (sizeof(T) == 2) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), reinterpret_cast<u32x4 *>(to));
                    else {
                        struct Two { u32x4 lo, hi; };
                        const Two two = __builtin_bit_cast(Two, v);
                        __builtin_nontemporal_store(two.lo, reinterpret_cast<u32x4 *>(to));
                        __builtin_nontemporal_store(two.hi, reinterpret_cast<u32x4 *>(to) + 1);
                    }
                } else
                    store8(to, room, __builtin_convertvector(v, f32x8));
            }
        }
    }
};

}  // namespace saber_ops
