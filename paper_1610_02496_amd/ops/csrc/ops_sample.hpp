// A word per row of logits, for a given random number.
//
//   z_v = (l_v - max l) / T,  words in the order of their logits, equal ones in the order of their numbers;
//   of these the first top_k, of them the fewest that hold top_p of their mass (sum of e^z), of them those of e^z >= min_p;
//   word: the first one, by number, with  sum of e^z of the words up to it  >  u * (sum of e^z of all that are left).
//
// Every limit leaves a head of the order, so what is left is known by a border: all logits above it, and of those equal to it the first few.
// The borders are found without sorting, by histograms of counts and of masses.
//
// Masses are whole numbers, round(e^z 2^S) with S = 45 (less beyond 2^17 words, so that the sum of all stays below 2^62): their sums are
// exact, so that neither their order nor atomics change a result, and e^z is computed to 2^-50, so that a border falls where 64-bit arithmetic
// puts it.  A word of less than 2^-(S + 1) of the likeliest one's mass has none and is never drawn.
#pragma once
#include "ops_common.hpp"

namespace saber_ops {

struct Sample {
    const void *logits; int64_t stride;
    int64_t rows, words;
    const float *u;
    // a value per row, or null: the same for all rows
    const float *temperatures; float temperature;
    const void *top_ks; int top_k64; int64_t top_k;
    const float *top_ps; float top_p;
    const float *min_ps; float min_p;
    int64_t *word; float *p;
    int tile_log, mass_log;         // words of a tile: 512 << tile_log; S
};

constexpr int kBins = 2048;         // of a histogram
constexpr int kList = 2048;         // logits of a bin that are looked at in LDS
constexpr int kTiles = 2048;        // of a row, at most
constexpr float kBinsPerUnit = 64.f;
constexpr int kZeroBin = 2046;      // bins from here on hold no mass: z < -31.9, e^z 2^45 < 1/2

// 2^r, |r| <= 1/2, to 3e-16: the interpolation at the Chebyshev nodes of degree 10
__device__ __forceinline__ double exp2_near(double r) {
    double p = 0x1.e6063f7217bc6p-28;
    p = fma(p, r, 0x1.b675bca4eeebbp-24);
    p = fma(p, r, 0x1.62bfd47773353p-20);
    p = fma(p, r, 0x1.ffcb54062e698p-17);
    p = fma(p, r, 0x1.430913096fd9fp-13);
    p = fma(p, r, 0x1.5d87fe9d7a584p-10);
    p = fma(p, r, 0x1.3b2ab6fba1ddap-7);
    p = fma(p, r, 0x1.c6b08d703ce49p-5);
    p = fma(p, r, 0x1.ebfbdff82c598p-3);
    p = fma(p, r, 0x1.62e42fefa3a19p-1);
    return fma(p, r, 1.0);
}

// The logits of a row relative to its largest.
struct Scale {
    float top, per;      // largest logit; bins per unit of a logit
    double log2_per;     // log2(e) / T
    double least;        // least difference that min_p leaves
    double up;           // 2^S
    // (of two infinities too)
    __device__ __forceinline__ double down(float l) const { return l == top ? 0.0 : (double)l - (double)top; }
    __device__ __forceinline__ int bin(float l) const {   // rises as the logit falls, by steps of 1/64 of z
        const float b = l == top ? 0.f : (top - l) * per;
        return b < (float)kZeroBin ? (int)b : kZeroBin;   // (NaN, of -inf and T = inf, as well)
    }
    // e^z; 0 for what is too small to have a mass
    __device__ __forceinline__ double part(double d) const {
        const double t = d * log2_per, n = t + 0x1.8p52, r = t - (n - 0x1.8p52);
        const double e = exp2_near(r);
        const uint64_t bits = __double_as_longlong(e) + ((uint64_t)__double_as_longlong(n) << 52);
        return t > -64.0 ? __longlong_as_double((long long)bits) : 0.0;
    }
    __device__ __forceinline__ uint64_t mass(float l) const {
        const double v = fma(part(down(l)), up, 0x1p52);   // rounded to a whole number
        return (uint64_t)__double_as_longlong(v) & 0xfffffffffffffull;
    }
};

__device__ __forceinline__ uint32_t key_of(float f) {   // the order of the floats; -0 and 0 are equal
    const uint32_t b = __float_as_uint(f + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

template <int CTRL>
__device__ __forceinline__ uint64_t dpp64(uint64_t v) { return (uint64_t)dpp<CTRL>((uint32_t)(v >> 32)) << 32 | dpp<CTRL>((uint32_t)v); }
__device__ __forceinline__ uint64_t lane64(uint64_t v, int lane) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}
__device__ __forceinline__ uint64_t wave_total(uint64_t v) {
    v += dpp64<0x128>(v);
    v += dpp64<0x124>(v);
    v += dpp64<0x122>(v);
    v += dpp64<0x121>(v);
    return lane64(v, 0) + lane64(v, 16) + lane64(v, 32) + lane64(v, 48);
}
__device__ __forceinline__ float wave_largest(float v) {
#pragma unroll
    for (int i = 32; i; i >>= 1) v = fmaxf(v, __shfl_xor(v, i));
    return v;
}
// sum over this lane and those before it
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) {
        const uint64_t below = (uint64_t)__shfl_up((unsigned long long)v, i);
        if (lane >= i) v += below;
    }
    return v;
}

template <int THREADS>
struct SampleLds {
    uint64_t mass[kBins];            // of a bin; later of a tile
    uint32_t count[kBins];           // the same; of a tile: logits equal to the border
    float list[kList];
    uint64_t waves[2][THREADS / 64];
    uint64_t found[4];
    uint32_t listed, key_lo, key_hi;
};

// sum over the threads up to and including this one, and over all of them
template <int THREADS>
__device__ __forceinline__ uint64_t block_scan(SampleLds<THREADS> &s, int which, uint64_t v, uint64_t &total) {
    const uint64_t own = wave_scan(v);
    if ((threadIdx.x & 63) == 63) s.waves[which][threadIdx.x >> 6] = own;
    __syncthreads();
    uint64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const uint64_t x = s.waves[which][w];
        if (w < (int)(threadIdx.x >> 6)) before += x;
        total += x;
    }
    __syncthreads();
    return before + own;
}

// f(first word, eight logits, how many of them exist) for all of a row, a tile of 512 words per wavefront at a time; four are on their way.
template <class T, int THREADS, class F>
__device__ __forceinline__ void walk(const T *row, int64_t words, F &&f) {
    const int lane = threadIdx.x & 63;
    const int64_t step = THREADS / 64 * 512;
    for (int64_t c0 = (int64_t)(threadIdx.x >> 6) * 512; c0 < words; c0 += 4 * step) {
        Raw8<T> raw[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t c = c0 + k * step + lane * 8;
            raw[k] = load_raw8(row + c, words - c);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c0 + k * step < words) {
                const int64_t c = c0 + k * step + lane * 8, left = words - c;
                f(c, widen(raw[k]), left < 8 ? (int)left : 8);
            }
    }
}

// The border of the fewest logits in falling order that hold `goal` (a count, or a mass): its value, and how many of those equal to it take
// part.  Only logits above `above` count, and `ties` of those equal to it.  Fewer than goal in all bins that have mass: -inf.
struct Border { float value; uint64_t ties; };

template <class T, int THREADS, bool MASS>
__device__ __forceinline__ Border find_border(SampleLds<THREADS> &s, const T *row, int64_t words, const Scale &sc, Border above, double share, uint64_t goal) {
    const int tid = threadIdx.x;
    constexpr int EACH = kBins / THREADS;
    auto clear = [&] {
        for (int i = tid; i < kBins; i += THREADS) {
            s.mass[i] = 0;
            s.count[i] = 0;
        }
    };
    auto add = [&](int bin, float l) {
        if constexpr (MASS) {
            const uint64_t m = sc.mass(l);
            if (m) atomicAdd((unsigned long long *)&s.mass[bin], (unsigned long long)m);
        } else
            atomicAdd(&s.count[bin], 1u);
    };
    auto add_ties = [&](int bin) {   // by one thread
        if constexpr (MASS)
            if (above.value > -INFINITY) atomicAdd((unsigned long long *)&s.mass[bin], (unsigned long long)(above.ties * sc.mass(above.value)));
    };
    // the bin in which the sum from the first bin on reaches the goal, and the sum before it; kBins if there is none
    auto reach = [&](uint64_t before, bool first) {
        uint64_t v[EACH], sum = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += v[i] = MASS ? s.mass[tid * EACH + i] : s.count[tid * EACH + i];
        if (tid == 0) s.found[0] = kBins;
        const uint64_t upto = block_scan(s, 0, sum, total);
        if (MASS && first) {
            const double want = share * (double)total;
            goal = (uint64_t)want;
            goal += (double)goal < want;
            if (goal < 1) goal = 1;
            if (goal > total) goal = total;
        }
        uint64_t at = before + upto - sum;
        if (at < goal && at + sum >= goal) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (at < goal && at + v[i] >= goal) {
                    s.found[0] = (uint64_t)(tid * EACH + i);
                    s.found[1] = at;
                    s.found[2] = v[i];
                }
                at += v[i];
            }
        }
        __syncthreads();
    };

    __syncthreads();
    clear();
    __syncthreads();
    walk<T, THREADS>(row, words, [&](int64_t, f32x8 v, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int b = sc.bin(v[i]);
            if (i < n && b < kZeroBin && v[i] > above.value) add(b, v[i]);
        }
    });
    if (tid == 0 && above.value > -INFINITY && sc.bin(above.value) < kZeroBin) add_ties(sc.bin(above.value));
    __syncthreads();
    reach(0, true);
    if (s.found[0] >= kBins) return above;
    const int bin = (int)s.found[0];
    uint64_t before = s.found[1];

    // the logits of that bin (those at the border above stay out): a list of them, if they are few, and their range
    if (tid == 0) { s.listed = 0; s.key_lo = 0xffffffffu; s.key_hi = 0; }
    __syncthreads();
    uint32_t lo = 0xffffffffu, hi = 0;
    walk<T, THREADS>(row, words, [&](int64_t, f32x8 v, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n && v[i] > above.value && sc.bin(v[i]) == bin) {
                const uint32_t at = atomicAdd(&s.listed, 1u);
                if (at < kList) s.list[at] = v[i];
                const uint32_t k = key_of(v[i]);
                lo = min(lo, k);
                hi = max(hi, k);
            }
    });
    const bool tied = MASS && above.value > -INFINITY && sc.bin(above.value) == bin;
    if (tied) lo = key_of(above.value);
    if (lo <= hi || tied) { atomicMin(&s.key_lo, lo); atomicMax(&s.key_hi, max(lo, hi)); }
    __syncthreads();
    lo = s.key_lo; hi = s.key_hi;
    const uint32_t listed = s.listed;
    // a histogram of the keys lo .. hi, the largest first, in ever smaller ranges
    while (lo < hi) {
        const int shift = 32 - __builtin_clz((hi - lo) >> 10 | 1u) - 1;   // ((hi - lo) >> shift) < 2048
        __syncthreads();
        clear();
        __syncthreads();
        auto take = [&](float l) {
            const uint32_t k = key_of(l);
            if (k >= lo && k <= hi) add((int)((hi - k) >> shift), l);
        };
        if (listed <= kList) {
            for (uint32_t i = tid; i < listed; i += THREADS) take(s.list[i]);
        } else {
            walk<T, THREADS>(row, words, [&](int64_t, f32x8 v, int n) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < n && v[i] > above.value && sc.bin(v[i]) == bin) take(v[i]);
            });
        }
        if (tid == 0 && tied && key_of(above.value) >= lo && key_of(above.value) <= hi) add_ties((int)((hi - key_of(above.value)) >> shift));
        __syncthreads();
        reach(before, false);
        if (s.found[0] >= kBins) break;   // (cannot be: the range holds what is missing)
        const uint32_t part = (uint32_t)s.found[0], top = hi - (part << shift), width = (1u << shift) - 1;
        before = s.found[1];
        lo = top - lo > width ? top - width : lo;
        hi = top;
    }
    __syncthreads();
    const float value = of_key(hi);
    uint64_t ties = goal - before;
    if constexpr (MASS) {
        const uint64_t m = sc.mass(value);
        ties = m ? (ties + m - 1) / m : 1;
    }
    if (value == above.value && ties > above.ties) ties = above.ties;
    return Border{value, ties};
}

// A row per workgroup, read once for its largest logit, again for every histogram, and for the sums of its tiles; the word is found in its
// tile.
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void sample_kernel(Sample a) {
    __shared__ SampleLds<THREADS> s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *logits = static_cast<const T *>(a.logits) + row * a.stride;
        const int64_t V = a.words;
        const float temperature = a.temperatures ? a.temperatures[row] : a.temperature;
        const int64_t top_k = a.top_ks ? (a.top_k64 ? static_cast<const int64_t *>(a.top_ks)[row] : (int64_t)static_cast<const int32_t *>(a.top_ks)[row]) : a.top_k;
        const float top_p = a.top_ps ? a.top_ps[row] : a.top_p, min_p = a.min_ps ? a.min_ps[row] : a.min_p;
        const float u = a.u[row];

        float top = -INFINITY;
        bool odd = false;
        walk<T, THREADS>(logits, V, [&](int64_t, f32x8 v, int n) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float l = i < n ? v[i] : -INFINITY;
                top = fmaxf(top, l);
                odd |= l != l;
            }
        });
        top = wave_largest(top);
        odd = __builtin_amdgcn_ballot_w64(odd) != 0;
        __syncthreads();             // (the row before is done)
        if (lane == 0) s.waves[0][wave] = (uint64_t)odd << 32 | __float_as_uint(top);
        __syncthreads();
        odd = false;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            odd |= (s.waves[0][w] >> 32) != 0;
            top = fmaxf(top, __uint_as_float((uint32_t)s.waves[0][w]));
        }
        __syncthreads();
        if (odd || top == -INFINITY) {   // a NaN among the logits, or nothing to draw from
            if (tid == 0) {
                a.word[row] = -1;
                a.p[row] = odd ? NAN : 0.f;
            }
            continue;
        }
        if (!(temperature > 0.f)) {      // the first of the largest
            uint32_t at = 0xffffffffu;
            walk<T, THREADS>(logits, V, [&](int64_t c, f32x8 v, int n) {
#pragma unroll
                for (int i = 7; i >= 0; --i)
                    if (i < n && v[i] == top) at = min(at, (uint32_t)(c + i));
            });
            if (tid == 0) s.listed = 0xffffffffu;
            __syncthreads();
            if (at != 0xffffffffu) atomicMin(&s.listed, at);
            __syncthreads();
            if (tid == 0) {
                a.word[row] = (int64_t)s.listed;
                a.p[row] = 1.f;
            }
            continue;
        }
        Scale sc;
        sc.top = top;
        sc.per = kBinsPerUnit / temperature;
        sc.log2_per = 1.44269504088896340736 / (double)temperature;
        sc.least = min_p > 0.f ? (min_p < 1.f ? log((double)min_p) * (double)temperature : 0.0) : -INFINITY;
        sc.up = (double)((uint64_t)1 << a.mass_log);

        Border border{-INFINITY, 0};
        if (top_k > 0 && top_k < V) border = find_border<T, THREADS, false>(s, logits, V, sc, border, 0.0, (uint64_t)top_k);
        if (top_p < 1.f) border = find_border<T, THREADS, true>(s, logits, V, sc, border, top_p > 0.f ? (double)top_p : 0.0, 0);

        // masses of the tiles above the border, and how many logits are equal to it
        __syncthreads();
        for (int i = tid; i < kTiles; i += THREADS) {
            s.mass[i] = 0;
            s.count[i] = 0;
        }
        __syncthreads();
        auto above = [&](float l) { return l > border.value && sc.down(l) >= sc.least; };
        walk<T, THREADS>(logits, V, [&](int64_t c, f32x8 v, int n) {
            uint64_t sum = 0;
            uint32_t equal = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i < n && above(v[i])) sum += sc.mass(v[i]);
                equal += i < n && v[i] == border.value;
            }
            sum = wave_total(sum);
            if (__builtin_amdgcn_ballot_w64(equal != 0)) equal = (uint32_t)wave_total(equal);
            if (lane == 0) {
                const int tile = (int)(c >> (9 + a.tile_log));
                if (sum) atomicAdd((unsigned long long *)&s.mass[tile], (unsigned long long)sum);
                if (equal) atomicAdd(&s.count[tile], equal);
            }
        });
        __syncthreads();
        constexpr int EACH = kTiles / THREADS;
        const uint64_t tie = border.value > -INFINITY && sc.down(border.value) >= sc.least ? sc.mass(border.value) : 0;
        uint64_t masses[EACH], equals[EACH], sum = 0, equal = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            masses[i] = s.mass[tid * EACH + i];
            equal += equals[i] = border.value > -INFINITY ? s.count[tid * EACH + i] : 0;
        }
        uint64_t equal_before = block_scan(s, 0, equal, total) - equal;
        const uint64_t first_equal = equal_before;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const uint64_t room = equal_before < border.ties ? border.ties - equal_before : 0;
            masses[i] += (equals[i] < room ? equals[i] : room) * tie;
            equal_before += equals[i];
            sum += masses[i];
        }
        uint64_t at = block_scan(s, 1, sum, total) - sum;
        const float v01 = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
        const uint64_t target = (uint64_t)((double)v01 * (double)total);
        equal_before = first_equal;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (at <= target && at + masses[i] > target) {
                s.found[0] = (uint64_t)(tid * EACH + i);
                s.found[1] = at;
                s.found[2] = equal_before;
            }
            at += masses[i];
            equal_before += equals[i];
        }
        __syncthreads();
        if (wave == 0) {                 // the word, in its tile
            int64_t c = (int64_t)s.found[0] << (9 + a.tile_log);
            uint64_t before = s.found[1], seen = s.found[2];
            const int64_t end = c + ((int64_t)512 << a.tile_log) < V ? c + ((int64_t)512 << a.tile_log) : V;
            for (; c < end; c += 512) {
                const int64_t first = c + lane * 8;
                const int n = end - first < 8 ? (end - first > 0 ? (int)(end - first) : 0) : 8;
                const f32x8 v = load8(logits + first, n);
                uint32_t mine = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) mine += i < n && tie && v[i] == border.value;
                const uint64_t to_here = wave_scan(mine);
                uint64_t rank = seen + to_here - mine, m[8], own = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] = 0;
                    if (i < n) {
                        if (above(v[i])) m[i] = sc.mass(v[i]);
                        else if (tie && v[i] == border.value) m[i] = rank++ < border.ties ? tie : 0;
                    }
                    own += m[i];
                }
                const uint64_t upto = wave_scan(own);
                uint64_t sum_at = before + upto - own;
                if (sum_at <= target && sum_at + own > target) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (sum_at <= target && sum_at + m[i] > target) {
                            a.word[row] = first + i;
                            a.p[row] = (float)(sc.part(sc.down(v[i])) / ((double)total / sc.up));
                        }
                        sum_at += m[i];
                    }
                }
                before += lane64(upto, 63);
                seen += lane64(to_here, 63);
            }
        }
    }
}

}  // namespace saber_ops
