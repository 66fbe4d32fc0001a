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
// exact, so that neither their order nor atomics change a result, and e^z is computed in 64 bits to 1.1e-12, so that a border falls where 64-bit
// arithmetic puts it but for some 1e-7 of the random numbers (V 1e-12; in 32 bits it would be one in a hundred).  A word of less than 2^-(S + 1) of the likeliest one's mass has none and is never drawn.
// The histogram of all words adds up e^z relative to the middle of a bin, in whole multiples of 2^-40, which takes half the arithmetic and no
// largest logit; one factor per bin makes masses of its sums.  They differ from the sums of the masses, which are rounded word by word, by half a
// unit per word and by 3.2e-12 of the sum (errors of both exponentials, the multiples).  Where a border lies so near to the edge of a word's mass
// that this could move it, it is searched for again by the masses themselves: with natural logits and top_p 0.95 in one row of 7,700 of 100,000 words, in
// one of 1,900 of 141,000 (2048 such rows take 3 % longer for it).  A share counts as held from 2^-40 of the whole below it.
//
// What bounds it: for many rows the arithmetic in 64 bits, 20 instructions a logit for the histogram and 25 for a word that is left, beside two reads of the
// row, the second mostly from caches (2048 rows of 141,000 in binary32 with top_p 0.95 440 to 480 us, of which two reads alone 330; of top_k 50 333; four reads, of
// top_k 5000 and top_p, 730); for few rows one CU's arithmetic and a dozen phases of a workgroup that follow from each other, 0.5 to 3 us each (one row of 100,000
// with all limits 30 us, with top_p alone 48, with top_k 5000 and top_p 81, two reads 11); for rows of equal logits additions to one word of LDS (1024 rows of
// 100,000 in bf16 with top_k 50 935 us, 79 for natural ones; one row of binary32 239 and 22).
#pragma once
#include "ops_common.hpp"

namespace saber_ops {

struct Sample {
    const void *logits; int64_t stride;
    int64_t first_row, words;   // of the launch, a workgroup per row
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
template <int THREADS> constexpr int kList = THREADS == 256 ? 2048 : 4096;   // logits that are looked at in LDS
constexpr int kMaxima = 4;          // that a thread keeps
constexpr float kBinsPerUnit = 32.f;
constexpr int kZeroBin = 2046;      // bins from here on hold no mass: z < -31.9, e^z 2^45 < 1/2
constexpr float kRoom = 31.f;       // z of the first bin above the first logits' largest, where that of all is not known yet
constexpr double kBinLog2 = 1.44269504088896340736 / 32;   // log2 of e^z over a bin

// p r + c with c in scalar registers.  (The compiler keeps such constants in vector registers, two each, and has none left for them.)
__device__ __forceinline__ double times_plus(double p, double r, double c) {
#if defined(__HIP_DEVICE_COMPILE__)
    double o;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(o) : "v"(p), "v"(r), "s"(c));
    return o;
#else
    return fma(p, r, c);
#endif
}
// 2^r, |r| <= 1/2, to 1.1e-12: the interpolation at the Chebyshev nodes of degree 8
__device__ __forceinline__ double exp2_near(double r) {
    double p = times_plus(0x1.63d136366db24p-20, r, 0x1.00dc4a532fb8ep-16);
    p = times_plus(p, r, 0x1.4308ac85aa947p-13);
    p = times_plus(p, r, 0x1.5d8745a728441p-10);
    p = times_plus(p, r, 0x1.3b2ab7181b755p-7);
    p = times_plus(p, r, 0x1.c6b08dd6fd234p-5);
    p = times_plus(p, r, 0x1.ebfbdff823cedp-3);
    p = times_plus(p, r, 0x1.62e42fef84cf0p-1);
    return fma(p, r, 1.0);
}

// 2^r, |r| <= kBinLog2 / 2 and a hundredth more, to 5.2e-13: the same of degree 4
__device__ __forceinline__ double exp2_in_bin(double r) {
    double p = times_plus(0x1.3b2b8f7b7e9dfp-7, r, 0x1.c6b25d473c852p-5);
    p = times_plus(p, r, 0x1.ebfbdff7b8a25p-3);
    p = times_plus(p, r, 0x1.62e42feead6b2p-1);
    return fma(p, r, 1.0);
}

// The logits of a row relative to its largest.
struct Scale {
    float top, per;      // largest logit; bins per unit of a logit times `unit`
    float edge;          // where the first bin begins: at the largest logit or above it
    // 1, and 1/2 from T of 2^122 on: there a word may have mass whose logit is further from the largest than binary32 reaches, so both are halved
    // before they are subtracted (below, such a difference is 2046 bins or more)
    float unit;
    double log2_per;     // log2(e) / T
    double least;        // least difference that min_p leaves
    double up;           // 2^S
    double bin_up;       // 2^40, or 2^S if that is less
    // (of two infinities too)
    __device__ __forceinline__ double down(float l) const { return l == top ? 0.0 : (double)l - (double)top; }
    __device__ __forceinline__ int bin(float l) const {   // rises as the logit falls, by steps of 1/32 of z
        const float b = l == edge ? 0.f : fmaf(l, -unit, edge * unit) * per;
        return b < (float)kZeroBin ? (int)b : kZeroBin;   // (NaN, of -inf and T = inf, as well)
    }
    // the same for a finite edge and a unit of 1, and 0 above the edge; and e^z relative to the middle of that bin, in multiples of 1 / bin_up
    __device__ __forceinline__ int bin_below(float l) const { return (int)__builtin_amdgcn_fmed3f((edge - l) * per, 0.f, (float)kZeroBin); }
    __device__ __forceinline__ uint64_t mass_in_bin(float l, int b) const {
        const double r = fma((double)l - (double)edge, log2_per, times_plus((double)b, kBinLog2, kBinLog2 / 2));
        return (uint64_t)__double_as_longlong(fma(exp2_in_bin(r), bin_up, 0x1p52)) & 0xfffffffffffffull;
    }
    // masses of a bin, from the sum of the above
    __device__ __forceinline__ uint64_t mass_of_bin(uint64_t sum, int b) const {
        const double t = ((double)edge - (double)top) * log2_per - ((double)b + 0.5) * kBinLog2;
        return b < kZeroBin ? (uint64_t)((double)sum * (power(t) * (up / bin_up)) + 0.5) : 0;
    }
    // 2^t, t > -64
    __device__ __forceinline__ double power_near(double t) const {
        const double n = t + 0x1.8p52, r = t - (n - 0x1.8p52);
        const double e = exp2_near(r);
        return __longlong_as_double(__double_as_longlong(e) + (long long)((uint64_t)__double_as_longlong(n) << 52));
    }
    // 0 for what is too small to have a mass
    __device__ __forceinline__ double power(double t) const { return t > -64.0 ? power_near(t) : 0.0; }
    // e^z
    __device__ __forceinline__ double part(double d) const { return power(d * log2_per); }
    __device__ __forceinline__ uint64_t mass_of(double d) const {
        const double v = fma(part(d), up, 0x1p52);   // rounded to a whole number
        return (uint64_t)__double_as_longlong(v) & 0xfffffffffffffull;
    }
    __device__ __forceinline__ uint64_t mass(float l) const { return mass_of(down(l)); }
    // of a logit of a bin before kZeroBin, or one that min_p leaves: finite, or equal to the largest
    __device__ __forceinline__ uint64_t mass_left(float l) const {
        const double d = (double)fminf(l, 0x1.fffffep127f) - (double)fminf(top, 0x1.fffffep127f);
        const double v = fma(power_near(fmax(d * log2_per, -64.0)), up, 0x1p52);
        return (uint64_t)__double_as_longlong(v) & 0xfffffffffffffull;
    }
};

__device__ __forceinline__ uint32_t key_of(float f) {   // the order of the floats; -0 and 0 are equal
    const uint32_t b = __float_as_uint(f + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }

// a value that all lanes share, in scalar registers
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }
__device__ __forceinline__ float uniform(float v) { return __uint_as_float(uniform(__float_as_uint(v))); }
__device__ __forceinline__ uint64_t uniform(uint64_t v) { return (uint64_t)uniform((uint32_t)(v >> 32)) << 32 | uniform((uint32_t)v); }
__device__ __forceinline__ double uniform(double v) { return __longlong_as_double((long long)uniform((uint64_t)__double_as_longlong(v))); }

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
    v = fmaxf(v, dpp<0x128>(v));
    v = fmaxf(v, dpp<0x124>(v));
    v = fmaxf(v, dpp<0x122>(v));
    v = fmaxf(v, dpp<0x121>(v));
    const int b = __float_as_int(v);
    return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 0)), __int_as_float(__builtin_amdgcn_readlane(b, 16))),
                 fmaxf(__int_as_float(__builtin_amdgcn_readlane(b, 32)), __int_as_float(__builtin_amdgcn_readlane(b, 48))));
}
// sum over this lane and those before it: within the rows of 16 lanes by shifts (0 comes in), then the last lane of a row to the next one, then
// that of the second row to the third and fourth
template <int CTRL, int ROWS>
__device__ __forceinline__ uint64_t from_below(uint64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(v >> 32), CTRL, ROWS, 0xf, true);
    return (uint64_t)hi << 32 | lo;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v) {
    v += from_below<0x111, 0xf>(v);   // row_shr:1
    v += from_below<0x112, 0xf>(v);
    v += from_below<0x114, 0xf>(v);
    v += from_below<0x118, 0xf>(v);
    v += from_below<0x142, 0xa>(v);   // row_bcast:15, to rows 1 and 3
    v += from_below<0x143, 0xc>(v);   // row_bcast:31, to rows 2 and 3
    return v;
}

struct Border { float value; uint64_t ties; };   // all logits above the value, and the first few of those equal to it (one at least)

template <int THREADS, int TILES, int LIST>
struct SampleLds {
    union {
        uint64_t sums[kBins];                // of a bin's masses, or the number of its logits
        struct { float l[512]; uint32_t at[512]; } some[THREADS / 64];   // a wavefront's logits of a tile that are left, and their words
    };
    uint64_t tile_mass[TILES];       // above the border
    uint32_t tile_equal[TILES];      // logits equal to it
    float list[LIST];
    uint32_t at[LIST];              // their words
    uint64_t waves[2][THREADS / 64];
    uint64_t found[3];               // the last: sum of a histogram of masses, until the word is looked for
    uint32_t listed;
};

// f(first word, four logits) for all of a row, a tile of 512 words per wavefront at a time, AHEAD of them on their way; done(first word of
// the lane in the tile) after a lane's eight.  The logits after the last whole tile come one by one, -inf past the row's end (the kernel's code
// has to fit the instruction cache: with a check at every load it was 85 KB).
template <class T, int THREADS, int AHEAD, class F, class D>
__device__ __forceinline__ void walk(const T *row, int64_t words, F &&f, D &&done) {
    typedef float f32x4_ __attribute__((ext_vector_type(4)));
    struct __attribute__((packed, aligned(1))) Any { Raw8<T> r; };
    const int lane = threadIdx.x & 63;
    constexpr int64_t step = THREADS / 64 * 512;
    const int64_t whole = words & ~(int64_t)511;
#pragma unroll 1
    for (int64_t c0 = (int64_t)uniform(threadIdx.x >> 6) * 512; c0 < whole; c0 += AHEAD * step) {
        Raw8<T> raw[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t c = c0 + (c0 + k * step < whole ? k * step : 0);   // (past the end: any)
            raw[k] = reinterpret_cast<const Any *>(row + c + lane * 8)->r;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (c0 + k * step < whole) {
                const int64_t c = c0 + k * step + lane * 8;
                const f32x8 v = widen(raw[k]);
                const f32x4_ lo = v.lo, hi = v.hi;
                f(c, lo);
                __builtin_amdgcn_sched_barrier(0);
                f(c + 4, hi);
                __builtin_amdgcn_sched_barrier(0);
                done(c);
            }
    }
#pragma unroll 1
    for (int64_t c0 = whole + (int64_t)uniform(threadIdx.x >> 6) * 256; c0 < words; c0 += THREADS * 4) {
        const int64_t c = c0 + lane * 4;
        f32x4_ v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < words ? (float)row[c + i] : -INFINITY;
        f(c, v);
        done(c);
    }
}
template <class T, int THREADS, int AHEAD, class F>
__device__ __forceinline__ void walk(const T *row, int64_t words, F &&f) { walk<T, THREADS, AHEAD>(row, words, f, [](int64_t) {}); }

// A row of logits and a workgroup's work on it.
template <class T, int THREADS, int TILES>
struct Row {
    SampleLds<THREADS, TILES, kList<THREADS>> &s;
    const T *row;
    int64_t words;
    int tile_log;
    Scale sc;
    bool all_listed;                 // the list holds every logit that can be left
    int tid = threadIdx.x;

    __device__ __forceinline__ void clear() {
        __syncthreads();
        for (int i = tid; i < kBins; i += THREADS) s.sums[i] = 0;
        __syncthreads();
    }
    // sum over the threads up to and including this one, and over all of them
    __device__ __forceinline__ uint64_t scan(int which, uint64_t v, uint64_t &total) {
        constexpr int W = THREADS / 64;
        static_assert(W <= 16, "a row of lanes");
        const uint64_t own = wave_scan(v);
        if ((tid & 63) == 63) s.waves[which][tid >> 6] = own;
        __syncthreads();
        uint64_t upto = s.waves[which][tid & (W - 1)];   // the wavefronts' sums, in every row of lanes
        upto += from_below<0x111, 0xf>(upto);
        upto += from_below<0x112, 0xf>(upto);
        upto += from_below<0x114, 0xf>(upto);
        upto += from_below<0x118, 0xf>(upto);
        total = lane64(upto, W - 1);
        const int wave = (int)uniform(threadIdx.x >> 6);
        const uint64_t before = wave ? lane64(upto, wave - 1) : 0;
        __syncthreads();
        return before + own;
    }
    // The bin at which the sum of the bins from the first one on, and `before`, reaches the goal (kBins if there is none); `before` is then the
    // sum before it.  Where a share is asked for, the goal is that of the whole.
    __device__ __forceinline__ int reach(uint64_t &before, bool of_whole, double share, uint64_t &goal) {
        constexpr int EACH = kBins / THREADS;
        __syncthreads();
        uint64_t v[EACH], sum = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += v[i] = s.sums[tid * EACH + i];
        if (tid == 0) s.found[0] = kBins;
        const uint64_t upto = scan(0, sum, total);
        if (of_whole) {
            const double want = fmax((share - 0x1p-40) * (double)total, 1.0);   // (a share of 0: one word's, the likeliest)
            goal = (uint64_t)want;
            goal += (double)goal < want;
            goal = uniform(goal > total ? total : goal);
            if (tid == 0) s.found[2] = total;
        }
        uint64_t at = before + upto - sum;
        if (at < goal && at + sum >= goal) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                if (at < goal && at + v[i] >= goal) {
                    s.found[0] = (uint64_t)(tid * EACH + i);
                    s.found[1] = at;
                }
                at += v[i];
            }
        }
        __syncthreads();
        before = uniform(s.found[1]);
        return (int)uniform((uint32_t)s.found[0]);
    }
    // what a logit adds to its bin
    __device__ __forceinline__ void add(bool mass, int bin, float l) {
        atomicAdd((unsigned long long *)&s.sums[bin], mass ? (unsigned long long)sc.mass(l) : 1ull);
    }
    // the mass of the logits equal to the border above that count; by one thread
    __device__ __forceinline__ void add_ties(int bin, Border above) {
        atomicAdd((unsigned long long *)&s.sums[bin], (unsigned long long)(above.ties * sc.mass(above.value)));
    }
    __device__ __forceinline__ void put(float l, int64_t word) {
        const uint32_t n = atomicAdd(&s.listed, 1u);
        if (n < kList<THREADS>) {
            s.list[n] = l;
            s.at[n] = (uint32_t)word;
        }
    }
    __device__ __forceinline__ int tile_of(int64_t word) const { return (int)(word >> (9 + tile_log)); }

    // The least logit that holds, where all above a logit that holds do; NaN if the largest does not.  The 64 lanes try as many at a time.
    template <class F>
    __device__ __forceinline__ float least_of(F &&holds) const {
        if (!holds(sc.top)) return NAN;
        uint32_t lo = key_of(-INFINITY), hi = key_of(sc.top);
#pragma unroll 1
        while (lo < hi) {
            const uint32_t step = (hi - lo) / 64 + 1;
            const uint64_t yes = __builtin_amdgcn_ballot_w64(holds(of_key(lo + min((uint32_t)(tid & 63) * step, hi - lo))));   // (that of hi holds)
            const uint32_t first = yes ? (uint32_t)__builtin_ctzll(yes) : 64u;   // (64: beyond the last one tried)
            const uint32_t from = first ? lo + (first - 1) * step + 1 : lo;
            if (yes) hi = lo + min(first * step, hi - lo);
            lo = from;
        }
        return of_key(hi);
    }
    __device__ __forceinline__ float least_of_bin(int bin) const {
        return least_of([&](float l) { return sc.bin(l) <= bin; });
    }

    // Four logits of a lane that are not below `from`, after the n that the wavefront has put side by side already.
    template <class S, class V>
    __device__ __forceinline__ void side_by_side(S &some, uint32_t &n, int64_t c, V v, float from) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool is = v[i] >= from;
            const uint64_t all = __builtin_amdgcn_ballot_w64(is);
            if (is) {
                const uint32_t to = __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, n));
                some.l[to] = v[i];
                some.at[to] = (uint32_t)c + i;
            }
            n += (uint32_t)__builtin_popcountll(all);
        }
    }
    // the wavefront's lanes see what they wrote to LDS
    __device__ __forceinline__ void wave_lds_fence() const {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
    }

    // Lists all logits of the bins up to `last`, which is before kZeroBin; false if they are too many.
    __device__ __forceinline__ bool list_upto(int last) {
        if (tid == 0) s.listed = 0;
        __syncthreads();
        const float least = least_of_bin(last);
        walk<T, THREADS, 4>(row, words, [&](int64_t c, auto v) {   // (few: each takes its place by itself)
            bool hit[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) hit[i] = v[i] >= least;
            if (__builtin_amdgcn_ballot_w64(hit[0] | hit[1] | hit[2] | hit[3])) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (hit[i]) put(v[i], c + i);
            }
        });
        __syncthreads();
        return uniform(s.listed) <= (uint32_t)kList<THREADS>;
    }

    // First half of a border's search: the bin in which the logits in falling order reach the goal, or kZeroBin if they do not.  Only logits
    // above `above` count, and above.ties of those equal to it.  `ready`: the sums are there.
    __device__ __forceinline__ int find_bin(bool ready, bool mass, Border above, double share, uint64_t &goal, uint64_t &before) {
        if (!ready) clear();
        auto take = [&](float l) {
            const int b = sc.bin(l);
            if (b < kZeroBin && l > above.value) add(mass, b, l);
        };
        if (ready) ;
        else if (all_listed) {
            for (uint32_t i = tid; i < s.listed; i += THREADS) take(s.list[i]);
        } else
            walk<T, THREADS, 4>(row, words, [&](int64_t, auto v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) take(v[i]);
            });
        if (mass && tid == 0 && above.value > -INFINITY && sc.bin(above.value) < kZeroBin) add_ties(sc.bin(above.value), above);
        before = 0;
        const int bin = reach(before, mass, share, goal);
        return bin < kZeroBin ? bin : kZeroBin;
    }

    // Masses of the tiles (if `sums`) of the bins before `bin`, of logits that min_p leaves; and a list of that bin's logits, unless all are
    // listed.  Of a tile's logits few are left, as a rule: a wavefront puts them side by side first, so that it computes 64 masses that count at
    // a time (2048 rows of 141,000 words in binary32, min_p 0.05: 335 us; without a limit, with the masses of all, 386).
    __device__ __forceinline__ void sum_and_list(bool sums, int bin) {
        __syncthreads();
        for (int i = tid; i < TILES; i += THREADS) {
            s.tile_mass[i] = 0;
            s.tile_equal[i] = 0;
        }
        if (tid == 0 && !all_listed) s.listed = 0;
        __syncthreads();
        if (all_listed) {
            if (sums)
                for (uint32_t i = tid; i < s.listed; i += THREADS) {
                    const float l = s.list[i];
                    if (sc.bin(l) < bin && sc.down(l) >= sc.least) atomicAdd((unsigned long long *)&s.tile_mass[tile_of(s.at[i])], (unsigned long long)sc.mass(l));
                }
        } else if (bin < kZeroBin || sc.least > -INFINITY) {
            const int lane = tid & 63;
            auto &some = s.some[uniform(threadIdx.x >> 6)];
            // from `above` on: before the bin; from `left` on: of them, what min_p leaves; NaN: none
            const float above = bin == kZeroBin ? -INFINITY : bin ? least_of_bin(bin - 1) : NAN;
            float left = sums ? above : NAN;
            if (sums && sc.least > -INFINITY && above == above) left = fmaxf(above, least_of([&](float l) { return sc.down(l) >= sc.least; }));
            const float from = bin < kZeroBin ? least_of_bin(bin) : left;
            uint32_t n = 0;
            walk<T, THREADS, 4>(row, words, [&](int64_t c, auto v) { side_by_side(some, n, c, v, from); }, [&](int64_t c) {
                if (!n) return;
                wave_lds_fence();
                uint64_t sum = 0;
#pragma unroll 1
                for (uint32_t i = lane; i < n; i += 64) {
                    const float l = some.l[i];
                    if (l >= left) sum += sc.mass_left(l);
                    else if (!(l >= above)) put(l, some.at[i]);
                }
                wave_lds_fence();
                n = 0;
                if (!sums) return;
                sum = wave_total(sum);
                if (lane == 0 && sum) atomicAdd((unsigned long long *)&s.tile_mass[tile_of(c)], (unsigned long long)sum);
            });
        } else if (sums) {
            uint64_t sum = 0;
            walk<T, THREADS, 4>(row, words, [&](int64_t, auto v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += sc.mass(v[i]);
            }, [&](int64_t c) {
                sum = wave_total(sum);
                if ((tid & 63) == 0 && sum) atomicAdd((unsigned long long *)&s.tile_mass[tile_of(c)], (unsigned long long)sum);
                sum = 0;
            });
        }
        __syncthreads();
    }

    // f(logit, word) for the logits of a bin: of the list, or if they did not fit, of the row.
    template <class F>
    __device__ __forceinline__ void of_bin(int bin, F &&f) {
        if (s.listed <= (uint32_t)kList<THREADS>) {
            for (uint32_t i = tid; i < s.listed; i += THREADS)
                if (sc.bin(s.list[i]) == bin) f(s.list[i], (int64_t)s.at[i]);
        } else
            walk<T, THREADS, 1>(row, words, [&](int64_t c, auto v) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (sc.bin(v[i]) == bin) f(v[i], c + i);
            });
    }

    // Second half: within the bin, by histograms of the keys lo .. hi, the largest first, in ever smaller ranges.  `rough`: goal and sum are of the
    // histogram of all words; no ties then: the border is not sure.
    __device__ __forceinline__ Border border_in(bool mass, int bin, Border above, uint64_t goal, uint64_t before, bool rough, int mass_log) {
        const uint32_t above_key = key_of(above.value);
        const bool tied = mass && above.value > -INFINITY && sc.bin(above.value) == bin;
        uint32_t lo = 0, hi = 0xffffffffu;
#pragma unroll 1
        while (true) {
            // to the keys that are there: often a single one
            uint32_t least = 0xffffffffu, most = 0;
            of_bin(bin, [&](float l, int64_t) {
                const uint32_t k = key_of(l);
                if (l > above.value && k >= lo && k <= hi) {
                    least = min(least, k);
                    most = max(most, k);
                }
            });
            if (tied && above_key >= lo && above_key <= hi) {
                least = min(least, above_key);
                most = max(most, above_key);
            }
            least = ~wave_max(~least);
            most = wave_max(most);
            if ((tid & 63) == 0) s.waves[0][tid >> 6] = (uint64_t)least << 32 | most;
            __syncthreads();
            const uint64_t other = s.waves[0][tid & (THREADS / 64 - 1)];
            lo = uniform(~wave_max(~(uint32_t)(other >> 32)));
            hi = uniform(wave_max((uint32_t)other));
            if (lo >= hi) {
                __syncthreads();
                break;
            }
            const int shift = 31 - __builtin_clz((hi - lo) >> 10 | 1u);   // ((hi - lo) >> shift) < 2048
            clear();
            of_bin(bin, [&](float l, int64_t) {
                const uint32_t k = key_of(l);
                if (l > above.value && k >= lo && k <= hi) add(mass, (int)((hi - k) >> shift), l);
            });
            if (tied && tid == 0 && above_key >= lo && above_key <= hi) add_ties((int)((hi - above_key) >> shift), above);
            const int part = reach(before, false, 0.0, goal);
            if (part >= kBins) return Border{-INFINITY, 0};   // (the bin's sum was greater by its rounding)
            const uint32_t top = hi - ((uint32_t)part << shift), width = (1u << shift) - 1;
            lo = top - lo > width ? top - width : lo;
            hi = top;
        }
        const float value = of_key(hi);
        uint64_t ties = goal - before;
        if (mass) {
            const uint64_t m = uniform(sc.mass(value));
            ties = m ? (ties + m - 1) / m : 1;
            if (rough) {
                // The sum before a word is off by the errors of the words before it, the goal by the share of all of them: their difference by no more than
                // all words' errors are.  Half a unit for a word and for a bin; 3.2e-12 of the whole, 2^-(S + 1) more where the multiples are 2^-S.
                const uint64_t off = (uint64_t)(words + kBins) / 2 + 2 + (uniform(s.found[2]) >> min(mass_log - 2, 38)), at = before + (ties - 1) * m;
                if ((at && goal - at <= off) || at + m - goal < off) return Border{-INFINITY, 0};
            }
        }
        if (value == above.value && ties > above.ties) ties = above.ties;
        return Border{value, ties};
    }

    // what of the border's bin is above it, and how many are equal
    __device__ __forceinline__ void add_bin(int bin, Border border) {
        of_bin(bin, [&](float l, int64_t word) {
            if (l > border.value) {
                if (sc.down(l) >= sc.least) atomicAdd((unsigned long long *)&s.tile_mass[tile_of(word)], (unsigned long long)sc.mass(l));
            } else if (l == border.value)
                atomicAdd(&s.tile_equal[tile_of(word)], 1u);
        });
        __syncthreads();
    }
};

// A row per workgroup.  It is read once for its largest logit and, if top_k is not small or top_p is given, the first limit's histogram; then, if
// top_k is small, once to list the few logits that can be left, among them the top_k largest of the threads' own maxima; else once for the masses of
// its tiles of 512 words and a list of the bin with the border (top_k not small and top_p: both a second time, for top_p).  The word is found
// in its tile.  A top_k is small up to twice the workgroup's threads: of 2048 rows of 141,000 in binary32 1000 words with top_p 0.9 take 361 us, 1100 669.
// (No loop over rows: what the compiler moved out of one did not fit the registers and took a third longer for 2048 rows of 141,000 with top_p.  As it is
// some 45 scalar registers wait in lanes of vector registers, and two vector registers of the variant of 256 threads in memory.)
template <class T, int THREADS, int TILES>
__global__ __launch_bounds__(THREADS, 4) void sample_kernel(Sample a) {
    __shared__ SampleLds<THREADS, TILES, kList<THREADS>> s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = a.first_row + blockIdx.x;
    const T *logits = static_cast<const T *>(a.logits) + row * a.stride;
    const int64_t V = a.words;
    const float temperature = uniform(a.temperatures ? a.temperatures[row] : a.temperature);
    const int64_t top_k = (int64_t)uniform((uint64_t)(a.top_ks ? (a.top_k64 ? static_cast<const int64_t *>(a.top_ks)[row] : (int64_t)static_cast<const int32_t *>(a.top_ks)[row]) : a.top_k));
    const float top_p = uniform(a.top_ps ? a.top_ps[row] : a.top_p), min_p = uniform(a.min_ps ? a.min_ps[row] : a.min_p);
    const float u = a.u[row];

    const bool greedy = !(temperature > 0.f), has_k = !greedy && top_k > 0 && top_k < V, has_p = !greedy && top_p < 1.f;
    const bool few = has_k && top_k <= kMaxima * THREADS / 2;
    Scale sc;
    sc.unit = uniform(temperature > 0x1p122f ? 0.5f : 1.f);
    sc.per = uniform(fminf(kBinsPerUnit / temperature, 0x1.fffffep127f) / sc.unit);
    sc.log2_per = uniform(1.44269504088896340736 / (double)temperature);
    sc.up = (double)((uint64_t)1 << a.mass_log);
    sc.bin_up = (double)((uint64_t)1 << (a.mass_log < 40 ? a.mass_log : 40));
    Row<T, THREADS, TILES> r{s, logits, V, a.tile_log, sc, false};

    // a wave's largest value and whether any is odd, over the workgroup
    auto join = [&](float &most, bool &any) {
        most = wave_largest(most);
        any = __builtin_amdgcn_ballot_w64(any) != 0;
        __syncthreads();
        if (lane == 0) s.waves[0][wave] = (uint64_t)any << 32 | __float_as_uint(most);
        __syncthreads();
        const uint64_t other = s.waves[0][lane & (THREADS / 64 - 1)];
        any = __builtin_amdgcn_ballot_w64((other >> 32) != 0) != 0;
        most = wave_largest(__uint_as_float((uint32_t)other));
    };
    bool ready = !few && (has_k || has_p), odd = false;
    if (ready) {                     // a histogram at once, from the largest of the first logits plus some room on
        const int64_t c = (int64_t)tid * 8;
        const f32x8 v = load8(logits + c, V - c);
        float first = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) first = fmaxf(first, c + i < V ? v[i] : -INFINITY);
        join(first, odd);
        r.sc.edge = uniform(first + kRoom * temperature);
        // (its masses are of bins of 1/32 of z: not where 32 / T is no number of binary32 and `per` is less; its differences are not halved)
        ready = fabsf(r.sc.edge) < INFINITY && kBinsPerUnit / temperature < INFINITY && r.sc.unit == 1.f;
        r.clear();
    }
    float own[kMaxima];
#pragma unroll
    for (int i = 0; i < kMaxima; ++i) own[i] = -INFINITY;
    odd = false;
    auto largest = [&](auto v) {
#pragma unroll
        for (int i = 0; i < kMaxima; ++i) {
            own[i] = fmaxf(own[i], v[i]);
            if (i & 1) odd |= __builtin_isunordered(v[i - 1], v[i]);
        }
    };
    if (ready && has_k)
        walk<T, THREADS, 4>(logits, V, [&](int64_t, auto v) {
            largest(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = r.sc.bin_below(v[i]);
                if (b < kZeroBin) atomicAdd((unsigned long long *)&s.sums[b], 1ull);
            }
        });
    else if (ready)
        walk<T, THREADS, 4>(logits, V, [&](int64_t, auto v) {
            largest(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int b = r.sc.bin_below(v[i]);
                if (b < kZeroBin) atomicAdd((unsigned long long *)&s.sums[b], (unsigned long long)r.sc.mass_in_bin(v[i], b));   // (many masked words would meet there)
            }
        });
    else
        walk<T, THREADS, 4>(logits, V, [&](int64_t, auto v) { largest(v); });
    float top = fmaxf(fmaxf(own[0], own[1]), fmaxf(own[2], own[3]));
    join(top, odd);
    __syncthreads();
    if (odd || top == -INFINITY) {   // a NaN among the logits, or nothing to draw from
        if (tid == 0) {
            a.word[row] = -1;
            a.p[row] = odd ? NAN : 0.f;
        }
        return;
    }
    if (greedy) {                    // the first of the largest
        uint32_t at = 0xffffffffu;
        walk<T, THREADS, 4>(logits, V, [&](int64_t c, auto v) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (v[i] == top) at = min(at, (uint32_t)(c + i));
        });
        if (tid == 0) s.listed = 0xffffffffu;
        __syncthreads();
        if (at != 0xffffffffu) atomicMin(&s.listed, at);
        __syncthreads();
        if (tid == 0) {
            a.word[row] = (int64_t)s.listed;
            a.p[row] = 1.f;
        }
        return;
    }
    ready = ready && top <= r.sc.edge;   // (else a later logit was far above the first ones)
    r.sc.top = top;
    if (!ready) r.sc.edge = top;
    r.sc.least = uniform(min_p > 0.f ? (min_p < 1.f ? log((double)min_p) * (double)temperature : 0.0) : -INFINITY);
    if (ready && !has_k)
        for (int i = tid; i < kBins; i += THREADS) s.sums[i] = r.sc.mass_of_bin(s.sums[i], i);

    Border border{-INFINITY, 0};
    uint64_t goal = (uint64_t)top_k, before = 0;
    if (few) {
        // the k-th largest logit is not below the k-th largest of the threads' maxima
        r.clear();
#pragma unroll
        for (int i = 0; i < kMaxima; ++i)
            if (own[i] > -INFINITY && r.sc.bin(own[i]) < kZeroBin) r.add(false, r.sc.bin(own[i]), own[i]);
        const int last = r.reach(before, false, 0.0, goal);
        if (last < kZeroBin) r.all_listed = r.list_upto(last);
    }
    int summed = -1;                 // bin whose list and tiles' masses are there
#pragma unroll 1
    for (int limit = 0; limit < 3; ++limit) {       // top_k, top_p, and where there is neither the sums alone
        if (limit == 0 ? !has_k : limit == 1 ? !has_p : has_k || has_p) continue;
        const bool mass = limit == 1, sums = limit > 0 || !has_p;
        const int bin = limit == 2 ? kZeroBin : r.find_bin(ready, mass, border, top_p > 0.f ? (double)top_p : 0.0, goal, before);
        const bool rough = ready;
        ready = false;
        if (bin != summed) r.sum_and_list(sums, bin);
        summed = -1;
        if (bin < kZeroBin) {
            border = r.border_in(mass, bin, border, goal, before, rough, a.mass_log);
            if (rough && !border.ties) {          // once more, by the masses; as a rule in the same bin
                --limit;
                summed = bin;
            } else if (sums) r.add_bin(bin, border);
        }
    }

    constexpr int EACH = (TILES + THREADS - 1) / THREADS;
    const uint64_t tie = border.value > -INFINITY && r.sc.down(border.value) >= r.sc.least ? r.sc.mass(border.value) : 0;
    uint64_t masses[EACH], equals[EACH], sum = 0, equal = 0, total;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool is = tid * EACH + i < TILES;
        masses[i] = is ? s.tile_mass[tid * EACH + i] : 0;
        equal += equals[i] = is ? s.tile_equal[tid * EACH + i] : 0;
    }
    uint64_t equal_before = r.scan(0, equal, total) - equal;
    const uint64_t first_equal = equal_before;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const uint64_t room = equal_before < border.ties ? border.ties - equal_before : 0;
        masses[i] += (equals[i] < room ? equals[i] : room) * tie;
        equal_before += equals[i];
        sum += masses[i];
    }
    uint64_t at = r.scan(1, sum, total) - sum;
    const float within = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
    const uint64_t target = (uint64_t)((double)within * (double)total);
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
        uint64_t sum_before = s.found[1], seen = s.found[2];
        const int64_t end = c + ((int64_t)512 << a.tile_log) < V ? c + ((int64_t)512 << a.tile_log) : V;
        for (; c < end; c += 512) {
            const int64_t first = c + lane * 8;
            const int n = end - first < 8 ? (end - first > 0 ? (int)(end - first) : 0) : 8;
            const f32x8 v = load8(logits + first, n);
            uint32_t mine = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) mine += i < n && tie && v[i] == border.value;
            const uint64_t to_here = wave_scan(mine);
            uint64_t rank = seen + to_here - mine, m[8], own_sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = 0;
                if (i < n) {
                    if (v[i] > border.value && r.sc.down(v[i]) >= r.sc.least) m[i] = r.sc.mass(v[i]);
                    else if (tie && v[i] == border.value) m[i] = rank++ < border.ties ? tie : 0;
                }
                own_sum += m[i];
                __builtin_amdgcn_sched_barrier(0);
            }
            const uint64_t upto = wave_scan(own_sum);
            uint64_t sum_at = sum_before + upto - own_sum;
            if (sum_at <= target && sum_at + own_sum > target) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (sum_at <= target && sum_at + m[i] > target) {
                        a.word[row] = first + i;
                        a.p[row] = (float)(r.sc.part(r.sc.down(v[i])) / ((double)total / r.sc.up));
                    }
                    sum_at += m[i];
                }
            }
            sum_before += lane64(upto, 63);
            seen += lane64(to_here, 63);
        }
    }
}

}  // namespace saber_ops
