// Matrix products of the head on the matrix cores: D[m][n] = sum over k of A[m][k] B[n][k], with either operand stored with k
// fastest or with k slowest, and an epilogue that consumes the tile from registers.
//
// A workgroup of four wavefronts computes a BM x BN tile in steps of 64 along k.  Operands go from memory to LDS directly (16 bytes a
// lane), up to two steps ahead of the arithmetic.  LDS is written in order of the lanes; what a lane fetches is permuted instead, so
// that the reads of a fragment meet different banks:
//   k fastest: a row of 64 k is 8 pieces of 16 bytes; piece p of row r lies at p ^ (r & 7); a lane reads its 8 values of k at once.
//   k slowest: a row holds U = 128 (64) columns in pieces of 16 bytes; piece p of row k lies at p ^ 2 f(k), f(k) = (k & 3) | (k & 8) >> 1
//              (k & 3); a lane's 8 values of k come through two transposing reads of 4 rows x 16 columns each.
// What bounds it: the matrix cores, which draw so much power here that a loop of nothing but these products reaches 1.55 to 1.6 PFLOP/s;
// and the requests, which take turns with them in each wave.  In bf16, 256 x 256: logits of 4096 rows of 1024 and 100,000 words 0.93 ms,
// 900 TFLOP/s; 8192 rows of 1000 and 141,000 words 2.70 ms, 855; the products of both gradients, of 32,768 words, 230 us, 1.19 PFLOP/s.
// Tried and slower: products of 32 x 32 (fewer cycles, more power), steps of 32 along k (twice the requests), operands through registers,
// eight waves a tile.
// Rows and columns outside the operands are read as zeros (the bounds of the buffer descriptors), so no tile reads out of range.
//
// Operands of binary32 come as planes, and the products of planes that matter are added as further steps along k ("segments"):
//   three planes of bfloat16, x = x1 + x2 + x3 exactly (8 bits of the significand each), six segments, any range of values; what is left
//   out (x2 y3, x3 y2, x3 y3) is up to 2^-21 of the product, always to the side of zero, as the planes are cut off;
//   two planes of binary16, x = x1 + x2 to 2^-23, three segments, for operands whose rows were brought to one magnitude and hold little
//   that is far below it; what is left out is up to 2^-22 of the product of two magnitudes.  Tiles of other rows are left to another
//   kernel.
#pragma once
#include <type_traits>
#include <utility>

#include "ops_common.hpp"

namespace saber_ops {

constexpr int kStep = 64;   // k per step

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// One operand: `major` rows (of m or n) by k, 16-bit elements.
struct Operand {
    const void *p;
    int64_t stride;      // elements between its stored rows (multiple of 8; p is aligned to 16 bytes)
    int64_t plane;       // elements between its planes
    int64_t major;       // extent of m (n); a multiple of 8 if k is slowest
};
struct Product {
    Operand a, b;
    uint32_t k;          // extent of k; where k is fastest the stored rows go on to the next multiple of 8, with zeros in one operand
    int segments;        // 1, or 6 or 3 for planes
    int tiles_m, tiles_n;
    int splits;          // parts of the steps along k, each a workgroup of its own
};

// planes that a segment multiplies: the largest two last
__device__ __forceinline__ int plane_a(int seg, int segments) { return ((segments == 6 ? 0x001012 : segments == 3 ? 0x001 : 0) >> (4 * seg)) & 15; }
__device__ __forceinline__ int plane_b(int seg, int segments) { return ((segments == 6 ? 0x010210 : segments == 3 ? 0x010 : 0) >> (4 * seg)) & 15; }

// f(0), f(1) .. f(N - 1) with the number as a constant
template <int... I, class F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F &&f) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F &&f) { each(std::make_integer_sequence<int, N>{}, f); }

// One product.  With 64 of them a wave's sums are 256 registers, which have to stay in accumulation registers, each in its place; the
// compiler moves them about, so here they are bound in assembly.  Two waits are the program's then: an operand that a vector
// instruction wrote may be read two states later (FIRST: of a row of fragments; all of them come from LDS, which has a counter), and
// the sums may be read seven states after their last product (settled()).  Waiting before every product would cost 2 to 4 % of a training
// step, so that the compiler puts no vector instruction in between is checked in the built code (tests/test_ops_waits.py).
template <class T, bool FIRST>
__device__ __forceinline__ void mfma(u32x4 a, u32x4 b, f32x4 &c) {
    if constexpr (FIRST) asm volatile("s_nop 1");
    if constexpr (std::is_same<T, bf16>::value) asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
    else asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b));
}
template <int M, int N>
__device__ __forceinline__ void settled(f32x4 (&c)[M][N]) {
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int j = 0; j < N; j += 2) asm volatile("s_nop 7" : "+a"(c[i][j]), "+a"(c[i][j + 1]));
}

using LdsBytes = __attribute__((address_space(3))) char;

template <int U>
__device__ __forceinline__ int slow_swizzle(int k) { return ((k & 3) | (U == 128 ? (k & 8) >> 1 : 0)) << 1; }

// 16 bytes per lane from the buffer to LDS, lane after lane from `lds` on, past the registers.  Nothing waits for it but a wait for
// the vector memory counter; in assembly, because the compiler puts such a wait in front of every later read of LDS.  The load has no
// result register, so there is none that could be used too early.  m0 needs a state between its write and its use, the addition; the
// descriptor five if a vector instruction wrote it, which the same test checks.
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, LdsBytes *lds, uint32_t off, uint32_t more) {
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
    uint32_t sum;
    asm volatile("s_mov_b32 m0, %1\n\tv_add_u32 %0, %2, %3\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds" : "=&v"(sum) : "s"(at), "s"(more), "v"(off), "s"(rsrc) : "memory");
}
// a raw buffer: base, bytes; accesses outside read zeros
__device__ __forceinline__ u32x4 buffer_of(const char *p, uint32_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// LDS is a ring of units: U = 128 (64) rows of m (n) by 64 k, in the layout above; 16 (8) KB.
// How a wave fetches its share of one operand's tile of W columns (or rows) of m, unit by unit.
template <bool SLOW, int W, int U, int WAVES>
struct Loader {
    static constexpr int kEach = U * kStep * 2 / 1024 / WAVES;   // requests of a wave per unit, 1 KB each
    static constexpr int kAll = kEach * (W / U);                 // and per step
    static constexpr int kPieces = SLOW ? U / 8 : 8;             // of 16 bytes, in a stored row
    static constexpr int kRows = 64 / kPieces;                   // stored rows that one request covers
    static_assert(WAVES == 4 && (U == 128 || U == 64), "the permutation's dependence on the request");
    const char *base;        // first element of the tile, plane 0
    uint32_t stride_bytes;
    int64_t plane_bytes;
    uint32_t extent;         // k fastest: bytes from the tile's first row to its last one's start; k slowest: bytes of a row
    uint32_t voff;           // of the wave's first request
    int piece_k;             // k fastest: first k of the lane's piece; k slowest: its piece
    int lane_k, wave_k;      // k slowest: the stored row of the lane's piece within a request, and of the wave's first request

    __device__ __forceinline__ void init(const Operand &o, int64_t origin, int wave, int lane) {
        stride_bytes = (uint32_t)o.stride * 2;
        plane_bytes = o.plane * 2;
        if constexpr (SLOW) {
            base = static_cast<const char *>(o.p) + origin * 2;
            extent = (uint32_t)((o.major - origin < W ? o.major - origin : W) * 2);
            voff = (wave * kEach * kRows + lane / kPieces) * stride_bytes;
            piece_k = lane % kPieces;
            lane_k = lane / kPieces;
            wave_k = wave * kEach * kRows;
        } else {
            base = static_cast<const char *>(o.p) + origin * (int64_t)stride_bytes;
            extent = (uint32_t)((o.major - origin < W ? o.major - origin : W) - 1) * stride_bytes;
            const int c = (lane & 7) ^ (lane >> 3);
            piece_k = c * 8;
            voff = (wave * kEach * kRows + (lane >> 3)) * stride_bytes + c * 16;
        }
    }
    // the step that is being asked for: its descriptor and the lane's offset in it (for a unit's first two requests, for the others)
    u32x4 rsrc;
    uint32_t off[2];
    int left;                // steps of the segment from it on
    __device__ __forceinline__ void begin(int plane, uint32_t k0, uint32_t k_end, bool any) {
        const char *p = base + plane * plane_bytes;
        uint32_t bytes, at = voff;
        left = any ? (int)((k_end - k0 + kStep - 1) / kStep) : 0x7fffffff;
        if constexpr (SLOW) {
            p += (uint64_t)k0 * stride_bytes;
            bytes = ((k_end - k0 < kStep ? k_end - k0 : kStep) - 1) * stride_bytes + extent;
        } else {
            p += k0 * 2;
            const uint32_t more = (k_end + 7) / 8 * 8 - k0;
            bytes = extent + more * 2;
            if ((uint32_t)piece_k >= more) at = 0x80000000u;     // past the row's end: out of the descriptor's bounds
        }
        rsrc = buffer_of(p, any ? bytes : 0);                    // past the last step: zeros that nobody uses
        off[0] = off[1] = at;
        if constexpr (SLOW) {                                    // the permutation is one for the first two requests, one for the others
            off[0] += (uint32_t)(piece_k ^ slow_swizzle<U>(lane_k + wave_k)) * 16;
            off[1] += (uint32_t)(piece_k ^ slow_swizzle<U>(lane_k + wave_k + 2 * kRows)) * 16;
        }
    }
    // the next step of a segment that has one after it which is whole
    __device__ __forceinline__ void next() {
        uint64_t p = rsrc[0] | (uint64_t)rsrc[1] << 32;
        p += SLOW ? kStep * (uint64_t)stride_bytes : kStep * 2;
        rsrc[0] = (uint32_t)p;
        rsrc[1] = (uint32_t)(p >> 32);
        if constexpr (!SLOW) rsrc[2] -= kStep * 2;
        --left;
    }
    // request j of the step; lds: the wave's place in the unit that it belongs to
    __device__ __forceinline__ void one(LdsBytes *lds, int j) const {
        const int u = j / kEach, i = j % kEach;
        load_to_lds(rsrc, lds + i * 1024, off[SLOW ? i >> 1 : 0], i * kRows * stride_bytes + (SLOW ? u * U * 2 : u * U * stride_bytes));
    }
};

// Fragments of 16 rows of m by 32 values of k: lane l holds row l % 16, k 8 (l / 16) .. + 7.  The addresses of a lane differ between
// fragments by constants, up to the permutation: a register per distinct one, the rest are the instructions' own offsets.
template <bool SLOW, int U, int N>
struct Reader {
    uint32_t at[SLOW ? N : 2];
    __device__ __forceinline__ void init(int row, int lane) {   // row: of the unit
        if constexpr (SLOW) {
            // lane l of 16 addresses row k + l / 4 of four, columns 4 (l % 4) .. + 3; it receives column l of the four rows
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2), col = row + 4 * (lane & 3);
#pragma unroll
            for (int i = 0; i < N; ++i) at[i] = k * U * 2 + (((col + 16 * i) * 2) ^ (slow_swizzle<U>(k) * 16));
        } else {
            at[0] = (row + (lane & 15)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
            at[1] = at[0] ^ 64;
        }
    }
    // fragment i along m of the unit at lds; kk: 0 or 32
    __device__ __forceinline__ u32x4 get(const LdsBytes *lds, int i, int kk) const {
        if constexpr (SLOW) {   // (k + 4 and k + 32 are permuted like k)
            using P = __attribute__((address_space(3))) s16x4 *;
            union { s16x4 h[2]; u32x4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at[i] + kk * U * 2));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at[i] + (kk + 4) * U * 2));
            return u.v;
        } else
            return *(const __attribute__((address_space(3))) u32x4 *)(lds + at[kk / 32] + i * 16 * 128);
    }
};

// Workgroups go round the eight XCDs; each XCD gets a run of neighbouring tiles, eight of n by all of m, so that what its
// workgroups read at a time meets in its L2.
__device__ __forceinline__ void tile_of_workgroup(const Product &p, uint32_t id, int &split, int &tm, int &tn) {
    const uint32_t plane_tiles = (uint32_t)p.tiles_m * p.tiles_n, tiles = plane_tiles * p.splits;
    {
        const uint32_t each = tiles / 8, more = tiles % 8, x = id % 8;
        id = x * each + (x < more ? x : more) + id / 8;
    }
    split = (int)(id / plane_tiles);
    id -= split * plane_tiles;
    const int group = (int)(id / (p.tiles_m * 8u));
    const int width = p.tiles_n - group * 8 < 8 ? p.tiles_n - group * 8 : 8;
    const int in_group = (int)(id - group * (p.tiles_m * 8u));
    tm = in_group / width;
    tn = group * 8 + in_group % width;
}

// the tiles that a product leaves to another kernel
struct None {
    template <int BM, int BN>
    __device__ __forceinline__ bool has(int64_t, int64_t, int64_t, int64_t, int) const { return false; }
};

template <class T, bool A_SLOW, bool B_SLOW, int BM, int BN, int WM, int WN, class Epilogue, class LeftOut>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product p, Epilogue e, LeftOut left_out) {
#if defined(__HIP_DEVICE_COMPILE__)   // (the host pass knows neither the matrix instructions nor their types)
    constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int U = BM < 128 ? BM : 128, kUnitBytes = U * kStep * 2;
    constexpr int UA = BM / U, UB = BN / U, UNITS = UA + UB, RING = UNITS * 5 / 2;           // units of a step, and in LDS
    static_assert(UA == UB, "the order of requests");
    __shared__ __attribute__((aligned(1024))) char smem[RING * kUnitBytes];
    LdsBytes *const lds = (LdsBytes *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    int split, tm, tn;
    tile_of_workgroup(p, blockIdx.x, split, tm, tn);
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;
    if (left_out.template has<BM, BN>(m0, n0, p.a.major, p.b.major, lane)) return;

    Loader<A_SLOW, BM, U, WAVES> la;
    Loader<B_SLOW, BN, U, WAVES> lb;
    la.init(p.a, m0, wave, lane);
    lb.init(p.b, n0, wave, lane);
    const int wm = (wave / WN) * TM * 16, wn = (wave % WN) * TN * 16;
    Reader<A_SLOW, U, TM> ra;
    Reader<B_SLOW, U, TN> rb;
    ra.init(wm % U, lane);
    rb.init(wn % U, lane);

    const int per_seg = (int)((p.k + kStep - 1) / kStep), steps = per_seg * p.segments;
    const int first = (int)((int64_t)steps * split / p.splits), last = (int)((int64_t)steps * (split + 1) / p.splits);

    typename Epilogue::template State<TN> state;       // what the epilogue reads of its columns: on its way during the loop
    e.prepare(state, n0 + wn + (lane & 15));

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    // A step has two halves of 32 k: while the matrix cores work on one half's fragments, the next half's are read.  It goes in GROUPS
    // groups of one row of fragments each, with one request for data to come in each group: the path from memory to LDS serves
    // requests at just the pace of the products, and a wave that has to wait for it is one that multiplies nothing.
    // Before group FREE everyone has read all of step s.  The ring has room for two and a half steps, so B of step s + 2 then goes where
    // A of step s was, and A of step s + 3 where B of step s was.  Before group NEED step s + 1 has arrived.
    constexpr int LA = Loader<A_SLOW, BM, U, WAVES>::kAll, LB = Loader<B_SLOW, BN, U, WAVES>::kAll, EACH = Loader<A_SLOW, BM, U, WAVES>::kEach;
    constexpr int GROUPS = 2 * TM, FREE = TM / 2 + 1, NEED = TM + TM / 2;
    static_assert(LA + LB == GROUPS, "one request per group");
    constexpr int READ1 = (TM + TN + FREE - 2) / (FREE - 1);                 // reads per group: of k 32 .. 63, in groups 0 .. FREE - 2
    constexpr int READ0 = (TM + TN + GROUPS - NEED - 1) / (GROUPS - NEED);   // of the next step's k 0 .. 31, from group NEED on
    constexpr int MOVE = TN > 3 ? TN - 3 : 0;                                // the product after which the next step is gone to
    constexpr int AHEAD = GROUPS - FREE - LB;                                // requests for A of step s + 2 before step s begins
    u32x4 fa[2][TM], fb[2][TN];
    // where a step's data is asked for: the next step of its segment, or, rarely, another segment, a step that ends in mid-air, or none
    int seg_a = first / per_seg, seg_b = seg_a, todo_a = last - first, todo_b = todo_a;
    const uint32_t k_first = (uint32_t)(first - seg_a * per_seg) * kStep;
    la.begin(plane_a(seg_a, p.segments), k_first, p.k, todo_a > 0);
    lb.begin(plane_b(seg_b, p.segments), k_first, p.k, todo_b > 0);
    auto next_a = [&] {
        --todo_a;
        if (la.left > 2) la.next();
        else if (la.left == 2) la.begin(plane_a(seg_a, p.segments), (per_seg - 1) * kStep, p.k, todo_a > 0);
        else { seg_a += todo_a > 0; la.begin(plane_a(seg_a, p.segments), 0, p.k, todo_a > 0); }
        if (todo_a <= 0) la.rsrc[2] = 0;
    };
    auto next_b = [&] {
        --todo_b;
        if (lb.left > 2) lb.next();
        else if (lb.left == 2) lb.begin(plane_b(seg_b, p.segments), (per_seg - 1) * kStep, p.k, todo_b > 0);
        else { seg_b += todo_b > 0; lb.begin(plane_b(seg_b, p.segments), 0, p.k, todo_b > 0); }
        if (todo_b <= 0) lb.rsrc[2] = 0;
    };
    // places in the ring; the wave's own part of a unit
    auto after = [&](LdsBytes *q, int units) { q += units * kUnitBytes; return q >= lds + RING * kUnitBytes ? q - RING * kUnitBytes : q; };
    const int own = wave * EACH * 1024;
    LdsBytes *to_a = lds, *to_b = lds + UA * kUnitBytes;                     // of the step that is asked for
    auto request_a = [&](int j) { la.one((UA > 1 && j >= EACH ? after(to_a, 1) : to_a) + own, j); };
    auto request_b = [&](int j) { lb.one((UB > 1 && j >= EACH ? after(to_b, 1) : to_b) + own, j); };
    LdsBytes *from_a = lds + wm / U * kUnitBytes, *from_b = lds + (UA + wn / U) * kUnitBytes;   // of the step that is read
    auto read = [&](int set, int j, int kk) {
        if (j < TN) fb[set][j] = rb.get(from_b, j, kk);
        else if (j < TN + TM) fa[set][j - TN] = ra.get(from_a, j - TN, kk);
    };
    auto barrier = [&] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    // all but the last n requests have arrived
#define SABER_OPS_ARRIVED(n) __builtin_amdgcn_s_waitcnt(0x0f70 | ((n) & 15) | ((n) >> 4) << 14)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int j = 0; j < LA; ++j) request_a(j);
#pragma unroll
        for (int j = 0; j < LB; ++j) request_b(j);
        next_a();
        to_a = after(to_a, UNITS);
        if (q == 0) {
            next_b();
            to_b = after(to_b, UNITS);
        }
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) request_a(j);
    SABER_OPS_ARRIVED(LA + LB + AHEAD);
    barrier();
#pragma unroll
    for (int j = 0; j < TM + TN; ++j) read(0, j, 0);
    for (int s = first; s < last; ++s) {
        each<GROUPS>([&](auto group) {
            constexpr int g = group.value;
            if constexpr (g == FREE) barrier();
            if constexpr (g == NEED) {
                SABER_OPS_ARRIVED(NEED + GROUPS - FREE - LB);
                barrier();
                from_a = after(from_a, UNITS);
                from_b = after(from_b, UNITS);
            }
            // a product, then one other instruction or two while it is at work
            each<TN>([&](auto col) {
                constexpr int j = col.value;
                mfma<T, j == 0>(fa[g / TM][g % TM], fb[g / TM][j], acc[g % TM][j]);
                if constexpr (g < FREE - 1) {
#pragma unroll
                    for (int r = j; r < READ1; r += TN) read(1, g * READ1 + r, 32);
                }
                if constexpr (g >= NEED) {
#pragma unroll
                    for (int r = j; r < READ0; r += TN) read(0, (g - NEED) * READ0 + r, 0);   // (after the last step: zeros, never used)
                }
                if constexpr (j == MOVE && g == FREE - 1) { next_b(); to_b = after(to_b, UNITS); }
                if constexpr (j == MOVE && g == FREE + LB - 1) { next_a(); to_a = after(to_a, UNITS); }
                if constexpr (j == TN - 1) {
                    if constexpr (g < FREE) request_a(AHEAD + g);
                    else if constexpr (g < FREE + LB) request_b(g - FREE);
                    else request_a(g - FREE - LB);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    }
#undef SABER_OPS_ARRIVED
    settled(acc);
    __builtin_amdgcn_s_waitcnt(0x0f70);                    // nothing is on its way to LDS any more: the epilogue may use it
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    e.template finish<BM, BN, WM, WN>(acc, state, m0, n0, wm, wn, lane, wave, split, tm, (void *)smem);
#endif
}

}  // namespace saber_ops
