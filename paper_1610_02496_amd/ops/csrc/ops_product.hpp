// Matrix products of the head on the matrix cores: D[m][n] = sum over k of A[m][k] B[n][k], with either operand stored with k
// fastest or with k slowest, and an epilogue that consumes the tile from registers.
//
// A workgroup computes a BM x BN tile in steps of 64 along k.  Operands go from memory to LDS directly (16 bytes a lane), one step
// ahead of the arithmetic, into two buffers.  LDS is written in order of the lanes; what a lane fetches is permuted instead, so that
// the reads of a fragment meet different banks:
//   k fastest: a row of 64 k is 8 pieces of 16 bytes; piece p of row r lies at p ^ (r & 7); a lane reads its 8 values of k at once.
//   k slowest: a row holds BM (BN) columns in pieces of 16 bytes; piece p of row k lies at p ^ 2 f(k), f(k) = (k & 3) | (k & 8) >> 1;
//              a lane's 8 values of k come through two transposing reads of 4 rows x 16 columns each.
// Rows and columns outside the operands are read as zeros (the bounds of the buffer descriptors), so no tile reads out of range.
//
// Operands of binary32 come as three planes of bfloat16, x = x1 + x2 + x3 exactly (8 bits of the significand each); the six
// products of planes whose weights exceed 2^-24 are added as further steps along k ("segments"), smallest first.
#pragma once
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
    int64_t k;           // extent of k; where k is fastest the stored rows go on to the next multiple of 8, with zeros in one operand
    int segments;        // 1, or 6 for planes
    int tiles_m, tiles_n;
    int splits;          // parts of the steps along k, each a workgroup of its own
};

// planes of the six segments: (0,0) last, as it is the largest
__device__ __forceinline__ int plane_a(int seg, int segments) { return segments == 1 ? 0 : (0x001012 >> (4 * seg)) & 15; }
__device__ __forceinline__ int plane_b(int seg, int segments) { return segments == 1 ? 0 : (0x010210 >> (4 * seg)) & 15; }

template <class T> struct Mfma;
template <> struct Mfma<bf16> {
    static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<f16> {
    static __device__ __forceinline__ f32x4 run(u32x4 a, u32x4 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

using LdsBytes = __attribute__((address_space(3))) char;

__device__ __forceinline__ int slow_swizzle(int k) { return ((k & 3) | ((k & 8) >> 1)) << 1; }

// 16 bytes per lane from the buffer to LDS, lane after lane from `lds` on, past the registers.  Nothing waits for it but a wait for
// the vector memory counter; in assembly, because the compiler puts such a wait in front of every later read of LDS.  It has no
// result register, so there is none that could be used too early.  s_nop: a write of m0 needs a state before its use.
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, LdsBytes *lds, uint32_t off) {
    const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)lds);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" : : "s"(at), "v"(off), "s"(rsrc) : "memory");
}
// a raw buffer: base, bytes; accesses outside read zeros
__device__ __forceinline__ u32x4 buffer_of(const char *p, uint32_t bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return u32x4{(uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((uint32_t)(a >> 32) & 0xffffu),
                 (uint32_t)__builtin_amdgcn_readfirstlane(bytes), 0x00020000u};
}

// How a wave fetches its share of one operand's tile of W columns (or rows) of m.
template <bool SLOW, int W, int WAVES>
struct Loader {
    static constexpr int kEach = W * kStep * 2 / 1024 / WAVES;   // instructions of a wave per step, 1 KB each
    static constexpr int kRows = SLOW ? 1024 / (W * 2) : 8;      // stored rows that one instruction covers
    const char *base;        // first element of the tile, plane 0
    uint32_t stride_bytes;
    int64_t plane_bytes;
    uint32_t extent;         // k fastest: bytes from the tile's first row to its last one's start; k slowest: bytes of a row
    uint32_t voff, vstep;    // of the wave's first instruction, and from one to the next
    int piece_k;             // k fastest: first k of the lane's piece

    __device__ __forceinline__ void init(const Operand &o, int64_t origin, int wave, int lane) {
        stride_bytes = (uint32_t)o.stride * 2;
        plane_bytes = o.plane * 2;
        vstep = kRows * stride_bytes;
        if constexpr (SLOW) {
            base = static_cast<const char *>(o.p) + origin * 2;
            extent = (uint32_t)((o.major - origin < W ? o.major - origin : W) * 2);
            constexpr int per_row = W / 8;                       // pieces of a row
            const int k = wave * kEach * kRows + lane / per_row;
            voff = k * stride_bytes;
            piece_k = lane % per_row;
        } else {
            base = static_cast<const char *>(o.p) + origin * (int64_t)stride_bytes;
            extent = (uint32_t)((o.major - origin < W ? o.major - origin : W) - 1) * stride_bytes;
            const int c = (lane & 7) ^ (lane >> 3);
            piece_k = c * 8;
            voff = (wave * kEach * kRows + (lane >> 3)) * stride_bytes + c * 16;
        }
    }
    __device__ __forceinline__ void fetch(LdsBytes *lds, int plane, int64_t k0, int64_t k_end, int wave, int lane) const {
        const char *p = base + plane * plane_bytes;
        uint32_t bytes, at = voff;
        if constexpr (SLOW) {
            const uint32_t left = k_end - k0 < kStep ? (uint32_t)(k_end - k0) : kStep;
            p += k0 * stride_bytes;
            bytes = (left - 1) * stride_bytes + extent;
        } else {
            p += k0 * 2;
            const uint32_t left = (uint32_t)((k_end + 7) / 8 * 8 - k0);
            bytes = extent + left * 2;
            if ((uint32_t)piece_k >= left) at = 0x80000000u;     // past the row's end: out of the descriptor's bounds
        }
        const u32x4 rsrc = buffer_of(p, bytes);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            uint32_t off = at + j * vstep;
            if constexpr (SLOW) {
                const int k = (wave * kEach + j) * kRows + lane / (W / 8);
                off += (uint32_t)(piece_k ^ slow_swizzle(k)) * 16;
            }
            load_to_lds(rsrc, lds + (wave * kEach + j) * 1024, off);
        }
    }
};

// Fragments of 16 rows of m by 32 values of k: lane l holds row l % 16, k 8 (l / 16) .. + 7.  The addresses of a lane differ between
// fragments by constants, up to the permutation: a register per distinct one, the rest are the instructions' own offsets.
template <bool SLOW, int W, int N>
struct Reader {
    uint32_t at[SLOW ? N : 2];
    __device__ __forceinline__ void init(int row, int lane) {
        if constexpr (SLOW) {
            // lane l of 16 addresses row k + l / 4 of four, columns 4 (l % 4) .. + 3; it receives column l of the four rows
            const int k = 8 * (lane >> 4) + ((lane & 15) >> 2), col = row + 4 * (lane & 3);
#pragma unroll
            for (int i = 0; i < N; ++i) at[i] = k * W * 2 + (((col + 16 * i) * 2) ^ (slow_swizzle(k) * 16));
        } else {
            at[0] = (row + (lane & 15)) * 128 + (((lane >> 4) ^ (lane & 7)) << 4);
            at[1] = at[0] ^ 64;
        }
    }
    // fragment i along m; kk: 0 or 32
    __device__ __forceinline__ u32x4 get(const LdsBytes *lds, int i, int kk) const {
        if constexpr (SLOW) {   // (k + 4 and k + 32 are permuted like k)
            using P = __attribute__((address_space(3))) s16x4 *;
            union { s16x4 h[2]; u32x4 v; } u;
            u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at[i] + kk * W * 2));
            u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds + at[i] + (kk + 4) * W * 2));
            return u.v;
        } else
            return *(const __attribute__((address_space(3))) u32x4 *)(lds + at[kk / 32] + i * 16 * 128);
    }
};

template <class T, bool A_SLOW, bool B_SLOW, int BM, int BN, int WM, int WN, class Epilogue>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product p, Epilogue e) {
#if defined(__HIP_DEVICE_COMPILE__)   // (the host pass knows neither the matrix instructions nor their types)
    constexpr int WAVES = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int kA = BM * kStep * 2, kB = BN * kStep * 2;
    __shared__ __attribute__((aligned(1024))) char smem[2 * (kA + kB)];
    LdsBytes *const lds = (LdsBytes *)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

    // Workgroups go round the eight XCDs; each XCD gets a run of neighbouring tiles, eight of n by all of m, so that what its
    // workgroups read at a time meets in its L2.
    const uint32_t plane_tiles = (uint32_t)p.tiles_m * p.tiles_n, tiles = plane_tiles * p.splits;
    uint32_t id = blockIdx.x;
    {
        const uint32_t each = tiles / 8, more = tiles % 8, x = id % 8;
        id = x * each + (x < more ? x : more) + id / 8;
    }
    const int split = (int)(id / plane_tiles);
    id -= split * plane_tiles;
    const int group = (int)(id / (p.tiles_m * 8u));
    const int width = p.tiles_n - group * 8 < 8 ? p.tiles_n - group * 8 : 8;
    const int in_group = (int)(id - group * (p.tiles_m * 8u));
    const int tm = in_group / width, tn = group * 8 + in_group % width;
    const int64_t m0 = (int64_t)tm * BM, n0 = (int64_t)tn * BN;

    Loader<A_SLOW, BM, WAVES> la;
    Loader<B_SLOW, BN, WAVES> lb;
    la.init(p.a, m0, wave, lane);
    lb.init(p.b, n0, wave, lane);
    const int wm = (wave / WN) * TM * 16, wn = (wave % WN) * TN * 16;
    Reader<A_SLOW, BM, TM> ra;
    Reader<B_SLOW, BN, TN> rb;
    ra.init(wm, lane);
    rb.init(wn, lane);

    const int per_seg = (int)((p.k + kStep - 1) / kStep), steps = per_seg * p.segments;
    const int first = (int)((int64_t)steps * split / p.splits), last = (int)((int64_t)steps * (split + 1) / p.splits);
    int seg = first / per_seg;                         // of the step that is fetched next
    int64_t k0 = (int64_t)(first - seg * per_seg) * kStep;

    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    auto fetch = [&](int buf) {
        la.fetch(lds + buf * kA, plane_a(seg, p.segments), k0, p.k, wave, lane);
        lb.fetch(lds + 2 * kA + buf * kB, plane_b(seg, p.segments), k0, p.k, wave, lane);
        k0 += kStep;
        if (k0 >= p.k) { k0 = 0; ++seg; }
    };
    auto step = [&](int buf, int s) {
        if (s + 1 < last) {
            fetch(buf ^ 1);
            __builtin_amdgcn_s_waitcnt(0x0f70 | (la.kEach + lb.kEach));   // all but what has just been asked for
        } else
            __builtin_amdgcn_s_waitcnt(0x0f70);
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        const LdsBytes *a = lds + buf * kA, *b = lds + 2 * kA + buf * kB;
#pragma unroll
        for (int kk = 0; kk < kStep; kk += 32) {
            u32x4 fb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j) fb[j] = rb.get(b, j, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const u32x4 fa = ra.get(a, i, kk);
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = Mfma<T>::run(fa, fb[j], acc[i][j]);
            }
            __builtin_amdgcn_sched_barrier(0);   // the fragments of one half at a time: both do not fit the registers
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();   // the buffer may be written again
    };
    static_assert(Loader<A_SLOW, BM, WAVES>::kEach + Loader<B_SLOW, BN, WAVES>::kEach < 16, "the wait's count");
    if (first < last) fetch(0);
    int s = first;
    for (; s + 1 < last; s += 2) {
        step(0, s);
        step(1, s + 1);
    }
    if (s < last) step(0, s);
    e.template finish<BM, BN, WM, WN>(acc, m0, n0, wm, wn, lane, wave, split, tm, (void *)smem);
#endif
}

}  // namespace saber_ops
