// Tiled products on the matrix units, in bfloat16 and in float32 that is taken apart into bfloat16 numbers, for kernels
// whose ends differ: what becomes of a tile's sums is the caller's.
//
// All products are of one form, C[m, n] = sum over k of P[m, k] Q[n, k].  An operand lies in memory row by row, with a row's k's next
// to each other, or k by k, with a k's rows next to each other (`turned`); local memory holds it as it lies, and the
// transposing read takes it from there.
#pragma once

#include <string.h>

#include <type_traits>

#include "device_utils.h"
#include "elements.h"
#include "tagc_internal.h"

namespace tagc {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kSlab = 64;        // k's of a stage in local memory: 128 bytes of a row
constexpr uint32_t kPackRows = 64;
constexpr uint32_t kParts = 3;        // bfloat16 numbers that a float32 is taken apart into


// rows up to which few_kernel goes; from there on tiles are faster (weights of 4096 by 11008, 17, 32, 64 rows, us: bfloat16
// 32, 35, 48, as tiles 23, 24, 26; float32 76, 95, 164, as tiles 74, 75, 80)
constexpr uint32_t kFewRows = 16;

// The three bfloat16 numbers, in the upper halves, that add up to a float32: it cut off behind 8 bits (what is finite stays finite),
// the rest rounded to 8 bits, and what is then left, which has no more than 8.  (Of an infinity the second is NaN.)
__device__ inline void split(float x, uint32_t (&out)[kParts])
{
    out[0] = __float_as_uint(x);
    const float y = x - __uint_as_float(out[0] & 0xFFFF0000u);
    out[1] = __float_as_uint(y) + 0x8000u;
    out[2] = __float_as_uint(y - __uint_as_float(out[1] & 0xFFFF0000u));
}
// ------------------------------------------------------------------ the product

struct Product {
    const void *p, *q;              // [m, k] and [n, k], or turned [k, m] and [k, n]: bfloat16, float32 taken apart, or float32 as it lies
    uint64_t ldp, ldq;              // bfloat16: multiples of 2; k a multiple of 8 where rows lie row by row
    uint32_t part_p, part_q;        // taken apart: elements from one of the three parts of a row to the next
    uint32_t m, n, k;
    uint32_t tiles_m, tiles_n;
    uint32_t slabs;                 // slabs of one part of the sum
    uint32_t splits;                // parts of the sum; 1: finished here
};

// What a product kernel does with a tile's sums is its argument's: a struct E that begins as a Product, with
//   put<RM, RN>(acc, strip, lane, m0, n0, part)   a wave's sums, rows from m0 and columns from n0 on, of a part of the sum;
//                 strip: local memory of its own, 32 rows of RN * 16 + 4 floats
//   kPartByPart   see place()
//   kCounted      whether a number on the device says how many of the m rows (of the k's, `of_k`) there are: settle() then
//                 cuts the product to them, and says whether there is anything to do for a workgroup
struct Counted : Product {
    static constexpr bool kPartByPart = false;
    const uint32_t *there;
    bool of_k;
    __device__ inline bool settle(uint32_t tile)
    {
        const uint32_t n = *there;
        if (of_k) {
            k = min(k, n);
            return true;
        }
        m = min(m, n);
        tiles_m = (m + tile - 1) / tile;
        return blockIdx.x < tiles_m * tiles_n * splits;
    }
};

// The six products of parts whose sum is a float32 product but for 2^-22 of it at most, smallest first.
__device__ inline uint32_t term_p(uint32_t t) { return (0x001102u >> (4 * t)) & 3; }
__device__ inline uint32_t term_q(uint32_t t) { return (0x010120u >> (4 * t)) & 3; }

// Which tile and which part of its sum a workgroup takes.  Workgroups go to the eight XCDs in turn.  Each XCD gets
// neighbouring tiles, and goes through them in groups of eight rows of tiles, so that what its L2 holds is used again: of each part
// of the sum (E::kPartByPart), or of all parts one behind the other, so that an XCD has most tiles of few parts.  (Float32, 1024 rows' dx of 768 from three
// pieces of 50257 columns, 48 tiles of five parts each: 158 / 132 us a piece.  Linear layers, whose parts are few: 512 by 4096 by 512 in float32 27 / 31, 512 by 11008 by 512 in
// bfloat16 23 / 20.)
struct Place {
    uint32_t m0, n0, part;
};
template <uint32_t TM, uint32_t TN, bool PART_BY_PART>
__device__ inline Place place(const Product &a)
{
    const uint32_t tiles = a.tiles_m * a.tiles_n, all = PART_BY_PART ? tiles : tiles * a.splits, b = blockIdx.x % all;
    const uint32_t xcd = b % 8, extra = all % 8, in_all = xcd * (all / 8) + min(xcd, extra) + b / 8;
    const uint32_t part = PART_BY_PART ? blockIdx.x / tiles : in_all / tiles, at = PART_BY_PART ? in_all : in_all % tiles;
    const uint32_t group = at / (8 * a.tiles_n), left = min(a.tiles_m - group * 8, 8u), in = at - group * 8 * a.tiles_n;
    return Place{(group * 8 + in % left) * TM, in / left * TN, part};
}

// The same of a part without terms.
template <int RM, int RN, typename E>
__device__ inline void put_zeros(const E &a, float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t part)
{
    const f32x4 acc[RM][RN] = {};
    a.template put<RM, RN>(acc, strip, lane, m0, n0, part);
}

// One operand of a workgroup's tile: how its slabs get into local memory, 16 bytes a lane, and from there into the matrix
// instruction's registers (lane l holds row l % 16, k's 8 (l / 16) to 8 (l / 16) + 7).  R rows, kSlab k's.  The
// loads go through a buffer descriptor that ends where the operand ends: what lies behind comes as zeros.
template <bool TURNED, uint32_t R, uint32_t THREADS>
struct Side;

constexpr uint32_t kMostBytes = 1u << 31;  // of a descriptor, and ...
constexpr uint32_t kNowhere = 3u << 30;    // ... an offset behind every one; what a tile reads has smaller offsets

// Where an operand's next slab begins, and how many elements there are from there to the operand's end.
template <typename T>
struct Walk {
    const T *p;
    uint64_t left;
    uint32_t step;  // elements from one slab to the next
    __device__ inline void advance(bool on)
    {
        p += on ? step : 0;
        left -= on ? step : 0;
    }
    __device__ inline __amdgpu_buffer_rsrc_t described() const
    {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<T *>(p), 0, left < kMostBytes / sizeof(T) ? uint32_t(left) * uint32_t(sizeof(T)) : kMostBytes, 0x00020000);
    }
};

__device__ inline void load_lds(__amdgpu_buffer_rsrc_t from, uint32_t off, char *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)to, 16, off, 0, 0, 0);
}

// Row by row: 128 bytes of k's to a row.  Its eight pieces of 16 bytes lie in an order turned by the row's
// number, so that lanes that read the same piece of 16 rows meet no bank twice.
template <uint32_t R, uint32_t THREADS>
struct Side<false, R, THREADS> {
    static constexpr uint32_t kLoads = R * 8 / THREADS;
    uint32_t off[kLoads], k, lane;
    __device__ inline Side(uint32_t, uint64_t ld)
    {
        const uint32_t sub = threadIdx.x >> 3, piece = (threadIdx.x & 7) ^ ((sub >> 1) & 7);
        lane = threadIdx.x & 63;
        k = piece * 8;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) off[i] = (sub + i * (THREADS / 8)) * uint32_t(ld * 2) + piece * 16;
    }
    // the operand from row r0 and k0 on (of a row whose k's are no multiple of eight there are zeros up to one)
    __device__ static inline Walk<uint16_t> walk(const void *base, uint32_t r0, uint32_t rows, uint32_t k0, uint32_t end, uint64_t ld)
    {
        const uint16_t *p = static_cast<const uint16_t *>(base);
        return Walk<uint16_t>{p + r0 * ld + k0, (rows - r0 - 1) * ld + ((end + 7) & ~7u) - k0, kSlab};
    }
    __device__ inline void fetch(__amdgpu_buffer_rsrc_t from, uint32_t k0, uint32_t end, char *stage, uint32_t wave) const
    {
        const bool there = k0 + k < end;  // (the next row lies behind the last k)
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) load_lds(from, there ? off[i] : kNowhere, stage + (i * THREADS + wave * 64) * 16);
    }
    // N tiles of 16 rows from `tile` on, 32 k's
    template <int N>
    __device__ inline void read(const char *stage, uint32_t tile, uint32_t step, bf16x8 (&to)[N]) const
    {
        const uint32_t row = lane & 15, c = step * 4 + (lane >> 4);
#pragma unroll
        for (int i = 0; i < N; ++i)
            to[i] = *reinterpret_cast<const bf16x8 *>(stage + (tile * 16 + row + 16 * i) * 128 + ((c ^ (row >> 1)) << 4));
    }
};

// K by k: 2 R bytes of rows to a k.  The transposing read gives each of 16 lanes one row of four k's, whose 32
// bytes each lie in four k's places; a wave reads 16 k's so.  Pairs of pieces lie in an order turned by the k's number,
// so that those 16 places share all banks evenly.
template <uint32_t R, uint32_t THREADS>
struct Side<true, R, THREADS> {
    static constexpr uint32_t kAcross = R / 8, kLoads = R * 8 / THREADS, kDown = THREADS / kAcross;
    static_assert(kAcross >= 16, "eight pairs of pieces at least");
    uint32_t off[kLoads], lane;
    __device__ static inline uint32_t turn(uint32_t k) { return (k & 3) | ((k >> 1) & 4); }
    __device__ inline Side(uint32_t r0, uint64_t ld)
    {
        lane = threadIdx.x & 63;
        const uint32_t k = threadIdx.x / kAcross;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i)
            off[i] = (k + i * kDown) * uint32_t(ld * 2) + (r0 + (threadIdx.x % kAcross ^ (2 * turn(k + i * kDown))) * 8) * 2;
    }
    // the operand from k0 on (a descriptor ends with a word: of an odd number of rows there is one more)
    __device__ static inline Walk<uint16_t> walk(const void *base, uint32_t, uint32_t rows, uint32_t k0, uint32_t end, uint64_t ld)
    {
        const uint16_t *p = static_cast<const uint16_t *>(base);
        return Walk<uint16_t>{p + k0 * ld, (end - k0 - 1) * ld + ((rows + 1) & ~1u), uint32_t(ld) * kSlab};
    }
    __device__ inline void fetch(__amdgpu_buffer_rsrc_t from, uint32_t, uint32_t, char *stage, uint32_t wave) const
    {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; ++i) load_lds(from, off[i], stage + (i * THREADS + wave * 64) * 16);
    }
    template <int N>
    __device__ inline void read(const char *stage, uint32_t tile, uint32_t step, bf16x8 (&to)[N]) const
    {
        typedef short s4 __attribute__((ext_vector_type(4)));
        const uint32_t at = step * 32 + 8 * (lane >> 4) + ((lane >> 2) & 3), s = turn(at);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            // (one sum: the compiler loses sight of which stage is read behind a few steps of a pointer, and would wait for loads)
            const uint32_t from = at * (R * 2) + (((tile + i) ^ s) << 5) + ((lane & 3) << 3);
            s4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)  // (four k's further on the turn is the same)
                half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(stage + (from + h * 4 * (R * 2))));
            to[i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// A wave computes RM by RN tiles of 16 by 16, WM by WN waves a workgroup's tile.  Q's rows go in as the matrix
// instruction's first operand, so that a lane ends up with neighbours of a row of C.
//
// Slabs of 64 k's pass through two stages of local memory, which global memory is read into directly.  A slab is four parts:
// two steps of 32 k's by two halves of P's rows, and what a part multiplies is read into registers during the part
// before, so that a wave waits for local memory only where the waves meet.  That is before a slab's last
// part: by then all have read the slab's last pieces, its stage is free for the slab after the next, and
// the next one has come.
//
// Bound by the matrix units, and by the power they draw: at 8192 by 8192 by 8192 they are busy for 71 % of the cycles,
// and the clock falls to some 1.7 GHz: 833 us, 1320 TFLOP/s.  What was measured on the way (TFLOP/s there): products in the order the
// compiler found 1113, woven with the reads 1196; 32 x 32 x 16 instructions, which move their sums twice as often, 1196, 16 x 16 x 32 1236;
// four waves of 128 by 128 1163; eight waves in two groups that take turns at reading and multiplying 1041; slabs
// of 32 in a ring of four stages, whose loads take half a cache line, 1172.
template <int WM, int WN, int RM, int RN, bool PT, bool QT, typename E>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(E a)
{
    constexpr uint32_t kThreads = WM * WN * 64, TM = WM * RM * 16, TN = WN * RN * 16;
    constexpr uint32_t kStage = (TM + TN) * kSlab * 2;
    constexpr int kLoads = int((TM + TN) * 8 / kThreads);
    constexpr uint32_t kRow = RN * 16 + 4;  // floats of a row of a wave's strip
    static_assert(WM * WN * 32 * kRow * 4 <= 2 * kStage, "the strips fit");
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave % WM, wn = wave / WM;
    if constexpr (E::kCounted)
        if (!a.settle(TM)) return;
    const Place at = place<TM, TN, E::kPartByPart>(a);
    const uint32_t m0 = at.m0, n0 = at.n0;

    const Side<PT, TM, kThreads> side_p(m0, a.ldp);
    const Side<QT, TN, kThreads> side_q(n0, a.ldq);

    float *strip = reinterpret_cast<float *>(wave * 32 * kRow * 4 + 32 * kRow * 4 <= kStage ? stage0 + wave * 32 * kRow * 4
                                                                                            : stage1 + (wave - kStage / (32 * kRow * 4)) * 32 * kRow * 4);
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab - 1) / kSlab - first);
    if constexpr (E::kCounted)
        if (first * kSlab >= a.k) return put_zeros<RM, RN>(a, strip, lane, m0 + wm * RM * 16, n0 + wn * RN * 16, at.part);

    // The next slab to fetch, found before the waves meet.  Behind the last one it is the last one again.
    struct Aim {
        __amdgpu_buffer_rsrc_t p, q;
        uint32_t k0;
    };
    uint32_t k0 = first * kSlab, to_come = count;
    Walk<uint16_t> walk_p = side_p.walk(a.p, m0, a.m, k0, a.k, a.ldp), walk_q = side_q.walk(a.q, n0, a.n, k0, a.k, a.ldq);
    auto aim = [&]() __attribute__((always_inline)) {
        const Aim at{walk_p.described(), walk_q.described(), k0};
        const bool on = to_come > 1;
        to_come -= on;
        k0 += on ? kSlab : 0;
        walk_p.advance(on);
        walk_q.advance(on);
        return at;
    };
    auto fetch = [&](const Aim &at, char *stage) __attribute__((always_inline)) {
        side_p.fetch(at.p, at.k0, a.k, stage, wave);
        side_q.fetch(at.q, at.k0, a.k, stage + TM * 128, wave);
    };

    f32x4 acc[RM][RN];
#pragma unroll
    for (int i = 0; i < RM; ++i)
#pragma unroll
        for (int j = 0; j < RN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;

    constexpr int H = RM / 2;
    bf16x8 fp[2][H], fq[2][RN];
    auto read_q = [&](const char *stage, uint32_t step) __attribute__((always_inline)) { side_q.template read<RN>(stage + TM * 128, wn * RN, step, fq[step]); };
    auto read_p = [&](const char *stage, uint32_t step, int half) __attribute__((always_inline)) { side_p.template read<H>(stage, wm * RM + half * H, step, fp[half]); };
    auto multiply = [&](int step, int half) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j)
                acc[half * H + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fq[step][j], fp[half][i], acc[half * H + i][j], 0, 0, 0);
    };
    // (a turned operand takes two reads of half the size)
    constexpr int kEachP = PT ? 2 : 1, kEachQ = QT ? 2 : 1, kReads = H * kEachP + RN * kEachQ;
    constexpr int kOnce = (kReads + H * RN - 1) / (H * RN), kBoth = (kReads + kOnce - 1) / kOnce;
    // The next pieces are read while the products of the last ones run, one read behind each of the first products.
    auto woven = [&](auto reads) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < H * RN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < decltype(reads)::value) __builtin_amdgcn_sched_group_barrier(0x100, kOnce, 0);
        }
    };
    // What this wave has asked for has come, then what the others have.
    auto arrived = [&]() __attribute__((always_inline)) {
        wait_own_memory_ops();
        __syncthreads();
    };
    // One slab: its first pieces are in registers, the next slab is on its way to `next`.  (Behind the last slab the
    // last one is fetched again, and never used: a branch here would cost the registers that the loop lacks.)
    auto slab = [&](char *now, const char *next) __attribute__((always_inline)) {
        read_p(now, 0, 1);
        multiply(0, 0);
        woven(std::integral_constant<int, (H * kEachP + kOnce - 1) / kOnce>());
        read_q(now, 1);
        read_p(now, 1, 0);
        multiply(0, 1);
        woven(std::integral_constant<int, kBoth>());
        const Aim at = aim();
        read_p(now, 1, 1);
        multiply(1, 0);
        woven(std::integral_constant<int, (H * kEachP + kOnce - 1) / kOnce>());
        // (from here to the next meeting a wave goes before those that have not got here)
        __builtin_amdgcn_s_setprio(0);
        arrived();
        __builtin_amdgcn_s_setprio(1);
        read_q(next, 0);
        read_p(next, 0, 0);
        fetch(at, now);
        multiply(1, 1);
        // (of turned operands, whose reads are more, the reads go first; woven with the loads they take the same time)
#pragma unroll
        for (int i = 0; i < H * RN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if constexpr (PT || QT || H * RN < kLoads) {
                if (i < (kReads + 1) / 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                else if (i < (kReads + 1) / 2 + kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            } else {
                if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                if (i % (H * RN / kLoads) == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
        }
    };

    fetch(aim(), stage0);
    fetch(aim(), stage1);
    arrived();
    read_q(stage0, 0);
    read_p(stage0, 0, 0);
    for (uint32_t s = 0; s < count; s += 2) {
        slab(stage0, stage1);
        if (s + 1 < count) slab(stage1, stage0);
    }
    arrived();

    a.template put<RM, RN>(acc, strip, lane, m0 + wm * RM * 16, n0 + wn * RN * 16, at.part);
}

// The product where there is no more than a tile of 128 by 128 for each compute unit, which its eight waves have to themselves: what
// they wait for is memory, so four stages keep three slabs on their way, and a slab's pieces are all read
// while the one before is multiplied.  (us, here / by two workgroups of product_kernel to a compute unit: 2048 by 2048 by 4096 35 / 47,
// 700 by 4096 by 4096 31 / 43, 1024 by 4096 by 1024 14 / 18, 4096 by 1024 by 2048 20 / 27; with two tiles for each
// compute unit, one behind the other here, 8192 by 1024 by 4096 74 / 65.)
template <bool PT, bool QT, typename E>
__global__ __launch_bounds__(512, 2) void lone_kernel(E a)
{
    constexpr int RM = 4, RN = 2, kSteps = kSlab / 32;
    constexpr uint32_t T = 128, kStage = 2 * T * kSlab * 2, kRow = RN * 16 + 4;
    constexpr int kLoads = 2 * T * 8 / 512, kReads = kSteps * (RM * (PT ? 2 : 1) + RN * (QT ? 2 : 1)), kProducts = kSteps * RM * RN;
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    __shared__ __attribute__((aligned(1024))) char stage2[kStage];
    __shared__ __attribute__((aligned(1024))) char stage3[kStage];
    static_assert(4 * 32 * kRow * 4 <= kStage, "half the strips fit");
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1, wn = wave >> 1;
    if constexpr (E::kCounted)
        if (!a.settle(T)) return;
    const Place at = place<T, T, E::kPartByPart>(a);
    const Side<PT, T, 512> side_p(at.m0, a.ldp);
    const Side<QT, T, 512> side_q(at.n0, a.ldq);
    float *strip = reinterpret_cast<float *>(wave < 4 ? stage0 : stage1) + (wave & 3) * 32 * kRow;
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab - 1) / kSlab - first);
    if constexpr (E::kCounted)
        if (first * kSlab >= a.k) return put_zeros<RM, RN>(a, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
    uint32_t k0 = first * kSlab, to_come = count;
    Walk<uint16_t> walk_p = side_p.walk(a.p, at.m0, a.m, k0, a.k, a.ldp), walk_q = side_q.walk(a.q, at.n0, a.n, k0, a.k, a.ldq);
    // (behind the last slab the last one again, which nobody uses)
    auto fetch = [&](char *stage) __attribute__((always_inline)) {
        side_p.fetch(walk_p.described(), k0, a.k, stage, wave);
        side_q.fetch(walk_q.described(), k0, a.k, stage + T * 128, wave);
        const bool on = to_come > 1;
        to_come -= on;
        k0 += on ? kSlab : 0;
        walk_p.advance(on);
        walk_q.advance(on);
    };
    f32x4 acc[RM][RN] = {};
    bf16x8 fp[2][kSteps][RM], fq[2][kSteps][RN];
    auto read = [&](const char *stage, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            side_q.template read<RN>(stage + T * 128, wn * RN, h, fq[to][h]);
            side_p.template read<RM>(stage, wm * RM, h, fp[to][h]);
        }
    };
    // All that this wave has read, and what it has asked for but for `slabs` slabs; then the same for the others.
    auto meet = [&](auto slabs) __attribute__((always_inline)) {
        static_assert(decltype(slabs)::value * kLoads < 16, "fits the count");
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | decltype(slabs)::value * kLoads);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // A slab, whose pieces are in registers: its stage, `now`, is free.
    auto slab = [&](int from, char *now, const char *next) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(0);
        meet(std::integral_constant<int, 2>());
        __builtin_amdgcn_s_setprio(1);
        read(next, from ^ 1);
        fetch(now);
#pragma unroll
        for (int h = 0; h < kSteps; ++h)
#pragma unroll
            for (int i = 0; i < RM; ++i)
#pragma unroll
                for (int j = 0; j < RN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fq[from][h][j], fp[from][h][i], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kProducts; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (2 * i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            if (i >= kProducts - kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    };
    fetch(stage0);
    fetch(stage1);
    fetch(stage2);
    fetch(stage3);
    meet(std::integral_constant<int, 3>());
    read(stage0, 0);
    // (a way round a slab inside the loop would have the compiler expect any stage to be the newest one, and wait)
    uint32_t left = count;
    for (; left >= 4; left -= 4) {
        slab(0, stage0, stage1);
        slab(1, stage1, stage2);
        slab(0, stage2, stage3);
        slab(1, stage3, stage0);
    }
    if (left > 0) slab(0, stage0, stage1);
    if (left > 1) slab(1, stage1, stage2);
    if (left > 2) slab(0, stage2, stage3);
    meet(std::integral_constant<int, 0>());
    a.template put<RM, RN>(acc, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
}

// One operand of the float32 product's tile, taken apart: slabs of 32 k's of all three parts, R rows, a load of 16
// bytes to a thread for each part.  As Side otherwise, but that rows are 64 bytes of k's and that every k that a slab
// has is there, if only as a zero.
constexpr uint32_t kSlab3 = 32;
template <bool TURNED, uint32_t R>
struct Side3 {
    static constexpr uint32_t kThreads = R * 4;  // (32 k's of R rows, in pieces of 8)
    uint32_t off[kParts], lane;
    __device__ static inline uint32_t turn(uint32_t k) { return Side<true, R, kThreads>::turn(k); }
    __device__ inline Side3(uint32_t r0, uint64_t ld, uint32_t part)
    {
        lane = threadIdx.x & 63;
        uint32_t at;
        if constexpr (TURNED) {
            const uint32_t k = threadIdx.x / (R / 8);
            at = k * uint32_t(ld * 2) + (r0 + (threadIdx.x % (R / 8) ^ (2 * turn(k))) * 8) * 2;
        } else {
            const uint32_t row = threadIdx.x >> 2;
            at = row * uint32_t(ld * 2) + ((threadIdx.x & 3) ^ ((row >> 2) & 3)) * 16;
        }
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q) off[q] = at + q * part * 2;
    }
    __device__ static inline Walk<uint16_t> walk(const void *base, uint32_t r0, uint32_t rows, uint32_t k0, uint32_t end, uint64_t ld)
    {
        const uint16_t *p = static_cast<const uint16_t *>(base);
        if constexpr (TURNED) return Walk<uint16_t>{p + k0 * ld, (end - k0) * ld, uint32_t(ld) * kSlab3};
        else return Walk<uint16_t>{p + r0 * ld + k0, (rows - r0) * ld - k0, kSlab3};
    }
    __device__ inline void fetch(__amdgpu_buffer_rsrc_t from, char *stage, uint32_t wave) const
    {
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q) load_lds(from, off[q], stage + q * R * 64 + wave * 1024);
    }
    template <int N>
    __device__ inline void read(const char *stage, uint32_t tile, bf16x8 (&to)[kParts][N]) const
    {
        if constexpr (TURNED) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            const uint32_t at = 8 * (lane >> 4) + ((lane >> 2) & 3), s = turn(at);
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint32_t from = q * R * 64 + at * (R * 2) + (((tile + i) ^ s) << 5) + ((lane & 3) << 3);
                    s4 half[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4 *)(stage + (from + h * 4 * (R * 2))));
                    to[q][i] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
                }
        } else {
            const uint32_t row = lane & 15;
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    to[q][i] = *reinterpret_cast<const bf16x8 *>(stage + q * R * 64 + ((tile + i) * 16 + row) * 64 + (((lane >> 4) ^ (row >> 2)) << 4));
        }
    }
};

template <int RM, int RN>
__device__ inline __attribute__((always_inline)) void six_products(f32x4 (&acc)[RM][RN], const bf16x8 (&p)[kParts][RM], const bf16x8 (&q)[kParts][RN])
{
#pragma unroll
    for (uint32_t t = 0; t < 6; ++t)
#pragma unroll
        for (int i = 0; i < RM; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[term_q(t)][j], p[term_p(t)][i], acc[i][j], 0, 0, 0);
}

// The product of operands taken apart: 128 by 128 to a workgroup of two by four waves, 64 by 32 to a wave.  All six products
// of parts are taken from one fetch and one read of the three: the next slab's pieces are read while this one's 48
// products run, from three stages, two of which are on their way while the third is multiplied.
//
// Bound by the matrix units and their power at large sizes (4096 by 4096 by 4096: 677 us, 203
// TFLOP/s, 1220 of bfloat16 products; the units are busy for 69 % of the cycles at 1.8 GHz).  A bfloat16
// product of six times as many k's, tile of 256 by 256, fetches and reads each part two or three times: 616 us there, but 70
// instead of 56 at 1024 by 4096 by 1024, 146 instead of 114 for both gradients at 1024 by 1024 by 4096, and 755 instead of 665 for
// those at 8192 by 1024 by 4096.
template <bool PT, bool QT, typename E>
__global__ __launch_bounds__(512, 2) void product3_kernel(E a)
{
    constexpr int RM = 4, RN = 2;
    constexpr uint32_t T = 128, kStage = 2 * T * kParts * 64, kRow = RN * 16 + 4;
    constexpr int kLoads = 2 * kParts, kReads = kParts * (RM * (PT ? 2 : 1) + RN * (QT ? 2 : 1));
    static_assert(8 * 32 * kRow * 4 <= kStage, "the strips fit");
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    __shared__ __attribute__((aligned(1024))) char stage2[kStage];
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1, wn = wave >> 1;
    if constexpr (E::kCounted)
        if (!a.settle(T)) return;
    const Place at = place<T, T, E::kPartByPart>(a);
    const Side3<PT, T> side_p(at.m0, a.ldp, a.part_p);
    const Side3<QT, T> side_q(at.n0, a.ldq, a.part_q);
    float *strip = reinterpret_cast<float *>(stage0) + wave * 32 * kRow;
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab3 - 1) / kSlab3 - first);
    if constexpr (E::kCounted)
        if (first * kSlab3 >= a.k) return put_zeros<RM, RN>(a, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
    uint32_t to_come = count;
    Walk<uint16_t> walk_p = side_p.walk(a.p, at.m0, a.m, first * kSlab3, a.k, a.ldp), walk_q = side_q.walk(a.q, at.n0, a.n, first * kSlab3, a.k, a.ldq);
    // (behind the last slab the last one again, which nobody uses)
    auto fetch = [&](char *stage) __attribute__((always_inline)) {
        side_p.fetch(walk_p.described(), stage, wave);
        side_q.fetch(walk_q.described(), stage + T * kParts * 64, wave);
        const bool on = to_come > 1;
        to_come -= on;
        walk_p.advance(on);
        walk_q.advance(on);
    };
    f32x4 acc[RM][RN] = {};
    bf16x8 fp[2][kParts][RM], fq[2][kParts][RN];
    auto read = [&](const char *stage, int to) __attribute__((always_inline)) {
        side_q.template read<RN>(stage + T * kParts * 64, wn * RN, fq[to]);
        side_p.template read<RM>(stage, wm * RM, fp[to]);
    };
    // All that this wave has read, and what it has asked for but for `slabs` slabs; then the same for the others.
    auto meet = [&](auto slabs) __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070 | decltype(slabs)::value * kLoads);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // A slab, whose pieces are in registers: its stage, `now`, is free.
    auto slab = [&](int from, char *now, const char *next) __attribute__((always_inline)) {
        __builtin_amdgcn_s_setprio(0);
        meet(std::integral_constant<int, 1>());
        __builtin_amdgcn_s_setprio(1);
        read(next, from ^ 1);
        fetch(now);
        six_products(acc, fp[from], fq[from]);
#pragma unroll
        for (int i = 0; i < 48; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            else if (i < kReads + kLoads) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    };
    fetch(stage0);
    fetch(stage1);
    fetch(stage2);
    meet(std::integral_constant<int, 2>());
    read(stage0, 0);
    // (a way round a slab inside the loop would have the compiler expect any stage to be the newest one, and wait)
    uint32_t left = count;
    for (; left >= 6; left -= 6) {
        slab(0, stage0, stage1);
        slab(1, stage1, stage2);
        slab(0, stage2, stage0);
        slab(1, stage0, stage1);
        slab(0, stage1, stage2);
        slab(1, stage2, stage0);
    }
    if (left > 0) slab(0, stage0, stage1);
    if (left > 1) slab(1, stage1, stage2);
    if (left > 2) slab(0, stage2, stage0);
    if (left > 3) slab(1, stage0, stage1);
    if (left > 4) slab(0, stage1, stage2);
    meet(std::integral_constant<int, 0>());
    a.template put<RM, RN>(acc, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
}

// A float32 operand as it lies, row by row: a thread's eight k's of a row are taken apart on the way into local memory, to where
// Side3 has them.
template <uint32_t R>
struct Raw3 {
    uint32_t off, k;
    __device__ inline explicit Raw3(uint64_t ld)
    {
        const uint32_t row = threadIdx.x >> 2;
        k = ((threadIdx.x & 3) ^ ((row >> 2) & 3)) * 8;
        off = row * uint32_t(ld * 4) + k * 4;
    }
    __device__ static inline Walk<float> walk(const void *base, uint32_t r0, uint32_t rows, uint32_t k0, uint32_t end, uint64_t ld)
    {
        return Walk<float>{static_cast<const float *>(base) + r0 * ld + k0, (rows - r0 - 1) * ld + end - k0, kSlab3};
    }
    struct Piece {
        u32x4 x[2];
    };
    __device__ inline Piece load(__amdgpu_buffer_rsrc_t from) const
    {
        Piece r;
#pragma unroll
        for (int h = 0; h < 2; ++h) r.x[h] = __builtin_amdgcn_raw_buffer_load_b128(from, off + h * 16, 0, 0);
        return r;
    }
    // of a slab with `have` k's (behind a row's last one lies the next row)
    __device__ inline void cut(Piece &r, uint32_t have) const
    {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (k + j >= have) r.x[j / 4][j % 4] = 0;
    }
    __device__ inline void put(const Piece &r, char *stage) const
    {
        u32x4 to[kParts];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            uint32_t s[2][kParts];
#pragma unroll
            for (uint32_t h = 0; h < 2; ++h) split(__uint_as_float(r.x[j / 2][j % 2 * 2 + h]), s[h]);
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q) to[q][j] = __builtin_amdgcn_perm(s[1][q], s[0][q], 0x07060302);
        }
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q) *reinterpret_cast<u32x4 *>(stage + (q * R * 64 + threadIdx.x * 16)) = to[q];
    }
};

// The same product of operands as they lie: while a slab's 48 products run, the next one's pieces are read from one stage, the one
// after that is taken apart into the other, and two more are on their way to registers.
//
// It saves the launch and the bytes of laying out, but takes an operand apart once for each tile that reads it, and
// the vector unit's instructions cost the matrix units a sixth of their rate: taken where operands are many bytes for their
// products (raw_pays).  (us, as they lie / laid out: 333 by 1001 by 777 19 / 26, 1024 by 1024 by 1024 25 / 32, 512 by 4096 by 4096
// 100 / 124, 8192 by 1024 by 4096 356 / 382, 2048 by 2048 by 4096 178 / 185; 8192 by 4096 by 1024 388 / 371, 4096 cubed 717 / 677.  Of
// turned operands, whose laying out dx and dw share, both gradients at 8192 by 1024 by 4096 took 722 / 666.)
template <typename E>
__global__ __launch_bounds__(512, 2) void raw3_kernel(E a)
{
    constexpr int RM = 4, RN = 2;
    constexpr uint32_t T = 128, kStage = 2 * T * kParts * 64, kRow = RN * 16 + 4;
    constexpr int kReads = kParts * (RM + RN);
    static_assert(8 * 32 * kRow * 4 <= kStage, "the strips fit");
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1, wn = wave >> 1;
    if constexpr (E::kCounted)
        if (!a.settle(T)) return;
    const Place at = place<T, T, E::kPartByPart>(a);
    const Raw3<T> side_p(a.ldp), side_q(a.ldq);
    const Side3<false, T> parts(0, 0, 0);
    float *strip = reinterpret_cast<float *>(stage0) + wave * 32 * kRow;
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab3 - 1) / kSlab3 - first), last = first + count - 1;
    if constexpr (E::kCounted)
        if (first * kSlab3 >= a.k) return put_zeros<RM, RN>(a, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
    // The last slab, which alone may have fewer k's, goes first; `load` asks for the others (behind the last of them for that one
    // again, which nobody uses).
    uint32_t to_come = count;
    Walk<float> walk_p = side_p.walk(a.p, at.m0, a.m, first * kSlab3, a.k, a.ldp), walk_q = side_q.walk(a.q, at.n0, a.n, first * kSlab3, a.k, a.ldq);
    Raw3<T>::Piece raw_p[2], raw_q[2];
    auto load = [&](int to) __attribute__((always_inline)) {
        raw_p[to] = side_p.load(walk_p.described());
        raw_q[to] = side_q.load(walk_q.described());
        const bool on = to_come > 2;
        to_come -= on;
        walk_p.advance(on);
        walk_q.advance(on);
    };
    auto put = [&](int from, char *stage) __attribute__((always_inline)) {
        side_p.put(raw_p[from], stage);
        side_q.put(raw_q[from], stage + T * kParts * 64);
    };
    f32x4 acc[RM][RN] = {};
    bf16x8 fp[2][kParts][RM], fq[2][kParts][RN];
    auto read = [&](const char *stage, int to) __attribute__((always_inline)) {
        parts.template read<RN>(stage + T * kParts * 64, wn * RN, fq[to]);
        parts.template read<RM>(stage, wm * RM, fp[to]);
    };
    // What this wave has read has come, and what it has written is there; then the same for the others.
    auto meet = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    // A slab, whose pieces are in registers: its stage, `now`, is free.
    auto slab = [&](int from, char *now, const char *next) __attribute__((always_inline)) {
        meet();
        read(next, from ^ 1);
        put(from, now);
        load(from);
        six_products(acc, fp[from], fq[from]);
#pragma unroll
        for (int i = 0; i < 48; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (i < 42) __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);
            if ((i >= 20 && i < 23) || (i >= 42 && i < 45)) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            if (i >= 44) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    };
    const Walk<float> end_p = side_p.walk(a.p, at.m0, a.m, last * kSlab3, a.k, a.ldp), end_q = side_q.walk(a.q, at.n0, a.n, last * kSlab3, a.k, a.ldq);
    raw_p[0] = side_p.load(end_p.described());
    raw_q[0] = side_q.load(end_q.described());
    load(1);
    side_p.cut(raw_p[0], a.k - last * kSlab3);
    side_q.cut(raw_q[0], a.k - last * kSlab3);
    put(0, stage0);
    load(0);
    put(1, stage1);
    load(1);
    meet();
    read(stage0, 0);
    uint32_t left = count;
    for (; left >= 2; left -= 2) {
        slab(0, stage0, stage1);
        slab(1, stage1, stage0);
    }
    if (left) slab(0, stage0, stage1);
    meet();
    a.template put<RM, RN>(acc, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
}

// ------------------------------------------------------------------ few rows

struct FewArgs {
    const void *x, *w;
    uint64_t ldx, ldw;
    uint32_t rows, in, out;
};

// Sixteen k's of a row from `k` on as they lie in memory, zeros from `end` on.
template <typename T>
struct Piece {
    T x[16];
    __device__ inline void load(const T *row, uint32_t k, uint32_t end)
    {
        if (k + 16 <= end) {
            typedef T vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
#pragma unroll
            for (uint32_t i = 0; i < sizeof(T); ++i) {
                const vec v = *reinterpret_cast<const vec *>(row + k + i * (16 / sizeof(T)));
#pragma unroll
                for (uint32_t j = 0; j < 16 / sizeof(T); ++j) x[i * (16 / sizeof(T)) + j] = v[j];
            }
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 16; ++j) x[j] = k + j < end ? row[k + j] : T(0);
        }
    }
    // the first or the second eight as the matrix instruction takes them
    __device__ inline void half(int h, bf16x8 (&to)[sizeof(T) == 2 ? 1 : 3]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if constexpr (sizeof(T) == 2) {
                to[0][e] = __builtin_bit_cast(__bf16, x[8 * h + e]);
            } else {
                uint32_t s[kParts];
                split(x[8 * h + e], s);
#pragma unroll
                for (uint32_t q = 0; q < kParts; ++q) to[q][e] = __builtin_bit_cast(__bf16, uint16_t(s[q] >> 16));
            }
        }
    }
};

// Up to kFewRows rows, an argument that begins as a FewArgs and has put(row, first of eight features out, how many of them there are, sums): the
// weights are read once, straight into registers, in pieces of 64 k's of 16 features out; rows of x,
// which all workgroups read, come from the caches.  kFewWaves waves share the k's of 16 features out and add up their
// sums in local memory.  The matrix instruction's k's may be in any order that both operands share: a lane takes 16
// neighbours, so that four lanes read a whole cache line.  float32 is taken apart in registers.
//
// Bound by the weights' bytes (one row of bfloat16 through 4096 by 11008, not in any cache: 17.5 us, 5.2 TB/s; 16 features
// out to a workgroup, 32 take half as long again; four or sixteen waves a sixth and a twelfth more; eight pieces on their way instead
// of four a tenth), at 16 rows also by x, which is as many bytes to a workgroup then (26.0).
constexpr int kFewWaves = 8;
template <typename T, typename E>
__global__ __launch_bounds__(kFewWaves * 64, 2) void few_kernel(E a)
{
    constexpr int planes = sizeof(T) == 2 ? 1 : 3, D = sizeof(T) == 2 ? 4 : 2;  // pieces on their way
    __shared__ f32x4 sums[kFewWaves][64];
    const uint32_t lane = lane_id(), wave = threadIdx.x >> 6, at = lane & 15, k0 = (lane >> 4) * 16;
    const uint32_t n0 = blockIdx.x * 16;
    const T *w = static_cast<const T *>(a.w) + min(n0 + at, a.out - 1) * a.ldw;
    const T *x = static_cast<const T *>(a.x) + min(at, a.rows - 1) * a.ldx;
    f32x4 acc = {};
    for (uint32_t k = wave * 64; k < a.in; k += kFewWaves * 64 * D) {
        Piece<T> pw[D], px[D];
#pragma unroll
        for (int d = 0; d < D; ++d) {
            const uint32_t from = k + d * kFewWaves * 64 + k0;
            pw[d].load(w, from, a.in);
            px[d].load(x, from, a.in);
        }
#pragma unroll
        for (int d = 0; d < D; ++d)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                bf16x8 fw[planes], fx[planes];
                pw[d].half(h, fw);
                px[d].half(h, fx);
                if constexpr (planes == 1) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[0], fx[0], acc, 0, 0, 0);
                } else {
#pragma unroll
                    for (uint32_t t = 0; t < 6; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[term_q(t)], fx[term_p(t)], acc, 0, 0, 0);
                }
            }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    // Eight neighbours of a row, features 8 h to 8 h + 7, are in two lanes' words.
    const uint32_t m = threadIdx.x / 2, h = threadIdx.x % 2, n = n0 + 8 * h;
    if (m >= a.rows || n >= a.out) return;
    float z[8] = {};
#pragma unroll
    for (int s = 0; s < kFewWaves; ++s)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const f32x4 v = sums[s][(2 * h + q) * 16 + m];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * q + e] += v[e];
        }
    a.put(m, n, min(8u, a.out - n), z);
}

// ------------------------------------------------------------------ host

// How a product is cut (into at most `most` parts of the sum: 16, 1, or 64 of sums as long as a vocabulary): tiles of `rows` by 256 (256 rows) or 128, and the parts of the sum that make up for few tiles.
struct Shape {
    uint32_t rows, tiles_m, tiles_n, slabs, splits;
    bool lone;  // bfloat16 tiles of 128 that each have a compute unit to themselves: lone_kernel
};

// By what the candidates would take, in us, from measurements at sizes from 333 by 1001 by 832 to 8192 by 8192 by 8192 (within 15 %
// of them): a slab of 256 by 256 takes a compute unit to itself for 1.68; two of 128 by 128 share one for 1.01, one
// that is left over takes 0.70, one alone by lone_kernel 0.50, a slab of 32 float32 1.1; parts of a sum cost a launch, and their bytes written and read.  (us, 256 by 256 / 128 by 128
// in one, two, four parts: 4096 cubed 107 / 124; 8192 by 2560 by 1024 64 / 53; 2048 by 2048 by 4096 81 / 35, 49; 1024 by 4096 by
// 1024 31 / 14, 27; 1024 by 1024 by 4096 - / -, -, 23; 333 by 1001 by 832 - / 10, -, -.)
inline Shape shape_of(uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, bool turned_p, uint64_t most = 16)
{
    Shape s{};
    const uint64_t cus = uint64_t(device_cu_count()), slab = dtype == TAGC_F32 ? kSlab3 : kSlab, slabs = up(k, slab) / slab;
    if (!slabs) return s;
    uint64_t splits = 1;
    if (dtype == TAGC_BF16 && !turned_p && m <= 64) {
        // thin tiles: the weights' bytes count, and many workgroups to ask for them
        s.rows = m <= 32 ? 32 : 64;
        s.tiles_m = 1;
        s.tiles_n = uint32_t((n + 127) / 128);
        splits = 2 * cus / s.tiles_n;
        if (splits > slabs / 4) splits = slabs / 4;
        if (most == 1) splits = 1;
        if (splits < 1) splits = 1;
    } else {
        double best = 0;
        for (const uint32_t t : {256u, 128u}) {
            if (t == 256 && dtype == TAGC_F32) continue;
            const uint64_t tm = (m + t - 1) / t, tn = (n + t - 1) / t, tiles = tm * tn;
            for (uint64_t parts = 1; parts <= most && parts <= slabs; ++parts) {
                const uint64_t each = (slabs + parts - 1) / parts, groups = tiles * parts;
                double rounds;
                if (dtype == TAGC_F32) {
                    rounds = 1.1 * double((groups + cus - 1) / cus);
                } else if (t == 256) {
                    rounds = 1.68 * double((groups + cus - 1) / cus);
                } else {
                    const uint64_t rest = groups % (2 * cus);
                    rounds = groups <= cus ? 0.50 : 1.01 * double(groups / (2 * cus)) + (!rest ? 0.0 : rest <= cus ? 0.70 : 1.01);
                }
                const double us = rounds * double(each) + (parts > 1 ? 4.5 + double(parts * m * n * 8) / 4e6 : 0.0);
                if (s.rows && us >= best) continue;
                best = us;
                s.rows = t;
                s.tiles_m = uint32_t(tm);
                s.tiles_n = uint32_t(tn);
                splits = parts;
            }
        }
    }
    s.slabs = uint32_t((slabs + splits - 1) / splits);
    s.splits = uint32_t((slabs + s.slabs - 1) / s.slabs);
    s.lone = dtype == TAGC_BF16 && s.rows == 128 && uint64_t(s.tiles_m) * s.tiles_n * s.splits <= cus;
    return s;
}

struct Operand {
    const void *p;
    uint64_t ld;
    uint32_t part;  // of float32 the three parts of a row, one behind the other, are so far apart
};

// whether a matrix with `cols` elements to a row can be read as it lies: in words, and, where a row is k's, in pieces of 16 bytes
// that do not straddle the last of them
inline bool as_it_lies(uint32_t dtype, const void *p, uint64_t ld, uint64_t cols, bool turned)
{
    return dtype == TAGC_BF16 && (reinterpret_cast<uintptr_t>(p) & 3) == 0 && ld % 2 == 0 && ld < kMaxSide && cols % (turned ? 2 : 8) == 0;
}

// Whether float32 rows of k's are read as they lie (raw3_kernel): laying out (m + n) k elements takes 2.1 us a million, and m n k products
// of what lies as it did 1.6 us a thousand million more.
inline bool raw_pays(uint64_t m, uint64_t n) { return m * n < 1300 * (m + n); }

// Room for an operand laid out anew: rows of whole slabs.
inline Operand room(Places &w, uint32_t dtype, uint64_t rows, uint64_t cols)
{
    const uint64_t part = up(cols, 64), ld = part * (dtype == TAGC_F32 ? kParts : 1);
    return Operand{w.take<uint16_t>(rows * ld), ld, uint32_t(part)};
}

// The cut of a product, and its operands, as the kernels take them.
inline void aim(Product &a, const Operand &p, const Operand &q, uint64_t m, uint64_t n, uint64_t k, const Shape &f)
{
    a.p = p.p;
    a.q = q.p;
    a.ldp = p.ld;
    a.ldq = q.ld;
    a.part_p = p.part;
    a.part_q = q.part;
    a.m = uint32_t(m);
    a.n = uint32_t(n);
    a.k = uint32_t(k);
    a.tiles_m = f.tiles_m;
    a.tiles_n = f.tiles_n;
    a.slabs = f.slabs;
    a.splits = f.splits;
}

// The launch of a product: its kernel by the shape, float32 operands as they lie (RAW) or taken apart.
template <typename T, bool PT, bool QT, typename E>
void launch(const E &a, const Shape &f, hipStream_t s)
{
    const uint32_t grid = f.tiles_m * f.tiles_n * f.splits;
    if (!grid) return;
    if constexpr (sizeof(T) == 4) {
        if constexpr (!PT && !QT) {
            if (!a.part_p) raw3_kernel<<<grid, 512, 0, s>>>(a);
            else product3_kernel<PT, QT><<<grid, 512, 0, s>>>(a);
        } else {
            product3_kernel<PT, QT><<<grid, 512, 0, s>>>(a);
        }
    } else {
        if (f.rows == 256) product_kernel<2, 4, 8, 4, PT, QT><<<grid, 512, 0, s>>>(a);
        else if (f.lone) lone_kernel<PT, QT><<<grid, 512, 0, s>>>(a);
        else if (f.rows == 128) product_kernel<2, 4, 4, 2, PT, QT><<<grid, 512, 0, s>>>(a);
        else if constexpr (!PT) {
            if (f.rows == 64) product_kernel<1, 4, 4, 2, PT, QT><<<grid, 256, 0, s>>>(a);
            else product_kernel<1, 4, 2, 2, PT, QT><<<grid, 256, 0, s>>>(a);
        }
    }
}

}  // namespace

}  // namespace tagc
