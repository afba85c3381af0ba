// Linear layers at the two ends of the exchange: y = act(x w^T + b) + r, and its gradients.
//
// All products are of one form, C[m, n] = sum over k of P[m, k] Q[n, k] with both operands' k contiguous:
//   forward       P = x,     Q = w      (k: features in)
//   dx            P = dz,    Q = w^T    (k: features out)
//   dw            P = dz^T,  Q = x^T    (k: tokens)
// What does not lie like that -- operands to be turned, rows off a 16-byte boundary, a k that is no multiple
// of a slab, float32 -- is first laid out anew in the workspace by pack_kernel; its cost is in
// the order of an operand's bytes, the product's in that of rows times operand.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "device_utils.h"
#include "tagc_internal.h"
#include "tagc_train.h"

namespace tagc {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kSlab = 64;        // k's of a stage in local memory: 128 bytes of a row
constexpr uint32_t kPackTile = 64;
constexpr uint32_t kPlanes = 3;       // bfloat16 numbers that a float32 is taken apart into
constexpr uint32_t kFewRows = 4;      // rows up to which the weights are streamed past the rows instead

constexpr uint64_t kMaxSide = 1u << 22;  // rows, features and direct strides are fewer

inline uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b * b; }

// ------------------------------------------------------------------ activations

__device__ inline float sigmoid(float z) { return 1.0f / (1.0f + __expf(-z)); }

// (tanh form: 0.5 (1 + tanh a) = sigmoid(2 a))
constexpr float kTanhIn = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;

__device__ inline float activate(float z, uint32_t act)
{
    switch (act) {
        case TAGC_ACT_RELU: return z > 0 ? z : (z != z ? z : 0.0f);
        case TAGC_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
        case TAGC_ACT_GELU_TANH: return z * sigmoid(kTanhIn * (z + kCubic * z * z * z));
        case TAGC_ACT_SILU: return z * sigmoid(z);
        default: return z;
    }
}

__device__ inline float slope(float z, uint32_t act)
{
    switch (act) {
        case TAGC_ACT_RELU: return z > 0 ? 1.0f : 0.0f;
        case TAGC_ACT_GELU:
            return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * __expf(-0.5f * z * z);
        case TAGC_ACT_GELU_TANH: {
            // (beyond 16 the sigmoid is 0 or 1, and z^2 would meet its 0 as an infinity)
            const float s = sigmoid(kTanhIn * (z + kCubic * z * z * z)), c = fminf(fmaxf(z, -16.0f), 16.0f);
            return s + c * s * (1.0f - s) * kTanhIn * (1.0f + 3.0f * kCubic * c * c);
        }
        case TAGC_ACT_SILU: {
            const float s = sigmoid(z);
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
}

// ------------------------------------------------------------------ elements

template <typename T>
__device__ inline float widen(T x)
{
    if constexpr (sizeof(T) == 2) return __uint_as_float(uint32_t(x) << 16);
    else return x;
}
template <typename T>
__device__ inline T narrow(float x)
{
    if constexpr (sizeof(T) == 2) return T(round_to_bf16(x));
    else return x;
}

// N neighbours at an element's address
template <typename T, int N>
__device__ inline void load_n(const T *p, float (&out)[N])
{
    typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    const vec v = *reinterpret_cast<const vec *>(p);
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = widen(T(v[j]));
}
template <typename T, int N>
__device__ inline void store_n(T *p, const float (&in)[N])
{
    typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    vec v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = narrow<T>(in[j]);
    *reinterpret_cast<vec *>(p) = v;
}

// ------------------------------------------------------------------ laying operands out

struct PackArgs {
    const void *src;      // [rows, cols], ld elements a row
    const void *pre;      // [rows, cols] or NULL: the source is dy, and what is packed dy act'(pre)
    uint64_t ld, ldp;
    uint32_t rows, cols;
    uint32_t act;
    uint16_t *straight;   // [rows, straight_ld] or NULL, zeros behind cols
    uint16_t *turned;     // [cols, turned_ld] or NULL, zeros behind rows
    uint64_t straight_ld, turned_ld, straight_plane, turned_plane;
    float *sums;          // [tiles of rows, cols] or NULL: sums over a tile's rows
};

// The bfloat16 numbers that a packed value goes to: itself rounded, or three that add up to it but for
// 2^-24 of it (an infinity or NaN stays in the first).
template <typename T>
__device__ inline void split(float x, uint16_t (&out)[sizeof(T) == 2 ? 1 : 3])
{
    out[0] = uint16_t(round_to_bf16(x));
    if constexpr (sizeof(T) == 4) {
        const bool finite = (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u;
        // (cut off, not rounded: what is finite stays finite)
        if (finite) out[0] = uint16_t(__float_as_uint(x) >> 16);
        const float y = finite ? x - __uint_as_float(uint32_t(out[0]) << 16) : 0.0f;
        out[1] = uint16_t(round_to_bf16(y));
        const float w = y - __uint_as_float(uint32_t(out[1]) << 16);
        out[2] = uint16_t(round_to_bf16(w));
    }
}

// A workgroup takes a tile of 64 by 64: reads it once, along the source's rows, and writes what is asked for.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackArgs a)
{
    constexpr int planes = sizeof(T) == 2 ? 1 : 3;
    __shared__ float tile[kPackTile][kPackTile + 1];
    const uint32_t tiles_c = (a.cols + kPackTile - 1) / kPackTile;
    const uint32_t r0 = blockIdx.x / tiles_c * kPackTile, c0 = blockIdx.x % tiles_c * kPackTile;
    const T *src = static_cast<const T *>(a.src), *pre = static_cast<const T *>(a.pre);
    const uint32_t c4 = threadIdx.x % 16 * 4;
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) {
        const uint32_t lr = threadIdx.x / 16 + 16 * i, r = r0 + lr, c = c0 + c4;
        float x[4] = {0, 0, 0, 0}, z[4] = {0, 0, 0, 0};
        if (r < a.rows) {
            if (c + 4 <= a.cols) {
                load_n<T, 4>(src + r * a.ld + c, x);
                if (pre) load_n<T, 4>(pre + r * a.ldp + c, z);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + j >= a.cols) continue;
                    x[j] = widen(src[r * a.ld + c + j]);
                    if (pre) z[j] = widen(pre[r * a.ldp + c + j]);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // (rows and columns that do not exist are 0 whatever the slope at 0 is)
            if (pre) x[j] *= slope(z[j], a.act);
            tile[lr][c4 + j] = x[j];
        }
        if (a.straight && r < a.rows) {
            typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
            u16x4 out[planes];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint16_t s[planes];
                split<T>(x[j], s);
#pragma unroll
                for (int q = 0; q < planes; ++q) out[q][j] = s[q];
            }
            if (c < a.straight_ld)
#pragma unroll
                for (int q = 0; q < planes; ++q)
                    *reinterpret_cast<u16x4 *>(a.straight + q * a.straight_plane + r * a.straight_ld + c) = out[q];
        }
    }
    __syncthreads();
    if (a.turned) {
        const uint32_t r4 = threadIdx.x % 16 * 4;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t lc = threadIdx.x / 16 + 16 * i;
            if (c0 + lc >= a.cols || r0 + r4 >= a.turned_ld) continue;
            typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
            u16x4 out[planes];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint16_t s[planes];
                split<T>(tile[r4 + j][lc], s);
#pragma unroll
                for (int q = 0; q < planes; ++q) out[q][j] = s[q];
            }
#pragma unroll
            for (int q = 0; q < planes; ++q)
                *reinterpret_cast<u16x4 *>(a.turned + q * a.turned_plane + uint64_t(c0 + lc) * a.turned_ld + r0 + r4) = out[q];
        }
    }
    if (a.sums && threadIdx.x < kPackTile && c0 + threadIdx.x < a.cols) {
        float sum = 0;
        for (uint32_t r = 0; r < kPackTile; ++r) sum += tile[r][threadIdx.x];
        a.sums[uint64_t(r0 / kPackTile) * a.cols + c0 + threadIdx.x] = sum;
    }
}

// db from the tiles' sums, added up in their order.
template <typename T>
__global__ __launch_bounds__(256) void bias_kernel(const float *sums, uint32_t tiles, uint32_t cols, T *db, uint32_t accumulate)
{
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    float s = 0;
    for (uint32_t t = 0; t < tiles; ++t) s += sums[uint64_t(t) * cols + c];
    db[c] = narrow<T>(accumulate ? s + widen(db[c]) : s);
}

// ------------------------------------------------------------------ results

struct Result {
    const void *bias;      // [n] or NULL
    const void *residual;  // [m, n] or NULL
    void *out;
    void *pre;             // or NULL
    uint64_t ldr, ldo, ldp;
    uint32_t act, accumulate;
};

// Eight neighbours of a row of the result, of which `count` exist.
template <typename T>
__device__ inline void finish(const Result &r, uint32_t m, uint32_t n, uint32_t count, float (&z)[8])
{
    const T *bias = static_cast<const T *>(r.bias), *res = static_cast<const T *>(r.residual);
    T *out = static_cast<T *>(r.out) + m * r.ldo + n, *pre = static_cast<T *>(r.pre);
    float t[8];
    if (count == 8) {
        if (bias) {
            load_n<T, 8>(bias + n, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += t[j];
        }
        if (pre) store_n<T, 8>(pre + m * r.ldp + n, z);
        if (r.act)
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = activate(z[j], r.act);
        if (res) {
            load_n<T, 8>(res + m * r.ldr + n, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += t[j];
        }
        if (r.accumulate) {
            load_n<T, 8>(out, t);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += t[j];
        }
        store_n<T, 8>(out, z);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (uint32_t(j) >= count) continue;
        float x = z[j];
        if (bias) x += widen(bias[n + j]);
        if (pre) pre[m * r.ldp + n + j] = narrow<T>(x);
        x = activate(x, r.act);
        if (res) x += widen(res[m * r.ldr + n + j]);
        if (r.accumulate) x += widen(out[j]);
        out[j] = narrow<T>(x);
    }
}

// ------------------------------------------------------------------ the product

struct Product {
    const uint16_t *p, *q;          // [m, k], [n, k] bfloat16, 16-byte aligned, k a multiple of kSlab
    uint64_t ldp, ldq;              // multiples of 8
    uint64_t plane_p, plane_q;      // from one of the three parts of a float32 to the next
    uint32_t m, n, k;
    uint32_t tiles_m, tiles_n;
    uint32_t slabs;                 // slabs of one part of the sum, in all terms
    uint32_t splits;                // parts of the sum; 1: finished here
    float *partial;                 // [splits][m][n]
    Result result;
};

// The six products of parts whose sum is a float32 product but for 2^-24 of it, smallest first.
__device__ inline uint32_t term_p(uint32_t t) { return (0x001102u >> (4 * t)) & 3; }
__device__ inline uint32_t term_q(uint32_t t) { return (0x010120u >> (4 * t)) & 3; }

// A wave computes RM by RN tiles of 16 by 16, WM by WN waves a workgroup's tile.  Q's rows go in as the matrix
// instruction's first operand, so that a lane ends up with neighbours of a row of C.
//
// Slabs of 64 k's pass through two stages of local memory, which global memory is read into directly.  A slab is four parts:
// two steps of 32 k's by two halves of P's rows, and what a part multiplies is read into registers during the part
// before, so that a wave waits for local memory only where the waves meet.  That is before a slab's last
// part: by then all have read the slab's last pieces, its stage is free for the slab after the next, and
// the next one has come.
//
// Bound by the matrix units, and by the power they draw: at 8192 by 8192 by 8192 they are busy for 72 % of the cycles,
// and the clock falls to some 1.6 GHz.  What was measured on the way (TFLOP/s there): products in the order the compiler
// found 1113, woven with the reads 1196; 32 x 32 x 16 instructions, which move their sums twice as often, 1196, 16 x 16 x 32 1236;
// four waves of 128 by 128 1163; eight waves in two groups that take turns at reading and multiplying 1041; slabs
// of 32 in a ring of four stages, whose loads take half a cache line, 1172.
template <typename T, int WM, int WN, int RM, int RN>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(Product a)
{
    constexpr uint32_t kThreads = WM * WN * 64, TM = WM * RM * 16, TN = WN * RN * 16;
    constexpr uint32_t terms = sizeof(T) == 2 ? 1 : 6;
    constexpr uint32_t kStage = (TM + TN) * kSlab * 2;
    constexpr uint32_t kLoadsP = TM * 8 / kThreads, kLoadsQ = TN * 8 / kThreads;
    constexpr uint32_t kRow = RN * 16 + 4;  // floats of a row of a wave's strip
    static_assert(WM * WN * 32 * kRow * 4 <= 2 * kStage, "the strips fit");
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave % WM, wn = wave / WM;
    uint32_t b = blockIdx.x;
    const uint32_t tiles = a.tiles_m * a.tiles_n, part = b / tiles;
    b %= tiles;
    // Workgroups go to the eight XCDs in turn.  Each XCD gets neighbouring tiles, and goes through them in groups of
    // eight rows of tiles, so that what its L2 holds is used again.
    const uint32_t xcd = b % 8, extra = tiles % 8;
    b = xcd * (tiles / 8) + min(xcd, extra) + b / 8;
    const uint32_t group = b / (8 * a.tiles_n), left = min(a.tiles_m - group * 8, 8u), in = b - group * 8 * a.tiles_n;
    const uint32_t m0 = (group * 8 + in % left) * TM, n0 = in / left * TN;

    // Where this lane's 16 bytes of each load come from.  A row's eight pieces lie in the stage in an order
    // turned by the row's number, so that lanes that read the same piece of 16 rows meet no
    // bank twice.
    uint32_t off_p[kLoadsP], off_q[kLoadsQ];
    const uint32_t sub = threadIdx.x >> 3, piece = (threadIdx.x & 7) ^ ((sub >> 1) & 7);
#pragma unroll
    for (uint32_t i = 0; i < kLoadsP; ++i)
        off_p[i] = (min(m0 + sub + i * (kThreads / 8), a.m - 1) - m0) * uint32_t(a.ldp * 2) + piece * 16;
#pragma unroll
    for (uint32_t i = 0; i < kLoadsQ; ++i)
        off_q[i] = (min(n0 + sub + i * (kThreads / 8), a.n - 1) - n0) * uint32_t(a.ldq * 2) + piece * 16;
    const char *p0 = reinterpret_cast<const char *>(a.p + uint64_t(m0) * a.ldp), *q0 = reinterpret_cast<const char *>(a.q + uint64_t(n0) * a.ldq);

    const uint32_t first = part * a.slabs, all = a.k / kSlab * terms;
    const uint32_t count = min(a.slabs, all - first);

    auto fetch = [&](uint32_t s, char *stage) {
        uint32_t ks = s, t = 0;
        if constexpr (terms > 1) {
            ks = s / terms;
            t = s % terms;
        }
        const char *p = p0 + ks * (kSlab * 2), *q = q0 + ks * (kSlab * 2);
        if constexpr (terms > 1) {
            p += term_p(t) * a.plane_p * 2;
            q += term_q(t) * a.plane_q * 2;
        }
#pragma unroll
        for (uint32_t i = 0; i < kLoadsP; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(p + off_p[i]),
                (__attribute__((address_space(3))) void *)(stage + (i * kThreads + wave * 64) * 16), 16, 0, 0);
#pragma unroll
        for (uint32_t i = 0; i < kLoadsQ; ++i)
            __builtin_amdgcn_global_load_lds(
                (const __attribute__((address_space(1))) void *)(q + off_q[i]),
                (__attribute__((address_space(3))) void *)(stage + TM * 128 + (i * kThreads + wave * 64) * 16), 16, 0, 0);
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
    const uint32_t row_p = wm * RM * 16 + (lane & 15), row_q = wn * RN * 16 + (lane & 15);
    // (rows 16 further on are turned the same way)
    auto read_q = [&](const char *stage, uint32_t step) {
        const uint32_t c = step * 4 + (lane >> 4);
#pragma unroll
        for (int j = 0; j < RN; ++j)
            fq[step][j] = *reinterpret_cast<const bf16x8 *>(stage + TM * 128 + (row_q + 16 * j) * 128 + ((c ^ ((row_q >> 1) & 7)) << 4));
    };
    auto read_p = [&](const char *stage, uint32_t step, int half) {
        const uint32_t c = step * 4 + (lane >> 4);
#pragma unroll
        for (int i = 0; i < H; ++i)
            fp[half][i] = *reinterpret_cast<const bf16x8 *>(stage + (row_p + 16 * (half * H + i)) * 128 + ((c ^ ((row_p >> 1) & 7)) << 4));
    };
    auto multiply = [&](int step, int half) {
#pragma unroll
        for (int i = 0; i < H; ++i)
#pragma unroll
            for (int j = 0; j < RN; ++j)
                acc[half * H + i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fq[step][j], fp[half][i], acc[half * H + i][j], 0, 0, 0);
    };
    // The next pieces are read while the products of the last ones run, one read behind each of the first products.
    auto woven = [&](auto reads) {
#pragma unroll
        for (int i = 0; i < H * RN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < decltype(reads)::value) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };
    // What this wave has asked for has come, then what the others have.
    auto arrived = [&]() {
        wait_own_memory_ops();
        __syncthreads();
    };
    // One slab: its first pieces are in registers, the next slab is on its way to `next`.  (Behind the last slab the
    // last one is fetched again, and never used: a branch here would cost the registers that the loop lacks.)
    auto slab = [&](uint32_t s, char *now, char *next) {
        read_p(now, 0, 1);
        multiply(0, 0);
        woven(std::integral_constant<int, H>());
        read_q(now, 1);
        read_p(now, 1, 0);
        multiply(0, 1);
        woven(std::integral_constant<int, H + RN>());
        read_p(now, 1, 1);
        multiply(1, 0);
        woven(std::integral_constant<int, H>());
        // (from here to the next meeting a wave goes before those that have not got here)
        __builtin_amdgcn_s_setprio(0);
        arrived();
        __builtin_amdgcn_s_setprio(1);
        fetch(first + min(s + 2, count - 1), now);
        read_q(next, 0);
        read_p(next, 0, 0);
        multiply(1, 1);
#pragma unroll
        for (int i = 0; i < H * RN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < H + RN) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if (i % (H * RN / (kLoadsP + kLoadsQ)) == 0) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    };

    fetch(first, stage0);
    fetch(first + min(1u, count - 1), stage1);
    arrived();
    read_q(stage0, 0);
    read_p(stage0, 0, 0);
    for (uint32_t s = 0; s < count; s += 2) {
        slab(s, stage0, stage1);
        if (s + 1 < count) slab(s + 1, stage1, stage0);
    }
    arrived();

    // Results go through the wave's own strip of local memory, 32 rows at a time, so that a row's neighbours
    // are written together.
    float *strip = reinterpret_cast<float *>(wave * 32 * kRow * 4 + 32 * kRow * 4 <= kStage ? stage0 + wave * 32 * kRow * 4
                                                                                            : stage1 + (wave - kStage / (32 * kRow * 4)) * 32 * kRow * 4);
#pragma unroll
    for (int i = 0; i < RM; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < RN; ++j)
                *reinterpret_cast<f32x4 *>(strip + (16 * h + (lane & 15)) * kRow + 16 * j + 4 * (lane >> 4)) = acc[i + h][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        constexpr uint32_t across = RN * 2, rows = 64 / across;
#pragma unroll 1
        for (uint32_t r = 0; r < 32; r += rows) {
            const uint32_t lr = r + lane / across, ln = lane % across * 8;
            const uint32_t m = m0 + (wm * RM + i) * 16 + lr, n = n0 + wn * RN * 16 + ln;
            float z[8];
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(strip + lr * kRow + ln + h);
                z[h] = v.x;
                z[h + 1] = v.y;
                z[h + 2] = v.z;
                z[h + 3] = v.w;
            }
            if (m >= a.m || n >= a.n) continue;
            const uint32_t have = min(8u, a.n - n);
            if (a.splits == 1) {
                finish<T>(a.result, m, n, have, z);
            } else {
                float *to = a.partial + (uint64_t(part) * a.m + m) * a.n + n;
                if (have == 8) {
                    store_n<float, 8>(to, z);
                } else {
#pragma unroll
                    for (uint32_t h = 0; h < 8; ++h)
                        if (h < have) to[h] = z[h];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// The parts of a split sum, added up in their order; a sum without terms is no parts.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float *partial, uint32_t splits, uint32_t rows, uint32_t cols, Result r)
{
    const uint32_t across = (cols + 7) / 8;
    for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < uint64_t(rows) * across; i += uint64_t(gridDim.x) * 256) {
        const uint32_t m = uint32_t(i / across), n = uint32_t(i % across) * 8, have = min(8u, cols - n);
        float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        for (uint32_t s = 0; s < splits; ++s) {
            const float *from = partial + (uint64_t(s) * rows + m) * cols + n;
            if (have == 8) {
                float t[8];
                load_n<float, 8>(from, t);
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] += t[j];
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    if (j < have) z[j] += from[j];
            }
        }
        finish<T>(r, m, n, have, z);
    }
}

// ------------------------------------------------------------------ few rows

struct FewArgs {
    const void *x, *w;
    uint64_t ldx, ldw;
    uint32_t in, out;
    Result result;
};

// Up to kFewRows rows: the weights are read once, in the order they lie in, and are all there is to read.  A
// wave takes a feature out at a time and its lanes the features in, sixteen bytes each.
template <typename T, int ROWS>
__global__ __launch_bounds__(256) void few_kernel(FewArgs a)
{
    constexpr uint32_t V = 16 / sizeof(T);
    const uint32_t lane = lane_id(), n = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (n >= a.out) return;
    const T *w = static_cast<const T *>(a.w) + n * a.ldw, *x = static_cast<const T *>(a.x);
    float sum[ROWS] = {};
    uint32_t k = lane * V;
#pragma unroll 4
    for (; k + V <= a.in; k += 64 * V) {
        float wv[V];
        load_n<T, V>(w + k, wv);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float xv[V];
            load_n<T, V>(x + r * a.ldx + k, xv);
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) sum[r] += wv[j] * xv[j];
        }
    }
    for (uint32_t j = 0; j < V; ++j)
        if (k + j < a.in)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) sum[r] += widen(w[k + j]) * widen(x[r * a.ldx + k + j]);
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        sum[r] = wave_sum(sum[r]);
        if (lane == 0) {
            float z[8] = {sum[r]};
            finish<T>(a.result, r, n, 1, z);
        }
    }
}

// ------------------------------------------------------------------ host

// How a product is cut: the tile, and the parts of the sum that make up for few tiles.
struct Shape {
    bool large;
    uint32_t tiles_m, tiles_n, slabs, splits;
};

Shape shape_of(uint64_t m, uint64_t n, uint64_t k, uint32_t terms)
{
    Shape s;
    const uint64_t cus = uint64_t(device_cu_count());
    const uint64_t slabs = k / kSlab * terms;
    if (!slabs) return Shape{};
    s.large = (m + 255) / 256 * ((n + 255) / 256) >= cus;
    const uint64_t t = s.large ? 256 : 128;
    s.tiles_m = uint32_t((m + t - 1) / t);
    s.tiles_n = uint32_t((n + t - 1) / t);
    const uint64_t tiles = uint64_t(s.tiles_m) * s.tiles_n;
    // two of the smaller workgroups share a compute unit; a part has four slabs at least
    uint64_t splits = 1;
    if (!s.large && tiles < 2 * cus) {
        splits = 2 * cus / tiles;
        if (splits > slabs / 4) splits = slabs / 4;
        if (splits < 1) splits = 1;
    }
    s.slabs = uint32_t((slabs + splits - 1) / splits);
    s.splits = uint32_t((slabs + s.slabs - 1) / s.slabs);
    return s;
}

// What a call lays out in its workspace, in order; at() hands out places.
struct Places {
    char *base;
    uint64_t at = 0;
    explicit Places(void *b) : base(static_cast<char *>(b)) {}
    template <typename T>
    T *take(uint64_t n)
    {
        T *p = reinterpret_cast<T *>(base + at);
        at += up(n * sizeof(T), 256);
        return p;
    }
};

struct Operand {
    const uint16_t *p;
    uint64_t ld, plane;
};

// whether rows of k elements can be read as they lie
bool as_it_lies(uint32_t dtype, const void *p, uint64_t ld, uint64_t k)
{
    return dtype == TAGC_BF16 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && ld < kMaxSide && k % kSlab == 0;
}

uint32_t planes_of(uint32_t dtype) { return dtype == TAGC_F32 ? kPlanes : 1; }

Operand room(Places &w, uint32_t dtype, uint64_t rows, uint64_t k)
{
    const uint64_t ld = up(k, kSlab), plane = rows * ld;
    return Operand{w.take<uint16_t>(plane * planes_of(dtype)), ld, plane};
}

template <typename T>
void launch_pack(const PackArgs &a, hipStream_t s)
{
    const uint64_t tiles = up(a.rows, kPackTile) / kPackTile * (up(a.cols, kPackTile) / kPackTile);
    if (!tiles) return;
    ProfileScope prof("linear_pack", s);
    pack_kernel<T><<<uint32_t(tiles), 256, 0, s>>>(a);
}

template <typename T>
void launch_product(const Operand &p, const Operand &q, uint64_t m, uint64_t n, uint64_t k, float *partial, const Result &r, hipStream_t s)
{
    Product a;
    a.p = p.p;
    a.q = q.p;
    a.ldp = p.ld;
    a.ldq = q.ld;
    a.plane_p = p.plane;
    a.plane_q = q.plane;
    a.m = uint32_t(m);
    a.n = uint32_t(n);
    a.k = uint32_t(up(k, kSlab));
    const Shape f = shape_of(m, n, a.k, sizeof(T) == 4 ? 6 : 1);
    a.tiles_m = f.tiles_m;
    a.tiles_n = f.tiles_n;
    a.slabs = f.slabs;
    a.splits = f.splits;
    a.partial = partial;
    a.result = r;
    const uint32_t grid = f.tiles_m * f.tiles_n * f.splits;
    if (grid) {
        ProfileScope prof("linear_product", s);
        if (f.large) product_kernel<T, 2, 4, 8, 4><<<grid, 512, 0, s>>>(a);
        else product_kernel<T, 2, 2, 4, 4><<<grid, 256, 0, s>>>(a);
    }
    if (f.splits != 1) {
        ProfileScope prof("linear_join", s);
        const uint64_t groups = (m * ((n + 7) / 8) + 255) / 256;
        join_kernel<T><<<uint32_t(groups < 65536 ? groups : 65536), 256, 0, s>>>(partial, f.splits, a.m, a.n, r);
    }
}

// elements of the partial sums of a product
uint64_t partial_elems(uint64_t m, uint64_t n, uint64_t k, uint32_t dtype)
{
    const Shape f = shape_of(m, n, up(k, kSlab), dtype == TAGC_F32 ? 6 : 1);
    return f.splits > 1 ? f.splits * m * n : 0;
}

bool aligned_to(const void *p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// a matrix that must or may be there
bool good(const void *p, uint64_t ld, uint64_t cols, uint64_t bytes) { return !p || (aligned_to(p, bytes) && ld >= cols && ld < (1ull << 40)); }

int check_sizes(uint64_t rows, uint64_t in, uint64_t out, uint32_t dtype, uint32_t act)
{
    if (dtype > TAGC_BF16 || act > TAGC_ACT_SILU) return TAGC_EINVAL;
    // a tile's 256 rows span fewer than 2^32 bytes
    if (rows >= kMaxSide || in >= kMaxSide || out >= kMaxSide) return TAGC_ESIZE;
    // a launch has fewer than 2^32 threads: at most a workgroup of 256 for a tile of 64 by 64
    const uint64_t r = up(rows, 64) / 64, i = up(in, 64) / 64, o = up(out, 64) / 64;
    if (r * i >= (1ull << 24) || r * o >= (1ull << 24) || i * o >= (1ull << 24)) return TAGC_ESIZE;
    return TAGC_OK;
}

template <typename T>
int forward(const tagc_linear *l, Places &w, bool enqueue, hipStream_t s)
{
    Result r{l->bias, l->residual, l->y, l->pre, l->ldr, l->ldy, l->ldp, l->activation, 0};
    const uint64_t M = l->rows, K = l->in, N = l->out;
    if (!M || !N) return TAGC_OK;
    if (M <= kFewRows) {
        if (!enqueue) return TAGC_OK;
        const FewArgs a{l->x, l->w, l->ldx, l->ldw, uint32_t(K), uint32_t(N), r};
        const uint32_t grid = uint32_t((N + 3) / 4);
        ProfileScope prof("linear_few", s);
        switch (M) {
            case 1: few_kernel<T, 1><<<grid, 256, 0, s>>>(a); break;
            case 2: few_kernel<T, 2><<<grid, 256, 0, s>>>(a); break;
            case 3: few_kernel<T, 3><<<grid, 256, 0, s>>>(a); break;
            default: few_kernel<T, 4><<<grid, 256, 0, s>>>(a); break;
        }
        return hip_ok(hipGetLastError());
    }
    Operand p{static_cast<const uint16_t *>(l->x), l->ldx, 0}, q{static_cast<const uint16_t *>(l->w), l->ldw, 0};
    PackArgs a{};
    a.rows = uint32_t(M);
    a.cols = uint32_t(K);
    if (!as_it_lies(l->dtype, l->x, l->ldx, K)) {
        p = room(w, l->dtype, M, K);
        a.src = l->x;
        a.ld = l->ldx;
        a.straight = const_cast<uint16_t *>(p.p);
        a.straight_ld = p.ld;
        a.straight_plane = p.plane;
        if (enqueue) launch_pack<T>(a, s);
    }
    if (!as_it_lies(l->dtype, l->w, l->ldw, K)) {
        q = room(w, l->dtype, N, K);
        a.src = l->w;
        a.ld = l->ldw;
        a.rows = uint32_t(N);
        a.straight = const_cast<uint16_t *>(q.p);
        a.straight_ld = q.ld;
        a.straight_plane = q.plane;
        if (enqueue) launch_pack<T>(a, s);
    }
    float *partial = w.take<float>(partial_elems(M, N, K, l->dtype));
    if (!enqueue) return TAGC_OK;
    launch_product<T>(p, q, M, N, K, partial, r, s);
    return hip_ok(hipGetLastError());
}

template <typename T>
int backward(const tagc_linear_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows, K = l->in, N = l->out;
    // dz as it is needed: by rows for dx, turned for dw
    Operand dz{static_cast<const uint16_t *>(l->dy), l->lddy, 0}, dzt{};
    PackArgs a{};
    a.src = l->dy;
    a.ld = l->lddy;
    a.pre = l->pre;
    a.ldp = l->ldp;
    a.act = l->activation;
    a.rows = uint32_t(M);
    a.cols = uint32_t(N);
    const bool dx = l->dx && M && K, dw = l->dw && N && K, db = l->db && N;
    if (dx && (l->pre || !as_it_lies(l->dtype, l->dy, l->lddy, N))) {
        dz = room(w, l->dtype, M, N);
        a.straight = const_cast<uint16_t *>(dz.p);
        a.straight_ld = dz.ld;
        a.straight_plane = dz.plane;
    }
    if (dw) {
        dzt = room(w, l->dtype, N, M);
        a.turned = const_cast<uint16_t *>(dzt.p);
        a.turned_ld = dzt.ld;
        a.turned_plane = dzt.plane;
    }
    const uint32_t tiles = uint32_t(up(M, kPackTile) / kPackTile);
    if (db) a.sums = w.take<float>(uint64_t(tiles) * N);
    if (enqueue && (a.straight || a.turned || db)) launch_pack<T>(a, s);
    if (enqueue && db) {
        ProfileScope prof("linear_bias", s);
        bias_kernel<T><<<uint32_t((N + 255) / 256), 256, 0, s>>>(a.sums, tiles, uint32_t(N), static_cast<T *>(l->db), l->accumulate);
    }
    const uint64_t mark = w.at;
    uint64_t most = mark;
    if (dx) {
        const Operand wt = room(w, l->dtype, K, N);
        float *partial = w.take<float>(partial_elems(M, K, N, l->dtype));
        if (enqueue) {
            PackArgs b{};
            b.src = l->w;
            b.ld = l->ldw;
            b.rows = uint32_t(N);
            b.cols = uint32_t(K);
            b.turned = const_cast<uint16_t *>(wt.p);
            b.turned_ld = wt.ld;
            b.turned_plane = wt.plane;
            launch_pack<T>(b, s);
            const Result r{nullptr, nullptr, l->dx, nullptr, 0, l->lddx, 0, TAGC_ACT_NONE, 0};
            launch_product<T>(dz, wt, M, K, N, partial, r, s);
        }
        most = w.at;
    }
    if (dw) {
        w.at = mark;  // what dx needed is done with
        const Operand xt = room(w, l->dtype, K, M);
        float *partial = w.take<float>(partial_elems(N, K, M, l->dtype));
        if (enqueue) {
            PackArgs b{};
            b.src = l->x;
            b.ld = l->ldx;
            b.rows = uint32_t(M);
            b.cols = uint32_t(K);
            b.turned = const_cast<uint16_t *>(xt.p);
            b.turned_ld = xt.ld;
            b.turned_plane = xt.plane;
            launch_pack<T>(b, s);
            const Result r{nullptr, nullptr, l->dw, nullptr, 0, l->lddw, 0, TAGC_ACT_NONE, l->accumulate};
            launch_product<T>(dzt, xt, N, K, M, partial, r, s);
        }
        if (w.at > most) most = w.at;
    }
    w.at = most;
    return enqueue ? hip_ok(hipGetLastError()) : TAGC_OK;
}

int check_forward(const tagc_linear *l, bool pointers)
{
    if (!l) return TAGC_EINVAL;
    const int rc = check_sizes(l->rows, l->in, l->out, l->dtype, l->activation);
    if (rc) return rc;
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2;
    if (pointers && l->rows && l->out && (!l->y || (l->in && (!l->x || !l->w)))) return TAGC_EINVAL;
    if (!good(l->x, l->ldx, l->in, e) || !good(l->w, l->ldw, l->in, e) || !aligned_to(l->bias, e) ||
        !good(l->residual, l->ldr, l->out, e) || !good(l->y, l->ldy, l->out, e) || !good(l->pre, l->ldp, l->out, e))
        return TAGC_EINVAL;
    return TAGC_OK;
}

int check_backward(const tagc_linear_grad *l, bool pointers)
{
    if (!l || l->reserved || l->accumulate > 1) return TAGC_EINVAL;
    const int rc = check_sizes(l->rows, l->in, l->out, l->dtype, l->activation);
    if (rc) return rc;
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2;
    if (pointers) {
        const bool any = l->rows && l->out;
        if (any && (!l->dy || (l->activation != TAGC_ACT_NONE) != (l->pre != nullptr))) return TAGC_EINVAL;
        if (any && l->in && ((l->dx && !l->w) || (l->dw && !l->x))) return TAGC_EINVAL;
    }
    if (!good(l->x, l->ldx, l->in, e) || !good(l->w, l->ldw, l->in, e) || !good(l->pre, l->ldp, l->out, e) ||
        !good(l->dy, l->lddy, l->out, e) || !good(l->dx, l->lddx, l->in, e) || !good(l->dw, l->lddw, l->in, e) ||
        !aligned_to(l->db, e))
        return TAGC_EINVAL;
    return TAGC_OK;
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_linear_forward_workspace(const tagc_linear *l, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check_forward(l, true);
    if (rc) return rc;
    Places w(nullptr);
    if (l->dtype == TAGC_F32) forward<float>(l, w, false, nullptr);
    else forward<uint16_t>(l, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_linear_backward_workspace(const tagc_linear_grad *l, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check_backward(l, true);
    if (rc) return rc;
    Places w(nullptr);
    if (l->dtype == TAGC_F32) backward<float>(l, w, false, nullptr);
    else backward<uint16_t>(l, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_linear_forward(const tagc_linear *l, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_linear_forward_workspace(l, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return l->dtype == TAGC_F32 ? forward<float>(l, w, true, s) : forward<uint16_t>(l, w, true, s);
}

extern "C" int tagc_linear_backward(const tagc_linear_grad *l, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_linear_backward_workspace(l, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return l->dtype == TAGC_F32 ? backward<float>(l, w, true, s) : backward<uint16_t>(l, w, true, s);
}
