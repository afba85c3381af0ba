// Linear layers at the two ends of the exchange: y = act(x w^T + b) + r, and its gradients.
//
// All products are of one form, C[m, n] = sum over k of P[m, k] Q[n, k]:
//   forward       P = x,               Q = w                   (k: features in)
//   dx            P = dz,              Q = w, k by k           (k: features out)
//   dw            P = dz, k by k       Q = x, k by k           (k: tokens)
// An operand lies in memory row by row, with a row's k's next to each other, or k by k, with a k's rows next
// to each other (`turned`); local memory holds it as it lies, and the transposing read takes it from there.
// What cannot be read as it lies -- bfloat16 rows that are no whole pieces of 16 bytes, float32 that many tiles
// read, dz where there is an activation -- is first laid out anew in the workspace by pack_kernel; its cost is in the order of an
// operand's bytes, the product's in that of rows times operand.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "device_utils.h"
#include "tagc_internal.h"
#include "tagc_test.h"
#include "tagc_train.h"

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

constexpr uint64_t kMaxSide = 1u << 22;  // rows, features (in float32 a quarter) and strides as they lie are fewer

inline uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b * b; }

// ------------------------------------------------------------------ activations

// (the hardware's exp2 and reciprocal: within 2 ulp each)
__device__ inline float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z)); }

// (tanh form: 0.5 (1 + tanh a) = sigmoid(2 a))
constexpr float kTanhIn = 1.5957691216057308f;  // 2 sqrt(2 / pi)
constexpr float kCubic = 0.044715f;

// erfc(-z / sqrt(2)) / 2 and exp(-z^2 / 2).  For bfloat16, left of 0, the bell times t P(t), t = 1 / (1 + 0.4149 |z|): six coefficients
// by a linear program that keeps the error under both 1.2e-7 and 1.9e-4 of the result down to -13.2, where the bell leaves float32's
// normal numbers.  Rounding a result to bfloat16 leaves ten times as much of it.  (In float32 as it stands here: 2.1e-7, 1.4e-4.)
template <typename T>
__device__ inline float normal_below(float z, float &bell)
{
    bell = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    if constexpr (sizeof(T) == 4) return 0.5f * erfcf(z * -0.70710678118654752f);  // (1 + erf would lose the left tail's bits)
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.4149f * fabsf(z));
    const float tail = bell * t * (0.16451882f + t * (0.17968506f + t * (0.061874557f + t * (0.27448904f + t * (-0.23748873f + t * 0.05692133f)))));
    return z < 0 ? tail : 1.0f - tail;
}

template <typename T, int N>
__device__ inline void activate(float (&z)[N], uint32_t act)
{
    float bell;
    switch (act) {
        case TAGC_ACT_RELU:
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] = z[j] > 0 ? z[j] : (z[j] != z[j] ? z[j] : 0.0f);
            break;
        case TAGC_ACT_GELU:
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] *= normal_below<T>(z[j], bell);
            break;
        case TAGC_ACT_GELU_TANH:
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] *= sigmoid(kTanhIn * (z[j] + kCubic * z[j] * z[j] * z[j]));
            break;
        case TAGC_ACT_SILU:
#pragma unroll
            for (int j = 0; j < N; ++j) z[j] *= sigmoid(z[j]);
            break;
        default: break;
    }
}

// x times the activation's slope at z
template <typename T, int N>
__device__ inline void times_slope(float (&x)[N], const float (&z)[N], uint32_t act)
{
    float bell;
    switch (act) {
        case TAGC_ACT_RELU:
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] *= z[j] > 0 ? 1.0f : (z[j] != z[j] ? z[j] : 0.0f);
            break;
        case TAGC_ACT_GELU:
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float below = normal_below<T>(z[j], bell);
                x[j] *= below + z[j] * 0.39894228040143268f * bell;
            }
            break;
        case TAGC_ACT_GELU_TANH:
#pragma unroll
            for (int j = 0; j < N; ++j) {
                // (beyond 16 the sigmoid is 0 or 1, and z^2 would meet its 0 as an infinity)
                const float s = sigmoid(kTanhIn * (z[j] + kCubic * z[j] * z[j] * z[j])), c = fminf(fmaxf(z[j], -16.0f), 16.0f);
                x[j] *= s + c * s * (1.0f - s) * kTanhIn * (1.0f + 3.0f * kCubic * c * c);
            }
            break;
        case TAGC_ACT_SILU:
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float s = sigmoid(z[j]);
                x[j] *= s * (1.0f + z[j] * (1.0f - s));
            }
            break;
        default: break;
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
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(T, static_cast<__bf16>(x));  // to nearest, ties to even
    else return x;
}

// N neighbours at an element's address
template <typename T, int N>
struct Lane {
    typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    vec v;
    __device__ inline void load(const T *p) { v = *reinterpret_cast<const vec *>(p); }
    __device__ inline float operator[](int j) const { return widen(T(v[j])); }
};
template <typename T, int N>
__device__ inline void load_n(const T *p, float (&out)[N])
{
    Lane<T, N> in;
    in.load(p);
#pragma unroll
    for (int j = 0; j < N; ++j) out[j] = in[j];
}
template <typename T, int N>
__device__ inline void store_n(T *p, const float (&in)[N])
{
    typename Lane<T, N>::vec v;
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = narrow<T>(in[j]);
    *reinterpret_cast<typename Lane<T, N>::vec *>(p) = v;
}

// ------------------------------------------------------------------ laying operands out

struct PackArgs {
    const void *src;      // [rows, cols], ld elements a row
    const void *pre;      // [rows, cols] or NULL: the source is dy, and what is packed dy act'(pre)
    uint64_t ld, ldp;
    uint32_t rows, cols;
    uint32_t act;
    uint16_t *to;         // [rows, to_ld] or NULL, zeros behind cols
    uint64_t to_ld;
    uint32_t to_part;     // float32: elements from one of the three parts of a row to the next
    float *sums;          // [tiles of rows, cols] or NULL: sums over a tile's rows
};

// What a call lays out, in one launch.
struct PackJobs {
    PackArgs job[3];
    uint32_t first[3];    // workgroup of each (one that there is not begins behind the last)
};

// The three bfloat16 numbers, in the upper halves, that add up to a float32: it cut off behind 8 bits (what is finite stays finite),
// the rest rounded to 8 bits, and what is then left, which has no more than 8.  (Of an infinity the second is NaN.)
__device__ inline void split(float x, uint32_t (&out)[kParts])
{
    out[0] = __float_as_uint(x);
    const float y = x - __uint_as_float(out[0] & 0xFFFF0000u);
    out[1] = __float_as_uint(y) + 0x8000u;
    out[2] = __float_as_uint(y - __uint_as_float(out[1] & 0xFFFF0000u));
}

// A workgroup takes a tile of kPackRows by 64, a thread four neighbours of each sixteenth row.
template <typename T>
__global__ __launch_bounds__(256) void pack_kernel(PackJobs jobs)
{
    const uint32_t which = blockIdx.x >= jobs.first[2] ? 2 : blockIdx.x >= jobs.first[1] ? 1 : 0;
    const PackArgs a = which == 0 ? jobs.job[0] : which == 1 ? jobs.job[1] : jobs.job[2];
    const uint32_t block = blockIdx.x - jobs.first[which];
    constexpr int planes = sizeof(T) == 2 ? 1 : 3;
    typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));
    __shared__ float sums[16][64];
    const uint32_t tiles_c = (a.cols + 63) / 64;
    const uint32_t tile = block / tiles_c, r0 = tile * kPackRows, c = block % tiles_c * 64 + threadIdx.x % 16 * 4;
    const T *src = static_cast<const T *>(a.src), *pre = static_cast<const T *>(a.pre);
    float x[kPackRows / 16][4] = {}, sum[4] = {};
#pragma unroll
    for (uint32_t i = 0; i < kPackRows / 16; ++i) {
        const uint32_t r = r0 + threadIdx.x / 16 + 16 * i;
        float z[4] = {};
        if (r < a.rows) {
            if (c + 4 <= a.cols) {
                load_n<T, 4>(src + r * a.ld + c, x[i]);
                if (pre) load_n<T, 4>(pre + r * a.ldp + c, z);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (c + j >= a.cols) continue;
                    x[i][j] = widen(src[r * a.ld + c + j]);
                    if (pre) z[j] = widen(pre[r * a.ldp + c + j]);
                }
            }
        }
        // (rows and columns that do not exist are 0 whatever the slope at 0 is)
        if (pre) times_slope<T>(x[i], z, a.act);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += x[i][j];
    }
    if (a.to)
#pragma unroll
        for (uint32_t i = 0; i < kPackRows / 16; ++i) {
            const uint32_t r = r0 + threadIdx.x / 16 + 16 * i;
            if (r >= a.rows) break;
            u16x4 out[planes];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (planes == 1) {
                    out[0][j] = narrow<T>(x[i][j]);
                } else {
                    uint32_t s[kParts];
                    split(x[i][j], s);
#pragma unroll
                    for (int q = 0; q < planes; ++q) out[q][j] = uint16_t(s[q] >> 16);
                }
            }
#pragma unroll
            for (int q = 0; q < planes; ++q) *reinterpret_cast<u16x4 *>(a.to + r * a.to_ld + q * a.to_part + c) = out[q];
        }
    if (!a.sums) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[threadIdx.x / 16][threadIdx.x % 16 * 4 + j] = sum[j];
    __syncthreads();
    const uint32_t at = block % tiles_c * 64 + threadIdx.x;
    if (threadIdx.x < 64 && at < a.cols) {
        float all = 0;
#pragma unroll
        for (uint32_t r = 0; r < 16; ++r) all += sums[r][threadIdx.x];
        a.sums[uint64_t(tile) * a.cols + at] = all;
    }
}

// db from the tiles' sums, added up in their order.
template <typename T>
__global__ __launch_bounds__(256) void bias_kernel(const float *sums, uint32_t tiles, uint32_t cols, T *db, uint32_t accumulate)
{
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    float s = 0;
#pragma unroll 8
    for (uint32_t t = 0; t < tiles; ++t) s += sums[uint64_t(t) * cols + c];
    db[c] = narrow<T>(accumulate ? s + widen(db[c]) : s);
}

// ------------------------------------------------------------------ results

struct Result {
    const void *bias;   // [n] or NULL
    const void *added;  // [m, n] or NULL: the residual, or the result itself where it is added to
    void *out;
    void *pre;          // or NULL
    uint64_t lda, ldo, ldp;
    uint32_t act;
};

// Eight neighbours of a row of the result, all there; what is added has been read.
template <typename T>
__device__ inline void finish(const Result &r, uint32_t m, uint32_t n, const float (&bias)[8], const Lane<T, 8> &added, float (&z)[8])
{
    if (r.bias)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] += bias[j];
    if (r.pre) store_n<T, 8>(static_cast<T *>(r.pre) + m * r.ldp + n, z);
    activate<T>(z, r.act);
    if (r.added)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] += added[j];
    store_n<T, 8>(static_cast<T *>(r.out) + m * r.ldo + n, z);
}

// The same of which `count` are there.
template <typename T>
__device__ inline void finish(const Result &r, uint32_t m, uint32_t n, uint32_t count, float (&z)[8])
{
    const T *bias = static_cast<const T *>(r.bias) + n, *add = static_cast<const T *>(r.added) + m * r.lda + n;
    if (count == 8) {
        float b[8];
        Lane<T, 8> added;
        if (r.bias) load_n<T, 8>(bias, b);
        if (r.added) added.load(add);
        return finish<T>(r, m, n, b, added, z);
    }
    T *out = static_cast<T *>(r.out) + m * r.ldo + n, *pre = static_cast<T *>(r.pre) + m * r.ldp + n;
#pragma unroll
    for (uint32_t j = 0; j < 8; ++j) {
        if (j >= count) break;
        float x[1] = {z[j]};
        if (r.bias) x[0] += widen(bias[j]);
        if (r.pre) pre[j] = narrow<T>(x[0]);
        activate<T>(x, r.act);
        if (r.added) x[0] += widen(add[j]);
        out[j] = narrow<T>(x[0]);
    }
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
    float *partial;                 // [splits][m][n]
    Result result;
};

// The six products of parts whose sum is a float32 product but for 2^-22 of it at most, smallest first.
__device__ inline uint32_t term_p(uint32_t t) { return (0x001102u >> (4 * t)) & 3; }
__device__ inline uint32_t term_q(uint32_t t) { return (0x010120u >> (4 * t)) & 3; }

// Which tile and which part of its sum a workgroup takes.  Workgroups go to the eight XCDs in turn.  Each XCD gets
// neighbouring tiles, and goes through them in groups of eight rows of tiles, so that what its L2 holds is used again.
struct Place {
    uint32_t m0, n0, part;
};
template <uint32_t TM, uint32_t TN>
__device__ inline Place place(const Product &a)
{
    const uint32_t tiles = a.tiles_m * a.tiles_n, part = blockIdx.x / tiles, b = blockIdx.x % tiles;
    const uint32_t xcd = b % 8, extra = tiles % 8, at = xcd * (tiles / 8) + min(xcd, extra) + b / 8;
    const uint32_t group = at / (8 * a.tiles_n), left = min(a.tiles_m - group * 8, 8u), in = at - group * 8 * a.tiles_n;
    return Place{(group * 8 + in % left) * TM, in / left * TN, part};
}

// A wave's sums, rows from m0 and columns from n0 on, go through its own strip of local memory, 32 rows at a time, so that a
// row's neighbours are written together.
template <typename T, int RM, int RN>
__device__ inline __attribute__((always_inline)) void write_out(const Product &a, const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0,
                                                                uint32_t part)
{
    constexpr uint32_t kRow = RN * 16 + 4, across = RN * 2, rows = 64 / across, kLines = 32 / rows;
    const uint32_t ln = lane % across * 8, n = n0 + ln, have = n < a.n ? min(8u, a.n - n) : 0;
    const Result &res = a.result;
    float bias[8] = {};
    if (res.bias && have == 8) load_n<T, 8>(static_cast<const T *>(res.bias) + n, bias);
#pragma unroll 1
    for (int i = 0; i < RM; i += 2) {
        // (one copy of what follows for all strips; registers are not found by a number at run time)
#pragma unroll
        for (int at = 0; at < RM; at += 2)
            if (at == i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < RN; ++j)
                        *reinterpret_cast<f32x4 *>(strip + (16 * h + (lane & 15)) * kRow + 16 * j + 4 * (lane >> 4)) = acc[at + h][j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        const uint32_t m = m0 + i * 16 + lane / across;
        Lane<T, 8> added[kLines];
        if (res.added && a.splits == 1 && have == 8)
#pragma unroll
            for (uint32_t l = 0; l < kLines; ++l)
                if (m + l * rows < a.m) added[l].load(static_cast<const T *>(res.added) + (m + l * rows) * res.lda + n);
#pragma unroll
        for (uint32_t l = 0; l < kLines; ++l) {
            if (m + l * rows >= a.m || !have) continue;
            float z[8];
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(strip + (l * rows + lane / across) * kRow + ln + h);
                z[h] = v.x;
                z[h + 1] = v.y;
                z[h + 2] = v.z;
                z[h + 3] = v.w;
            }
            if (a.splits != 1) {
                float *to = a.partial + (uint64_t(part) * a.m + m + l * rows) * a.n + n;
                if (have == 8) {
                    store_n<float, 8>(to, z);
                } else {
#pragma unroll
                    for (uint32_t h = 0; h < 8; ++h)
                        if (h < have) to[h] = z[h];
                }
            } else if (have == 8) {
                finish<T>(res, m + l * rows, n, bias, added[l], z);
            } else {
                finish<T>(res, m + l * rows, n, have, z);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
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
template <int WM, int WN, int RM, int RN, bool PT, bool QT>
__global__ __launch_bounds__(WM *WN * 64, 2) void product_kernel(Product a)
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
    const Place at = place<TM, TN>(a);
    const uint32_t m0 = at.m0, n0 = at.n0;

    const Side<PT, TM, kThreads> side_p(m0, a.ldp);
    const Side<QT, TN, kThreads> side_q(n0, a.ldq);

    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab - 1) / kSlab - first);

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

    float *strip = reinterpret_cast<float *>(wave * 32 * kRow * 4 + 32 * kRow * 4 <= kStage ? stage0 + wave * 32 * kRow * 4
                                                                                            : stage1 + (wave - kStage / (32 * kRow * 4)) * 32 * kRow * 4);
    write_out<uint16_t, RM, RN>(a, acc, strip, lane, m0 + wm * RM * 16, n0 + wn * RN * 16, at.part);
}

// The product where there is no more than a tile of 128 by 128 for each compute unit, which its eight waves have to themselves: what
// they wait for is memory, so four stages keep three slabs on their way, and a slab's pieces are all read
// while the one before is multiplied.  (us, here / by two workgroups of product_kernel to a compute unit: 2048 by 2048 by 4096 35 / 47,
// 700 by 4096 by 4096 31 / 43, 1024 by 4096 by 1024 14 / 18, 4096 by 1024 by 2048 20 / 27; with two tiles for each
// compute unit, one behind the other here, 8192 by 1024 by 4096 74 / 65.)
template <bool PT, bool QT>
__global__ __launch_bounds__(512, 2) void lone_kernel(Product a)
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
    const Place at = place<T, T>(a);
    const Side<PT, T, 512> side_p(at.m0, a.ldp);
    const Side<QT, T, 512> side_q(at.n0, a.ldq);
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab - 1) / kSlab - first);
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
    float *strip = reinterpret_cast<float *>(wave < 4 ? stage0 : stage1) + (wave & 3) * 32 * kRow;
    write_out<uint16_t, RM, RN>(a, acc, strip, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
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
template <bool PT, bool QT>
__global__ __launch_bounds__(512, 2) void product3_kernel(Product a)
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
    const Place at = place<T, T>(a);
    const Side3<PT, T> side_p(at.m0, a.ldp, a.part_p);
    const Side3<QT, T> side_q(at.n0, a.ldq, a.part_q);
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab3 - 1) / kSlab3 - first);
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
    write_out<float, RM, RN>(a, acc, reinterpret_cast<float *>(stage0) + wave * 32 * kRow, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
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
__global__ __launch_bounds__(512, 2) void raw3_kernel(Product a)
{
    constexpr int RM = 4, RN = 2;
    constexpr uint32_t T = 128, kStage = 2 * T * kParts * 64, kRow = RN * 16 + 4;
    constexpr int kReads = kParts * (RM + RN);
    static_assert(8 * 32 * kRow * 4 <= kStage, "the strips fit");
    __shared__ __attribute__((aligned(1024))) char stage0[kStage];
    __shared__ __attribute__((aligned(1024))) char stage1[kStage];
    const uint32_t lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t wm = wave & 1, wn = wave >> 1;
    const Place at = place<T, T>(a);
    const Raw3<T> side_p(a.ldp), side_q(a.ldq);
    const Side3<false, T> parts(0, 0, 0);
    const uint32_t first = at.part * a.slabs, count = min(a.slabs, (a.k + kSlab3 - 1) / kSlab3 - first), last = first + count - 1;
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
    write_out<float, RM, RN>(a, acc, reinterpret_cast<float *>(stage0) + wave * 32 * kRow, lane, at.m0 + wm * RM * 16, at.n0 + wn * RN * 16, at.part);
}

// The parts of a split sum, added up in their order; a sum without terms is no parts.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float *partial, uint32_t splits, uint32_t rows, uint32_t cols, Result r)
{
    const uint32_t across = (cols + 7) / 8;
    for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < uint64_t(rows) * across; i += uint64_t(gridDim.x) * 256) {
        const uint32_t m = uint32_t(i / across), n = uint32_t(i % across) * 8, have = min(8u, cols - n);
        float z[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        const float *from = partial + uint64_t(m) * cols + n;
        const uint64_t next = uint64_t(rows) * cols;
#pragma unroll 4
        for (uint32_t s = 0; s < splits; ++s, from += next) {
            float t[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (have == 8) {
                load_n<float, 8>(from, t);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    if (j < have) t[j] = from[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += t[j];
        }
        finish<T>(r, m, n, have, z);
    }
}

// ------------------------------------------------------------------ few rows

struct FewArgs {
    const void *x, *w;
    uint64_t ldx, ldw;
    uint32_t rows, in, out;
    Result result;
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

// Up to kFewRows rows: the weights are read once, straight into registers, in pieces of 64 k's of 16 features out; rows of x,
// which all workgroups read, come from the caches.  kFewWaves waves share the k's of 16 features out and add up their
// sums in local memory.  The matrix instruction's k's may be in any order that both operands share: a lane takes 16
// neighbours, so that four lanes read a whole cache line.  float32 is taken apart in registers.
//
// Bound by the weights' bytes (one row of bfloat16 through 4096 by 11008, not in any cache: 17.5 us, 5.2 TB/s; 16 features
// out to a workgroup, 32 take half as long again; four or sixteen waves a sixth and a twelfth more; eight pieces on their way instead
// of four a tenth), at 16 rows also by x, which is as many bytes to a workgroup then (26.0).
constexpr int kFewWaves = 8;
template <typename T>
__global__ __launch_bounds__(kFewWaves * 64, 2) void few_kernel(FewArgs a)
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
    finish<T>(a.result, m, n, min(8u, a.out - n), z);
}

// ------------------------------------------------------------------ host

// How a product is cut: tiles of `rows` by 256 (256 rows) or 128, and the parts of the sum that make up for few tiles.
struct Shape {
    uint32_t rows, tiles_m, tiles_n, slabs, splits;
    bool lone;  // bfloat16 tiles of 128 that each have a compute unit to themselves: lone_kernel
};

// By what the candidates would take, in us, from measurements at sizes from 333 by 1001 by 832 to 8192 by 8192 by 8192 (within 15 %
// of them): a slab of 256 by 256 takes a compute unit to itself for 1.68; two of 128 by 128 share one for 1.01, one
// that is left over takes 0.70, one alone by lone_kernel 0.50, a slab of 32 float32 1.1; parts of a sum cost a launch, and their bytes written and read.  (us, 256 by 256 / 128 by 128
// in one, two, four parts: 4096 cubed 107 / 124; 8192 by 2560 by 1024 64 / 53; 2048 by 2048 by 4096 81 / 35, 49; 1024 by 4096 by
// 1024 31 / 14, 27; 1024 by 1024 by 4096 - / -, -, 23; 333 by 1001 by 832 - / 10, -, -.)
Shape shape_of(uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, bool turned_p)
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
        if (splits < 1) splits = 1;
    } else {
        double best = 0;
        for (const uint32_t t : {256u, 128u}) {
            if (t == 256 && dtype == TAGC_F32) continue;
            const uint64_t tm = (m + t - 1) / t, tn = (n + t - 1) / t, tiles = tm * tn;
            for (uint64_t parts = 1; parts <= 16 && parts <= slabs; ++parts) {
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
    const void *p;
    uint64_t ld;
    uint32_t part;  // of float32 the three parts of a row, one behind the other, are so far apart
};

// whether a matrix with `cols` elements to a row can be read as it lies: in words, and, where a row is k's, in pieces of 16 bytes
// that do not straddle the last of them
bool as_it_lies(uint32_t dtype, const void *p, uint64_t ld, uint64_t cols, bool turned)
{
    return dtype == TAGC_BF16 && (reinterpret_cast<uintptr_t>(p) & 3) == 0 && ld % 2 == 0 && ld < kMaxSide && cols % (turned ? 2 : 8) == 0;
}

// Whether float32 rows of k's are read as they lie (raw3_kernel): laying out (m + n) k elements takes 2.1 us a million, and m n k products
// of what lies as it did 1.6 us a thousand million more.
bool raw_pays(uint64_t m, uint64_t n) { return m * n < 1300 * (m + n); }

Operand room(Places &w, uint32_t dtype, uint64_t rows, uint64_t cols)
{
    const uint64_t part = up(cols, 64), ld = part * (dtype == TAGC_F32 ? kParts : 1);
    return Operand{w.take<uint16_t>(rows * ld), ld, uint32_t(part)};
}

PackArgs packed(const void *src, uint64_t ld, uint64_t rows, uint64_t cols, const Operand &to)
{
    PackArgs a{};
    a.src = src;
    a.ld = ld;
    a.rows = uint32_t(rows);
    a.cols = uint32_t(cols);
    a.to = static_cast<uint16_t *>(const_cast<void *>(to.p));
    a.to_ld = to.ld;
    a.to_part = to.part;
    return a;
}

// What a call has to lay out, gathered while its workspace is handed out.
struct Packs {
    PackJobs jobs{};
    uint64_t groups = 0;
    int n = 0;
    void add(const PackArgs &a)
    {
        jobs.job[n] = a;
        jobs.first[n++] = uint32_t(groups);
        groups += up(a.rows, kPackRows) / kPackRows * (up(a.cols, 64) / 64);
    }
    // a matrix as it lies, or laid out anew
    Operand operand(Places &w, uint32_t dtype, const void *src, uint64_t ld, uint64_t rows, uint64_t cols, bool turned)
    {
        if (as_it_lies(dtype, src, ld, cols, turned)) return Operand{src, ld, 0};
        const Operand to = room(w, dtype, rows, cols);
        add(packed(src, ld, rows, cols, to));
        return to;
    }
    template <typename T>
    void launch(hipStream_t s)
    {
        if (!groups) return;
        for (int i = n; i < 3; ++i) jobs.first[i] = uint32_t(groups);
        ProfileScope prof("linear_pack", s);
        pack_kernel<T><<<uint32_t(groups), 256, 0, s>>>(jobs);
    }
};

template <typename T, bool PT, bool QT>
void launch_product(const Operand &p, const Operand &q, uint64_t m, uint64_t n, uint64_t k, float *partial, const Result &r, hipStream_t s)
{
    Product a;
    a.p = p.p;
    a.q = q.p;
    a.ldp = p.ld;
    a.ldq = q.ld;
    a.part_p = p.part;
    a.part_q = q.part;
    a.m = uint32_t(m);
    a.n = uint32_t(n);
    a.k = uint32_t(k);
    const Shape f = shape_of(m, n, k, sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16, PT);
    a.tiles_m = f.tiles_m;
    a.tiles_n = f.tiles_n;
    a.slabs = f.slabs;
    a.splits = f.splits;
    a.partial = partial;
    a.result = r;
    const uint32_t grid = f.tiles_m * f.tiles_n * f.splits;
    if (grid) {
        ProfileScope prof("linear_product", s);
        if constexpr (sizeof(T) == 4) {
            if constexpr (!PT && !QT) {
                if (!p.part) raw3_kernel<<<grid, 512, 0, s>>>(a);
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
    if (f.splits != 1) {
        ProfileScope prof("linear_join", s);
        const uint64_t groups = (m * ((n + 7) / 8) + 255) / 256;
        join_kernel<T><<<uint32_t(groups < 65536 ? groups : 65536), 256, 0, s>>>(partial, f.splits, a.m, a.n, r);
    }
}

// elements of the partial sums of a product
uint64_t partial_elems(uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, bool turned_p)
{
    const Shape f = shape_of(m, n, k, dtype, turned_p);
    return f.splits > 1 ? f.splits * m * n : 0;
}

bool aligned_to(const void *p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// a matrix that must or may be there
bool good(const void *p, uint64_t ld, uint64_t cols, uint64_t bytes) { return !p || (aligned_to(p, bytes) && ld >= cols && ld < (1ull << 40)); }

// Rows of a matrix as bytes in memory.
struct Rows {
    const char *p;
    uint64_t rows, width, ld;
    Rows(const void *at, uint64_t n, uint64_t bytes, uint64_t step) : p(static_cast<const char *>(at)), rows(at && bytes ? n : 0), width(bytes), ld(step)
    {
        if (rows > 1 && ld == width) {  // one row as well
            width *= rows;
            rows = 1;
        }
    }
    const char *end() const { return p + (rows - 1) * ld + width; }
    // whether one of them meets [from, to): the last that begins before `to` ends last
    bool meets(const char *from, const char *to) const
    {
        if (to <= p) return false;
        const uint64_t before = uint64_t(to - p - 1) / ld, last = before < rows ? before : rows - 1;
        return p + last * ld + width > from;
    }
};

// Whether two matrices share a byte.  Matrices side by side in one buffer, whose rows alternate, do not.
bool meet(const Rows &a, const Rows &b)
{
    if (!a.rows || !b.rows || a.end() <= b.p || b.end() <= a.p) return false;
    if (a.rows == 1) return b.meets(a.p, a.end());
    if (b.rows == 1) return a.meets(b.p, b.end());
    if (a.ld == b.ld) {
        // row j of b begins `in` bytes into row j + down of a and what lies behind it, and may reach row j + down + 1
        const int64_t d = b.p - a.p, ld = int64_t(a.ld), down = d >= 0 ? d / ld : -((-d + ld - 1) / ld), in = d - down * ld;
        const int64_t ra = int64_t(a.rows), rb = int64_t(b.rows);
        return (in < int64_t(a.width) && down < ra && down + rb > 0) || (in + int64_t(b.width) > ld && down + 1 < ra && down + 1 + rb > 0);
    }
    const Rows &few = a.rows < b.rows ? a : b, &many = a.rows < b.rows ? b : a;
    for (uint64_t i = 0; i < few.rows; ++i)
        if (many.meets(few.p + i * few.ld, few.p + i * few.ld + few.width)) return true;
    return false;
}

int check_sizes(uint64_t rows, uint64_t in, uint64_t out, uint32_t dtype, uint32_t act)
{
    if (dtype > TAGC_BF16 || act > TAGC_ACT_SILU) return TAGC_EINVAL;
    // a tile's 256 rows span fewer than 2^32 bytes
    const uint64_t most = dtype == TAGC_F32 ? kMaxSide / 4 : kMaxSide;
    if (rows >= most || in >= most || out >= most) return TAGC_ESIZE;
    // a launch has fewer than 2^32 threads: at most a workgroup of 256 for each tile of 64 by 64 of all three matrices
    const uint64_t r = up(rows, 64) / 64, i = up(in, 64) / 64, o = up(out, 64) / 64;
    if (r * i + r * o + i * o >= (1ull << 24)) return TAGC_ESIZE;
    return TAGC_OK;
}

template <typename T>
int forward(const tagc_linear *l, Places &w, bool enqueue, hipStream_t s)
{
    const Result r{l->bias, l->residual, l->y, l->pre, l->ldr, l->ldy, l->ldp, l->activation};
    const uint64_t M = l->rows, K = l->in, N = l->out;
    if (!M || !N) return TAGC_OK;
    if (M <= kFewRows) {
        if (!enqueue) return TAGC_OK;
        ProfileScope prof("linear_few", s);
        few_kernel<T><<<uint32_t((N + 15) / 16), kFewWaves * 64, 0, s>>>(FewArgs{l->x, l->w, l->ldx, l->ldw, uint32_t(M), uint32_t(K), uint32_t(N), r});
        return hip_ok(hipGetLastError());
    }
    Packs packs;
    Operand p{l->x, l->ldx, 0}, q{l->w, l->ldw, 0};
    if (sizeof(T) == 2 || !raw_pays(M, N) || l->ldx >= kMaxSide || l->ldw >= kMaxSide) {
        p = packs.operand(w, l->dtype, l->x, l->ldx, M, K, false);
        q = packs.operand(w, l->dtype, l->w, l->ldw, N, K, false);
    }
    float *partial = w.take<float>(partial_elems(M, N, K, l->dtype, false));
    if (!enqueue) return TAGC_OK;
    packs.launch<T>(s);
    launch_product<T, false, false>(p, q, M, N, K, partial, r, s);
    return hip_ok(hipGetLastError());
}

// Behind an activation dz is held in the operands' type: the two products read it, and bfloat16 is what the matrix units take.
// That is one rounding more than dz in float32 has (bfloat16, 4096 by 4096 by 11008, silu: gradients are off by 0.00235 of their
// norm instead of 0.00166, which is what rounding the results leaves by itself); dz in two parts of bfloat16 would keep it and
// double both products.  Where there is no activation dz is dy, and db is summed from dz before it is rounded.
template <typename T>
int backward(const tagc_linear_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows, K = l->in, N = l->out;
    const bool dx = l->dx && M && K, dw = l->dw && N && K, db = l->db && N;
    Operand dz{l->dy, l->lddy, 0};
    PackArgs a = packed(l->dy, l->lddy, M, N, Operand{});
    if ((dx || dw) && (l->pre || !as_it_lies(l->dtype, l->dy, l->lddy, N, !dx))) {
        dz = room(w, l->dtype, M, N);
        a = packed(l->dy, l->lddy, M, N, dz);
    }
    a.pre = l->pre;
    a.ldp = l->ldp;
    a.act = l->activation;
    const uint32_t tiles = uint32_t(up(M, kPackRows) / kPackRows);
    if (db) a.sums = w.take<float>(uint64_t(tiles) * N);
    Packs packs;
    if (a.to || db) packs.add(a);
    Operand wq{}, xq{};
    if (dx) wq = packs.operand(w, l->dtype, l->w, l->ldw, N, K, true);
    if (dw) xq = packs.operand(w, l->dtype, l->x, l->ldx, M, K, true);
    // (dx is done with its partial sums when dw begins)
    const uint64_t for_dx = dx ? partial_elems(M, K, N, l->dtype, false) : 0, for_dw = dw ? partial_elems(N, K, M, l->dtype, true) : 0;
    float *partial = w.take<float>(for_dx > for_dw ? for_dx : for_dw);
    if (!enqueue) return TAGC_OK;
    packs.launch<T>(s);
    if (db) {
        ProfileScope prof("linear_bias", s);
        bias_kernel<T><<<uint32_t((N + 255) / 256), 256, 0, s>>>(a.sums, tiles, uint32_t(N), static_cast<T *>(l->db), l->accumulate);
    }
    if (dx) launch_product<T, false, true>(dz, wq, M, K, N, partial, Result{nullptr, nullptr, l->dx, nullptr, 0, l->lddx, 0, TAGC_ACT_NONE}, s);
    if (dw)
        launch_product<T, true, true>(dz, xq, N, K, M, partial,
                                      Result{nullptr, l->accumulate ? l->dw : nullptr, l->dw, nullptr, l->lddw, l->lddw, 0, TAGC_ACT_NONE}, s);
    return hip_ok(hipGetLastError());
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

// Results are written while other workgroups read operands: they lie apart, but that y may be the residual, each of whose elements
// is read where y's is written, and pre may be y where both are the same numbers.
int check_apart(const tagc_linear *l)
{
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, M = l->rows, K = l->in * e, N = l->out * e;
    const Rows x(l->x, M, K, l->ldx * e), w(l->w, l->out, K, l->ldw * e), bias(l->bias, 1, N, N), residual(l->residual, M, N, l->ldr * e);
    const Rows y(l->y, M, N, l->ldy * e), pre(l->pre, M, N, l->ldp * e);
    const bool over = l->y == l->residual && (M <= 1 || l->ldy == l->ldr);
    const bool one = l->y == l->pre && (M <= 1 || l->ldy == l->ldp) && l->activation == TAGC_ACT_NONE && !l->residual;
    if (meet(y, x) || meet(y, w) || meet(y, bias) || (!over && meet(y, residual)) || meet(pre, x) || meet(pre, w) || meet(pre, bias) ||
        meet(pre, residual) || (!one && meet(pre, y)))
        return TAGC_EINVAL;
    return TAGC_OK;
}

// What is laid out anew has been read before the first result is written: float32 operands, and dy and pre behind an activation.
int check_apart(const tagc_linear_grad *l)
{
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, M = l->rows, K = l->in * e, N = l->out * e;
    const bool lies = l->dtype == TAGC_BF16;
    const Rows in[] = {Rows(lies && l->dw ? l->x : nullptr, M, K, l->ldx * e), Rows(lies && l->dx ? l->w : nullptr, l->out, K, l->ldw * e),
                       Rows(lies && !l->pre ? l->dy : nullptr, M, N, l->lddy * e)};
    const Rows out[] = {Rows(l->dx, M, K, l->lddx * e), Rows(l->dw, l->out, K, l->lddw * e), Rows(l->db, 1, N, N)};
    for (int i = 0; i < 3; ++i) {
        for (const Rows &r : in)
            if (meet(out[i], r)) return TAGC_EINVAL;
        for (int j = 0; j < i; ++j)
            if (meet(out[i], out[j])) return TAGC_EINVAL;
    }
    return TAGC_OK;
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_rows_meet_host(uint64_t a, uint64_t a_rows, uint64_t a_width, uint64_t a_ld, uint64_t b, uint64_t b_rows,
                                   uint64_t b_width, uint64_t b_ld)
{
    return meet(Rows(reinterpret_cast<const void *>(a), a_rows, a_width, a_ld), Rows(reinterpret_cast<const void *>(b), b_rows, b_width, b_ld));
}

extern "C" int tagc_linear_path_host(uint32_t pass, uint64_t rows, uint64_t in, uint64_t out, uint32_t dtype, uint32_t *path)
{
    if (!path || pass > TAGC_PASS_DW) return TAGC_EINVAL;
    const int rc = check_sizes(rows, in, out, dtype, TAGC_ACT_NONE);
    if (rc) return rc;
    path[0] = path[1] = path[2] = 0;
    if (pass == TAGC_PASS_FORWARD && rows <= kFewRows) return TAGC_OK;
    const Shape f = pass == TAGC_PASS_FORWARD ? shape_of(rows, out, in, dtype, false)
                    : pass == TAGC_PASS_DX    ? shape_of(rows, in, out, dtype, false)
                                              : shape_of(out, in, rows, dtype, true);
    if (dtype == TAGC_BF16) path[0] = f.lone ? TAGC_PATH_LONE : TAGC_PATH_PRODUCT;
    else path[0] = pass == TAGC_PASS_FORWARD && raw_pays(rows, out) ? TAGC_PATH_RAW3 : TAGC_PATH_PRODUCT3;
    path[1] = f.rows;
    path[2] = f.splits;
    return TAGC_OK;
}

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
    int rc = tagc_linear_forward_workspace(l, &need);
    if (!rc) rc = check_apart(l);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return l->dtype == TAGC_F32 ? forward<float>(l, w, true, s) : forward<uint16_t>(l, w, true, s);
}

extern "C" int tagc_linear_backward(const tagc_linear_grad *l, void *workspace, void *stream)
{
    uint64_t need = 0;
    int rc = tagc_linear_backward_workspace(l, &need);
    if (!rc) rc = check_apart(l);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    hipStream_t s = static_cast<hipStream_t>(stream);
    return l->dtype == TAGC_F32 ? backward<float>(l, w, true, s) : backward<uint16_t>(l, w, true, s);
}
