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

#include "product.h"
#include "tagc_test.h"
#include "tagc_train.h"

namespace tagc {

namespace {

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
};// A workgroup takes a tile of kPackRows by 64, a thread four neighbours of each sixteenth row.
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

// A product whose sums go through finish(), or as parts of them to be joined.
template <typename T>
struct Written : Product {
    static constexpr bool kCounted = false, kPartByPart = true;
    float *partial;                 // [splits][m][n]
    Result result;
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t part) const;
};

// A wave's sums, rows from m0 and columns from n0 on, go through its own strip of local memory, 32 rows at a time, so that a
// row's neighbours are written together.
template <typename T, int RM, int RN>
__device__ inline __attribute__((always_inline)) void write_out(const Written<T> &a, const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0,
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

template <typename T>
template <int RM, int RN>
__device__ inline __attribute__((always_inline)) void Written<T>::put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t part) const
{
    write_out<T, RM, RN>(*this, acc, strip, lane, m0, n0, part);
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

template <typename T>
struct FewWritten : FewArgs {
    Result result;
    __device__ inline void put(uint32_t m, uint32_t n, uint32_t have, float (&z)[8]) const { finish<T>(result, m, n, have, z); }
};

// ------------------------------------------------------------------ host

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
    Written<T> a;
    const Shape f = shape_of(m, n, k, sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16, PT);
    aim(a, p, q, m, n, k, f);
    a.partial = partial;
    a.result = r;
    if (f.tiles_m * f.tiles_n * f.splits) {
        ProfileScope prof("linear_product", s);
        launch<T, PT, QT>(a, f, s);
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
        few_kernel<T><<<uint32_t((N + 15) / 16), kFewWaves * 64, 0, s>>>(FewWritten<T>{{l->x, l->w, l->ldx, l->ldw, uint32_t(M), uint32_t(K), uint32_t(N)}, r});
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
