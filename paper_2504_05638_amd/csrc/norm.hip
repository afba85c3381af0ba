// Norms of rows, forward and backward.
//
//   y = (x - mean) r w + b,  r = 1 / sqrt(mean of (x - mean)^2 + eps)
//   h = (x - mean) r, u = dy w:  dx = r (u - mean u - h mean(u h)),  dw = sum of dy h over the rows,  db = sum of dy
//
// A row is held in registers by a wave, four or sixteen of them, so that it is read once; its sums go through the waves' lanes and
// local memory.  Rows need a dozen operations an element: both passes are bound by the bytes of rows, and at few rows by
// the latency of a load, two meetings and a store.
#include <math.h>

#include "device_utils.h"
#include "elements.h"
#include "tagc_internal.h"
#include "tagc_train.h"

namespace tagc {

namespace {

// The sum over a wave's lanes, in all of them.  (Shifts inside the rows of 16 lanes, then the two broadcasts across them: the order is the
// lanes', whatever runs beside.)
template <int CTRL, int ROWS>
__device__ inline float dpp_add(float x)
{
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xF, ROWS == 0xF));
}
__device__ inline float wave_total(float x)
{
    x = dpp_add<0x111, 0xF>(x);
    x = dpp_add<0x112, 0xF>(x);
    x = dpp_add<0x114, 0xF>(x);
    x = dpp_add<0x118, 0xF>(x);
    x = dpp_add<0x142, 0xA>(x);
    x = dpp_add<0x143, 0xC>(x);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// The same of N numbers over the LANES that share a row.  `room`: [2][LANES / 64][N], its halves used in turn, so that one meeting is
// enough: what was read from a half has been read when the next sum's waves have met.
template <int LANES, int N>
__device__ inline void row_totals(float (&x)[N], float *room, uint32_t &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = wave_total(x[i]);
    if constexpr (LANES > 64) {
        constexpr int W = LANES / 64;
        float *half = room + turn * W * N;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) half[threadIdx.x / 64 * N + i] = x[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) s += half[w * N + i];
            x[i] = s;
        }
    }
}

// A thread's part of a row as it lies in memory: STEPS pieces of 16 bytes, LANES pieces apart; zeros behind the row's end.
template <typename T, int LANES, int STEPS>
struct Part {
    static constexpr int V = 16 / int(sizeof(T)), N = V * STEPS;
    u32x4_t v[STEPS];
    __device__ static inline uint32_t column(int s) { return (uint32_t(s) * LANES + threadIdx.x % LANES) * V; }
    // Asks for it.  Behind the row's end a lane asks for the row's last 16 bytes, and settle() takes from them what is its own: lanes that write zeros
    // while others' loads are on their way have the wave wait for those (8000 rows of 4095 in bfloat16, backward: 173 us, 62 so).
    __device__ inline void load(const T *row, uint32_t width)
    {
        if (width >= V) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                Lane<T, V> in;
                in.load(row + min(column(s), width - V));
                v[s] = __builtin_bit_cast(u32x4_t, in.v);
            }
        } else {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                v[s] = u32x4_t{0, 0, 0, 0};
                // (in words: held by themselves, bfloat16 numbers would take a register each)
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (column(s) + j < width) v[s][j * int(sizeof(T)) / 4] |= bits(row[column(s) + j]) << (j * sizeof(T) * 8 % 32);
            }
        }
    }
    __device__ inline void settle(uint32_t width)
    {
        if (width < V || width == LANES * N) return;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t end = column(s) + V;
            if (end > width) v[s] = end - width >= V ? u32x4_t{0, 0, 0, 0} : __builtin_bit_cast(u32x4_t, __builtin_bit_cast(unsigned __int128, v[s]) >> ((end - width) * sizeof(T) * 8));
        }
    }
    __device__ static inline uint32_t bits(T x)
    {
        if constexpr (sizeof(T) == 2) return x;
        else return __float_as_uint(x);
    }
    __device__ inline void fill(uint32_t word)
    {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) v[s] = u32x4_t{word, word, word, word};
    }
    __device__ inline float operator[](int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(v[i / 4][i % 4]);
        const uint32_t word = v[i / 8][i % 8 / 2];
        return __uint_as_float(i % 2 ? word & 0xFFFF0000u : word << 16);
    }
    // what was computed from it is computed again
    __device__ inline void forget()
    {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) asm volatile("" : "+v"(v[s]));
    }
    // f(i): what becomes of element i
    template <typename F>
    __device__ static inline void store(T *row, uint32_t width, F f)
    {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint32_t c = column(s);
            float y[V];
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = f(s * V + j);
            if (c + V <= width) {
                store_n<T, V>(row + c, y);
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (c + j < width) row[c + j] = narrow<T>(y[j]);
            }
        }
    }
    // whether element i is the row's
    __device__ static inline bool there(int i, uint32_t width) { return column(i / V) + i % V < width; }
};
template <typename T>
constexpr uint32_t kOnes = sizeof(T) == 4 ? 0x3F800000u : 0x3F803F80u;

struct Norm {
    const void *x, *w, *b;
    void *y;
    float *stats;
    uint64_t ldx, ldy;
    uint32_t rows, width, kind;
    float eps;
};

// LANES threads a row, 256 or LANES threads a workgroup.
template <int LANES>
constexpr int kNormThreads = LANES < 256 ? 256 : LANES;

template <typename T, int LANES, int STEPS>
__global__ __launch_bounds__(kNormThreads<LANES>) void norm_kernel(Norm a)
{
    typedef Part<T, LANES, STEPS> P;
    constexpr uint32_t kRows = kNormThreads<LANES> / LANES;
    __shared__ float room[2 * (LANES / 64)];
    uint32_t turn = 0;
    const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.w), *b = static_cast<const T *>(a.b);
    const uint64_t row = uint64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    if (row >= a.rows) return;  // (LANES of 256 and more: a workgroup has one row, and all its waves go on to the meetings)
    P in;
    in.load(x + row * a.ldx, a.width);
    in.settle(a.width);
    float z[P::N], sum[1] = {0};
#pragma unroll
    for (int i = 0; i < P::N; ++i) {
        z[i] = in[i];
        sum[0] += z[i];
    }
    float mean = 0;
    if (a.kind == TAGC_NORM_LAYER) {
        row_totals<LANES>(sum, room, turn);
        mean = sum[0] / float(a.width);  // (a reciprocal's rounding would leave something of a row that is all mean)
#pragma unroll
        for (int i = 0; i < P::N; ++i) z[i] = P::there(i, a.width) ? z[i] - mean : 0.0f;
    }
    // (the squares of what is left, not a difference of sums: exact to rounding also where the mean is large)
    sum[0] = 0;
#pragma unroll
    for (int i = 0; i < P::N; ++i) sum[0] += z[i] * z[i];
    row_totals<LANES>(sum, room, turn);
    const float r = 1.0f / sqrtf(sum[0] / float(a.width) + a.eps);
    P weight, bias;
    weight.fill(kOnes<T>);
    bias.fill(0);
    if (w) weight.load(w, a.width);
    if (b) bias.load(b, a.width);
    weight.settle(a.width);
    bias.settle(a.width);
    P::store(static_cast<T *>(a.y) + row * a.ldy, a.width, [&](int i) { return z[i] * r * weight[i] + bias[i]; });
    if (a.stats && threadIdx.x % LANES == 0) *reinterpret_cast<float2 *>(a.stats + 2 * row) = make_float2(mean, r);
}

struct NormGrad {
    const void *x, *w, *dy, *residual;
    const float *stats;
    void *dx;
    float *sums;  // [workgroups][2][width] or NULL: what the workgroups' rows add to dw and db
    uint64_t ldx, lddy, ldr, lddx;
    uint32_t rows, width;
    float over;    // 1 / width
    uint32_t groups;  // workgroups that take rows; those behind them take columns, for which `sums` is NULL
    void *dw, *db;    // theirs
    uint32_t accumulate;
};

// Few rows' dw and db without a launch to join them: a workgroup takes 8 * V columns of all rows, eight lanes to a row, and adds up what its
// eighths of waves and its waves have, in their order.  It reads x and dy once more, from the caches.
template <typename T, int THREADS>
__device__ inline void norm_columns(const NormGrad &a)
{
    constexpr uint32_t V = 16 / sizeof(T), kSlices = THREADS / 8, kAhead = 4, W = THREADS / 64;
    __shared__ float parts[2][W][8 * V];
    const uint32_t lane = threadIdx.x % 8, slice = threadIdx.x / 8, c = (blockIdx.x - a.groups) * 8 * V + lane * V;
    // (as Part: of a row's last piece that is not whole the row's last 16 bytes)
    const bool thin = a.width < V;
    const uint32_t at = thin ? 0 : min(c, a.width - V);
    const T *x = static_cast<const T *>(a.x) + at, *dy = static_cast<const T *>(a.dy) + at;
    float dw[V] = {}, db[V] = {};
    for (uint32_t first = slice; first < a.rows; first += kSlices * kAhead) {
        float px[kAhead][V], py[kAhead][V];
        float2 stats[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            const uint64_t row = min(first + k * kSlices, a.rows - 1);
            stats[k] = *reinterpret_cast<const float2 *>(a.stats + 2 * row);
            if (!thin) {
                load_n<T, V>(x + row * a.ldx, px[k]);
                load_n<T, V>(dy + row * a.lddy, py[k]);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < V; ++j) {
                    px[k][j] = widen(x[row * a.ldx + min(j, a.width - 1)]);
                    py[k][j] = widen(dy[row * a.lddy + min(j, a.width - 1)]);
                }
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) {
                const float g = first + k * kSlices < a.rows ? py[k][j] : 0.0f;
                // (a row that is not there again, whose numbers may be infinite)
                dw[j] += first + k * kSlices < a.rows ? g * ((px[k][j] - stats[k].x) * stats[k].y) : 0.0f;
                db[j] += g;
            }
    }
#pragma unroll
    for (uint32_t j = 0; j < V; ++j)
#pragma unroll
        for (int d = 8; d < 64; d *= 2) {
            dw[j] += __shfl_xor(dw[j], d, 64);
            db[j] += __shfl_xor(db[j], d, 64);
        }
    if (threadIdx.x % 64 < 8)
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) {
            parts[0][threadIdx.x / 64][lane * V + j] = dw[j];
            parts[1][threadIdx.x / 64][lane * V + j] = db[j];
        }
    __syncthreads();
    if (threadIdx.x >= 16 * V) return;
    const uint32_t which = threadIdx.x / (8 * V), own = threadIdx.x % (8 * V);
    float sum = 0;
#pragma unroll
    for (uint32_t w = 0; w < W; ++w) sum += parts[which][w][own];
    T *to = static_cast<T *>(which ? a.db : a.dw);
    // (lanes behind the row's end, and elements of its last piece that are another lane's, are not stored)
    const uint32_t begin = (blockIdx.x - a.groups) * 8 * V + own / V * V, place = (thin ? 0 : min(begin, a.width - V)) + own % V;
    if (!to || begin >= a.width || place < begin || place >= a.width) return;
    to[place] = narrow<T>(a.accumulate ? sum + widen(to[place]) : sum);
}

// A workgroup takes every gridDim.x-th row (group of rows), and keeps their part of dw and db in registers.  What lies between the sums
// and dx is computed twice from the row as it lies: held, it would take as many registers as all the rest.
template <typename T, int LANES, int STEPS, bool LAYER>
__global__ __launch_bounds__(kNormThreads<LANES>) void norm_grad_kernel(NormGrad a)
{
    typedef Part<T, LANES, STEPS> P;
    constexpr uint32_t kThreads = kNormThreads<LANES>, kRows = kThreads / LANES;
    if (blockIdx.x >= a.groups) return norm_columns<T, kThreads>(a);
    __shared__ float room[2 * 2 * (LANES / 64)];
    uint32_t turn = 0;
    const T *x = static_cast<const T *>(a.x), *dy = static_cast<const T *>(a.dy), *res = static_cast<const T *>(a.residual);
    P weight;
    weight.fill(kOnes<T>);
    if (a.w) weight.load(static_cast<const T *>(a.w), a.width);
    weight.settle(a.width);
    // (sixteen waves of a row leave a thread 128 registers: their sums are in local memory, each thread's its own, and what
    // is added to dx is asked for last)
    constexpr bool kNarrow = LANES > 256;
    __shared__ float held[kNarrow ? (LAYER ? 2 : 1) * P::N * LANES : 1];
    float dw[P::N] = {}, db[LAYER ? P::N : 1] = {};
    if constexpr (kNarrow)
#pragma unroll
        for (int i = 0; i < (LAYER ? 2 : 1) * P::N; ++i) held[i * LANES + threadIdx.x] = 0.0f;
    // (the next row comes while this one's sums meet, where there are registers for it: 3 % at 8192 by 4096)
    constexpr bool kAhead = P::N <= 16 && !kNarrow;
    P ax, ay, ar;
    float2 next_stats = make_float2(0, 0);
    ar.fill(0);
    auto fetch = [&](uint64_t row) __attribute__((always_inline)) {
        ax.load(x + row * a.ldx, a.width);
        ay.load(dy + row * a.lddy, a.width);
        if (res && !kNarrow) ar.load(res + row * a.ldr, a.width);
        next_stats = *reinterpret_cast<const float2 *>(a.stats + 2 * row);
    };
    const uint64_t step = uint64_t(a.groups) * kRows;
    uint64_t row = uint64_t(blockIdx.x) * kRows + threadIdx.x / LANES;
    if (kAhead && row < a.rows) fetch(row);
    for (; row < a.rows; row += step) {
        if (!kAhead) fetch(row);
        P px = ax, py = ay, pr = ar;
        const float2 stats = next_stats;
        if (kAhead && row + step < a.rows) fetch(row + step);
        px.settle(a.width);
        py.settle(a.width);
        if (!kNarrow) pr.settle(a.width);
        float sum[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < P::N; ++i) {
            const float g = py[i], h = LAYER ? (px[i] - stats.x) * stats.y : px[i] * stats.y, u = g * weight[i];
            // (dy is 0 behind the row's end)
            if constexpr (kNarrow) held[i * LANES + threadIdx.x] += g * h;
            else dw[i] += g * h;
            if constexpr (LAYER) {
                if constexpr (kNarrow) held[(P::N + i) * LANES + threadIdx.x] += g;
                else db[i] += g;
                sum[0] += u;
            }
            sum[1] += u * h;
        }
        if (!a.dx) continue;
        row_totals<LANES>(sum, room, turn);
        const float m = LAYER ? sum[0] * a.over : 0.0f, s = sum[1] * a.over;
        px.forget();
        py.forget();
        T *to = static_cast<T *>(a.dx) + row * a.lddx;
        const auto dx = [&](int i) __attribute__((always_inline)) {
            const float h = LAYER ? (px[i] - stats.x) * stats.y : px[i] * stats.y, u = py[i] * weight[i];
            return stats.y * (u - m - h * s);
        };
        if (kNarrow && !res) {
            P::store(to, a.width, dx);
            continue;
        }
        if (kNarrow) {
            pr.load(res + row * a.ldr, a.width);
            pr.settle(a.width);
        }
        P::store(to, a.width, [&](int i) __attribute__((always_inline)) { return dx(i) + pr[i]; });
    }
    if (!a.sums) return;
    float *to = a.sums + uint64_t(blockIdx.x) * 2 * a.width;
    if constexpr (kNarrow)
#pragma unroll
        for (int i = 0; i < P::N; ++i) {
            dw[i] = held[i * LANES + threadIdx.x];
            if constexpr (LAYER) db[i] = held[(P::N + i) * LANES + threadIdx.x];
        }
    if constexpr (kRows > 1) {
        // a wave's rows after another's, in their order
        __shared__ float both[LAYER ? 2 : 1][LANES * P::N];
        for (uint32_t r = 0; r < kRows; ++r) {
            if (threadIdx.x / LANES == r)
#pragma unroll
                for (int i = 0; i < P::N; ++i) {
                    float *at = &both[0][i * LANES + threadIdx.x % LANES], *bt = &both[LAYER][i * LANES + threadIdx.x % LANES];
                    *at = r ? *at + dw[i] : dw[i];
                    if (LAYER) *bt = r ? *bt + db[i] : db[i];
                }
            __syncthreads();
        }
        if (threadIdx.x / LANES) return;
#pragma unroll
        for (int i = 0; i < P::N; ++i) {
            dw[i] = both[0][i * LANES + threadIdx.x];
            if constexpr (LAYER) db[i] = both[1][i * LANES + threadIdx.x];
        }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
#pragma unroll
        for (int j = 0; j < P::V; ++j) {
            const uint32_t c = P::column(s) + j;
            if (c >= a.width) continue;
            to[c] = dw[s * P::V + j];
            if (LAYER) to[a.width + c] = db[s * P::V + j];
        }
}

// dw (the first workgroups) or db (the others) from the workgroups' sums: 16 columns to a workgroup, whose 64 groups of threads take
// every 64th sum, eight of them on their way at once: they come from other XCDs' writes, a microsecond each.
constexpr uint32_t kJoinSlices = 64, kJoinColumns = 16, kJoinAhead = 8;
template <typename T>
__global__ __launch_bounds__(1024) void norm_join_kernel(const float *sums, uint32_t groups, uint32_t width, T *dw, T *db, uint32_t accumulate)
{
    __shared__ float parts[kJoinSlices][kJoinColumns];
    const uint32_t across = (width + kJoinColumns - 1) / kJoinColumns;
    const bool second = !dw || blockIdx.x >= across;
    const uint32_t at = threadIdx.x % kJoinColumns, slice = threadIdx.x / kJoinColumns, c = blockIdx.x % across * kJoinColumns + at;
    float sum = 0;
    if (c < width)
        for (uint32_t g = slice; g < groups; g += kJoinSlices * kJoinAhead) {
            float x[kJoinAhead];
#pragma unroll
            for (uint32_t i = 0; i < kJoinAhead; ++i) {
                const uint32_t which = g + i * kJoinSlices;
                x[i] = which < groups ? sums[(uint64_t(which) * 2 + second) * width + c] : 0.0f;
            }
#pragma unroll
            for (uint32_t i = 0; i < kJoinAhead; ++i) sum += x[i];
        }
    parts[slice][at] = sum;
    __syncthreads();
    if (slice || c >= width) return;
    T *to = second ? db : dw;
    float s = 0;
#pragma unroll
    for (uint32_t i = 0; i < kJoinSlices; ++i) s += parts[i][at];
    to[c] = narrow<T>(accumulate ? s + widen(to[c]) : s);
}

// ------------------------------------------------------------------ host

// By width: how many lanes share a row, and the elements of each.
template <typename T, typename F>
void by_width(uint64_t width, F f)
{
    constexpr int V = 16 / int(sizeof(T));
    if (width <= 64 * 8) f(std::integral_constant<int, 64>(), std::integral_constant<int, 8 / V>());
    else if (width <= 64 * 16) f(std::integral_constant<int, 64>(), std::integral_constant<int, 16 / V>());
    else if (width <= 256 * 8) f(std::integral_constant<int, 256>(), std::integral_constant<int, 8 / V>());
    else if (width <= 256 * 16) f(std::integral_constant<int, 256>(), std::integral_constant<int, 16 / V>());
    else if (width <= 256 * 32) f(std::integral_constant<int, 256>(), std::integral_constant<int, 32 / V>());
    else f(std::integral_constant<int, 1024>(), std::integral_constant<int, 16 / V>());
}
static_assert(TAGC_MAX_NORM_WIDTH == 1024 * 16, "the widest rows that registers hold");

uint32_t rows_at_once(uint64_t width) { return width <= 64 * 16 ? 4 : 1; }

// Workgroups of the backward pass.  The fewer there are, the fewer sums are left to be joined, and a row on its way behind the one in work keeps
// the memory busy.  (us, one / two / three / four to a compute unit: bfloat16 8192 by 4096 54 / 57 / 60 / 62, 4096 by 8192 66 / 66 / 76 / 80,
// 16384 by 2048 64 / 55 / 57 / 61, 32768 by 512 36 / 30 / 32 / 33; float32 8192 by 768 32 / 27 / 32 / 32, 2048 by
// 8192 67 / 77 / 87 / 99.)
uint32_t grad_groups(uint64_t rows, uint64_t width)
{
    const uint64_t all = (rows + rows_at_once(width) - 1) / rows_at_once(width), most = (width > 2048 ? 1 : 2) * uint64_t(device_cu_count());
    return uint32_t(all < most ? all : most);
}

// Rows up to which dw and db are a part of the one launch.  (us, so / joined by a second one: bfloat16 64 rows of 4096 4.7 / 9.0, 256 8.5 / 12.9, 512
// 13.0 / 13.7, 512 of 16384 24 / 34, of 512 8.2 / 7.0; float32 512 of 768 6.5 / 10.1, of 8192 23 / 31.)
constexpr uint32_t kDirect = 512;

int check(uint64_t rows, uint64_t width, uint32_t dtype, uint32_t kind)
{
    if (dtype > TAGC_BF16 || kind > TAGC_NORM_RMS) return TAGC_EINVAL;
    return rows >> 31 || width > TAGC_MAX_NORM_WIDTH ? TAGC_ESIZE : TAGC_OK;
}

int check(const tagc_norm *n)
{
    if (!n) return TAGC_EINVAL;
    const int rc = check(n->rows, n->width, n->dtype, n->kind);
    if (rc) return rc;
    const uint64_t e = n->dtype == TAGC_F32 ? 4 : 2, M = n->rows, bytes = n->width * e;
    if (!(n->eps >= 0) || !isfinite(float(n->eps)) || (n->kind == TAGC_NORM_RMS && n->b)) return TAGC_EINVAL;
    if (M && n->width && (!n->x || !n->y)) return TAGC_EINVAL;
    if (!good(n->x, n->ldx, n->width, e) || !good(n->y, n->ldy, n->width, e) || !aligned_to(n->w, e) || !aligned_to(n->b, e) || !aligned_to(n->stats, 8))
        return TAGC_EINVAL;
    const Rows x(n->x, M, bytes, n->ldx * e), y(n->y, M, bytes, n->ldy * e), w(n->w, 1, bytes, bytes), b(n->b, 1, bytes, bytes), stats(n->stats, 1, M * 8, M * 8);
    const bool over = n->x == n->y && (M <= 1 || n->ldx == n->ldy);
    if ((!over && meet(y, x)) || meet(y, w) || meet(y, b) || meet(y, stats) || meet(stats, x) || meet(stats, w) || meet(stats, b)) return TAGC_EINVAL;
    return TAGC_OK;
}

int check(const tagc_norm_grad *n)
{
    if (!n || n->reserved || n->accumulate > 1) return TAGC_EINVAL;
    const int rc = check(n->rows, n->width, n->dtype, n->kind);
    if (rc) return rc;
    const uint64_t e = n->dtype == TAGC_F32 ? 4 : 2, M = n->rows, bytes = n->width * e;
    if ((n->kind == TAGC_NORM_RMS && n->db) || (n->residual && !n->dx)) return TAGC_EINVAL;
    if (M && n->width && (!n->x || !n->dy || !n->stats)) return TAGC_EINVAL;
    if (!good(n->x, n->ldx, n->width, e) || !good(n->dy, n->lddy, n->width, e) || !good(n->residual, n->ldr, n->width, e) || !good(n->dx, n->lddx, n->width, e) ||
        !aligned_to(n->w, e) || !aligned_to(n->dw, e) || !aligned_to(n->db, e) || !aligned_to(n->stats, 8))
        return TAGC_EINVAL;
    const Rows x(n->x, M, bytes, n->ldx * e), dy(n->dy, M, bytes, n->lddy * e), res(n->residual, M, bytes, n->ldr * e), dx(n->dx, M, bytes, n->lddx * e);
    const Rows w(n->w, 1, bytes, bytes), stats(n->stats, 1, M * 8, M * 8), dw(n->dw, 1, bytes, bytes), db(n->db, 1, bytes, bytes);
    const auto one = [&](const void *p, uint64_t ld) { return n->dx == p && (M <= 1 || n->lddx == ld); };
    if ((!one(n->x, n->ldx) && meet(dx, x)) || (!one(n->dy, n->lddy) && meet(dx, dy)) || (!one(n->residual, n->ldr) && meet(dx, res)) || meet(dx, w) ||
        meet(dx, stats) || meet(dx, dw) || meet(dx, db) || meet(dw, db))
        return TAGC_EINVAL;
    for (const Rows &in : {x, dy, res, w, stats})
        if (meet(dw, in) || meet(db, in)) return TAGC_EINVAL;
    return TAGC_OK;
}

// (a launch has fewer than 2^32 threads, and a row up to 1024 of them)
constexpr uint64_t kLaunchRows = 1u << 21;

template <typename T>
int forward(const tagc_norm *n, hipStream_t s)
{
    if (!n->width) return TAGC_OK;
    ProfileScope prof("norm", s);
    for (uint64_t first = 0; first < n->rows; first += kLaunchRows) {
        const uint64_t rows = n->rows - first < kLaunchRows ? n->rows - first : kLaunchRows;
        const Norm a{static_cast<const T *>(n->x) + first * n->ldx, n->w, n->b, static_cast<T *>(n->y) + first * n->ldy, n->stats ? n->stats + 2 * first : nullptr,
                     n->ldx, n->ldy, uint32_t(rows), uint32_t(n->width), n->kind, float(n->eps)};
        by_width<T>(n->width, [&](auto lanes, auto steps) {
            constexpr int L = decltype(lanes)::value, threads = kNormThreads<L>;
            norm_kernel<T, L, decltype(steps)::value><<<uint32_t((rows + threads / L - 1) / (threads / L)), threads, 0, s>>>(a);
        });
    }
    return hip_ok(hipGetLastError());
}

template <typename T>
int backward(const tagc_norm_grad *n, Places &w, bool enqueue, hipStream_t s)
{
    if (!n->width) return TAGC_OK;
    // (columns are read while rows' dx is written)
    const bool direct = n->rows && n->rows <= kDirect && !(n->dx && (n->dx == n->x || n->dx == n->dy)), sums = (n->dw || n->db) && !direct, columns = (n->dw || n->db) && direct;
    const uint32_t groups = grad_groups(n->rows, n->width);
    float *room = sums ? w.take<float>(uint64_t(groups) * 2 * n->width) : nullptr;
    if (!enqueue) return TAGC_OK;
    if (groups && (sums || columns || n->dx)) {
        constexpr uint32_t kColumns = 8 * 16 / sizeof(T);
        const NormGrad a{n->x, n->w, n->dy, n->residual, n->stats, n->dx, room, n->ldx, n->lddy, n->ldr, n->lddx, uint32_t(n->rows), uint32_t(n->width),
                         float(1.0 / double(n->width)), sums || n->dx ? groups : 0, n->dw, n->db, n->accumulate};
        const uint32_t grid = a.groups + (columns ? uint32_t((n->width + kColumns - 1) / kColumns) : 0);
        ProfileScope prof("norm_grad", s);
        by_width<T>(n->width, [&](auto lanes, auto steps) {
            constexpr int L = decltype(lanes)::value;
            if (n->kind == TAGC_NORM_LAYER) norm_grad_kernel<T, L, decltype(steps)::value, true><<<grid, kNormThreads<L>, 0, s>>>(a);
            else norm_grad_kernel<T, L, decltype(steps)::value, false><<<grid, kNormThreads<L>, 0, s>>>(a);
        });
    }
    if (sums) {
        ProfileScope prof("norm_join", s);
        norm_join_kernel<T><<<uint32_t((n->width + kJoinColumns - 1) / kJoinColumns) * ((n->dw ? 1 : 0) + (n->db ? 1 : 0)), 1024, 0, s>>>(room, groups, uint32_t(n->width), static_cast<T *>(n->dw), static_cast<T *>(n->db),
                                                                          n->accumulate);
    }
    return hip_ok(hipGetLastError());
}

int backward(const tagc_norm_grad *n, Places &w, bool enqueue, hipStream_t s)
{
    return n->dtype == TAGC_F32 ? backward<float>(n, w, enqueue, s) : backward<uint16_t>(n, w, enqueue, s);
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_norm_forward(const tagc_norm *n, void *stream)
{
    const int rc = check(n);
    if (rc) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return n->dtype == TAGC_F32 ? forward<float>(n, s) : forward<uint16_t>(n, s);
}

extern "C" int tagc_norm_backward_workspace(const tagc_norm_grad *n, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check(n);
    if (rc) return rc;
    Places w(nullptr);
    backward(n, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_norm_backward(const tagc_norm_grad *n, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_norm_backward_workspace(n, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    return backward(n, w, true, static_cast<hipStream_t>(stream));
}
