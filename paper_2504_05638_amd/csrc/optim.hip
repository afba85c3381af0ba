// The optimizer behind the exchange: norm over all gradients, AdamW over many tensors.
//
// A plan's tensors are cut into chunks of kChunk elements; a workgroup finds its chunk's tensor in a
// device table, so that one launch covers any number of tensors of any lengths.  Tensors start
// at any element: vector accesses are declared with the element's alignment, which the
// hardware's global loads and stores take.
#include <math.h>
#include <string.h>

#include <new>
#include <vector>

#include "device_utils.h"
#include "tagc_internal.h"
#include "tagc_train.h"

namespace tagc {

namespace {

constexpr uint32_t kOptimThreads = 256;
constexpr uint32_t kSteps = 4;                                   // times that a thread takes four neighbours
constexpr uint32_t kChunk = kOptimThreads * 4 * kSteps;          // elements of a workgroup
constexpr uint32_t kNormGroups = 2048;                           // most workgroups of the norm
constexpr uint32_t kArriveTogether = 32, kArriveWords = 16;      // workgroups that a count is for; words from count to count
constexpr uint32_t kArriveBytes = 4 * kArriveWords * (1 + kNormGroups / kArriveTogether);
constexpr uint64_t kMaxLength = 1ull << 34;                      // an element's number / 4 fits 32 bits
// (8-bit moments: half the steps; 202 M with bf16 gradients 549 -> 539 us, 9 M at odd places 30.1 -> 27.4; with 32 bits two steps
// are the slower ones, 151 M 717 -> 733 us)
constexpr uint32_t kCodeThreads = 512, kCodeSteps = 2;
static_assert(kCodeThreads * 4 * kCodeSteps == kChunk, "the same chunks");
// a launch has fewer than 2^32 threads: chunks of a plan are fewer than these, the norm's workgroups take many each
constexpr uint64_t kMaxChunks = (1ull << 32) / kOptimThreads, kMaxCodeChunks = (1ull << 32) / kCodeThreads;
static_assert(kChunk % TAGC_MOMENT_BLOCK == 0 && TAGC_MOMENT_BLOCK == 4 * 64, "a wave's step is a block");

struct TensorDev {
    void *param;
    const void *grad;
    void *m, *v;
    uint32_t *bases;
    uint16_t *copy;
    uint64_t length;
    uint64_t first;   // elements of the tensors before
    uint32_t types;   // kParamBf16 | kGradBf16
    uint32_t group;
    uint32_t reserved[2];
};
static_assert(sizeof(TensorDev) == 80, "TensorDev layout");
constexpr uint32_t kParamBf16 = 1, kGradBf16 = 2;

struct ChunkDev {
    uint32_t tensor, chunk;
};

}  // namespace

}  // namespace tagc

struct tagc_optim_s {
    tagc_optim_config cfg;
    std::vector<tagc::TensorDev> rows;
    std::vector<tagc::ChunkDev> chunks;
    bool has_params;
    uint32_t n_groups;  // groups that the tensors name
    tagc_optim_sizes sizes;

    // the table: rows, chunks, then the device state: arrivals, the norm's partial sums
    uint64_t chunks_at() const { return rows.size() * sizeof(tagc::TensorDev); }
    uint64_t state_at() const { return (chunks_at() + chunks.size() * sizeof(tagc::ChunkDev) + 15) & ~uint64_t(15); }
};

namespace tagc {

namespace {


template <typename T>
__device__ inline void load4(const T *p, T (&out)[4])
{
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    const vec v = __builtin_nontemporal_load(reinterpret_cast<const vec *>(p));
#pragma unroll
    for (int j = 0; j < 4; ++j) out[j] = v[j];
}
template <typename T>
__device__ inline void store4(T *p, const T (&in)[4])
{
    typedef T vec __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    vec v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = in[j];
    __builtin_nontemporal_store(v, reinterpret_cast<vec *>(p));
}

// Four elements from `i` on as float32, zeros from `n` on.
template <typename T>
__device__ inline void load_f32(const T *p, uint64_t i, uint64_t n, float (&out)[4])
{
    T raw[4] = {};
    if (i + 4 <= n) {
        load4(p + i, raw);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < n) raw[j] = p[i + j];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) out[j] = __uint_as_float(uint32_t(raw[j]) << 16);
        else out[j] = raw[j];
    }
}

template <typename T>
__device__ inline void store_f32(T *p, uint64_t i, uint64_t n, const float (&x)[4])
{
    T raw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) raw[j] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[j]));  // to nearest, ties to even
        else raw[j] = x[j];
    }
    if (i + 4 <= n) {
        store4(p + i, raw);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i + j < n) p[i + j] = raw[j];
    }
}

// ------------------------------------------------------------------ norm

// Sum of the squares of a chunk's elements that this thread takes, in float64: the square of
// any float32 is finite there, and 2^33 of them lose nothing that a float32 shows.
template <typename T>
__device__ inline double chunk_squares(const T *grad, uint64_t at, uint64_t n)
{
    float g[kSteps][4];
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) load_f32(grad, at + 4 * (k * kOptimThreads + threadIdx.x), n, g[k]);
    double sum = 0;
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += double(g[k][j]) * double(g[k][j]);
    return sum;
}

__device__ inline double power(double b, uint32_t n)
{
    double r = 1;
    for (; n; n >>= 1, b *= b)
        if (n & 1) r *= b;
    return r;
}

struct NormArgs {
    const TensorDev *rows;
    const ChunkDev *chunks;
    uint32_t *arrived;
    uint64_t *partial;
    tagc_optim_control *control;
    double grad_scale, max_norm, beta1, beta2;
    uint32_t n_chunks;
};

// Each workgroup leaves its part of the sum; the last to arrive adds the parts up, in their order.  Arrivals are counted
// by 32 and then by those: 2048 adds to one word took some 12 ns each (9 M gradients 33 us, and 12 so).
//
// Bound by the gradients' bytes: 809 M in bfloat16 take 255 us, 151 M in float32 95, 6.3 TB/s both; a
// call takes 5 us at least.
__global__ __launch_bounds__(kOptimThreads) void norm_kernel(NormArgs a)
{
    __shared__ double smem[kOptimThreads / 64];
    __shared__ uint32_t last;
    double sum = 0;
    for (uint32_t c = blockIdx.x; c < a.n_chunks; c += gridDim.x) {
        const ChunkDev ch = a.chunks[c];
        const TensorDev &t = a.rows[ch.tensor];
        const uint64_t at = uint64_t(ch.chunk) * kChunk;
        if (t.types & kGradBf16) sum += chunk_squares(as_global(static_cast<const uint16_t *>(t.grad)), at, t.length);
        else sum += chunk_squares(as_global(static_cast<const float *>(t.grad)), at, t.length);
    }
    sum = block_sum<double, kOptimThreads / 64>(sum, smem);
    if (threadIdx.x == 0) {
        __hip_atomic_store(&a.partial[blockIdx.x], uint64_t(__double_as_longlong(sum)), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        wait_own_memory_ops();
        const uint32_t group = blockIdx.x / kArriveTogether, groups = (gridDim.x + kArriveTogether - 1) / kArriveTogether;
        const uint32_t of = min(kArriveTogether, gridDim.x - group * kArriveTogether);
        uint32_t *mine = a.arrived + kArriveWords * (1 + group);
        last = 0;
        if (__hip_atomic_fetch_add(mine, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1) {
            // (counts are left as the next call expects them)
            __hip_atomic_store(mine, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            last = __hip_atomic_fetch_add(a.arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == groups - 1;
        }
    }
    __syncthreads();
    if (!last) return;
    double all = 0;
    for (uint32_t i = threadIdx.x; i < gridDim.x; i += kOptimThreads)
        all += __longlong_as_double(int64_t(__hip_atomic_load(&a.partial[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)));
    all = block_sum<double, kOptimThreads / 64>(all, smem);
    if (threadIdx.x) return;
    __hip_atomic_store(a.arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    tagc_optim_control *c = a.control;
    const double norm = a.grad_scale * sqrt(all);
    // (a norm that float32 cannot hold is not finite either)
    const bool finite = norm <= 3.4028234663852886e38;
    c->norm = float(norm);
    c->apply = finite;
    c->factor = float(a.max_norm > 0 && norm > a.max_norm ? a.grad_scale * (a.max_norm / norm) : a.grad_scale);
    if (finite) {
        const uint32_t step = c->step + 1;
        c->step = step;
        c->bias1 = 1 / (1 - power(a.beta1, step));
        c->bias2 = 1 / sqrt(1 - power(a.beta2, step));
    } else {
        c->skipped += 1;
    }
}

// ------------------------------------------------------------------ AdamW

struct StepArgs {
    const TensorDev *rows;
    const ChunkDev *chunks;
    const tagc_optim_control *control;  // NULL: the three below
    double bias1, bias2;
    uint32_t step;
    float factor;
    float beta1, beta2, rest1, rest2, eps;  // rest = 1 - beta, rounded once
    uint64_t seed;
    double lr[TAGC_MAX_GROUPS], weight_decay[TAGC_MAX_GROUPS];
};

// What is the same for a workgroup's elements.
struct Hyper {
    float factor, beta1, beta2, rest1, rest2, eps, decay, size, bias2;
};

// m, v and p of one element after the step.  Products and sums are rounded one by one (a product that
// went into a sum unrounded would make the 8-bit moments differ from what the formula gives in
// float32).
template <bool SMALL_EPS>
__device__ inline void adamw(const Hyper &h, float grad, float &m, float &v, float &p)
{
#pragma clang fp contract(off)
    const float g = grad * h.factor;
    m = m * h.beta1 + g * h.rest1;
    v = v * h.beta2 + (g * g) * h.rest2;
    // (root and reciprocal as the hardware has them, within an ulp each, where what they go into is more than a subnormal
    // number's root, which the hardware takes for 0: see small_eps)
    if constexpr (SMALL_EPS) p = p * h.decay - m / (sqrtf(v) * h.bias2 + h.eps) * h.size;
    else p = p * h.decay - m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v) * h.bias2 + h.eps) * h.size;
}

// Bound by bytes: 151 M elements in float32 (28 bytes each) take 713 us, 5.9 TB/s.  All loads of a thread, four times four
// neighbours of four arrays, go out before the first is used, and none is kept by the caches (with
// ordinary loads and stores 779 us).
template <typename P, typename G, bool SMALL_EPS>
__device__ inline void adamw32_chunk(const TensorDev &t, uint64_t at, const Hyper &h)
{
    const G *grad = as_global(static_cast<const G *>(t.grad));
    P *param = as_global(static_cast<P *>(t.param));
    float *mp = as_global(static_cast<float *>(t.m)), *vp = as_global(static_cast<float *>(t.v));
    uint16_t *copy = as_global(t.copy);
    const uint64_t n = t.length;
    float g[kSteps][4], p[kSteps][4], m[kSteps][4], v[kSteps][4];
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
        const uint64_t i = at + 4 * (k * kOptimThreads + threadIdx.x);
        load_f32(grad, i, n, g[k]);
        load_f32(mp, i, n, m[k]);
        load_f32(vp, i, n, v[k]);
        load_f32(param, i, n, p[k]);
    }
#pragma unroll
    for (uint32_t k = 0; k < kSteps; ++k) {
        const uint64_t i = at + 4 * (k * kOptimThreads + threadIdx.x);
        if (i >= n) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) adamw<SMALL_EPS>(h, g[k][j], m[k][j], v[k][j], p[k][j]);
        store_f32(mp, i, n, m[k]);
        store_f32(vp, i, n, v[k]);
        store_f32(param, i, n, p[k]);
        if (copy) store_f32(copy, i, n, p[k]);
    }
}

// Four codes from `i` on, the first in the low byte; zeros from `n` on.
__device__ inline uint32_t load_codes(const uint8_t *p, uint64_t i, uint64_t n)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (i + 4 <= n) return __builtin_nontemporal_load(reinterpret_cast<const word *>(p + i));
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) c |= uint32_t(p[i + j]) << (8 * j);
    return c;
}
__device__ inline void store_codes(uint8_t *p, uint64_t i, uint64_t n, uint32_t c)
{
    typedef uint32_t word __attribute__((aligned(1)));
    if (i + 4 <= n) {
        __builtin_nontemporal_store(c, reinterpret_cast<word *>(p + i));
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) p[i + j] = uint8_t(c >> (8 * j));
}

// float32 bits of a code's magnitude under a base
__device__ inline uint32_t code_bits(uint32_t c, uint32_t base) { return c ? (c + base) << 20 : 0; }

// (bits + 16 u) >> 20 of a magnitude; what is finite stays finite, what is not stays that
__device__ inline uint32_t rounded(uint32_t bits, uint32_t u)
{
    const uint32_t q = (bits + 16 * u) >> 20, most = bits >> 20;
    return min(q, most > 0x7F7u ? most : 0x7F7u);
}

// Two 16-bit numbers' largest over a wave, each for itself, by the VALU alone.
__device__ inline uint32_t max2(uint32_t a, uint32_t b)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <int CTRL>
__device__ inline uint32_t max2_from(uint32_t x)
{
    return max2(x, uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, true)));
}
__device__ inline uint32_t wave_max2(uint32_t x)
{
    x = max2_from<0x111>(x);  // row_shr:1, 2, 4, 8: a row's last lane has the row's
    x = max2_from<0x112>(x);
    x = max2_from<0x114>(x);
    x = max2_from<0x118>(x);
    x = max2_from<0x142>(x);  // row_bcast:15, 31: the last lane has the wave's
    x = max2_from<0x143>(x);
    return uint32_t(__builtin_amdgcn_readlane(int(x), 63));
}

// whether one of a word's bytes is 0
__device__ inline bool zero_byte(uint32_t x) { return ((x - 0x01010101u) & ~x & 0x80808080u) != 0; }

// A wave's step is a block: its 64 lanes hold four neighbours each, and the base takes one maximum over the wave.
//
// Bound by bytes where weights are float32 (202 M with bfloat16 gradients and copies, 16 bytes each, 540 us, 6.0 TB/s), by
// the VALU where they are not (10 bytes each, 363 us, 5.6 TB/s): some 50 instructions an element, after root and
// reciprocal by the hardware (659 -> 587 us, 535 -> 464), the maximum of both moments at once without local memory, and
// what is seldom behind branches (587 -> 549, 464 -> 401).
template <typename P, typename G, bool SMALL_EPS>
__device__ inline void adamw8_chunk(const TensorDev &t, uint64_t at, const Hyper &h, uint32_t key)
{
    const G *grad = as_global(static_cast<const G *>(t.grad));
    P *param = as_global(static_cast<P *>(t.param));
    uint8_t *mp = as_global(static_cast<uint8_t *>(t.m)), *vp = as_global(static_cast<uint8_t *>(t.v));
    uint32_t *bases = as_global(t.bases);
    uint16_t *copy = as_global(t.copy);
    const uint64_t n = t.length;
    float g[kCodeSteps][4], p[kCodeSteps][4];
    uint32_t mc[kCodeSteps], vc[kCodeSteps], base[kCodeSteps];
#pragma unroll
    for (uint32_t k = 0; k < kCodeSteps; ++k) {
        const uint64_t i = at + 4 * (k * kCodeThreads + threadIdx.x);
        const uint64_t block = i / TAGC_MOMENT_BLOCK;
        base[k] = block * TAGC_MOMENT_BLOCK < n ? bases[block] : 0;
        mc[k] = load_codes(mp, i, n);
        vc[k] = load_codes(vp, i, n);
        load_f32(grad, i, n, g[k]);
        load_f32(param, i, n, p[k]);
    }
#pragma unroll
    for (uint32_t k = 0; k < kCodeSteps; ++k) {
        const uint64_t i = at + 4 * (k * kCodeThreads + threadIdx.x);
        const uint64_t block = i / TAGC_MOMENT_BLOCK;
        if (block * TAGC_MOMENT_BLOCK >= n) break;  // (the same for a whole wave)
        const uint32_t word = mix32(uint32_t(i / 4) ^ key), base_m = base[k] & 0xFFFF, base_v = base[k] >> 16;
        float m[4], v[4];
        uint32_t u[4], bits_m[4], bits_v[4], q[4], most = 0;
        // Codes of 0, numbers that are not finite and numbers far under the block's largest are seldom: what they
        // take is a branch that whole waves go past.
        const bool zeros = zero_byte(mc[k] & 0x7F7F7F7Fu) | zero_byte(vc[k]);
        if (__builtin_expect(__any(zeros), 0)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = (mc[k] >> (8 * j)) & 0xFF, d = (vc[k] >> (8 * j)) & 0xFF;
                m[j] = __uint_as_float(code_bits(c & 127, base_m) | (c & 128) << 24);
                v[j] = __uint_as_float(code_bits(d, base_v));
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = (mc[k] >> (8 * j)) & 0xFF, d = (vc[k] >> (8 * j)) & 0xFF;
                m[j] = __uint_as_float(((c & 127) + base_m) << 20 | (c & 128) << 24);
                v[j] = __uint_as_float((d + base_v) << 20);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            adamw<SMALL_EPS>(h, g[k][j], m[j], v[j], p[k][j]);
            u[j] = j ? (word >> (8 * j)) | (word << (32 - 8 * j)) : word;
            bits_m[j] = __float_as_uint(m[j]);
            bits_v[j] = __float_as_uint(v[j]);
            q[j] = ((bits_m[j] & 0x7FFFFFFFu) + (u[j] & 0xFFFF) * 16) >> 20 | ((bits_v[j] & 0x7FFFFFFFu) + (u[j] >> 16) * 16) >> 20 << 16;
            most = max2(most, q[j]);
        }
        most = wave_max2(most);
        uint32_t new_m = 0, new_v = 0, bm = max(most & 0xFFFF, 127u) - 127, bv = max(most >> 16, 255u) - 255;
        bool low = false;
#pragma unroll
        for (int j = 0; j < 4; ++j) low |= (q[j] & 0xFFFF) <= bm || q[j] >> 16 <= bv;
        if (__builtin_expect((most & 0xFFFF) < 0x7F8 && most >> 16 < 0x7F8 && !__any(low), 1)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                new_m |= ((q[j] & 0xFFFF) - bm | (bits_m[j] >> 24 & 128)) << (8 * j);
                new_v |= ((q[j] >> 16) - bv) << (8 * j);
            }
        } else {
            uint32_t qm[4], qv[4];
            most = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                qm[j] = rounded(bits_m[j] & 0x7FFFFFFFu, u[j] & 0xFFFF);
                qv[j] = rounded(bits_v[j] & 0x7FFFFFFFu, u[j] >> 16);
                most = max2(most, qm[j] | qv[j] << 16);
            }
            most = wave_max2(most);
            bm = max(most & 0xFFFF, 127u) - 127;
            bv = max(most >> 16, 255u) - 255;
            const float least = __uint_as_float((bm + 1) << 20);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t low_m = float(u[j] & 0xFFFF) * 0x1p-16f * least < fabsf(m[j]), low_v = v[j] > 0;
                new_m |= ((qm[j] > bm ? qm[j] - bm : low_m) | (m[j] < 0 ? 128u : 0u)) << (8 * j);
                new_v |= (qv[j] > bv ? qv[j] - bv : low_v) << (8 * j);
            }
        }
        if (i < n) {
            store_codes(mp, i, n, new_m);
            store_codes(vp, i, n, new_v);
            store_f32(param, i, n, p[k]);
            if (copy) store_f32(copy, i, n, p[k]);
        }
        if ((threadIdx.x & 63) == 0) bases[block] = bm | bv << 16;
    }
}

template <int BITS, bool SMALL_EPS>
__global__ __launch_bounds__(BITS == 32 ? kOptimThreads : kCodeThreads) void adamw_kernel(StepArgs a)
{
    const ChunkDev ch = a.chunks[blockIdx.x];
    const TensorDev &t = a.rows[ch.tensor];
    uint32_t step = a.step;
    Hyper h{a.factor, a.beta1, a.beta2, a.rest1, a.rest2, a.eps, 0, 0, 0};
    double bias1 = a.bias1, bias2 = a.bias2, lr = a.lr[t.group];
    if (a.control) {
        if (!a.control->apply) return;
        step = a.control->step;
        h.factor = a.control->factor;
        bias1 = a.control->bias1;
        bias2 = a.control->bias2;
        lr *= a.control->lr_scale;
    }
    h.decay = float(1 - lr * a.weight_decay[t.group]);
    h.size = float(lr * bias1);
    h.bias2 = float(bias2);
    const uint64_t at = uint64_t(ch.chunk) * kChunk;
    if constexpr (BITS == 32) {
        switch (t.types) {
            case 0: return adamw32_chunk<float, float, SMALL_EPS>(t, at, h);
            case kParamBf16: return adamw32_chunk<uint16_t, float, SMALL_EPS>(t, at, h);
            case kGradBf16: return adamw32_chunk<float, uint16_t, SMALL_EPS>(t, at, h);
            default: return adamw32_chunk<uint16_t, uint16_t, SMALL_EPS>(t, at, h);
        }
    } else {
        const uint32_t key = mix32(ch.tensor * 0x9E3779B9u + seed_word(a.seed, step));
        switch (t.types) {
            case 0: return adamw8_chunk<float, float, SMALL_EPS>(t, at, h, key);
            case kParamBf16: return adamw8_chunk<uint16_t, float, SMALL_EPS>(t, at, h, key);
            case kGradBf16: return adamw8_chunk<float, uint16_t, SMALL_EPS>(t, at, h, key);
            default: return adamw8_chunk<uint16_t, uint16_t, SMALL_EPS>(t, at, h, key);
        }
    }
}

// A code's bfloat16: the upper half of (base + c) << 20, and the sign.
__global__ __launch_bounds__(kCodeThreads) void unpack_kernel(const TensorDev *rows, const ChunkDev *chunks,
                                                               uint16_t *m_out, uint16_t *v_out)
{
    const ChunkDev ch = chunks[blockIdx.x];
    const TensorDev &t = rows[ch.tensor];
    const uint8_t *mp = as_global(static_cast<const uint8_t *>(t.m)), *vp = as_global(static_cast<const uint8_t *>(t.v));
    const uint32_t *bases = as_global(t.bases);
    const uint64_t n = t.length;
    uint16_t *mo = m_out + t.first, *vo = v_out + t.first;
    uint32_t mc[kCodeSteps], vc[kCodeSteps], base[kCodeSteps];
#pragma unroll
    for (uint32_t k = 0; k < kCodeSteps; ++k) {
        const uint64_t i = uint64_t(ch.chunk) * kChunk + 4 * (k * kCodeThreads + threadIdx.x);
        base[k] = i < n ? bases[i / TAGC_MOMENT_BLOCK] : 0;
        mc[k] = load_codes(mp, i, n);
        vc[k] = load_codes(vp, i, n);
    }
#pragma unroll
    for (uint32_t k = 0; k < kCodeSteps; ++k) {
        const uint64_t i = uint64_t(ch.chunk) * kChunk + 4 * (k * kCodeThreads + threadIdx.x);
        uint16_t m[4], v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t c = (mc[k] >> (8 * j)) & 0xFF, d = (vc[k] >> (8 * j)) & 0xFF;
            m[j] = uint16_t(code_bits(c & 127, base[k] & 0xFFFF) >> 16 | (c & 128) << 8);
            v[j] = uint16_t(code_bits(d, base[k] >> 16) >> 16);
        }
        if (i + 4 <= n) {
            store4(mo + i, m);
            store4(vo + i, v);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i + j >= n) continue;
                mo[i + j] = m[j];
                vo[i + j] = v[j];
            }
        }
    }
}

bool aligned(const void *p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
uint64_t type_bytes(uint32_t type) { return type == TAGC_F32 ? 4 : 2; }

// Whether the update's denominator, sqrt(v) / sqrt(1 - beta2^t) + eps, can be changed by more than a rounding, 2^-24, where a subnormal
// v, whose root is 2^-63 at most, is taken for 0; the first root's divisor is sqrt(1 - beta2) at least.  Then root and quotient
// are IEEE's.  (An eps of 1e-8 is small for a beta2 from 1 - 3.3e-8 on only.)
bool small_eps(const tagc_optim_config &cfg) { return cfg.eps * sqrt(1 - cfg.beta2) < 0x1p-39; }

// one tensor's pointers and fields
int check_tensor(const tagc_optim_config &cfg, const tagc_tensor &t)
{
    if (t.param_type > TAGC_BF16 || t.grad_type > TAGC_BF16 || t.group >= TAGC_MAX_GROUPS || t.reserved) return TAGC_EINVAL;
    if (t.length >= kMaxLength) return TAGC_ESIZE;
    if (!t.length) return TAGC_OK;
    if (!t.grad || !aligned(t.grad, type_bytes(t.grad_type))) return TAGC_EINVAL;
    if (!t.param) return t.m || t.v || t.bases || t.copy ? TAGC_EINVAL : TAGC_OK;
    const uint64_t moment = cfg.moment_bits / 8;
    if (!aligned(t.param, type_bytes(t.param_type)) || !t.m || !t.v || !aligned(t.m, moment) || !aligned(t.v, moment) ||
        !aligned(t.copy, 2) || !aligned(t.bases, 4))
        return TAGC_EINVAL;
    return (t.bases != nullptr) == (cfg.moment_bits == 8) ? TAGC_OK : TAGC_EINVAL;
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_optim_plan(const tagc_optim_config *cfg, const tagc_tensor *tensors, uint32_t n_tensors,
                               tagc_optim_t **out)
{
    if (!cfg || !out || (n_tensors && !tensors)) return TAGC_EINVAL;
    *out = nullptr;
    if (!(cfg->beta1 >= 0 && cfg->beta1 < 1) || !(cfg->beta2 >= 0 && cfg->beta2 < 1) || !(cfg->eps >= 0 && cfg->eps <= 1e30) ||
        !(cfg->grad_scale > 0 && cfg->grad_scale <= 1e30) || !(cfg->max_norm >= 0 && cfg->max_norm <= 1e30) ||
        (cfg->moment_bits != 32 && cfg->moment_bits != 8) || cfg->reserved)
        return TAGC_EINVAL;
    tagc_optim_t *p = new (std::nothrow) tagc_optim_s();
    if (!p) return TAGC_ENOMEM;
    p->cfg = *cfg;
    p->has_params = true;
    int rc = TAGC_OK;
    try {
        uint64_t chunks = 0, most = kMaxChunks;
        for (uint32_t i = 0; i < n_tensors && !rc; ++i) {
            rc = check_tensor(*cfg, tensors[i]);
            chunks += (tensors[i].length + kChunk - 1) / kChunk;
            if (tensors[i].param && cfg->moment_bits == 8) most = kMaxCodeChunks;
            if (!rc && chunks >= most) rc = TAGC_ESIZE;
        }
        if (rc) {
            delete p;
            return rc;
        }
        p->rows.reserve(n_tensors);
        p->chunks.reserve(chunks);
        for (uint32_t i = 0; i < n_tensors; ++i) {
            const tagc_tensor &t = tensors[i];
            TensorDev d{};
            d.param = t.param;
            d.grad = t.grad;
            d.m = t.m;
            d.v = t.v;
            d.bases = t.bases;
            d.copy = static_cast<uint16_t *>(t.copy);
            d.length = t.length;
            d.first = p->sizes.n_elems;
            d.types = (t.param_type == TAGC_BF16 ? kParamBf16 : 0) | (t.grad_type == TAGC_BF16 ? kGradBf16 : 0);
            d.group = t.group;
            p->rows.push_back(d);
            for (uint64_t c = 0; c * kChunk < t.length; ++c) p->chunks.push_back({i, uint32_t(c)});
            p->sizes.n_elems += t.length;
            p->sizes.n_blocks += (t.length + TAGC_MOMENT_BLOCK - 1) / TAGC_MOMENT_BLOCK;
            if (t.length && !t.param) p->has_params = false;
            if (t.length && t.group >= p->n_groups) p->n_groups = t.group + 1;
        }
    } catch (const std::exception &) {
        delete p;
        return TAGC_ENOMEM;
    }
    p->sizes.n_chunks = p->chunks.size();
    p->sizes.table_bytes = p->state_at() + kArriveBytes + 8 * kNormGroups;
    *out = p;
    return TAGC_OK;
}

extern "C" void tagc_optim_destroy(tagc_optim_t *p) { delete p; }

extern "C" int tagc_optim_plan_sizes(const tagc_optim_t *p, tagc_optim_sizes *out)
{
    if (!p || !out) return TAGC_EINVAL;
    *out = p->sizes;
    return TAGC_OK;
}

extern "C" int tagc_optim_upload(const tagc_optim_t *p, void *table, void *stream)
{
    if (!p || !table || !aligned(table, 16)) return TAGC_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char *t = static_cast<char *>(table);
    if (!p->rows.empty() &&
        hipMemcpyAsync(t, p->rows.data(), p->rows.size() * sizeof(TensorDev), hipMemcpyHostToDevice, s) != hipSuccess)
        return TAGC_EHIP;
    if (!p->chunks.empty() && hipMemcpyAsync(t + p->chunks_at(), p->chunks.data(), p->chunks.size() * sizeof(ChunkDev),
                                             hipMemcpyHostToDevice, s) != hipSuccess)
        return TAGC_EHIP;
    return hip_ok(hipMemsetAsync(t + p->state_at(), 0, kArriveBytes, s));
}

extern "C" int tagc_grad_norm(const tagc_optim_t *p, void *table, tagc_optim_control *control, void *stream)
{
    if (!p || !table || !aligned(table, 16) || !control || !aligned(control, 16)) return TAGC_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    char *t = static_cast<char *>(table);
    NormArgs a;
    a.rows = reinterpret_cast<const TensorDev *>(t);
    a.chunks = reinterpret_cast<const ChunkDev *>(t + p->chunks_at());
    a.arrived = reinterpret_cast<uint32_t *>(t + p->state_at());
    a.partial = reinterpret_cast<uint64_t *>(t + p->state_at() + kArriveBytes);
    a.control = control;
    a.grad_scale = p->cfg.grad_scale;
    a.max_norm = p->cfg.max_norm;
    a.beta1 = p->cfg.beta1;
    a.beta2 = p->cfg.beta2;
    a.n_chunks = uint32_t(p->chunks.size());
    uint32_t grid = uint32_t(device_cu_count()) * 8;
    if (grid > kNormGroups) grid = kNormGroups;
    if (grid > a.n_chunks) grid = a.n_chunks ? a.n_chunks : 1;
    ProfileScope prof("grad_norm", s);
    norm_kernel<<<grid, kOptimThreads, 0, s>>>(a);
    return hip_ok(hipGetLastError());
}

extern "C" int tagc_adamw_step(const tagc_optim_t *p, const void *table, const tagc_group *groups, uint32_t n_groups,
                               uint32_t step, const tagc_optim_control *control, void *stream)
{
    if (!p || !table || !aligned(table, 16) || (n_groups && !groups) || n_groups > TAGC_MAX_GROUPS || n_groups < p->n_groups ||
        !p->has_params || (!step && (!control || !aligned(control, 16))))
        return TAGC_EINVAL;
    for (uint32_t i = 0; i < n_groups; ++i)
        if (!isfinite(groups[i].lr) || !isfinite(groups[i].weight_decay)) return TAGC_EINVAL;
    if (p->chunks.empty()) return TAGC_OK;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const char *t = static_cast<const char *>(table);
    StepArgs a{};
    a.rows = reinterpret_cast<const TensorDev *>(t);
    a.chunks = reinterpret_cast<const ChunkDev *>(t + p->chunks_at());
    a.control = step ? nullptr : control;
    a.step = step;
    if (step) {
        a.bias1 = 1 / (1 - pow(p->cfg.beta1, double(step)));
        a.bias2 = 1 / sqrt(1 - pow(p->cfg.beta2, double(step)));
    }
    a.factor = float(p->cfg.grad_scale);
    a.beta1 = float(p->cfg.beta1);
    a.beta2 = float(p->cfg.beta2);
    a.rest1 = float(1 - p->cfg.beta1);
    a.rest2 = float(1 - p->cfg.beta2);
    a.eps = float(p->cfg.eps);
    a.seed = p->cfg.seed;
    for (uint32_t i = 0; i < n_groups; ++i) {
        a.lr[i] = groups[i].lr;
        a.weight_decay[i] = groups[i].weight_decay;
    }
    const uint32_t grid = uint32_t(p->chunks.size());
    if (p->cfg.moment_bits == 32) {
        ProfileScope prof("adamw32", s);
        if (small_eps(p->cfg)) adamw_kernel<32, true><<<grid, kOptimThreads, 0, s>>>(a);
        else adamw_kernel<32, false><<<grid, kOptimThreads, 0, s>>>(a);
    } else {
        ProfileScope prof("adamw8", s);
        if (small_eps(p->cfg)) adamw_kernel<8, true><<<grid, kCodeThreads, 0, s>>>(a);
        else adamw_kernel<8, false><<<grid, kCodeThreads, 0, s>>>(a);
    }
    return hip_ok(hipGetLastError());
}

extern "C" int tagc_adamw_unpack(const tagc_optim_t *p, const void *table, void *m_out, void *v_out, void *stream)
{
    if (!p || !table || !aligned(table, 16) || !p->has_params) return TAGC_EINVAL;
    if (p->cfg.moment_bits != 8) return TAGC_EUNSUPPORTED;
    if (p->chunks.empty()) return TAGC_OK;
    if (!m_out || !v_out || !aligned(m_out, 2) || !aligned(v_out, 2)) return TAGC_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const char *t = static_cast<const char *>(table);
    ProfileScope prof("adamw_unpack", s);
    unpack_kernel<<<uint32_t(p->chunks.size()), kCodeThreads, 0, s>>>(
        reinterpret_cast<const TensorDev *>(t), reinterpret_cast<const ChunkDev *>(t + p->chunks_at()),
        static_cast<uint16_t *>(m_out), static_cast<uint16_t *>(v_out));
    return hip_ok(hipGetLastError());
}
