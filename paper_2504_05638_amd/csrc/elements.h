// What the training kernels share: elements and rows of both types in registers, workspaces, and matrices as the host
// sees them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tagc_train.h"

namespace tagc {

namespace {

constexpr uint64_t kMaxSide = 1u << 22;  // rows, features (in float32 a quarter) and strides as they lie are fewer

inline uint64_t up(uint64_t a, uint64_t b) { return (a + b - 1) / b * b; }

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
// ------------------------------------------------------------------ host

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

inline bool aligned_to(const void *p, uint64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// a matrix that must or may be there
inline bool good(const void *p, uint64_t ld, uint64_t cols, uint64_t bytes) { return !p || (aligned_to(p, bytes) && ld >= cols && ld < (1ull << 40)); }

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
inline bool meet(const Rows &a, const Rows &b)
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

}  // namespace

}  // namespace tagc
