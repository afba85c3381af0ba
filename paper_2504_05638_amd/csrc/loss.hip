// Losses over a vocabulary, and their gradients, without the scores.
//
//   s = x w^T / T,  lse = log of the sum of e^s;  loss = sum over a row's terms of q (log q - s + lse)
//   ds = dloss (e^(s - lse) - q) / T;  dx = ds w,  dw = ds^T x
//
// Forward, the scores stay in the registers of the product that makes them: of every row a wave leaves its columns' largest score
// and the sum of exponentials against it, and these are put together when the product is done.  Terms' own scores
// are taken from there, too.  Backward, the product is made again, a piece of the vocabulary at a time, and ends in ds of that piece,
// which the two products behind it read; the terms' few elements are put right between them.  What is held of a piece is bounded, whatever the
// vocabulary.
//
// Rows without a term take no part: the others are laid out one behind the other, and how many there are is a number on the
// device that cuts the products short.
#include <math.h>

#include "product.h"
#include "tagc_train.h"

namespace tagc {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f, kLeast = 1.17549435e-38f;

// Up to so many rows and scores, these are held between the product and what becomes of them.  (us, held / not: bfloat16 1 row of 4096 over 32000 54 / 80,
// 128 rows 72 / 83, 512 rows 144 / 133; 333 of 777 over 1001 21 / 27, in float32 24 / 49; 4096 rows of 256 over 2048 35 / 28.)
constexpr uint64_t kHeldRows = 1024, kHeld = 1u << 23;

// Terms of a row from which on they are listed by strips: few are found sooner than a launch makes lists.
constexpr uint32_t kListTerms = 5;

// Elements up to which a vocabulary that is one piece is laid out in the launch that lays out x.  (us, backward, so / by a launch of its own: float32
// 26 rows of 863 over 1977 49 / 52, bfloat16 1200 of 777 over 8001 91 / 95; float32 1024 of 1024 over 32000 1065 / 1068.)
constexpr uint64_t kAtOnce = 1u << 26;

// What a piece of the vocabulary may hold (ds, operands laid out, the waves' sums), and its fewest rows.  (us, a quarter / a half / one GiB, backward in
// bfloat16: 8192 rows of 768 over 50257 2613 / 2317 / 2170, of 4096 over 32000 5314 / 5251 / 5256, over 128256 21161 / 20707 / 20662: dx of narrow
// rows has few tiles, and more parts the longer its sums are; float32, a quarter / a half: 1024 of 768 over 50257 1202 / 1235, 2048 of 4096 over 32000
// 7575 / 7215.)
constexpr uint64_t kPieceBytes = 512ull << 20, kPieceRows = 1024;

// ------------------------------------------------------------------ terms and rows

__device__ inline uint32_t id_at(const void *ids, uint32_t wide, uint64_t at, uint32_t vocab)
{
    const uint64_t id = wide ? static_cast<const uint64_t *>(ids)[at] : uint64_t(int64_t(static_cast<const int32_t *>(ids)[at]));
    return id < vocab ? uint32_t(id) : vocab;
}

struct Terms {
    const void *ids;
    const float *logits;
    float *q;        // [rows, terms] with logits: a term's share, 0 for none
    uint8_t *any;    // [rows] with logits: whether a row has a term
    uint32_t rows, terms, vocab, wide;
    float over;      // 1 / temperature
};

__device__ inline float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

// A teacher's shares, a row to a wave.  (Logits are divided by the temperature once the largest is taken from them: a row whose
// logits are all the type's lowest value, some masks' mark, has shares alike.)
__global__ __launch_bounds__(256) void terms_kernel(Terms a)
{
    const uint64_t row = uint64_t(blockIdx.x) * 4 + threadIdx.x / 64;
    if (row >= a.rows) return;
    const uint32_t lane = threadIdx.x & 63;
    const float *logits = a.logits + row * a.terms;
    const float over2 = a.over * kLog2e;
    float top = -INFINITY, sum = 0;
    bool any = false;
    for (uint32_t k = lane; k < a.terms; k += 64) {
        const float x = logits[k];
        if (id_at(a.ids, a.wide, row * a.terms + k, a.vocab) == a.vocab || x == -INFINITY) continue;
        any = true;
        top = fmaxf(top, x);
    }
    top = wave_max(top);
    if (top == -INFINITY) top = 0;  // (all there is is NaN)
    for (uint32_t k = lane; k < a.terms; k += 64) {
        const float x = logits[k];
        if (id_at(a.ids, a.wide, row * a.terms + k, a.vocab) == a.vocab || x == -INFINITY) continue;
        sum += __builtin_amdgcn_exp2f((x - top) * over2);
    }
    sum = wave_sum(sum);
    for (uint32_t k = lane; k < a.terms; k += 64) {
        const float x = logits[k];
        const bool none = id_at(a.ids, a.wide, row * a.terms + k, a.vocab) == a.vocab || x == -INFINITY;
        float q = __builtin_amdgcn_exp2f((x - top) * over2) / sum;
        if (q < kLeast) q = kLeast;  // (a term, if one that does not count: its score is saved)
        a.q[row * a.terms + k] = none ? 0.0f : q;
    }
    any = __any(any);
    if (lane == 0) a.any[row] = any;
}

// A row's weight of a term, 0 for none.
__device__ inline float share(const Terms &a, uint64_t at, uint32_t id) { return a.q ? a.q[at] : id < a.vocab ? 1.0f : 0.0f; }

struct List {
    uint32_t *rows;   // those with a term in order, then the others
    uint32_t *count;  // of the first
};

__device__ inline bool has_term(const Terms &a, uint32_t row) { return a.logits ? a.any[row] != 0 : id_at(a.ids, a.wide, row, a.vocab) < a.vocab; }

constexpr uint32_t kListThreads = 1024, kListEach = 8;
__global__ __launch_bounds__(kListThreads) void list_kernel(Terms a, List l)
{
    __shared__ uint32_t room[kListThreads / 64];
    uint32_t done = 0;
    for (uint32_t first = 0; first < a.rows; first += kListThreads * kListEach) {
        const uint32_t from = first + threadIdx.x * kListEach;
        uint32_t bits = 0;
#pragma unroll
        for (uint32_t i = 0; i < kListEach; ++i)
            if (from + i < a.rows) bits |= uint32_t(has_term(a, from + i)) << i;
        uint32_t total;
        uint32_t at = done + block_excl_scan<uint32_t, kListThreads / 64>(__popc(bits), &total, room);
#pragma unroll
        for (uint32_t i = 0; i < kListEach; ++i) {
            const uint32_t row = from + i;
            if (row >= a.rows) break;
            if (!(bits >> i & 1)) {
                l.rows[a.rows - 1 - (row - at)] = row;  // (row - at: those without a term before it)
                continue;
            }
            l.rows[at++] = row;
        }
        done += total;
    }
    if (threadIdx.x == 0) *l.count = done;
}

// ------------------------------------------------------------------ operands laid out

struct Gather {
    const void *src;  // rows of `cols`, ld elements apart
    void *to;
    uint64_t ld, to_ld;
    uint32_t n, cols, part;  // part: float32 taken apart, elements from one part to the next; 0: as they are
    uint32_t across;         // pieces of eight elements to a row, zeros behind cols
};

template <typename T>
__device__ inline void lay_piece(const Gather &a, uint32_t from, uint32_t r, uint32_t c)
{
    const T *src = static_cast<const T *>(a.src) + from * a.ld + c;
    float x[8];
    if (c + 8 <= a.cols) {
        load_n<T, 8>(src, x);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) x[j] = c + j < a.cols ? widen(src[j]) : 0.0f;
    }
    if (sizeof(T) == 4 && a.part) {
        uint16_t *to = static_cast<uint16_t *>(a.to) + r * a.to_ld + c;
        u32x4 out[kParts];
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            uint32_t s[2][kParts];
            split(x[2 * j], s[0]);
            split(x[2 * j + 1], s[1]);
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q) out[q][j] = __builtin_amdgcn_perm(s[1][q], s[0][q], 0x07060302);
        }
#pragma unroll
        for (uint32_t q = 0; q < kParts; ++q) *reinterpret_cast<u32x4 *>(to + q * a.part) = out[q];
    } else {
        store_n<T, 8>(static_cast<T *>(a.to) + r * a.to_ld + c, x);
    }
}

template <typename T>
__device__ inline void lay_all(const Gather &a, uint32_t group)
{
    const uint64_t i = uint64_t(group) * 256 + threadIdx.x;
    const uint32_t r = uint32_t(i / a.across);
    if (r < a.n) lay_piece<T>(a, r, r, uint32_t(i % a.across) * 8);
}
template <typename T>
__global__ __launch_bounds__(256) void gather_kernel(Gather a)
{
    lay_all<T>(a, blockIdx.x);
}

// The rows that have a term, one behind the other: x's, their terms' ids, and what the backward pass needs of each.
struct Lay {
    Terms terms;
    List list;
    Gather x;
    uint32_t groups;   // workgroups for x; those behind them are for ids
    Gather w;          // a vocabulary that is one piece
    uint32_t w_from;   // workgroups from there on are its
    uint32_t *ids;     // [rows][2^shift]: a row's terms, kNone for none
    uint32_t shift;
    const float *saved, *dloss;
    float2 *row;       // backward: of a row the log2 of its sum of exponentials, and dloss / temperature
    uint32_t step;
};
constexpr uint32_t kNone = 0xFFFFFFFFu;

// SCAN: up to 1024 rows' list is made here, by each workgroup for itself: a launch less.
constexpr uint32_t kScanRows = 1024;
template <typename T, bool SCAN>
__global__ __launch_bounds__(256) void lay_kernel(Lay a)
{
    __shared__ uint32_t rows[SCAN ? kScanRows : 1], room[4];
    if (blockIdx.x >= a.w_from) return lay_all<T>(a.w, blockIdx.x - a.w_from);
    uint32_t count;
    if constexpr (SCAN) {
        uint32_t bits = 0;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
            if (threadIdx.x * 4 + i < a.terms.rows) bits |= uint32_t(has_term(a.terms, threadIdx.x * 4 + i)) << i;
        uint32_t at = block_excl_scan<uint32_t, 4>(__popc(bits), &count, room);
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const uint32_t row = threadIdx.x * 4 + i;
            if (row >= a.terms.rows) break;
            const uint32_t to = bits >> i & 1 ? at++ : a.terms.rows - 1 - (row - at);
            rows[to] = row;
            if (blockIdx.x == 0) a.list.rows[to] = row;
        }
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.list.count = count;
        __syncthreads();
    } else {
        count = *a.list.count;
    }
    const auto row_at = [&](uint32_t r) { return SCAN ? rows[r] : a.list.rows[r]; };
    if (blockIdx.x < a.groups) {
        const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
        const uint32_t r = uint32_t(i / a.x.across);
        if (r < count) lay_piece<T>(a.x, row_at(r), r, uint32_t(i % a.x.across) * 8);
        return;
    }
    const uint64_t i = uint64_t(blockIdx.x - a.groups) * 256 + threadIdx.x;
    const uint32_t r = uint32_t(i >> a.shift), k = uint32_t(i) & ((1u << a.shift) - 1);
    if (r >= count) return;
    const uint32_t row = row_at(r);
    uint32_t id = kNone;
    if (k < a.terms.terms) {
        const uint64_t at = uint64_t(row) * a.terms.terms + k;
        id = id_at(a.terms.ids, a.terms.wide, at, a.terms.vocab);
        if (id == a.terms.vocab || share(a.terms, at, id) == 0) id = kNone;
    }
    a.ids[i] = id;
    if (a.row && k == 0) a.row[r] = make_float2(a.saved[uint64_t(row) * (1 + a.terms.terms)] * kLog2e, a.dloss[uint64_t(row) * a.step] * a.terms.over);
}

// Many terms, by strips of 32 of the vocabulary's tokens: a workgroup counts and places those of 32 rows.  (Their order within a strip does not
// matter: each is copied to a place of its own.)
constexpr uint32_t kStripsRows = 32, kStrip = 32, kMostStrips = 8192;
struct Strips {
    uint32_t *starts;   // [groups of rows][strips + 1]: where the terms of a strip begin, NULL: there are no lists
    uint32_t *entries;  // row of the group << 20 | term << 10 | lowest ten bits of the id
    uint32_t strips;
};
__global__ __launch_bounds__(256) void strips_kernel(const uint32_t *ids, uint32_t shift, const uint32_t *count, Strips to)
{
    __shared__ uint32_t at[kMostStrips], room[4];
    const uint32_t first = blockIdx.x * kStripsRows;
    if (first >= *count) return;
    const uint32_t n = min(kStripsRows, *count - first) << shift, base = first << shift;
    for (uint32_t s = threadIdx.x; s < to.strips; s += 256) at[s] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += 256) {
        const uint32_t id = ids[base + i];
        if (id != kNone) atomicAdd(&at[id / kStrip], 1u);
    }
    __syncthreads();
    const uint32_t each = (to.strips + 255) / 256, from = min(threadIdx.x * each, to.strips), end = min(from + each, to.strips);
    uint32_t sum = 0, all;
    for (uint32_t s = from; s < end; ++s) sum += at[s];
    uint32_t place = block_excl_scan<uint32_t, 4>(sum, &all, room);
    uint32_t *starts = to.starts + uint64_t(blockIdx.x) * (to.strips + 1);
    for (uint32_t s = from; s < end; ++s) {
        const uint32_t have = at[s];
        at[s] = place;
        starts[s] = base + place;
        place += have;
    }
    if (threadIdx.x == 0) starts[to.strips] = base + all;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < n; i += 256) {
        const uint32_t id = ids[base + i];
        if (id != kNone) to.entries[base + atomicAdd(&at[id / kStrip], 1u)] = (i >> shift) << 20 | (i & ((1u << shift) - 1)) << 10 | (id & 1023);
    }
}

// ------------------------------------------------------------------ ends of the products

// A wave's sums in rows, eight neighbours at a time, by way of its strip: f(m, n, z) for rows under `rows` and columns, by eights, under
// `cols`.  (What f reads may be asked for 32 rows ahead; that won nothing.)
template <int RM, int RN, typename F>
__device__ inline __attribute__((always_inline)) void in_rows(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t rows,
                                                              uint32_t cols, F f)
{
    constexpr uint32_t kRow = RN * 16 + 4, across = RN * 2, lines = 64 / across;
    const uint32_t ln = lane % across * 8, n = n0 + ln;
#pragma unroll 1
    for (int i = 0; i < RM; i += 2) {
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
#pragma unroll
        for (uint32_t l = 0; l < 32 / lines; ++l) {
            if (m + l * lines >= rows || n >= cols) continue;
            float z[8];
#pragma unroll
            for (int h = 0; h < 8; h += 4) {
                const float4 v = *reinterpret_cast<const float4 *>(strip + (l * lines + lane / across) * kRow + ln + h);
                z[h] = v.x;
                z[h + 1] = v.y;
                z[h + 2] = v.z;
                z[h + 3] = v.w;
            }
            f(m + l * lines, n, z);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Forward: of a row's scores in a wave's columns the largest, and the sum of 2^(score - largest), scores times log2(e) / T; and those of
// its terms.  These come from lists by strips, or are looked for among the terms' ids, 32 rows at a time; where there is one the rows go
// through local memory.  (us, lists / looked for, the whole call over 32000 by 4096, 2048 rows of 8, 64, 128 terms: 448, 457, 462 / 461, 474, 503, of one
// term 442; 4096 rows of 768 over 50257, 64 terms: 381 / 445.  By themselves, as products of two rows each, 64 terms took 164.)
struct Scores : Counted {
    static constexpr bool kCounted = true;
    float2 *stats;  // [strips of columns][rows]
    uint32_t rows;
    float over2;    // log2(e) / T
    const uint32_t *ids;  // [rows][2^shift]
    float *scores;        // [rows][terms]
    uint32_t shift, terms, base;  // base: the id of the piece's first column
    float over;           // 1 / T
    Strips lists;         // of groups of 32 rows, pieces of whole strips
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t) const
    {
        if (lists.starts) listed_terms(acc, strip, lane, m0, n0);
        else searched_terms(acc, strip, lane, m0, n0);
        float2 *to = stats + uint64_t(n0 / (RN * 16)) * rows;
        const uint32_t c0 = n0 + 4 * (lane >> 4);
        const bool whole = n0 + RN * 16 <= n;
#pragma unroll
        for (int i = 0; i < RM; ++i) {
            const uint32_t row = m0 + i * 16 + (lane & 15);
            const float2 of = whole ? summed<true>(acc[i], c0) : summed<false>(acc[i], c0);
            if (lane < 16 && row < m) to[row] = of;
        }
    }
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void searched_terms(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0) const
    {
        constexpr uint32_t kRow = RN * 16 + 4, kQuads = 8;  // quads of ids on their way
        const uint32_t first = base + n0, quads = 32u << (shift - 2);
        // (rows that there are not have no ids)
        const uint4 *from = reinterpret_cast<const uint4 *>(ids + (uint64_t(m0) << shift));
        const auto quad = [&](uint32_t q) { return m0 + (q >> (shift - 2)) < m ? from[q] : make_uint4(kNone, kNone, kNone, kNone); };
        const auto in = [&](uint32_t id) { return id - first < RN * 16; };
        // (up to four terms a row: three of four waves have none)
        bool search = shift > 2;
        if (!search) {
            for (uint32_t q = lane; q < RM * 16; q += 64) {
                const uint4 id = quad(q);
                search = search || in(id.x) || in(id.y) || in(id.z) || in(id.w);
            }
            search = __any(search);
        }
#pragma unroll 1
        for (int i = search ? 0 : RM; i < RM; i += 2) {
            bool written = false;
            for (uint32_t at_quad = 0; at_quad < quads; at_quad += 64 * kQuads) {  // (all lanes, which write the strip together)
                const uint32_t q0 = at_quad + lane;
                uint4 id[kQuads];
                bool any = false;
#pragma unroll
                for (uint32_t b = 0; b < kQuads; ++b) id[b] = q0 + 64 * b < quads ? quad(q0 + 64 * b + i / 2 * quads) : make_uint4(kNone, kNone, kNone, kNone);
#pragma unroll
                for (uint32_t b = 0; b < kQuads; ++b) any = any || in(id[b].x) || in(id[b].y) || in(id[b].z) || in(id[b].w);
                if (!__any(any)) continue;
                if (!written) {
                    written = true;
#pragma unroll
                    for (int at = 0; at < RM; at += 2)
                        if (at == i)
#pragma unroll
                            for (int h = 0; h < 2; ++h)
#pragma unroll
                                for (int j = 0; j < RN; ++j)
                                    *reinterpret_cast<f32x4 *>(strip + (16 * h + (lane & 15)) * kRow + 16 * j + 4 * (lane >> 4)) = acc[at + h][j];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                }
#pragma unroll
                for (uint32_t b = 0; b < kQuads; ++b) {
                    const uint32_t q = q0 + 64 * b, r = q >> (shift - 2), k = (q << 2) & ((1u << shift) - 1);
                    float *to = scores + uint64_t(m0 + i * 16 + r) * terms + k;
                    if (in(id[b].x)) to[0] = strip[r * kRow + id[b].x - first] * over;
                    if (in(id[b].y)) to[1] = strip[r * kRow + id[b].y - first] * over;
                    if (in(id[b].z)) to[2] = strip[r * kRow + id[b].z - first] * over;
                    if (in(id[b].w)) to[3] = strip[r * kRow + id[b].w - first] * over;
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void listed_terms(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0) const
    {
        constexpr uint32_t kRow = RN * 16 + 4;
        static_assert(RN * 16 % kStrip == 0, "whole strips");
        if (n0 >= n) return;
        const uint32_t first = base + n0, s = first / kStrip, end_s = min(s + RN * 16 / kStrip, lists.strips);
#pragma unroll 1
        for (int i = 0; i < RM; i += 2) {
            if (m0 + i * 16 >= m) break;
            const uint32_t *starts = lists.starts + uint64_t((m0 + i * 16) / kStripsRows) * (lists.strips + 1);
            const uint32_t from = __builtin_amdgcn_readfirstlane(starts[s]), end = __builtin_amdgcn_readfirstlane(starts[end_s]);
            if (from == end) continue;
#pragma unroll
            for (int at = 0; at < RM; at += 2)
                if (at == i)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < RN; ++j)
                            *reinterpret_cast<f32x4 *>(strip + (16 * h + (lane & 15)) * kRow + 16 * j + 4 * (lane >> 4)) = acc[at + h][j];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            for (uint32_t e = from + lane; e < end; e += 64) {
                const uint32_t entry = lists.entries[e], r = entry >> 20, k = entry >> 10 & 1023, c = (entry - first) & 1023;
                scores[uint64_t(m0 + i * 16 + r) * terms + k] = strip[r * kRow + c] * over;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    // of a row's scores in columns c0 + 16 j + (0 .. 3) of four lanes; WHOLE: all these columns are there
    template <bool WHOLE, int RN>
    __device__ inline float2 summed(const f32x4 (&row)[RN], uint32_t c0) const
    {
        float top = -INFINITY, sum = 0;
#pragma unroll
        for (int j = 0; j < RN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (WHOLE || c0 + 16 * j + e < n) top = fmaxf(top, row[j][e]);
        top *= over2;
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float against = top == -INFINITY ? 0.0f : top;  // (no column, or nothing but -infinity and NaN)
#pragma unroll
        for (int j = 0; j < RN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (WHOLE || c0 + 16 * j + e < n) sum += __builtin_amdgcn_exp2f(row[j][e] * over2 - against);
        sum += __shfl_xor(sum, 16, 64);
        sum += __shfl_xor(sum, 32, 64);
        return make_float2(top, sum);
    }
};

// Backward: ds of a piece of the vocabulary but for a teacher's terms, as an operand: bfloat16, or float32 taken apart.
//
// In bfloat16 that is one rounding more than float32 scores would need.  It is what the matrix units take; ds in two bfloat16 numbers would keep it, for
// twice the products of dx and of dw: two thirds more of the whole (4096 rows of 4096 over 32000: 1.6 ms to 2.5).  What it costs (errors against float64 as
// 2-norms, dx / dw; rounding results by itself leaves 0.00166 / 0.00165): those rows 0.00195 / 0.00189, 2048 rows against 64 terms 0.00234 / 0.00168.
// That is float64's products of ds so rounded but for 0.00014 of their norm: nothing else has fewer bits than float32.
template <typename T>
struct Slopes : Counted {
    static constexpr bool kCounted = true;
    uint16_t *ds;
    uint64_t ld;
    uint32_t part;
    const float2 *row;
    const uint32_t *ids;  // [rows][4]: a row's target, whose weight is 1, or NULL: a teacher's terms are put right afterwards
    uint32_t shift, base;
    float over2;
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t) const
    {
        in_rows(acc, strip, lane, m0, n0, m, part, [&](uint32_t r, uint32_t c, float(&z)[8]) __attribute__((always_inline)) { finish(r, c, z); });
    }
    // of eight products of a row
    __device__ inline __attribute__((always_inline)) void finish(uint32_t r, uint32_t c, float (&z)[8]) const
    {
        const float2 by = row[r];
        const uint32_t term = ids ? ids[uint64_t(r) << shift] - base : kNone;
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) z[j] = c + j < n ? by.y * (__builtin_amdgcn_exp2f(z[j] * over2 - by.x) - (c + j == term ? 1.0f : 0.0f)) : 0.0f;
        uint16_t *to = ds + r * ld + c;
        if constexpr (sizeof(T) == 2) {
            store_n<uint16_t, 8>(to, z);
        } else {
            u32x4 out[kParts];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                uint32_t s[2][kParts];
                split(z[2 * j], s[0]);
                split(z[2 * j + 1], s[1]);
#pragma unroll
                for (uint32_t q = 0; q < kParts; ++q) out[q][j] = __builtin_amdgcn_perm(s[1][q], s[0][q], 0x07060302);
            }
#pragma unroll
            for (uint32_t q = 0; q < kParts; ++q) *reinterpret_cast<u32x4 *>(to + q * part) = out[q];
        }
    }
};

// Elements of a float32 result as far as there are columns.
__device__ inline void put_f32(float *to, uint32_t have, const float (&z)[8])
{
    if (have >= 8) {
        store_n<float, 8>(to, z);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < have) to[j] = z[j];
    }
}

// The sum of N neighbours over planes `step` apart, of which `have` are there: in the planes' order, four on their way at once.  (us, so / one after
// the other: 16 planes of 26 rows of 863 6 / 20.)
template <int N>
__device__ inline void sum_planes(const float *from, uint64_t step, uint32_t planes, uint32_t have, float (&z)[N])
{
    constexpr uint32_t kAhead = 4;
#pragma unroll
    for (int j = 0; j < N; ++j) z[j] = 0;
    for (uint32_t p = 0; p < planes; p += kAhead) {
        float x[kAhead][N];
        if (have >= N) {
#pragma unroll
            for (uint32_t k = 0; k < kAhead; ++k) load_n<float, N>(from + min(p + k, planes - 1) * step, x[k]);
        } else {
#pragma unroll
            for (uint32_t k = 0; k < kAhead; ++k)
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) x[k][j] = (from + min(p + k, planes - 1) * step)[min(j, have - 1)];
        }
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) z[j] += p + k < planes ? x[k][j] : 0.0f;
    }
}

// A result in float32, a plane for each part of its sum: dx of the rows that have a term (Counted), added to from piece to piece, or a
// few tiles' scores (Product).
template <typename Base>
struct Planes : Base {
    static constexpr bool kCounted = std::is_same<Base, Counted>::value, kPartByPart = false;
    float *planes;  // [parts][rows][n]
    uint32_t rows, add;
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t p) const
    {
        const uint32_t n = this->n;
        in_rows(acc, strip, lane, m0, n0, this->m, n, [&](uint32_t r, uint32_t c, float(&z)[8]) __attribute__((always_inline)) {
            float *to = planes + (uint64_t(p) * rows + r) * n + c;
            const uint32_t have = n - c;
            if (kCounted && add) {
#pragma unroll
                for (uint32_t j = 0; j < 8; ++j)
                    if (j < have) z[j] += to[j];
            }
            put_f32(to, have, z);
        });
    }
};

// The scores of a few rows.
struct FewScores : FewArgs {
    float *plane;  // [rows][out]
    __device__ inline void put(uint32_t m, uint32_t n, uint32_t have, float (&z)[8]) const { put_f32(plane + uint64_t(m) * out + n, have, z); }
};

// dw of a piece, or parts of its sum.
template <typename T>
__device__ inline void put_dw(T *to, uint32_t have, uint32_t add, float (&z)[8])
{
    if (have >= 8) {
        if (add) {
            float was[8];
            load_n<T, 8>(to, was);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] += was[j];
        }
        store_n<T, 8>(to, z);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < have) to[j] = narrow<T>(add ? z[j] + widen(to[j]) : z[j]);
    }
}

template <typename T>
struct Weights : Counted {
    static constexpr bool kCounted = true;
    T *dw;
    uint64_t ld;
    float *partial;  // [parts][m][n] where there are several
    uint32_t add;
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t p) const
    {
        in_rows(acc, strip, lane, m0, n0, m, n, [&](uint32_t r, uint32_t c, float(&z)[8]) __attribute__((always_inline)) {
            if (splits > 1) put_f32(partial + (uint64_t(p) * m + r) * n + c, n - c, z);
            else put_dw<T>(dw + r * ld + c, n - c, add, z);
        });
    }
};

// dx of a vocabulary that is one piece, whole sums: in the rows' own places at once.  (us, backward, so / by way of float32: bfloat16 4096 rows of
// 4096 over 32000 2618 / 2638, 8192 of 2048 over 2000 231 / 250.)
template <typename T>
struct Placed : Counted {
    static constexpr bool kCounted = true;
    T *dx;
    uint64_t ld;
    const uint32_t *list;
    template <int RM, int RN>
    __device__ inline __attribute__((always_inline)) void put(const f32x4 (&acc)[RM][RN], float *strip, uint32_t lane, uint32_t m0, uint32_t n0, uint32_t) const
    {
        in_rows(acc, strip, lane, m0, n0, m, n,
                [&](uint32_t r, uint32_t c, float(&z)[8]) __attribute__((always_inline)) { put_dw<T>(dx + list[r] * ld + c, n - c, 0, z); });
    }
};

template <typename T>
__global__ __launch_bounds__(256) void weights_join_kernel(Weights<T> a)
{
    const uint32_t across = (a.n + 7) / 8;
    for (uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x; i < uint64_t(a.m) * across; i += uint64_t(gridDim.x) * 256) {
        const uint32_t r = uint32_t(i / across), c = uint32_t(i % across) * 8, have = a.n - c;
        float z[8] = {};
        for (uint32_t p = 0; p < a.splits; ++p) {
            const float *from = a.partial + (uint64_t(p) * a.m + r) * a.n + c;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
                if (j < have) z[j] += from[j];
        }
        put_dw<T>(a.dw + r * a.ld + c, have, a.add, z);
    }
}

// ------------------------------------------------------------------ between and behind the products

struct Close {
    Terms terms;
    List list;
    const float2 *stats;  // [strips][rows]
    float2 *run;          // [rows]: what earlier pieces of the vocabulary left, or this one leaves
    uint32_t strips, earlier, last;
    const float *scores;  // [rows with a term, terms]
    float *loss, *saved;
};

// Puts the waves' sums together, 16 rows to a workgroup, and ends in the loss where the piece is the last one.
__global__ __launch_bounds__(256) void close_kernel(Close a)
{
    __shared__ float2 parts[16][17];
    const uint32_t r = threadIdx.x % 16, slice = threadIdx.x / 16, count = *a.list.count, i = blockIdx.x * 16 + r;
    float top = -INFINITY, sum = 0;
    auto join = [&](float2 by) {
        const float most = fmaxf(top, by.x), against = most == -INFINITY ? 0.0f : most;
        sum = sum * __builtin_amdgcn_exp2f(top - against) + by.y * __builtin_amdgcn_exp2f(by.x - against);
        top = most;
    };
    if (i < count) {
        if (a.earlier && slice == 0) join(a.run[i]);
#pragma unroll 4
        for (uint32_t s = slice; s < a.strips; s += 16) join(a.stats[uint64_t(s) * a.terms.rows + i]);
    }
    parts[slice][r] = make_float2(top, sum);
    __syncthreads();
    const uint32_t row_in = threadIdx.x / 16, at = threadIdx.x % 16, j = blockIdx.x * 16 + row_in;
    if (j >= a.terms.rows) return;
    top = -INFINITY;
    sum = 0;
#pragma unroll
    for (uint32_t s = 0; s < 16; ++s) join(parts[s][row_in]);
    const bool there = j < count;
    if (!a.last) {
        if (there && at == 0) a.run[j] = make_float2(top, sum);
        return;
    }
    // sixteen threads to a row
    const uint32_t row = a.list.rows[j], K = a.terms.terms;
    const float lse = there ? (top + __builtin_amdgcn_logf(sum)) * kLn2 : 0.0f;
    float loss = 0;
    for (uint32_t k = at; k < K; k += 16) {
        const uint64_t t = uint64_t(row) * K + k;
        float s = 0;
        const float q = there ? share(a.terms, t, id_at(a.terms.ids, a.terms.wide, t, a.terms.vocab)) : 0.0f;
        if (q != 0) {
            s = a.scores[uint64_t(j) * K + k];
            loss += q * (__builtin_amdgcn_logf(q) * kLn2 + (lse - s));
        }
        if (a.saved) a.saved[uint64_t(row) * (1 + K) + 1 + k] = s;
    }
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) loss += __shfl_xor(loss, d, 64);
    if (at == 0) {
        a.loss[row] = loss;
        if (a.saved) a.saved[uint64_t(row) * (1 + K)] = lse;
    }
}

// Scores that are held, a row to a workgroup.
struct Held {
    Terms terms;
    const float *planes;  // [parts][rows][vocab], before they are divided by the temperature
    uint32_t parts;
    float *loss, *saved;
};

template <int THREADS>
__global__ __launch_bounds__(THREADS) void held_kernel(Held a)
{
    constexpr int W = THREADS / 64;
    __shared__ float2 tops[W];
    __shared__ float room[W], q[TAGC_MAX_TERMS];
    const uint32_t row = blockIdx.x, K = a.terms.terms, V = a.terms.vocab, wave = threadIdx.x / 64;
    const uint64_t first = uint64_t(row) * K, next = uint64_t(a.terms.rows) * V;
    const float *scores = a.planes + uint64_t(row) * V;
    // largest number of all threads, and the sum of 2^(theirs - largest) numbers
    auto together = [&](float &top, float &sum) {
        auto join = [&](float t, float s) {
            const float most = fmaxf(top, t), against = most == -INFINITY ? 0.0f : most;
            sum = sum * __builtin_amdgcn_exp2f(top - against) + s * __builtin_amdgcn_exp2f(t - against);
            top = most;
        };
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) join(__shfl_xor(top, d, 64), __shfl_xor(sum, d, 64));
        __syncthreads();
        if ((threadIdx.x & 63) == 0) tops[wave] = make_float2(top, sum);
        __syncthreads();
        top = -INFINITY;
        sum = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) join(tops[w].x, tops[w].y);
    };
    // a term's share: 1, or the teacher's
    bool any = false;
    float top = -INFINITY, sum = 0;
    for (uint32_t k = threadIdx.x; k < K; k += THREADS) {
        const bool none = id_at(a.terms.ids, a.terms.wide, first + k, V) == V;
        float x = none ? -INFINITY : 0.0f;
        if (a.terms.logits && !none) x = a.terms.logits[first + k];
        q[k] = x;
        any = any || x != -INFINITY;
        top = fmaxf(top, x);
    }
    any = __syncthreads_or(any);
    if (!any) {
        if (threadIdx.x == 0) a.loss[row] = 0;
        if (a.saved)
            for (uint32_t k = threadIdx.x; k < 1 + K; k += THREADS) a.saved[uint64_t(row) * (1 + K) + k] = 0;
        return;
    }
    const float over2 = a.terms.over * kLog2e;
    if (a.terms.logits) {
        together(top, sum);
        const float against = top == -INFINITY ? 0.0f : top;
        sum = 0;
        for (uint32_t k = threadIdx.x; k < K; k += THREADS) sum += __builtin_amdgcn_exp2f((q[k] - against) * over2);
        sum = block_sum<float, W>(sum, room);
        for (uint32_t k = threadIdx.x; k < K; k += THREADS) {
            const float x = q[k], share = __builtin_amdgcn_exp2f((x - against) * over2) / sum;
            q[k] = x == -INFINITY ? 0.0f : share < kLeast ? kLeast : share;
        }
    } else if (threadIdx.x == 0) {
        q[0] = 1;
    }
    // the scores, four neighbours at a time, times log2(e) / T
    top = -INFINITY;
    sum = 0;
    for (uint32_t c = threadIdx.x * 4; c < V; c += THREADS * 4) {
        float z[4];
        const uint32_t have = min(4u, V - c);
        sum_planes<4>(scores + c, next, a.parts, have, z);
        float most = top;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
            z[j] *= over2;
            if (j < have) most = fmaxf(most, z[j]);
        }
        const float against = most == -INFINITY ? 0.0f : most;
        sum *= __builtin_amdgcn_exp2f(top - against);
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j)
            if (j < have) sum += __builtin_amdgcn_exp2f(z[j] - against);
        top = most;
    }
    together(top, sum);
    const float lse = (top + __builtin_amdgcn_logf(sum)) * kLn2;
    float loss[1] = {0};
    for (uint32_t k = threadIdx.x; k < K; k += THREADS) {
        float s = 0;
        if (q[k] != 0) {  // (each thread's own)
            const uint32_t id = id_at(a.terms.ids, a.terms.wide, first + k, V);
            for (uint32_t p = 0; p < a.parts; ++p) s += scores[p * next + id];
            s *= a.terms.over;
            loss[0] += q[k] * (__builtin_amdgcn_logf(q[k]) * kLn2 + (lse - s));
        }
        if (a.saved) a.saved[uint64_t(row) * (1 + K) + 1 + k] = s;
    }
    const float all = block_sum<float, W>(loss[0], room);
    if (threadIdx.x == 0) {
        a.loss[row] = all;
        if (a.saved) a.saved[uint64_t(row) * (1 + K)] = lse;
    }
}

// ds from parts of the scores' sums, as the product's end makes it of whole ones.
template <typename T>
__global__ __launch_bounds__(256) void slopes_kernel(Slopes<T> a, const float *planes, uint32_t parts)
{
    const uint32_t across = (a.n + 63) / 64 * 8;  // (zeros up to a whole slab of the next product)
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    const uint32_t r = uint32_t(i / across), c = uint32_t(i % across) * 8;
    if (r >= *a.there) return;
    float z[8];
    sum_planes<8>(planes + uint64_t(r) * a.n + min(c, a.n - 1), uint64_t(a.m) * a.n, parts, c < a.n ? a.n - c : 1, z);
    a.finish(r, c, z);
}

// ds where a row has a term, in its place: from the score that the forward pass saved, so that 1 - q's difference is taken before
// anything is rounded.  A token that is a row's term twice gets the same value twice.
//
// A workgroup takes rows of 2^shift terms, 256 terms together or a row of more: ids and weights lie in local memory, where each term looks for itself.
// (64 terms of 2048 rows: 10 us; each reading its row's terms from memory, 18.)
template <typename T>
__global__ __launch_bounds__(256) void terms_slope_kernel(Terms a, List l, const uint32_t *ids, uint32_t shift, const float2 *rows, const float *saved, uint16_t *ds,
                                                          uint64_t ld, uint32_t part, uint32_t begin, uint32_t end)
{
    __shared__ uint32_t id[TAGC_MAX_TERMS];
    __shared__ float q[TAGC_MAX_TERMS];
    const uint32_t width = 1u << shift, each = width < 256 ? 256 >> shift : 1, count = *l.count;
    for (uint32_t s = threadIdx.x; s < each * width; s += 256) {
        const uint32_t i = blockIdx.x * each + (s >> shift), k = s & (width - 1);
        id[s] = i < count ? ids[(uint64_t(i) << shift) + k] : kNone;
        q[s] = id[s] != kNone ? share(a, uint64_t(l.rows[i]) * a.terms + k, id[s]) : 0.0f;
    }
    __syncthreads();
    for (uint32_t s = threadIdx.x; s < each * width; s += 256) {
        const uint32_t own = id[s], i = blockIdx.x * each + (s >> shift), k = s & (width - 1);
        if (own < begin || own >= end) continue;  // (kNone is behind every end)
        float sum = 0;
        for (uint32_t j = s - k; j < s - k + a.terms; ++j) sum += id[j] == own ? q[j] : 0.0f;
        const uint32_t row = l.rows[i];
        const float2 by = rows[i];
        const float x = by.y * (__builtin_amdgcn_exp2f(saved[uint64_t(row) * (1 + a.terms) + 1 + k] * kLog2e - by.x) - sum);
        uint16_t *to = ds + i * ld + (own - begin);
        if constexpr (sizeof(T) == 2) {
            *to = narrow<uint16_t>(x);
        } else {
            uint32_t parts[kParts];
            split(x, parts);
#pragma unroll
            for (uint32_t p = 0; p < kParts; ++p) to[p * part] = uint16_t(parts[p] >> 16);
        }
    }
}

// dx in the rows' own places: the planes' sum, zeros where a row has no term.
template <typename T>
__global__ __launch_bounds__(256) void place_kernel(const float *planes, uint32_t n_planes, List l, uint32_t rows, uint32_t cols, T *dx, uint64_t ld)
{
    const uint32_t across = (cols + 7) / 8, count = *l.count;
    const uint64_t i = uint64_t(blockIdx.x) * 256 + threadIdx.x;
    const uint32_t r = uint32_t(i / across), c = uint32_t(i % across) * 8, have = min(8u, cols - c);
    if (r >= rows) return;
    float z[8] = {};
    if (r < count) sum_planes<8>(planes + uint64_t(r) * cols + c, uint64_t(rows) * cols, n_planes, have, z);
    T *to = dx + l.rows[r] * ld + c;
    if (have == 8) {
        store_n<T, 8>(to, z);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j)
            if (j < have) to[j] = narrow<T>(z[j]);
    }
}

// Zeros in dx where a row has no term, a wave to a row.
template <typename T>
__global__ __launch_bounds__(256) void blank_kernel(List l, uint32_t rows, uint32_t cols, T *dx, uint64_t ld)
{
    const uint32_t r = blockIdx.x * 4 + threadIdx.x / 64;
    if (r >= rows || r < *l.count) return;
    T *to = dx + l.rows[r] * ld;
    for (uint32_t c = threadIdx.x % 64 * 8; c < cols; c += 64 * 8) {
        float z[8] = {};
        put_dw<T>(to + c, cols - c, 0, z);
    }
}

// ------------------------------------------------------------------ host

int check_sizes(uint64_t rows, uint64_t in, uint64_t vocab, uint32_t terms, uint32_t dtype, uint32_t id_type, double temperature, const float *logits)
{
    if (dtype > TAGC_BF16 || id_type > TAGC_ID_I64 || !in || !vocab || !terms || (!logits && terms != 1)) return TAGC_EINVAL;
    if (!(temperature > 0) || !isfinite(temperature) || !(float(1 / temperature) > 0) || !isfinite(float(kLog2e / temperature))) return TAGC_EINVAL;
    const uint64_t most = dtype == TAGC_F32 ? kMaxSide / 4 : kMaxSide;
    if (rows >= most || in >= most || vocab >= most || terms > TAGC_MAX_TERMS) return TAGC_ESIZE;
    // a launch has fewer than 2^32 threads: one to eight elements of a row, a wave to a term, a workgroup to a tile of 64 by 64
    const uint64_t r = up(rows, 64) / 64, i = up(in, 64) / 64, v = up(vocab, 64) / 64;
    if (r * i + r * v + i * v >= (1ull << 24) || rows * terms >= (1ull << 25) || up(rows, 64) * up(in, 64) >= (1ull << 34) || up(vocab, 64) * up(in, 64) >= (1ull << 34))
        return TAGC_ESIZE;
    return TAGC_OK;
}

// The operands as the products take them: rows with a term, and a piece of the vocabulary at a time.
struct Operands {
    bool raw;      // float32 as it lies
    bool lay;      // whether w's pieces are laid out anew
};

template <typename T>
Operands operands_of(uint64_t M, uint64_t D, uint64_t V, const void *w, uint64_t ldw, bool forward)
{
    if (sizeof(T) == 2) return Operands{false, !as_it_lies(TAGC_BF16, w, ldw, D, false)};
    const bool raw = forward && raw_pays(M, V) && ldw < kMaxSide;
    return Operands{raw, !raw};
}

// Rows of a piece of the vocabulary that holds so many bytes a row: pieces alike, but in whole rounds of tiles, of which 4096 rows make so many
// that they fill 256 compute units at most sizes.  (Float32, 1024 rows of 768 over 50257, three pieces: of 20480
// rows 1350 us, alike, of 16768, 1386.)
uint64_t piece_rows(uint64_t vocab, uint64_t bytes)
{
    uint64_t n = kPieceBytes / (bytes ? bytes : 1);
    if (n < kPieceRows) n = kPieceRows;
    const uint64_t pieces = (vocab + n - 1) / n, each = (vocab + pieces - 1) / pieces;
    return up(each, 4096) <= n ? up(each, 4096) : up(each, 256);
}

template <typename T>
Gather gather(const void *src, uint64_t ld, uint64_t n, uint64_t cols, const Operand &to)
{
    Gather a{};
    a.src = src;
    a.to = const_cast<void *>(to.p);
    a.ld = ld;
    a.to_ld = to.ld;
    a.n = uint32_t(n);
    a.cols = uint32_t(cols);
    a.part = to.part;
    a.across = uint32_t((sizeof(T) == 4 && to.part ? to.part : to.ld) / 8);
    return a;
}

template <typename T>
void launch_gather(const Gather &a, hipStream_t s)
{
    ProfileScope prof("loss_lay", s);
    gather_kernel<T><<<uint32_t((uint64_t(a.n) * a.across + 255) / 256), 256, 0, s>>>(a);
}

// x's rows that have a term, laid out: an operand for products, zeros behind a row's last element up to a whole slab.
template <typename T>
Operand room_for_x(Places &w, uint64_t M, uint64_t D, bool raw)
{
    if (sizeof(T) == 4 && raw) return Operand{w.take<float>(M * up(D, 8)), up(D, 8), 0};
    Operand to = room(w, sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16, M, D);
    if (sizeof(T) == 2) to.part = 0;
    return to;
}

template <typename G>
Terms terms_of(const G *l, Places &w)
{
    Terms t{l->ids, l->logits, nullptr, nullptr, uint32_t(l->rows), l->terms, uint32_t(l->vocab), l->id_type, float(1 / l->temperature)};
    if (l->logits) {
        t.q = w.take<float>(l->rows * l->terms);
        t.any = w.take<uint8_t>(l->rows);
    }
    return t;
}

// What the backward pass gives to a row's part.
struct Rowwise {
    const float *saved, *dloss;
    float2 *row;
    uint32_t step;
};

// Room for the list of the rows that have a term, and for the ids of their terms.
struct Listed {
    List list;
    uint32_t *ids, shift;
    Listed(Places &w, uint64_t rows, uint32_t terms) : shift(2)
    {
        while (1u << shift < terms) ++shift;
        list = List{w.take<uint32_t>(rows), w.take<uint32_t>(1)};
        ids = w.take<uint32_t>(rows << shift);
    }
};

template <typename T>
void launch_rows(const Terms &t, const Listed &l, const Gather &x, const Gather &w, const Rowwise &r, hipStream_t s)
{
    ProfileScope prof("loss_rows", s);
    if (t.logits && t.rows) terms_kernel<<<(t.rows + 3) / 4, 256, 0, s>>>(t);
    const uint64_t groups = (uint64_t(x.n) * x.across + 255) / 256, more = ((uint64_t(t.rows) << l.shift) + 255) / 256;
    const bool scan = t.rows <= kScanRows;
    const uint32_t w_from = uint32_t(groups + more + scan), w_groups = w.n ? uint32_t((uint64_t(w.n) * w.across + 255) / 256) : 0;
    const Lay a{t, l.list, x, uint32_t(groups), w, w_from, l.ids, l.shift, r.saved, r.dloss, r.row, r.step};
    if (scan) {
        lay_kernel<T, true><<<w_from + w_groups, 256, 0, s>>>(a);
    } else {
        list_kernel<<<1, kListThreads, 0, s>>>(t, l.list);
        lay_kernel<T, false><<<w_from + w_groups, 256, 0, s>>>(a);
    }
}

// Scores of few rows or of a small vocabulary are held, all rows', as parts of their sums: two launches, and as many workgroups as the
// parts make.
template <typename T>
int forward_held(const tagc_loss *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows, D = l->in, V = l->vocab;
    constexpr uint32_t dtype = sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16;
    Operand x{l->x, l->ldx, 0}, q{l->w, l->ldw, 0};
    // (us, few_kernel / thin tiles: bfloat16 1, 8, 16 rows of 4096 over 32000 55, 63, 73 / 59, 64, 65, of 768 over 50257 48, 50, 52 / 30, 31, 31, whose rows
    // leave most of its waves nothing; float32 of 768 over 50257 50, 54, 59 / 170, 88, 76)
    const bool lies = as_it_lies(dtype, l->w, l->ldw, D, false);
    const bool few = M <= kFewRows && (sizeof(T) == 4 || !lies || (M <= 8 && D >= 2048)), raw = sizeof(T) == 4 && raw_pays(M, V) && l->ldx < kMaxSide && l->ldw < kMaxSide;
    const bool lay_x = !few && !raw && !as_it_lies(dtype, l->x, l->ldx, D, false), lay_w = !few && !raw && !lies;
    if (lay_x) x = room(w, dtype, M, D);
    if (lay_w) q = room(w, dtype, V, D);
    const Shape f = few ? Shape{} : shape_of(M, V, D, dtype, false);
    const uint32_t parts = few ? 1 : f.splits;
    float *planes = w.take<float>(parts * M * V);
    if (!enqueue) return TAGC_OK;
    if (lay_x) launch_gather<T>(gather<T>(l->x, l->ldx, M, D, x), s);
    if (lay_w) launch_gather<T>(gather<T>(l->w, l->ldw, V, D, q), s);
    {
        ProfileScope prof("loss_product", s);
        if (few) {
            few_kernel<T><<<uint32_t((V + 15) / 16), kFewWaves * 64, 0, s>>>(FewScores{{l->x, l->w, l->ldx, l->ldw, uint32_t(M), uint32_t(D), uint32_t(V)}, planes});
        } else {
            Planes<Product> a{};
            aim(a, x, q, M, V, D, f);
            a.planes = planes;
            a.rows = uint32_t(M);
            launch<T, false, false>(a, f, s);
        }
    }
    ProfileScope prof("loss_close", s);
    const Terms terms{l->ids, l->logits, nullptr, nullptr, uint32_t(M), l->terms, uint32_t(V), l->id_type, float(1 / l->temperature)};
    const Held h{terms, planes, parts, l->loss, l->saved};
    if (V <= 8192) held_kernel<256><<<uint32_t(M), 256, 0, s>>>(h);
    else held_kernel<1024><<<uint32_t(M), 1024, 0, s>>>(h);
    return hip_ok(hipGetLastError());
}

template <typename T>
int forward(const tagc_loss *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows, D = l->in, V = l->vocab;
    constexpr uint32_t dtype = sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16;
    if (!M) return TAGC_OK;
    if (M <= kHeldRows && M * V <= kHeld) return forward_held<T>(l, w, enqueue, s);
    Close close{};
    const Terms terms = terms_of(l, w);
    const Listed listed(w, M, l->terms);
    const List list = listed.list;
    const Operands ops = operands_of<T>(M, D, V, l->w, l->ldw, true);
    const Operand x = room_for_x<T>(w, M, D, ops.raw);
    // (a wave's strip of columns has 32 at least)
    const uint64_t piece = piece_rows(V, M * 8 / 32 + (ops.lay ? up(D, 64) * (sizeof(T) == 4 ? 6 : 2) : 0));
    Operand wq{};
    if (ops.lay) {
        wq = room(w, dtype, piece, D);
        if (sizeof(T) == 2) wq.part = 0;
    }
    float2 *stats = w.take<float2>(up(piece, 256) / 32 * M);
    float2 *run = w.take<float2>(piece < V ? M : 0);
    float *scores = w.take<float>(M * l->terms);
    Strips lists{};
    lists.strips = uint32_t((V + kStrip - 1) / kStrip);
    const bool listing = l->terms >= kListTerms && lists.strips <= kMostStrips;
    if (listing) {
        lists.starts = w.take<uint32_t>((M + kStripsRows - 1) / kStripsRows * (lists.strips + 1));
        lists.entries = w.take<uint32_t>(M << listed.shift);
    }
    if (!enqueue) return TAGC_OK;

    const bool at_once = ops.lay && piece >= V && V * D < kAtOnce;
    launch_rows<T>(terms, listed, gather<T>(l->x, l->ldx, M, D, x), at_once ? gather<T>(l->w, l->ldw, V, D, wq) : Gather{}, Rowwise{}, s);
    if (listing) {
        ProfileScope prof("loss_strips", s);
        strips_kernel<<<uint32_t((M + kStripsRows - 1) / kStripsRows), 256, 0, s>>>(listed.ids, listed.shift, list.count, lists);
    }
    for (uint64_t v = 0; v < V; v += piece) {
        const uint64_t n = V - v < piece ? V - v : piece;
        const T *from = static_cast<const T *>(l->w) + v * l->ldw;
        Operand q{from, l->ldw, 0};
        if (ops.lay) {
            if (!at_once) launch_gather<T>(gather<T>(from, l->ldw, n, D, wq), s);
            q = wq;
        }
        Scores a{};
        const Shape f = shape_of(M, n, D, dtype, false, 1);
        aim(a, x, q, M, n, D, f);
        a.there = list.count;
        a.stats = stats;
        a.rows = uint32_t(M);
        a.over2 = float(kLog2e / l->temperature);
        a.ids = listed.ids;
        a.scores = scores;
        a.shift = listed.shift;
        a.terms = l->terms;
        a.base = uint32_t(v);
        a.over = terms.over;
        a.lists = lists;
        {
            ProfileScope prof("loss_product", s);
            launch<T, false, false>(a, f, s);
        }
        ProfileScope prof("loss_close", s);
        // (four waves share a tile's columns, whatever its size)
        close = Close{terms, list, stats, run, 4 * f.tiles_n, uint32_t(v > 0), uint32_t(v + n == V), scores, l->loss, l->saved};
        close_kernel<<<uint32_t((M + 15) / 16), 256, 0, s>>>(close);
    }
    return hip_ok(hipGetLastError());
}

template <typename T>
int backward(const tagc_loss_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows, D = l->in, V = l->vocab;
    constexpr uint32_t dtype = sizeof(T) == 4 ? TAGC_F32 : TAGC_BF16;
    if ((!l->dx && !l->dw) || (!M && (l->accumulate || !l->dw))) return TAGC_OK;
    const uint64_t rows = M ? M : 1;  // (no rows: dw becomes zeros by a product without terms)
    const Terms terms = terms_of(l, w);
    const Listed listed(w, rows, l->terms);
    const List list = listed.list;
    const Rowwise by{l->saved, l->dloss, w.take<float2>(rows), l->dloss_step};
    const Operands ops = operands_of<T>(rows, D, V, l->w, l->ldw, false);
    const Operand x = room_for_x<T>(w, rows, D, false);
    const uint64_t e = sizeof(T) == 4 ? 6 : 2, piece = piece_rows(V, (rows + (ops.lay ? up(D, 64) : 0)) * e);
    Operand wq{};
    if (ops.lay) {
        wq = room(w, dtype, piece, D);
        if (sizeof(T) == 2) wq.part = 0;
    }
    const Operand ds = room(w, dtype, rows, piece);
    // (us, dx of float32 64 rows of 768 over 50257 in up to 64 parts / 16: the whole call 264 / 295)
    const Shape fx = shape_of(rows, D, piece, dtype, false, 64), fw = shape_of(piece, D, rows, dtype, true);
    const bool placed = piece >= V && fx.splits == 1;
    // Scores' sums in parts, as planes, where that pays a launch more: few rows, a small vocabulary.  (us, so / by tiles that hold whole sums: float32 26
    // rows of 863 over 1977 49 / 59, 490 of 1152 over 980 66 / 83, bfloat16 64 of 2048 over 16000, 125 thin tiles, 81 / 87, 16 of 4096 over
    // 32000, 250 of them, 220 / 214.)
    const auto in_parts = [&](uint64_t n) {
        if (!M || !n || M > kHeldRows || M * n > kHeld) return Shape{};
        const Shape f = shape_of(M, n, D, dtype, false);
        return sizeof(T) == 2 && 2 * f.tiles_m * f.tiles_n > uint32_t(device_cu_count()) ? Shape{} : f;
    };
    uint64_t held = 0;
    for (const uint64_t n : {piece < V ? piece : V, V % piece})
        if (const Shape f = in_parts(n); f.splits > 1 && f.splits * M * n > held) held = f.splits * M * n;
    float *scores = w.take<float>(held);
    float *planes = w.take<float>(l->dx && !placed ? fx.splits * rows * D : 0), *partial = w.take<float>(l->dw && fw.splits > 1 ? fw.splits * piece * D : 0);
    if (!enqueue) return TAGC_OK;

    const bool at_once = ops.lay && M && piece >= V && V * D < kAtOnce;  // (without rows there need be no w)
    launch_rows<T>(terms, listed, gather<T>(l->x, l->ldx, M, D, x), at_once ? gather<T>(l->w, l->ldw, V, D, wq) : Gather{}, by, s);
    for (uint64_t v = 0; v < V; v += piece) {
        const uint64_t n = V - v < piece ? V - v : piece;
        const T *from = static_cast<const T *>(l->w) + v * l->ldw;
        Operand q{from, l->ldw, 0};
        if (ops.lay && M) {
            if (!at_once) launch_gather<T>(gather<T>(from, l->ldw, n, D, wq), s);
            q = wq;
        }
        if (M) {
            Slopes<T> a{};
            const Shape parts = in_parts(n), f = parts.splits > 1 ? parts : shape_of(M, n, D, dtype, false, 1);
            aim(a, x, q, M, n, D, f);
            a.there = list.count;
            a.ds = static_cast<uint16_t *>(const_cast<void *>(ds.p));
            a.ld = ds.ld;
            a.part = ds.part;
            a.row = by.row;
            a.ids = l->logits ? nullptr : listed.ids;
            a.shift = listed.shift;
            a.base = uint32_t(v);
            a.over2 = float(kLog2e / l->temperature);
            {
                ProfileScope prof("loss_slopes", s);
                if (f.splits > 1) {
                    Planes<Counted> b{};
                    static_cast<Counted &>(b) = a;
                    b.planes = scores;
                    b.rows = uint32_t(M);
                    launch<T, false, false>(b, f, s);
                    slopes_kernel<T><<<uint32_t((M * (up(n, 64) / 8) + 255) / 256), 256, 0, s>>>(a, scores, f.splits);
                } else {
                    launch<T, false, false>(a, f, s);
                }
            }
            if (l->logits) {  // (of a single term, too: its weight is not 1 but NaN where its logit is not finite)
                ProfileScope prof("loss_terms", s);
                const uint64_t each = listed.shift < 8 ? 256 >> listed.shift : 1;
                terms_slope_kernel<T><<<uint32_t((M + each - 1) / each), 256, 0, s>>>(terms, list, listed.ids, listed.shift, by.row, l->saved, a.ds, ds.ld, ds.part, uint32_t(v),
                                                                                      uint32_t(v + n));
            }
        }
        Operand p = ds;
        if (sizeof(T) == 2) p.part = 0;
        if (l->dx && M && placed) {
            Placed<T> a{};
            aim(a, p, q, M, D, n, fx);
            a.there = list.count;
            a.dx = static_cast<T *>(l->dx);
            a.ld = l->lddx;
            a.list = list.rows;
            ProfileScope prof("loss_dx", s);
            launch<T, false, true>(a, fx, s);
        } else if (l->dx && M) {
            Planes<Counted> a{};
            aim(a, p, q, M, D, n, fx);
            const uint64_t slab = dtype == TAGC_F32 ? kSlab3 : kSlab;
            a.slabs = uint32_t((up(n, slab) / slab + fx.splits - 1) / fx.splits);
            a.there = list.count;
            a.planes = planes;
            a.rows = uint32_t(M);
            a.add = v > 0;
            ProfileScope prof("loss_dx", s);
            launch<T, false, true>(a, fx, s);
        }
        if (l->dw) {
            Weights<T> a{};
            Shape f = fw;
            f.tiles_m = uint32_t((n + f.rows - 1) / f.rows);
            aim(a, p, x, n, D, rows, f);
            a.there = list.count;
            a.of_k = true;
            a.dw = static_cast<T *>(l->dw) + v * l->lddw;
            a.ld = l->lddw;
            a.partial = partial;
            a.add = l->accumulate;
            {
                ProfileScope prof("loss_dw", s);
                launch<T, true, true>(a, f, s);
            }
            if (f.splits > 1) {
                ProfileScope prof("loss_dw_join", s);
                const uint64_t groups = (n * ((D + 7) / 8) + 255) / 256;
                weights_join_kernel<T><<<uint32_t(groups < 65536 ? groups : 65536), 256, 0, s>>>(a);
            }
        }
    }
    if (l->dx && M) {
        ProfileScope prof("loss_place", s);
        if (placed) blank_kernel<T><<<uint32_t((M + 3) / 4), 256, 0, s>>>(list, uint32_t(M), uint32_t(D), static_cast<T *>(l->dx), l->lddx);
        else place_kernel<T><<<uint32_t((M * ((D + 7) / 8) + 255) / 256), 256, 0, s>>>(planes, fx.splits, list, uint32_t(M), uint32_t(D), static_cast<T *>(l->dx), l->lddx);
    }
    return hip_ok(hipGetLastError());
}

template <typename G>
bool good_operands(const G *l)
{
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2;
    return good(l->x, l->ldx, l->in, e) && good(l->w, l->ldw, l->in, e) && aligned_to(l->ids, l->id_type == TAGC_ID_I64 ? 8 : 4) && aligned_to(l->logits, 4);
}

// Whether [at, at + bytes) or rows of a result meet an operand of the call.
template <typename G>
bool meets_operands(const G *l, const Rows &r)
{
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, row = l->in * e, K = l->rows * l->terms, id = l->id_type == TAGC_ID_I64 ? 8 : 4;
    const Rows in[] = {Rows(l->x, l->rows, row, l->ldx * e), Rows(l->w, l->vocab, row, l->ldw * e), Rows(l->ids, 1, K * id, K * id), Rows(l->logits, 1, K * 4, K * 4)};
    for (const Rows &i : in)
        if (meet(r, i)) return true;
    return false;
}

int check(const tagc_loss *l)
{
    if (!l || l->reserved) return TAGC_EINVAL;
    const int rc = check_sizes(l->rows, l->in, l->vocab, l->terms, l->dtype, l->id_type, l->temperature, l->logits);
    if (rc) return rc;
    if (l->rows && (!l->x || !l->w || !l->ids || !l->loss)) return TAGC_EINVAL;
    if (!good_operands(l) || !aligned_to(l->loss, 4) || !aligned_to(l->saved, 4)) return TAGC_EINVAL;
    const uint64_t n = l->rows * 4, m = n * (1 + l->terms);
    const Rows loss(l->loss, 1, n, n), saved(l->saved, 1, m, m);
    return meets_operands(l, loss) || meets_operands(l, saved) || meet(loss, saved) ? TAGC_EINVAL : TAGC_OK;
}

int check(const tagc_loss_grad *l)
{
    if (!l || l->reserved || l->accumulate > 1 || l->dloss_step > 1) return TAGC_EINVAL;
    const int rc = check_sizes(l->rows, l->in, l->vocab, l->terms, l->dtype, l->id_type, l->temperature, l->logits);
    if (rc) return rc;
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, M = l->rows, row = l->in * e;
    if (M && (!l->x || !l->w || !l->ids || !l->saved || !l->dloss)) return TAGC_EINVAL;
    if (!good_operands(l) || !aligned_to(l->saved, 4) || !aligned_to(l->dloss, 4) || !good(l->dx, l->lddx, l->in, e) || !good(l->dw, l->lddw, l->in, e)) return TAGC_EINVAL;
    const uint64_t m = M * 4 * (1 + l->terms), n = M ? 4 * (1 + (M - 1) * l->dloss_step) : 0;
    const Rows saved(l->saved, 1, m, m), dloss(l->dloss, 1, n, n), dx(l->dx, M, row, l->lddx * e), dw(l->dw, l->vocab, row, l->lddw * e);
    if (meets_operands(l, dx) || meets_operands(l, dw) || meet(dx, saved) || meet(dw, saved) || meet(dx, dloss) || meet(dw, dloss) || meet(dx, dw)) return TAGC_EINVAL;
    return TAGC_OK;
}

int forward(const tagc_loss *l, Places &w, bool enqueue, hipStream_t s)
{
    return l->dtype == TAGC_F32 ? forward<float>(l, w, enqueue, s) : forward<uint16_t>(l, w, enqueue, s);
}

int backward(const tagc_loss_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    return l->dtype == TAGC_F32 ? backward<float>(l, w, enqueue, s) : backward<uint16_t>(l, w, enqueue, s);
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_loss_forward_workspace(const tagc_loss *l, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check(l);
    if (rc) return rc;
    Places w(nullptr);
    forward(l, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_loss_backward_workspace(const tagc_loss_grad *l, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check(l);
    if (rc) return rc;
    Places w(nullptr);
    backward(l, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_loss_forward(const tagc_loss *l, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_loss_forward_workspace(l, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    return forward(l, w, true, static_cast<hipStream_t>(stream));
}

extern "C" int tagc_loss_backward(const tagc_loss_grad *l, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_loss_backward_workspace(l, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    return backward(l, w, true, static_cast<hipStream_t>(stream));
}
