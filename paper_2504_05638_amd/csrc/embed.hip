// Token embeddings: rows of a table, and the table's gradient.
//
//   y[t] = scale * table[ids[t]] + residual[t]            dtable[v] (+)= scale * sum over t with ids[t] = v of dy[t]
//
// The gradient's sums have an order of their own: tokens are sorted by id, and by place where ids are equal, so that
// a row's terms lie one behind the other.  A workgroup sorts kChunk tokens, four bits of their ids at a time; sorted chunks are merged by searching
// each one for every token of the others, kMerge of them at a time.  Pieces of sorted tokens are summed side by side; a run of one id that goes on into the next piece
// leaves a partial sum there, and these are joined in order.  No atomics on sums, nothing to clear.
//
// Batches of up to kDirect tokens are not sorted: the first token of an id finds the others, and all is one launch.
//
// Bound by bytes: the rows looked up, or dy and the table's gradient, most of which is zeros; these are written while the tokens are
// sorted.
#include <math.h>

#include <type_traits>

#include "device_utils.h"
#include "elements.h"
#include "tagc_internal.h"
#include "tagc_train.h"

namespace tagc {

namespace {

// Tokens sorted together, in local memory.
constexpr uint32_t kChunk = 4096, kSortThreads = 1024, kSlots = kChunk / kSortThreads, kSortWaves = kSortThreads / 64;
constexpr uint32_t kMerge = 16;        // sorted lists merged at once
// Sorted tokens summed by a workgroup: many leave fewer partial sums behind, few make more workgroups of a short batch.  (us, eight / 16 /
// 32: 16384 tokens into 32000 by 4096 in bfloat16 111 / 101 / 96, 65536 into 50257 by 768 101 / 93 / 88, 1023 there in float32 41 / 44 / 48.)
constexpr uint32_t kShortPiece = 8, kLongPiece = 32, kShort = 8192;
constexpr uint32_t kSumThreads = 256, kRunSlices = kSumThreads / 64;
constexpr uint32_t kZeroRows = 64;     // most table rows that a workgroup looks after for want of tokens
// Tokens up to which it looks at all of them, while they are sorted; at more it searches the sorted ones, while these are summed.  (us, 65536 tokens into 50257
// by 768 in bfloat16: 139 / 90.)
constexpr uint32_t kZerosFirst = 16384;

// Tokens up to which there is one launch.  (us, with it / with the sort: 128 tokens into 1000 by 512 7 / 12; 512 there 18 / 13, and 512 of one id into
// 32000 by 4096 116 / 62, for which a workgroup adds them all.)
constexpr uint32_t kDirect = 128;

// An id, or `vocab` for what is no token.
__device__ inline uint32_t id_at(const void *ids, uint32_t wide, uint64_t t, uint32_t vocab)
{
    const uint64_t id = wide ? static_cast<const uint64_t *>(ids)[t] : uint64_t(int64_t(static_cast<const int32_t *>(ids)[t]));
    return id < vocab ? uint32_t(id) : vocab;
}

// ------------------------------------------------------------------ forward

struct Lookup {
    const void *ids, *table, *residual;
    void *y;
    uint64_t ldt, ldr, ldy;
    uint32_t rows, width, vocab, wide, spans;
    float scale;
};

// Where a lane whose piece begins at column c loads from: the piece, or, of a row's last one that is not whole, the row's last 16 bytes, of which
// its own elements are the last ones.  Rows shorter than that are not loaded so.  (us, so / such a piece one element after the other, bfloat16:
// lookup of 8192 rows of 4095 with a residual 36 / 40; gradient of 16384 tokens into 32000 by 4095 103 / 132, added to a table 84 / 136.)
template <uint32_t V>
__device__ inline uint32_t load_at(uint32_t c, uint32_t width) { return min(c, width - V); }

// A wave takes kSteps pieces of 16 bytes to a lane of one row.
constexpr uint32_t kSteps = 4;
template <typename T>
__global__ __launch_bounds__(256) void lookup_kernel(Lookup a)
{
    constexpr uint32_t V = 16 / sizeof(T), kSpan = 64 * V * kSteps;
    const uint64_t job = uint64_t(blockIdx.x) * 4 + threadIdx.x / 64;
    const uint64_t t = job / a.spans;
    if (t >= a.rows) return;
    const uint32_t from = uint32_t(job % a.spans) * kSpan + threadIdx.x % 64 * V;
    const uint32_t id = id_at(a.ids, a.wide, t, a.vocab);
    const T *row = static_cast<const T *>(a.table) + (id < a.vocab ? id : 0) * a.ldt, *res = static_cast<const T *>(a.residual) + t * a.ldr;
    T *y = static_cast<T *>(a.y) + t * a.ldy;
    const bool token = id < a.vocab;
    Lane<T, V> in[kSteps] = {}, add[kSteps] = {};
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) {
        const uint32_t c = from + s * 64 * V;
        if (c >= a.width || a.width < V) continue;
        if (token) in[s].load(row + load_at<V>(c, a.width));
        if (a.residual) add[s].load(res + load_at<V>(c, a.width));
    }
#pragma unroll
    for (uint32_t s = 0; s < kSteps; ++s) {
        const uint32_t c = from + s * 64 * V;
        if (c >= a.width) break;
        if (a.width < V) {
            for (uint32_t j = 0; j < a.width; ++j) {
                const float z = token ? a.scale * widen(row[j]) : 0.0f;
                y[j] = narrow<T>(a.residual ? z + widen(res[j]) : z);
            }
            break;
        }
        float z[V];
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) z[j] = a.residual ? a.scale * in[s][j] + add[s][j] : a.scale * in[s][j];
        if (!token)
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) z[j] = add[s][j];
        if (c + V <= a.width) {
            store_n<T, V>(y + c, z);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < V; ++j)
                if (a.width - V + j >= c) y[a.width - V + j] = narrow<T>(z[j]);
        }
    }
}

// ------------------------------------------------------------------ sorting

struct Sorted {
    uint32_t *keys, *order;  // [rows] ids in order, and the tokens that have them
};

struct Tokens {
    const void *ids;
    Sorted to;
    void *dtable;        // NULL: no zeros are wanted
    uint64_t ldt;
    uint32_t rows, width, vocab, wide, groups;
    uint32_t zero_rows;  // table rows of a workgroup
    uint32_t bits;       // of the largest id, which is `vocab`
};

// Zeros in those of a workgroup's rows, from `first` on, that no token has been found for.
template <typename T, uint32_t THREADS>
__device__ inline void write_zeros(T *dtable, uint64_t ld, uint32_t width, uint32_t first, uint32_t rows, const uint32_t *found)
{
    constexpr uint32_t V = 16 / sizeof(T);
    const uint32_t across = (width + V - 1) / V;
    const float zeros[V] = {};
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < rows * across; i += THREADS) {
        const uint32_t r = i / across, c = (i - r * across) * V;
        if (found[r]) continue;
        T *row = dtable + (first + r) * ld;
        if (width >= V) {
            store_n<T, V>(row + load_at<V>(c, width), zeros);
        } else {
            for (uint32_t j = 0; j < width; ++j) row[j] = T(0);
        }
    }
}

// The same for some rows of the table, whose tokens are looked for among all.  `found`: local memory for kZeroRows words.
template <typename T, uint32_t THREADS>
__device__ inline void zero_rows(const Tokens &a, uint32_t which, uint32_t *found)
{
    const uint32_t first = which * a.zero_rows;
    if (threadIdx.x < a.zero_rows) found[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll 4
    for (uint32_t t = threadIdx.x; t < a.rows; t += THREADS) {
        const uint32_t v = id_at(a.ids, a.wide, t, a.vocab) - first;
        if (v < a.zero_rows) found[v] = 1;
    }
    __syncthreads();
    write_zeros<T, THREADS>(static_cast<T *>(a.dtable), a.ldt, a.width, first, min(a.zero_rows, a.vocab - first), found);
}

// The first workgroups sort a chunk each: by four bits at a time, lowest first, each time in the order that there was, so that equal ids stay in the
// tokens' order.  A token's new place is the number of smaller digits, of the same digit in the waves before and, by ballots, in the lanes
// before it.  The others write zeros: bytes that keep the memory busy meanwhile (16384 tokens into 32000 by 4096 in bfloat16: 218 MB, 40 to 51 us by what
// the caches have to write back; sorting alone takes 15 at 65536 tokens).
template <typename T>
__global__ __launch_bounds__(kSortThreads) void sort_kernel(Tokens a)
{
    __shared__ uint32_t keys[kChunk], counts[16 * kSlots * kSortWaves], room[kSortWaves];
    __shared__ uint16_t order[kChunk];
    static_assert(16 * kSlots * kSortWaves == kSortThreads, "a count to a thread");
    if (blockIdx.x >= a.groups) return zero_rows<T, kSortThreads>(a, blockIdx.x - a.groups, keys);
    const uint32_t chunk = blockIdx.x * kChunk, have = min(kChunk, a.rows - chunk), slots = (have + kSortThreads - 1) / kSortThreads;
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint64_t before = (1ull << lane) - 1;
    uint32_t key[kSlots], at[kSlots];
#pragma unroll
    for (uint32_t s = 0; s < kSlots; ++s) {
        at[s] = s * kSortThreads + threadIdx.x;
        key[s] = at[s] < have ? id_at(a.ids, a.wide, chunk + at[s], a.vocab) : 0xFFFFFFFFu;  // (behind all others)
    }
    for (uint32_t shift = 0; shift < a.bits; shift += 4) {
        counts[threadIdx.x] = 0;
        __syncthreads();
        uint32_t place[kSlots];
#pragma unroll
        for (uint32_t s = 0; s < kSlots; ++s) {
            if (s >= slots) break;
            const uint32_t digit = key[s] >> shift & 15;
            uint64_t same = ~0ull;
#pragma unroll
            for (uint32_t b = 0; b < 4; ++b) {
                const uint64_t set = __ballot(digit >> b & 1);
                same &= digit >> b & 1 ? set : ~set;
            }
            place[s] = uint32_t(__popcll(same & before));
            if (!place[s]) counts[(digit * kSlots + s) * kSortWaves + wave] = uint32_t(__popcll(same));
        }
        __syncthreads();
        uint32_t all;
        const uint32_t first = block_excl_scan<uint32_t, kSortWaves>(counts[threadIdx.x], &all, room);
        counts[threadIdx.x] = first;
        __syncthreads();
#pragma unroll
        for (uint32_t s = 0; s < kSlots; ++s) {
            if (s >= slots) break;
            const uint32_t to = counts[((key[s] >> shift & 15) * kSlots + s) * kSortWaves + wave] + place[s];
            keys[to] = key[s];
            order[to] = uint16_t(at[s]);
        }
        __syncthreads();
#pragma unroll
        for (uint32_t s = 0; s < kSlots; ++s) {
            if (s >= slots) break;
            key[s] = keys[s * kSortThreads + threadIdx.x];
            at[s] = order[s * kSortThreads + threadIdx.x];
        }
    }
#pragma unroll
    for (uint32_t s = 0; s < kSlots; ++s) {
        const uint32_t i = s * kSortThreads + threadIdx.x;
        if (i >= have) break;
        a.to.keys[chunk + i] = key[s];
        a.to.order[chunk + i] = chunk + at[s];
    }
}

// How many of `n` sorted keys are under `key`.
__device__ inline uint32_t under(const uint32_t *keys, uint32_t n, uint32_t key)
{
    uint32_t lo = 0;
    while (n) {
        const uint32_t half = n / 2;
        const bool less = keys[lo + half] < key;
        lo = less ? lo + half + 1 : lo;
        n = less ? n - half - 1 : half;
    }
    return lo;
}

// Sorted lists of `run` tokens, kMerge of them to one: a token's place is its own list's, and what the others have before it.  The first half
// of each search is among 64 of a list's ids in local memory.  (65536 tokens: 29 us without, 23 with.)
constexpr uint32_t kSamples = 64;
__global__ __launch_bounds__(256) void merge_kernel(Sorted from, uint32_t rows, uint32_t run, Sorted to)
{
    __shared__ uint32_t samples[kMerge][kSamples];
    static_assert(kChunk % 256 == 0, "a workgroup's tokens are of one list");
    const uint32_t i = blockIdx.x * 256 + threadIdx.x, own = blockIdx.x * 256 / run, first = own / kMerge * kMerge, step = run / kSamples;
#pragma unroll
    for (uint32_t s = threadIdx.x; s < kMerge * kSamples; s += 256) {
        const uint64_t at = uint64_t(first + s / kSamples) * run + s % kSamples * step;
        samples[s / kSamples][s % kSamples] = at < rows ? from.keys[at] : 0xFFFFFFFFu;
    }
    __syncthreads();
    if (i >= rows) return;
    const uint32_t key = from.keys[i];
    uint32_t place = i % run;
#pragma unroll 4
    for (uint32_t k = 0; k < kMerge; ++k) {
        const uint32_t c = first + k;
        if (c == own || uint64_t(c) * run >= rows) continue;
        const uint32_t want = key + (c < own), some = under(samples[k], kSamples, want);
        if (!some) continue;
        // (the last sample under it is, and the next one is not)
        const uint32_t begin = (some - 1) * step + 1, length = min(run, rows - c * run);
        place += begin + under(from.keys + c * run + begin, min(step - 1, length - begin), want);
    }
    to.keys[first * run + place] = key;
    to.order[first * run + place] = from.order[i];
}

// ------------------------------------------------------------------ sums

struct Sums {
    Sorted sorted;
    const void *dy;
    void *dtable;
    float *partial;  // [pieces][2][width]: of a piece the sum of its first run, if that began before it, and of the run that goes on behind it
    uint64_t lddy, ldt;
    uint32_t rows, width, vocab, pieces, spans, accumulate;
    uint32_t zero_rows;  // as Tokens has them, where this launch writes the zeros
    float scale;
};

// By width: rows of whole pieces of V elements, of V at least, of less.
enum { kWhole, kTail, kThin };

// Of the piece that begins at column c; `sum` as load_piece has it.  A row's last piece that is not whole overlaps the one before it, whose sums are
// the same: without what is there to be added to, both may write them.
template <typename T, int ROWS>
__device__ inline void finish_row(const Sums &a, uint32_t key, uint32_t c, const float (&sum)[16 / sizeof(T)])
{
    constexpr uint32_t V = 16 / sizeof(T);
    T *row = static_cast<T *>(a.dtable) + key * a.ldt;
    if constexpr (ROWS != kThin) {
        const uint32_t at = ROWS == kWhole ? c : load_at<V>(c, a.width);
        float z[V], was[V];
        if (a.accumulate) load_n<T, V>(row + at, was);
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) z[j] = a.accumulate ? a.scale * sum[j] + was[j] : a.scale * sum[j];
        if (ROWS == kWhole || !a.accumulate || at == c) return store_n<T, V>(row + at, z);
#pragma unroll
        for (uint32_t j = 1; j < V; ++j)
            if (at + j >= c) row[at + j] = narrow<T>(z[j]);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j)
            if (j < a.width) row[j] = narrow<T>(a.accumulate ? a.scale * sum[j] + widen(row[j]) : a.scale * sum[j]);
    }
}

// A lane's piece of a row of dy, for finish_row.  (Lanes behind the row's end have its last piece as well, and no use for it: loads without
// branches go out together.)
template <typename T, int ROWS, bool PAST>
__device__ inline void load_piece(const T *row, uint32_t c, uint32_t width, Lane<T, 16 / sizeof(T)> &to)
{
    constexpr uint32_t V = 16 / sizeof(T);
    if constexpr (ROWS != kThin) {
        const T *from = row + load_at<V>(c, width);
        if constexpr (PAST) to.v = __builtin_nontemporal_load(reinterpret_cast<const typename Lane<T, V>::vec *>(from));
        else to.load(from);
    } else {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) to.v[j] = c + j < width ? row[c + j] : T(0);
    }
}

// Up to kDirect tokens: a workgroup to a token and 256 * V columns, if it is the first of its id, and the zeros beside them.
template <typename T, int ROWS>
__global__ __launch_bounds__(kSumThreads) void direct_kernel(Tokens a, Sums b)
{
    constexpr uint32_t V = 16 / sizeof(T), kAhead = 16;
    __shared__ uint32_t keys[kDirect], list[kDirect + kAhead];
    if (blockIdx.x >= a.groups) return zero_rows<T, kSumThreads>(a, blockIdx.x - a.groups, keys);
    const uint32_t t = blockIdx.x / b.spans, c = (blockIdx.x % b.spans * kSumThreads + threadIdx.x) * V;
    for (uint32_t i = threadIdx.x; i < a.rows; i += kSumThreads) keys[i] = id_at(a.ids, a.wide, i, a.vocab);
    __syncthreads();
    const uint32_t key = keys[t];
    if (key == a.vocab) return;
    bool earlier = false;
    for (uint32_t i = threadIdx.x; i < t; i += kSumThreads) earlier |= keys[i] == key;
    if (__syncthreads_or(earlier)) return;
    // each wave finds its tokens, 64 at a time, and one of them writes the list
    uint32_t n = 0;
    for (uint32_t i = t / 64 * 64; i < a.rows; i += 64) {
        const uint32_t at = i + (threadIdx.x & 63);
        const bool mine = at < a.rows && keys[at] == key;
        const uint64_t mask = __ballot(mine);
        if (threadIdx.x < 64 && mine) list[n + __popcll(mask & ((1ull << threadIdx.x) - 1))] = at;
        n += uint32_t(__popcll(mask));
    }
    __syncthreads();
    float sum[V] = {};
    for (uint32_t k = 0; k < n; k += kAhead) {
        Lane<T, V> x[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) load_piece<T, ROWS, false>(static_cast<const T *>(b.dy) + list[min(k + i, n - 1)] * b.lddy, c, a.width, x[i]);
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i)
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) sum[j] += k + i < n ? x[i][j] : 0.0f;
    }
    if (c < a.width) finish_row<T, ROWS>(b, key, c, sum);
}

// A workgroup sums a piece of sorted tokens, 256 * V columns of them; workgroups behind those write zeros.  Bound by the bytes of dy, of the rows that
// are finished and of the partial sums: 16384 tokens of 4096 in bfloat16 35 us for 134, 43 and 9 MB, 5.3 TB/s.
template <typename T, uint32_t PIECE, int ROWS>
__global__ __launch_bounds__(kSumThreads) void sum_kernel(Sums a)
{
    constexpr uint32_t V = 16 / sizeof(T);
    const uint32_t span = blockIdx.x % a.spans, c = (span * kSumThreads + threadIdx.x) * V;
    const uint32_t piece = blockIdx.x / a.spans;
    if (piece >= a.pieces) {
        __shared__ uint32_t found[kZeroRows];
        const uint32_t first = (blockIdx.x - a.pieces * a.spans) * a.zero_rows, rows = min(a.zero_rows, a.vocab - first);
        if (threadIdx.x < rows) {
            const uint32_t v = first + threadIdx.x, at = under(a.sorted.keys, a.rows, v);
            found[threadIdx.x] = at < a.rows && a.sorted.keys[at] == v;
        }
        __syncthreads();
        return write_zeros<T, kSumThreads>(static_cast<T *>(a.dtable), a.ldt, a.width, first, rows, found);
    }
    const uint32_t begin = piece * PIECE, n = min(PIECE, a.rows - begin);
    // a lane has a token's id and row, the piece's neighbours' ids behind them; all rows are asked for before the first is needed
    const uint32_t lane = threadIdx.x % 64, at = lane < n ? begin + lane : lane == PIECE ? begin - 1 : begin + n;
    const bool there = lane < n || (lane == PIECE && begin) || (lane == PIECE + 1 && begin + n < a.rows);
    const uint32_t mine = there ? a.sorted.keys[at] : 0xFFFFFFFFu, row = a.sorted.order[lane < n ? at : begin];
    // (taken from the lanes before lanes part: behind that, those that are done with a register may write to it)
    uint32_t rows[PIECE], keys[PIECE + 2];
#pragma unroll
    for (uint32_t k = 0; k < PIECE; ++k) rows[k] = __builtin_amdgcn_readlane(row, k);
#pragma unroll
    for (uint32_t k = 0; k < PIECE + 2; ++k) keys[k] = __builtin_amdgcn_readlane(mine, k);
    const uint32_t before = keys[PIECE], behind = keys[PIECE + 1];
    float sum[V] = {};
    uint32_t now = keys[0];
    bool began = now == before;
    auto flush = [&](bool goes_on) {
        if (now >= a.vocab || c >= a.width) return;
        if (!began && !goes_on) return finish_row<T, ROWS>(a, now, c, sum);
        // (a run that fills its piece and goes on both ways has the first place)
        float *to = a.partial + (uint64_t(piece) * 2 + (began ? 0 : 1)) * a.width;
        if constexpr (ROWS != kThin) {
            store_n<float, V>(to + load_at<V>(c, a.width), sum);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < V; ++j)
                if (j < a.width) to[j] = sum[j];
        }
    };
    // rows come four at a time, past the caches' order, which the table's rows are left to (16384 tokens of 4096: 40 us, 61 through the caches), the
    // next ones while these are added (two, eight: 1 % slower, the same; all at once, which leaves fewer workgroups room, half as long again)
    constexpr uint32_t kAhead = 4;
    Lane<T, V> x[2][kAhead];
    auto fetch = [&](uint32_t first, Lane<T, V>(&to)[kAhead]) __attribute__((always_inline)) {
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) load_piece<T, ROWS, true>(static_cast<const T *>(a.dy) + rows[first + k] * a.lddy, c, a.width, to[k]);
    };
    fetch(0, x[0]);
#pragma unroll
    for (uint32_t g = 0; g < PIECE; g += kAhead) {
        if (g + kAhead < PIECE) fetch(g + kAhead, x[g / kAhead + 1 & 1]);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
            if (g + k >= n) break;
            if (keys[g + k] != now) {
                flush(false);
                now = keys[g + k];
                began = false;
#pragma unroll
                for (uint32_t j = 0; j < V; ++j) sum[j] = 0;
            }
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) sum[j] += x[g / kAhead & 1][k][j];
        }
    }
    flush(now == behind);
}

// Runs that go on behind the piece that they begin in: their partial sums in order, a quarter to each of the four waves that share 64 * V
// columns, eight on their way at once.  (A token's share of text can be a tenth: 50 pieces of 16384 tokens, 10 us; one
// part after the other, four on their way, 31.)
template <typename T, uint32_t PIECE, int ROWS>
__global__ __launch_bounds__(kSumThreads) void run_kernel(Sums a)
{
    constexpr uint32_t V = 16 / sizeof(T), kAhead = 8;
    __shared__ float parts[kRunSlices][V][64];
    const uint32_t spans = (a.width + 64 * V - 1) / (64 * V), piece = blockIdx.x / spans, lane = threadIdx.x % 64, slice = threadIdx.x / 64;
    const uint32_t c = (blockIdx.x % spans * 64 + lane) * V;
    const uint32_t begin = piece * PIECE, next = begin + PIECE;
    if (next >= a.rows) return;
    const uint32_t key = a.sorted.keys[next];
    if (key >= a.vocab || a.sorted.keys[next - 1] != key || (begin && a.sorted.keys[begin - 1] == key)) return;
    const uint32_t end = under(a.sorted.keys, a.rows, key + 1), count = (end - 1) / PIECE - piece + 1;
    // (the first part is its piece's second sum, the others are their pieces' first)
    const uint32_t each = (count + kRunSlices - 1) / kRunSlices, from = slice * each, to = min(from + each, count);
    float sum[V] = {};
    for (uint32_t p = from; p < to; p += kAhead) {
        float x[kAhead][V];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k) {
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) x[k][j] = 0;
            if (p + k >= to) continue;
            const float *part = a.partial + (uint64_t(piece + p + k) * 2 + (p + k == 0)) * a.width;
            if constexpr (ROWS != kThin) {
                load_n<float, V>(part + load_at<V>(c, a.width), x[k]);
            } else {
#pragma unroll
                for (uint32_t j = 0; j < V; ++j)
                    if (c + j < a.width) x[k][j] = part[c + j];
            }
        }
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
#pragma unroll
            for (uint32_t j = 0; j < V; ++j) sum[j] += x[k][j];
    }
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) parts[slice][j][lane] = sum[j];
    __syncthreads();
    if (slice || c >= a.width) return;
#pragma unroll
    for (uint32_t s = 1; s < kRunSlices; ++s)
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) sum[j] += parts[s][j][lane];
    finish_row<T, ROWS>(a, key, c, sum);
}

// ------------------------------------------------------------------ host

int check(uint64_t rows, uint64_t width, uint64_t vocab, uint32_t dtype, uint32_t id_type, double scale)
{
    if (dtype > TAGC_BF16 || id_type > TAGC_ID_I64 || !isfinite(scale) || !isfinite(float(scale))) return TAGC_EINVAL;
    if (rows >= kMaxSide || width >= kMaxSide || vocab >= kMaxSide) return TAGC_ESIZE;
    // a launch has fewer than 2^32 threads: a workgroup of 256 to eight rows and 256 columns at least
    if ((up(rows, 8) / 8 + 1) * (up(width, 256) / 256) >= (1ull << 24)) return TAGC_ESIZE;
    return TAGC_OK;
}

int check(const tagc_embedding *l)
{
    if (!l) return TAGC_EINVAL;
    const int rc = check(l->rows, l->width, l->vocab, l->dtype, l->id_type, l->scale);
    if (rc) return rc;
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, id = l->id_type == TAGC_ID_I64 ? 8 : 4, M = l->rows, bytes = l->width * e;
    if (M && l->width && (!l->ids || !l->y || (l->vocab && !l->table))) return TAGC_EINVAL;
    if (!aligned_to(l->ids, id) || !good(l->table, l->ldt, l->width, e) || !good(l->residual, l->ldr, l->width, e) || !good(l->y, l->ldy, l->width, e)) return TAGC_EINVAL;
    const Rows y(l->y, M, bytes, l->ldy * e), table(l->table, l->vocab, bytes, l->ldt * e), res(l->residual, M, bytes, l->ldr * e), ids(l->ids, 1, M * id, M * id);
    const bool over = l->y == l->residual && (M <= 1 || l->ldy == l->ldr);
    return meet(y, table) || meet(y, ids) || (!over && meet(y, res)) ? TAGC_EINVAL : TAGC_OK;
}

int check(const tagc_embedding_grad *l)
{
    if (!l || l->reserved || l->accumulate > 1) return TAGC_EINVAL;
    const int rc = check(l->rows, l->width, l->vocab, l->dtype, l->id_type, l->scale);
    if (rc) return rc;
    const uint64_t e = l->dtype == TAGC_F32 ? 4 : 2, id = l->id_type == TAGC_ID_I64 ? 8 : 4, M = l->rows, bytes = l->width * e;
    if (l->vocab && l->width && (!l->dtable || (M && (!l->ids || !l->dy)))) return TAGC_EINVAL;
    if (!aligned_to(l->ids, id) || !good(l->dy, l->lddy, l->width, e) || !good(l->dtable, l->ldt, l->width, e)) return TAGC_EINVAL;
    const Rows dtable(l->dtable, l->vocab, bytes, l->ldt * e), dy(l->dy, M, bytes, l->lddy * e), ids(l->ids, 1, M * id, M * id);
    return meet(dtable, dy) || meet(dtable, ids) ? TAGC_EINVAL : TAGC_OK;
}

template <typename T>
int forward(const tagc_embedding *l, hipStream_t s)
{
    if (!l->rows || !l->width) return TAGC_OK;
    constexpr uint32_t kSpan = 64 * (16 / sizeof(T)) * kSteps;
    const uint32_t spans = uint32_t((l->width + kSpan - 1) / kSpan);
    const Lookup a{l->ids, l->table, l->residual, l->y, l->ldt, l->ldr, l->ldy, uint32_t(l->rows), uint32_t(l->width), uint32_t(l->vocab), l->id_type, spans, float(l->scale)};
    ProfileScope prof("embed_lookup", s);
    lookup_kernel<T><<<uint32_t((l->rows * spans + 3) / 4), 256, 0, s>>>(a);
    return hip_ok(hipGetLastError());
}

template <uint32_t V, typename F>
void by_rows(uint64_t width, F f)
{
    if (width < V) f(std::integral_constant<int, kThin>());
    else if (width % V) f(std::integral_constant<int, kTail>());
    else f(std::integral_constant<int, kWhole>());
}

template <typename T>
int backward(const tagc_embedding_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    const uint64_t M = l->rows;
    if (!l->vocab || !l->width || (!M && l->accumulate)) return TAGC_OK;
    const bool direct = M <= kDirect;
    const uint32_t piece = M <= kShort ? kShortPiece : kLongPiece, pieces = uint32_t((M + piece - 1) / piece);
    constexpr uint32_t V = 16 / sizeof(T);
    Sorted sorted{}, other{};
    if (!direct) sorted = Sorted{w.take<uint32_t>(M), w.take<uint32_t>(M)};
    if (M > kChunk) other = Sorted{w.take<uint32_t>(M), w.take<uint32_t>(M)};
    Sums a{};
    a.partial = w.take<float>(direct ? 0 : uint64_t(pieces) * 2 * l->width);
    if (!enqueue) return TAGC_OK;
    a.dy = l->dy;
    a.dtable = l->dtable;
    a.lddy = l->lddy;
    a.ldt = l->ldt;
    a.rows = uint32_t(M);
    a.width = uint32_t(l->width);
    a.vocab = uint32_t(l->vocab);
    a.pieces = pieces;
    a.spans = uint32_t((l->width + kSumThreads * V - 1) / (kSumThreads * V));
    a.accumulate = l->accumulate;
    a.scale = float(l->scale);
    uint32_t zeros = 0;
    {
        // (rows to a workgroup so that there are two workgroups to a compute unit)
        Tokens t{l->ids, sorted, l->dtable, l->ldt, a.rows, a.width, a.vocab, l->id_type, uint32_t((M + kChunk - 1) / kChunk), 1, 0};
        while (l->vocab >> t.bits) ++t.bits;
        while (t.zero_rows < kZeroRows && l->vocab / t.zero_rows > 2 * uint64_t(device_cu_count())) t.zero_rows *= 2;
        if (!l->accumulate) zeros = (a.vocab + t.zero_rows - 1) / t.zero_rows;
        a.zero_rows = t.zero_rows;
        if (direct) {
            t.groups = a.rows * a.spans;
            ProfileScope prof("embed_sum", s);
            by_rows<V>(l->width, [&](auto rows) { direct_kernel<T, decltype(rows)::value><<<t.groups + zeros, kSumThreads, 0, s>>>(t, a); });
            return hip_ok(hipGetLastError());
        }
        ProfileScope prof("embed_sort", s);
        sort_kernel<T><<<t.groups + (M <= kZerosFirst ? zeros : 0), kSortThreads, 0, s>>>(t);
        if (M <= kZerosFirst) zeros = 0;
        for (uint64_t run = kChunk; run < M; run *= kMerge) {
            merge_kernel<<<uint32_t((M + 255) / 256), 256, 0, s>>>(sorted, a.rows, uint32_t(run), other);
            const Sorted was = sorted;
            sorted = other;
            other = was;
        }
    }
    if (pieces) {
        a.sorted = sorted;
        ProfileScope prof("embed_sum", s);
        const uint32_t runs = (pieces - 1) * uint32_t((l->width + 64 * V - 1) / (64 * V));
        const auto go = [&](auto size) {
            by_rows<V>(l->width, [&](auto rows) {
                constexpr uint32_t P = decltype(size)::value, R = decltype(rows)::value;
                sum_kernel<T, P, R><<<pieces * a.spans + zeros, kSumThreads, 0, s>>>(a);
                if (runs) run_kernel<T, P, R><<<runs, kSumThreads, 0, s>>>(a);
            });
        };
        if (piece == kShortPiece) go(std::integral_constant<uint32_t, kShortPiece>());
        else go(std::integral_constant<uint32_t, kLongPiece>());
    }
    return hip_ok(hipGetLastError());
}

int backward(const tagc_embedding_grad *l, Places &w, bool enqueue, hipStream_t s)
{
    return l->dtype == TAGC_F32 ? backward<float>(l, w, enqueue, s) : backward<uint16_t>(l, w, enqueue, s);
}

}  // namespace

}  // namespace tagc

using namespace tagc;

extern "C" int tagc_embedding_forward(const tagc_embedding *e, void *stream)
{
    const int rc = check(e);
    if (rc) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return e->dtype == TAGC_F32 ? forward<float>(e, s) : forward<uint16_t>(e, s);
}

extern "C" int tagc_embedding_backward_workspace(const tagc_embedding_grad *e, uint64_t *bytes)
{
    if (!bytes) return TAGC_EINVAL;
    const int rc = check(e);
    if (rc) return rc;
    Places w(nullptr);
    backward(e, w, false, nullptr);
    *bytes = w.at;
    return TAGC_OK;
}

extern "C" int tagc_embedding_backward(const tagc_embedding_grad *e, void *workspace, void *stream)
{
    uint64_t need = 0;
    const int rc = tagc_embedding_backward_workspace(e, &need);
    if (rc) return rc;
    if (need && (!workspace || !aligned_to(workspace, 256))) return TAGC_EINVAL;
    Places w(workspace);
    return backward(e, w, true, static_cast<hipStream_t>(stream));
}
