// lookup.hip -- rows of a table by id, and the table's gradient by sorted ids.
//   out_i = scale table[id_i],  dtable_r = scale sum over id_i = r of dout_i
// Forward: bound by reading rows at random places and writing them in order.
// Backward: the places i are sorted by id (radix passes over pairs of id and
// place, ids that are no rows left out by the first), so that each row's
// gradients stand together and are summed in the order of their places, without
// atomics; bound by reading dout's rows at random places.
//   The sorted places are split into runs of equal length, a group of lanes each.
// A group sums the rows that begin in its run, into the next run where a row ends
// there; one that goes further (a popular id) is split: every run that it
// touches leaves its part's sum, and a last launch joins them in order.
// Measured: 3 000 000 ids, a third of them empty, rows of 128 bf16 values: 185 us
// forward (5.0 TB/s; 180 to 215 by what else is in the caches); the gradient of the
// rows that occur 290: three passes of 9 bits (5 to 10 us counting, 6.5 scanning,
// 14 to 18 scattering each), 8 for the list's places, 163 for the sums (4.3 TB/s,
// what rows at random places reach), 27 to join popular rows.  240 000 ids, 17 000
// rows of 100 fp32 values, whole: 76 us, of which 27 the sums and 27 the sort.
#include <type_traits>

#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kThreads = 256;
constexpr int kSortThreads = 512, kWaves = kSortThreads / 64;
// Entries that a workgroup sorts: 8 a thread, 2 where that leaves CUs idle (a
// pass of few tiles takes as long as one does: 240 000 ids 11 us with 8).
constexpr uint32_t tile_of(uint32_t n) { return kSortThreads * (n < 1u << 20 ? 2 : 8); }
constexpr uint32_t kMaxBits = 9, kMaxDigits = 1u << kMaxBits;

template <typename T> struct Chunk { static constexpr int n = 16 / sizeof(T); };

// 16 bytes of values from c on of a row of `width`, zeros past its end.
template <typename T> __device__ __forceinline__ u32x4 load_chunk(const uint8_t *row, uint32_t c, uint32_t width) {
    constexpr uint32_t n = Chunk<T>::n;
    const uint8_t *p = row + (size_t)c * sizeof(T);
    u32x4 x = {0, 0, 0, 0};
    if (c + n <= width) {
        x = *(const u32x4_any *)p;
    } else {
#pragma unroll
        for (uint32_t i = 0; i < n - 1; i++)
            if (c + i < width) {
                if constexpr (sizeof(T) == 4) x[i] = ((const uint32_t *)p)[i];
                else x[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (16 * (i % 2));
            }
    }
    return x;
}
// (Past the caches: 3 000 000 rows of 256 bytes 242 us with ordinary stores, 185 so.)
template <typename T> __device__ __forceinline__ void store_chunk(uint8_t *row, uint32_t c, uint32_t width, u32x4 x) {
    constexpr uint32_t n = Chunk<T>::n;
    uint8_t *p = row + (size_t)c * sizeof(T);
    if (c + n <= width) {
        __builtin_nontemporal_store(x, (u32x4_any *)p);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < n - 1; i++)
            if (c + i < width) {
                if constexpr (sizeof(T) == 4) ((uint32_t *)p)[i] = x[i];
                else ((uint16_t *)p)[i] = (uint16_t)(x[i / 2] >> (16 * (i % 2)));
            }
    }
}
template <typename T> __device__ __forceinline__ void unpack(u32x4 x, float (&f)[Chunk<T>::n]) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
        if constexpr (sizeof(T) == 4) {
            f[i] = __uint_as_float(x[i]);
        } else {
            f[2 * i] = __uint_as_float(x[i] << 16);
            f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        }
    }
}
template <typename T> __device__ __forceinline__ u32x4 packed(const float (&f)[Chunk<T>::n], float scale) {
    T v[Chunk<T>::n];
#pragma unroll
    for (int i = 0; i < Chunk<T>::n; i++) v[i] = (T)(f[i] * scale);
    u32x4 u;
    __builtin_memcpy(&u, v, 16);
    return u;
}

// ---------------------------------------------------------------- rows
struct Rows {
    const uint8_t *table;
    uint8_t *out;
    int64_t table_row, out_row;                            // bytes
    const int32_t *ids;
    uint32_t n, rows, width, chunks, per;                  // chunks of a row, rows of a tile
    uint64_t magic;                                        // division by chunks
    float scale;
};

// A workgroup takes `per` rows at a time, a thread four of their chunks.  FILL:
// zeros for all rows of `out`, without a table.
template <typename T, bool FILL> __global__ __launch_bounds__(kThreads) void copy_rows(Rows a) {
    const uint32_t tiles = (a.n + a.per - 1) / a.per;
    for (uint32_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint32_t first = tile * a.per, all = min(a.per, a.n - first) * a.chunks;
        for (uint32_t l0 = threadIdx.x; l0 < all; l0 += 4 * kThreads) {
            uint32_t row[4], c[4];
            int32_t id[4];
            u32x4 x[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const uint32_t l = l0 + i * kThreads, r = nlb_div(l, a.magic);
                row[i] = first + r;
                c[i] = (l - r * a.chunks) * Chunk<T>::n;
                id[i] = -1;
                if (!FILL && l < all) id[i] = a.ids[row[i]];
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[i] = u32x4{0, 0, 0, 0};
                if (!FILL && (uint32_t)id[i] < a.rows)
                    x[i] = load_chunk<T>(a.table + (int64_t)id[i] * a.table_row, c[i], a.width);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) {
                if (l0 + i * kThreads >= all) continue;
                if constexpr (!FILL) {
                    float f[Chunk<T>::n];
                    unpack<T>(x[i], f);
                    if ((uint32_t)id[i] < a.rows) x[i] = packed<T>(f, a.scale);
                }
                store_chunk<T>(a.out + (int64_t)row[i] * a.out_row, c[i], a.width, x[i]);
            }
        }
    }
}

// ---------------------------------------------------------------- sorting
struct Sort {
    const int32_t *ids;
    const uint64_t *from;                                  // id in the upper half, place in the lower
    uint64_t *to;
    uint32_t *hist, *totals, *valid;                       // [tiles][digits], [digits], one word
    uint32_t n, rows, tiles, shift, bits;
};

template <bool FIRST> __device__ __forceinline__ uint64_t entry(const Sort &a, uint32_t i, uint32_t n) {
    if constexpr (FIRST) {
        const int32_t id = i < n ? a.ids[i] : -1;
        return (uint32_t)id < a.rows ? (uint64_t)(uint32_t)id << 32 | i : ~0ull;
    } else {
        return i < n ? a.from[i] : ~0ull;
    }
}
__device__ __forceinline__ uint32_t digit_of(const Sort &a, uint64_t e) {
    return (uint32_t)(e >> (32 + a.shift)) & ((1u << a.bits) - 1);
}

// How many of a tile's entries have each digit.
template <bool FIRST, int kItems> __global__ __launch_bounds__(kSortThreads) void count_digits(Sort a) {
    constexpr uint32_t kTile = kSortThreads * kItems;
    __shared__ uint32_t count[kMaxDigits];
    const uint32_t digits = 1u << a.bits, n = FIRST ? a.n : *a.valid;
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) count[d] = 0;
    __syncthreads();
    uint64_t e[kItems];
#pragma unroll
    for (int i = 0; i < kItems; i++) e[i] = entry<FIRST>(a, blockIdx.x * kTile + i * kSortThreads + threadIdx.x, n);
#pragma unroll
    for (int i = 0; i < kItems; i++)
        if (e[i] != ~0ull) atomicAdd(&count[digit_of(a, e[i])], 1u);
    __syncthreads();
    for (uint32_t d = threadIdx.x; d < digits; d += kSortThreads) a.hist[((size_t)blockIdx.x << a.bits) + d] = count[d];
}

// The sum of x over the workgroup's threads before this one; `all` that of all.
__device__ __forceinline__ uint32_t sum_before(uint32_t x, uint32_t &all, uint32_t *lds) {
    const uint32_t lane = threadIdx.x % 64, waves = blockDim.x / 64;
    uint32_t s = x;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t y = __shfl_up(s, o);
        if (lane >= (uint32_t)o) s += y;
    }
    __syncthreads();
    if (lane == 63) lds[threadIdx.x / 64] = s;
    __syncthreads();
    uint32_t w = lane < waves ? lds[lane] : 0;             // of wavefronts, at most 16
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
        const uint32_t y = __shfl_up(w, o);
        if (lane >= (uint32_t)o) w += y;
    }
    all = __shfl(w, waves - 1);
    const uint32_t before = threadIdx.x / 64 ? __shfl(w, threadIdx.x / 64 - 1) : 0;
    return before + s - x;
}

// A digit's counts become those of the tiles before each; their sum goes to
// totals.  16 digits a workgroup, 64 threads each, a stretch of the tiles a thread.
__global__ __launch_bounds__(1024) void scan_digits(Sort a) {
    __shared__ uint32_t sums[64][17];
    const uint32_t c = threadIdx.x % 16, t = threadIdx.x / 16, d = blockIdx.x * 16 + c, digits = 1u << a.bits;
    const uint32_t per = (a.tiles + 63) / 64, t0 = min(t * per, a.tiles), t1 = d < digits ? min(t0 + per, a.tiles) : t0;
    uint32_t *h = a.hist + d;
    uint32_t sum = 0;
    for (uint32_t k = t0; k < t1; k += 8) {
        uint32_t x[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) x[i] = k + i < t1 ? h[(size_t)(k + i) << a.bits] : 0;
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) sum += x[i];
    }
    sums[t][c] = sum;
    __syncthreads();
    uint32_t at = 0, all = 0;
#pragma unroll 16
    for (uint32_t i = 0; i < 64; i++) {
        const uint32_t x = sums[i][c];
        at += i < t ? x : 0;
        all += x;
    }
    for (uint32_t k = t0; k < t1; k += 8) {
        uint32_t x[8];
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) x[i] = k + i < t1 ? h[(size_t)(k + i) << a.bits] : 0;
#pragma unroll
        for (uint32_t i = 0; i < 8; i++) {
            if (k + i < t1) h[(size_t)(k + i) << a.bits] = at;
            at += x[i];
        }
    }
    if (t == 0 && d < digits) a.totals[d] = all;
}

// Each entry's rank among its wavefront's entries of its digit, in their order;
// `counts` gets how many there are of each.
template <int kItems>
__device__ __forceinline__ void rank_digits(const Sort &a, const uint64_t (&e)[kItems], uint16_t *counts,
                                            uint32_t (&rank)[kItems]) {
    const uint32_t lane = threadIdx.x % 64;
#pragma unroll
    for (int i = 0; i < kItems; i++) {
        const bool there = e[i] != ~0ull;
        const uint32_t d = there ? digit_of(a, e[i]) : 0;
        uint64_t same = __ballot(there);
        for (uint32_t b = 0; b < a.bits; b++) {
            const uint64_t one = __ballot(d >> b & 1);
            same &= d >> b & 1 ? one : ~one;
        }
        const uint32_t before = __popcll(same & ((1ull << lane) - 1));
        volatile uint16_t *count = counts + d;
        const uint32_t c = there ? *count : 0;
        rank[i] = c + before;
        if (there && before == 0) *count = (uint16_t)(c + __popcll(same));
    }
}

// Each entry of a tile to its place: behind all of lower digits, the earlier
// tiles' of its own and the earlier of its own in the tile.  The tile is put in
// order in LDS first, so that neighbours go out together.
template <bool FIRST, int kItems> __global__ __launch_bounds__(kSortThreads) void scatter(Sort a) {
    constexpr uint32_t kTile = kSortThreads * kItems;
    __shared__ uint64_t items[kTile];
    __shared__ uint16_t waves[kWaves][kMaxDigits];
    __shared__ uint32_t start[kMaxDigits], base[kMaxDigits], lds[kWaves];
    const uint32_t digits = 1u << a.bits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t n = FIRST ? a.n : *a.valid;
    if (!FIRST && blockIdx.x * kTile >= n) return;
    for (uint32_t d = threadIdx.x; d < kWaves * kMaxDigits; d += kSortThreads) waves[d / kMaxDigits][d % kMaxDigits] = 0;
    uint64_t e[kItems];
#pragma unroll
    for (int i = 0; i < kItems; i++)
        e[i] = entry<FIRST>(a, blockIdx.x * kTile + (wave * kItems + i) * 64 + lane, n);
    const uint32_t total = threadIdx.x < digits ? a.totals[threadIdx.x] : 0;
    const uint32_t earlier = threadIdx.x < digits ? a.hist[((size_t)blockIdx.x << a.bits) + threadIdx.x] : 0;
    __syncthreads();
    uint32_t rank[kItems];
    rank_digits<kItems>(a, e, waves[wave], rank);
    __syncthreads();
    // a digit a thread: its counts' sums over wavefronts, digits and tiles
    uint32_t sum = 0, all, total_all;
    const uint32_t mine = threadIdx.x;
    if (mine < digits) {
#pragma unroll
        for (int w = 0; w < kWaves; w++) {
            const uint32_t c = waves[w][mine];
            waves[w][mine] = (uint16_t)sum;
            sum += c;
        }
    }
    const uint32_t at = sum_before(sum, all, lds), to = sum_before(total, total_all, lds);
    if (FIRST && blockIdx.x == 0 && threadIdx.x == 0) *a.valid = total_all;
    if (mine < digits) {
        start[mine] = at;
        base[mine] = to + earlier - at;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kItems; i++) {
        if (e[i] == ~0ull) continue;
        const uint32_t d = digit_of(a, e[i]);
        items[start[d] + waves[wave][d] + rank[i]] = e[i];
    }
    __syncthreads();
    for (uint32_t p = threadIdx.x; p < all; p += kSortThreads) {
        const uint64_t x = items[p];
        a.to[base[digit_of(a, x)] + p] = x;
    }
}

// All passes of a call of up to 4096 ids, in one workgroup, in place of three
// launches each (the rows that occur of 4000 ids, three passes: 44 us a call, of
// 5000 ids, by launches: 55).
constexpr uint32_t kSmall = kSortThreads * 8;
template <int kItems> __global__ __launch_bounds__(kSortThreads) void sort_small(Sort a, uint32_t passes) {
    __shared__ uint64_t items[kSortThreads * kItems];
    __shared__ uint16_t waves[kWaves][kMaxDigits];
    __shared__ uint32_t start[kMaxDigits], lds[kWaves];
    const uint32_t digits = 1u << a.bits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint64_t e[kItems];
#pragma unroll
    for (int i = 0; i < kItems; i++) e[i] = entry<true>(a, (wave * kItems + i) * 64 + lane, a.n);
    uint32_t all = 0;
    for (uint32_t p = 0; p < passes; p++) {
        a.shift = p * a.bits;
        for (uint32_t d = threadIdx.x; d < kWaves * kMaxDigits; d += kSortThreads) waves[d / kMaxDigits][d % kMaxDigits] = 0;
        __syncthreads();
        uint32_t rank[kItems], sum = 0;
        rank_digits<kItems>(a, e, waves[wave], rank);
        __syncthreads();
        const uint32_t mine = threadIdx.x;
        if (mine < digits) {
#pragma unroll
            for (int w = 0; w < kWaves; w++) {
                const uint32_t c = waves[w][mine];
                waves[w][mine] = (uint16_t)sum;
                sum += c;
            }
        }
        const uint32_t at = sum_before(sum, all, lds);
        if (mine < digits) start[mine] = at;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kItems; i++) {
            if (e[i] == ~0ull) continue;
            const uint32_t d = digit_of(a, e[i]);
            items[start[d] + waves[wave][d] + rank[i]] = e[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kItems; i++) {
            const uint32_t at = (wave * kItems + i) * 64 + lane;
            e[i] = at < all ? items[at] : ~0ull;
        }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kItems; i++)
        if (e[i] != ~0ull) a.to[(wave * kItems + i) * 64 + lane] = e[i];
    if (threadIdx.x == 0) *a.valid = all;
}

// ---------------------------------------------------------------- sums
struct Sums {
    const uint8_t *dout;
    uint8_t *out;
    int64_t dout_row, out_row;                             // bytes
    const uint64_t *sorted;
    const uint32_t *valid;
    float *part;                                           // [runs][2][width]
    int32_t *list;                                         // NULL: rows go to their ids
    uint32_t *heads, *blocks;                              // [runs], [their blocks + 1]: rows that begin before
    uint32_t *count;
    uint32_t n, width, lanes, run, runs;
    float scale;
};

__device__ __forceinline__ uint32_t id_at(const Sums &a, uint32_t i) { return (uint32_t)(a.sorted[i] >> 32); }

// How many rows begin in the runs before each, within the workgroup's 64 runs
// (16 lanes each), and in all of those.
constexpr uint32_t kBlock = 64;
__global__ __launch_bounds__(1024) void count_heads(Sums a) {
    __shared__ uint32_t count[kBlock];
    const uint32_t n = *a.valid, r = blockIdx.x * kBlock + threadIdx.x / 16, lane = threadIdx.x % 16;
    uint32_t k = 0;
#pragma unroll 4
    for (uint32_t i = lane; i < a.run && r < a.runs; i += 16) {
        const uint32_t j = r * a.run + i;
        if (j < n && (j == 0 || id_at(a, j) != id_at(a, j - 1))) k++;
    }
    for (int o = 8; o; o /= 2) k += __shfl_xor(k, o);
    if (lane == 0) count[threadIdx.x / 16] = k;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    k = count[threadIdx.x];
    uint32_t sum = k;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t y = __shfl_up(sum, o);
        if (threadIdx.x >= (uint32_t)o) sum += y;
    }
    const uint32_t at = blockIdx.x * kBlock + threadIdx.x;
    if (at < a.runs) a.heads[at] = sum - k;
    if (threadIdx.x == 63) a.blocks[blockIdx.x] = sum;
}

// The blocks' counts become those of the blocks before each; behind the last,
// all of them.
__global__ __launch_bounds__(1024) void scan_blocks(Sums a) {
    __shared__ uint32_t lds[16];
    const uint32_t blocks = (a.runs + kBlock - 1) / kBlock;
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < blocks; b0 += 1024) {
        const uint32_t b = b0 + threadIdx.x, x = b < blocks ? a.blocks[b] : 0;
        uint32_t all;
        const uint32_t at = before + sum_before(x, all, lds);
        if (b < blocks) a.blocks[b] = at;
        before += all;
    }
    if (threadIdx.x == 0) {
        a.blocks[blocks] = before;
        *a.count = before;
    }
}

// Rows that begin in the runs before r (all of them behind the last run).
__device__ __forceinline__ uint32_t heads_before(const Sums &a, uint32_t r) {
    return r < a.runs ? a.heads[r] + a.blocks[r / kBlock] : a.blocks[(a.runs + kBlock - 1) / kBlock];
}

// Whether the entry at place `at` is one of row `id`.
__device__ __forceinline__ bool goes_on(const Sums &a, uint32_t id, uint32_t at, uint32_t n) {
    return at < n && id_at(a, at) == id;
}

// A group of lanes sums the rows that begin in its run.  One that ends in the next
// run is summed to its end there; one that goes on behind the next run is summed in
// parts: `tail`, this run's part of a row that begins in it, and in the runs behind
// it `head`, their parts of a row that began before (join_parts finds the same rows
// by the same two places, the first ones of the next run and of the run behind it).
template <typename T> __global__ __launch_bounds__(kThreads) void sum_runs(Sums a) {
    constexpr int N = Chunk<T>::n, U = 8;
    const uint32_t n = *a.valid, lane = threadIdx.x % a.lanes;
    const uint32_t r = blockIdx.x * (kThreads / a.lanes) + threadIdx.x / a.lanes;
    const uint32_t c = (blockIdx.y * a.lanes + lane) * N;
    if (r >= a.runs) return;
    const uint32_t begin = r * a.run, end = min(begin + a.run, n);
    uint32_t slot = 0;
    if (a.list) {
        slot = heads_before(a, r);
        const uint32_t all = heads_before(a, a.runs);
        if (blockIdx.y == 0)                               // behind the last row's id
            for (uint32_t i = begin + lane; i < begin + a.run && i < a.n; i += a.lanes)
                if (i >= all) a.list[i] = -1;
    }
    if (begin >= n) return;
    uint32_t id = id_at(a, begin), i = begin, stop = end;
    bool head = begin > 0 && id_at(a, begin - 1) == id, tail = false;
    if (head) {
        // in parts if it goes on behind this run, or began before the last one
        const bool parts = goes_on(a, id, end, n) && end == begin + a.run;
        if (!parts && !(begin > a.run && id_at(a, begin - a.run - 1) == id)) {
            // the run before has summed it to its end
            for (uint32_t step = end - i; step;) {         // the first place behind it
                const uint32_t half = step / 2;
                if (id_at(a, i + half) == id) i += half + 1, step -= half + 1;
                else step = half;
            }
            head = false;
        }
    }
    if (i >= end) return;
    const uint32_t last = id_at(a, end - 1);
    if (goes_on(a, last, end, n) && !(head && last == id)) {
        const uint32_t far = min(end + a.run, n);
        tail = far == end + a.run && goes_on(a, last, far, n);
        if (!tail) {
            stop = end;
            for (uint32_t step = far - end; step;) {
                const uint32_t half = step / 2;
                if (id_at(a, stop + half) == last) stop += half + 1, step -= half + 1;
                else step = half;
            }
        }
    }
    float sum[N];
#pragma unroll
    for (int k = 0; k < N; k++) sum[k] = 0.0f;
    id = id_at(a, i);
    const auto leave_part = [&](int which) {
        float *p = a.part + ((size_t)r * 2 + which) * a.width;
#pragma unroll
        for (int k = 0; k < N; k++)
            if (c + k < a.width) p[c + k] = sum[k];
    };
    const auto leave = [&](uint32_t id) {
        if (c < a.width)
            store_chunk<T>(a.out + (int64_t)(a.list ? slot : id) * a.out_row, c, a.width, packed<T>(sum, a.scale));
        if (a.list) {
            if (c == 0) a.list[slot] = (int32_t)id;
            slot++;
        }
    };
    uint64_t e[U], ahead[U];
#pragma unroll
    for (int u = 0; u < U; u++) ahead[u] = a.sorted[min(i + u, stop - 1)];
    for (; i < stop; i += U) {
        u32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; u++) e[u] = ahead[u];
#pragma unroll
        for (int u = 0; u < U; u++) {
            x[u] = u32x4{0, 0, 0, 0};
            if (i + u < stop && c < a.width) x[u] = load_chunk<T>(a.dout + (int64_t)(uint32_t)e[u] * a.dout_row, c, a.width);
        }
#pragma unroll
        for (int u = 0; u < U; u++) ahead[u] = a.sorted[min(i + U + u, stop - 1)];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const uint32_t now = (uint32_t)(e[u] >> 32);
            if (now != id) {
                if (head) leave_part(0);
                else leave(id);
                head = false;
                id = now;
#pragma unroll
                for (int k = 0; k < N; k++) sum[k] = 0.0f;
            }
            float f[N];
            unpack<T>(x[u], f);
            if (i + u < stop)
#pragma unroll
                for (int k = 0; k < N; k++) sum[k] += f[k];
        }
    }
    if (head) leave_part(0);
    else if (tail) leave_part(1);
    else leave(id);
}

// Rows that were summed in parts: a workgroup looks at 32 runs and joins the
// rows that begin in them: a wavefront each those of up to 64 parts more, all of
// them together the longer ones; groups of lanes take a stretch of the parts
// each, whose sums are added in order.
constexpr uint32_t kLook = 32, kJoinThreads = 1024;

// The sum over parts p0 to p1 - 1 of the row that begins in run `first`: the
// run's second part, then the first ones of the runs behind it.
template <int N>
__device__ __forceinline__ void add_parts(const Sums &a, uint32_t first, uint32_t p0, uint32_t p1, uint32_t c,
                                          float (&sum)[N]) {
    constexpr int U = 8;
#pragma unroll
    for (int i = 0; i < N; i++) sum[i] = 0.0f;
    for (uint32_t p = p0; p < p1; p += U) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const float *f = a.part + ((size_t)(first + p + u) * 2 + (p + u == 0)) * a.width + c;
            if (c + N <= a.width) {
#pragma unroll
                for (int i = 0; i < N; i += 4) {
                    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
                    if (p + u < p1) v = *(const f32x4_at4 *)(f + i);
                    x[u][i] = v[0], x[u][i + 1] = v[1], x[u][i + 2] = v[2], x[u][i + 3] = v[3];
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; i++) x[u][i] = p + u < p1 && c + i < a.width ? f[i] : 0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int i = 0; i < N; i++) sum[i] += x[u][i];
    }
}

template <typename T> __global__ __launch_bounds__(kJoinThreads) void join_parts(Sums a) {
    constexpr int N = Chunk<T>::n;
    __shared__ uint32_t found[kLook], number, large[kLook], larges, reach;
    __shared__ float sums[kJoinThreads][N + 1];
    const uint32_t n = *a.valid, r = blockIdx.x * kLook + threadIdx.x;
    if (blockIdx.x * kLook * a.run >= n) return;
    if (threadIdx.x == 0) number = larges = 0;
    __syncthreads();
    if (threadIdx.x < kLook && r < a.runs && (uint64_t)(r + 2) * a.run < n) {
        const uint32_t begin = r * a.run, end = begin + a.run, id = id_at(a, end - 1);
        // the run's last row: begins in this run, and goes on behind the next
        const bool from_before = id_at(a, begin) == id && begin > 0 && id_at(a, begin - 1) == id;
        if (!from_before && id_at(a, end) == id && id_at(a, end + a.run) == id) found[atomicAdd(&number, 1u)] = r;
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x % a.lanes, c = (blockIdx.y * a.lanes + lane) * N;
    const auto leave = [&](uint32_t first, uint32_t id, const float (&sum)[N]) {
        const uint32_t row = a.list ? heads_before(a, first + 1) - 1 : id;
        store_chunk<T>(a.out + (int64_t)row * a.out_row, c, a.width, packed<T>(sum, a.scale));
        if (a.list && c == 0) a.list[row] = (int32_t)id;
    };
    const auto in_run = [&](uint64_t q, uint32_t id) {
        return q < a.runs && q * a.run < n && id_at(a, (uint32_t)q * a.run) == id;
    };
    for (uint32_t k = threadIdx.x / 64; k < number; k += kJoinThreads / 64) {
        const uint32_t first = found[k], id = id_at(a, first * a.run + a.run - 1), in_wave = threadIdx.x % 64;
        const uint32_t more = __popcll(__ballot(in_run((uint64_t)first + 1 + in_wave, id)));
        if (more == 64) {
            if (in_wave == 0) large[atomicAdd(&larges, 1u)] = first;
            continue;
        }
        const uint32_t groups = 64 / a.lanes, per = (more + groups) / groups, p0 = in_wave / a.lanes * per;
        float sum[N];
        add_parts<N>(a, first, min(p0, more + 1), min(p0 + per, more + 1), c, sum);
        for (uint32_t g = 1; g < groups; g++)
#pragma unroll
            for (int i = 0; i < N; i++) {
                const float x = __shfl(sum[i], (in_wave + g * a.lanes) % 64);
                if (in_wave < a.lanes) sum[i] += x;
            }
        if (in_wave < a.lanes && c < a.width) leave(first, id, sum);
    }
    __syncthreads();
    const uint32_t group = threadIdx.x / a.lanes, groups = kJoinThreads / a.lanes;
    for (uint32_t k = 0; k < larges; k++) {
        const uint32_t first = large[k], id = id_at(a, first * a.run + a.run - 1);
        // the last run that holds it, as many tried at once as there are threads
        uint32_t last = first + 1, step = (a.runs - first + kJoinThreads - 1) / kJoinThreads;
        for (;; step = (step + kJoinThreads - 1) / kJoinThreads) {
            if (threadIdx.x == 0) reach = 0;
            __syncthreads();
            if (in_run((uint64_t)last + (uint64_t)step * threadIdx.x, id)) atomicMax(&reach, threadIdx.x);
            __syncthreads();
            last += step * reach;
            __syncthreads();
            if (step == 1) break;
        }
        const uint32_t parts = last - first + 1, per = (parts + groups - 1) / groups;
        float sum[N];
        add_parts<N>(a, first, min(group * per, parts), min(group * per + per, parts), c, sum);
#pragma unroll
        for (int i = 0; i < N; i++) sums[threadIdx.x][i] = sum[i];
        __syncthreads();
        if (group == 0 && c < a.width) {
            for (uint32_t g = 1; g < groups; g++)
#pragma unroll
                for (int i = 0; i < N; i++) sum[i] += sums[g * a.lanes + lane][i];
            leave(first, id, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host
uint32_t chunks_of(uint32_t width, int32_t dtype) {
    const uint32_t n = dtype == NLB_DTYPE_BF16 ? 8 : 4;
    return (width + n - 1) / n;
}

// Passes and the bits of each for ids below `rows`.
void passes_of(uint32_t rows, uint32_t &passes, uint32_t &bits) {
    uint32_t all = 1;
    while (all < 31 && (1ull << all) < rows) all++;
    passes = (all + kMaxBits - 1) / kMaxBits;
    bits = (all + passes - 1) / passes;
}

// Places a run: enough runs to fill the card, few enough that popular rows have
// few parts (3 000 000 places: runs of 256 228 us for the sums, of 64 172; 240 000:
// runs of 16 26 us and 32 to join, of 32 27 and 15).
uint32_t run_of(uint32_t n) {
    uint32_t run = 16;
    while (run < 64 && run < n / 8192) run *= 2;
    return run;
}

size_t align16z(size_t n) { return (n + 15) & ~(size_t)15; }

struct Work {                                              // places in the working memory
    size_t pairs[2], hist, totals, valid, heads, blocks, part, all;
    uint32_t tiles, passes, bits, run, runs;
    Work(const nlb_lookup_call *c, bool listed) {
        passes_of(c->rows, passes, bits);
        tiles = (uint32_t)(((uint64_t)c->n + tile_of(c->n) - 1) / tile_of(c->n));
        run = run_of(c->n);
        runs = (uint32_t)(((uint64_t)c->n + run - 1) / run);
        size_t at = 0;
        const auto take = [&](size_t n) {
            const size_t p = at;
            at += align16z(n);
            return p;
        };
        for (size_t &p : pairs) p = take((size_t)c->n * 8);
        hist = take(((size_t)tiles << bits) * 4);
        totals = take(4ull << bits);
        valid = take(4);
        heads = take(listed ? (size_t)runs * 4 : 0);
        blocks = take(listed ? ((runs + kBlock - 1) / kBlock + 1) * 4ull : 0);
        part = take((size_t)runs * 2 * c->width * 4);
        all = at;
    }
};

int check(const nlb_lookup_call *c) {
    if (!c || (c->dtype != NLB_DTYPE_F32 && c->dtype != NLB_DTYPE_BF16)) return NLB_EINVAL;
    if (c->width < 1 || c->width > NLB_LOOKUP_MAX_WIDTH || c->n > INT32_MAX || c->rows < 1 || c->rows > INT32_MAX)
        return NLB_EINVAL;
    if ((c->n && !c->ids) || (uintptr_t)c->ids % 4 || !std::isfinite(c->scale)) return NLB_EINVAL;
    return NLB_OK;
}

bool bad_rows(const void *p, int64_t stride, bool some, int32_t dtype) {
    return (some && !p) || (uintptr_t)p % (dtype == NLB_DTYPE_BF16 ? 2 : 4) || stride < 0 || stride > INT32_MAX;
}

Rows rows_of(const nlb_lookup_call *c, void *out, int64_t out_stride, uint32_t n) {
    Rows a = {};
    a.out = (uint8_t *)out;
    a.out_row = out_stride * (c->dtype == NLB_DTYPE_BF16 ? 2 : 4);
    a.ids = c->ids;
    a.n = n;
    a.rows = c->rows;
    a.width = (uint32_t)c->width;
    a.chunks = chunks_of(a.width, c->dtype);
    a.per = a.chunks < 4 * kThreads ? 4 * kThreads / a.chunks : 1;
    a.magic = nlb_div_magic(a.chunks);
    a.scale = c->scale;
    return a;
}

template <bool FILL> int copy(const Rows &a, int32_t dtype, hipStream_t s) {
    const uint32_t tiles = (uint32_t)(((uint64_t)a.n + a.per - 1) / a.per), blocks = tiles < 1u << 20 ? tiles : 1u << 20;
    if (!blocks) return NLB_OK;
    return enqueue(dtype == NLB_DTYPE_BF16 ? copy_rows<__bf16, FILL> : copy_rows<float, FILL>, blocks, kThreads, 0, s, a);
}

// Sorts; *sorted is where the pairs end up.
template <int ITEMS> int sort(const nlb_lookup_call *c, const Work &w, uint8_t *work, const uint64_t **sorted, hipStream_t s) {
    Sort a = {};
    a.ids = c->ids;
    a.hist = (uint32_t *)(work + w.hist);
    a.totals = (uint32_t *)(work + w.totals);
    a.valid = (uint32_t *)(work + w.valid);
    a.n = c->n;
    a.rows = c->rows;
    a.tiles = w.tiles;
    a.bits = w.bits;
    if (c->n <= kSmall) {
        a.to = (uint64_t *)(work + w.pairs[0]);
        *sorted = a.to;
        return enqueue(c->n <= 2 * kSortThreads ? sort_small<2> : sort_small<8>, 1, kSortThreads, 0, s, a, w.passes);
    }
    for (uint32_t p = 0; p < w.passes; p++) {
        a.shift = p * w.bits;
        a.from = (const uint64_t *)(work + w.pairs[(p + 1) % 2]);
        a.to = (uint64_t *)(work + w.pairs[p % 2]);
        int rc = enqueue(p ? count_digits<false, ITEMS> : count_digits<true, ITEMS>, w.tiles, kSortThreads, 0, s, a);
        if (rc == NLB_OK) rc = enqueue(scan_digits, ((1u << w.bits) + 15) / 16, 1024, 0, s, a);
        if (rc == NLB_OK) rc = enqueue(p ? scatter<false, ITEMS> : scatter<true, ITEMS>, w.tiles, kSortThreads, 0, s, a);
        if (rc != NLB_OK) return rc;
        *sorted = a.to;
    }
    return NLB_OK;
}

}  // namespace

extern "C" int nlb_lookup(const nlb_lookup_call *c, const void *table, int64_t table_stride, void *out,
                          int64_t out_stride, void *stream) {
    const int rc = check(c);
    if (rc != NLB_OK) return rc;
    if (bad_rows(table, table_stride, c->n, c->dtype) || bad_rows(out, out_stride, c->n, c->dtype)) return NLB_EINVAL;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    Rows a = rows_of(c, out, out_stride, c->n);
    a.table = (const uint8_t *)table;
    a.table_row = table_stride * (c->dtype == NLB_DTYPE_BF16 ? 2 : 4);
    return copy<false>(a, c->dtype, (hipStream_t)stream);
}

extern "C" int nlb_lookup_work(const nlb_lookup_call *c, int32_t listed, size_t *bytes) {
    if (!bytes) return NLB_EINVAL;
    const int rc = check(c);
    if (rc != NLB_OK) return rc;
    *bytes = Work(c, listed != 0).all;
    return NLB_OK;
}

extern "C" int nlb_lookup_backward(const nlb_lookup_call *c, const void *dout, int64_t dout_stride, void *dtable,
                                   int64_t dtable_stride, int32_t *list, uint32_t *count, void *work, size_t work_bytes,
                                   void *stream) {
    int rc = check(c);
    if (rc != NLB_OK) return rc;
    const bool listed = list || count;
    if (bad_rows(dout, dout_stride, c->n, c->dtype) || bad_rows(dtable, dtable_stride, !listed || c->n, c->dtype))
        return NLB_EINVAL;
    if (listed && ((c->n && !list) || !count)) return NLB_EINVAL;
    if (((uintptr_t)list | (uintptr_t)count) % 4 || (uintptr_t)work % 16) return NLB_EINVAL;
    const Work w(c, listed);
    if (w.all && (!work || work_bytes < w.all)) return NLB_ESCRATCH;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    const hipStream_t s = (hipStream_t)stream;
    if (!listed) {
        rc = copy<true>(rows_of(c, dtable, dtable_stride, c->rows), c->dtype, s);
        if (rc != NLB_OK || !c->n) return rc;
    }
    Sums a = {};
    a.dout = (const uint8_t *)dout;
    a.out = (uint8_t *)dtable;
    a.dout_row = dout_stride * (c->dtype == NLB_DTYPE_BF16 ? 2 : 4);
    a.out_row = dtable_stride * (c->dtype == NLB_DTYPE_BF16 ? 2 : 4);
    uint8_t *m = (uint8_t *)work;
    a.valid = (const uint32_t *)(m + w.valid);
    a.part = (float *)(m + w.part);
    a.list = list;
    a.heads = (uint32_t *)(m + w.heads);
    a.blocks = (uint32_t *)(m + w.blocks);
    a.count = count;
    a.n = c->n;
    a.width = (uint32_t)c->width;
    a.lanes = 4;
    const uint32_t chunks = chunks_of(a.width, c->dtype);
    while (a.lanes < 64 && a.lanes < chunks) a.lanes *= 2;
    a.run = w.run;
    a.runs = w.runs;
    a.scale = c->scale;
    if (c->n) rc = tile_of(c->n) == 2 * kSortThreads ? sort<2>(c, w, m, &a.sorted, s) : sort<8>(c, w, m, &a.sorted, s);
    if (rc == NLB_OK && listed) {
        if (c->n) rc = enqueue(count_heads, (w.runs + kBlock - 1) / kBlock, 1024, 0, s, a);
        if (rc == NLB_OK) rc = enqueue(scan_blocks, 1, 1024, 0, s, a);
    }
    if (rc != NLB_OK || !c->n) return rc;
    const bool bf16 = c->dtype == NLB_DTYPE_BF16;
    const uint32_t groups = kThreads / a.lanes, columns = (chunks + a.lanes - 1) / a.lanes;
    rc = enqueue(bf16 ? sum_runs<__bf16> : sum_runs<float>, dim3((w.runs + groups - 1) / groups, columns), kThreads, 0, s, a);
    if (rc != NLB_OK) return rc;
    return enqueue(bf16 ? join_parts<__bf16> : join_parts<float>, dim3((w.runs + kLook - 1) / kLook, columns),
                   kJoinThreads, 0, s, a);
}
