// attention.h -- what the attention kernels share: a call's arguments on the
// device, the packed sequences' tiles, the position bias, tile staging and the
// matrix products.  Private to libnlb.so.
//
// The mathematics, for query row i and key j of one sequence and one head:
//   t_ij = (scale q_i.k_j + bias[bucket(pos_i - pos_j)]) log2(e)
//   L_i  = log2 sum_j 2^t_ij over the open keys,  p_ij = 2^(t_ij - L_i)
//   o_i  = sum_j p_ij v_j
// Everything after the products of q and k works in powers of two (one
// hardware exponential); what a caller sees (lse) is natural.
//
// Matrix products.  Tiles are 32 x 32 matrix-core blocks.  A block of scores
// is computed transposed to its use: its columns (one per lane of a half
// wavefront) are the rows that a wavefront owns, its rows lie in registers,
// half a wavefront's registers holding rows 8 (r / 4) + 4 (half) + r % 4.
// Products that contract over those rows take the block as their right
// operand straight from the registers (any order of the contracted index
// serves, so the left operand is read in that order), and everything kept per
// owned row (running maximum, sum, log of the sum) is one value per lane.
// bf16 inputs run on 32x32x16 products, fp32 inputs on 32x32x2 fp32 products;
// sums are fp32.  The bf16 kernels round p and ds to bf16 for the products
// that contract over them (up to 2^-8 of each term, like the rounding of
// the result itself); sums and statistics take them unrounded.
#pragma once

#include <algorithm>

#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef int16_t i16x4 __attribute__((ext_vector_type(4)));
// 16 and 8 bytes of a row at its element's alignment (global accesses of any
// alignment are legal on gfx950).
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr uint32_t kNoKey = 0xFFFFFFFFu;
constexpr int32_t kNoKeyFlipped = INT32_MAX;
constexpr int kThreads = 256;            // four wavefronts, everywhere
constexpr int kOwned = 128;              // rows that a tiled workgroup owns, 32 per wavefront
constexpr int kMaxBuckets = NLB_ATT_MAX_BUCKETS;
constexpr uint32_t kMostRows = INT32_MAX - 1023;   // a tile past any row still has a 32-bit place
static_assert(kMaxBuckets == 64, "bucket_of takes six steps");
constexpr float kBiasCloses = -0x1p100f; // bias values at or below this close their bucket
constexpr float kBiasMost = 0x1p20f;     // others count as at most this in magnitude (see bias2_of)

struct Strided {
    const uint8_t *p;
    int64_t row, head;                   // bytes
};

// One call on the device.
struct Attend {
    Strided q, k, v, o, dout;            // o: written forward, read backward
    Strided dq, dk, dv;
    float *lse;                          // [q_rows][heads], natural
    float2 *stats;                       // [q_rows][heads]: log2 of the sum, and D
    const int32_t *q_start, *k_start;
    uint32_t batch, q_rows, k_rows, q_len, k_len;   // *_len: rows of every sequence where *_start is null
    uint32_t heads, kv_heads, group, dim;
    uint32_t causal, buckets, dtype_bytes;
    float scale, scale2, signed2;        // scale2: |scale| log2(e), 1 where scale is 0; signed2: scale log2(e)
    const int32_t *bounds;
    const void *bias;                    // [buckets][heads]
    const uint32_t *q_pos, *k_pos;
    float *part;                         // partial results (see the kernels)
    float *kpart;                        // [2][split][k_rows][kv_heads][dim rounded up to 4]: shares of dk, dv
    uint32_t slots, chunk, split;
    uint32_t first;                      // the launch's first workgroup (see enqueue_blocks)
};

struct Seq {
    uint32_t q0, k0;                     // first rows
    int32_t lq, lk;
    uint32_t tile;                       // the workgroup's tile in it
};

__device__ __forceinline__ uint32_t first_row(const int32_t *start, uint32_t len, uint32_t total, uint32_t b) {
    if (!start) return b * len;
    const int32_t s = start[b];
    return s < 0 ? 0u : min((uint32_t)s, total);
}

// A sequence's rows, whatever its start values say, lie inside its tensor.
__device__ __forceinline__ void sequence(const Attend &a, uint32_t b, Seq &s) {
    s.q0 = first_row(a.q_start, a.q_len, a.q_rows, b);
    s.lq = max(0, (int32_t)(first_row(a.q_start, a.q_len, a.q_rows, b + 1) - s.q0));
    s.k0 = first_row(a.k_start, a.k_len, a.k_rows, b);
    s.lk = max(0, (int32_t)(first_row(a.k_start, a.k_len, a.k_rows, b + 1) - s.k0));
}

// Packed sequences in tiles of n rows without a list of tiles: sequence b owns
// the slots from start[b] / n + b on, of which the next sequence's first
// leaves it at least as many as it has tiles (rounded up), so total / n +
// batch slots cover any lengths and the host need not know them.  The owner
// of a slot is found 64 candidates at a time.
__device__ __forceinline__ uint32_t slot_owner(const int32_t *start, uint32_t len, uint32_t total, uint32_t batch,
                                               uint32_t n, uint32_t slot, uint32_t &tile) {
    uint32_t lo = 0, hi = batch;
    const uint32_t lane = threadIdx.x & 63u;
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 63u) / 64u, b = lo + lane * step;
        const bool below = b < hi && first_row(start, len, total, b) / n + b <= slot;
        const uint64_t m = __ballot(below);
        if (!m) break;
        lo += (63u - (uint32_t)__builtin_clzll(m)) * step;
        hi = min(hi, lo + step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    tile = __builtin_amdgcn_readfirstlane(slot - (first_row(start, len, total, lo) / n + lo));
    return lo;
}

// ---------------------------------------------------------------- values
template <typename T> __device__ __forceinline__ float to_float(T x) { return (float)x; }

template <typename T> struct Chunk;      // 16 bytes of a row
template <> struct Chunk<__bf16> { static constexpr int n = 8; };
template <> struct Chunk<float> { static constexpr int n = 4; };

// Drops the first `gone` bytes (the same for all lanes) of a chunk.
template <typename T> __device__ __forceinline__ u32x4 drop_bytes(u32x4 x, uint32_t gone) {
    if (gone & 8) x = u32x4{x[2], x[3], 0, 0};
    if (gone & 4) x = u32x4{x[1], x[2], x[3], 0};
    if (sizeof(T) == 2 && (gone & 2))
        x = u32x4{__builtin_amdgcn_alignbit(x[1], x[0], 16), __builtin_amdgcn_alignbit(x[2], x[1], 16),
                  __builtin_amdgcn_alignbit(x[3], x[2], 16), x[3] >> 16};
    return x;
}

// 16 bytes from value c0 of a row of dim values, zeros past its end: a row's
// last chunk is loaded where the row ends, and moved.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const uint8_t *row, uint32_t c0, uint32_t dim) {
    constexpr uint32_t n = Chunk<T>::n;
    u32x4 x = {0, 0, 0, 0};
    if (c0 >= dim) return x;
    if (dim >= n) {
        x = *(const u32x4_any *)(row + min(c0, dim - n) * sizeof(T));
        if (dim % n) {
            const u32x4 y = drop_bytes<T>(x, (n - dim % n) * sizeof(T));
            if (c0 + n > dim) x = y;
        }
        return x;
    }
#pragma unroll
    for (uint32_t i = 0; i < n - 1; i++)
        if (i < dim) {
            if constexpr (sizeof(T) == 4) x[i] = ((const uint32_t *)row)[i];
            else x[i / 2] |= (uint32_t)((const uint16_t *)row)[i] << (16 * (i % 2));
        }
    return x;
}

template <typename T> __device__ __forceinline__ void unpack(u32x4 x, float (&f)[Chunk<T>::n]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; i++) f[i] = __uint_as_float(x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            f[2 * i] = __uint_as_float(x[i] << 16);
            f[2 * i + 1] = __uint_as_float(x[i] & 0xFFFF0000u);
        }
    }
}

// Values c0 .. c0 + n - 1 of a row of dim values (those past its end are not written).
template <typename T, int N>
__device__ __forceinline__ void store_values(uint8_t *row, uint32_t c0, uint32_t dim, const float (&f)[N]) {
    T v[N];
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = (T)f[i];
    T *p = (T *)row + c0;
    if (c0 + N <= dim) {
        if constexpr (N * sizeof(T) == 16) {
            u32x4 w;
            __builtin_memcpy(&w, v, 16);
            *(u32x4_any *)p = w;
        } else {
            static_assert(N * sizeof(T) == 8, "");
            u32x2 w;
            __builtin_memcpy(&w, v, 8);
            *(u32x2_any *)p = w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N - 1; i++)
            if (c0 + i < dim) p[i] = v[i];
    }
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_fast(float x) { return __builtin_amdgcn_logf(x); }

// A lane's value with the one of its column in the other half wavefront.
__device__ __forceinline__ float halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The sum over each group of N neighbouring lanes, in every lane of the group.
template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
template <int N> __device__ __forceinline__ float lanes_sum(float x) {
    if constexpr (N > 1) x = dpp_add<0xB1>(x);     // lane ^ 1
    if constexpr (N > 2) x = dpp_add<0x4E>(x);     // lane ^ 2
    if constexpr (N > 4) x = dpp_add<0x141>(x);    // the other half of eight (groups of 4 are equal by now)
    if constexpr (N > 8) x = dpp_add<0x140>(x);    // the other half of sixteen
    if constexpr (N > 16) x += __uint_as_float(__builtin_amdgcn_ds_swizzle(__float_as_uint(x), 0x401F));
    return x;
}

// ---------------------------------------------------------------- bias
// The gap between two positions, unsigned 32-bit values, clamped to int32
// (flipped positions are order-preserving signed ones).
__device__ __forceinline__ int32_t flip(uint32_t p) { return (int32_t)(p ^ 0x80000000u); }
__device__ __forceinline__ int32_t gap_of(int32_t qf, int32_t kf) { return __builtin_elementwise_sub_sat(qf, kf); }

// The bounds in LDS, padded to 64 with the largest value.
__device__ __forceinline__ uint32_t bucket_of(const int32_t *bounds, uint32_t buckets, int32_t gap) {
    uint32_t n = 0;
#pragma unroll
    for (uint32_t step = 32; step; step >>= 1)
        if (bounds[n + step - 1] <= gap) n += step;
    return min(n, buckets - 1);
}

// One head's bias in powers of two.  Scores and lse are fp32, so a row whose
// scores are of magnitude x has weights that are off by some 2^-22 x of
// themselves: at 2^20 by a quarter, at 2^31 (a mask of -1e9 is 2^30) by factors
// that no longer fit, and the row, with the gradients of all of its keys, would
// be infinite or zero.  So biases are held within 2^20: a row's weights change
// only where two of them beyond that lead it, or where all of its keys have one.
template <typename T> __device__ __forceinline__ float bias2_of(const Attend &a, uint32_t b, uint32_t head) {
    const float x = (float)((const T *)a.bias)[(size_t)b * a.heads + head];
    const float most = x > kBiasMost ? kBiasMost : x < -kBiasMost ? -kBiasMost : x;   // (NaN stays)
    return x <= kBiasCloses ? -INFINITY : most * kLog2e;
}

// The bounds of a workgroup's buckets and one head's bias as tiled kernels add
// it, to scores in steps of 1 / scale2.
template <typename T>
__device__ __forceinline__ void stage_bias(const Attend &a, uint32_t head, int32_t *bounds, float *bias) {
    for (uint32_t i = threadIdx.x; i < kMaxBuckets; i += kThreads) {
        if (bounds) bounds[i] = i + 1 < a.buckets ? a.bounds[i] : INT32_MAX;
        bias[i] = i < a.buckets ? bias2_of<T>(a, i, head) / a.scale2 : 0.0f;
    }
}

// Whether all gaps from lo to hi lie in the first or in the last bucket, and
// which it is.
__device__ __forceinline__ bool one_bucket(const int32_t *bounds, uint32_t buckets, int32_t lo, int32_t hi,
                                           uint32_t &bucket) {
    const bool last = buckets == 1 || lo >= bounds[buckets - 2], first = buckets > 1 && hi < bounds[0];
    bucket = last ? buckets - 1 : 0;
    return __builtin_amdgcn_readfirstlane(last || first);
}

// Buckets of many gaps.  The gaps are cut into cells, four to a power of two
// on either side of zero (by a gap's sign, exponent and two bits of its
// mantissa); a table in LDS has each cell's first bucket, and a gap takes as
// many further comparisons as the fullest cell has bounds (`more`; one or two
// for bounds in steps of one, then in equal ratios).  Against a search of six
// dependent LDS reads, two or three.
constexpr int kCells = 256;
__device__ __forceinline__ int32_t cell_of(int32_t gap) {
    // |gap| in fp32 rounds monotonically; 1 is cell 1, 2^31 cell 125
    const int32_t bits = (int32_t)(__float_as_uint(fabsf((float)gap)) >> 21) - 507;
    const int32_t n = max(bits, 0);
    return gap < 0 ? 128 - n : 128 + n;
}
struct Buckets {
    int32_t *bounds;                     // [64]
    uint8_t *cells;                      // [kCells]
    uint32_t last, more;                 // the last bucket; comparisons after a cell's first
};
// Fills the table; bounds are there, and `ends` has room for 64 words.  Ends
// with a barrier.
__device__ __forceinline__ void fill_cells(Buckets &t, int32_t *ends) {
    if (threadIdx.x < kMaxBuckets)
        ends[threadIdx.x] = threadIdx.x < t.last ? cell_of(t.bounds[threadIdx.x]) : INT32_MAX;
    __syncthreads();
    // bounds below cell c, and in it
    static_assert(kCells == kThreads, "a thread a cell");
    const int32_t c = threadIdx.x;
    uint32_t below = 0, upto = 0;
#pragma unroll
    for (uint32_t step = 32; step; step >>= 1) {
        if (ends[below + step - 1] < c) below += step;
        if (ends[upto + step - 1] <= c) upto += step;
    }
    t.cells[c] = (uint8_t)min(below, t.last);                 // (also where bounds do not increase)
    uint32_t in = upto - below;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) in = max(in, (uint32_t)__shfl_xor((int)in, w));
    __syncthreads();
    if (threadIdx.x % 64 == 0) ends[threadIdx.x / 64] = in;
    __syncthreads();
    t.more = __builtin_amdgcn_readfirstlane(max(max(ends[0], ends[1]), max(ends[2], ends[3])));
}
// The buckets of 16 gaps at once, so that each step's LDS reads overlap.
__device__ __forceinline__ void buckets_in(const Buckets &t, const int32_t (&gap)[16], uint32_t (&n)[16]) {
#pragma unroll
    for (int r = 0; r < 16; r++) n[r] = t.cells[cell_of(gap[r])];
    for (uint32_t i = 0; i < t.more; i++) {
        int32_t next[16];
#pragma unroll
        for (int r = 0; r < 16; r++) next[r] = t.bounds[min(n[r], (uint32_t)kMaxBuckets - 1)];
#pragma unroll
        for (int r = 0; r < 16; r++) n[r] += n[r] < t.last && next[r] <= gap[r] ? 1u : 0u;
    }
}

// ---------------------------------------------------------------- tiles
// Streamed rows of a tiled kernel, in LDS.  What pads a row depends on how the
// tile is read, 256 bytes a cycle: by rows (16 lanes read 16 bytes of 16
// rows: rows 16 bytes apart modulo 256 use every bank once), by columns (bf16:
// 32 lanes read 64 bytes of each of 4 rows; fp32: 128 bytes of rows 4 apart),
// or both ways, each at half speed.
enum Use { kByRows, kByColumns, kBothWays };

// NARROW: see Span.
template <typename T, int DP, Use USE, bool NARROW> struct Tile {
    typedef T Value;
    static constexpr bool narrow = NARROW;
    static constexpr int rows = NARROW ? 128 : sizeof(T) == 2 ? 64 : 32;
    static constexpr int chunks = DP * sizeof(T) / 16;              // per row
    static constexpr int pad = USE == kByRows ? 16 : USE == kBothWays || sizeof(T) == 4 ? 32 : DP == 32 ? 0 : 64;
    static constexpr int stride = DP * sizeof(T) + pad;             // bytes
    static constexpr int bytes = rows * stride;
    static constexpr int step = kThreads / chunks;                  // rows of one load of the workgroup
    static constexpr int per_thread = rows / step;
    static_assert(rows * chunks % kThreads == 0, "");
    typedef u32x4 Regs[per_thread];
    typedef uint32_t Positions[per_thread];
};

// What a workgroup owns and what its wavefronts take of a tile.  Usually it
// owns 128 rows, 32 a wavefront, every wavefront takes the whole tile, and the
// next tile is staged in a second buffer.  A NARROW workgroup owns 32 rows;
// tiles have 128 rows, a wavefront takes every fourth 32 of them, and their
// results are joined at the end: for sequences of few rows, and for calls of
// few workgroups, whose time is that of one workgroup's way along its tiles (37
// sequences of up to 1000 keys, two fp32 heads of 50: 207 and 62 us).
template <bool NARROW, int ROWS> struct Span {
    static constexpr int owned = NARROW ? 32 : kOwned;
    static constexpr int buffers = NARROW ? 1 : 2;
    static constexpr int rows = NARROW ? 32 : ROWS;                 // of a tile, a wavefront's
    static constexpr int blocks = rows / 32;
    uint32_t own, take;                  // a wavefront's first owned row, and first row of a tile
    __device__ __forceinline__ Span() {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        own = NARROW ? 0 : wave * 32;
        take = NARROW ? wave * 32 : 0;
    }
};

// The sum of the wavefronts' results, in the first one; lds: 3 DP 128 bytes
// that no wavefront reads any more.
template <int DP> __device__ __forceinline__ void join_waves(f32x16 (&acc)[DP / 32], float *lds) {
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    if (wave)
#pragma unroll
        for (int i = 0; i < DP / 2; i++) lds[((wave - 1) * (DP / 2) + i) * 64 + lane] = acc[i / 16][i % 16];
    __syncthreads();
    if (wave == 0)
#pragma unroll
        for (int w = 0; w < 3; w++)
#pragma unroll
            for (int i = 0; i < DP / 2; i++) acc[i / 16][i % 16] += lds[(w * (DP / 2) + i) * 64 + lane];
}

// This thread's chunks of the tile whose first row is `base`, which has n > 0
// rows; rows from n on repeat the last one (their scores are masked, or their
// probabilities zero), so that the loads of a tile are nothing but loads (with
// a test for each chunk, vector operations for them took as long as the
// exponentials).  EXACT: a row is a whole number of chunks and a tile's rows
// lie within 2^31 bytes.  Else a row's last chunk is loaded where the row
// ends, and moved into place by tile_settle when it is staged.  Chunks past a
// row's end stay as tile_clear left them.
template <typename G> __device__ __forceinline__ void tile_clear(typename G::Regs &reg) {
#pragma unroll
    for (int i = 0; i < G::per_thread; i++) reg[i] = u32x4{0, 0, 0, 0};
}

template <typename G, bool EXACT>
__device__ __forceinline__ void tile_load(typename G::Regs &reg, const uint8_t *base, int64_t stride, int32_t n,
                                          uint32_t dim) {
    using T = typename G::Value;
    constexpr uint32_t N = Chunk<T>::n;
    const uint32_t c0 = threadIdx.x % G::chunks * N, r0 = threadIdx.x / G::chunks;
    if (c0 >= dim) return;
    if (EXACT || dim >= N) {
        const uint32_t at = (EXACT ? c0 : min(c0, dim - N)) * (uint32_t)sizeof(T);
        const auto load = [&](int i) {
            const uint32_t r = min(r0 + i * G::step, (uint32_t)n - 1);
            if constexpr (EXACT) reg[i] = *(const u32x4_any *)(base + (r * (uint32_t)stride + at));
            else reg[i] = *(const u32x4_any *)(base + (r * stride + at));
        };
        if (!G::narrow || n >= G::rows) {
#pragma unroll
            for (int i = 0; i < G::per_thread; i++) load(i);
        } else {
#pragma unroll
            for (int i = 0; i < G::per_thread; i++)
                if (i * G::step < n) load(i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < G::per_thread; i++)
            reg[i] = load_chunk<T>(base + min(r0 + i * G::step, (uint32_t)n - 1) * stride, 0, dim);
    }
}

// A row's last chunk, whose `dim % N` values were loaded as the last of N.
template <typename G> __device__ __forceinline__ void tile_settle(typename G::Regs &reg, uint32_t dim) {
    using T = typename G::Value;
    constexpr uint32_t N = Chunk<T>::n;
    const uint32_t c0 = threadIdx.x % G::chunks * N, gone = (N - dim % N) % N * sizeof(T);   // bytes to drop
    if (dim < N || gone == 0) return;
    const bool last = c0 < dim && c0 + N > dim;
#pragma unroll
    for (int i = 0; i < G::per_thread; i++) {
        const u32x4 x = drop_bytes<T>(reg[i], gone);
        if (last) reg[i] = x;
    }
}

// A narrow tile of n rows is written as far as wavefronts read it.
template <typename G> __device__ __forceinline__ void tile_store(uint8_t *lds, const typename G::Regs &reg, int32_t n) {
    const uint32_t c = threadIdx.x % G::chunks, r0 = threadIdx.x / G::chunks;
#pragma unroll
    for (int i = 0; i < G::per_thread; i++) {
        if (G::narrow && i * G::step >= (n + 31) / 32 * 32) break;
        *(u32x4 *)(lds + (r0 + i * G::step) * G::stride + c * 16) = reg[i];
    }
}

// The positions of the rows of this thread's chunks; from row n on none.
template <typename G>
__device__ __forceinline__ void tile_positions(typename G::Positions &pos, const uint32_t *p, int32_t n) {
    const uint32_t r0 = threadIdx.x / G::chunks;
#pragma unroll
    for (int i = 0; i < G::per_thread; i++) {
        const int32_t r = r0 + i * G::step;
        pos[i] = r < n ? p[r] : kNoKey;
    }
}

// Rows of closed keys may hold anything: they are multiplied as zeros.
template <typename G>
__device__ __forceinline__ void tile_close(typename G::Regs &reg, const typename G::Positions &pos) {
#pragma unroll
    for (int i = 0; i < G::per_thread; i++)
        if (pos[i] == kNoKey) reg[i] = u32x4{0, 0, 0, 0};
}

template <typename G>
__device__ __forceinline__ void tile_store_positions(int32_t *lds, const typename G::Positions &pos) {
    if (threadIdx.x % G::chunks == 0)
#pragma unroll
        for (int i = 0; i < G::per_thread; i++)
            lds[threadIdx.x / G::chunks + i * G::step] = flip(pos[i]);
}

// Owned rows as the right operand of products that contract over the row's
// values: lane (column c, half h) holds row c's values 16 s + 8 h + (0..7) of
// step s (bf16) or 8 s + 4 h + (0..3) (fp32): 16 bytes each.
template <typename T, int DP> struct Owned {
    static constexpr int steps = DP * sizeof(T) / 32;
    u32x4 x[steps];
};

// A score in steps of 1 / scale2: q (or k) takes the sign of scale, and zero.
template <typename T, int DP> __device__ __forceinline__ void sign_owned(Owned<T, DP> &f, float scale) {
    const uint32_t sign = scale < 0.0f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
    const uint32_t keep = scale == 0.0f ? 0u : 0xFFFFFFFFu;
#pragma unroll
    for (int s = 0; s < Owned<T, DP>::steps; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) f.x[s][i] = (f.x[s][i] ^ sign) & keep;
}

template <typename T, int DP>
__device__ __forceinline__ void load_owned(Owned<T, DP> &f, const uint8_t *row, bool there, uint32_t dim) {
    const uint32_t h = (threadIdx.x >> 5) & 1u;
#pragma unroll
    for (int s = 0; s < Owned<T, DP>::steps; s++) {
        f.x[s] = u32x4{0, 0, 0, 0};
        if (there) f.x[s] = load_chunk<T>(row, (2 * s + h) * Chunk<T>::n, dim);
    }
}

// acc[row][c] += sum over values of tile[blk + row] . owned[c]
template <typename G, typename T, int DP>
__device__ __forceinline__ void product_rows(f32x16 &acc, const uint8_t *tile, int blk, const Owned<T, DP> &own) {
    const uint32_t lane = threadIdx.x & 63u;
    const uint8_t *p = tile + (blk + (lane & 31u)) * G::stride + (lane >> 5) * 16;
#pragma unroll
    for (int s = 0; s < Owned<T, DP>::steps; s++) {
        const u32x4 x = *(const u32x4 *)(p + s * 32);
        if constexpr (sizeof(T) == 2) {
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x),
                                                          __builtin_bit_cast(bf16x8, own.x[s]), acc, 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x[e]), __uint_as_float(own.x[s][e]), acc, 0,
                                                           0, 0);
        }
    }
}

// A score block as the right operand of a product that contracts over its rows.
template <typename T> struct Scores;
template <> struct Scores<__bf16> { bf16x8 x[2]; };
template <> struct Scores<float> { float x[16]; };

__device__ __forceinline__ void pack(Scores<__bf16> &s, const float (&p)[16]) {
#pragma unroll
    for (int u = 0; u < 2; u++)
#pragma unroll
        for (int e = 0; e < 8; e++) s.x[u][e] = (__bf16)p[8 * u + e];
}
__device__ __forceinline__ void pack(Scores<float> &s, const float (&p)[16]) {
#pragma unroll
    for (int e = 0; e < 16; e++) s.x[e] = p[e];
}

// Four rows of one column of a row-major bf16 tile per lane, by the LDS
// transposing read: in each group of 16 lanes, lanes 4 r .. 4 r + 3 name the
// 16 columns of row r, and lane c gets column c of rows 0 .. 3.
__device__ __forceinline__ i16x4 read_columns(const uint8_t *p) {
    typedef __attribute__((address_space(3))) i16x4 *lds_ptr;
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)p);
}

// acc[d block][value][c] += sum over the block's rows of tile[blk + row][value] scores[row][c]
template <typename G, typename T, int D>
__device__ __forceinline__ void product_columns(f32x16 (&acc)[D], const uint8_t *tile, int blk, const Scores<T> &s) {
    const uint32_t lane = threadIdx.x & 63u, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
        const uint8_t *p = tile + (blk + 4 * h + ((lane & 15u) >> 2)) * G::stride +
                           (16 * ((lane >> 4) & 1u) + 4 * (lane & 3u)) * 2;
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int d = 0; d < D; d++) {
                const i16x4 lo = read_columns(p + (16 * u) * G::stride + d * 64);
                const i16x4 hi = read_columns(p + (16 * u + 8) * G::stride + d * 64);
                const auto x = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), s.x[u], acc[d], 0, 0,
                                                                 0);
            }
    } else {
        const uint8_t *p = tile + (blk + 4 * h) * G::stride + (lane & 31u) * 4;
#pragma unroll
        for (int r = 0; r < 16; r++)
#pragma unroll
            for (int d = 0; d < D; d++)
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                    *(const float *)(p + (8 * (r / 4) + r % 4) * G::stride + d * 128), s.x[r], acc[d], 0, 0, 0);
    }
}

// The transposed result of a wavefront's rows: acc[d][r] is value
// 32 d + 8 (r / 4) + 4 h + r % 4 of the lane's row.
template <typename T, int DP>
__device__ __forceinline__ void store_owned(uint8_t *row, uint32_t dim, const f32x16 (&acc)[DP / 32], float factor) {
    const uint32_t h = (threadIdx.x >> 5) & 1u;
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const float f[4] = {acc[d][r] * factor, acc[d][r + 1] * factor, acc[d][r + 2] * factor,
                                acc[d][r + 3] * factor};
            const uint32_t c = 32 * d + 2 * r + 4 * h;
            if (c < dim) store_values<T, 4>(row, c, dim, f);
        }
}

// Row r of a score block, of the lane's half.
__device__ __forceinline__ int block_row(int r) {
    return 8 * (r / 4) + 4 * ((threadIdx.x >> 5) & 1u) + r % 4;
}

// ---------------------------------------------------------------- lists
// How a row's values lie across lanes where rows are read one by one.
template <typename T, int DP> struct Lanes {
    static constexpr int per_row = DP / Chunk<T>::n;
    static constexpr int rows = 64 / per_row;
};
constexpr int kListKeys = 64;            // keys of a list whose open ones are looked up at once

// The positions of KEYS (64 at most) keys from j0 on of each lane group's list:
// a lane loads every PER-th.
template <int PER, int KEYS> struct ListPositions {
    uint32_t pos[KEYS / PER];
    __device__ __forceinline__ void load(const Attend &a, uint32_t k0, int32_t lk, int32_t j0) {
        const int32_t c = threadIdx.x % PER;
#pragma unroll
        for (int i = 0; i < KEYS / PER; i++) {
            const int32_t j = j0 + i * PER + c;
            pos[i] = j < lk ? (uint32_t)j : kNoKey;
            if (a.k_pos && j < lk) pos[i] = a.k_pos[k0 + j];
        }
    }
};

// The open keys among them as a bit mask in each lane of the group, and their
// buckets in codes[group][64]: each is searched once.
template <int PER, int KEYS>
__device__ __forceinline__ uint64_t open_keys(const Attend &a, const int32_t *bounds, uint8_t *codes,
                                              const ListPositions<PER, KEYS> &at, int32_t lk, int32_t j0,
                                              int32_t qpos) {
    const uint32_t lane = threadIdx.x & 63u, c = lane % PER, base = lane - c;
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < KEYS / PER; i++) {
        if (!__any(j0 + i * PER < lk)) break;
        const uint64_t m = __ballot(at.pos[i] != kNoKey);
        mine |= ((m >> base) & ((1ull << PER) - 1)) << (i * PER);
        if (a.buckets)
            codes[base / PER * kListKeys + i * PER + c] = bucket_of(bounds, a.buckets, gap_of(qpos, flip(at.pos[i])));
    }
    return mine;
}

// The LDS writes of the wavefront's lanes before its reads after.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// ---------------------------------------------------------------- host
// Rows of a call as the kernels take them.
inline int fill_rows(const nlb_att_call *c, const nlb_att_rows *r, bool needed, Strided &out) {
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (!r) return NLB_EINVAL;
    if (needed && !r->data) return NLB_EINVAL;
    if ((uintptr_t)r->data % e) return NLB_EINVAL;
    if (r->row_stride < 0 || r->head_stride < 0 || r->row_stride > INT32_MAX || r->head_stride > INT32_MAX)
        return NLB_EINVAL;
    out = {(const uint8_t *)r->data, r->row_stride * e, r->head_stride * e};
    return NLB_OK;
}

inline int fill_call(const nlb_att_call *c, Attend &a) {
    a = {};
    if (!c) return NLB_EINVAL;
    if (c->dtype != NLB_DTYPE_F32 && c->dtype != NLB_DTYPE_BF16) return NLB_EINVAL;
    if (c->dim < 1 || c->dim > NLB_ATT_MAX_DIM || c->heads < 1 || c->heads > NLB_ATT_MAX_HEADS) return NLB_EINVAL;
    if (c->kv_heads < 1 || c->heads % c->kv_heads) return NLB_EINVAL;
    const float size = std::fabs(c->scale);
    if (!(size == 0.0f || (size >= 0x1p-20f && size <= 0x1p20f))) return NLB_EINVAL;
    if (c->causal != 0 && c->causal != 1) return NLB_EINVAL;
    if (c->batch < 1 || c->batch > INT32_MAX / NLB_ATT_MAX_HEADS || c->q_rows > kMostRows || c->k_rows > kMostRows)
        return NLB_EINVAL;
    if ((!c->q_start && c->q_rows % c->batch) || (!c->k_start && c->k_rows % c->batch)) return NLB_EINVAL;
    if (c->buckets < 0 || c->buckets > NLB_ATT_MAX_BUCKETS) return NLB_EINVAL;
    if ((c->buckets > 0) != (c->bias != nullptr) || (c->buckets > 1 && !c->bounds)) return NLB_EINVAL;
    if (c->q_pos && !c->k_pos && c->k_rows) return NLB_EINVAL;
    if (c->buckets > 0 && !c->q_pos && c->k_pos && c->q_rows) return NLB_EINVAL;
    if (((uintptr_t)c->q_start | (uintptr_t)c->k_start | (uintptr_t)c->bounds | (uintptr_t)c->q_pos |
         (uintptr_t)c->k_pos) % 4)
        return NLB_EINVAL;
    if ((uintptr_t)c->bias % (c->dtype == NLB_DTYPE_BF16 ? 2 : 4)) return NLB_EINVAL;
    if (fill_rows(c, &c->q, c->q_rows > 0, a.q) != NLB_OK || fill_rows(c, &c->k, c->k_rows > 0, a.k) != NLB_OK ||
        fill_rows(c, &c->v, c->k_rows > 0, a.v) != NLB_OK)
        return NLB_EINVAL;
    a.q_start = c->q_start;
    a.k_start = c->k_start;
    a.batch = c->batch;
    a.q_rows = c->q_rows;
    a.k_rows = c->k_rows;
    a.q_len = c->q_rows / c->batch;
    a.k_len = c->k_rows / c->batch;
    a.heads = c->heads;
    a.kv_heads = c->kv_heads;
    a.group = c->heads / c->kv_heads;
    a.dim = c->dim;
    a.causal = c->causal;
    a.buckets = c->buckets;
    a.dtype_bytes = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    a.scale = c->scale;
    a.signed2 = c->scale * kLog2e;
    a.scale2 = c->scale == 0.0f ? 1.0f : std::fabs(c->scale) * kLog2e;
    a.bounds = c->bounds;
    a.bias = c->bias;
    a.q_pos = c->q_pos;
    a.k_pos = c->k_pos;
    return NLB_OK;
}

// Whether rows take the short form of tile_load.
inline bool exact_rows(const Attend &a, const Strided &r) {
    return a.dim * a.dtype_bytes % 16 == 0 && r.row <= 1 << 25;
}

// Kernels that take more LDS than 64 KiB need to be allowed it.
template <typename K> bool allow_lds(K kernel, uint32_t bytes) {
    if (bytes <= 65536) return true;
    if (hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess)
        return true;
    (void)hipGetLastError();
    return false;
}

// Starts `blocks` (2^31 - 1 at most) workgroups.  A launch holds fewer than
// 2^32 work items, so more than 2^24 - 1 workgroups (a million sequences with
// 16 heads) take several launches, each of which is told its first one.
inline int enqueue_blocks(void (*kernel)(Attend), Attend a, uint64_t blocks, uint32_t lds, hipStream_t stream) {
    constexpr uint64_t most = (1ull << 32) / kThreads - 1;
    for (uint64_t first = 0; first < blocks; first += most) {
        a.first = (uint32_t)first;
        const int rc = enqueue(kernel, (uint32_t)std::min(most, blocks - first), kThreads, lds, stream, a);
        if (rc != NLB_OK) return rc;
    }
    return NLB_OK;
}

inline size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

// Which kernels a call runs.
enum Form { kTiles, kOne, kLists };
constexpr uint64_t kNarrowBlocks = 128;

// Calls of tiles: narrow workgroups where sequences have 64 owned rows or fewer
// on average, or where the others are so few that half of the card idles (480
// of the others, 8 sequences of 128 to 2048 rows: 49 us, narrow 62).
inline bool narrow_tiles(const Attend &a, uint64_t rows, uint32_t heads) {
    if ((a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128) * a.dtype_bytes > 256) return false;   // (LDS)
    return rows / 64 <= a.batch || (rows / kOwned + 1) * heads <= kNarrowBlocks;
}

struct Forward {
    Form form;
    bool narrow;
    uint32_t chunk;                      // kOne: keys of a wavefront
    uint64_t slots, most;
    size_t bytes;
};

// One query row per sequence.  Many short lists take a group of lanes each
// (kLists), however long it is: the host knows the average length only, and a
// call waits for its longest list (see the header).  Else a wavefront takes a
// list (kOne), or where lists are too few to fill the card (8 wavefronts on each
// of 1024 SIMDs) a chunk of its keys, of 256 rows at least.  A chunk writes a
// group's heads of fp32 values, which the join reads again, for 512 rows of
// keys and values that it reads: group / 256 of the bytes for bf16, group / 512
// for fp32 rows, so 1.6 % at 4 heads on one, a quarter at 64.
// Lists times key/value heads from which a group of lanes each fills the card
// (4000 lists of 63 slots in two heads, bf16: 37 us, a wavefront each 28; 8000:
// 44 and 49; 6000 of 10 slots: 14 and 18).
constexpr uint64_t kManyLists = 8192;
inline bool short_lists(const Attend &a) { return a.k_rows / kListKeys <= a.batch; }

inline Forward plan_forward(const Attend &a) {
    Forward f = {};
    if (a.q_start || a.q_len != 1) {
        f.narrow = narrow_tiles(a, a.q_rows, a.heads);
        f.slots = (uint64_t)a.q_rows / (f.narrow ? 32 : kOwned) + a.batch;
        f.most = INT32_MAX / a.heads;
        return f;
    }
    f.most = INT32_MAX;
    f.slots = a.batch;
    f.form = kLists;
    if (short_lists(a) && (uint64_t)a.batch * a.kv_heads >= kManyLists) return f;
    f.form = kOne;
    const uint64_t even = ((uint64_t)a.k_rows * a.kv_heads + 8191) / 8192;
    f.chunk = (uint32_t)(((even < 256 ? 256 : even) + 63) / 64 * 64);
    const bool split = a.k_start ? a.k_rows > f.chunk : a.k_len > f.chunk;
    if (split) f.slots += (uint64_t)a.k_rows / f.chunk;
    f.bytes = split ? align256(f.slots * a.heads * (a.dim + 2) * 4) : 0;
    return f;
}

struct Backward {
    bool lists, narrow_rows, narrow_keys;
    uint32_t blocks, keep;               // kLists: workgroups; keys whose probabilities stay in LDS
    uint32_t shares;                     // shares of the first sum of bias gradients
    uint64_t q_slots, q_most, k_slots, k_most;
    uint32_t split;                      // workgroups that share a group's query heads
    uint64_t parts;                      // partial bias gradients
    size_t stat_bytes, part_bytes, bytes;
};

// Short lists with one query row, and longer ones where they are many, take a
// group of lanes each; a group's heads are in registers there, four at most.
// Everything else, single rows over long histories among it, goes through
// tiles.  Their second kernel spreads over the keys; the first gives a row and
// head to one workgroup, which walks all keys (bf16 rows twice) and sets the
// time where rows are few.
inline Backward plan_backward(const Attend &a) {
    Backward p = {};
    p.lists = !a.q_start && a.q_len == 1 && a.group <= 4 &&
              (short_lists(a) || (a.k_rows / 1024 <= a.batch && (uint64_t)a.batch * a.kv_heads >= kManyLists));
    if (p.lists) {
        const uint32_t n = a.dtype_bytes == 2 ? 8 : 4, dp = a.dim <= 32 ? 32 : a.dim <= 64 ? 64 : 128;
        const uint32_t rows = 64 / (dp / n), gb = a.group > 2 ? 4 : a.group;
        // every lane group keeps its key/value head: a whole number of heads in a turn of all groups
        uint32_t x = a.kv_heads, y = 4 * rows;
        while (y) {
            const uint32_t z = x % y;
            x = y;
            y = z;
        }
        const uint32_t unit = a.kv_heads / x, cap = (a.heads * a.buckets > 1024 ? 512 : 2048) / unit * unit;
        const uint64_t need = ((uint64_t)a.batch * a.kv_heads + 4 * rows - 1) / (4 * rows);
        p.blocks = (uint32_t)std::min<uint64_t>(cap, (need + unit - 1) / unit * unit);
        // (beside the other tables of a workgroup, which take 132 KiB at most)
        const uint32_t rest = kMaxBuckets * 4 + 8 + a.buckets * (a.heads + gb * 4 * rows) * 4 + 4 * rows * kListKeys;
        p.keep = std::min<uint32_t>(kListKeys, std::min(65536u, 155648u - rest) / (4 * rows * gb * 8));
        p.parts = p.blocks;
    } else {
        p.narrow_rows = narrow_tiles(a, a.q_rows, a.heads);
        p.narrow_keys = narrow_tiles(a, a.k_rows, a.heads);   // (a group's heads can be spread, see split)
        p.q_slots = (uint64_t)a.q_rows / (p.narrow_rows ? 32 : kOwned) + a.batch;
        p.k_slots = (uint64_t)a.k_rows / (p.narrow_keys ? 32 : kOwned) + a.batch;
        p.q_most = INT32_MAX / a.heads;
        p.k_most = INT32_MAX / a.heads;
        p.parts = a.q_rows ? p.q_slots : 0;
        p.stat_bytes = align256((size_t)a.q_rows * a.heads * 8);
        // Two workgroups of backward_keys run on a CU.  Where key tiles are too
        // few for two turns of them (which causal sequences of one length need
        // to even out), a group's heads are spread over workgroups, whose
        // shares of dk and dv are summed afterwards.
        const uint64_t tiles = p.k_slots * a.kv_heads;
        p.split = (uint32_t)std::min<uint64_t>(a.group, (1024 + tiles - 1) / tiles);
    }
    // (a workgroup a head sums 2048 partial gradients in 9 us; two steps take 10)
    p.shares = p.parts > 2048 ? 64 : 0;
    p.part_bytes = align256((p.parts + p.shares) * a.heads * a.buckets * 4);
    p.bytes = p.stat_bytes + p.part_bytes;
    if (p.split > 1) p.bytes += 2 * p.split * (size_t)a.k_rows * a.kv_heads * ((a.dim + 3) / 4) * 16;
    return p;
}

}  // namespace
