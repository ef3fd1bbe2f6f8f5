// gated_scan.hip -- gated linear recurrence over packed sequences, forward and
// backward.
//   z = sigmoid(g),  h_t = z_t h_{t-1} + (1 - z_t) x_t
//   d_t = dh_t + e_{t+1},  e_t = z_t d_t  (e past a sequence's end: dlast)
//   dx = (1 - z) d,  dg = z (1 - z) d (h_{t-1} - x),  dh0 = e at the first row
// A stretch of rows maps the state before it to A h + B, and two maps join to
// one: (A2 A1, A2 B1 + B2).  All sequences are one such scan over the call's
// rows, in which a sequence's first row forgets what came before it, so that
// neither their number nor their lengths matter to how the work is split.
//   A thread holds 16 (backward: 8) rows of its channels in registers, a workgroup's
// 4 wavefronts stand one below the other: maps of those rows are joined over the
// workgroup through LDS, then every thread walks its rows again, in registers.
// A workgroup walks a chunk of the rows tile by tile.  Where there are several
// chunks, a first launch makes their maps (it reads x and g once more, but only
// from the last first row in the chunk on), a second joins them.
// Measured: one sequence of a million rows of 128 bf16 values: 97 us for the maps
// (5.3 TB/s), 8 to join them, 149 for h (5.2 TB/s); 48 sequences of 16 to 4096
// rows of 1024: 33, 5 and 45 us, backward 29, 5 and 92; 20 000 of 1 to 60 rows of
// 100 fp32 values: 18, 6 and 105, backward 10, 6 and 215.  Forward, HBM bounds it
// (vector instructions: 0.73 to 0.83 of the cycles); backward of long sequences
// vector instructions (57 a value, 0.75); short sequences each tile's chain of loads.
#include <algorithm>
#include <type_traits>

#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef uint32_t u32_any __attribute__((aligned(2)));

constexpr int kThreads = 256, kRows = 16, kRowsBack = 8;   // rows a thread holds
constexpr uint32_t kStateRows = NLB_SCAN_STATE_ROWS, kChunks = 1024;

struct Scan {
    const uint8_t *x, *g, *dh;
    uint8_t *h, *dx, *dg;
    int64_t x_row, g_row, dh_row, h_row, dx_row, dg_row;   // bytes
    const int32_t *start;                                  // NULL: len rows each
    const float *h0, *dlast;
    float *last, *dh0, *states;
    float *maps, *into;                                    // [chunks][2][width], [chunks][width]
    uint32_t rows, width, batch, len;
    uint32_t lanes, chunk_rows, chunks, groups;            // lanes of a row, groups of them for all its channels
};

// A lane's channels of a row: one fp32 value, or two bf16 ones in a word.  The
// last bf16 value of an odd width comes in the upper half of the word that ends
// with it, and goes out by itself; a width of one has a type of its own.  bf16
// results go out past the caches, whose room the inputs can use, which are read
// twice (a million rows of 128 values: the first reading takes 118 us with
// ordinary stores, 97 so; fp32 rows of short lists are 2 % slower so).
struct OneBf16 {};
template <typename T> struct Piece;
template <> struct Piece<float> {
    static constexpr int n = 1;
    uint32_t off;
    bool there;
    __device__ __forceinline__ Piece(uint32_t c, uint32_t width) : off(c < width ? 4 * c : 0), there(c < width) {}
    __device__ __forceinline__ uint32_t load(const uint8_t *row) const { return *(const uint32_t *)(row + off); }
    __device__ __forceinline__ void unpack(uint32_t w, float (&f)[1]) const { f[0] = __uint_as_float(w); }
    __device__ __forceinline__ void store(uint8_t *row, const float (&f)[1]) const { *(float *)(row + off) = f[0]; }
};
template <> struct Piece<__bf16> {
    static constexpr int n = 2;
    uint32_t off, shift;
    bool there;
    __device__ __forceinline__ Piece(uint32_t c, uint32_t width) : there(c < width) {
        shift = c + 1 == width ? 16 : 0;
        off = there ? 2 * c - (shift ? 2 : 0) : 0;
    }
    __device__ __forceinline__ uint32_t load(const uint8_t *row) const { return *(const u32_any *)(row + off); }
    __device__ __forceinline__ void unpack(uint32_t w, float (&f)[2]) const {
        w >>= shift;
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xFFFF0000u);
    }
    __device__ __forceinline__ void store(uint8_t *row, const float (&f)[2]) const {
        __bf16 v[2] = {(__bf16)f[0], (__bf16)f[1]};
        uint32_t w;
        __builtin_memcpy(&w, v, 4);
        if (!shift) __builtin_nontemporal_store(w, (u32_any *)(row + off));
        else *(uint16_t *)(row + off + 2) = (uint16_t)w;
    }
};
template <> struct Piece<OneBf16> {
    static constexpr int n = 1;
    bool there;
    __device__ __forceinline__ Piece(uint32_t c, uint32_t width) : there(c < width) {}
    __device__ __forceinline__ uint32_t load(const uint8_t *row) const { return *(const uint16_t *)row; }
    __device__ __forceinline__ void unpack(uint32_t w, float (&f)[1]) const { f[0] = __uint_as_float(w << 16); }
    __device__ __forceinline__ void store(uint8_t *row, const float (&f)[1]) const { *(__bf16 *)row = (__bf16)f[0]; }
};

// Gates beyond 80 in magnitude become 80 (NaN stays): few calls have one, so a
// wavefront looks at the largest of its words' magnitudes first.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <typename T, int R> __device__ __forceinline__ void limit(uint32_t (&raw)[R]) {
    if constexpr (std::is_same<T, float>::value) {
        float most = 0.0f;
#pragma unroll
        for (int k = 0; k < R; k++) most = fmaxf(most, fabsf(__uint_as_float(raw[k])));
        if (!__any(most > 80.0f)) return;
#pragma unroll
        for (int k = 0; k < R; k++) {
            const float g = __uint_as_float(raw[k]);
            if (fabsf(g) > 80.0f) raw[k] = __float_as_uint(copysignf(80.0f, g));
        }
    } else {
        u16x2 most = {0, 0};
#pragma unroll
        for (int k = 0; k < R; k++) {
            const uint32_t w = raw[k] & 0x7FFF7FFFu;
            u16x2 v;
            __builtin_memcpy(&v, &w, 4);
            most = __builtin_elementwise_max(most, v);
        }
        if (!__any(most[0] > 0x42A0 || most[1] > 0x42A0)) return;
#pragma unroll
        for (int k = 0; k < R; k++)
#pragma unroll
            for (int i = 0; i < 32; i += 16) {
                const uint32_t m = raw[k] >> i & 0x7FFF;
                if (m > 0x42A0 && m <= 0x7F80) raw[k] = (raw[k] & ~(0x7FFFu << i)) | 0x42A0u << i;
            }
    }
}

// z = sigmoid(g) = 1 / (1 + e) and 1 - z = e z with e = exp(-g) = 2^t, t = -g / ln
// 2, |g| up to 80.  EXACT: e (1 + lo) with what t's rounding left, lo = -g - t ln 2,
// so that both have relative errors of some 2^-21.  Without it, for bf16 gates, t is
// off by 2^-24 (its rounding) and 2^-26 (its constant) of itself, and z and 1 - z by
// less than |g| 2^-23 more of themselves (z by less than 2^-24 absolutely): below the
// rounding of what goes out as bf16, and two operations of 14 less.  The states,
// which are fp32, have it too.
template <bool EXACT> __device__ __forceinline__ void gate(float g, float &z, float &y) {
    const float t = g * -1.44269504f;
    float e = __builtin_amdgcn_exp2f(t);
    if constexpr (EXACT) e = fmaf(e, fmaf(t, -0.693147181f, -g), e);
    z = __builtin_amdgcn_rcpf(1.0f + e);
    y = e * z;
}

// The map h -> a h + b of a stretch of rows.  A stretch that holds a first row
// (in the other direction: a last row) does not see the state before it: its
// a is -0, the sign telling it from a product that came to 0.
struct Map {
    float a, b;
    __device__ __forceinline__ float of(float h) const { return __float_as_int(a) < 0 ? b : fmaf(a, h, b); }
    // this stretch after `before`
    __device__ __forceinline__ Map after(Map before) const {
        if (__float_as_int(a) < 0) return *this;
        return {a * before.a, fmaf(a, before.b, b)};
    }
};
constexpr float kForgets = -0.0f;

struct Edges {                                             // of a tile's sequences, in LDS
    uint32_t begins[kThreads / 8], ends[kThreads / 8];     // a bit for each row, a word for a thread's rows
    int32_t begin[kThreads / 8 * kRows], end[kThreads / 8 * kRows];   // their sequences
    uint32_t next, s[kThreads], e[kThreads];               // the next tile's sequence; rows of those looked at
};

// The first row of sequence b, the rows' end for b = batch.
__device__ __forceinline__ uint32_t start_of(const Scan &a, uint32_t b) {
    if (!a.start) return b * a.len;
    const int32_t s = a.start[b];
    return s < 0 ? 0u : (uint32_t)s < a.rows ? (uint32_t)s : a.rows;
}

// The last sequence that begins at row r or before it (0 if none does): a
// wavefront tries 64 of them at once.
__device__ __forceinline__ uint32_t find_sequence(const Scan &a, uint32_t r) {
    if (!a.start) return r / a.len;
    uint32_t lo = 0, n = a.batch;
    const uint32_t lane = threadIdx.x % 64;
    for (;;) {
        const uint32_t step = (n + 63) / 64, i = lane * step;
        const bool before = i < n && a.start[lo + i] <= (int32_t)r;
        const uint32_t k = __popcll(__ballot(before));
        if (k > 1) lo += (k - 1) * step, n -= (k - 1) * step;
        if (step == 1) return __builtin_amdgcn_readfirstlane(lo);
        n = n < step ? n : step;
    }
}

// Walks the sequences along with the tiles (BACK: from the last one on).  b is
// the last sequence that begins at the tile's first row (BACK: its last row) or
// before it, s and e its rows; where they go beyond the tile to both sides, no
// edge is in it, and the tile needs no barrier for them.
template <int R, bool BACK> struct Cursor {
    uint32_t b, s, e;
    __device__ __forceinline__ void at(const Scan &a, uint32_t to) {
        b = to;
        s = __builtin_amdgcn_readfirstlane(start_of(a, b));
        e = __builtin_amdgcn_readfirstlane(start_of(a, b + 1));
    }
    __device__ __forceinline__ bool plain(uint32_t r0, uint32_t n) const { return s < r0 && e > r0 + n; }
    // This thread's share of the sequences that may have edges in the tile, a
    // workgroup of them from `from` on, and the last of these.
    struct Look {
        uint32_t from, i, s, e, last;
        bool more;
    };
    __device__ __forceinline__ void look(const Scan &a, uint32_t from, Look &l) const {
        l.from = from;
        l.i = BACK ? from - threadIdx.x : from + threadIdx.x;
        l.s = l.e = 0;
        if (l.i < a.batch) l.s = start_of(a, l.i), l.e = start_of(a, l.i + 1);
        l.more = from < a.batch && (BACK ? from >= kThreads - 1 : from + (kThreads - 1) < a.batch);
        l.last = l.more ? start_of(a, BACK ? from - (kThreads - 1) : from + (kThreads - 1)) : 0;
    }
    // Fills `edges`, whose words are 0 and whose `next` is 0, for the rows r0 ..
    // r0 + n - 1, and moves on to the next tile; ends with a barrier.
    __device__ __forceinline__ void find(const Scan &a, uint32_t r0, uint32_t n, Look &l, Edges &edges) {
        for (;;) {
            if (l.i < a.batch) {
                if (l.s < l.e && l.s - r0 < n) {
                    atomicOr(&edges.begins[(l.s - r0) / R], 1u << ((l.s - r0) % R));
                    edges.begin[l.s - r0] = l.i;
                }
                if (l.s < l.e && l.e - 1 - r0 < n) {
                    atomicOr(&edges.ends[(l.e - 1 - r0) / R], 1u << ((l.e - 1 - r0) % R));
                    edges.end[l.e - 1 - r0] = l.i;
                }
                // where the next tile begins to look
                if (BACK ? l.s < r0 : l.s <= r0 + n) atomicMax(&edges.next, l.i);
                edges.s[threadIdx.x] = l.s;
                edges.e[threadIdx.x] = l.e;
            }
            __syncthreads();
            if (!(l.more && (BACK ? l.last >= r0 : l.last < r0 + n))) break;
            look(a, BACK ? l.from - kThreads : l.from + kThreads, l);
            if (l.from >= a.batch) break;                  // (BACK: below the first)
        }
        b = __builtin_amdgcn_readfirstlane(edges.next);
        const uint32_t at_ = BACK ? l.from - b : b - l.from;
        if (l.from < a.batch && at_ < kThreads) {
            s = __builtin_amdgcn_readfirstlane(edges.s[at_]);
            e = __builtin_amdgcn_readfirstlane(edges.e[at_]);
        } else {
            at(a, b);
        }
    }
};

// Joins the maps of the workgroup's stretches (`own`, a thread's rows each): returns
// that of all stretches before this one (REVERSE: behind it), `all` that of
// all of them.  A barrier within; another has to follow before the next use.
template <int C, bool REVERSE>
__device__ __forceinline__ void join(const Map (&own)[C], uint32_t lanes, Map (&before)[C], Map (&all)[C],
                                     Map (&lds)[kThreads / 64][64 * C]) {
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = lane % lanes;
    Map in[C];                                              // all of this wavefront's up to this one
#pragma unroll
    for (int i = 0; i < C; i++) in[i] = own[i], before[i] = {1.0f, 0.0f};
    for (uint32_t o = lanes; o < 64; o *= 2) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            const int from = REVERSE ? lane + o : lane - o;
            const Map p = {__shfl(in[i].a, from), __shfl(in[i].b, from)};
            if (REVERSE ? lane + o < 64 : lane >= o) in[i] = in[i].after(p);
        }
    }
    if (lanes < 64) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            const int from = REVERSE ? lane + lanes : lane - lanes;
            const Map p = {__shfl(in[i].a, from), __shfl(in[i].b, from)};
            if (REVERSE ? lane + lanes < 64 : lane >= lanes) before[i] = p;
        }
    }
    if (REVERSE ? lane < lanes : lane >= 64 - lanes) {
#pragma unroll
        for (int i = 0; i < C; i++) lds[wave][c * C + i] = in[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < C; i++) {
        Map up = {1.0f, 0.0f}, sum = {1.0f, 0.0f};
#pragma unroll 2
        for (uint32_t k = 0; k < kThreads / 64; k++) {
            const uint32_t w = REVERSE ? kThreads / 64 - 1 - k : k;
            if (w == wave) up = sum;
            sum = lds[w][c * C + i].after(sum);
        }
        before[i] = before[i].after(up);
        all[i] = sum;
    }
}

// Where a thread's rows and channels are.  ONE: a wavefront holds one stretch
// of rows, so that rows and what is asked of them are the wavefront's.
//   The groups of a chunk's channels are eight workgroups apart, so that the same
// XCD takes them, side by side: rows that do not begin at a cache line share
// lines between groups (288 654 rows of 100 fp32 values, a training step: 385 us
// with the groups one after the other, 366 so).
template <int R, bool ONE> struct Place {
    uint32_t chunk, sub, c, tile;                          // its stretch in a tile, its first channel, rows of a tile
    uint32_t first, last;                                  // rows that sequences have
    __device__ __forceinline__ Place(const Scan &a, int n) {
        const uint32_t in = blockIdx.x % (8 * a.groups);
        chunk = blockIdx.x / (8 * a.groups) * 8 + in % 8;
        sub = ONE ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / a.lanes;
        c = (in / 8 * a.lanes + threadIdx.x % a.lanes) * n;
        tile = kThreads / a.lanes * R;
        first = __builtin_amdgcn_readfirstlane(start_of(a, 0));
        last = __builtin_amdgcn_readfirstlane(start_of(a, a.batch));
    }
    __device__ __forceinline__ bool none() const { return first >= last; }
    __device__ __forceinline__ bool there(uint32_t r) const { return r >= first && r < last; }
    __device__ __forceinline__ bool all_there(uint32_t r) const { return r >= first && r + R <= last; }
    __device__ __forceinline__ uint32_t word(const uint32_t *words) const {
        return ONE ? __builtin_amdgcn_readfirstlane(words[sub]) : words[sub];
    }
};

// The words of a thread's rows.  IN: all of them are rows of sequences; else the
// nearest of those are read where they are not.  (No choice within the loop: each
// load would be waited for before the next.)
template <bool IN, typename T, int R, bool ONE>
__device__ __forceinline__ void load_rows(const uint8_t *p, int64_t stride, uint32_t r, const Place<R, ONE> &at,
                                          const Piece<T> &piece, uint32_t (&raw)[R]) {
    if constexpr (IN) {
        p += (int64_t)r * stride;
#pragma unroll
        for (int i = 0; i < R; i++, p += stride) raw[i] = piece.load(p);
    } else {
#pragma unroll
        for (int i = 0; i < R; i++) raw[i] = piece.load(p + (int64_t)min(max(r + i, at.first), at.last - 1) * stride);
        asm volatile("");                                  // (keeps the two kinds of loads apart)
    }
}
template <typename T, int R, bool ONE>
__device__ __forceinline__ void store_rows(uint8_t *p, int64_t stride, uint32_t r, const Place<R, ONE> &at,
                                           const Piece<T> &piece, bool whole, const float (&f)[R][Piece<T>::n]) {
    p += (int64_t)r * stride;
    if (!piece.there) return;
    if (whole) {
#pragma unroll
        for (int i = 0; i < R; i++, p += stride) piece.store(p, f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < R; i++, p += stride)
            if (at.there(r + i)) piece.store(p, f[i]);
    }
}

// Values c on of row b of an fp32 array [batch][width], zeros without one.
template <int C>
__device__ __forceinline__ void load_state(const Scan &a, const float *p, uint32_t b, uint32_t c, float (&f)[C]) {
#pragma unroll
    for (int i = 0; i < C; i++) f[i] = p && c + i < a.width ? p[(size_t)b * a.width + c + i] : 0.0f;
}
template <int C>
__device__ __forceinline__ void store_state(const Scan &a, float *p, uint32_t b, uint32_t c, const float (&f)[C]) {
#pragma unroll
    for (int i = 0; i < C; i++)
        if (c + i < a.width) p[(size_t)b * a.width + c + i] = f[i];
}

// Sequences without rows, which no tile holds: their states go through.
template <int C>
__device__ __forceinline__ void pass_on(const Scan &a, const float *from, float *to, uint32_t chunk, uint32_t c) {
    if (!to || (!a.start && a.len)) return;
    for (uint32_t b = chunk; b < a.batch; b += max(a.chunks, 1u)) {
        if (start_of(a, b) < start_of(a, b + 1) || threadIdx.x >= a.lanes) continue;
        float f[C];
        load_state(a, from, b, c, f);
        store_state(a, to, b, c, f);
    }
}

// Has the compiler unpack the words again behind it, instead of keeping what they
// held in registers of its own.
template <int R> __device__ __forceinline__ void forget(uint32_t (&raw)[R]) {
#pragma unroll
    for (int k = 0; k < R; k++) asm volatile("" : "+v"(raw[k]));
}
// Keeps the compiler from starting what follows among what comes before: that
// would take more registers than there are.
__device__ __forceinline__ void phase() { __builtin_amdgcn_sched_barrier(0); }

// APPLY = false: the chunks' maps; true: h, the last states and the states
// that the backward pass starts from.
template <typename T, bool ONE, bool APPLY>
__global__ __launch_bounds__(kThreads, 4) void scan_rows(Scan a) {
    constexpr int C = Piece<T>::n, R = kRows;
    constexpr bool EXACT = std::is_same<T, float>::value;
    __shared__ Edges edges;
    __shared__ Map lds[kThreads / 64][64 * C];
    const Place<R, ONE> at(a, C);
    const Piece<T> piece(at.c, a.width);
    if (at.chunk >= max(a.chunks, 1u)) return;
    const uint32_t from = at.chunk * a.chunk_rows, to = min(a.rows, from + a.chunk_rows);
    float state[C];
    Map chunk[C];
    load_state(a, APPLY ? a.into : nullptr, at.chunk, at.c, state);
#pragma unroll
    for (int i = 0; i < C; i++) chunk[i] = {1.0f, 0.0f};
    if (threadIdx.x < kThreads / 8) edges.begins[threadIdx.x] = edges.ends[threadIdx.x] = 0;
    if (threadIdx.x == 0) edges.next = 0;
    __syncthreads();
    uint32_t tiles = at.none() ? 0 : (to - from + at.tile - 1) / at.tile, t0 = 0;
    Cursor<R, !APPLY> cursor;
    if (tiles) {
        cursor.at(a, find_sequence(a, APPLY ? from : to - 1));
        // rows before the last first row in the chunk do not matter
        if (!APPLY && cursor.s > from) t0 = (cursor.s - from) / at.tile;
    }
    for (uint32_t n = t0; n < tiles; n++) {
        const uint32_t t = APPLY ? n : tiles - 1 - (n - t0), r0 = from + t * at.tile, r = r0 + at.sub * R;
        const bool plain = cursor.plain(r0, at.tile);
        uint32_t rx[R], rg[R], begins = 0, ends = 0;
        typename Cursor<R, !APPLY>::Look look;
        if (!plain) cursor.look(a, cursor.b, look);
        const bool whole = plain || at.all_there(r);
        if (whole) {
            load_rows<true>(a.x, a.x_row, r, at, piece, rx);
            load_rows<true>(a.g, a.g_row, r, at, piece, rg);
        } else {
            load_rows<false>(a.x, a.x_row, r, at, piece, rx);
            load_rows<false>(a.g, a.g_row, r, at, piece, rg);
        }
        if (!plain) {
            cursor.find(a, r0, at.tile, look, edges);
            begins = at.word(edges.begins);
            if constexpr (APPLY) ends = at.word(edges.ends);
        }
        limit<T>(rg);
        float z[APPLY ? R : 1][C], y[APPLY ? R : 1][C];
        Map own[C], before[C], all[C];
#pragma unroll
        for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
        phase();
#pragma unroll
        for (int k = 0; k < R; k++) {
            constexpr int one = APPLY ? 1 : 0;
            float x[C], g[C], (&zk)[C] = z[one * k], (&yk)[C] = y[one * k];
            piece.unpack(rx[k], x);
            piece.unpack(rg[k], g);
#pragma unroll
            for (int i = 0; i < C; i++) {
                gate<EXACT>(g[i], zk[i], yk[i]);
                yk[i] *= x[i];
                if (!whole && !at.there(r + k)) zk[i] = 1.0f, yk[i] = 0.0f;
            }
            if (begins >> k & 1) {
                float h0[C];
                load_state(a, a.h0, edges.begin[at.sub * R + k], at.c, h0);
#pragma unroll
                for (int i = 0; i < C; i++) {
                    yk[i] = fmaf(zk[i], h0[i], yk[i]);
                    zk[i] = kForgets;
                    own[i] = {kForgets, yk[i]};
                }
            } else {
#pragma unroll
                for (int i = 0; i < C; i++) {                // (a forgetting map's -0 stays one times z)
                    own[i].a *= zk[i];
                    own[i].b = fmaf(zk[i], own[i].b, yk[i]);
                }
            }
            if (k % 4 == 3) phase();
        }
        join<C, false>(own, a.lanes, before, all, lds);
        if (!plain && threadIdx.x < kThreads / 8) edges.begins[threadIdx.x] = edges.ends[threadIdx.x] = 0;
        if (!plain && threadIdx.x == 0) edges.next = 0;
        if constexpr (APPLY) {
            float h[C];
#pragma unroll
            for (int i = 0; i < C; i++) h[i] = before[i].of(state[i]);
            if (a.states && r % kStateRows == 0 && r < a.rows) store_state(a, a.states, r / kStateRows, at.c, h);
            if (!begins) {
#pragma unroll
                for (int k = 0; k < R; k++)
#pragma unroll
                    for (int i = 0; i < C; i++) y[k][i] = h[i] = fmaf(z[k][i], h[i], y[k][i]);
            } else {
#pragma unroll
                for (int k = 0; k < R; k++)
#pragma unroll
                    for (int i = 0; i < C; i++) y[k][i] = h[i] = Map{z[k][i], y[k][i]}.of(h[i]);
            }
            store_rows<T>(a.h, a.h_row, r, at, piece, whole, y);
            if (a.last && ends) {
#pragma unroll
                for (int k = 0; k < R; k++)
                    if (ends >> k & 1) store_state(a, a.last, edges.end[at.sub * R + k], at.c, y[k]);
            }
#pragma unroll
            for (int i = 0; i < C; i++) state[i] = all[i].of(state[i]);
        } else {
#pragma unroll
            for (int i = 0; i < C; i++) chunk[i] = chunk[i].after(all[i]);
        }
        __syncthreads();
    }
    if constexpr (APPLY) {
        pass_on<C>(a, a.h0, a.last, at.chunk, at.c);
    } else if (threadIdx.x < a.lanes) {
        float *m = a.maps + (size_t)at.chunk * 2 * a.width;
#pragma unroll
        for (int i = 0; i < C; i++)
            if (at.c + i < a.width) m[at.c + i] = chunk[i].a, m[a.width + at.c + i] = chunk[i].b;
    }
}

// The same backwards: APPLY = false: the chunks' maps of e; true: the gradients.
template <typename T, bool ONE, bool APPLY>
__global__ __launch_bounds__(kThreads, 4) void scan_rows_backward(Scan a) {
    constexpr int C = Piece<T>::n, R = kRowsBack;
    constexpr bool EXACT = std::is_same<T, float>::value;
    __shared__ Edges edges;
    __shared__ Map lds[2][kThreads / 64][64 * C];
    const Place<R, ONE> at(a, C);
    const Piece<T> piece(at.c, a.width);
    if (at.chunk >= max(a.chunks, 1u)) return;
    const uint32_t from = at.chunk * a.chunk_rows, to = min(a.rows, from + a.chunk_rows);
    float state[C];
    Map chunk[C];
    load_state(a, APPLY ? a.into : nullptr, at.chunk, at.c, state);
#pragma unroll
    for (int i = 0; i < C; i++) chunk[i] = {1.0f, 0.0f};
    if (threadIdx.x < kThreads / 8) edges.begins[threadIdx.x] = edges.ends[threadIdx.x] = 0;
    if (threadIdx.x == 0) edges.next = 0;
    __syncthreads();
    uint32_t tiles = (to - from + at.tile - 1) / at.tile;
    Cursor<R, APPLY> cursor;
    if (at.none()) tiles = 0;
    if (tiles) {
        cursor.at(a, find_sequence(a, APPLY ? to - 1 : from));
        // rows behind the first last row in the chunk do not matter
        if (!APPLY && cursor.e > from && cursor.e <= to) tiles = (cursor.e - from + at.tile - 1) / at.tile;
    }
    for (uint32_t n = 0; n < tiles; n++) {
        const uint32_t t = APPLY ? tiles - 1 - n : n, r0 = from + t * at.tile, r = r0 + at.sub * R;
        const bool plain = cursor.plain(r0, at.tile);
        uint32_t rx[R], rg[R], rd[R], begins = 0, ends = 0;
        typename Cursor<R, APPLY>::Look look;
        if (!plain) cursor.look(a, cursor.b, look);
        const bool whole = plain || at.all_there(r);
        if (whole) {
            load_rows<true>(a.g, a.g_row, r, at, piece, rg);
            load_rows<true>(a.dh, a.dh_row, r, at, piece, rd);
            if constexpr (APPLY) load_rows<true>(a.x, a.x_row, r, at, piece, rx);
        } else {
            load_rows<false>(a.g, a.g_row, r, at, piece, rg);
            load_rows<false>(a.dh, a.dh_row, r, at, piece, rd);
            if constexpr (APPLY) load_rows<false>(a.x, a.x_row, r, at, piece, rx);
        }
        float h[C];
        load_state(a, APPLY ? a.states : nullptr, r0 / kStateRows, at.c, h);
        if (!plain) {
            cursor.find(a, r0, at.tile, look, edges);
            ends = at.word(edges.ends);
            if constexpr (APPLY) begins = at.word(edges.begins);
        }
        limit<T>(rg);
        float z[R][C], y[R][C];
        Map own[C], before[C], all[C];
#pragma unroll
        for (int k = 0; k < R; k++) {
            float g[C];
            piece.unpack(rg[k], g);
#pragma unroll
            for (int i = 0; i < C; i++) gate<EXACT>(g[i], z[k][i], y[k][i]);
            if (k % 4 == 3) phase();
        }
        if (!whole) {
#pragma unroll
            for (int k = 0; k < R; k++)
#pragma unroll
                for (int i = 0; i < C; i++)
                    if (!at.there(r + k)) z[k][i] = 1.0f, y[k][i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
#pragma unroll
        for (int k = R - 1; k >= 0; k--) {
            float d[C];
            piece.unpack(rd[k], d);
            if (ends >> k & 1) {
                float last[C];
                load_state(a, a.dlast, edges.end[at.sub * R + k], at.c, last);
#pragma unroll
                for (int i = 0; i < C; i++) own[i] = {kForgets, z[k][i] * (d[i] + last[i])};
            } else {
#pragma unroll
                for (int i = 0; i < C; i++) {                // (a forgetting map's -0 stays one times z)
                    own[i].a *= z[k][i];
                    own[i].b = fmaf(z[k][i], own[i].b, z[k][i] * d[i]);
                }
            }
        }
        phase();
        join<C, true>(own, a.lanes, before, all, lds[0]);
        phase();
        if (!plain && threadIdx.x < kThreads / 8) edges.begins[threadIdx.x] = edges.ends[threadIdx.x] = 0;
        if (!plain && threadIdx.x == 0) edges.next = 0;
        float e[C];
#pragma unroll
        for (int i = 0; i < C; i++) {
            e[i] = before[i].of(state[i]);
            if constexpr (APPLY) state[i] = all[i].of(state[i]);
            else chunk[i] = chunk[i].after(all[i]);
        }
        if constexpr (APPLY) {
            // h before each row again: forward maps from the state that was kept
            float w[R][C];
#pragma unroll
            for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < R; k++) {
                float x[C];
                piece.unpack(rx[k], x);
                if (begins >> k & 1) {
                    load_state(a, a.h0, edges.begin[at.sub * R + k], at.c, w[k]);
#pragma unroll
                    for (int i = 0; i < C; i++) own[i] = {kForgets, fmaf(z[k][i], w[k][i], y[k][i] * x[i])};
                } else {
#pragma unroll
                    for (int i = 0; i < C; i++) {
                        own[i].a *= z[k][i];
                        own[i].b = fmaf(z[k][i], own[i].b, y[k][i] * x[i]);
                    }
                }
            }
            phase();
            join<C, false>(own, a.lanes, before, all, lds[1]);
            forget(rx);
            phase();
#pragma unroll
            for (int i = 0; i < C; i++) h[i] = before[i].of(h[i]);
#pragma unroll
            for (int k = 0; k < R; k++) {
                float x[C];
                piece.unpack(rx[k], x);
                if (!(begins >> k & 1)) {
#pragma unroll
                    for (int i = 0; i < C; i++) w[k][i] = h[i];
                }
#pragma unroll
                for (int i = 0; i < C; i++) h[i] = fmaf(z[k][i], w[k][i], y[k][i] * x[i]);
                if (k % 4 == 3) phase();
            }
            forget(rx);
            forget(rd);
            phase();
            // y becomes dx, w dg, z what goes on to the row before
#pragma unroll
            for (int k = R - 1; k >= 0; k--) {
                float x[C], d[C];
                piece.unpack(rx[k], x);
                piece.unpack(rd[k], d);
                if (ends >> k & 1) load_state(a, a.dlast, edges.end[at.sub * R + k], at.c, e);
#pragma unroll
                for (int i = 0; i < C; i++) {
                    const float q = d[i] + e[i];
                    y[k][i] *= q;
                    w[k][i] = y[k][i] * z[k][i] * (w[k][i] - x[i]);
                    e[i] = z[k][i] *= q;
                }
                if (k % 4 == 0) phase();
            }
            store_rows<T>(a.dx, a.dx_row, r, at, piece, whole, y);
            store_rows<T>(a.dg, a.dg_row, r, at, piece, whole, w);
            if (a.dh0 && begins) {
#pragma unroll
                for (int k = 0; k < R; k++)
                    if (begins >> k & 1) store_state(a, a.dh0, edges.begin[at.sub * R + k], at.c, z[k]);
            }
        }
        __syncthreads();
    }
    if constexpr (APPLY) {
        pass_on<C>(a, a.dlast, a.dh0, at.chunk, at.c);
    } else if (threadIdx.x < a.lanes) {
        float *m = a.maps + (size_t)at.chunk * 2 * a.width;
#pragma unroll
        for (int i = 0; i < C; i++)
            if (at.c + i < a.width) m[at.c + i] = chunk[i].a, m[a.width + at.c + i] = chunk[i].b;
    }
}

// One row a sequence, as it comes: a thread a few channels of one row.
template <typename T> __global__ __launch_bounds__(256) void single_rows(Scan a) {
    constexpr int C = Piece<T>::n;
    constexpr bool EXACT = std::is_same<T, float>::value;
    const uint32_t pieces = (a.width + C - 1) / C;
    const uint64_t all = (uint64_t)a.rows * pieces, step = (uint64_t)gridDim.x * 256;
    for (uint64_t l = (uint64_t)blockIdx.x * 256 + threadIdx.x; l < all; l += step) {
        const uint32_t r = (uint32_t)(l / pieces), c = (uint32_t)(l - (uint64_t)r * pieces) * C;
        const Piece<T> piece(c, a.width);
        float x[C], g[C], h[C];
        piece.unpack(piece.load(a.x + (int64_t)r * a.x_row), x);
        uint32_t w[1] = {piece.load(a.g + (int64_t)r * a.g_row)};
        limit<T>(w);
        piece.unpack(w[0], g);
        load_state(a, a.h0, r, c, h);
#pragma unroll
        for (int i = 0; i < C; i++) {
            float z, y;
            gate<EXACT>(g[i], z, y);
            h[i] = fmaf(z, h[i], y * x[i]);
        }
        piece.store(a.h + (int64_t)r * a.h_row, h);
        if (a.last) store_state(a, a.last, r, c, h);
    }
}

// The state before each chunk (REVERSE: e behind it) from the chunks' maps: 16
// channels a workgroup, 64 threads each, a run of chunks a thread.
template <bool REVERSE> __global__ __launch_bounds__(1024) void join_chunks(Scan a) {
    __shared__ Map lds[2][64][16];
    const uint32_t t = threadIdx.x / 16, c = blockIdx.x * 16 + threadIdx.x % 16;
    const uint32_t per = (a.chunks + 63) / 64, k0 = min(t * per, a.chunks), k1 = min(k0 + per, a.chunks);
    const auto chunk = [&](uint32_t k) { return (size_t)(REVERSE ? a.chunks - 1 - k : k); };
    Map run = {1.0f, 0.0f};
    const bool there = c < a.width;
    for (uint32_t k = k0; k < k1 && there; k += 8) {
        Map m[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            m[i] = {1.0f, 0.0f};
            if (k + i < k1) m[i] = {a.maps[chunk(k + i) * 2 * a.width + c], a.maps[(chunk(k + i) * 2 + 1) * a.width + c]};
        }
#pragma unroll
        for (int i = 0; i < 8; i++) run = m[i].after(run);
    }
    uint32_t at = 0;
    lds[0][t][threadIdx.x % 16] = run;
    __syncthreads();
    for (uint32_t o = 1; o < 64; o *= 2, at ^= 1) {
        Map m = lds[at][t][threadIdx.x % 16];
        if (t >= o) m = m.after(lds[at][t - o][threadIdx.x % 16]);
        lds[at ^ 1][t][threadIdx.x % 16] = m;
        __syncthreads();
    }
    float h = t ? lds[at][t - 1][threadIdx.x % 16].of(0.0f) : 0.0f;
    for (uint32_t k = k0; k < k1 && there; k += 8) {
        Map m[8];
#pragma unroll
        for (int i = 0; i < 8; i++) {
            m[i] = {1.0f, 0.0f};
            if (k + i < k1) m[i] = {a.maps[chunk(k + i) * 2 * a.width + c], a.maps[(chunk(k + i) * 2 + 1) * a.width + c]};
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (k + i < k1) a.into[chunk(k + i) * a.width + c] = h;
            h = m[i].of(h);
        }
    }
}

// ---------------------------------------------------------------- host
// Lanes that share a row: a power of two from 8 to 64 that holds the channels.
// Chunks: as many workgroups as the card holds (four on each of 256 CUs), of whole
// tiles; twice as many are no faster, and their maps take twice as long to join.
void split(Scan &a, int n) {
    a.lanes = 8;
    while (a.lanes < 64 && a.lanes * n < a.width) a.lanes *= 2;
    const uint32_t tile = kThreads / a.lanes * kRows, tiles = (a.rows + tile - 1) / tile;
    a.groups = (a.width + a.lanes * n - 1) / (a.lanes * n);
    const uint32_t most = a.groups < kChunks ? kChunks / a.groups : 1;
    const uint32_t per = (tiles + most - 1) / most;
    a.chunk_rows = per * tile;
    a.chunks = per ? (tiles + per - 1) / per : 0;
}

// Whether a chunk sees the one before it.
bool carried(const Scan &a) { return a.chunks > 1 && (a.start || a.chunk_rows % a.len); }

size_t align16z(size_t n) { return (n + 15) & ~(size_t)15; }
size_t work_of(const Scan &a) {
    return carried(a) ? align16z((size_t)a.chunks * 2 * a.width * 4) + align16z((size_t)a.chunks * a.width * 4) : 0;
}

bool bad_rows(const nlb_scan_rows &r, uint32_t rows, int64_t e) {
    return (rows && !r.data) || (uintptr_t)r.data % e || r.row_stride < 0 || r.row_stride > INT32_MAX;
}

int fill(const nlb_scan_call *c, Scan &a) {
    a = {};
    if (!c || (c->dtype != NLB_DTYPE_F32 && c->dtype != NLB_DTYPE_BF16)) return NLB_EINVAL;
    if (c->width < 1 || c->width > NLB_SCAN_MAX_WIDTH || c->rows > NLB_SCAN_MAX_ROWS) return NLB_EINVAL;
    if (c->batch < 1 || c->batch > INT32_MAX - 1) return NLB_EINVAL;
    if (!c->start && c->rows % c->batch) return NLB_EINVAL;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (bad_rows(c->x, c->rows, e) || bad_rows(c->g, c->rows, e)) return NLB_EINVAL;
    if (((uintptr_t)c->start | (uintptr_t)c->h0) % 4) return NLB_EINVAL;
    a.x = (const uint8_t *)c->x.data;
    a.g = (const uint8_t *)c->g.data;
    a.x_row = c->x.row_stride * e;
    a.g_row = c->g.row_stride * e;
    a.start = c->start;
    a.h0 = c->h0;
    a.rows = c->rows;
    a.width = (uint32_t)c->width;
    a.batch = c->batch;
    a.len = c->start ? 0 : c->rows / c->batch;
    split(a, c->dtype == NLB_DTYPE_BF16 ? 2 : 1);
    return NLB_OK;
}

// Two arrays [batch][width] that share memory?
bool overlap(const Scan &a, const float *p, const float *q) {
    const size_t n = (size_t)a.batch * a.width;
    return p && q && p < q + n && q < p + n;
}

template <typename T, bool ONE, bool BACKWARD> int launch(Scan &a, void *work, hipStream_t s) {
    // (a call of no rows still has states to pass on)
    const uint32_t grid = (a.chunks ? (a.chunks + 7) / 8 : 1) * 8 * a.groups;
    if (carried(a)) {
        a.maps = (float *)work;
        float *into = (float *)((uint8_t *)work + align16z((size_t)a.chunks * 2 * a.width * 4));
        int rc = enqueue(BACKWARD ? scan_rows_backward<T, ONE, false> : scan_rows<T, ONE, false>, grid, kThreads, 0, s, a);
        if (rc != NLB_OK) return rc;
        a.into = into;
        rc = enqueue(join_chunks<BACKWARD>, (a.width + 15) / 16, 1024, 0, s, a);
        if (rc != NLB_OK) return rc;
    }
    return enqueue(BACKWARD ? scan_rows_backward<T, ONE, true> : scan_rows<T, ONE, true>, grid, kThreads, 0, s, a);
}
template <typename T, bool BACKWARD> int launch(Scan &a, void *work, hipStream_t s) {
    if (!BACKWARD && !a.start && a.len == 1 && !a.states) {
        const uint64_t pieces = (uint64_t)a.rows * ((a.width + Piece<T>::n - 1) / Piece<T>::n);
        return enqueue(single_rows<T>, (uint32_t)std::min<uint64_t>((pieces + 255) / 256, 1u << 20), 256, 0, s, a);
    }
    return a.lanes == 64 ? launch<T, true, BACKWARD>(a, work, s) : launch<T, false, BACKWARD>(a, work, s);
}

template <bool BACKWARD> int launch_bf16(Scan &a, void *work, hipStream_t s) {
    return a.width == 1 ? launch<OneBf16, false, BACKWARD>(a, work, s) : launch<__bf16, BACKWARD>(a, work, s);
}

}  // namespace

extern "C" int nlb_gated_scan_work(const nlb_scan_call *c, size_t *bytes) {
    Scan a;
    if (!bytes) return NLB_EINVAL;
    const int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    *bytes = work_of(a);
    return NLB_OK;
}

extern "C" int nlb_gated_scan(const nlb_scan_call *c, const nlb_scan_rows *h, float *last, float *states, void *work,
                              size_t work_bytes, void *stream) {
    Scan a;
    int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (!h || bad_rows(*h, c->rows, e) || ((uintptr_t)last | (uintptr_t)states) % 4 || (uintptr_t)work % 16)
        return NLB_EINVAL;
    // a sequence's last state may be written before another workgroup reads its first
    if (overlap(a, a.h0, last) && !(a.h0 == last && !a.start && a.len == 1)) return NLB_EINVAL;
    if (work_of(a) && (!work || work_bytes < work_of(a))) return NLB_ESCRATCH;
    a.h = (uint8_t *)h->data;
    a.h_row = h->row_stride * e;
    a.last = last;
    a.states = states;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    return c->dtype == NLB_DTYPE_BF16 ? launch_bf16<false>(a, work, (hipStream_t)stream)
                                      : launch<float, false>(a, work, (hipStream_t)stream);
}

extern "C" int nlb_gated_scan_backward(const nlb_scan_call *c, const float *states, const nlb_scan_rows *dh,
                                       const float *dlast, const nlb_scan_rows *dx, const nlb_scan_rows *dg, float *dh0,
                                       void *work, size_t work_bytes, void *stream) {
    Scan a;
    int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (!dh || !dx || !dg || bad_rows(*dh, c->rows, e) || bad_rows(*dx, c->rows, e) || bad_rows(*dg, c->rows, e))
        return NLB_EINVAL;
    if ((c->rows && !states) || ((uintptr_t)states | (uintptr_t)dlast | (uintptr_t)dh0) % 4 || (uintptr_t)work % 16)
        return NLB_EINVAL;
    if (overlap(a, dlast, dh0) || overlap(a, a.h0, dh0)) return NLB_EINVAL;
    if (work_of(a) && (!work || work_bytes < work_of(a))) return NLB_ESCRATCH;
    a.states = (float *)states;
    a.dh = (const uint8_t *)dh->data;
    a.dx = (uint8_t *)dx->data;
    a.dg = (uint8_t *)dg->data;
    a.dh_row = dh->row_stride * e;
    a.dx_row = dx->row_stride * e;
    a.dg_row = dg->row_stride * e;
    a.dlast = dlast;
    a.dh0 = dh0;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    return c->dtype == NLB_DTYPE_BF16 ? launch_bf16<true>(a, work, (hipStream_t)stream)
                                      : launch<float, true>(a, work, (hipStream_t)stream);
}
