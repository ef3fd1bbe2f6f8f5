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
// 8 wavefronts stand one below the other: maps of those rows are joined over the
// workgroup through LDS, then every thread walks its rows again, in registers.
// A workgroup walks a chunk of the rows tile by tile.  Where there are several
// chunks, a first launch makes their maps (it reads x and g once more, but only
// from the last first row in the chunk on), a second joins them.
#include <type_traits>

#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef uint32_t u32_any __attribute__((aligned(2)));

constexpr int kThreads = 512, kRows = 16, kRowsBack = 8;   // rows a thread holds
constexpr uint32_t kStateRows = NLB_SCAN_STATE_ROWS;

struct Scan {
    const uint8_t *x, *g, *dh;
    uint8_t *h, *dx, *dg;
    int64_t x_row, g_row, dh_row, h_row, dx_row, dg_row;   // bytes
    const int32_t *start;                                  // NULL: len rows each
    const float *h0, *dlast;
    float *last, *dh0, *states;
    float *maps, *into;                                    // [chunks][2][width], [chunks][width]
    uint32_t rows, width, batch, len;
    uint32_t lanes, chunk_rows, chunks;
};

// Values c and c + 1 of a row (fp32: c), 0 past its end.
template <typename T> struct Lane;
template <> struct Lane<float> {
    static constexpr int n = 1;
    static __device__ __forceinline__ uint32_t load(const uint8_t *row, uint32_t c, uint32_t) {
        return ((const uint32_t *)row)[c];
    }
    static __device__ __forceinline__ void unpack(uint32_t w, float (&f)[1]) { f[0] = __uint_as_float(w); }
    static __device__ __forceinline__ void store(uint8_t *row, uint32_t c, uint32_t, const float (&f)[1]) {
        ((float *)row)[c] = f[0];
    }
};
template <> struct Lane<__bf16> {
    static constexpr int n = 2;
    static __device__ __forceinline__ uint32_t load(const uint8_t *row, uint32_t c, uint32_t width) {
        const uint8_t *p = row + 2 * c;
        return c + 1 < width ? *(const u32_any *)p : *(const uint16_t *)p;
    }
    static __device__ __forceinline__ void unpack(uint32_t w, float (&f)[2]) {
        f[0] = __uint_as_float(w << 16);
        f[1] = __uint_as_float(w & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void store(uint8_t *row, uint32_t c, uint32_t width, const float (&f)[2]) {
        __bf16 v[2] = {(__bf16)f[0], (__bf16)f[1]};
        uint32_t w;
        __builtin_memcpy(&w, v, 4);
        uint8_t *p = row + 2 * c;
        if (c + 1 < width) *(u32_any *)p = w;
        else *(uint16_t *)p = (uint16_t)w;
    }
};

// z = sigmoid(g) and 1 - z, each with its own relative error of some 2^-22:
// from e = exp(-|g|), the larger of them 1 / (1 + e) and the smaller e times
// that.  e is 2^(t + lo) with t + lo = -|g| / ln 2 in two words.  Gates beyond
// 80 in magnitude (e below 2^-115) count as 80.
__device__ __forceinline__ void gate(float g, float &z, float &y) {
    const float m = fabsf(g) > 80.0f ? 80.0f : fabsf(g);      // (a NaN stays one)
    const float t = m * -1.44269504f;
    const float lo = fmaf(m, -1.92596299e-8f, fmaf(m, -1.44269504f, -t));
    float e = __builtin_amdgcn_exp2f(t);
    e = fmaf(e, lo * 0.693147181f, e);
    const float big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    z = g < 0.0f ? small : big;
    y = g < 0.0f ? big : small;
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
};

// Rows that sequences have: first to last.
__device__ __forceinline__ uint32_t clamped(const int32_t *start, uint32_t b, uint32_t rows) {
    const int32_t s = start[b];
    return s < 0 ? 0u : (uint32_t)s < rows ? (uint32_t)s : rows;
}

// The last sequence that begins at row r or before it (0 if none does): a
// wavefront tries 64 of them at once.
__device__ __forceinline__ uint32_t find_sequence(const int32_t *start, uint32_t batch, uint32_t r) {
    uint32_t lo = 0, n = batch;
    const uint32_t lane = threadIdx.x % 64;
    for (;;) {
        const uint32_t step = (n + 63) / 64, i = lane * step;
        const bool before = i < n && start[lo + i] <= (int32_t)r;
        const uint32_t k = __popcll(__ballot(before));
        if (k > 1) lo += (k - 1) * step, n -= (k - 1) * step;
        if (step == 1) return lo;
        n = n < step ? n : step;
    }
}

// Fills `edges` for the rows r0 .. r0 + n - 1; two barriers, so that what was
// read before it may be written, and what it writes may be read.
template <int R> __device__ __forceinline__ void find_edges(const Scan &a, uint32_t r0, uint32_t n, Edges &edges) {
    if (threadIdx.x < kThreads / 8) edges.begins[threadIdx.x] = edges.ends[threadIdx.x] = 0;
    __syncthreads();
    if (!a.start) {
        for (uint32_t i = threadIdx.x; i < n; i += kThreads) {
            const uint32_t b = (r0 + i) / a.len, at = r0 + i - b * a.len;
            if (r0 + i >= a.rows) break;
            if (at == 0) {
                atomicOr(&edges.begins[i / R], 1u << (i % R));
                edges.begin[i] = b;
            }
            if (at == a.len - 1) {
                atomicOr(&edges.ends[i / R], 1u << (i % R));
                edges.end[i] = b;
            }
        }
        __syncthreads();
        return;
    }
    uint32_t b = find_sequence(a.start, a.batch, r0) + threadIdx.x;
    for (;; b += kThreads) {
        bool more = false;
        if (b < a.batch) {
            const uint32_t s = clamped(a.start, b, a.rows), e = clamped(a.start, b + 1, a.rows);
            more = s < r0 + n;                                // rows end before 2^31
            if (s < e && s - r0 < n) {
                atomicOr(&edges.begins[(s - r0) / R], 1u << ((s - r0) % R));
                edges.begin[s - r0] = b;
            }
            if (s < e && e - 1 - r0 < n) {
                atomicOr(&edges.ends[(e - 1 - r0) / R], 1u << ((e - 1 - r0) % R));
                edges.end[e - 1 - r0] = b;
            }
        }
        if (threadIdx.x != kThreads - 1) more = false;
        if (!__syncthreads_or(more)) return;
    }
}

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
#pragma unroll
        for (uint32_t k = 0; k < kThreads / 64; k++) {
            const uint32_t w = REVERSE ? kThreads / 64 - 1 - k : k;
            if (w == wave) up = sum;
            sum = lds[w][c * C + i].after(sum);
        }
        before[i] = before[i].after(up);
        all[i] = sum;
    }
}

// Where a thread's rows and channels are.
struct Place {
    uint32_t sub, c, tile;                                 // its stretch in a tile, its first channel, rows of a tile
    uint32_t first, last;                                  // rows that sequences have
    __device__ __forceinline__ Place(const Scan &a, int n, int rows) {
        sub = threadIdx.x / a.lanes;
        c = (blockIdx.y * a.lanes + threadIdx.x % a.lanes) * n;
        tile = kThreads / a.lanes * rows;
        first = a.start ? clamped(a.start, 0, a.rows) : 0;
        last = a.start ? clamped(a.start, a.batch, a.rows) : a.rows;
    }
};

template <typename T, int R>
__device__ __forceinline__ void load_rows(const uint8_t *p, int64_t stride, uint32_t r, const Place &at, uint32_t width,
                                          uint32_t (&raw)[R]) {
#pragma unroll
    for (int i = 0; i < R; i++) {
        raw[i] = 0;
        if (at.c < width && r + i >= at.first && r + i < at.last)
            raw[i] = Lane<T>::load(p + (int64_t)(r + i) * stride, at.c, width);
    }
}

// Sequences without rows, which no tile holds: their states go through.
__device__ __forceinline__ void pass_on(const Scan &a, const float *from, float *to, uint32_t c, int n) {
    if (!to || (!a.start && a.len)) return;
    for (uint32_t b = blockIdx.x; b < a.batch; b += gridDim.x) {
        if (a.start && clamped(a.start, b, a.rows) < clamped(a.start, b + 1, a.rows)) continue;
        if (threadIdx.x < a.lanes)
            for (int i = 0; i < n; i++)
                if (c + i < a.width)
                    to[(size_t)b * a.width + c + i] = from ? from[(size_t)b * a.width + c + i] : 0.0f;
    }
}

// APPLY = false: the chunks' maps; true: h, the last states and the states
// that the backward pass starts from.
template <typename T, bool APPLY>
__global__ __launch_bounds__(kThreads, 4) void scan_rows(Scan a) {
    constexpr int C = Lane<T>::n, R = kRows;
    __shared__ Edges edges;
    __shared__ Map lds[kThreads / 64][64 * C];
    const Place at(a, C, R);
    const uint32_t from = blockIdx.x * a.chunk_rows, to = min(a.rows, from + a.chunk_rows);
    float state[C];
    Map chunk[C];
#pragma unroll
    for (int i = 0; i < C; i++) {
        chunk[i] = {1.0f, 0.0f};
        state[i] = APPLY && a.into && at.c + i < a.width ? a.into[(size_t)blockIdx.x * a.width + at.c + i] : 0.0f;
    }
    uint32_t r0 = from;
    if constexpr (!APPLY) {
        // rows before the last first row in the chunk do not matter
        const uint32_t b = a.start ? find_sequence(a.start, a.batch, to - 1) : (to - 1) / a.len;
        const uint32_t s = a.start ? clamped(a.start, b, a.rows) : b * a.len;
        if (s > from) r0 = from + (s - from) / at.tile * at.tile;
    }
    for (; r0 < to; r0 += at.tile) {
        const uint32_t r = r0 + at.sub * R;
        uint32_t rx[R], rg[R];
        load_rows<T, R>(a.x, a.x_row, r, at, a.width, rx);
        load_rows<T, R>(a.g, a.g_row, r, at, a.width, rg);
        find_edges<R>(a, r0, at.tile, edges);
        const uint32_t begins = edges.begins[at.sub], ends = APPLY ? edges.ends[at.sub] : 0;
        float z[R][C], y[R][C];
        Map own[C], before[C], all[C];
#pragma unroll
        for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < R; k++) {
            float x[C], g[C];
            Lane<T>::unpack(rx[k], x);
            Lane<T>::unpack(rg[k], g);
            const bool there = r + k >= at.first && r + k < at.last;
#pragma unroll
            for (int i = 0; i < C; i++) {
                gate(g[i], z[k][i], y[k][i]);
                y[k][i] *= x[i];
                if (!there) z[k][i] = 1.0f, y[k][i] = 0.0f;
            }
            if (begins >> k & 1) {
                const int32_t b = edges.begin[at.sub * R + k];
#pragma unroll
                for (int i = 0; i < C; i++) {
                    const float h0 = a.h0 && at.c + i < a.width ? a.h0[(size_t)b * a.width + at.c + i] : 0.0f;
                    y[k][i] = fmaf(z[k][i], h0, y[k][i]);
                    z[k][i] = kForgets;
                }
            }
#pragma unroll
            for (int i = 0; i < C; i++) own[i] = Map{z[k][i], y[k][i]}.after(own[i]);
        }
        join<C, false>(own, a.lanes, before, all, lds);
        if constexpr (APPLY) {
            float h[C];
#pragma unroll
            for (int i = 0; i < C; i++) h[i] = before[i].of(state[i]);
            if (a.states && r % kStateRows == 0 && r < a.rows)
#pragma unroll
                for (int i = 0; i < C; i++)
                    if (at.c + i < a.width) a.states[(size_t)(r / kStateRows) * a.width + at.c + i] = h[i];
#pragma unroll
            for (int k = 0; k < R; k++) {
#pragma unroll
                for (int i = 0; i < C; i++) h[i] = Map{z[k][i], y[k][i]}.of(h[i]);
                if (at.c < a.width && r + k >= at.first && r + k < at.last) {
                    Lane<T>::store(a.h + (int64_t)(r + k) * a.h_row, at.c, a.width, h);
                    if (a.last && (ends >> k & 1)) {
                        const int32_t b = edges.end[at.sub * R + k];
#pragma unroll
                        for (int i = 0; i < C; i++)
                            if (at.c + i < a.width) a.last[(size_t)b * a.width + at.c + i] = h[i];
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < C; i++) state[i] = all[i].of(state[i]);
        } else {
#pragma unroll
            for (int i = 0; i < C; i++) chunk[i] = all[i].after(chunk[i]);
        }
        __syncthreads();
    }
    if constexpr (APPLY) {
        pass_on(a, a.h0, a.last, at.c, C);
    } else if (threadIdx.x < a.lanes) {
        float *m = a.maps + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
        for (int i = 0; i < C; i++)
            if (at.c + i < a.width) m[at.c + i] = chunk[i].a, m[a.width + at.c + i] = chunk[i].b;
    }
}

// The same backwards: APPLY = false: the chunks' maps of e; true: the gradients.
template <typename T, bool APPLY>
__global__ __launch_bounds__(kThreads, 2) void scan_rows_backward(Scan a) {
    constexpr int C = Lane<T>::n, R = kRowsBack;
    __shared__ Edges edges;
    __shared__ Map lds[2][kThreads / 64][64 * C];
    const Place at(a, C, R);
    const uint32_t from = blockIdx.x * a.chunk_rows, to = min(a.rows, from + a.chunk_rows);
    float state[C];
    Map chunk[C];
#pragma unroll
    for (int i = 0; i < C; i++) {
        chunk[i] = {1.0f, 0.0f};
        state[i] = APPLY && a.into && at.c + i < a.width ? a.into[(size_t)blockIdx.x * a.width + at.c + i] : 0.0f;
    }
    uint32_t tiles = (to - from + at.tile - 1) / at.tile;
    if constexpr (!APPLY) {
        // rows behind the first last row in the chunk do not matter
        const uint32_t b = a.start ? find_sequence(a.start, a.batch, from) : from / a.len;
        const uint32_t e = a.start ? clamped(a.start, b + 1, a.rows) : (b + 1) * a.len;
        if (e > from && e <= to) tiles = min(tiles, (e - from + at.tile - 1) / at.tile);
    }
    for (uint32_t t = tiles; t-- > 0;) {
        const uint32_t r0 = from + t * at.tile, r = r0 + at.sub * R;
        uint32_t rx[R], rg[R], rd[R];
        load_rows<T, R>(a.g, a.g_row, r, at, a.width, rg);
        load_rows<T, R>(a.dh, a.dh_row, r, at, a.width, rd);
        if constexpr (APPLY) load_rows<T, R>(a.x, a.x_row, r, at, a.width, rx);
        float h[C];
#pragma unroll
        for (int i = 0; i < C; i++)
            h[i] = APPLY && at.c + i < a.width ? a.states[(size_t)(r0 / kStateRows) * a.width + at.c + i] : 0.0f;
        find_edges<R>(a, r0, at.tile, edges);
        const uint32_t begins = APPLY ? edges.begins[at.sub] : 0, ends = edges.ends[at.sub];
        float z[R][C], y[R][C], d[R][C];
        Map own[C], before[C], all[C];
#pragma unroll
        for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
#pragma unroll
        for (int k = R - 1; k >= 0; k--) {
            float g[C];
            Lane<T>::unpack(rg[k], g);
            Lane<T>::unpack(rd[k], d[k]);
            const bool there = r + k >= at.first && r + k < at.last, end = ends >> k & 1;
#pragma unroll
            for (int i = 0; i < C; i++) {
                gate(g[i], z[k][i], y[k][i]);
                if (!there) z[k][i] = 1.0f, y[k][i] = 0.0f;
            }
            if (end && a.dlast) {
                const int32_t b = edges.end[at.sub * R + k];
#pragma unroll
                for (int i = 0; i < C; i++)
                    if (at.c + i < a.width) d[k][i] += a.dlast[(size_t)b * a.width + at.c + i];
            }
#pragma unroll
            for (int i = 0; i < C; i++)
                own[i] = Map{end ? kForgets : z[k][i], z[k][i] * d[k][i]}.after(own[i]);
        }
        join<C, true>(own, a.lanes, before, all, lds[0]);
        float e[C];
#pragma unroll
        for (int i = 0; i < C; i++) {
            e[i] = before[i].of(state[i]);
            if constexpr (APPLY) state[i] = all[i].of(state[i]);
            else chunk[i] = all[i].after(chunk[i]);
        }
        if constexpr (APPLY) {
            // h before each row again: forward maps from the state that was kept
            const auto forward = [&](int k, int i, const float (&x)[C]) {
                Map m = {z[k][i], y[k][i] * x[i]};
                if (begins >> k & 1) {
                    const float h0 = a.h0 && at.c + i < a.width
                                         ? a.h0[(size_t)edges.begin[at.sub * R + k] * a.width + at.c + i] : 0.0f;
                    m = {kForgets, fmaf(m.a, h0, m.b)};
                }
                return m;
            };
#pragma unroll
            for (int i = 0; i < C; i++) own[i] = {1.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < R; k++) {
                float x[C];
                Lane<T>::unpack(rx[k], x);
#pragma unroll
                for (int i = 0; i < C; i++) own[i] = forward(k, i, x).after(own[i]);
            }
            join<C, false>(own, a.lanes, before, all, lds[1]);
            float w[R][C];                               // h before the row
#pragma unroll
            for (int i = 0; i < C; i++) h[i] = before[i].of(h[i]);
#pragma unroll
            for (int k = 0; k < R; k++) {
                float x[C];
                Lane<T>::unpack(rx[k], x);
#pragma unroll
                for (int i = 0; i < C; i++) {
                    w[k][i] = h[i];
                    if (begins >> k & 1)
                        w[k][i] = a.h0 && at.c + i < a.width
                                      ? a.h0[(size_t)edges.begin[at.sub * R + k] * a.width + at.c + i] : 0.0f;
                    h[i] = forward(k, i, x).of(h[i]);
                }
            }
#pragma unroll
            for (int k = R - 1; k >= 0; k--) {
                float x[C], dx[C], dg[C];
                Lane<T>::unpack(rx[k], x);
#pragma unroll
                for (int i = 0; i < C; i++) {
                    const float q = (ends >> k & 1) ? d[k][i] : d[k][i] + e[i];
                    dx[i] = y[k][i] * q;
                    e[i] = z[k][i] * q;
                    dg[i] = dx[i] * z[k][i] * (w[k][i] - x[i]);
                }
                if (at.c >= a.width || r + k < at.first || r + k >= at.last) continue;
                Lane<T>::store(a.dx + (int64_t)(r + k) * a.dx_row, at.c, a.width, dx);
                Lane<T>::store(a.dg + (int64_t)(r + k) * a.dg_row, at.c, a.width, dg);
                if (a.dh0 && (begins >> k & 1)) {
                    const int32_t b = edges.begin[at.sub * R + k];
#pragma unroll
                    for (int i = 0; i < C; i++)
                        if (at.c + i < a.width) a.dh0[(size_t)b * a.width + at.c + i] = e[i];
                }
            }
        }
        __syncthreads();
    }
    if constexpr (APPLY) {
        pass_on(a, a.dlast, a.dh0, at.c, C);
    } else if (threadIdx.x < a.lanes) {
        float *m = a.maps + (size_t)blockIdx.x * 2 * a.width;
#pragma unroll
        for (int i = 0; i < C; i++)
            if (at.c + i < a.width) m[at.c + i] = chunk[i].a, m[a.width + at.c + i] = chunk[i].b;
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
uint32_t groups_of(const Scan &a, int n) { return (a.width + a.lanes * n - 1) / (a.lanes * n); }

// Lanes that share a row: a power of two from 8 to 64 that holds the channels.
// Chunks: as many workgroups as the card holds twice, of whole tiles.
void split(Scan &a, int n) {
    a.lanes = 8;
    while (a.lanes < 64 && a.lanes * n < a.width) a.lanes *= 2;
    const uint32_t tile = kThreads / a.lanes * kRows, tiles = (a.rows + tile - 1) / tile;
    const uint32_t groups = groups_of(a, n), most = groups < 1024 ? 1024 / groups : 1;
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

template <typename T, bool BACKWARD> int launch(Scan &a, void *work, hipStream_t s) {
    const uint32_t groups = groups_of(a, Lane<T>::n);
    // (a call of no rows still has states to pass on)
    const dim3 grid(a.chunks ? a.chunks : 1, groups);
    if (carried(a)) {
        a.maps = (float *)work;
        float *into = (float *)((uint8_t *)work + align16z((size_t)a.chunks * 2 * a.width * 4));
        int rc = enqueue(BACKWARD ? scan_rows_backward<T, false> : scan_rows<T, false>, grid, kThreads, 0, s, a);
        if (rc != NLB_OK) return rc;
        a.into = into;
        rc = enqueue(join_chunks<BACKWARD>, (a.width + 15) / 16, 1024, 0, s, a);
        if (rc != NLB_OK) return rc;
    }
    return enqueue(BACKWARD ? scan_rows_backward<T, true> : scan_rows<T, true>, grid, kThreads, 0, s, a);
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
    return c->dtype == NLB_DTYPE_BF16 ? launch<__bf16, false>(a, work, (hipStream_t)stream)
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
    return c->dtype == NLB_DTYPE_BF16 ? launch<__bf16, true>(a, work, (hipStream_t)stream)
                                      : launch<float, true>(a, work, (hipStream_t)stream);
}
