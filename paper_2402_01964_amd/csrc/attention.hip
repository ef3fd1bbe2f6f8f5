// attention.hip -- softmax attention over packed sequences, forward: tiles of
// query rows (attend_tiles), and one query row per sequence (attend_one,
// attend_join).
#include "attention.h"

namespace {

// ---------------------------------------------------------------- tiles
// A workgroup owns 128 query rows of one head and streams the keys and values
// in tiles of 64 (fp32: 32) rows through two LDS buffers: the next tile's
// global loads are in flight in registers while this one is multiplied, one
// barrier a tile.  A wavefront owns 32 rows; its scores are columns (see
// attention.h), so its softmax statistics are one value per lane and the
// probabilities go to the second product from the registers they are in.
// The running maximum follows a row's scores only when they pass it by more
// than 2^8: until then the sums carry factors of at most 2^8 and the
// accumulated values need no scaling.
//
// POS: 0 no bias and no closed keys; 1 bias by places: of a tile's gaps there
// are 32 + 128 - 1 at most, so their bias values are looked up once per tile;
// 2 positions given (bias by their gaps, closed keys).
//
// What the vector units do for a score bounds the kernel beside the matrix
// products (16 products of 32 cycles a block of 32 x 32 for 128 values, 16
// exponentials of 16 cycles and four other operations a lane's score), so
// scores stay in steps of 1 / scale2 and meet scale and maximum in the one
// fused operation before the exponential; masks run only in tiles that need
// them, and tiles whose gaps are all in one bucket add their bias to the
// maximum's term.  Measured (128 bf16 values, 16 heads): one causal sequence of
// 8000 rows with the bias 321 us (820 TFLOP/s of the open pairs, two thirds of
// what a large library product reaches), 24 sequences of 16 to 2048 rows 120 us
// (490).  The matrix cores are busy 43 % of the time, the vector units about as
// long; LDS reads are free of bank conflicts.  Finding the maximum only where a
// sum would overflow saved a tenth of the vector work and lost more than that,
// since the exponentials of one block then no longer ran beside the products of
// the other (355 to 385 us).
constexpr int kGaps = 192;

template <typename T, int DP, bool NARROW> constexpr uint32_t tiles_lds() {
    return (NARROW ? 1 : 2) * (Tile<T, DP, kByRows, NARROW>::bytes + Tile<T, DP, kByColumns, NARROW>::bytes) +
           2 * kGaps * 4 + kMaxBuckets * 8 +
           kCells + kMaxBuckets * 4;
}

template <typename T, int DP, int POS, bool EXACT, bool NARROW>
__global__ __launch_bounds__(kThreads, 2) void attend_tiles(Attend a) {
    using KT = Tile<T, DP, kByRows, NARROW>;
    using VT = Tile<T, DP, kByColumns, NARROW>;
    using G = KT;
    using S = Span<NARROW, G::rows>;
    const S span;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    float *extra = (float *)(lds + S::buffers * (KT::bytes + VT::bytes));   // [2][kGaps]: bias by gap, or positions
    float *bias = extra + 2 * kGaps;
    Buckets buckets = {(int32_t *)(bias + kMaxBuckets), (uint8_t *)(bias + 2 * kMaxBuckets), a.buckets - 1, 0};
    const uint32_t lane = threadIdx.x & 63u, col = lane & 31u;

    // heads of one key/value head follow each other at a distance of kv_heads:
    // workgroups that are dispatched to one XCD share keys and values
    const uint32_t id = a.first + blockIdx.x, hid = id % a.heads, slot = a.slots - 1 - id / a.heads;
    const uint32_t kvh = hid % a.kv_heads, head = kvh * a.group + hid / a.kv_heads;
    Seq sq;
    const uint32_t b = slot_owner(a.q_start, a.q_len, a.q_rows, a.batch, S::owned, slot, sq.tile);
    sequence(a, b, sq);
    if (sq.tile >= ((uint32_t)sq.lq + S::owned - 1) / S::owned) return;
    const int32_t row0 = sq.tile * S::owned, row = row0 + (int32_t)span.own + (int32_t)col, off = sq.lk - sq.lq;
    const bool there = row < sq.lq;

    Owned<T, DP> q;
    load_owned(q, a.q.p + (int64_t)(sq.q0 + row) * a.q.row + head * a.q.head, there, a.dim);
    sign_owned(q, a.scale);
    int32_t qpos = 0;
    if constexpr (POS == 2)
        if (there && a.q_pos) qpos = flip(a.q_pos[sq.q0 + row]);
    // keys [0, kend) are open to some row of the workgroup, [0, wend) of the wavefront
    const int32_t last = min(row0 + S::owned, sq.lq) - 1, wrow0 = row0 + (int32_t)span.own;
    const int32_t kend = a.causal ? min(sq.lk, last + off + 1) : sq.lk;
    const int32_t wend = a.causal ? min(sq.lk, min(wrow0 + 32, sq.lq) + off) : sq.lk;
    const int32_t limit = a.causal ? min(sq.lk, row + off + 1) : sq.lk;   // keys open to this lane's row
    const int32_t whole = a.causal ? min(sq.lk, wrow0 + off + 1) : sq.lk; // and to all of the wavefront's
    const uint8_t *kbase = a.k.p + (int64_t)sq.k0 * a.k.row + kvh * a.k.head;
    const uint8_t *vbase = a.v.p + (int64_t)sq.k0 * a.v.row + kvh * a.v.head;

    typename G::Regs kreg, vreg;
    tile_clear<G>(kreg);
    tile_clear<G>(vreg);
    uint32_t preg[POS == 2 ? G::per_thread : 1];
    const auto fetch = [&](int32_t k0) {
        tile_load<G, EXACT>(kreg, kbase + (int64_t)k0 * a.k.row, a.k.row, kend - k0, a.dim);
        tile_load<G, EXACT>(vreg, vbase + (int64_t)k0 * a.v.row, a.v.row, kend - k0, a.dim);
        if constexpr (POS == 2) tile_positions<G>(preg, a.k_pos + sq.k0 + k0, kend - k0);
    };
    // the gaps of the tile at k0: from least to least + owned + rows - 2
    const auto least = [&](int32_t k0) { return row0 + off - k0 - (G::rows - 1); };
    // writes the fetched tile and what the bias needs of it
    const auto stage = [&](int32_t k0, int buf) {
        uint8_t *kt = lds + buf * (KT::bytes + VT::bytes);
        if constexpr (!EXACT) {
            tile_settle<G>(kreg, a.dim);
            tile_settle<G>(vreg, a.dim);
        }
        if constexpr (POS == 2) {
            tile_close<G>(kreg, preg);
            tile_close<G>(vreg, preg);
            tile_store_positions<G>((int32_t *)extra + buf * kGaps, preg);
        }
        tile_store<KT>(kt, kreg, kend - k0);
        tile_store<VT>(kt + KT::bytes, vreg, kend - k0);
        if constexpr (POS == 1) {
            const int32_t x = (int32_t)threadIdx.x, lo = least(k0);
            uint32_t one;
            if (!one_bucket(buckets.bounds, a.buckets, lo, lo + S::owned + G::rows - 2, one) &&
                x < S::owned + G::rows - 1)
                extra[buf * kGaps + x] = bias[bucket_of(buckets.bounds, a.buckets, lo + x)];
        }
    };

    f32x16 acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) acc[d] = f32x16{};
    // m: the maximum in the scores' steps; up to 2^8 behind it
    float m = -INFINITY, sum = 0.0f;
    const float behind = 8.0f / a.scale2;

    if (kend > 0) fetch(0);                                    // (in flight beside the bias tables' loads)
    if (POS != 0 && a.buckets) {
        stage_bias<T>(a, head, buckets.bounds, bias);
        int32_t *ends = (int32_t *)(buckets.cells + kCells);
        __syncthreads();
        if constexpr (POS == 2) {
            fill_cells(buckets, ends);
        }
    }
    if (kend > 0) stage(0, 0);
    __syncthreads();
    int buf = 0;
    for (int32_t k0 = 0; k0 < kend; k0 += G::rows, buf ^= S::buffers - 1) {
        const bool more = k0 + G::rows < kend;
        if (more) fetch(k0 + G::rows);
        if (k0 + (int32_t)span.take < wend) {
            const uint8_t *kt = lds + buf * (KT::bytes + VT::bytes), *vt = kt + KT::bytes;
            const float *ex = extra + buf * kGaps;
            const bool ragged = k0 + (int32_t)span.take + S::rows > whole;
            float shift = 0.0f;                                // the bias where the tile has one bucket
            bool far = true, shut = false;
            if constexpr (POS == 1) {
                uint32_t one;
                far = one_bucket(buckets.bounds, a.buckets, least(k0), least(k0) + S::owned + G::rows - 2, one);
                if (far) shift = bias[one];
            }
            if constexpr (POS == 2) shut = __any(((const int32_t *)ex)[span.take + lane % S::rows] == kNoKeyFlipped);
            f32x16 s[S::blocks];
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < S::blocks; n++) {
                const int blk = span.take + n * 32;
                s[n] = f32x16{};
                product_rows<KT>(s[n], kt, blk, q);
                if (POS == 1 && !far) {
                    const float *e = ex + span.own + col + (G::rows - 1) - blk;
#pragma unroll
                    for (int r = 0; r < 16; r++) s[n][r] += e[-block_row(r)];
                }
                if (POS == 2 && a.buckets) {
                    int32_t gap[16];
                    uint32_t bk[16];
#pragma unroll
                    for (int r = 0; r < 16; r++) gap[r] = gap_of(qpos, ((const int32_t *)ex)[blk + block_row(r)]);
                    buckets_in(buckets, gap, bk);
#pragma unroll
                    for (int r = 0; r < 16; r++) s[n][r] += bias[bk[r]];
                }
                if (POS == 2 && shut) {
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        if (((const int32_t *)ex)[blk + block_row(r)] == kNoKeyFlipped) s[n][r] = -INFINITY;
                }
                if (ragged) {
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        if (k0 + blk + block_row(r) >= limit) s[n][r] = -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < 16; r++) top = fmaxf(top, s[n][r]);
            }
            top = halves_max(top) + shift;
            if (__any(top > m + behind)) {
                const float up = fmaxf(m, top);
                const float f = up == -INFINITY ? 1.0f : exp2_fast((m - up) * a.scale2);
                m = up;
                sum *= f;
#pragma unroll
                for (int d = 0; d < DP / 32; d++)
#pragma unroll
                    for (int r = 0; r < 16; r++) acc[d][r] *= f;
            }
            const float base = fmaf(shift, a.scale2, m == -INFINITY ? 0.0f : -m * a.scale2);
#pragma unroll
            for (int n = 0; n < S::blocks; n++) {
                float t[16];
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    t[r] = exp2_fast(fmaf(s[n][r], a.scale2, base));
                    sum += t[r];
                }
                Scores<T> p;
                pack(p, t);
                product_columns<VT>(acc, vt, span.take + n * 32, p);
            }
        }
        if (NARROW && more) __syncthreads();
        if (more) stage(k0 + G::rows, NARROW ? 0 : buf ^ 1);
        __syncthreads();
    }
    sum = halves_sum(sum);
    if constexpr (NARROW) {
        float *tops = (float *)lds, *sums = tops + 256;
        tops[threadIdx.x] = m;
        __syncthreads();
        float top = tops[lane];
#pragma unroll
        for (int w = 1; w < 4; w++) top = fmaxf(top, tops[w * 64 + lane]);
        const float f = m == top ? 1.0f : exp2_fast((m - top) * a.scale2);
        m = top;
        sums[threadIdx.x] = sum * f;
#pragma unroll
        for (int d = 0; d < DP / 32; d++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[d][r] *= f;
        __syncthreads();
        sum = sums[lane] + sums[64 + lane] + sums[128 + lane] + sums[192 + lane];
        join_waves<DP>(acc, sums + 256);
        if (threadIdx.x >= 64) return;
    }
    if (!there) return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    store_owned<T, DP>((uint8_t *)a.o.p + (int64_t)(sq.q0 + row) * a.o.row + head * a.o.head, a.dim, acc, inv);
    if (a.lse && lane < 32)
        a.lse[(size_t)(sq.q0 + row) * a.heads + head] =
            sum == 0.0f ? -INFINITY : (m * a.scale2 + log2_fast(sum)) * kLn2;
}

// ---------------------------------------------------------------- one query row
// A sequence's single query row (a retrieved list, or a new token over a long
// history) is bound by reading its keys and values once.  A wavefront takes up
// to GB query heads of one key/value head over at most `chunk` keys; a row's
// values lie across DP / (values in 16 bytes) neighbouring lanes, so one load
// takes a row from each of 64 / that many keys, and U such loads of keys and
// of values are in flight.  Each group of lanes keeps its own running maximum,
// sum and weighted values; the groups join once at the end.  Longer sequences
// have several chunks, whose results (maximum, sum, values in fp32) go to
// `part` and are joined by attend_join.  Wavefronts take chunk after chunk, so
// the bias table is staged once.  Measured: 16 sequences of 1 to 65 536 keys,
// 32 heads on 8, 128 bf16 values (2.03 GB): 386 us and 11 us for the join, 5.1
// TB/s, a plain copy's rate.
template <typename T, int DP, int GB>
__global__ __launch_bounds__(kThreads) void attend_one(Attend a) {
    using L = Lanes<T, DP>;
    constexpr int N = Chunk<T>::n, U = 4;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    int32_t *bounds = (int32_t *)lds;
    float *bias = (float *)(bounds + kMaxBuckets);            // [buckets][heads]
    if (a.buckets) {
        for (uint32_t i = threadIdx.x; i < kMaxBuckets; i += kThreads)
            bounds[i] = i + 1 < a.buckets ? a.bounds[i] : INT32_MAX;
        for (uint32_t i = threadIdx.x; i < a.buckets * a.heads; i += kThreads)
            bias[i] = bias2_of<T>(a, i / a.heads, i % a.heads);
        __syncthreads();
    }
    const uint32_t lane = threadIdx.x & 63u, c0 = (lane % L::per_row) * N, kr = lane / L::per_row;
    const uint32_t parts = (a.group + GB - 1) / GB, per_slot = a.kv_heads * parts;
    const uint64_t units = (uint64_t)a.slots * per_slot;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint64_t unit = blockIdx.x * 4ull + wave; unit < units; unit += gridDim.x * 4ull) {
        const uint32_t slot = unit / per_slot, kvh = unit % a.kv_heads, g0 = (unit % per_slot) / a.kv_heads * GB;
        const uint32_t head0 = kvh * a.group + g0, ng = min((uint32_t)GB, a.group - g0);
        Seq sq;
        uint32_t b = slot;
        sq.tile = 0;
        if (a.slots != a.batch) b = slot_owner(a.k_start, a.k_len, a.k_rows, a.batch, a.chunk, slot, sq.tile);
        sequence(a, b, sq);
        const uint32_t chunks = max(1u, ((uint32_t)sq.lk + a.chunk - 1) / a.chunk);
        if (sq.tile >= chunks) continue;
        const int32_t first = sq.tile * a.chunk, n = min((int32_t)a.chunk, sq.lk - first);

        float q[GB][N], acc[GB][N], m[GB], sum[GB];
#pragma unroll
        for (int g = 0; g < GB; g++) {
            u32x4 x = {0, 0, 0, 0};
            if ((uint32_t)g < ng)
                x = load_chunk<T>(a.q.p + (int64_t)b * a.q.row + (head0 + g) * a.q.head, c0, a.dim);
            unpack<T>(x, q[g]);
#pragma unroll
            for (int i = 0; i < N; i++) {
                q[g][i] *= a.signed2;
                acc[g][i] = 0.0f;
            }
            m[g] = -INFINITY;
            sum[g] = 0.0f;
        }
        const int32_t qpos = a.buckets ? (a.q_pos ? flip(a.q_pos[b]) : flip((uint32_t)sq.lk - 1)) : 0;
        const uint8_t *kp = a.k.p + (int64_t)(sq.k0 + first) * a.k.row + kvh * a.k.head;
        const uint8_t *vp = a.v.p + (int64_t)(sq.k0 + first) * a.v.row + kvh * a.v.head;
        for (int32_t j0 = 0; j0 < n; j0 += L::rows * U) {
            u32x4 k[U], v[U];
            uint32_t pos[U];
            bool open[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int32_t j = j0 + u * L::rows + kr;
                open[u] = j < n;
                pos[u] = first + j;
                if (a.k_pos && open[u]) {
                    pos[u] = a.k_pos[sq.k0 + first + j];
                    open[u] = pos[u] != kNoKey;
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int32_t j = j0 + u * L::rows + kr;
                k[u] = v[u] = u32x4{0, 0, 0, 0};
                if (open[u]) {
                    k[u] = load_chunk<T>(kp + j * a.k.row, c0, a.dim);
                    v[u] = load_chunk<T>(vp + j * a.v.row, c0, a.dim);
                }
            }
            float t[U][GB];
#pragma unroll
            for (int u = 0; u < U; u++) {
                float x[N];
                unpack<T>(k[u], x);
#pragma unroll
                for (int g = 0; g < GB; g++) {
                    float s = 0.0f;
#pragma unroll
                    for (int i = 0; i < N; i++) s = fmaf(q[g][i], x[i], s);
                    t[u][g] = lanes_sum<L::per_row>(s);
                }
                const uint32_t at =
                    a.buckets ? bucket_of(bounds, a.buckets, gap_of(qpos, flip(pos[u]))) * a.heads + head0 : 0;
#pragma unroll
                for (int g = 0; g < GB; g++) {
                    if (a.buckets && (uint32_t)g < ng) t[u][g] += bias[at + g];
                    if (!open[u]) t[u][g] = -INFINITY;
                }
            }
            float p[U][GB];
#pragma unroll
            for (int g = 0; g < GB; g++) {
                float up = m[g];
#pragma unroll
                for (int u = 0; u < U; u++) up = fmaxf(up, t[u][g]);
                const float base = up == -INFINITY ? 0.0f : up, f = exp2_fast(m[g] - base);
                m[g] = up;
                sum[g] *= f;
#pragma unroll
                for (int i = 0; i < N; i++) acc[g][i] *= f;
#pragma unroll
                for (int u = 0; u < U; u++) {
                    p[u][g] = exp2_fast(t[u][g] - base);
                    sum[g] += p[u][g];
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                float x[N];
                unpack<T>(v[u], x);
#pragma unroll
                for (int g = 0; g < GB; g++)
#pragma unroll
                    for (int i = 0; i < N; i++) acc[g][i] = fmaf(p[u][g], x[i], acc[g][i]);
            }
        }
#pragma unroll
        for (int g = 0; g < GB; g++) {
            if ((uint32_t)g >= ng) break;
            float up = m[g];
#pragma unroll
            for (int w = L::per_row; w < 64; w *= 2) up = fmaxf(up, __shfl_xor(up, w));
            const float base = up == -INFINITY ? 0.0f : up, f = exp2_fast(m[g] - base);
            sum[g] *= f;
#pragma unroll
            for (int i = 0; i < N; i++) acc[g][i] *= f;
#pragma unroll
            for (int w = L::per_row; w < 64; w *= 2) {
                sum[g] += __shfl_xor(sum[g], w);
#pragma unroll
                for (int i = 0; i < N; i++) acc[g][i] += __shfl_xor(acc[g][i], w);
            }
            const uint32_t head = head0 + g;
            if (chunks == 1) {
                const float inv = sum[g] == 0.0f ? 0.0f : 1.0f / sum[g];
#pragma unroll
                for (int i = 0; i < N; i++) acc[g][i] *= inv;
                if (kr == 0 && c0 < a.dim)
                    store_values<T, N>((uint8_t *)a.o.p + (int64_t)b * a.o.row + head * a.o.head, c0, a.dim, acc[g]);
                if (lane == 0 && a.lse)
                    a.lse[(size_t)b * a.heads + head] =
                        sum[g] == 0.0f ? -INFINITY : (up + log2_fast(sum[g])) * kLn2;
            } else {
                float *part = a.part + ((size_t)slot * a.heads + head) * (a.dim + 2);
                if (lane == 0) {
                    part[0] = up;
                    part[1] = sum[g];
                }
                if (kr == 0)
#pragma unroll
                    for (int i = 0; i < N; i++)
                        if (c0 + i < a.dim) part[2 + c0 + i] = acc[g][i];
            }
        }
    }
}

// Joins the chunks of the sequences that have more than one: a workgroup per
// sequence and head, values across the lanes, every fourth run of 64 chunks a
// wavefront.
template <typename T>
__global__ __launch_bounds__(kThreads) void attend_join(Attend a) {
    __shared__ float tops[4], sums[4], values[4][128];
    const uint32_t id = a.first + blockIdx.x, b = id / a.heads, head = id % a.heads;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    Seq sq;
    sequence(a, b, sq);
    const uint32_t chunks = ((uint32_t)sq.lk + a.chunk - 1) / a.chunk;
    if (chunks < 2) return;
    const size_t step = (size_t)a.heads * (a.dim + 2);
    const float *part = a.part + (size_t)(sq.k0 / a.chunk + b) * step + head * (a.dim + 2);
    float m = -INFINITY;
    for (uint32_t i = threadIdx.x; i < chunks; i += kThreads) m = fmaxf(m, part[i * step]);
#pragma unroll
    for (int w = 1; w < 64; w *= 2) m = fmaxf(m, __shfl_xor(m, w));
    if (lane == 0) tops[wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float base = m == -INFINITY ? 0.0f : m;
    const uint32_t c0 = min(lane, a.dim - 1), c1 = min(lane + 64, a.dim - 1);
    float sum = 0.0f, x0 = 0.0f, x1 = 0.0f;
    for (uint32_t i0 = wave * 64; i0 < chunks; i0 += kThreads) {
        const uint32_t n = min(64u, chunks - i0);
        const float f = lane < n ? exp2_fast(part[(i0 + lane) * step] - base) : 0.0f;
        if (lane < n) sum = fmaf(f, part[(i0 + lane) * step + 1], sum);
        for (uint32_t u0 = 0; u0 < n; u0 += 8) {              // sixteen loads in flight
            float v0[8], v1[8];
#pragma unroll
            for (uint32_t u = 0; u < 8; u++) {
                const float *p = part + (i0 + min(u0 + u, n - 1)) * step + 2;
                v0[u] = p[c0];
                v1[u] = p[c1];
            }
#pragma unroll
            for (uint32_t u = 0; u < 8; u++) {
                const float g = u0 + u < n ? __shfl(f, u0 + u) : 0.0f;
                x0 = fmaf(g, v0[u], x0);
                x1 = fmaf(g, v1[u], x1);
            }
        }
    }
#pragma unroll
    for (int w = 1; w < 64; w *= 2) sum += __shfl_xor(sum, w);
    values[wave][lane] = x0;
    values[wave][lane + 64] = x1;
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = sums[0] + sums[1] + sums[2] + sums[3];
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const uint32_t t = threadIdx.x;
    if (t < a.dim)
        ((T *)(a.o.p + (int64_t)b * a.o.row + head * a.o.head))[t] =
            (T)((values[0][t] + values[1][t] + values[2][t] + values[3][t]) * inv);
    if (t == 0 && a.lse) a.lse[(size_t)b * a.heads + head] = sum == 0.0f ? -INFINITY : (m + log2_fast(sum)) * kLn2;
}

// ---------------------------------------------------------------- short lists
// Many short lists with a query row each: a group of lanes that spans one row
// takes a whole list (and up to GB query heads of one key/value head), so a
// wavefront works on 4 to 16 lists and nothing is joined across lanes but a
// score's own sum.  A list's open keys are found up to 64 at a time; closed ones
// are neither read nor multiplied.  Measured: 300 000 lists of 10 slots, six in
// ten open, two heads of 64 bf16 values (1.09 GB): 221 us, 4.9 TB/s (a wavefront
// a list 735 us: its joining across lanes took most of the instructions).
// (fp32 rows fit five wavefronts on a SIMD without spilling, 8300 lists of 20
// slots 41 to 26 us; bf16 rows spill there, 300 000 lists of 10 223 to 315 us)
template <typename T, int DP, int GB>
__global__ __launch_bounds__(kThreads, GB == 1 && sizeof(T) == 4 ? 5 : 1) void attend_lists(Attend a) {
    using L = Lanes<T, DP>;
    constexpr int N = Chunk<T>::n, U = 4;
    constexpr int K = std::min(kListKeys, 4 * L::per_row);    // (more positions in registers cost a wavefront)
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    int32_t *bounds = (int32_t *)lds;
    float *bias = (float *)(bounds + kMaxBuckets);            // [buckets][heads]
    uint8_t *codes = (uint8_t *)(bias + a.buckets * a.heads) + (threadIdx.x >> 6) * L::rows * kListKeys;
    if (a.buckets) {
        for (uint32_t i = threadIdx.x; i < kMaxBuckets; i += kThreads)
            bounds[i] = i + 1 < a.buckets ? a.bounds[i] : INT32_MAX;
        for (uint32_t i = threadIdx.x; i < a.buckets * a.heads; i += kThreads)
            bias[i] = bias2_of<T>(a, i / a.heads, i % a.heads);
        __syncthreads();
    }
    const uint32_t lane = threadIdx.x & 63u, c0 = (lane % L::per_row) * N, kr = lane / L::per_row;
    const uint32_t parts = (a.group + GB - 1) / GB, per_list = a.kv_heads * parts;
    const uint64_t units = (uint64_t)a.batch * per_list, turn = (uint64_t)gridDim.x * 4 * L::rows;
    for (uint64_t unit0 = (blockIdx.x * 4ull + (threadIdx.x >> 6)) * L::rows; unit0 < units; unit0 += turn) {
        const bool there = unit0 + kr < units;
        const uint64_t unit = there ? unit0 + kr : 0;
        const uint32_t b = unit / per_list, in = unit % per_list;
        const uint32_t kvh = in % a.kv_heads, g0 = in / a.kv_heads * GB;
        const uint32_t head0 = kvh * a.group + g0, ng = min((uint32_t)GB, a.group - g0);
        Seq sq;
        sequence(a, b, sq);
        if (!there) sq.lk = 0;
        // (the first positions are in flight with q)
        u32x4 raw[GB];
#pragma unroll
        for (int g = 0; g < GB; g++) {
            raw[g] = u32x4{0, 0, 0, 0};
            if ((uint32_t)g < ng)
                raw[g] = load_chunk<T>(a.q.p + (int64_t)b * a.q.row + (head0 + g) * a.q.head, c0, a.dim);
        }
        ListPositions<L::per_row, K> keys;
        keys.load(a, sq.k0, sq.lk, 0);
        float q[GB][N], acc[GB][N], m[GB], sum[GB];
#pragma unroll
        for (int g = 0; g < GB; g++) {
            unpack<T>(raw[g], q[g]);
#pragma unroll
            for (int i = 0; i < N; i++) {
                q[g][i] *= a.signed2;
                acc[g][i] = 0.0f;
            }
            m[g] = -INFINITY;
            sum[g] = 0.0f;
        }
        const int32_t qpos = a.buckets ? (a.q_pos ? flip(a.q_pos[b]) : flip((uint32_t)sq.lk - 1)) : 0;
        const uint8_t *kp = a.k.p + (int64_t)sq.k0 * a.k.row + kvh * a.k.head;
        const uint8_t *vp = a.v.p + (int64_t)sq.k0 * a.v.row + kvh * a.v.head;
        for (int32_t j0 = 0; __any(j0 < sq.lk); j0 += K) {
            if (j0) keys.load(a, sq.k0, sq.lk, j0);
            wave_lds_fence();
            uint64_t mine = open_keys(a, bounds, codes, keys, sq.lk, j0, qpos);
            wave_lds_fence();
            while (__any(mine != 0)) {
                u32x4 k[U], v[U];
                bool open[U];
                uint32_t at[U];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    open[u] = mine != 0;
                    at[u] = open[u] ? __builtin_ctzll(mine) : 0;
                    mine &= mine - 1;
                    k[u] = v[u] = u32x4{0, 0, 0, 0};
                    if (open[u]) {
                        k[u] = load_chunk<T>(kp + (int64_t)(j0 + at[u]) * a.k.row, c0, a.dim);
                        v[u] = load_chunk<T>(vp + (int64_t)(j0 + at[u]) * a.v.row, c0, a.dim);
                    }
                }
                float t[U][GB];
#pragma unroll
                for (int u = 0; u < U; u++) {
                    float x[N];
                    unpack<T>(k[u], x);
                    const uint32_t bk = a.buckets ? codes[kr * kListKeys + at[u]] * a.heads + head0 : 0;
#pragma unroll
                    for (int g = 0; g < GB; g++) {
                        float s = 0.0f;
#pragma unroll
                        for (int i = 0; i < N; i++) s = fmaf(q[g][i], x[i], s);
                        t[u][g] = lanes_sum<L::per_row>(s);
                        if (a.buckets && (uint32_t)g < ng) t[u][g] += bias[bk + g];
                        if (!open[u]) t[u][g] = -INFINITY;
                    }
                }
                float p[U][GB];
#pragma unroll
                for (int g = 0; g < GB; g++) {
                    float up = m[g];
#pragma unroll
                    for (int u = 0; u < U; u++) up = fmaxf(up, t[u][g]);
                    const float base = up == -INFINITY ? 0.0f : up, f = exp2_fast(m[g] - base);
                    m[g] = up;
                    sum[g] *= f;
#pragma unroll
                    for (int i = 0; i < N; i++) acc[g][i] *= f;
#pragma unroll
                    for (int u = 0; u < U; u++) {
                        p[u][g] = exp2_fast(t[u][g] - base);
                        sum[g] += p[u][g];
                    }
                }
#pragma unroll
                for (int u = 0; u < U; u++) {
                    float x[N];
                    unpack<T>(v[u], x);
#pragma unroll
                    for (int g = 0; g < GB; g++)
#pragma unroll
                        for (int i = 0; i < N; i++) acc[g][i] = fmaf(p[u][g], x[i], acc[g][i]);
                }
            }
        }
        if (!there) continue;
#pragma unroll
        for (int g = 0; g < GB; g++) {
            if ((uint32_t)g >= ng) break;
            const uint32_t head = head0 + g;
            const float inv = sum[g] == 0.0f ? 0.0f : 1.0f / sum[g];
#pragma unroll
            for (int i = 0; i < N; i++) acc[g][i] *= inv;
            if (c0 < a.dim)
                store_values<T, N>((uint8_t *)a.o.p + (int64_t)b * a.o.row + head * a.o.head, c0, a.dim, acc[g]);
            if (c0 == 0 && a.lse)
                a.lse[(size_t)b * a.heads + head] = sum[g] == 0.0f ? -INFINITY : (m[g] + log2_fast(sum[g])) * kLn2;
        }
    }
}

// ---------------------------------------------------------------- launches
template <typename T, int DP, bool EXACT, bool NARROW>
int launch_tiles(const Attend &a, hipStream_t stream) {
    const int pos = a.k_pos ? 2 : a.buckets ? 1 : 0;
    const auto kernel = pos == 2   ? attend_tiles<T, DP, 2, EXACT, NARROW>
                        : pos == 1 ? attend_tiles<T, DP, 1, EXACT, NARROW>
                                   : attend_tiles<T, DP, 0, EXACT, NARROW>;
    constexpr uint32_t bytes = tiles_lds<T, DP, NARROW>();
    if (!allow_lds(kernel, bytes)) return NLB_EDEVICE;
    return enqueue_blocks(kernel, a, (uint64_t)a.slots * a.heads, bytes, stream);
}

template <typename T, int DP>
int launch_single(const Attend &a, Form form, hipStream_t stream) {
    const int gb = a.group >= 4 ? 4 : a.group >= 2 ? 2 : 1;
    const uint64_t parts = (a.group + gb - 1) / gb;
    uint32_t bytes = kMaxBuckets * 4 + a.buckets * a.heads * 4;
    if (form == kLists) {
        constexpr uint32_t rows = 4 * Lanes<T, DP>::rows;
        const auto kernel = gb == 4   ? attend_lists<T, DP, 4>
                            : gb == 2 ? attend_lists<T, DP, 2>
                                      : attend_lists<T, DP, 1>;
        bytes += rows * kListKeys;
        if (!allow_lds(kernel, bytes)) return NLB_EDEVICE;
        const uint64_t need = ((uint64_t)a.batch * a.kv_heads * parts + rows - 1) / rows;
        return enqueue(kernel, (uint32_t)std::min<uint64_t>(need, 256 * 8), kThreads, bytes, stream, a);
    } else {
        const auto kernel = gb == 4 ? attend_one<T, DP, 4> : gb == 2 ? attend_one<T, DP, 2> : attend_one<T, DP, 1>;
        if (!allow_lds(kernel, bytes)) return NLB_EDEVICE;
        const uint64_t need = ((uint64_t)a.slots * a.kv_heads * parts + 3) / 4;
        const int rc = enqueue(kernel, (uint32_t)std::min<uint64_t>(need, 256 * 8), kThreads, bytes, stream, a);
        if (rc != NLB_OK || a.slots == a.batch) return rc;
        return enqueue_blocks(attend_join<T>, a, (uint64_t)a.batch * a.heads, 0, stream);
    }
}

template <typename T, int DP> int launch_form(const Attend &a, const Forward &f, hipStream_t s) {
    if (f.form != kTiles) return launch_single<T, DP>(a, f.form, s);
    if constexpr (DP * sizeof(T) <= 256)
        if (f.narrow) return launch_tiles<T, DP, false, true>(a, s);
    return exact_rows(a, a.k) && exact_rows(a, a.v) ? launch_tiles<T, DP, true, false>(a, s)
                                                    : launch_tiles<T, DP, false, false>(a, s);
}

template <typename T> int launch(const Attend &a, const Forward &f, hipStream_t s) {
    return a.dim <= 32   ? launch_form<T, 32>(a, f, s)
           : a.dim <= 64 ? launch_form<T, 64>(a, f, s)
                         : launch_form<T, 128>(a, f, s);
}

}  // namespace

extern "C" int nlb_attention_work(const nlb_att_call *c, int32_t backward, size_t *bytes) {
    Attend a;
    if (!bytes) return NLB_EINVAL;
    const int rc = fill_call(c, a);
    if (rc != NLB_OK) return rc;
    *bytes = backward ? plan_backward(a).bytes : plan_forward(a).bytes;
    return NLB_OK;
}

extern "C" int nlb_attention(const nlb_att_call *c, const nlb_att_rows *o, float *lse, void *work, size_t work_bytes,
                             void *stream) {
    Attend a;
    int rc = fill_call(c, a);
    if (rc != NLB_OK) return rc;
    if ((rc = fill_rows(c, o, true, a.o)) != NLB_OK || (uintptr_t)lse % 4 || (uintptr_t)work % 16) return NLB_EINVAL;
    const Forward f = plan_forward(a);
    if (f.slots > f.most) return NLB_EINVAL;
    if (work_bytes < f.bytes || (f.bytes && !work)) return NLB_ESCRATCH;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    if (a.q_rows == 0) return NLB_OK;
    a.lse = lse;
    a.part = (float *)work;
    a.slots = (uint32_t)f.slots;
    a.chunk = f.chunk;
    return c->dtype == NLB_DTYPE_BF16 ? launch<__bf16>(a, f, (hipStream_t)stream)
                                      : launch<float>(a, f, (hipStream_t)stream);
}
