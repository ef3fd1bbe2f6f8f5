// attention_backward.hip -- gradients of softmax attention over packed
// sequences.  With p_ij as in the forward pass and D_i = sum_j p_ij dp_ij:
//   dp_ij = do_i . v_j,   ds_ij = p_ij (dp_ij - D_i)
//   dq_i = scale sum_j ds_ij k_j,   dk_j = scale sum_i ds_ij q_i
//   dv_j = sum_i p_ij do_i,   dbias[b][h] = sum of ds_ij over the pairs of bucket b
// The probabilities are computed again from the scores and lse.  Sums over
// rows and sums over keys are taken by different kernels (backward_rows,
// backward_keys), each of which owns what it sums: no atomics on results, the
// same bits each time, at the price of computing the scores and dp twice.
#include "attention.h"

namespace {

constexpr int kGaps = 192;               // gaps of a tile of owned rows and streamed rows

// 2^(t - L) is zero for a row without open keys.
__device__ __forceinline__ float row_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// ---------------------------------------------------------------- rows
// A workgroup owns 128 query rows of one head and streams keys and values as
// the forward pass does.  D is do . o, which is as far off as o: rounded to
// bf16, and from probabilities rounded to bf16.  A first pass over the keys adds
// sum_j p_j (dp_j - do . o), so that the ds of a row add up to zero as they
// should (fp32 rows do without it unless a bias gradient is wanted, which is
// a difference of large sums).  Without it dq and dk of 128 bf16 values are
// 2.6e-3 to 3.1e-3 off (2-norm, relative) where rounding them and ds alone
// makes 2.4e-3, and of a bucket that takes most of a row's weight nothing is
// left; it takes two products of seven more.
//
// The bias gradient: each thread adds its ds to its own column of an LDS table
// [buckets][threads], four at a time: reads, sums over equal buckets among the
// four, writes in order (LDS float atomics, about three cycles a lane, made
// the pass four times as long).  Tiles whose gaps all lie in the first or the
// last bucket add to a register.  The columns are summed at the end in a fixed
// order into part[slot][head][bucket].
//
// Measured: 8095 causal rows in two sequences, 16 heads of 128 bf16 values: 365
// us for five products (920 TFLOP/s); 7584 rows in 8 sequences, 8 heads of 64
// with the bias and its gradient 108 us, 523 with atomics on its table.
template <typename T, int DP, bool NARROW> constexpr uint32_t rows_lds(uint32_t buckets) {
    return (NARROW ? 1 : 2) * (Tile<T, DP, kBothWays, NARROW>::bytes + Tile<T, DP, kByRows, NARROW>::bytes) +
           2 * kGaps * 8 + kMaxBuckets * 8 +
           kCells + kMaxBuckets * 4 + (1 + buckets) * kThreads * 4;
}

__device__ __forceinline__ void add_four(float *column, const uint32_t (&b)[4], const float (&x)[4]) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = column[b[i] * kThreads];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        v[i] += x[i];
#pragma unroll
        for (int j = 0; j < i; j++)
            if (b[j] == b[i]) v[i] += x[j];
    }
#pragma unroll
    for (int i = 0; i < 4; i++) column[b[i] * kThreads] = v[i];
}

// (rows of 512 bytes leave registers for one wavefront on a SIMD, rows of 256
// with the bias table LDS for one workgroup on a CU)
template <typename T, int DP, int POS, bool EXACT, bool NARROW>
__global__ __launch_bounds__(kThreads, DP * sizeof(T) > (POS ? 128 : 256) ? 1 : 2) void backward_rows(Attend a) {
    using KT = Tile<T, DP, kBothWays, NARROW>;
    using VT = Tile<T, DP, kByRows, NARROW>;
    using G = KT;
    using S = Span<NARROW, G::rows>;
    const S span;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    // [2][kGaps] bias by gap, or positions; [2][kGaps] buckets by gap
    float *extra = (float *)(lds + S::buffers * (KT::bytes + VT::bytes));
    uint32_t *code = (uint32_t *)(extra + 2 * kGaps);
    float *bias = (float *)(code + 2 * kGaps);
    Buckets buckets = {(int32_t *)(bias + kMaxBuckets), (uint8_t *)(bias + 2 * kMaxBuckets), a.buckets - 1, 0};
    int32_t *cell_ends = (int32_t *)(buckets.cells + kCells);
    float *shares = (float *)(cell_ends + kMaxBuckets);       // [threads]
    float *hist = shares + kThreads;                          // [buckets][threads]
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, col = lane & 31u;
    const uint32_t id = a.first + blockIdx.x, hid = id % a.heads, slot = a.slots - 1 - id / a.heads;
    const uint32_t kvh = hid % a.kv_heads, head = kvh * a.group + hid / a.kv_heads;
    const bool want = POS != 0 && a.part;                     // the bias gradient
    Seq sq;
    const uint32_t b = slot_owner(a.q_start, a.q_len, a.q_rows, a.batch, S::owned, slot, sq.tile);
    sequence(a, b, sq);
    if (sq.tile >= ((uint32_t)sq.lq + S::owned - 1) / S::owned) {
        if (want && threadIdx.x < a.buckets) a.part[((size_t)slot * a.heads + head) * a.buckets + threadIdx.x] = 0.0f;
        return;
    }
    const int32_t row0 = sq.tile * S::owned, row = row0 + (int32_t)span.own + (int32_t)col, off = sq.lk - sq.lq;
    const bool there = row < sq.lq;
    const size_t stat = (size_t)(sq.q0 + row) * a.heads + head;

    Owned<T, DP> q, dout;
    load_owned(q, a.q.p + (int64_t)(sq.q0 + row) * a.q.row + head * a.q.head, there, a.dim);
    load_owned(dout, a.dout.p + (int64_t)(sq.q0 + row) * a.dout.row + head * a.dout.head, there, a.dim);
    sign_owned(q, a.scale);
    int32_t qpos = 0;
    if constexpr (POS == 2)
        if (there && a.q_pos) qpos = flip(a.q_pos[sq.q0 + row]);
    float L = there ? row_log2(a.lse[stat]) : INFINITY;
    float D = 0.0f;                                           // do . o, corrected by the first pass
    {
        Owned<T, DP> o;
        load_owned(o, a.o.p + (int64_t)(sq.q0 + row) * a.o.row + head * a.o.head, there, a.dim);
#pragma unroll
        for (int s = 0; s < Owned<T, DP>::steps; s++) {
            float x[Chunk<T>::n], y[Chunk<T>::n];
            unpack<T>(o.x[s], x);
            unpack<T>(dout.x[s], y);
#pragma unroll
            for (int i = 0; i < Chunk<T>::n; i++) D = fmaf(x[i], y[i], D);
        }
        D = halves_sum(D);
    }
    float more_D = 0.0f, weight = 0.0f;
    const int32_t last = min(row0 + S::owned, sq.lq) - 1, wrow0 = row0 + (int32_t)span.own;
    const int32_t kend = a.causal ? min(sq.lk, last + off + 1) : sq.lk;
    const int32_t wend = a.causal ? min(sq.lk, min(wrow0 + 32, sq.lq) + off) : sq.lk;
    const int32_t limit = a.causal ? min(sq.lk, row + off + 1) : sq.lk;
    const int32_t whole = a.causal ? min(sq.lk, wrow0 + off + 1) : sq.lk;
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
    const auto least = [&](int32_t k0) { return row0 + off - k0 - (G::rows - 1); };
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
                x < S::owned + G::rows - 1) {
                const uint32_t n = bucket_of(buckets.bounds, a.buckets, lo + x);
                code[buf * kGaps + x] = n;
                extra[buf * kGaps + x] = bias[n];
            }
        }
    };

    if (kend > 0) fetch(0);                                    // (in flight beside the bias tables' loads)
    if (POS != 0 && a.buckets) {
        stage_bias<T>(a, head, buckets.bounds, bias);
        if (want)
            for (uint32_t i = 0; i < a.buckets; i++) hist[i * kThreads + threadIdx.x] = 0.0f;
        __syncthreads();
        if constexpr (POS == 2) {
            fill_cells(buckets, cell_ends);
        }
    }
    if (kend > 0) stage(0, 0);
    __syncthreads();

    f32x16 acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) acc[d] = f32x16{};
    float ends[2] = {0.0f, 0.0f};                             // ds of the first and the last bucket
    // one pass over the keys: FIRST sums D, the other dq (and the bias gradient)
    const auto pass = [&](auto first_pass) {
        constexpr bool FIRST = decltype(first_pass)::value;
        f32x16 minus_D;                                       // what the products of do and v start from
#pragma unroll
        for (int r = 0; r < 16; r++) minus_D[r] = -D;
        int buf = 0;
        for (int32_t k0 = 0; k0 < kend; k0 += G::rows, buf ^= S::buffers - 1) {
            const bool more = k0 + G::rows < kend;
            if (more) fetch(k0 + G::rows);
            if (k0 + (int32_t)span.take < wend) {
                const uint8_t *kt = lds + buf * (KT::bytes + VT::bytes), *vt = kt + KT::bytes;
                const float *ex = extra + buf * kGaps;
                const bool ragged = k0 + (int32_t)span.take + S::rows > whole;
                bool far = true, shut = false;
                uint32_t one = 0;
                float base = -L;
                if constexpr (POS == 1) {
                    far = one_bucket(buckets.bounds, a.buckets, least(k0), least(k0) + S::owned + G::rows - 2, one);
                    if (far) base = fmaf(bias[one], a.scale2, base);
                }
                if constexpr (POS == 2)
                    shut = __any(((const int32_t *)ex)[span.take + lane % S::rows] == kNoKeyFlipped);
#pragma unroll
                for (int n = 0; n < S::blocks; n++) {
                    const int blk = span.take + n * 32;
                    f32x16 s = {}, dp = minus_D;
                    product_rows<KT>(s, kt, blk, q);
                    product_rows<VT>(dp, vt, blk, dout);
                    uint32_t bk[POS == 0 ? 1 : 16];
                    if (POS == 1 && !far) {
                        const uint32_t at = span.own + col + (G::rows - 1) - blk;
#pragma unroll
                        for (int r = 0; r < 16; r++) {
                            s[r] += ex[at - block_row(r)];
                            if (!FIRST) bk[r % (POS == 0 ? 1 : 16)] = code[buf * kGaps + at - block_row(r)];
                        }
                    }
                    if (POS == 2 && a.buckets) {
                        int32_t gap[16];
                        uint32_t nb[16];
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            gap[r] = gap_of(qpos, ((const int32_t *)ex)[blk + block_row(r)]);
                        buckets_in(buckets, gap, nb);
#pragma unroll
                        for (int r = 0; r < 16; r++) {
                            s[r] += bias[nb[r]];
                            if (!FIRST) bk[r % (POS == 0 ? 1 : 16)] = nb[r];
                        }
                    }
                    if (POS == 2 && shut) {
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            if (((const int32_t *)ex)[blk + block_row(r)] == kNoKeyFlipped) s[r] = -INFINITY;
                    }
                    if (ragged) {
#pragma unroll
                        for (int r = 0; r < 16; r++)
                            if (k0 + blk + block_row(r) >= limit) s[r] = -INFINITY;
                    }
                    float ds[16];
#pragma unroll
                    for (int r = 0; r < 16; r++) {
                        const float p = exp2_fast(fmaf(s[r], a.scale2, base));
                        if constexpr (FIRST) more_D = fmaf(p, dp[r], more_D);
                        else ds[r] = p * dp[r];
                        if (FIRST && sizeof(T) == 4) weight += p;
                    }
                    if constexpr (!FIRST) {
                        if (want && POS == 1 && far) {
                            float x = 0.0f;
#pragma unroll
                            for (int r = 0; r < 16; r++) x += ds[r];
                            ends[0] += one == 0 ? x : 0.0f;
                            ends[1] += one == 0 ? 0.0f : x;
                        } else if (want) {
#pragma unroll
                            for (int r = 0; r < 16; r += 4) {
                                constexpr int kept = POS == 0 ? 1 : 16;
                                const uint32_t four[4] = {bk[r % kept], bk[(r + 1) % kept], bk[(r + 2) % kept],
                                                          bk[(r + 3) % kept]};
                                const float x[4] = {ds[r], ds[r + 1], ds[r + 2], ds[r + 3]};
                                add_four(hist + threadIdx.x, four, x);
                            }
                        }
                        Scores<T> p;
                        pack(p, ds);
                        product_columns<KT>(acc, kt, blk, p);
                    }
                }
            }
            if (NARROW && more) __syncthreads();
            if (more) stage(k0 + G::rows, NARROW ? 0 : buf ^ 1);
            __syncthreads();
        }
    };
    if (sizeof(T) == 2 || want) {
        pass(std::true_type{});
        if (kend > G::rows) {                                 // (else the one tile is still there)
            fetch(0);
            stage(0, 0);
        }
        __syncthreads();
        const auto row_sum = [&](float x) {
            x = halves_sum(x);
            if constexpr (NARROW) {
                shares[threadIdx.x] = x;
                __syncthreads();
                x = shares[lane] + shares[64 + lane] + shares[128 + lane] + shares[192 + lane];
                __syncthreads();
            }
            return x;
        };
        D += row_sum(more_D);
        // fp32: lse is rounded, and a row's probabilities with it
        if constexpr (sizeof(T) == 4) {
            weight = row_sum(weight);
            if (weight > 0.5f) L += log2_fast(weight);
        }
    }
    const bool first_wave = !NARROW || wave == 0;
    if (there && lane < 32 && first_wave) a.stats[stat] = make_float2(L, D);
    pass(std::false_type{});
    if constexpr (NARROW) join_waves<DP>(acc, (float *)lds);
    if (there && first_wave)
        store_owned<T, DP>((uint8_t *)a.dq.p + (int64_t)(sq.q0 + row) * a.dq.row + head * a.dq.head, a.dim, acc,
                           a.scale);
    if (want) {
        if (POS == 1) {
            hist[threadIdx.x] += ends[0];
            hist[(a.buckets - 1) * kThreads + threadIdx.x] += ends[1];
            __syncthreads();
        }
        for (uint32_t i = wave; i < a.buckets; i += 4) {
            float x = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; w++) x += hist[i * kThreads + w * 64 + lane];
#pragma unroll
            for (int w = 1; w < 64; w *= 2) x += __shfl_xor(x, w);
            if (lane == 0) a.part[((size_t)slot * a.heads + head) * a.buckets + i] = x;
        }
    }
}

// ---------------------------------------------------------------- keys
// A workgroup owns 128 keys of one key/value head and streams the query rows
// that see them, head by head of its group: q and do in tiles through two LDS
// buffers, lse and D beside them.  Blocks of scores have the owned keys as
// columns here, so p and ds go to the products that sum over rows from the
// registers they are in.
//
// WHAT: 1 dv, 2 dk, 3 both.  Both at once keep k, v, dk and dv of a
// wavefront's keys in registers: rows of 256 bytes and more take two launches
// instead, which compute the scores twice and run two wavefronts on a SIMD
// where the one would run one.  Measured (8095 causal rows in two sequences, 16
// heads in 4 groups of 128 bf16 values, a group's heads on four workgroups): 185
// and 245 us for two and three products, 24 for the sum of the heads; in one
// launch 565 us, and with a group on one workgroup 1030.
template <typename T, int DP, bool NARROW> constexpr uint32_t keys_lds(uint32_t group, bool bias) {
    return (NARROW ? 2 : 4) * Tile<T, DP, kBothWays, NARROW>::bytes +
           2 * (kGaps + 2 * Tile<T, DP, kBothWays, NARROW>::rows) * 4 +
           (bias ? kMaxBuckets * 4 * (1 + group) + kCells + kMaxBuckets * 4 : 0);
}

template <typename T, int DP, int POS, int WHAT, bool EXACT, bool NARROW>
__global__ __launch_bounds__(kThreads, DP * sizeof(T) > 256 ? 1 : 2) void backward_keys(Attend a) {
    using G = Tile<T, DP, kBothWays, NARROW>;
    using S = Span<NARROW, G::rows>;
    const S span;
    constexpr bool DK = WHAT & 2, DV = WHAT & 1;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int kExtra = kGaps + 2 * G::rows;
    // [2]: L, D of the tile's rows; bias by gap, or positions
    float *extra = (float *)(lds + S::buffers * 2 * G::bytes);
    float *bias = extra + 2 * kExtra;                         // [group][buckets]
    Buckets buckets = {(int32_t *)(bias + kMaxBuckets * a.group), (uint8_t *)(bias + kMaxBuckets * (1 + a.group)),
                       a.buckets - 1, 0};
    const uint32_t lane = threadIdx.x & 63u, col = lane & 31u;
    const uint32_t id = a.first + blockIdx.x, kvh = id % a.kv_heads, share = id / a.kv_heads % a.split;
    const uint32_t slot = id / (a.kv_heads * a.split);
    // query heads of the group: this workgroup's share
    const int32_t g0 = a.group * share / a.split, g1 = a.group * (share + 1) / a.split;
    Seq sq;
    const uint32_t b = slot_owner(a.k_start, a.k_len, a.k_rows, a.batch, S::owned, slot, sq.tile);
    sequence(a, b, sq);
    if (sq.tile >= ((uint32_t)sq.lk + S::owned - 1) / S::owned) return;
    const int32_t key0 = sq.tile * S::owned, key = key0 + (int32_t)span.own + (int32_t)col, off = sq.lk - sq.lq;
    const bool there = key < sq.lk;
    int32_t kpos = 0;
    if constexpr (POS == 2) kpos = there ? flip(a.k_pos[sq.k0 + key]) : kNoKeyFlipped;
    const bool open = there && (POS != 2 || kpos != kNoKeyFlipped);
    Owned<T, DP> k, v;
    load_owned(k, a.k.p + (int64_t)(sq.k0 + key) * a.k.row + kvh * a.k.head, open, a.dim);
    if constexpr (DK) load_owned(v, a.v.p + (int64_t)(sq.k0 + key) * a.v.row + kvh * a.v.head, open, a.dim);
    sign_owned(k, a.scale);
    // rows from `first` on see a key of the workgroup, from `whole` on all of the wavefront's
    const int32_t first = a.causal ? max(0, key0 - off) / G::rows * G::rows : 0;
    const int32_t tiles = sq.lq > first ? (sq.lq - first + G::rows - 1) / G::rows : 0;
    const int32_t seen = a.causal ? key - off : 0;            // the first row that sees this lane's key
    const int32_t wseen = a.causal ? key0 + (int32_t)span.own - off : 0;
    const int32_t whole = a.causal ? wseen + 31 : 0;
    const bool shut = __any(!open);

    typename G::Regs qreg, oreg;
    tile_clear<G>(qreg);
    tile_clear<G>(oreg);
    float Lreg = 0.0f, Dreg = 0.0f;
    uint32_t preg = 0;
    const auto fetch = [&](int32_t g, int32_t i0) {
        const uint32_t head = kvh * a.group + g;
        const int64_t r = sq.q0 + i0;
        tile_load<G, EXACT>(qreg, a.q.p + r * a.q.row + head * a.q.head, a.q.row, sq.lq - i0, a.dim);
        tile_load<G, EXACT>(oreg, a.dout.p + r * a.dout.row + head * a.dout.head, a.dout.row, sq.lq - i0, a.dim);
        if (threadIdx.x < G::rows) {
            const bool in = i0 + (int32_t)threadIdx.x < sq.lq;
            const size_t stat = (size_t)(r + threadIdx.x) * a.heads + head;
            const float2 x = in ? a.stats[stat] : make_float2(INFINITY, 0.0f);
            Lreg = x.x;
            Dreg = x.y;
            if (POS == 2 && a.q_pos) preg = in ? a.q_pos[r + threadIdx.x] : 0;
        }
    };
    const auto least = [&](int32_t i0) { return i0 + off - key0 - (S::owned - 1); };
    const auto stage = [&](int32_t g, int32_t i0, int buf) {
        uint8_t *qt = lds + buf * 2 * G::bytes;
        float *e = extra + buf * kExtra;
        if constexpr (!EXACT) {
            tile_settle<G>(qreg, a.dim);
            tile_settle<G>(oreg, a.dim);
        }
        tile_store<G>(qt, qreg, sq.lq - i0);
        tile_store<G>(qt + G::bytes, oreg, sq.lq - i0);
        if (threadIdx.x < G::rows) {
            e[threadIdx.x] = -Lreg;
            if (DK) e[G::rows + threadIdx.x] = Dreg;
            if (POS == 2) ((int32_t *)e)[2 * G::rows + threadIdx.x] = flip(preg);
        }
        if constexpr (POS == 1) {
            const int32_t x = (int32_t)threadIdx.x, lo = least(i0);
            uint32_t one;
            if (!one_bucket(buckets.bounds, a.buckets, lo, lo + S::owned + G::rows - 2, one) &&
                x < S::owned + G::rows - 1)
                e[2 * G::rows + x] = bias[g * kMaxBuckets + bucket_of(buckets.bounds, a.buckets, lo + x)];
        }
    };

    f32x16 dk[DK ? DP / 32 : 1], dv[DV ? DP / 32 : 1];
#pragma unroll
    for (int d = 0; d < DP / 32; d++) {
        if constexpr (DK) dk[d] = f32x16{};
        if constexpr (DV) dv[d] = f32x16{};
    }
    // (below 2^31: tiles have 32 rows and more, and lse and stats, 12 bytes a row
    // and head, of 2^36 rows times heads fit no memory)
    const int32_t total = tiles * (g1 - g0);
    if (total > 0) fetch(g0, first);                           // (in flight beside the bias tables' loads)
    if (POS != 0 && a.buckets) {
        for (uint32_t g = 0; g < a.group; g++)
            stage_bias<T>(a, kvh * a.group + g, g ? nullptr : buckets.bounds, bias + g * kMaxBuckets);
        int32_t *cell_ends = (int32_t *)(buckets.cells + kCells);
        __syncthreads();
        if constexpr (POS == 2) {
            fill_cells(buckets, cell_ends);
        }
    }
    if (total > 0) stage(g0, first, 0);
    __syncthreads();
    int buf = 0;
    int32_t g = g0, i0 = first;
    for (int32_t it = 0; it < total; it++, buf ^= S::buffers - 1) {
        int32_t gn = g, in = i0 + G::rows;
        if (in >= sq.lq) {
            in = first;
            gn++;
        }
        const bool more = it + 1 < total;
        if (more) fetch(gn, in);
        if (i0 + (int32_t)span.take + S::rows > wseen && i0 + (int32_t)span.take < sq.lq) {
            const uint8_t *qt = lds + buf * 2 * G::bytes, *ot = qt + G::bytes;
            const float *e = extra + buf * kExtra;
            const bool ragged = i0 + (int32_t)span.take < whole;
            bool far = true;
            float shift = 0.0f;
            if constexpr (POS == 1) {
                uint32_t one;
                far = one_bucket(buckets.bounds, a.buckets, least(i0), least(i0) + S::owned + G::rows - 2, one);
                if (far) shift = bias[g * kMaxBuckets + one];
            }
#pragma unroll
            for (int n = 0; n < S::blocks; n++) {
                const int blk = span.take + n * 32;
                f32x16 s = {}, dp = {};
                product_rows<G>(s, qt, blk, k);
                if constexpr (DK) product_rows<G>(dp, ot, blk, v);
                if (POS == 1) {
                    if (far) {
#pragma unroll
                        for (int r = 0; r < 16; r++) s[r] += shift;
                    } else {
                        const float *x = e + 2 * G::rows + blk + (S::owned - 1) - span.own - col;
#pragma unroll
                        for (int r = 0; r < 16; r++) s[r] += x[block_row(r)];
                    }
                }
                if (POS == 2 && a.buckets) {
                    int32_t gap[16];
                    uint32_t nb[16];
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        gap[r] = gap_of(((const int32_t *)e)[2 * G::rows + blk + block_row(r)], kpos);
                    buckets_in(buckets, gap, nb);
#pragma unroll
                    for (int r = 0; r < 16; r++) s[r] += bias[g * kMaxBuckets + nb[r]];
                }
                if (ragged) {
#pragma unroll
                    for (int r = 0; r < 16; r++)
                        if (i0 + blk + block_row(r) < seen) s[r] = -INFINITY;
                }
                if (shut) {
#pragma unroll
                    for (int r = 0; r < 16; r++) s[r] = open ? s[r] : -INFINITY;
                }
                float p[16], ds[16];
#pragma unroll
                for (int r = 0; r < 16; r++) {
                    const int ir = blk + block_row(r);
                    p[r] = exp2_fast(fmaf(s[r], a.scale2, e[ir]));
                    if constexpr (DK) ds[r] = p[r] * (dp[r] - e[G::rows + ir]);
                }
                Scores<T> w;
                if constexpr (DV) {
                    pack(w, p);
                    product_columns<G>(dv, ot, blk, w);
                }
                if constexpr (DK) {
                    pack(w, ds);
                    product_columns<G>(dk, qt, blk, w);
                }
            }
        }
        if (NARROW && more) __syncthreads();
        if (more) stage(gn, in, NARROW ? 0 : buf ^ 1);
        __syncthreads();
        g = gn;
        i0 = in;
    }
    if constexpr (NARROW) {
        if constexpr (DK) join_waves<DP>(dk, (float *)lds);
        if constexpr (DK && DV) __syncthreads();
        if constexpr (DV) join_waves<DP>(dv, (float *)lds);
        if (threadIdx.x >= 64) return;
    }
    if (!there) return;
    const int64_t at = sq.k0 + key;
    if (a.split > 1) {
        const size_t width = (a.dim + 3) / 4 * 4, all = (size_t)a.k_rows * a.kv_heads * width;
        float *p = a.kpart + share * all + (at * a.kv_heads + kvh) * width;
        if constexpr (DK) store_owned<float, DP>((uint8_t *)p, a.dim, dk, a.scale);
        if constexpr (DV) store_owned<float, DP>((uint8_t *)(p + a.split * all), a.dim, dv, 1.0f);
        return;
    }
    if constexpr (DK)
        store_owned<T, DP>((uint8_t *)a.dk.p + at * a.dk.row + kvh * a.dk.head, a.dim, dk, a.scale);
    if constexpr (DV) store_owned<T, DP>((uint8_t *)a.dv.p + at * a.dv.row + kvh * a.dv.head, a.dim, dv, 1.0f);
}

// The sum of the shares of dk (blockIdx.y 0) and dv: a thread four values.
template <typename T> __global__ __launch_bounds__(kThreads) void sum_heads(Attend a) {
    const uint32_t chunks = (a.dim + 3) / 4;
    const uint32_t lo = first_row(a.k_start, a.k_len, a.k_rows, 0);
    const uint32_t hi = first_row(a.k_start, a.k_len, a.k_rows, a.batch);
    const size_t all = (size_t)a.k_rows * a.kv_heads * chunks;
    const f32x4 *part = (const f32x4 *)a.kpart + blockIdx.y * a.split * all;
    const Strided &out = blockIdx.y ? a.dv : a.dk;
    for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < all; i += (size_t)gridDim.x * kThreads) {
        const size_t row = i / chunks / a.kv_heads;
        if (row < lo || row >= hi) continue;
        f32x4 x = part[i];
        for (uint32_t s = 1; s < a.split; s++) x += part[s * all + i];
        const float f[4] = {x[0], x[1], x[2], x[3]};
        store_values<T, 4>((uint8_t *)out.p + row * out.row + i / chunks % a.kv_heads * out.head, i % chunks * 4,
                           a.dim, f);
    }
}

// ---------------------------------------------------------------- short lists
// The gradients of many short lists with a query row each, of up to GB query
// heads on a key/value head: a group of lanes takes a list, as in attend_lists.
// One pass over a list's keys and values gives, with d_j = dp_j - dp of the
// first open key,
//   D' = sum p_j d_j,  A = sum p_j d_j k_j,  B = sum p_j k_j,  dq = scale (A - D' B)
// and ds_j = p_j (d_j - D'), so dk_j = scale ds_j q and dv_j = p_j do need
// neither k nor v again: p_j and d_j of the list's first `keep` keys wait in
// LDS, a longer list is read again for the others.  Bound by reading k and v
// and writing dk and dv once.  Measured: 12 000 lists of 20 slots, two heads of 50
// fp32 values (0.33 GB): 96 us, 3.4 TB/s.
struct PD {
    float p, d;
};

template <typename T, int DP, int GB>
__global__ __launch_bounds__(kThreads) void backward_lists(Attend a, uint32_t keep) {
    using L = Lanes<T, DP>;
    constexpr int N = Chunk<T>::n, U = 2;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63u, c = lane % L::per_row, c0 = c * N, kr = lane / L::per_row;
    const uint32_t wave = threadIdx.x >> 6, group = wave * L::rows + kr;   // lane group of the workgroup
    int32_t *bounds = (int32_t *)lds;
    float *bias = (float *)(bounds + kMaxBuckets);            // [buckets][heads]
    PD *kept = (PD *)(((uintptr_t)(bias + a.buckets * a.heads) + 7) & ~(uintptr_t)7);   // [groups][keep][GB]
    float *hist = (float *)(kept + 4 * L::rows * keep * GB);  // the bias gradient: [buckets][GB][groups]
    const bool want = a.part;
    uint8_t *codes = (uint8_t *)(hist + (want ? a.buckets * GB * 4 * L::rows : 0)) + wave * L::rows * kListKeys;
    kept += group * keep * GB;
    if (a.buckets) {
        for (uint32_t i = threadIdx.x; i < kMaxBuckets; i += kThreads)
            bounds[i] = i + 1 < a.buckets ? a.bounds[i] : INT32_MAX;
        for (uint32_t i = threadIdx.x; i < a.buckets * a.heads; i += kThreads)
            bias[i] = bias2_of<T>(a, i / a.heads, i % a.heads);
        if (want)
            for (uint32_t i = threadIdx.x; i < a.buckets * GB * 4 * L::rows; i += kThreads) hist[i] = 0.0f;
        __syncthreads();
    }
    // (all groups' turn is a multiple of kv_heads: each group keeps its heads)
    const uint64_t units = (uint64_t)a.batch * a.kv_heads, turn = (uint64_t)gridDim.x * 4 * L::rows;
    for (uint64_t unit0 = (blockIdx.x * 4ull + wave) * L::rows; unit0 < units; unit0 += turn) {
        const bool there = unit0 + kr < units;
        const uint64_t unit = there ? unit0 + kr : 0;
        const uint32_t b = unit / a.kv_heads, kvh = unit % a.kv_heads, head0 = kvh * a.group;
        Seq sq;
        sequence(a, b, sq);
        if (!there) sq.lk = 0;
        // (the first positions are in flight with q and do)
        u32x4 rawq[GB], rawo[GB];
        float q[GB][N], dout[GB][N], A[GB][N], B[GB][N], lse[GB], first[GB], D[GB], weight[GB];
#pragma unroll
        for (int g = 0; g < GB; g++) {
            rawq[g] = rawo[g] = u32x4{0, 0, 0, 0};
            lse[g] = -INFINITY;
            if ((uint32_t)g < a.group) {
                rawq[g] = load_chunk<T>(a.q.p + (int64_t)b * a.q.row + (head0 + g) * a.q.head, c0, a.dim);
                rawo[g] = load_chunk<T>(a.dout.p + (int64_t)b * a.dout.row + (head0 + g) * a.dout.head, c0, a.dim);
                lse[g] = a.lse[(size_t)b * a.heads + head0 + g];
            }
        }
        ListPositions<L::per_row, kListKeys> keys;
        keys.load(a, sq.k0, sq.lk, 0);
#pragma unroll
        for (int g = 0; g < GB; g++) {
            lse[g] = row_log2(lse[g]);
            first[g] = D[g] = weight[g] = 0.0f;
            unpack<T>(rawq[g], q[g]);
            unpack<T>(rawo[g], dout[g]);
#pragma unroll
            for (int i = 0; i < N; i++) A[g][i] = B[g][i] = 0.0f;
        }
        const int32_t qpos = a.buckets ? (a.q_pos ? flip(a.q_pos[b]) : flip((uint32_t)sq.lk - 1)) : 0;
        const uint8_t *kp = a.k.p + (int64_t)sq.k0 * a.k.row + kvh * a.k.head;
        const uint8_t *vp = a.v.p + (int64_t)sq.k0 * a.v.row + kvh * a.v.head;
        uint8_t *dkp = (uint8_t *)a.dk.p + (int64_t)sq.k0 * a.dk.row + kvh * a.dk.head;
        uint8_t *dvp = (uint8_t *)a.dv.p + (int64_t)sq.k0 * a.dv.row + kvh * a.dv.head;
        bool began = false;

        // p and d of U open keys (0 where there is none)
        const auto weigh = [&](int32_t j0, uint64_t &mine, uint32_t (&at)[U], bool (&open)[U], float (&p)[U][GB],
                               float (&d)[U][GB], auto summing) {
            u32x4 k[U], v[U];
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
#pragma unroll
            for (int u = 0; u < U; u++) {
                float x[N], y[N];
                unpack<T>(k[u], x);
                unpack<T>(v[u], y);
                const uint32_t bk = a.buckets ? codes[kr * kListKeys + at[u]] * a.heads + head0 : 0;
#pragma unroll
                for (int g = 0; g < GB; g++) {
                    float s = 0.0f, dp = 0.0f;
#pragma unroll
                    for (int i = 0; i < N; i++) {
                        s = fmaf(q[g][i], x[i], s);
                        dp = fmaf(dout[g][i], y[i], dp);
                    }
                    s = lanes_sum<L::per_row>(s) * a.signed2;
                    dp = lanes_sum<L::per_row>(dp);
                    if (a.buckets && (uint32_t)g < a.group) s += bias[bk + g];
                    p[u][g] = open[u] ? exp2_fast(s - lse[g]) : 0.0f;
                    if (!began && open[u]) first[g] = dp;
                    d[u][g] = open[u] ? dp - first[g] : 0.0f;
                    if constexpr (decltype(summing)::value) {
                        const float pd = p[u][g] * d[u][g];
                        D[g] += pd;
                        weight[g] += p[u][g];
#pragma unroll
                        for (int i = 0; i < N; i++) {
                            A[g][i] = fmaf(pd, x[i], A[g][i]);
                            B[g][i] = fmaf(p[u][g], x[i], B[g][i]);
                        }
                    }
                }
                began |= open[u];
            }
        };
        // dk, dv (and the bias gradient) of key j0 + at
        const auto give = [&](int32_t j0, uint32_t at, bool open, const float (&p)[GB], const float (&d)[GB]) {
            float dk[N] = {}, dv[N] = {}, mine = 0.0f;
#pragma unroll
            for (int g = 0; g < GB; g++) {
                const float w = p[g] * weight[g], ds = w * (d[g] - D[g]), dss = ds * a.scale;
                if (c == (uint32_t)g) mine = ds;
#pragma unroll
                for (int i = 0; i < N; i++) {
                    dk[i] = fmaf(dss, q[g][i], dk[i]);
                    dv[i] = fmaf(w, dout[g][i], dv[i]);
                }
            }
            if (!open) return;
            if (want && c < GB)
                __hip_atomic_fetch_add(hist + (codes[kr * kListKeys + at] * GB + c) * 4 * L::rows + group, mine,
                                       __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            if (c0 < a.dim) {
                store_values<T, N>(dkp + (int64_t)(j0 + at) * a.dk.row, c0, a.dim, dk);
                store_values<T, N>(dvp + (int64_t)(j0 + at) * a.dv.row, c0, a.dim, dv);
            }
        };

        uint64_t opened = 0;                                  // of the list's first 64 keys
        for (int32_t j0 = 0; __any(j0 < sq.lk); j0 += kListKeys) {
            if (j0) keys.load(a, sq.k0, sq.lk, j0);
            wave_lds_fence();
            uint64_t mine = open_keys(a, bounds, codes, keys, sq.lk, j0, qpos);
            wave_lds_fence();
            if (j0 == 0) opened = mine;
            while (__any(mine != 0)) {
                uint32_t at[U];
                bool open[U];
                float p[U][GB], d[U][GB];
                weigh(j0, mine, at, open, p, d, std::true_type{});
#pragma unroll
                for (int u = 0; u < U; u++)
                    if (c < GB && open[u] && j0 == 0 && at[u] < keep) {
                        float x = p[u][0], y = d[u][0];
#pragma unroll
                        for (int g = 1; g < GB; g++)
                            if (c == (uint32_t)g) {
                                x = p[u][g];
                                y = d[u][g];
                            }
                        kept[at[u] * GB + c] = PD{x, y};
                    }
            }
        }
        wave_lds_fence();
        // lse is rounded, and a list's probabilities with it: they add up to one
#pragma unroll
        for (int g = 0; g < GB; g++) {
            weight[g] = weight[g] > 0.5f ? 1.0f / weight[g] : 1.0f;
            D[g] *= weight[g];
        }
        for (int32_t j0 = 0; __any(j0 < sq.lk); j0 += kListKeys) {
            uint64_t mine = opened;
            if (__any(sq.lk > kListKeys)) {                   // (else the codes are still there)
                keys.load(a, sq.k0, sq.lk, j0);
                wave_lds_fence();
                mine = open_keys(a, bounds, codes, keys, sq.lk, j0, qpos);
                wave_lds_fence();
            }
            // rows of closed keys
            for (int32_t j = j0; __any(j < min(sq.lk, j0 + kListKeys)); j++)
                if (j < sq.lk && !((mine >> (j - j0)) & 1) && c0 < a.dim) {
                    const float zero[N] = {};
                    store_values<T, N>(dkp + (int64_t)j * a.dk.row, c0, a.dim, zero);
                    store_values<T, N>(dvp + (int64_t)j * a.dv.row, c0, a.dim, zero);
                }
            uint64_t waits = j0 == 0 ? mine & (keep < 64 ? (1ull << keep) - 1 : ~0ull) : 0;
            mine &= ~waits;
            while (__any(waits != 0)) {
                const bool open = waits != 0;
                const uint32_t at = open ? __builtin_ctzll(waits) : 0;
                waits &= waits - 1;
                float p[GB], d[GB];
#pragma unroll
                for (int g = 0; g < GB; g++) {
                    const PD x = kept[at * GB + g];
                    p[g] = open ? x.p : 0.0f;
                    d[g] = open ? x.d : 0.0f;
                }
                give(j0, at, open, p, d);
            }
            while (__any(mine != 0)) {
                uint32_t at[U];
                bool open[U];
                float p[U][GB], d[U][GB];
                weigh(j0, mine, at, open, p, d, std::false_type{});
#pragma unroll
                for (int u = 0; u < U; u++) give(j0, at[u], open[u], p[u], d[u]);
            }
        }
        if (!there) continue;
#pragma unroll
        for (int g = 0; g < GB; g++) {
            if ((uint32_t)g >= a.group) break;
            float dq[N];
#pragma unroll
            for (int i = 0; i < N; i++) dq[i] = a.scale * weight[g] * (A[g][i] - D[g] * B[g][i]);
            if (c0 < a.dim)
                store_values<T, N>((uint8_t *)a.dq.p + (int64_t)b * a.dq.row + (head0 + g) * a.dq.head, c0, a.dim, dq);
        }
    }
    if (!want) return;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < a.heads * a.buckets; i += kThreads) {
        const uint32_t bk = i % a.buckets, head = i / a.buckets, kvh = head / a.group, g = head % a.group;
        // the lane groups of this workgroup that work on the head
        float x = 0.0f;
        const uint32_t first = (blockIdx.x * 4ull * L::rows) % a.kv_heads;
        for (uint32_t r = (kvh + a.kv_heads - first) % a.kv_heads; r < 4 * L::rows; r += a.kv_heads)
            x += hist[(bk * GB + g) * 4 * L::rows + r];
        a.part[((size_t)blockIdx.x * a.heads + head) * a.buckets + bk] = x;
    }
}

// ---------------------------------------------------------------- bias gradient
// Sums n partial tables [heads][buckets] in a fixed order: block (head, p) the
// p-th of `outs` even shares into out[p], or the gradient itself where out is
// null; every 16th table a wavefront.  64-bit sums: the terms cancel.
template <typename T>
__global__ __launch_bounds__(1024) void sum_bias(const float *part, uint32_t n, uint32_t heads, uint32_t buckets,
                                                 uint32_t outs, float *out, T *dbias) {
    __shared__ double sums[16][64];
    const uint32_t head = blockIdx.x % heads, p = blockIdx.x / heads, lane = threadIdx.x & 63u, w = threadIdx.x >> 6;
    const uint32_t each = (n + outs - 1) / outs, hi = min(n, p * each + each);
    const size_t step = (size_t)heads * buckets;
    double x = 0.0;
    if (lane < buckets) {
        const float *t = part + (size_t)head * buckets + lane;
        uint32_t i = p * each + w;
        for (; i + 112 < hi; i += 128) {                      // eight loads in flight
            float v[8];
#pragma unroll
            for (uint32_t u = 0; u < 8; u++) v[u] = t[(i + 16 * u) * step];
#pragma unroll
            for (uint32_t u = 0; u < 8; u++) x += (double)v[u];
        }
        for (; i < hi; i += 16) x += (double)t[i * step];
    }
    sums[w][lane] = x;
    __syncthreads();
    if (w == 0 && lane < buckets) {
#pragma unroll
        for (int i = 1; i < 16; i++) x += sums[i][lane];
        if (out) out[((size_t)p * heads + head) * buckets + lane] = (float)x;
        else dbias[(size_t)lane * heads + head] = (T)(float)x;
    }
}

// ---------------------------------------------------------------- launches
template <typename T, int DP, bool EXACT, bool NARROW>
int launch_rows(const Attend &a, hipStream_t stream) {
    const int pos = a.k_pos ? 2 : a.buckets ? 1 : 0;
    const auto rows = pos == 2   ? backward_rows<T, DP, 2, EXACT, NARROW>
                      : pos == 1 ? backward_rows<T, DP, 1, EXACT, NARROW>
                                 : backward_rows<T, DP, 0, EXACT, NARROW>;
    const uint32_t bytes = rows_lds<T, DP, NARROW>(a.part ? a.buckets : 0);
    if (!allow_lds(rows, bytes)) return NLB_EDEVICE;
    return enqueue_blocks(rows, a, (uint64_t)a.slots * a.heads, bytes, stream);
}

template <typename T, int DP, int WHAT, bool EXACT, bool NARROW>
int launch_keys(const Attend &a, hipStream_t stream) {
    const int pos = a.k_pos ? 2 : a.buckets ? 1 : 0;
    const auto keys = pos == 2   ? backward_keys<T, DP, 2, WHAT, EXACT, NARROW>
                      : pos == 1 ? backward_keys<T, DP, 1, WHAT, EXACT, NARROW>
                                 : backward_keys<T, DP, 0, WHAT, EXACT, NARROW>;
    const uint32_t bytes = keys_lds<T, DP, NARROW>(a.group, a.buckets > 0);
    if (!allow_lds(keys, bytes)) return NLB_EDEVICE;
    return enqueue_blocks(keys, a, (uint64_t)a.slots * a.kv_heads * a.split, bytes, stream);
}

template <typename T, int DP, bool EXACT, bool NARROW> int launch_both_keys(const Attend &a, hipStream_t stream) {
    if constexpr (DP * sizeof(T) >= 256) {
        const int rc = launch_keys<T, DP, 1, EXACT, NARROW>(a, stream);
        return rc != NLB_OK ? rc : launch_keys<T, DP, 2, EXACT, NARROW>(a, stream);
    } else {
        return launch_keys<T, DP, 3, EXACT, NARROW>(a, stream);
    }
}

template <typename T, int DP> int launch_tiles(Attend a, const Backward &p, hipStream_t stream) {
    const bool exact = exact_rows(a, a.q) && exact_rows(a, a.k) && exact_rows(a, a.v) && exact_rows(a, a.dout);
    int rc = NLB_OK;
    a.slots = (uint32_t)p.q_slots;
    if (a.q_rows) {
        bool narrow = false;
        if constexpr (DP * sizeof(T) <= 256)
            if ((narrow = p.narrow_rows)) rc = launch_rows<T, DP, false, true>(a, stream);
        if (!narrow)
            rc = exact ? launch_rows<T, DP, true, false>(a, stream) : launch_rows<T, DP, false, false>(a, stream);
    }
    a.slots = (uint32_t)p.k_slots;
    if (a.k_rows && rc == NLB_OK) {
        bool narrow = false;
        if constexpr (DP * sizeof(T) <= 256)
            if ((narrow = p.narrow_keys)) rc = launch_both_keys<T, DP, false, true>(a, stream);
        if (!narrow)
            rc = exact ? launch_both_keys<T, DP, true, false>(a, stream)
                       : launch_both_keys<T, DP, false, false>(a, stream);
        if (a.split > 1 && rc == NLB_OK) rc = enqueue(sum_heads<T>, dim3(1024, 2), kThreads, 0, stream, a);
    }
    return rc;
}

template <typename T, int DP> int launch_lists(const Attend &a, const Backward &p, hipStream_t stream) {
    const int gb = a.group > 2 ? 4 : (int)a.group;
    const auto kernel =
        gb == 4 ? backward_lists<T, DP, 4> : gb == 2 ? backward_lists<T, DP, 2> : backward_lists<T, DP, 1>;
    const uint32_t groups = 4 * Lanes<T, DP>::rows;
    const uint32_t bytes = kMaxBuckets * 4 + a.buckets * a.heads * 4 + 8 + groups * p.keep * gb * 8 +
                           (a.part ? a.buckets * gb * groups * 4 : 0) + groups * kListKeys;
    if (!allow_lds(kernel, bytes)) return NLB_EDEVICE;
    return enqueue(kernel, p.blocks, kThreads, bytes, stream, a, p.keep);
}

template <typename T, int DP> int launch_form(const Attend &a, const Backward &p, hipStream_t s) {
    return p.lists ? launch_lists<T, DP>(a, p, s) : launch_tiles<T, DP>(a, p, s);
}

template <typename T> int launch(const Attend &a, const Backward &p, void *dbias, hipStream_t s) {
    int rc = a.dim <= 32   ? launch_form<T, 32>(a, p, s)
             : a.dim <= 64 ? launch_form<T, 64>(a, p, s)
                           : launch_form<T, 128>(a, p, s);
    if (rc != NLB_OK || !dbias) return rc;
    const float *from = a.part;
    uint32_t n = (uint32_t)p.parts;
    if (p.shares) {
        float *mid = a.part + (size_t)n * a.heads * a.buckets;
        rc = enqueue(sum_bias<T>, p.shares * a.heads, 1024, 0, s, from, n, a.heads, a.buckets, p.shares, mid, nullptr);
        if (rc != NLB_OK) return rc;
        from = mid;
        n = p.shares;
    }
    return enqueue(sum_bias<T>, a.heads, 1024, 0, s, from, n, a.heads, a.buckets, 1u, nullptr, (T *)dbias);
}

}  // namespace

extern "C" int nlb_attention_backward(const nlb_att_call *c, const nlb_att_rows *o, const float *lse,
                                      const nlb_att_rows *dout, const nlb_att_rows *dq, const nlb_att_rows *dk,
                                      const nlb_att_rows *dv, void *dbias, void *work, size_t work_bytes,
                                      void *stream) {
    Attend a;
    int rc = fill_call(c, a);
    if (rc != NLB_OK) return rc;
    const bool q = c->q_rows > 0, k = c->k_rows > 0;
    if (fill_rows(c, o, q, a.o) != NLB_OK || fill_rows(c, dout, q, a.dout) != NLB_OK ||
        fill_rows(c, dq, q, a.dq) != NLB_OK || fill_rows(c, dk, k, a.dk) != NLB_OK ||
        fill_rows(c, dv, k, a.dv) != NLB_OK)
        return NLB_EINVAL;
    if ((q && !lse) || (uintptr_t)lse % 4 || (uintptr_t)work % 16) return NLB_EINVAL;
    if ((uintptr_t)dbias % (c->dtype == NLB_DTYPE_BF16 ? 2 : 4) || (dbias && !a.buckets)) return NLB_EINVAL;
    const Backward p = plan_backward(a);
    if (p.q_slots > p.q_most || p.k_slots > p.k_most) return NLB_EINVAL;
    if (work_bytes < p.bytes || (p.bytes && !work)) return NLB_ESCRATCH;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    a.lse = const_cast<float *>(lse);
    a.stats = (float2 *)work;
    a.split = p.split;
    a.kpart = (float *)((uint8_t *)work + p.stat_bytes + p.part_bytes);
    a.part = dbias ? (float *)((uint8_t *)work + p.stat_bytes) : nullptr;
    return c->dtype == NLB_DTYPE_BF16 ? launch<__bf16>(a, p, dbias, (hipStream_t)stream)
                                      : launch<float>(a, p, dbias, (hipStream_t)stream);
}
