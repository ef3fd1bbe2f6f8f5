// norm_rotate.hip -- RMS norm of each head's queries and keys and their rotation
// by position, in one pass, forward and backward.
//   r = (mean x^2 + eps)^-1/2,  u = x r w,  a_i = pos f_i  (i < m)
//   y_i = u_i cos a_i - u_{m+i} sin a_i,  y_{m+i} = u_{m+i} cos a_i + u_i sin a_i
//   du = dy rotated by -a,  g = du w,  dx = r (g - x r^2 mean(g x)),  dw = sum du x r
// All of it is bound by reading the rows once and writing them once.  A head is
// held by a few lanes, each with the values of some pairs (i, m + i), so that a
// rotation needs no other lane; the values behind the 2 m rotated ones are taken
// as pairs that turn by nothing.  A lane makes the sines of its pairs once for a
// row and keeps them over the row's heads.
// Measured: 131 072 rows of 16 + 4 heads of 128 bf16 values 277 us (4.8 TB/s, a
// large copy's rate); 32 768 rows of 8 + 2 heads of 64, half of each turned, 24 us,
// backward 33 (3.5 and 3.8 TB/s) and 5 for the sum of the shares; 12 000 + 240 000
// rows of 2 heads of 50 fp32 values 32 us (of its cycles 0.8 vector instructions:
// sines for two heads), backward 58 and 6.
#include <type_traits>

#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kThreads = 256;

struct Side {                                              // the queries, or the keys
    const uint8_t *x, *dy;
    uint8_t *out;                                          // y or dx
    int64_t x_row, x_head, dy_row, dy_head, out_row, out_head;   // bytes
    const uint32_t *pos;
    const float *w;
    uint32_t rows, heads, blocks, per, parts;              // workgroups; heads a task, tasks a row
};

struct Rotate {
    Side side[2];
    const float *freq;
    uint32_t dim, m, rest;                                 // rest: pairs behind the rotated ones
    float eps;
    float *part;                                           // [workgroups][dim]: shares of dw
};

// sin and cos of `turns` revolutions: reduced to an eighth of one in 64 bits,
// then the series of both to beyond fp32's last bit.
__device__ __forceinline__ void sincos_turns(double turns, float &s, float &c) {
    const double q = __builtin_rint(turns * 4.0);
    const float t = (float)((turns - q * 0.25) * 6.283185307179586477);
    const float v = t * t;
    const float ps = fmaf(v, fmaf(v, fmaf(v, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f);
    const float pc = fmaf(v, fmaf(v, fmaf(v, fmaf(v, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f),
                          -0.5f);
    const float ss = fmaf(t * v, ps, t), cc = fmaf(v, pc, 1.0f);
    const int k = (int)(q - 4.0 * __builtin_floor(q * 0.25));   // quarter turns, 0 to 3
    const float a = k & 1 ? cc : ss, b = k & 1 ? ss : cc;
    s = k & 2 ? -a : a;
    c = (k + 1) & 2 ? -b : b;
}

// A lane's pairs: V of them, side by side where both halves can be read in whole
// chunks (kWhole; kOverlap: where the last chunk of the rotated pairs, or of those
// behind them, is not full, it is moved back over the one before, and the first
// `skip` of its pairs belong to that), else every L-th (kStrided).  Pair p is the
// values lo(p) and hi(p) of a head; the last pair behind the rotated ones may lack
// the second.
constexpr int kWhole = 0, kOverlap = 1, kStrided = 2;
template <typename T, int L, int MODE, bool BACK> struct Pairs {
    static constexpr int V = 16 / sizeof(T);
    uint32_t j, p0, skip;
    bool some;
    __device__ __forceinline__ Pairs(const Rotate &a, uint32_t lane) : j(lane), p0(0), skip(0), some(true) {
        if constexpr (MODE != kStrided) {
            const uint32_t turned = (a.m + V - 1) / V, in = j < turned ? j : j - turned;
            const uint32_t n = j < turned ? a.m : a.rest;
            some = in * V < n;
            p0 = in * V;
            if (some && p0 + V > n) skip = p0 + V - n, p0 = n - V;
            p0 += j < turned ? 0 : a.m;
        }
    }
    __device__ __forceinline__ uint32_t pair(int i) const { return MODE != kStrided ? p0 + i : i * L + j; }
    static __device__ __forceinline__ uint32_t lo(const Rotate &a, uint32_t p) { return p < a.m ? p : a.m + p; }
    static __device__ __forceinline__ uint32_t hi(const Rotate &a, uint32_t p) {
        return p < a.m ? a.m + p : a.m + a.rest + p;
    }
    // whether pair(i) is this lane's to add up
    __device__ __forceinline__ bool own(int i) const { return MODE != kOverlap || i >= (int)skip; }
    __device__ __forceinline__ bool has_lo(const Rotate &a, uint32_t p) const { return some && p < a.m + a.rest; }
    __device__ __forceinline__ bool has_hi(const Rotate &a, uint32_t p) const {
        return some && p < a.m + a.rest && hi(a, p) < a.dim;
    }
    // the values of one half, HI or not
    template <bool HI> __device__ __forceinline__ void load(const Rotate &a, const uint8_t *x, u32x4 &raw) const {
        raw = u32x4{0, 0, 0, 0};
        if constexpr (MODE != kStrided) {
            if (some) raw = *(const u32x4_any *)(x + (HI ? hi(a, p0) : lo(a, p0)) * sizeof(T));
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const uint32_t p = pair(i);
                if (HI ? !has_hi(a, p) : !has_lo(a, p)) continue;
                const uint32_t c = HI ? hi(a, p) : lo(a, p);
                if constexpr (sizeof(T) == 4) raw[i] = ((const uint32_t *)x)[c];
                else raw[i / 2] |= (uint32_t)((const uint16_t *)x)[c] << (16 * (i % 2));
            }
        }
    }
    static __device__ __forceinline__ void unpack(u32x4 raw, float (&f)[V]) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            if constexpr (sizeof(T) == 4) {
                f[i] = __uint_as_float(raw[i]);
            } else {
                f[2 * i] = __uint_as_float(raw[i] << 16);
                f[2 * i + 1] = __uint_as_float(raw[i] & 0xFFFF0000u);
            }
        }
    }
    // Gradients go out past the caches (lists of width 50: 67 us with ordinary stores,
    // 57 so), results, whose half lines the caches join, through them (rows of 64
    // values of which 32 turn: 23 us so, 29 past them).
    // (pairs of two chunks are written twice, the same values: a head's lanes are
    // in one wavefront, and all have read before any writes)
    template <bool HI> __device__ __forceinline__ void store(const Rotate &a, uint8_t *y, const float (&f)[V]) const {
        T v[V];
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = (T)f[i];
        if constexpr (MODE != kStrided) {
            u32x4 u;
            __builtin_memcpy(&u, v, 16);
            u32x4_any *to = (u32x4_any *)(y + (HI ? hi(a, p0) : lo(a, p0)) * sizeof(T));
            if (some && BACK) __builtin_nontemporal_store(u, to);
            else if (some) *to = u;
        } else {
#pragma unroll
            for (int i = 0; i < V; i++) {
                const uint32_t p = pair(i);
                if (HI ? !has_hi(a, p) : !has_lo(a, p)) continue;
                ((T *)y)[HI ? hi(a, p) : lo(a, p)] = v[i];
            }
        }
    }
    // of an fp32 vector of dim values; `other` without one or past its end
    template <bool HI>
    __device__ __forceinline__ void weights(const Rotate &a, const float *w, float other, float (&f)[V]) const {
#pragma unroll
        for (int i = 0; i < V; i++) {
            const uint32_t p = pair(i);
            f[i] = w && (HI ? has_hi(a, p) : has_lo(a, p)) ? w[HI ? hi(a, p) : lo(a, p)] : other;
        }
    }
};

template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
// The sum over the L lanes of a head, in each of them.
template <int L> __device__ __forceinline__ float head_sum(float x) {
    if constexpr (L > 1) x = dpp_add<0xB1>(x);
    if constexpr (L > 2) x = dpp_add<0x4E>(x);
    if constexpr (L > 4) x = dpp_add<0x141>(x);
    if constexpr (L > 8) x = dpp_add<0x140>(x);
    return x;
}

// A task is a row's `per` heads (the last task's may be fewer); L lanes take
// one, the workgroup's groups of lanes tasks side by side.
template <typename T, int L, int MODE, bool BACK>
__global__ __launch_bounds__(kThreads) void rotate_heads(Rotate a) {
    typedef Pairs<T, L, MODE, BACK> P;
    constexpr int V = P::V, U = BACK ? 2 : 4;              // heads whose loads are in flight at once
    const uint32_t is_k = blockIdx.x >= a.side[0].blocks;
    const Side &s = a.side[is_k];
    const uint32_t block = blockIdx.x - (is_k ? a.side[0].blocks : 0);
    const P pairs(a, threadIdx.x % L);
    const float inv = 1.0f / a.dim;
    float wlo[V], whi[V];
    pairs.template weights<false>(a, s.w, 1.0f, wlo);
    pairs.template weights<true>(a, s.w, 1.0f, whi);
    double f[V];                                           // revolutions a step of pos
#pragma unroll
    for (int i = 0; i < V; i++) {
        const uint32_t p = pairs.pair(i);
        f[i] = p < a.m ? (double)a.freq[p] * 0.15915494309189533577 : 0.0;
    }
    float dwlo[V], dwhi[V];
#pragma unroll
    for (int i = 0; i < V; i++) dwlo[i] = dwhi[i] = 0.0f;
    const uint64_t tasks = (uint64_t)s.rows * s.parts, step = (uint64_t)s.blocks * (kThreads / L);
    for (uint64_t t = (uint64_t)block * (kThreads / L) + threadIdx.x / L; t < tasks; t += step) {
        const uint32_t row = s.parts == 1 ? (uint32_t)t : (uint32_t)(t / s.parts);
        const uint32_t h0 = s.parts == 1 ? 0 : (uint32_t)(t - (uint64_t)row * s.parts) * s.per;
        const uint32_t h1 = min(h0 + s.per, s.heads);
        const uint32_t pos = s.pos ? s.pos[row] : 0;
        const uint8_t *x = s.x + (int64_t)row * s.x_row, *dy = BACK ? s.dy + (int64_t)row * s.dy_row : nullptr;
        uint8_t *out = s.out + (int64_t)row * s.out_row;
        if (pos == 0xFFFFFFFFu) {
            float none[V] = {};
            for (uint32_t h = h0; h < h1; h++) {
                pairs.template store<false>(a, out + (int64_t)h * s.out_head, none);
                pairs.template store<true>(a, out + (int64_t)h * s.out_head, none);
            }
            continue;
        }
        float sn[V], cs[V];
#pragma unroll
        for (int i = 0; i < V; i++) {
            sn[i] = 0.0f, cs[i] = 1.0f;
            if (a.m) sincos_turns((double)pos * f[i], sn[i], cs[i]);
        }
        for (uint32_t h = h0; h < h1; h += U) {
            u32x4 xl[U], xh[U], gl[U], gh[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (h + u >= h1) continue;
                pairs.template load<false>(a, x + (int64_t)(h + u) * s.x_head, xl[u]);
                pairs.template load<true>(a, x + (int64_t)(h + u) * s.x_head, xh[u]);
                if constexpr (BACK) {
                    pairs.template load<false>(a, dy + (int64_t)(h + u) * s.dy_head, gl[u]);
                    pairs.template load<true>(a, dy + (int64_t)(h + u) * s.dy_head, gh[u]);
                }
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (h + u >= h1) continue;
                float lo[V], hi[V], sq = 0.0f;
                P::unpack(xl[u], lo);
                P::unpack(xh[u], hi);
#pragma unroll
                for (int i = 0; i < V; i++) sq += pairs.own(i) ? fmaf(hi[i], hi[i], lo[i] * lo[i]) : 0.0f;
                float ol[V], oh[V];
                const float r = __builtin_amdgcn_rsqf(fmaf(head_sum<L>(sq), inv, a.eps));
                if constexpr (!BACK) {
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float ul = lo[i] * r * wlo[i], uh = hi[i] * r * whi[i];
                        ol[i] = fmaf(ul, cs[i], -(uh * sn[i]));
                        oh[i] = fmaf(uh, cs[i], ul * sn[i]);
                    }
                } else {
                    float yl[V], yh[V], sg = 0.0f;
                    P::unpack(gl[u], yl);
                    P::unpack(gh[u], yh);
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        const float dl = fmaf(yl[i], cs[i], yh[i] * sn[i]), dh = fmaf(yh[i], cs[i], -(yl[i] * sn[i]));
                        dwlo[i] = fmaf(dl, lo[i] * r, dwlo[i]);
                        dwhi[i] = fmaf(dh, hi[i] * r, dwhi[i]);
                        ol[i] = dl * wlo[i], oh[i] = dh * whi[i];
                        sg += pairs.own(i) ? fmaf(oh[i], hi[i], ol[i] * lo[i]) : 0.0f;
                    }
                    const float mean = head_sum<L>(sg) * inv * r * r;
#pragma unroll
                    for (int i = 0; i < V; i++) {
                        ol[i] = r * fmaf(-lo[i], mean, ol[i]);
                        oh[i] = r * fmaf(-hi[i], mean, oh[i]);
                    }
                }
                pairs.template store<false>(a, out + (int64_t)(h + u) * s.out_head, ol);
                pairs.template store<true>(a, out + (int64_t)(h + u) * s.out_head, oh);
            }
        }
    }
    if (!BACK || !a.part) return;
    // the groups' sums, in order
    constexpr int G = kThreads / L;
    __shared__ float sums[2][G][L * V + 1];
#pragma unroll
    for (int i = 0; i < V; i++) {
        sums[0][threadIdx.x / L][i * L + threadIdx.x % L] = dwlo[i];
        sums[1][threadIdx.x / L][i * L + threadIdx.x % L] = dwhi[i];
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < 2 * L * V; k += kThreads) {
        const uint32_t half = k / (L * V), at = k % (L * V);
        const P other(a, at % L);
        const uint32_t p = other.pair(at / L);
        if (!other.own(at / L) || (half ? !other.has_hi(a, p) : !other.has_lo(a, p))) continue;
        float x = 0.0f;
#pragma unroll 8
        for (int g = 0; g < G; g++) x += sums[half][g][at];
        a.part[(size_t)blockIdx.x * a.dim + (half ? P::hi(a, p) : P::lo(a, p))] = x;
    }
}

// dwq and dwk from the workgroups' shares (the queries' first), in 64 bits and a
// fixed order: 16 columns a workgroup, every 64th share a thread.
__global__ __launch_bounds__(1024) void sum_shares(const float *part, uint32_t q_blocks, uint32_t k_blocks, uint32_t dim,
                                                   float *dwq, float *dwk) {
    __shared__ double sums[64][17];
    const uint32_t at = threadIdx.x / 16, c = blockIdx.x * 16 + threadIdx.x % 16;
    const uint32_t first = blockIdx.y ? q_blocks : 0, n = blockIdx.y ? k_blocks : q_blocks;
    double x = 0.0;
    for (uint32_t i = at; i < n && c < dim; i += 512) {     // eight loads in flight
        float v[8];
#pragma unroll
        for (uint32_t u = 0; u < 8; u++) v[u] = i + 64 * u < n ? part[(size_t)(first + i + 64 * u) * dim + c] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; u++) x += (double)v[u];
    }
    const uint32_t col = threadIdx.x % 16;
    sums[at][col] = x;
    for (uint32_t o = 32; o; o /= 2) {
        __syncthreads();
        if (at < o) sums[at][col] += sums[at + o][col];
    }
    float *dw = blockIdx.y ? dwk : dwq;
    if (at || c >= dim || !dw) return;
    dw[c] = (float)sums[0][col];
}

// ---------------------------------------------------------------- host
// A head's sum stays within 16 lanes.
constexpr uint32_t kMaxLanes = 16;

// Lanes that hold a head of which each part's pairs are in chunks of their own.
template <typename T> uint32_t chunked_lanes(const Rotate &a) {
    const uint32_t v = 16 / sizeof(T);
    return (a.m + v - 1) / v + (a.rest + v - 1) / v;
}
template <typename T> int mode_of(const Rotate &a) {
    const uint32_t v = 16 / sizeof(T), rest = a.dim - 2 * a.m;
    if (a.m % v == 0 && rest % (2 * v) == 0) return kWhole;
    // half a chunk's lanes idle at most, pairs of both halves, and lanes enough
    // (fp32 heads of 62 to 64 pairs in two parts can need 17 chunks; pair by pair
    // they take 16 lanes: 32 768 rows of 16 + 4 heads of 128, 143 us with 32 pairs
    // turned, in whole chunks, 163 with 31; backward 155 and 203)
    return rest % 2 == 0 && (a.m == 0 || a.m >= v) && (rest == 0 || rest >= 2 * v) && chunked_lanes<T>(a) <= kMaxLanes
               ? kOverlap
               : kStrided;
}
template <typename T> uint32_t lanes_of(const Rotate &a) {
    const uint32_t v = 16 / sizeof(T);
    const uint32_t need = mode_of<T>(a) == kStrided ? (a.m + a.rest + v - 1) / v : chunked_lanes<T>(a);
    uint32_t l = 2;
    while (l < need) l *= 2;
    return l;
}

// Tasks of a side and its workgroups: a row's heads in one task where there are
// rows enough to fill the card, else spread over more lanes.
void split(Side &s, uint32_t lanes, uint32_t most) {
    s.per = s.heads;
    while (s.per > 1 && (uint64_t)s.rows * ((s.heads + s.per - 1) / s.per) * lanes < 262144) s.per = (s.per + 1) / 2;
    s.parts = s.per ? (s.heads + s.per - 1) / s.per : 0;
    const uint64_t need = ((uint64_t)s.rows * s.parts * lanes + kThreads - 1) / kThreads;
    s.blocks = need < most ? (uint32_t)need : most;
}

// Workgroups in all, of which queries and keys have shares by their values:
// eight on each of 256 CUs forward; backward, where each leaves a share of dw, as
// many as the CUs hold at once (registers: three for bf16 rows, four for fp32).
template <typename T> void split(Rotate &a, bool back) {
    const uint32_t lanes = lanes_of<T>(a), most = !back ? 2048 : sizeof(T) == 2 ? 768 : 1024;
    const uint64_t q = (uint64_t)a.side[0].rows * a.side[0].heads, k = (uint64_t)a.side[1].rows * a.side[1].heads;
    uint32_t for_q = q + k ? (uint32_t)((double)most * q / (q + k)) : 0;
    for_q = for_q < 64 ? 64 : for_q > most - 64 ? most - 64 : for_q;
    split(a.side[0], lanes, for_q);
    split(a.side[1], lanes, most - for_q);
}

bool bad_rows(const nlb_att_rows &r, uint32_t rows, int64_t e) {
    return (rows && !r.data) || (uintptr_t)r.data % e || r.row_stride < 0 || r.row_stride > INT32_MAX ||
           r.head_stride < 0 || r.head_stride > INT32_MAX;
}

int fill(const nlb_rotate_call *c, Rotate &a, bool back) {
    a = {};
    if (!c || (c->dtype != NLB_DTYPE_F32 && c->dtype != NLB_DTYPE_BF16)) return NLB_EINVAL;
    if (c->dim < 1 || c->dim > NLB_ATT_MAX_DIM || c->freqs < 0 || 2 * c->freqs > c->dim) return NLB_EINVAL;
    if (c->heads < 1 || c->heads > NLB_ATT_MAX_HEADS || c->kv_heads < 0 || c->kv_heads > NLB_ATT_MAX_HEADS)
        return NLB_EINVAL;
    if (c->q_rows > INT32_MAX || c->k_rows > INT32_MAX || (c->k_rows && !c->kv_heads)) return NLB_EINVAL;
    if (!(c->eps >= 0.0f) || std::isinf(c->eps)) return NLB_EINVAL;
    if (c->freqs && (!c->freq || (c->q_rows && !c->q_pos) || (c->k_rows && !c->k_pos))) return NLB_EINVAL;
    if (((uintptr_t)c->freq | (uintptr_t)c->q_pos | (uintptr_t)c->k_pos | (uintptr_t)c->wq | (uintptr_t)c->wk) % 4)
        return NLB_EINVAL;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (bad_rows(c->q, c->q_rows, e) || bad_rows(c->k, c->k_rows, e)) return NLB_EINVAL;
    a.freq = c->freq;
    a.dim = (uint32_t)c->dim;
    a.m = (uint32_t)c->freqs;
    a.rest = (a.dim - 2 * a.m + 1) / 2;
    a.eps = c->eps;
    for (int i = 0; i < 2; i++) {
        Side &s = a.side[i];
        const nlb_att_rows &r = i ? c->k : c->q;
        s.x = (const uint8_t *)r.data;
        s.x_row = r.row_stride * e;
        s.x_head = r.head_stride * e;
        s.pos = i ? c->k_pos : c->q_pos;
        s.w = i ? c->wk : c->wq;
        s.rows = i ? c->k_rows : c->q_rows;
        s.heads = (uint32_t)(i ? c->kv_heads : c->heads);
    }
    if (c->dtype == NLB_DTYPE_BF16) split<__bf16>(a, back);
    else split<float>(a, back);
    return NLB_OK;
}

size_t work_of(const Rotate &a) { return (size_t)(a.side[0].blocks + a.side[1].blocks) * a.dim * 4; }

template <typename T, bool BACK, int MODE> int launch(const Rotate &a, hipStream_t s) {
    const uint32_t blocks = a.side[0].blocks + a.side[1].blocks;
    switch (lanes_of<T>(a)) {
        case 2: return enqueue(rotate_heads<T, 2, MODE, BACK>, blocks, kThreads, 0, s, a);
        case 4: return enqueue(rotate_heads<T, 4, MODE, BACK>, blocks, kThreads, 0, s, a);
        case 8: return enqueue(rotate_heads<T, 8, MODE, BACK>, blocks, kThreads, 0, s, a);
        case 16: return enqueue(rotate_heads<T, 16, MODE, BACK>, blocks, kThreads, 0, s, a);
    }
    return NLB_EINVAL;
}
template <typename T, bool BACK> int launch(const Rotate &a, hipStream_t s) {
    switch (mode_of<T>(a)) {
        case kWhole: return launch<T, BACK, kWhole>(a, s);
        case kOverlap: return launch<T, BACK, kOverlap>(a, s);
    }
    return launch<T, BACK, kStrided>(a, s);
}
template <bool BACK> int launch(const Rotate &a, int32_t dtype, hipStream_t s) {
    if (!(a.side[0].blocks + a.side[1].blocks)) return NLB_OK;
    return dtype == NLB_DTYPE_BF16 ? launch<__bf16, BACK>(a, s) : launch<float, BACK>(a, s);
}

}  // namespace

extern "C" int nlb_norm_rotate(const nlb_rotate_call *c, const nlb_att_rows *q_out, const nlb_att_rows *k_out,
                               void *stream) {
    Rotate a;
    const int rc = fill(c, a, false);
    if (rc != NLB_OK) return rc;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (!q_out || bad_rows(*q_out, c->q_rows, e)) return NLB_EINVAL;
    if (c->k_rows && (!k_out || bad_rows(*k_out, c->k_rows, e))) return NLB_EINVAL;
    for (int i = 0; i < 2; i++) {
        const nlb_att_rows *r = i ? k_out : q_out;
        if (!a.side[i].rows) continue;
        a.side[i].out = (uint8_t *)r->data;
        a.side[i].out_row = r->row_stride * e;
        a.side[i].out_head = r->head_stride * e;
    }
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    return launch<false>(a, c->dtype, (hipStream_t)stream);
}

extern "C" int nlb_norm_rotate_work(const nlb_rotate_call *c, size_t *bytes) {
    Rotate a;
    if (!bytes) return NLB_EINVAL;
    const int rc = fill(c, a, true);
    if (rc != NLB_OK) return rc;
    *bytes = work_of(a);
    return NLB_OK;
}

extern "C" int nlb_norm_rotate_backward(const nlb_rotate_call *c, const nlb_att_rows *dq_out, const nlb_att_rows *dk_out,
                                        const nlb_att_rows *dq, const nlb_att_rows *dk, float *dwq, float *dwk,
                                        void *work, size_t work_bytes, void *stream) {
    Rotate a;
    int rc = fill(c, a, true);
    if (rc != NLB_OK) return rc;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (!dq_out || !dq || bad_rows(*dq_out, c->q_rows, e) || bad_rows(*dq, c->q_rows, e)) return NLB_EINVAL;
    if (c->k_rows && (!dk_out || !dk || bad_rows(*dk_out, c->k_rows, e) || bad_rows(*dk, c->k_rows, e)))
        return NLB_EINVAL;
    if (((uintptr_t)dwq | (uintptr_t)dwk) % 4 || (uintptr_t)work % 16) return NLB_EINVAL;
    if ((dwq || dwk) && work_of(a) && (!work || work_bytes < work_of(a))) return NLB_ESCRATCH;
    for (int i = 0; i < 2; i++) {
        const nlb_att_rows *r = i ? dk_out : dq_out, *d = i ? dk : dq;
        if (!a.side[i].rows) continue;
        a.side[i].dy = (const uint8_t *)r->data;
        a.side[i].dy_row = r->row_stride * e;
        a.side[i].dy_head = r->head_stride * e;
        a.side[i].out = (uint8_t *)d->data;
        a.side[i].out_row = d->row_stride * e;
        a.side[i].out_head = d->head_stride * e;
    }
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    a.part = dwq || dwk ? (float *)work : nullptr;
    rc = launch<true>(a, c->dtype, (hipStream_t)stream);
    if (rc != NLB_OK || !(dwq || dwk)) return rc;
    return enqueue(sum_shares, dim3((a.dim + 15) / 16, 2), 1024, 0, (hipStream_t)stream, (const float *)work,
                   a.side[0].blocks, a.side[1].blocks, a.dim, dwq, dwk);
}
