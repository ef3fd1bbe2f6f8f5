// layer_norm.hip -- layer norm of rows, forward and backward.
//   mean = sum x / d,  var = sum (x - mean)^2 / d,  rstd = (var + eps)^-1/2
//   xh = (x - mean) rstd,  y = xh w + b
//   g = dy w,  dx = rstd (g - mean(g) - xh mean(g xh))
//   dw = sum over rows of dy xh,  db = sum over rows of dy
// Both passes are bound by reading their rows and writing one of the same size.
// Measured (131 072 rows of 1024 bf16 values): 100 us forward (5.4 TB/s, a plain
// copy's rate), 167 us backward (4.8) and 6 us for the sum of the shares; 16 384
// rows of 8192 fp32 values 198 and 309 us (5.4 and 5.2 TB/s).
#include "call_device.h"
#include "nlb_internal.h"

namespace {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

struct Norm {
    const uint8_t *x, *dy;
    uint8_t *out;                        // y or dx
    int64_t x_row, dy_row, out_row;      // bytes
    const float *w, *b;
    float *mean, *rstd;
    uint32_t rows, width;
    float eps;
    float *part;                         // [workgroups][2][width]: shares of dw and db
};

template <typename T> struct Chunk { static constexpr int n = 16 / sizeof(T); };

// 16 bytes of values from c0 on of a row of `width`, zeros past its end.
template <typename T>
__device__ __forceinline__ u32x4 load_chunk(const uint8_t *row, uint32_t c0, uint32_t width) {
    constexpr uint32_t n = Chunk<T>::n;
    const uint8_t *p = row + c0 * sizeof(T);
    u32x4 x = {0, 0, 0, 0};
    if (c0 + n <= width) {
        x = *(const u32x4_any *)p;
    } else if (c0 < width) {
#pragma unroll
        for (uint32_t i = 0; i < n - 1; i++)
            if (c0 + i < width) {
                if constexpr (sizeof(T) == 4) x[i] = ((const uint32_t *)p)[i];
                else x[i / 2] |= (uint32_t)((const uint16_t *)p)[i] << (16 * (i % 2));
            }
    }
    return x;
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

// Values c0 .. c0 + n - 1 of a vector of `width`, `other` without one or past its end.
template <int n>
__device__ __forceinline__ void load_weights(const float *p, uint32_t c0, uint32_t width, float other, float (&f)[n]) {
#pragma unroll
    for (int i = 0; i < n; i++) f[i] = p && c0 + i < width ? p[c0 + i] : other;
}

template <typename T, int n>
__device__ __forceinline__ void store_row(uint8_t *row, uint32_t c0, uint32_t width, const float (&f)[n]) {
    T v[n];
#pragma unroll
    for (int i = 0; i < n; i++) v[i] = (T)f[i];
    T *p = (T *)row + c0;
    if (c0 + n <= width) {
#pragma unroll
        for (int i = 0; i < n; i += 16 / sizeof(T)) {
            u32x4 u;
            __builtin_memcpy(&u, v + i, 16);
            *(u32x4_any *)(p + i) = u;
        }
    } else {
#pragma unroll
        for (int i = 0; i < n - 1; i++)
            if (c0 + i < width) p[i] = v[i];
    }
}

// The sum of x over the N threads that share a row (a power of two, up to the
// 256 of the workgroup), in each of them: within a wavefront by lane
// permutations of the vector units, over wavefronts through LDS.
template <int CTRL> __device__ __forceinline__ float dpp_add(float x) {
    return x + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
template <int N> __device__ __forceinline__ float row_sum(float x, float (&lds)[4]) {
    x = dpp_add<0xB1>(x);
    x = dpp_add<0x4E>(x);
    if constexpr (N > 4) x = dpp_add<0x141>(x);
    if constexpr (N > 8) x = dpp_add<0x140>(x);
    if constexpr (N > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (N > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if constexpr (N > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = x;
        __syncthreads();
        x = lds[0];
#pragma unroll
        for (int i = 1; i < N / 64; i++) x += lds[i];
    }
    return x;
}

// A row is held in registers by N threads, C chunks of 16 bytes each (chunk
// i of a thread: values (i N + thread) n on), the next row's loads in flight
// while this one is summed; weights stay in registers over the rows of a
// workgroup.
template <typename T, int N, int C>
__global__ __launch_bounds__(256) void norm_rows(Norm a) {
    constexpr int n = Chunk<T>::n, per = 256 / N;
    __shared__ float lds[4];
    const uint32_t t = threadIdx.x % N, step = gridDim.x * per;
    const float inv = 1.0f / a.width;
    float w[C][n], b[C][n];
#pragma unroll
    for (int i = 0; i < C; i++) {
        load_weights<n>(a.w, (i * N + t) * n, a.width, 1.0f, w[i]);
        load_weights<n>(a.b, (i * N + t) * n, a.width, 0.0f, b[i]);
    }
    u32x4 raw[C];
    const auto fetch = [&](uint32_t r) {
#pragma unroll
        for (int i = 0; i < C; i++)
            raw[i] = load_chunk<T>(a.x + (int64_t)r * a.x_row, (i * N + t) * n, r < a.rows ? a.width : 0);
    };
    uint32_t r = blockIdx.x * per + threadIdx.x / N;
    fetch(r);
    // (as many turns for every thread of the workgroup: the first row decides)
    for (uint32_t r0 = blockIdx.x * per; r0 < a.rows; r0 += step, r += step) {
        float x[C][n], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < C; i++) {
            unpack<T>(raw[i], x[i]);
#pragma unroll
            for (int e = 0; e < n; e++) sum += x[i][e];
        }
        if (r0 + step < a.rows) fetch(r + step);
        const float mean = row_sum<N>(sum, lds) * inv;
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < C; i++)
#pragma unroll
            for (int e = 0; e < n; e++) {
                x[i][e] = (i * N + t) * n + e < a.width ? x[i][e] - mean : 0.0f;
                sq = fmaf(x[i][e], x[i][e], sq);
            }
        const float rstd = 1.0f / sqrtf(row_sum<N>(sq, lds) * inv + a.eps);
        if (r >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < C; i++) {
            const uint32_t c = (i * N + t) * n;
            if (c >= a.width) break;
#pragma unroll
            for (int e = 0; e < n; e++) x[i][e] = fmaf(x[i][e] * rstd, w[i][e], b[i][e]);
            store_row<T, n>(a.out + (int64_t)r * a.out_row, c, a.width, x[i]);
        }
        if (t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

// As norm_rows; a thread keeps its values' sums of dy xh and dy over the rows
// of its workgroup, which leaves them in part[workgroup].
template <typename T, int N, int C>
__global__ __launch_bounds__(256) void norm_rows_backward(Norm a) {
    constexpr int n = Chunk<T>::n, per = 256 / N;
    __shared__ float lds[4];
    const uint32_t t = threadIdx.x % N, step = gridDim.x * per;
    const float inv = 1.0f / a.width;
    float w[C][n], dw[C][n], db[C][n];
#pragma unroll
    for (int i = 0; i < C; i++) {
        load_weights<n>(a.w, (i * N + t) * n, a.width, 1.0f, w[i]);
#pragma unroll
        for (int e = 0; e < n; e++) dw[i][e] = db[i][e] = 0.0f;
    }
    u32x4 rawx[C], rawg[C];
    float mean = 0.0f, rstd = 0.0f;
    const auto fetch = [&](uint32_t r) {
        const uint32_t width = r < a.rows ? a.width : 0;
#pragma unroll
        for (int i = 0; i < C; i++) {
            rawx[i] = load_chunk<T>(a.x + (int64_t)r * a.x_row, (i * N + t) * n, width);
            rawg[i] = load_chunk<T>(a.dy + (int64_t)r * a.dy_row, (i * N + t) * n, width);
        }
        mean = width ? a.mean[r] : 0.0f;
        rstd = width ? a.rstd[r] : 0.0f;
    };
    uint32_t r = blockIdx.x * per + threadIdx.x / N;
    fetch(r);
    for (uint32_t r0 = blockIdx.x * per; r0 < a.rows; r0 += step, r += step) {
        float xh[C][n], g[C][n], s1 = 0.0f, s2 = 0.0f;
        const float sd = rstd;
#pragma unroll
        for (int i = 0; i < C; i++) {
            unpack<T>(rawx[i], xh[i]);
            unpack<T>(rawg[i], g[i]);
#pragma unroll
            for (int e = 0; e < n; e++) {
                xh[i][e] = (i * N + t) * n + e < a.width ? (xh[i][e] - mean) * sd : 0.0f;
                dw[i][e] = fmaf(g[i][e], xh[i][e], dw[i][e]);
                db[i][e] += g[i][e];
                g[i][e] *= w[i][e];
                s1 += g[i][e];
                s2 = fmaf(g[i][e], xh[i][e], s2);
            }
        }
        if (r0 + step < a.rows) fetch(r + step);
        s1 = row_sum<N>(s1, lds) * inv;
        s2 = row_sum<N>(s2, lds) * inv;
        if (r >= a.rows) continue;
#pragma unroll
        for (int i = 0; i < C; i++) {
            const uint32_t c = (i * N + t) * n;
            if (c >= a.width) break;
#pragma unroll
            for (int e = 0; e < n; e++) g[i][e] = sd * (g[i][e] - s1 - xh[i][e] * s2);
            store_row<T, n>(a.out + (int64_t)r * a.out_row, c, a.width, g[i]);
        }
    }
    if (!a.part) return;
    float *part = a.part + (size_t)blockIdx.x * 2 * a.width;
    if constexpr (per == 1) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            store_row<float, n>((uint8_t *)part, (i * N + t) * n, a.width, dw[i]);
            store_row<float, n>((uint8_t *)(part + a.width), (i * N + t) * n, a.width, db[i]);
        }
    } else {
        // the workgroup's rows side by side, one group of N threads after the other
        __shared__ float sums[2][N * C * n];
        for (int p = 0; p < per; p++) {
            if ((int)threadIdx.x / N == p)
#pragma unroll
                for (int i = 0; i < C; i++)
#pragma unroll
                    for (int e = 0; e < n; e++) {
                        const uint32_t c = (i * N + t) * n + e;
                        sums[0][c] = p ? sums[0][c] + dw[i][e] : dw[i][e];
                        sums[1][c] = p ? sums[1][c] + db[i][e] : db[i][e];
                    }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < a.width; c += 256) {
            part[c] = sums[0][c];
            part[a.width + c] = sums[1][c];
        }
    }
}

// dw and db from the workgroups' shares: 64 columns a workgroup, every 16th
// share a wavefront, in 64 bits and a fixed order.
__global__ __launch_bounds__(1024) void sum_shares(const float *part, uint32_t shares, uint32_t width, float *dw,
                                                   float *db) {
    __shared__ double sums[16][64];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane;
    double x = 0.0;
    if (c < 2 * width) {
        const size_t step = 2 * (size_t)width;
        uint32_t i = wave;
        for (; i + 112 < shares; i += 128) {                  // eight loads in flight
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; u++) v[u] = part[(i + 16 * u) * step + c];
#pragma unroll
            for (int u = 0; u < 8; u++) x += (double)v[u];
        }
        for (; i < shares; i += 16) x += (double)part[i * step + c];
    }
    sums[wave][lane] = x;
    __syncthreads();
    if (wave || c >= 2 * width) return;
#pragma unroll
    for (int i = 1; i < 16; i++) x += sums[i][lane];
    if (c < width) {
        if (dw) dw[c] = (float)x;
    } else if (db) {
        db[c - width] = (float)x;
    }
}

// Threads and chunks that hold a row: up to 256 threads of 4 chunks of 8 bf16
// values or 8 of 4 fp32 ones.
template <typename T, typename F> int with_shape(uint32_t width, F f) {
    const uint32_t chunks = (width + Chunk<T>::n - 1) / Chunk<T>::n;
#define SHAPE(N, C) \
    if (chunks <= N * C) return f(std::integral_constant<int, N>{}, std::integral_constant<int, C>{})
    SHAPE(4, 1);
    SHAPE(16, 1);
    SHAPE(32, 1);
    SHAPE(64, 1);
    SHAPE(64, 2);
    SHAPE(256, 1);
    SHAPE(256, 2);
    SHAPE(256, 4);
    if constexpr (Chunk<T>::n == 4) SHAPE(256, 8);
#undef SHAPE
    return NLB_EINVAL;
}

// Workgroups of the backward pass: each leaves a share of dw and db, so no
// more than the card holds at once (four of 256 threads on each of 256 CUs),
// and no fewer rows than 32 each.
inline uint32_t backward_blocks(uint32_t rows, uint32_t per) {
    const uint32_t need = (rows + 32 * per - 1) / (32 * per);
    return need < 1024 ? (need ? need : 1) : 1024;
}

template <typename T> int norm_per(uint32_t width) {
    return with_shape<T>(width, [](auto n, auto) { return 256 / (int)decltype(n)::value; });
}

int fill(const nlb_norm_call *c, Norm &a) {
    a = {};
    if (!c || (c->dtype != NLB_DTYPE_F32 && c->dtype != NLB_DTYPE_BF16)) return NLB_EINVAL;
    if (c->width < 1 || c->width > NLB_NORM_MAX_WIDTH || c->rows > INT32_MAX) return NLB_EINVAL;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    if (c->rows && !c->x) return NLB_EINVAL;
    if ((uintptr_t)c->x % e || ((uintptr_t)c->w | (uintptr_t)c->mean | (uintptr_t)c->rstd) % 4) return NLB_EINVAL;
    if (c->x_stride < 0 || c->x_stride > INT32_MAX) return NLB_EINVAL;
    a.x = (const uint8_t *)c->x;
    a.x_row = c->x_stride * e;
    a.w = c->w;
    a.mean = c->mean;
    a.rstd = c->rstd;
    a.rows = c->rows;
    a.width = (uint32_t)c->width;
    return NLB_OK;
}

bool bad_rows(const void *p, int64_t stride, uint32_t rows, int32_t dtype) {
    return (rows && !p) || (uintptr_t)p % (dtype == NLB_DTYPE_BF16 ? 2 : 4) || stride < 0 || stride > INT32_MAX;
}

size_t work_of(const nlb_norm_call *c) {
    const int per = c->dtype == NLB_DTYPE_BF16 ? norm_per<__bf16>(c->width) : norm_per<float>(c->width);
    return (size_t)backward_blocks(c->rows, per) * 2 * c->width * 4;
}

template <typename T> int launch(const Norm &a, hipStream_t s) {
    return with_shape<T>(a.width, [&](auto n, auto c) {
        constexpr int N = decltype(n)::value, C = decltype(c)::value;
        const uint32_t per = 256 / N, blocks = (a.rows + per - 1) / per;
        return enqueue(norm_rows<T, N, C>, blocks < 2048 ? blocks : 2048, 256, 0, s, a);
    });
}

template <typename T> int launch_backward(const Norm &a, float *dw, float *db, hipStream_t s) {
    return with_shape<T>(a.width, [&](auto n, auto c) {
        constexpr int N = decltype(n)::value, C = decltype(c)::value;
        const uint32_t blocks = backward_blocks(a.rows, 256 / N);
        const int rc = enqueue(norm_rows_backward<T, N, C>, blocks, 256, 0, s, a);
        if (rc != NLB_OK || !a.part) return rc;
        return enqueue(sum_shares, (2 * a.width + 63) / 64, 1024, 0, s, a.part, blocks, a.width, dw, db);
    });
}

}  // namespace

extern "C" int nlb_layer_norm(const nlb_norm_call *c, const float *b, float eps, void *y, int64_t y_stride,
                              void *stream) {
    Norm a;
    int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    if (bad_rows(y, y_stride, c->rows, c->dtype) || (uintptr_t)b % 4 || !(eps >= 0.0f) || std::isinf(eps))
        return NLB_EINVAL;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    if (c->rows == 0) return NLB_OK;
    a.b = b;
    a.eps = eps;
    a.out = (uint8_t *)y;
    a.out_row = y_stride * (c->dtype == NLB_DTYPE_BF16 ? 2 : 4);
    return c->dtype == NLB_DTYPE_BF16 ? launch<__bf16>(a, (hipStream_t)stream) : launch<float>(a, (hipStream_t)stream);
}

extern "C" int nlb_layer_norm_work(const nlb_norm_call *c, size_t *bytes) {
    Norm a;
    if (!bytes) return NLB_EINVAL;
    const int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    *bytes = work_of(c);
    return NLB_OK;
}

extern "C" int nlb_layer_norm_backward(const nlb_norm_call *c, const void *dy, int64_t dy_stride, void *dx,
                                       int64_t dx_stride, float *dw, float *db, void *work, size_t work_bytes,
                                       void *stream) {
    Norm a;
    int rc = fill(c, a);
    if (rc != NLB_OK) return rc;
    if (bad_rows(dy, dy_stride, c->rows, c->dtype) || bad_rows(dx, dx_stride, c->rows, c->dtype)) return NLB_EINVAL;
    if (c->rows && (!c->mean || !c->rstd)) return NLB_EINVAL;
    if (((uintptr_t)dw | (uintptr_t)db) % 4 || (uintptr_t)work % 16) return NLB_EINVAL;
    if ((dw || db) && (!work || work_bytes < work_of(c))) return NLB_ESCRATCH;
    CallDevice device(c->device);
    if (device.rc != NLB_OK) return device.rc;
    const int64_t e = c->dtype == NLB_DTYPE_BF16 ? 2 : 4;
    a.dy = (const uint8_t *)dy;
    a.dy_row = dy_stride * e;
    a.out = (uint8_t *)dx;
    a.out_row = dx_stride * e;
    a.part = dw || db ? (float *)work : nullptr;
    return c->dtype == NLB_DTYPE_BF16 ? launch_backward<__bf16>(a, dw, db, (hipStream_t)stream)
                                      : launch_backward<float>(a, dw, db, (hipStream_t)stream);
}
