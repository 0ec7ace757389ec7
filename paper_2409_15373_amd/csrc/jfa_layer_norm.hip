// Layer norm of the rows of a jagged tensor and its gradient (see jfa_layer_norm in jfa.h):
//   mean, rstd = 1 / sqrt(var + eps) of a row;  xh = (x - mean) rstd;  y = xh w + b
//   dx = rstd (w dy - mean(w dy) - xh mean(w dy xh));  dw = sum over rows of dy xh,  db = sum over rows of dy
// Bound by HBM: x in and y out, and x and dy in and dx out.  A row is read once: it stays in the registers of the lanes that share it for the
// mean, the variance about it and the result, in fp32.  A row has a wave or a part of one, or a workgroup; rows
// too long for registers (more than 16 KB) are read again from the caches.  dw and db are summed where a row passes through: a lane has the same columns of
// every row that its wave takes, so its sums are registers until the end, one partial row per workgroup; a second launch adds those in a fixed order.
#include "jfa_rows.h"

namespace jfa {

namespace {

constexpr int kLnThreads = 256;

// Sum over the `LANES` lanes that share a row: a power of two up to 64, or all 256 of a workgroup (`slots` [4] is free again after the next call's first barrier).
template <int LANES> __device__ inline float lanes_sum(float x, float *slots) {
#pragma unroll
    for (int d = 1; d < (LANES < 64 ? LANES : 64); d <<= 1) x += __shfl_xor(x, d, 64);
    if constexpr (LANES > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = x;
        __syncthreads();
        x = (slots[0] + slots[1]) + (slots[2] + slots[3]);
    }
    return x;
}

// The vectors of a row that a lane has, as they lie in memory; zero behind the row's end.
template <typename T, int ITEMS, int LANES, bool EVEN> struct RowPart {
    static constexpr int VEC = kRowVec<T>;
    RowRaw<T, VEC> v[ITEMS];
    __device__ void read(const T *tensor, int64_t r, int N, int lane) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
            v[i] = RowRaw<T, VEC>{};
            if (own < N) v[i] = read_vec<T, VEC, EVEN>(tensor + r * N + c, N - c);
        }
    }
};

// LANES lanes per row (a wave or part of one, or the workgroup), ITEMS vectors each, one row at a time.  (Two in flight: 586000 rows of 512 bf16 4.9 -> 5.0 TB/s, but
// 14848 of them 7.8 -> 8.3 us and 1000 3.0 -> 3.8.)
template <typename T, int ITEMS, int LANES, bool EVEN>
__global__ __launch_bounds__(kLnThreads) void layer_norm_kernel(const T *__restrict__ x, const T *__restrict__ weight, const T *__restrict__ bias,
                                                                const int64_t *__restrict__ offsets, int64_t B, int64_t rows, int64_t reps, int N, float eps,
                                                                T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int kPerBlock = kLnThreads / LANES, VEC = kRowVec<T>;
    __shared__ float slots[4];
    const int64_t n = rows_there(offsets, B, rows) * reps, step = (int64_t)gridDim.x * kPerBlock;
    const int lane = threadIdx.x % LANES;
    const float inv = 1.0f / (float)N;
    RowPart<T, ITEMS, LANES, EVEN> part;
    for (int64_t r = (int64_t)blockIdx.x * kPerBlock + threadIdx.x / LANES; r < n; r += step) {
        part.read(x, r, N, lane);
        float v[ITEMS][VEC], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
            widen_vec<T, VEC>(part.v[i], v[i]);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (EVEN || c + e >= own) sum += v[i][e];
        }
        const float m = lanes_sum<LANES>(sum, slots) * inv;
        float square = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (own < N && (EVEN || (c + e >= own && c + e < N))) square += (v[i][e] - m) * (v[i][e] - m);
        }
        const float rs = 1.0f / sqrtf(lanes_sum<LANES>(square, slots) * inv + eps);
        if (lane == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = rs;
        }
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
            if (own < N) {
                float w[VEC], b[VEC];
                if (weight) load_vec<T, VEC, EVEN>(weight + c, N - c, w);
                if (bias) load_vec<T, VEC, EVEN>(bias + c, N - c, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i][e] = (v[i][e] - m) * rs * (weight ? w[e] : 1.0f) + (bias ? b[e] : 0.0f);
                store_vec<T, VEC, EVEN>(y + r * N + c, N - c, v[i]);
            }
        }
    }
}

// Rows of any length, a workgroup per row.
template <typename T, bool EVEN>
__global__ __launch_bounds__(kLnThreads) void layer_norm_long_kernel(const T *__restrict__ x, const T *__restrict__ weight, const T *__restrict__ bias,
                                                                     const int64_t *__restrict__ offsets, int64_t B, int64_t rows, int64_t reps, int64_t N,
                                                                     float eps, T *__restrict__ y, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int VEC = kRowVec<T>;
    __shared__ float slots[4];
    const int64_t n = rows_there(offsets, B, rows) * reps;
    const float inv = 1.0f / (float)N;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const T *row = x + r * N;
        float sum = 0.0f, square = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < N; c += kLnThreads * VEC) {
            float v[VEC];
            load_vec<T, VEC, EVEN>(row + c, N - c, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += v[e];
        }
        const float m = lanes_sum<kLnThreads>(sum, slots) * inv;
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < N; c += kLnThreads * VEC) {
            float v[VEC];
            load_vec<T, VEC, EVEN>(row + c, N - c, v);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (c + (EVEN ? 0 : e) < N) square += (v[e] - m) * (v[e] - m);
        }
        const float rs = 1.0f / sqrtf(lanes_sum<kLnThreads>(square, slots) * inv + eps);
        if (threadIdx.x == 0) {
            if (mean) mean[r] = m;
            if (rstd) rstd[r] = rs;
        }
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < N; c += kLnThreads * VEC) {
            float v[VEC], w[VEC], b[VEC];
            load_vec<T, VEC, EVEN>(row + c, N - c, v);
            if (weight) load_vec<T, VEC, EVEN>(weight + c, N - c, w);
            if (bias) load_vec<T, VEC, EVEN>(bias + c, N - c, b);
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] = (v[e] - m) * rs * (weight ? w[e] : 1.0f) + (bias ? b[e] : 0.0f);
            store_vec<T, VEC, EVEN>(y + r * N + c, N - c, v);
        }
    }
}

// dx of LANES lanes' rows, and the workgroup's sums of dy xh and dy into partial[workgroup][2][N].
template <typename T, int ITEMS, int LANES, bool EVEN>
__global__ __launch_bounds__(kLnThreads) void layer_norm_backward_kernel(const T *__restrict__ x, const T *__restrict__ weight, const T *__restrict__ dy,
                                                                         const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                         const int64_t *__restrict__ offsets, int64_t B, int64_t rows, int64_t reps, int N,
                                                                         T *__restrict__ dx, float *__restrict__ partial) {
    constexpr int kPerBlock = kLnThreads / LANES, VEC = kRowVec<T>, kCols = LANES <= 64 ? ITEMS * VEC * LANES : 1;
    __shared__ float sums[4][kCols], slots[4];   // sums: of each wave
    const int64_t n = rows_there(offsets, B, rows) * reps, step = (int64_t)gridDim.x * kPerBlock;
    const int lane = threadIdx.x % LANES, wave = threadIdx.x >> 6;
    const float inv = 1.0f / (float)N;
    float dw[ITEMS][VEC], db[ITEMS][VEC];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) dw[i][e] = db[i][e] = 0.0f;
    RowPart<T, ITEMS, LANES, EVEN> part_x, part_dy;
    for (int64_t r = (int64_t)blockIdx.x * kPerBlock + threadIdx.x / LANES; r < n; r += step) {
        const float m = mean[r], rs = rstd[r];
        part_x.read(x, r, N, lane);
        part_dy.read(dy, r, N, lane);
        float h[ITEMS][VEC], g[ITEMS][VEC], s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
            widen_vec<T, VEC>(part_x.v[i], h[i]);
            widen_vec<T, VEC>(part_dy.v[i], g[i]);
            if (own < N) {
                float w[VEC];
                if (weight) load_vec<T, VEC, EVEN>(weight + c, N - c, w);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {   // (behind the row's end dy is zero)
                    h[i][e] = (h[i][e] - m) * rs;
                    const bool counts = EVEN || c + e >= own;
                    if (counts) {
                        dw[i][e] += g[i][e] * h[i][e];
                        db[i][e] += g[i][e];
                    }
                    if (weight) g[i][e] *= w[e];
                    if (counts) {
                        s1 += g[i][e];
                        s2 += g[i][e] * h[i][e];
                    }
                }
            }
        }
        s1 = lanes_sum<LANES>(s1, slots) * inv;
        s2 = lanes_sum<LANES>(s2, slots) * inv;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
            if (own < N) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) h[i][e] = rs * (g[i][e] - s1 - h[i][e] * s2);
                store_vec<T, VEC, EVEN>(dx + r * N + c, N - c, h[i]);
            }
        }
    }
    if (!partial) return;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
        float *const dst = partial + ((int64_t)blockIdx.x * 2 + pass) * N;
        if constexpr (LANES > 64) {   // every lane has columns of its own
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (own < N && (EVEN || (c + e >= own && c + e < N))) dst[c + e] = pass ? db[i][e] : dw[i][e];
            }
        } else {   // the lanes of a wave that share columns, then the four waves
            __syncthreads();
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int own = (i * LANES + lane) * VEC, c = vec_at<VEC, EVEN>(own, N) + e;
                    float s = pass ? db[i][e] : dw[i][e];
#pragma unroll
                    for (int d = LANES; d < 64; d <<= 1) s += __shfl_xor(s, d, 64);
                    if ((threadIdx.x & 63) < LANES && own < N && c >= own) sums[wave][c] = s;
                }
            __syncthreads();
            for (int c = threadIdx.x; c < N; c += kLnThreads) dst[c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
        }
    }
}

// dx of rows of any length, a workgroup per row.
template <typename T, bool EVEN>
__global__ __launch_bounds__(kLnThreads) void layer_norm_backward_long_kernel(const T *__restrict__ x, const T *__restrict__ weight, const T *__restrict__ dy,
                                                                              const float *__restrict__ mean, const float *__restrict__ rstd,
                                                                              const int64_t *__restrict__ offsets, int64_t B, int64_t rows, int64_t reps,
                                                                              int64_t N, T *__restrict__ dx) {
    constexpr int VEC = kRowVec<T>;
    __shared__ float slots[4];
    const int64_t n = rows_there(offsets, B, rows) * reps;
    const float inv = 1.0f / (float)N;
    for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
        const float m = mean[r], rs = rstd[r];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < N; c += kLnThreads * VEC) {
            float h[VEC], g[VEC], w[VEC];
            load_vec<T, VEC, EVEN>(x + r * N + c, N - c, h);
            load_vec<T, VEC, EVEN>(dy + r * N + c, N - c, g);
            if (weight) load_vec<T, VEC, EVEN>(weight + c, N - c, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float u = weight ? g[e] * w[e] : g[e];
                s1 += u;
                s2 += u * (h[e] - m) * rs;
            }
        }
        s1 = lanes_sum<kLnThreads>(s1, slots) * inv;
        s2 = lanes_sum<kLnThreads>(s2, slots) * inv;
        for (int64_t c = (int64_t)threadIdx.x * VEC; c < N; c += kLnThreads * VEC) {
            float h[VEC], g[VEC], w[VEC];
            load_vec<T, VEC, EVEN>(x + r * N + c, N - c, h);
            load_vec<T, VEC, EVEN>(dy + r * N + c, N - c, g);
            if (weight) load_vec<T, VEC, EVEN>(weight + c, N - c, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) h[e] = rs * ((weight ? g[e] * w[e] : g[e]) - s1 - (h[e] - m) * rs * s2);
            store_vec<T, VEC, EVEN>(dx + r * N + c, N - c, h);
        }
    }
}

// The sums of dy xh and dy for rows of any length: 256 columns and every gridDim.y-th row per workgroup, into partial[blockIdx.y][2][N].
template <typename T>
__global__ __launch_bounds__(kLnThreads) void layer_norm_columns_kernel(const T *__restrict__ x, const T *__restrict__ dy, const float *__restrict__ mean,
                                                                        const float *__restrict__ rstd, const int64_t *__restrict__ offsets, int64_t B,
                                                                        int64_t rows, int64_t reps, int64_t N, float *__restrict__ partial) {
    const int64_t n = rows_there(offsets, B, rows) * reps, c = (int64_t)blockIdx.x * kLnThreads + threadIdx.x;
    if (c >= N) return;
    float dw = 0.0f, db = 0.0f;
#pragma unroll 4
    for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
        const float g = (float)dy[r * N + c];
        dw += g * ((float)x[r * N + c] - mean[r]) * rstd[r];
        db += g;
    }
    partial[(int64_t)blockIdx.y * 2 * N + c] = dw;
    partial[((int64_t)blockIdx.y * 2 + 1) * N + c] = db;
}

// partial [parts][2][N] -> dweight, dbias: 64 columns per workgroup, its 16 waves every 16th part each; blockIdx.y: which of the two.  (Four waves:
// 17.6 us for 1024 parts of 1024 columns.)
constexpr int kReduceThreads = 1024;
template <typename T>
__global__ __launch_bounds__(kReduceThreads) void layer_norm_reduce_kernel(const float *__restrict__ partial, int parts, int64_t N, T *__restrict__ dweight,
                                                                       T *__restrict__ dbias) {
    constexpr int kWaves = kReduceThreads / 64;
    __shared__ float sums[kWaves][64];
    T *const dst = blockIdx.y ? dbias : dweight;
    if (!dst) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < N) {
#pragma unroll 8
        for (int p = wave; p < parts; p += kWaves) s += partial[((int64_t)p * 2 + blockIdx.y) * N + c];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < N) {
#pragma unroll
        for (int d = kWaves / 2; d > 0; d /= 2)
#pragma unroll
            for (int w = 0; w < d; ++w) sums[w][lane] += sums[w + d][lane];
        dst[c] = (T)sums[0][lane];
    }
}

constexpr int kLnMostParts = 1024;

// Workgroups of the row kernels.
int64_t ln_grid(int64_t rows, int per_block) {
    const int64_t need = (rows + per_block - 1) / per_block;
    return need < 1 ? 1 : need < kLnMostParts ? need : kLnMostParts;
}

// How a row of N elements of T is spread: up to a wave's lanes with a vector each, then up to four vectors of each of a wave's lanes, then up to four of a workgroup's
// (a wave with eight vectors a lane, 4096 bf16 a row: 2.9 TB/s forward, 1.8 backward; a workgroup with two 5.2 and 5.4).  Longer rows have kernels of their own
// (ITEMS = 0), which read them again from the caches: 16384 bf16 a row 3.5 and 2.7 TB/s.
template <typename T, typename Launch> hipError_t ln_spread(int64_t N, bool aligned, Launch launch) {
    constexpr int kVec = kRowVec<T>;
    const auto with = [&](auto even) {
        const int64_t vectors = (N + kVec - 1) / kVec;
        using std::integral_constant;
        if (vectors <= 8) return launch(even, integral_constant<int, 1>{}, integral_constant<int, 8>{});
        if (vectors <= 16) return launch(even, integral_constant<int, 1>{}, integral_constant<int, 16>{});
        if (vectors <= 32) return launch(even, integral_constant<int, 1>{}, integral_constant<int, 32>{});
        if (vectors <= 64) return launch(even, integral_constant<int, 1>{}, integral_constant<int, 64>{});
        if (vectors <= 128) return launch(even, integral_constant<int, 2>{}, integral_constant<int, 64>{});
        if (vectors <= 256) return launch(even, integral_constant<int, 4>{}, integral_constant<int, 64>{});
        if (vectors <= 512) return launch(even, integral_constant<int, 2>{}, integral_constant<int, 256>{});
        if (vectors <= 1024) return launch(even, integral_constant<int, 4>{}, integral_constant<int, 256>{});
        return launch(even, integral_constant<int, 0>{}, integral_constant<int, 0>{});
    };
    return aligned && N % kVec == 0 ? with(std::true_type{}) : with(std::false_type{});
}

template <typename T>
hipError_t layer_norm_t(const T *x, const T *weight, const T *bias, const int64_t *offsets, int64_t B, int64_t rows, int64_t reps, int64_t N, float eps, T *y,
                        float *mean, float *rstd, hipStream_t stream) {
    return ln_spread<T>(N, aligned16(x, weight, bias, y), [&](auto even, auto items, auto lanes) {
        constexpr bool EVEN = decltype(even)::value;
        constexpr int I = decltype(items)::value, L = decltype(lanes)::value;
        if constexpr (I == 0) {
            const int64_t all = rows * reps;
            hipLaunchKernelGGL((layer_norm_long_kernel<T, EVEN>), dim3((unsigned)(all < 4096 ? all : 4096)), dim3(kLnThreads), 0, stream, x, weight, bias, offsets, B, rows, reps, N,
                               eps, y, mean, rstd);
        } else {
            constexpr int kPerBlock = kLnThreads / L;
            const int64_t need = (rows * reps + kPerBlock - 1) / kPerBlock;
            hipLaunchKernelGGL((layer_norm_kernel<T, I, L, EVEN>), dim3((unsigned)(need < 8192 ? need : 8192)), dim3(kLnThreads), 0, stream, x, weight, bias, offsets, B, rows, reps,
                               (int)N, eps, y, mean, rstd);
        }
        return hipGetLastError();
    });
}

template <typename T>
hipError_t layer_norm_backward_t(const T *x, const T *weight, const T *dy, const float *mean, const float *rstd, const int64_t *offsets, int64_t B, int64_t rows,
                                 int64_t reps, int64_t N, T *dx, T *dweight, T *dbias, float *partial, hipStream_t stream) {
    const dim3 reduce_grid((unsigned)((N + 63) / 64), 2);
    if (rows == 0) {   // sums of nothing
        hipLaunchKernelGGL((layer_norm_reduce_kernel<T>), reduce_grid, dim3(kReduceThreads), 0, stream, partial, 0, N, dweight, dbias);
        return hipGetLastError();
    }
    return ln_spread<T>(N, aligned16(x, weight, dy, dx), [&](auto even, auto items, auto lanes) {
        constexpr bool EVEN = decltype(even)::value;
        constexpr int I = decltype(items)::value, L = decltype(lanes)::value;
        const bool sums = dweight || dbias;
        int64_t parts;
        if constexpr (I == 0) {
            const int64_t all = rows * reps;
            hipLaunchKernelGGL((layer_norm_backward_long_kernel<T, EVEN>), dim3((unsigned)(all < 4096 ? all : 4096)), dim3(kLnThreads), 0, stream, x, weight, dy, mean, rstd, offsets,
                               B, rows, reps, N, dx);
            parts = all < 64 ? all : 64;
            if (sums)
                hipLaunchKernelGGL((layer_norm_columns_kernel<T>), dim3((unsigned)((N + kLnThreads - 1) / kLnThreads), (unsigned)parts), dim3(kLnThreads), 0, stream, x, dy, mean,
                                   rstd, offsets, B, rows, reps, N, partial);
        } else {
            parts = ln_grid(rows * reps, kLnThreads / L);
            hipLaunchKernelGGL((layer_norm_backward_kernel<T, I, L, EVEN>), dim3((unsigned)parts), dim3(kLnThreads), 0, stream, x, weight, dy, mean, rstd, offsets, B, rows, reps,
                               (int)N, dx, sums ? partial : nullptr);
        }
        if (sums)
            hipLaunchKernelGGL((layer_norm_reduce_kernel<T>), reduce_grid, dim3(kReduceThreads), 0, stream, partial, (int)parts, N, dweight, dbias);
        return hipGetLastError();
    });
}

}  // namespace

// Partial sums of the gradients of weight and bias: at most one pair of rows per workgroup.
size_t layer_norm_workspace(int64_t rows, int64_t N) {
    const int64_t parts = rows < kLnMostParts ? rows : kLnMostParts;
    return (size_t)(parts * 2 * N) * sizeof(float);
}

hipError_t launch_layer_norm(bool f32, const void *x, const void *weight, const void *bias, const int64_t *offsets, int64_t B, int64_t rows, int64_t reps,
                             int64_t N, float eps, void *y, float *mean, float *rstd, hipStream_t stream) {
    if (f32) return layer_norm_t<float>((const float *)x, (const float *)weight, (const float *)bias, offsets, B, rows, reps, N, eps, (float *)y, mean, rstd, stream);
    return layer_norm_t<__bf16>((const __bf16 *)x, (const __bf16 *)weight, (const __bf16 *)bias, offsets, B, rows, reps, N, eps, (__bf16 *)y, mean, rstd, stream);
}
hipError_t launch_layer_norm_backward(bool f32, const void *x, const void *weight, const void *dy, const float *mean, const float *rstd, const int64_t *offsets,
                                      int64_t B, int64_t rows, int64_t reps, int64_t N, void *dx, void *dweight, void *dbias, void *workspace,
                                      hipStream_t stream) {
    if (f32)
        return layer_norm_backward_t<float>((const float *)x, (const float *)weight, (const float *)dy, mean, rstd, offsets, B, rows, reps, N, (float *)dx,
                                            (float *)dweight, (float *)dbias, (float *)workspace, stream);
    return layer_norm_backward_t<__bf16>((const __bf16 *)x, (const __bf16 *)weight, (const __bf16 *)dy, mean, rstd, offsets, B, rows, reps, N, (__bf16 *)dx,
                                         (__bf16 *)dweight, (__bf16 *)dbias, (float *)workspace, stream);
}

}  // namespace jfa
