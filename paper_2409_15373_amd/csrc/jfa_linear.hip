// Linear attention with a decay for each head on jagged samples (see jfa_linear_attention in jfa.h).  With g = exp(log_decay[h]),
//   S_i = g S_(i-1) + k_i^T v_i,   out_i = scale q_i S_i
// and its gradients are walks of the same kind.  With G_ij = g^(i-j) (dout_i . v_j) and P_ij = g^(i-j) (q_i . k_j), j <= i,
//   dq_i = scale sum_j G_ij k_j      : the walk with (dout, v, k) for (q, k, v)
//   dk_j = scale sum_i G_ij q_i      : the walk from the last row to the first, with (v, dout, q)
//   dv_j = scale sum_i P_ij dout_i   : the same direction, with (k, q, dout)
// so one kernel serves all four.  It goes through a (sample, head) pair kRows rows at a time (a chunk): inside the chunk by the product of its
// rows, P = (A B^T) o g^(i-j) and P C, from chunk to chunk through the D x D state, which stays in the accumulators of the matrix
// instructions from the first row to the last:
//   out = P C + g^(i+1) A S,   S <- g^rows S + (g^(rows-1-i) B)^T C         (A, B, C: the walk's first, second and third argument)
// From last row to first a row's product enters before the decay: exponents i and rows - i instead.
//
// Each row of a tensor is read once and each output row written once: at 96 flops a byte (D = 128, 64 rows) that is bound by HBM.
#include "jfa_common.h"
#include "jfa_mfma.h"

namespace jfa {

namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// The two element types.  An operand holds 16 contraction indices, eight per lane: slot e of a lane in half h = lane / 32 is index
// (e / 4) * 8 + 4 h + e % 4, the order in which an accumulator tile holds its rows, so that a tile is an operand as it stands.
// rows(): the tile's rows along the lanes, contraction along its columns; cols(): its columns along the lanes, contraction along its rows.
template <typename T> struct Elem;

template <> struct Elem<__bf16> {
    typedef bf16x8 Operand;
    static constexpr int kRows = 64;
    __host__ __device__ static constexpr int row_bytes(int d) { return d * 2 + 32; }
    __device__ static f32x16 product(Operand a, Operand b, f32x16 c) { return mfma_32x32x16(a, b, c); }
    __device__ static Operand rows(const char *tile, int stride, int row0, int k0, int lane) {
        const char *p = tile + (row0 + (lane & 31)) * stride + (k0 + 4 * (lane >> 5)) * 2;
        const u32x2 lo = *reinterpret_cast<const u32x2 *>(p), hi = *reinterpret_cast<const u32x2 *>(p + 16);
        return __builtin_bit_cast(bf16x8, u32x4{lo[0], lo[1], hi[0], hi[1]});
    }
    __device__ static Operand cols(const char *tile, int stride, int col0, int k0, int lane) {
        const char *p = tile + (k0 + 4 * (lane >> 5) + ((lane & 15) >> 2)) * stride + col0 * 2 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
        return concat(lds_read_tr16(p), lds_read_tr16(p + 8 * stride));
    }
    __device__ static Operand pack(const f32x8 &x) {
        Operand r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (__bf16)x[e];
        return r;
    }
    __device__ static f32x8 widen(Operand x) {
        f32x8 r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = (float)x[e];
        return r;
    }
    __device__ static void store4(__bf16 *dst, f32x4 x) {
        bf16x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = (__bf16)x[e];
        *reinterpret_cast<bf16x4 *>(dst) = r;
    }
};

template <> struct Elem<float> {
    typedef f32x8 Operand;
    static constexpr int kRows = 32;
    __host__ __device__ static constexpr int row_bytes(int d) { return d * 4 + 16; }
    __device__ static f32x16 product(Operand a, Operand b, f32x16 c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    __device__ static Operand rows(const char *tile, int stride, int row0, int k0, int lane) {
        const char *p = tile + (row0 + (lane & 31)) * stride + (k0 + 4 * (lane >> 5)) * 4;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(p), hi = *reinterpret_cast<const f32x4 *>(p + 32);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ static Operand cols(const char *tile, int stride, int col0, int k0, int lane) {
        const char *p = tile + (k0 + 4 * (lane >> 5)) * stride + (col0 + (lane & 31)) * 4;
        Operand r;
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = *reinterpret_cast<const float *>(p + ((e >> 2) * 8 + (e & 3)) * stride);
        return r;
    }
    __device__ static Operand pack(const f32x8 &x) { return x; }
    __device__ static f32x8 widen(Operand x) { return x; }
    __device__ static void store4(float *dst, f32x4 x) { *reinterpret_cast<f32x4 *>(dst) = x; }
};

__device__ inline f32x8 eight(const f32x16 &acc, int first) {
    f32x8 r;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = acc[first + e];
    return r;
}

// log2 of the decay.  A decay of zero (log_decay = -inf) becomes 2^-1024, whose first power is zero and whose zeroth is one.
__device__ inline float log2_decay(float log_decay) {
    const float x = log_decay * 1.4426950408889634f;
    return x < -1024.0f ? -1024.0f : x;
}
__device__ inline float power(float log2_g, int n) { return fast_exp2(log2_g * (float)n); }   // n >= 0

}  // namespace

// One walk per blockIdx.y, one (sample, head, segment) per blockIdx.x; D / 32 waves.  Wave w owns columns 32 w .. 32 w + 31 of the state and of
// the outputs.  kParts: into how many bf16 parts the decayed rows of C are split for the state's product: one where the state only
// feeds bf16 outputs, three (exact) where it is itself a result.
// kStateOnly: the state that a segment adds to, for those with a segment after them, into `carried`.
template <typename T, int D, int kParts, bool kStateOnly>
__global__ __launch_bounds__(2 * D) void linear_walk_kernel(LinearWalks walks, const float *__restrict__ log_decay, const int64_t *__restrict__ offsets,
                                                            int H, int segments, int segment_rows, float *__restrict__ carried) {
    typedef Elem<T> E;
    typedef typename E::Operand Operand;
    constexpr int kRows = E::kRows, kThreads = 2 * D, kRowBytes = E::row_bytes(D), kSize = (int)sizeof(T);
    constexpr int kTiles = kRows / 32, kStateTiles = D / 32, kSteps = D / 16;
    constexpr int kPRow = kRows * kSize + 16;
    constexpr int kChunksPerRow = D * kSize / 16, kLoads = kRows * kChunksPerRow / kThreads;   // 16-byte chunks of a tile per thread
    __shared__ __attribute__((aligned(16))) char at[kStateOnly ? 16 : kRows * kRowBytes], bt[kRows * kRowBytes], ct[kRows * kRowBytes], pt[kStateOnly ? 16 : kRows * kPRow];
    const LinearWalk &walk = walks.walk[blockIdx.y];
    const int pair = blockIdx.x / segments, segment = blockIdx.x - pair * segments;
    const int b = pair / H, h = pair - b * H;
    const int64_t first = offsets[b];
    const int64_t L = offsets[b + 1] - first;
    const int64_t t0 = (int64_t)segment * segment_rows;   // rows are counted in the order of the walk
    const bool last = t0 + segment_rows >= L;
    if (kStateOnly ? last || segment == segments - 1 : (t0 >= L && segment > 0)) return;
    const int64_t left = L - t0;
    const int n = (int)(left < segment_rows ? left : segment_rows);   // rows of this segment; 0 for an empty sample
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, half = lane >> 5;
    const bool reverse = walk.reverse;
    const float lg = log2_decay(log_decay[h]);
    float *const state_out = kStateOnly ? carried + (((int64_t)blockIdx.y * (gridDim.x / segments) + pair) * (segments - 1) + segment) * D * D
                                        : last && walk.state_out ? walk.state_out + (int64_t)pair * D * D : nullptr;
    const bool out_transposed = !kStateOnly && walk.transposed;

    f32x16 S[kStateTiles];   // tile m: rows 32 m .. (dimension of B), columns 32 wave .. (dimension of C)
#pragma unroll
    for (int m = 0; m < kStateTiles; ++m)
#pragma unroll
        for (int v = 0; v < 16; ++v) S[m][v] = 0.0f;
    if (!kStateOnly) {
        const float *from = segment > 0 ? carried + (((int64_t)blockIdx.y * (gridDim.x / segments) + pair) * (segments - 1) + segment - 1) * D * D
                            : walk.state_in ? walk.state_in + (int64_t)pair * D * D : nullptr;
        if (from) {
            const bool transposed = segment == 0 && walk.transposed;
#pragma unroll
            for (int m = 0; m < kStateTiles; ++m)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = m * 32 + acc_row(v, half), c = wave * 32 + col;
                    S[m][v] = from[transposed ? c * D + r : r * D + c];
                }
        }
    }

    // Row t of the walk is row first + t, or first + L - 1 - t, of the tensors.
    const int64_t row_stride = (int64_t)H * D, step = reverse ? -row_stride : row_stride;
    const int64_t base = (first + (reverse ? L - 1 - t0 : t0)) * row_stride + (int64_t)h * D;
    const T *const sources[3] = {(const T *)walk.a + base, (const T *)walk.b + base, (const T *)walk.c + base};
    u32x4 held[3][kLoads];
    auto fetch = [&](int r0) {
#pragma unroll
        for (int s = kStateOnly ? 1 : 0; s < 3; ++s)
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int c = tid + kThreads * u, r = r0 + c / kChunksPerRow;
                held[s][u] = u32x4{0, 0, 0, 0};   // rows past the sample's end
                if (r < n) held[s][u] = *reinterpret_cast<const u32x4 *>(sources[s] + r * step + (c % kChunksPerRow) * (16 / kSize));
            }
    };

    // Powers of the decay.  diag: P's factors in a tile on the diagonal (column i = this lane, rows j); below it g^(32 + i - j) = g^(i + 1) g^(31 - j).
    const float in_scale = walk.in_scale, out_scale = walk.out_scale;
    float diag[16], below[kTiles > 1 ? 16 : 1], late[8];
    if (!kStateOnly) {
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int j = acc_row(v, half);
            diag[v] = col >= j ? in_scale * power(lg, col - j) : 0.0f;
            if (kTiles > 1) below[v] = in_scale * power(lg, 31 - j + col + 1);
        }
    }
    // late[e]: g^(15 - index) of a contraction step's rows; times g^(16 (steps left)) it is a row's decay up to the chunk's end
#pragma unroll
    for (int e = 0; e < 8; ++e) late[e] = in_scale * power(lg, 15 - ((e >> 2) * 8 + 4 * half + (e & 3)));
    const float chunk_decay = power(lg, kRows);
    const int tail = reverse ? 1 : 0;   // the decay after a chunk's last row

    fetch(0);
    for (int r0 = 0; r0 < n; r0 += kRows) {
        const int rows = n - r0 < kRows ? n - r0 : kRows;
        __syncthreads();   // the previous chunk's tiles are free
#pragma unroll
        for (int s = kStateOnly ? 1 : 0; s < 3; ++s) {
            char *tile = s == 0 ? at : s == 1 ? bt : ct;
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int c = tid + kThreads * u;
                *reinterpret_cast<u32x4 *>(tile + (c / kChunksPerRow) * kRowBytes + (c % kChunksPerRow) * 16) = held[s][u];
            }
        }
        __syncthreads();
        if (r0 + kRows < n) fetch(r0 + kRows);
        if (!kStateOnly) {
            // P^T, tile (rows j of B) x (columns i of A) by tile; it is zero above the diagonal
            int t = 0;
#pragma unroll
            for (int ti = 0; ti < kTiles; ++ti)
#pragma unroll
                for (int tj = 0; tj <= ti; ++tj, ++t) {
                    if (t % kStateTiles != wave) continue;
                    f32x16 p;
#pragma unroll
                    for (int v = 0; v < 16; ++v) p[v] = 0.0f;
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks)
                        p = E::product(E::rows(bt, kRowBytes, tj * 32, ks * 16, lane), E::rows(at, kRowBytes, ti * 32, ks * 16, lane), p);
#pragma unroll
                    for (int v = 0; v < 16; ++v) p[v] = ti > tj ? p[v] * below[kTiles > 1 ? v : 0] : col < acc_row(v, half) ? 0.0f : p[v] * diag[v];
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        E::store4(reinterpret_cast<T *>(pt + (ti * 32 + col) * kPRow) + tj * 32 + g * 8 + half * 4, f32x4{p[4 * g], p[4 * g + 1], p[4 * g + 2], p[4 * g + 3]});
                }
            __syncthreads();
            // out^T = C^T P^T + g^(i + 1) S^T A^T, this wave's columns of C
#pragma unroll
            for (int ti = 0; ti < kTiles; ++ti) {
                f32x16 o;
#pragma unroll
                for (int v = 0; v < 16; ++v) o[v] = 0.0f;
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks)
                    o = E::product(E::pack(eight(S[ks >> 1], (ks & 1) * 8)), E::rows(at, kRowBytes, ti * 32, ks * 16, lane), o);
                const float since = power(lg, ti * 32 + col + 1 - tail);
#pragma unroll
                for (int v = 0; v < 16; ++v) o[v] *= since;
#pragma unroll
                for (int ks = 0; ks < 2 * (ti + 1); ++ks)
                    o = E::product(E::cols(ct, kRowBytes, wave * 32, ks * 16, lane), E::rows(pt, kPRow, ti * 32, ks * 16, lane), o);
                const int r = ti * 32 + col;
                if (r < rows) {
                    T *dst = (T *)walk.out + base + (r0 + r) * step + wave * 32 + half * 4;
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        E::store4(dst + g * 8, f32x4{o[4 * g] * out_scale, o[4 * g + 1] * out_scale, o[4 * g + 2] * out_scale, o[4 * g + 3] * out_scale});
                }
            }
        }
        // S <- g^rows S + (g^(rows - 1 - i) B)^T C, unless nobody looks at it any more
        if (r0 + kRows < n || state_out) {
            const float decay = rows == kRows ? chunk_decay : power(lg, rows);
#pragma unroll
            for (int m = 0; m < kStateTiles; ++m)
#pragma unroll
                for (int v = 0; v < 16; ++v) S[m][v] *= decay;
#pragma unroll
            for (int ks = 0; ks < kRows / 16; ++ks) {
                f32x8 c = E::widen(E::cols(ct, kRowBytes, wave * 32, ks * 16, lane));
                if (rows == kRows) {
                    const float rest = power(lg, kRows - 16 - ks * 16 + tail);
#pragma unroll
                    for (int e = 0; e < 8; ++e) c[e] *= late[e] * rest;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int after = rows - 1 - (ks * 16 + (e >> 2) * 8 + 4 * half + (e & 3));
                        c[e] *= after < 0 ? 0.0f : in_scale * power(lg, after + tail);
                    }
                }
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    const Operand x = E::pack(c);
#pragma unroll
                    for (int m = 0; m < kStateTiles; ++m) S[m] = E::product(E::cols(bt, kRowBytes, m * 32, ks * 16, lane), x, S[m]);
                    if (part + 1 < kParts) c -= E::widen(x);
                }
            }
        }
    }
    if (state_out) {
#pragma unroll
        for (int m = 0; m < kStateTiles; ++m)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = m * 32 + acc_row(v, half), c = wave * 32 + col;
                state_out[out_transposed ? c * D + r : r * D + c] = S[m][v];
            }
    }
}

// carried[m] (what segment m adds) -> the state in front of segment m + 1, for every (walk, sample, head) and element.
__global__ __launch_bounds__(256) void linear_carry_kernel(LinearWalks walks, const float *__restrict__ log_decay, const int64_t *__restrict__ offsets,
                                                           int H, int D, int segments, int segment_rows, float *__restrict__ carried) {
    const int blocks = D * D / 1024;   // 1024 elements, four per thread, per workgroup
    const int pair = blockIdx.x / blocks, at = (blockIdx.x - pair * blocks) * 1024 + threadIdx.x * 4;
    const LinearWalk &walk = walks.walk[blockIdx.y];
    const int b = pair / H;
    const int64_t L = offsets[b + 1] - offsets[b];
    const int64_t passed = (L + segment_rows - 1) / segment_rows - 1;   // segments with one after them
    const int n = (int)(passed < segments - 1 ? passed : segments - 1);
    if (n <= 0) return;
    const float decay = fast_exp2(log2_decay(log_decay[pair - b * H]) * (float)segment_rows);
    f32x4 S = {0.0f, 0.0f, 0.0f, 0.0f};
    if (walk.state_in) {
        const float *from = walk.state_in + (int64_t)pair * D * D;
        const int r = at / D, c = at % D;
#pragma unroll
        for (int e = 0; e < 4; ++e) S[e] = from[walk.transposed ? (c + e) * D + r : at + e];
    }
    f32x4 *x = reinterpret_cast<f32x4 *>(carried + ((int64_t)blockIdx.y * (gridDim.x / blocks) + pair) * (segments - 1) * D * D + at);
    const int64_t stride = (int64_t)D * D / 4;
    constexpr int kAhead = 8;
    for (int m0 = 0; m0 < n; m0 += kAhead) {
        f32x4 y[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (m0 + u < n) y[u] = x[(m0 + u) * stride];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (m0 + u < n) {
                S = S * decay + y[u];
                x[(m0 + u) * stride] = S;
            }
    }
}

// One token per sequence: S <- g S + k^T v, out = scale q S.  Bound by the state, read once and written once.  A workgroup has
// kCols columns of one (sequence, head)'s state; a thread four of them and every kLanes-th row.
template <typename T, int kCols>
__global__ __launch_bounds__(256) void linear_step_kernel(const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v,
                                                          const float *__restrict__ log_decay, int H, int D, float scale, const float *state,
                                                          T *__restrict__ out, float *new_state) {
    constexpr int kGroups = kCols / 4, kLanes = 256 / kGroups;
    __shared__ f32x4 sums[256];
    const int strips = D / kCols, pair = blockIdx.x / strips, strip = blockIdx.x - pair * strips;
    const int tid = threadIdx.x, g = tid % kGroups, r0 = tid / kGroups;
    const float decay = fast_exp2(log2_decay(log_decay[pair % H]));
    const int64_t row = (int64_t)pair * D, at = row * D + strip * kCols + g * 4;
    f32x4 vc, o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e) vc[e] = (float)v[row + strip * kCols + g * 4 + e];
#pragma unroll 8
    for (int r = r0; r < D; r += kLanes) {
        f32x4 s = *reinterpret_cast<const f32x4 *>(state + at + (int64_t)r * D);
        s = s * decay + vc * (float)k[row + r];
        *reinterpret_cast<f32x4 *>(new_state + at + (int64_t)r * D) = s;
        o += s * (float)q[row + r];
    }
    sums[tid] = o;
    __syncthreads();
    for (int n = kLanes / 2; n > 0; n >>= 1) {
        if (r0 < n) sums[tid] += sums[tid + n * kGroups];
        __syncthreads();
    }
    if (r0 == 0) Elem<T>::store4(out + row + strip * kCols + g * 4, sums[tid] * scale);
}

// Rows of a segment: so many that every compute unit has two walks, at least kLeastSegment, and always whole chunks.
int linear_segment_rows(int64_t B, int64_t max_len, int H, int walks, int cus) {
    constexpr int64_t kLeastSegment = 256;
    const int64_t pairs = B * H * walks, wanted = (2 * (int64_t)cus + pairs - 1) / pairs;   // segments per pair
    int64_t rows = (max_len + wanted - 1) / wanted;
    rows = (rows + 63) / 64 * 64;
    if (rows < kLeastSegment) rows = kLeastSegment;
    if (rows >= max_len) rows = (max_len + 63) / 64 * 64;
    return (int)(rows > 0 ? rows : 64);
}

template <typename T, int D>
static hipError_t launch_walks(const LinearWalks &walks, int n_walks, bool states, const float *log_decay, const int64_t *offsets, int64_t B, int H,
                               int segments, int segment_rows, float *carried, hipStream_t stream) {
    const dim3 grid((unsigned)(B * H * segments), n_walks), threads(2 * D);
    constexpr int kExact = sizeof(T) == 2 ? 3 : 1;
    if (segments > 1) {
        if (states) hipLaunchKernelGGL((linear_walk_kernel<T, D, kExact, true>), grid, threads, 0, stream, walks, log_decay, offsets, H, segments, segment_rows, carried);
        else hipLaunchKernelGGL((linear_walk_kernel<T, D, 1, true>), grid, threads, 0, stream, walks, log_decay, offsets, H, segments, segment_rows, carried);
        hipLaunchKernelGGL(linear_carry_kernel, dim3((unsigned)(B * H * (D * D / 1024)), n_walks), dim3(256), 0, stream, walks, log_decay, offsets, H, D, segments,
                           segment_rows, carried);
    }
    if (states) hipLaunchKernelGGL((linear_walk_kernel<T, D, kExact, false>), grid, threads, 0, stream, walks, log_decay, offsets, H, segments, segment_rows, carried);
    else hipLaunchKernelGGL((linear_walk_kernel<T, D, 1, false>), grid, threads, 0, stream, walks, log_decay, offsets, H, segments, segment_rows, carried);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_walks(const LinearWalks &walks, int n_walks, bool states, const float *log_decay, const int64_t *offsets, int64_t B, int H, int D,
                               int segments, int segment_rows, float *carried, hipStream_t stream) {
    switch (D) {
        case 32: return launch_walks<T, 32>(walks, n_walks, states, log_decay, offsets, B, H, segments, segment_rows, carried, stream);
        case 64: return launch_walks<T, 64>(walks, n_walks, states, log_decay, offsets, B, H, segments, segment_rows, carried, stream);
        case 128: return launch_walks<T, 128>(walks, n_walks, states, log_decay, offsets, B, H, segments, segment_rows, carried, stream);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_linear_walks(bool f32, const LinearWalks &walks, int n_walks, bool states, const float *log_decay, const int64_t *offsets, int64_t B, int H,
                               int D, int segments, int segment_rows, float *carried, hipStream_t stream) {
    return f32 ? launch_walks<float>(walks, n_walks, states, log_decay, offsets, B, H, D, segments, segment_rows, carried, stream)
               : launch_walks<__bf16>(walks, n_walks, states, log_decay, offsets, B, H, D, segments, segment_rows, carried, stream);
}

template <typename T>
static hipError_t launch_step(const void *q, const void *k, const void *v, const float *log_decay, int64_t B, int H, int D, float scale, const float *state,
                              void *out, float *new_state, hipStream_t stream) {
    hipLaunchKernelGGL((linear_step_kernel<T, 32>), dim3((unsigned)(B * H * (D / 32))), dim3(256), 0, stream, (const T *)q, (const T *)k, (const T *)v, log_decay, H, D,
                       scale, state, (T *)out, new_state);
    return hipGetLastError();
}
hipError_t launch_linear_step(bool f32, const void *q, const void *k, const void *v, const float *log_decay, int64_t B, int H, int D, float scale,
                              const float *state, void *out, float *new_state, hipStream_t stream) {
    return f32 ? launch_step<float>(q, k, v, log_decay, B, H, D, scale, state, out, new_state, stream)
               : launch_step<__bf16>(q, k, v, log_decay, B, H, D, scale, state, out, new_state, stream);
}

}  // namespace jfa
