// Embedding lookup into the rows of a jagged tensor and its gradient (see jfa_embedding in jfa.h):
//   out_i = scale table[id_i],   dtable[v] = scale sum over the i with id_i = v of dout_i
// The lookup is a copy of rows: bound by HBM, 16 bytes per lane, several rows of a lane in flight.
// The gradient adds the rows of an id in the order of their positions, so that it is the same every time: the positions are sorted by id (radix
// sort, stable, of (id, position) pairs of eight bytes: a few per cent of the rows' bytes), and every row of the table is then written
// once, the sum of its positions' rows or zeros.  Frequent ids (one that stands for anything unknown may have a third of all positions) would
// keep one row's lanes busy long after the others: blocks of 64 sorted positions that all have one id are added beforehand, each by lanes of its own, and
// blocks of 64 such blocks from those, so that a row adds at most 63 single rows, 63 blocks and the blocks of blocks at either end.
#include "jfa_common.h"
#include "jfa_mfma.h"

namespace jfa {

namespace {

constexpr int kEmThreads = 256;
constexpr int kEmTile = 4096;    // positions that a workgroup sorts at a time
constexpr int kEmBlock = 64;     // positions of a block, blocks of a block of blocks
constexpr int kEmMostBits = 10;  // of a sort's digit

template <typename T, int VEC> struct EmVec { typedef T Type __attribute__((ext_vector_type(VEC))); };
template <typename T> struct EmVec<T, 1> { typedef T Type; };

template <typename T, int VEC> __device__ inline void em_load(const T *p, float (&x)[VEC]) {
    const typename EmVec<T, VEC>::Type v = *reinterpret_cast<const typename EmVec<T, VEC>::Type *>(p);
    if constexpr (VEC == 1) x[0] = (float)v;
    else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) x[e] = (float)v[e];
    }
}
template <typename T, int VEC> __device__ inline void em_store(T *p, const float (&x)[VEC]) {
    typename EmVec<T, VEC>::Type v;
    if constexpr (VEC == 1) v = (T)x[0];
    else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = (T)x[e];
    }
    *reinterpret_cast<typename EmVec<T, VEC>::Type *>(p) = v;
}

__device__ inline int64_t em_rows_there(const int64_t *offsets, int64_t B, int64_t rows) {
    if (!offsets) return rows;
    const int64_t have = offsets[B];
    return have < 0 ? 0 : have < rows ? have : rows;
}

// LANES lanes per row, kInFlight rows at a time.
template <typename T, typename Id, int VEC, int LANES>
__global__ __launch_bounds__(kEmThreads) void embedding_kernel(const T *__restrict__ table, const Id *__restrict__ ids, const int64_t *__restrict__ offsets,
                                                               int64_t B, int64_t rows, int64_t V, int64_t N, float scale, T *__restrict__ out) {
    constexpr int kPerBlock = kEmThreads / LANES, kInFlight = 4;
    const int64_t n = em_rows_there(offsets, B, rows);
    const int lane = threadIdx.x % LANES;
    for (int64_t i0 = (int64_t)blockIdx.x * kPerBlock * kInFlight + threadIdx.x / LANES; i0 < n; i0 += (int64_t)gridDim.x * kPerBlock * kInFlight) {
        int64_t id[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) id[u] = i0 + u * kPerBlock < n ? (int64_t)ids[i0 + u * kPerBlock] : -1;
        for (int64_t c = lane * VEC; c < N; c += LANES * VEC) {
            float x[kInFlight][VEC];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[u][e] = 0.0f;
                if (id[u] >= 0 && id[u] < V) {
                    em_load<T, VEC>(table + id[u] * N + c, x[u]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[u][e] *= scale;
                }
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u)
                if (i0 + u * kPerBlock < n) em_store<T, VEC>(out + (i0 + u * kPerBlock) * N + c, x[u]);
        }
    }
}

// ---- positions by id ----
// What the first pass reads are the ids themselves; an id outside the table, or a row that is not there, has key V, behind all others.
struct SortSource {
    const void *ids;          // first pass; later ones read keys and positions
    const uint32_t *keys, *positions;
    const int64_t *offsets;
    int64_t B, V;
    int rows;
    bool ids64;
};
template <bool FIRST> __device__ inline uint32_t sort_key(const SortSource &s, int64_t there, int i) {
    if (!FIRST) return s.keys[i];
    const int64_t id = s.ids64 ? ((const int64_t *)s.ids)[i] : (int64_t)((const int32_t *)s.ids)[i];
    return i < there && id >= 0 && id < s.V ? (uint32_t)id : (uint32_t)s.V;
}

// counts[bin * tiles + tile]; the first pass also clears the table rows' bounds.
template <bool FIRST>
__global__ __launch_bounds__(kEmThreads) void sort_count_kernel(SortSource s, int shift, int bits, int tiles, uint32_t *__restrict__ counts, uint32_t *__restrict__ bounds) {
    __shared__ uint32_t bins[1 << kEmMostBits];
    const int n_bins = 1 << bits;
    for (int i = threadIdx.x; i < n_bins; i += kEmThreads) bins[i] = 0;
    __syncthreads();
    const int64_t there = FIRST ? em_rows_there(s.offsets, s.B, s.rows) : 0;
    const int first = (int)blockIdx.x * kEmTile, end = s.rows - first < kEmTile ? s.rows : first + kEmTile;
    for (int i = first + threadIdx.x; i < end; i += kEmThreads) atomicAdd(&bins[(sort_key<FIRST>(s, there, i) >> shift) & (n_bins - 1)], 1u);
    if (FIRST)
        for (int64_t i = (int64_t)blockIdx.x * kEmThreads + threadIdx.x; i < 2 * s.V; i += (int64_t)gridDim.x * kEmThreads) bounds[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n_bins; i += kEmThreads) counts[(int64_t)i * tiles + blockIdx.x] = bins[i];
}

// A wave per bin: counts -> the counts of the tiles before, and the bin's total.
__global__ __launch_bounds__(kEmThreads) void sort_scan_kernel(int n_bins, int tiles, uint32_t *__restrict__ counts, uint32_t *__restrict__ totals) {
    const int bin = blockIdx.x * (kEmThreads / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (bin >= n_bins) return;
    uint32_t *row = counts + (int64_t)bin * tiles, carry = 0;
    for (int t0 = 0; t0 < tiles; t0 += 64) {
        const uint32_t mine = t0 + lane < tiles ? row[t0 + lane] : 0;
        uint32_t sum = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t y = __shfl_up(sum, d, 64);
            if (lane >= d) sum += y;
        }
        if (t0 + lane < tiles) row[t0 + lane] = carry + sum - mine;
        carry += __shfl(sum, 63, 64);
    }
    if (lane == 0) totals[bin] = carry;
}

// Every key and position to its place.  A wave has a quarter of the tile in order; equal digits of a wave's 64 keys are ranked by ballots.
template <bool FIRST>
__global__ __launch_bounds__(kEmThreads) void sort_place_kernel(SortSource s, int shift, int bits, int tiles, const uint32_t *__restrict__ counts,
                                                                const uint32_t *__restrict__ totals, uint32_t *__restrict__ keys, uint32_t *__restrict__ positions) {
    constexpr int kWaves = kEmThreads / 64, kMine = kEmTile / kWaves, kRounds = kMine / 64;
    __shared__ uint32_t next[kWaves][1 << kEmMostBits];
    __shared__ uint32_t wave_totals[kWaves];
    const int n_bins = 1 << bits, mask = n_bins - 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t there = FIRST ? em_rows_there(s.offsets, s.B, s.rows) : 0;
    for (int i = threadIdx.x; i < n_bins; i += kEmThreads)
#pragma unroll
        for (int w = 0; w < kWaves; ++w) next[w][i] = 0;
    __syncthreads();
    const int first = (int)blockIdx.x * kEmTile + wave * kMine;
    uint32_t key[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = first + r * 64 + lane;
        key[r] = 0;
        if (i < s.rows) {
            key[r] = sort_key<FIRST>(s, there, i);
            atomicAdd(&next[wave][(key[r] >> shift) & mask], 1u);
        }
    }
    __syncthreads();
    // where a bin starts: the totals of the bins before it; a thread has kPer bins in a row
    const int per = n_bins / kEmThreads > 0 ? n_bins / kEmThreads : 1, bin0 = threadIdx.x * per;
    uint32_t mine = 0;
    if (bin0 < n_bins)
        for (int k = 0; k < per; ++k) mine += totals[bin0 + k];
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(sum, d, 64);
        if (lane >= d) sum += y;
    }
    if (lane == 63) wave_totals[wave] = sum;
    __syncthreads();
    uint32_t start = sum - mine;
    for (int w = 0; w < wave; ++w) start += wave_totals[w];
    if (bin0 < n_bins)
        for (int k = 0; k < per; ++k) {
            uint32_t at = start + counts[(int64_t)(bin0 + k) * tiles + blockIdx.x];
            start += totals[bin0 + k];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint32_t c = next[w][bin0 + k];
                next[w][bin0 + k] = at;
                at += c;
            }
        }
    __syncthreads();
    volatile uint32_t *const at = next[wave];   // the wave's own from here on; its LDS instructions are served in order
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = first + r * 64 + lane;
        const bool valid = i < s.rows;
        const int digit = (key[r] >> shift) & mask;
        uint64_t same = __builtin_amdgcn_ballot_w64(valid);
        for (int bit = 0; bit < bits; ++bit) {
            const bool set = (digit >> bit) & 1;
            const uint64_t votes = __builtin_amdgcn_ballot_w64(set);
            same &= set ? votes : ~votes;
        }
        uint32_t base = 0;
        if (valid) base = at[digit];
        const int before = __popcll(same & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (valid && before == 0) at[digit] = base + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
        if (valid) {
            keys[base + before] = key[r];
            positions[base + before] = FIRST ? (uint32_t)i : s.positions[i];
        }
    }
}

// bounds[2 v], bounds[2 v + 1]: the sorted positions of row v (cleared before: none).
__global__ __launch_bounds__(kEmThreads) void bounds_kernel(const uint32_t *__restrict__ keys, int rows, uint32_t V, uint32_t *__restrict__ bounds) {
    const int i = blockIdx.x * kEmThreads + threadIdx.x;
    if (i >= rows) return;
    const uint32_t key = keys[i];
    if (key >= V) return;
    if (i == 0 || keys[i - 1] != key) bounds[2 * (int64_t)key] = i;
    if (i == rows - 1 || keys[i + 1] != key) bounds[2 * (int64_t)key + 1] = i + 1;
}

// ---- sums of rows ----
// Adds `count` rows of `src`, row r at index(r); kAhead loads in flight.
template <typename S, int VEC, typename Index> __device__ inline void add_rows(const S *src, int64_t N, int64_t c, int from, int to, Index index, float (&sum)[VEC]) {
    constexpr int kAhead = 8;
    for (int r = from; r < to; r += kAhead) {
        float x[kAhead][VEC];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (r + u < to) em_load<S, VEC>(src + (int64_t)index(r + u) * N + c, x[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (r + u < to) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
            }
    }
}

// blocks[k][N]: the sum of sorted positions 64 k .. 64 k + 63 where all of them have one id.
template <typename T, int VEC, int LANES>
__global__ __launch_bounds__(kEmThreads) void block_sums_kernel(const T *__restrict__ dout, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ positions,
                                                                int n_blocks, uint32_t V, int64_t N, float *__restrict__ blocks) {
    const int k = blockIdx.x * (kEmThreads / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (k >= n_blocks) return;
    const int first = k * kEmBlock;
    const uint32_t key = keys[first];
    if (key >= V || keys[first + kEmBlock - 1] != key) return;
    for (int64_t c = lane * VEC; c < N; c += LANES * VEC) {
        float sum[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        add_rows<T, VEC>(dout, N, c, first, first + kEmBlock, [&](int r) { return positions[r]; }, sum);
        em_store<float, VEC>(blocks + (int64_t)k * N + c, sum);
    }
}

// supers[k][N]: the sum of blocks 64 k .. 64 k + 63 where all of their positions have one id.
template <int VEC, int LANES>
__global__ __launch_bounds__(kEmThreads) void super_sums_kernel(const uint32_t *__restrict__ keys, int n_supers, uint32_t V, int64_t N, const float *__restrict__ blocks,
                                                                float *__restrict__ supers) {
    const int k = blockIdx.x * (kEmThreads / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (k >= n_supers) return;
    const int64_t first = (int64_t)k * kEmBlock * kEmBlock;
    const uint32_t key = keys[first];
    if (key >= V || keys[first + kEmBlock * kEmBlock - 1] != key) return;
    for (int64_t c = lane * VEC; c < N; c += LANES * VEC) {
        float sum[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        add_rows<float, VEC>(blocks, N, c, k * kEmBlock, (k + 1) * kEmBlock, [](int r) { return r; }, sum);
        em_store<float, VEC>(supers + (int64_t)k * N + c, sum);
    }
}

// dtable: LANES lanes per row of the table.
template <typename T, int VEC, int LANES>
__global__ __launch_bounds__(kEmThreads) void table_rows_kernel(const T *__restrict__ dout, const uint32_t *__restrict__ positions, const uint32_t *__restrict__ bounds,
                                                                int64_t V, int64_t N, float scale, const float *__restrict__ blocks, const float *__restrict__ supers,
                                                                T *__restrict__ dtable) {
    constexpr int kPerBlock = kEmThreads / LANES;
    const int lane = threadIdx.x % LANES;
    for (int64_t v = (int64_t)blockIdx.x * kPerBlock + threadIdx.x / LANES; v < V; v += (int64_t)gridDim.x * kPerBlock) {
        const int first = (int)bounds[2 * v], end = (int)bounds[2 * v + 1];
        int block0 = (first + kEmBlock - 1) / kEmBlock, block1 = end / kEmBlock;   // the blocks inside
        if (block0 > block1) block0 = block1 = -1;
        int super0 = (block0 + kEmBlock - 1) / kEmBlock, super1 = block1 / kEmBlock;
        if (block0 < 0 || super0 > super1) super0 = super1 = -1;
        for (int64_t c = lane * VEC; c < N; c += LANES * VEC) {
            float sum[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
            const auto position = [&](int r) { return positions[r]; };
            const auto same = [](int r) { return r; };
            if (block0 < 0) add_rows<T, VEC>(dout, N, c, first, end, position, sum);
            else {
                add_rows<T, VEC>(dout, N, c, first, block0 * kEmBlock, position, sum);
                if (super0 < 0) add_rows<float, VEC>(blocks, N, c, block0, block1, same, sum);
                else {
                    add_rows<float, VEC>(blocks, N, c, block0, super0 * kEmBlock, same, sum);
                    add_rows<float, VEC>(supers, N, c, super0, super1, same, sum);
                    add_rows<float, VEC>(blocks, N, c, super1 * kEmBlock, block1, same, sum);
                }
                add_rows<T, VEC>(dout, N, c, block1 * kEmBlock, end, position, sum);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] *= scale;
            em_store<T, VEC>(dtable + v * N + c, sum);
        }
    }
}

template <typename T, typename Launch> hipError_t em_spread(int64_t N, bool aligned, Launch launch) {
    constexpr int kVec = 16 / (int)sizeof(T);
    const auto with = [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const int64_t vectors = (N + V - 1) / V;
        using std::integral_constant;
        if (vectors <= 4) return launch(vec, integral_constant<int, 4>{});
        if (vectors <= 8) return launch(vec, integral_constant<int, 8>{});
        if (vectors <= 16) return launch(vec, integral_constant<int, 16>{});
        if (vectors <= 32) return launch(vec, integral_constant<int, 32>{});
        return launch(vec, integral_constant<int, 64>{});
    };
    return aligned && N % kVec == 0 ? with(std::integral_constant<int, kVec>{}) : with(std::integral_constant<int, 1>{});
}

template <typename T, typename Id>
hipError_t embedding_t(const T *table, const Id *ids, const int64_t *offsets, int64_t B, int64_t rows, int64_t V, int64_t N, float scale, T *out, hipStream_t stream) {
    return em_spread<T>(N, aligned16(table, out), [&](auto vec, auto lanes) {
        constexpr int VEC = decltype(vec)::value, L = decltype(lanes)::value, kRows = kEmThreads / L * 4;
        const int64_t need = (rows + kRows - 1) / kRows;
        hipLaunchKernelGGL((embedding_kernel<T, Id, VEC, L>), dim3((unsigned)(need < 8192 ? need : 8192)), dim3(kEmThreads), 0, stream, table, ids, offsets, B, rows, V, N, scale,
                           out);
        return hipGetLastError();
    });
}

// The workspace's parts, in 4-byte words from its start.
struct EmPlan {
    int bits, passes, tiles;
    int n_blocks, n_supers;
    int64_t counts, totals, bounds, keys[2], positions[2], blocks, supers, words;
};
EmPlan em_plan(int64_t rows, int64_t V, int64_t N) {
    EmPlan p;
    int bits = 1;
    while (((int64_t)1 << bits) < V + 1) ++bits;   // keys 0 .. V
    p.passes = (bits + kEmMostBits - 1) / kEmMostBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = rows > 0 ? (int)((rows + kEmTile - 1) / kEmTile) : 1;   // (no rows: one tile with nothing in it)
    p.n_blocks = (int)(rows / kEmBlock);
    p.n_supers = (int)(rows / (kEmBlock * kEmBlock));
    int64_t at = 0;
    const auto take = [&](int64_t words) { const int64_t here = at; at += (words + 3) / 4 * 4; return here; };
    p.counts = take((int64_t)p.tiles << p.bits);
    p.totals = take((int64_t)1 << p.bits);
    p.bounds = take(2 * V);
    for (int i = 0; i < 2; ++i) { p.keys[i] = take(rows); p.positions[i] = take(rows); }
    p.blocks = take(p.n_blocks * N);
    p.supers = take(p.n_supers * N);
    p.words = at;
    return p;
}

template <typename T>
hipError_t embedding_backward_t(const T *dout, const void *ids, bool ids64, const int64_t *offsets, int64_t B, int64_t rows, int64_t V, int64_t N, float scale,
                                T *dtable, uint32_t *ws, hipStream_t stream) {
    const EmPlan p = em_plan(rows, V, N);
    const dim3 threads(kEmThreads);
    uint32_t *const counts = ws + p.counts, *const totals = ws + p.totals, *const bounds = ws + p.bounds;
    SortSource s{ids, nullptr, nullptr, offsets, B, V, (int)rows, ids64};
    for (int pass = 0; pass < p.passes; ++pass) {
        uint32_t *const keys = ws + p.keys[pass & 1], *const positions = ws + p.positions[pass & 1];
        const int shift = pass * p.bits;
        if (pass == 0) hipLaunchKernelGGL((sort_count_kernel<true>), dim3(p.tiles), threads, 0, stream, s, shift, p.bits, p.tiles, counts, bounds);
        else hipLaunchKernelGGL((sort_count_kernel<false>), dim3(p.tiles), threads, 0, stream, s, shift, p.bits, p.tiles, counts, bounds);
        hipLaunchKernelGGL(sort_scan_kernel, dim3(((1 << p.bits) + 3) / 4), threads, 0, stream, 1 << p.bits, p.tiles, counts, totals);
        if (pass == 0) hipLaunchKernelGGL((sort_place_kernel<true>), dim3(p.tiles), threads, 0, stream, s, shift, p.bits, p.tiles, counts, totals, keys, positions);
        else hipLaunchKernelGGL((sort_place_kernel<false>), dim3(p.tiles), threads, 0, stream, s, shift, p.bits, p.tiles, counts, totals, keys, positions);
        s.keys = keys;
        s.positions = positions;
    }
    hipLaunchKernelGGL(bounds_kernel, dim3((unsigned)(rows / kEmThreads + 1)), threads, 0, stream, s.keys, (int)rows, (uint32_t)V, bounds);
    float *const blocks = reinterpret_cast<float *>(ws + p.blocks), *const supers = reinterpret_cast<float *>(ws + p.supers);
    return em_spread<T>(N, aligned16(dout, dtable), [&](auto vec, auto lanes) {
        constexpr int VEC = decltype(vec)::value, L = decltype(lanes)::value, kPer = kEmThreads / L;
        if (p.n_blocks)
            hipLaunchKernelGGL((block_sums_kernel<T, VEC, L>), dim3((p.n_blocks + kPer - 1) / kPer), threads, 0, stream, dout, s.keys, s.positions, p.n_blocks, (uint32_t)V, N, blocks);
        if (p.n_supers)
            hipLaunchKernelGGL((super_sums_kernel<VEC, L>), dim3((p.n_supers + kPer - 1) / kPer), threads, 0, stream, s.keys, p.n_supers, (uint32_t)V, N, blocks, supers);
        const int64_t need = (V + kPer - 1) / kPer;
        hipLaunchKernelGGL((table_rows_kernel<T, VEC, L>), dim3((unsigned)(need < 65536 ? need : 65536)), threads, 0, stream, dout, s.positions, bounds, V, N, scale, blocks,
                           supers, dtable);
        return hipGetLastError();
    });
}

}  // namespace

size_t embedding_workspace(int64_t rows, int64_t V, int64_t N) { return (size_t)em_plan(rows, V, N).words * 4; }

hipError_t launch_embedding(bool f32, const void *table, const void *ids, bool ids64, const int64_t *offsets, int64_t B, int64_t rows, int64_t V, int64_t N,
                            float scale, void *out, hipStream_t stream) {
    if (f32) {
        if (ids64) return embedding_t((const float *)table, (const int64_t *)ids, offsets, B, rows, V, N, scale, (float *)out, stream);
        return embedding_t((const float *)table, (const int32_t *)ids, offsets, B, rows, V, N, scale, (float *)out, stream);
    }
    if (ids64) return embedding_t((const __bf16 *)table, (const int64_t *)ids, offsets, B, rows, V, N, scale, (__bf16 *)out, stream);
    return embedding_t((const __bf16 *)table, (const int32_t *)ids, offsets, B, rows, V, N, scale, (__bf16 *)out, stream);
}
hipError_t launch_embedding_backward(bool f32, const void *dout, const void *ids, bool ids64, const int64_t *offsets, int64_t B, int64_t rows, int64_t V,
                                     int64_t N, float scale, void *dtable, void *workspace, hipStream_t stream) {
    if (f32) return embedding_backward_t((const float *)dout, ids, ids64, offsets, B, rows, V, N, scale, (float *)dtable, (uint32_t *)workspace, stream);
    return embedding_backward_t((const __bf16 *)dout, ids, ids64, offsets, B, rows, V, N, scale, (__bf16 *)dtable, (uint32_t *)workspace, stream);
}

}  // namespace jfa
