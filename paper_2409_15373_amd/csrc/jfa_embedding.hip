// Embedding lookup into the rows of a jagged tensor and its gradient (see jfa_embedding in jfa.h):
//   out_i = scale table[id_i],   dtable[v] = scale sum over the i with id_i = v of dout_i
// The lookup is a copy of rows: bound by HBM, 16 bytes per lane, several rows of a lane in flight.
// The gradient adds the rows of an id in the order of their positions, so that it is the same every time: the positions are sorted by id (radix
// sort, stable, of (id, position) pairs of eight bytes: a few per cent of the rows' bytes), and every row of dout is then read once, in that order.
// The sorted positions are cut into blocks of kEmBlock, so that no id, however frequent (one that stands for anything unknown may
// have a third of all positions), keeps one row's lanes busy long after the others: what of a block belongs to an id with positions in other blocks is
// left as a partial sum, and those are added by the lanes of the block that the id begins in, kEmSuper of them at once where one
// id has that many.  The table's other rows are zeros: the sort, a few dozen workgroups that wait for memory, has the chip to itself, so its launches
// carry workgroups that clear the whole table (a row that is written again costs less than finding out that it will be).
#include "jfa_mfma.h"
#include "jfa_rows.h"

namespace jfa {

namespace {

constexpr int kEmThreads = 256;
constexpr int kEmBlock = 32;     // sorted positions of a block
constexpr int kEmSuper = 64;     // blocks that are added at once
constexpr int kEmMostBits = 10;  // of a sort's digit
constexpr int kSortThreads = 1024;

// LANES lanes per row, kInFlight rows at a time (2, 4 and 8: 29.7, 32.1 and 36.4 us for 322248 rows of 128).  PAST: rows are stored past the L2, for
// what has more of them than the L2s hold: the table's frequent rows stay (131072 rows of 512, 37 -> 25 us).
constexpr int kInFlight = 2;
constexpr int64_t kL2Bytes = 32 << 20;
template <typename T, typename Id, bool EVEN, int LANES, bool PAST>
__global__ __launch_bounds__(kEmThreads) void embedding_kernel(const T *__restrict__ table, const Id *__restrict__ ids, const int64_t *__restrict__ offsets,
                                                               int64_t B, int64_t rows, int64_t V, int64_t N, float scale, T *__restrict__ out) {
    constexpr int kPerBlock = kEmThreads / LANES, VEC = kRowVec<T>;
    const int64_t n = rows_there(offsets, B, rows);
    const int lane = threadIdx.x % LANES;
    for (int64_t i0 = (int64_t)blockIdx.x * kPerBlock * kInFlight + threadIdx.x / LANES; i0 < n; i0 += (int64_t)gridDim.x * kPerBlock * kInFlight) {
        int64_t id[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) id[u] = i0 + u * kPerBlock < n ? (int64_t)ids[i0 + u * kPerBlock] : -1;
        for (int64_t own = lane * VEC; own < N; own += LANES * VEC) {
            const int64_t c = vec_at<VEC, EVEN>(own, N);
            float x[kInFlight][VEC];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) x[u][e] = 0.0f;
                if (id[u] >= 0 && id[u] < V) {
                    load_vec<T, VEC, EVEN>(table + id[u] * N + c, N - c, x[u]);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[u][e] *= scale;
                }
            }
#pragma unroll
            for (int u = 0; u < kInFlight; ++u)
                if (i0 + u * kPerBlock < n) store_vec<T, VEC, EVEN, PAST>(out + (i0 + u * kPerBlock) * N + c, N - c, x[u]);
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

// What the workgroups behind a sort's own clear: `bytes` bytes from `dst` on, the ones of this launch from `from` to `to` (in units of kClearBytes).
struct Clearing {
    char *dst;
    int64_t bytes, from, to;
};
// Past the L2, where the rows of dout, which the block sums read next, may be (1000003 x 128: block sums 38 -> 21 us, and the next pass' lookup 30 -> 18).
constexpr int kClearBytes = kSortThreads * 16 * 4;
__device__ inline void clear_share(const Clearing &c, int64_t unit) {
    if (unit >= c.to) return;
    const int64_t at = unit * kClearBytes;
    if (((uintptr_t)c.dst & 15) == 0 && at + kClearBytes <= c.bytes) {
#pragma unroll
        for (int u = 0; u < 4; ++u) __builtin_nontemporal_store(u32x4{0, 0, 0, 0}, reinterpret_cast<u32x4 *>(c.dst + at + (u * kSortThreads + threadIdx.x) * 16));
        return;
    }
    for (int64_t i = at + threadIdx.x * 2; i < at + kClearBytes && i < c.bytes; i += kSortThreads * 2) *reinterpret_cast<uint16_t *>(c.dst + i) = 0;
}

// counts[tile][bin].  TILE: positions that a workgroup sorts at a time.
template <bool FIRST, int TILE>
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortSource s, int shift, int bits, int tiles, uint32_t *__restrict__ counts, Clearing clearing) {
    __shared__ uint32_t bins[1 << kEmMostBits];
    if ((int)blockIdx.x >= tiles) return clear_share(clearing, clearing.from + blockIdx.x - tiles);
    const int n_bins = 1 << bits;
    for (int i = threadIdx.x; i < n_bins; i += kSortThreads) bins[i] = 0;
    __syncthreads();
    const int64_t there = FIRST ? rows_there(s.offsets, s.B, s.rows) : 0;
    const int first = (int)blockIdx.x * TILE, end = s.rows - first < TILE ? s.rows : first + TILE;
    for (int i = first + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&bins[(sort_key<FIRST>(s, there, i) >> shift) & (n_bins - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < n_bins; i += kSortThreads) counts[(int64_t)blockIdx.x * n_bins + i] = bins[i];
}

// counts -> the counts of the tiles before, and the bins' totals: 64 bins per workgroup, a sixteenth of the tiles for each of its waves.
__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(int n_bins, int tiles, uint32_t *__restrict__ counts, uint32_t *__restrict__ totals, Clearing clearing) {
    constexpr int kWaves = kSortThreads / 64;
    __shared__ uint32_t sums[kWaves][64];
    const int own = (n_bins + 63) / 64;
    if ((int)blockIdx.x >= own) return clear_share(clearing, clearing.from + blockIdx.x - own);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bin = blockIdx.x * 64 + lane;
    const int each = (tiles + kWaves - 1) / kWaves, first = wave * each, end = first + each < tiles ? first + each : tiles;
    uint32_t sum = 0;
    if (bin < n_bins) {
#pragma unroll 8
        for (int t = first; t < end; ++t) sum += counts[(int64_t)t * n_bins + bin];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (bin >= n_bins) return;
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += sums[w][lane];
        total += sums[w][lane];
    }
    for (int t = first; t < end; ++t) {
        const uint32_t c = counts[(int64_t)t * n_bins + bin];
        counts[(int64_t)t * n_bins + bin] = before;
        before += c;
    }
    if (wave == 0) totals[bin] = total;
}

// Every key and position to its place.  A wave has a sixteenth of the tile in order; equal digits of a wave's 64 keys are ranked by ballots.
// totals: null where nobody has scanned the counts.  Up to kFewTiles tiles a workgroup adds its bins' counts itself, in less time than a launch takes
// (64 tiles, 131072 rows: 64 us, with a launch 69; 79 tiles of 4096, 322248 rows: 102 and 92).
constexpr int kFewTiles = 64;
template <bool FIRST, int TILE>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortSource s, int shift, int bits, int tiles, const uint32_t *__restrict__ counts,
                                                                  const uint32_t *__restrict__ totals, uint32_t *__restrict__ keys, uint32_t *__restrict__ positions,
                                                                  Clearing clearing) {
    constexpr int kWaves = kSortThreads / 64, kMine = TILE / kWaves, kRounds = kMine / 64;
    __shared__ uint32_t next[kWaves][1 << kEmMostBits];
    __shared__ uint32_t wave_totals[kWaves];
    if ((int)blockIdx.x >= tiles) return clear_share(clearing, clearing.from + blockIdx.x - tiles);
    const int n_bins = 1 << bits, mask = n_bins - 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t there = FIRST ? rows_there(s.offsets, s.B, s.rows) : 0;
    for (int i = threadIdx.x; i < n_bins * kWaves; i += kSortThreads) next[i >> bits][i & mask] = 0;
    const int first = (int)blockIdx.x * TILE + wave * kMine;
    uint32_t key[kRounds], position[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = first + r * 64 + lane;
        key[r] = i < s.rows ? sort_key<FIRST>(s, there, i) : 0;
        position[r] = FIRST ? (uint32_t)i : i < s.rows ? s.positions[i] : 0;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (first + r * 64 + lane < s.rows) atomicAdd(&next[wave][(key[r] >> shift) & mask], 1u);
    __syncthreads();
    // a thread per bin: what the waves have of it, then where the bin starts: behind the bins before it
    static_assert(1 << kEmMostBits <= kSortThreads, "a thread per bin");
    const int bin = threadIdx.x;
    uint32_t here = 0, before = 0, total = 0;
    if (bin < n_bins) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) here += next[w][bin];
        if (totals) {
            before = counts[(int64_t)blockIdx.x * n_bins + bin];
            total = totals[bin];
        } else if (tiles == 1) total = here;
        else {
#pragma unroll 16
            for (int t = 0; t < tiles; ++t) {
                const uint32_t c = counts[(int64_t)t * n_bins + bin];
                total += c;
                before += t < (int)blockIdx.x ? c : 0;
            }
        }
    }
    uint32_t sum = total;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(sum, d, 64);
        if (lane >= d) sum += y;
    }
    if (lane == 63) wave_totals[wave] = sum;
    __syncthreads();
    uint32_t at_bin = sum - total;
    for (int w = 0; w < wave; ++w) at_bin += wave_totals[w];
    if (bin < n_bins) {
        at_bin += before;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = next[w][bin];
            next[w][bin] = at_bin;
            at_bin += c;
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
            positions[base + before] = position[r];
        }
    }
}

// ---- sums of rows ----
// Block k: sorted positions kEmBlock k up to the next block's (or the end).  An id whose positions are all inside: its row of the table.  The sum of those that
// an earlier block's last id has in this one: heads[k]; of those of the last id, where it begins in this block and goes on in the next: tails[k].
template <typename T, bool EVEN, int LANES>
__global__ __launch_bounds__(kEmThreads) void block_sums_kernel(const T *__restrict__ dout, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ positions, int rows,
                                                                int n_blocks, uint32_t V, int64_t N, float scale, T *__restrict__ dtable, float *__restrict__ heads,
                                                                float *__restrict__ tails) {
    constexpr int kAhead = 8, VEC = kRowVec<T>;
    typedef RowRaw<T, VEC> Raw;
    const int k = blockIdx.x * (kEmThreads / LANES) + threadIdx.x / LANES, lane = threadIdx.x % LANES;
    if (k >= n_blocks) return;
    const int first = k * kEmBlock, end = rows - first < kEmBlock ? rows : first + kEmBlock;
    const uint32_t before = first > 0 ? keys[first - 1] : ~0u, after = end < rows ? keys[end] : ~0u;   // (no key is that large)
    // the block's keys and positions, kEach of them with every lane: read once, so that nothing but the rows themselves is waited for below
    constexpr int kEach = LANES < kEmBlock ? kEmBlock / LANES : 1;
    uint32_t my_key[kEach], my_position[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = first + i * LANES + lane < end ? first + i * LANES + lane : end - 1;
        my_key[i] = keys[r];
        my_position[i] = my_key[i] < V ? positions[r] : ~0u;   // a row that nobody adds (it may not be there) is not read
    }
    const auto of = [&](const uint32_t (&x)[kEach], int r) { return (uint32_t)__shfl((int)x[r / LANES], r % LANES, LANES); };   // r: a constant
    for (int64_t own = lane * VEC; own - lane * VEC < N; own += LANES * VEC) {   // (every lane takes part in the exchanges)
        const bool mine = own < N;
        const int64_t c = vec_at<VEC, EVEN>(own, N);
        Raw row[2][kAhead];
        auto read = [&](int from, int buffer) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t at = of(my_position, from + u);
                row[buffer][u] = mine && at != ~0u ? read_vec<T, VEC, EVEN>(dout + (int64_t)at * N + c, N - c) : Raw{};
            }
        };
        float sum[VEC];
        uint32_t current = of(my_key, 0);
        bool began = current != before;   // inside this block
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        auto row_is_done = [&]() {
            if (!mine) return;
            if (!began) store_vec<float, VEC, EVEN>(heads + (int64_t)k * N + c, N - c, sum);
            else if (current < V) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] *= scale;
                store_vec<T, VEC, EVEN>(dtable + (int64_t)current * N + c, N - c, sum);
            }
        };
        read(0, 0);
#pragma unroll
        for (int batch = 0; batch < kEmBlock / kAhead; ++batch) {
            if (first + batch * kAhead >= end) break;
            if (batch + 1 < kEmBlock / kAhead) read((batch + 1) * kAhead, (batch + 1) & 1);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const uint32_t key = of(my_key, batch * kAhead + u);
                if (first + batch * kAhead + u >= end) break;
                if (key != current) {
                    row_is_done();
                    current = key;
                    began = true;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
                }
                const Raw x = row[batch & 1][u];
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += (float)x[e];
            }
        }
        if (!began || current != after) row_is_done();
        else if (mine) store_vec<float, VEC, EVEN>(tails + (int64_t)k * N + c, N - c, sum);
    }
}

// Adds rows from .. to - 1 of `src`, kAhead loads in flight.
template <int VEC, bool EVEN> __device__ inline void add_rows(const float *src, int64_t N, int64_t c, int from, int to, float (&sum)[VEC]) {
    constexpr int kAhead = 8;
    for (int r = from; r < to; r += kAhead) {
        float x[kAhead][VEC];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (r + u < to) load_vec<float, VEC, EVEN>(src + (int64_t)(r + u) * N + c, N - c, x[u]);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (r + u < to) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += x[u][e];
            }
    }
}

// The sum of what the kPer lane groups of a workgroup have each added, in their order, with the first of them; `slots`: VEC floats a thread.
template <int VEC, int LANES> __device__ inline void groups_sum(float (&sum)[VEC], float (*slots)[VEC]) {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < VEC; ++e) slots[threadIdx.x][e] = sum[e];
    __syncthreads();
    if (threadIdx.x < LANES)
        for (int g = 1; g < kEmThreads / LANES; ++g)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] += slots[g * LANES + threadIdx.x][e];
}

// supers[k]: the sum of heads kEmSuper k .. kEmSuper (k + 1) - 1, where one id has all of their positions and began earlier.  A workgroup each.
template <int VEC, bool EVEN, int LANES>
__global__ __launch_bounds__(kEmThreads) void super_sums_kernel(const uint32_t *__restrict__ keys, uint32_t V, int64_t N, const float *__restrict__ heads,
                                                                float *__restrict__ supers) {
    constexpr int kPer = kEmThreads / LANES, kEach = kEmSuper > kPer ? kEmSuper / kPer : 1;   // heads of a lane group
    __shared__ float slots[kEmThreads][VEC];
    const int k = blockIdx.x, group = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const int64_t first = (int64_t)k * kEmSuper * kEmBlock;
    const uint32_t key = keys[first];
    if (key >= V || keys[first + kEmSuper * kEmBlock - 1] != key || first == 0 || keys[first - 1] != key) return;
    for (int64_t own = lane * VEC; own - lane * VEC < N; own += LANES * VEC) {
        const int64_t c = vec_at<VEC, EVEN>(own, N);
        float sum[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
        if (own < N && group * kEach < kEmSuper) add_rows<VEC, EVEN>(heads, N, c, k * kEmSuper + group * kEach, k * kEmSuper + (group + 1) * kEach, sum);
        groups_sum<VEC, LANES>(sum, slots);
        if (group == 0 && own < N) store_vec<float, VEC, EVEN>(supers + (int64_t)k * N + c, N - c, sum);
    }
}

// The rows of ids that begin in one block and end in another.  A workgroup has a block for each of its groups of LANES lanes; ids with more
// than kFewHeads heads are added by all of them together.
template <typename T, bool EVEN, int LANES>
__global__ __launch_bounds__(kEmThreads) void join_blocks_kernel(const uint32_t *__restrict__ keys, int n_blocks, uint32_t V, int64_t N, float scale,
                                                                 const float *__restrict__ heads, const float *__restrict__ tails, const float *__restrict__ supers,
                                                                 T *__restrict__ dtable) {
    constexpr int kPer = kEmThreads / LANES, kFewHeads = 16, VEC = kRowVec<T>;
    __shared__ float slots[kEmThreads][VEC];
    __shared__ int long_block[kPer], long_last[kPer];
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, k = blockIdx.x * kPer + group;
    const int64_t next = (int64_t)(k + 1) * kEmBlock;
    uint32_t key = V;
    if (k + 1 < n_blocks) {   // (the last block's ids end in it)
        key = keys[next - 1];
        if (key < V && (keys[next] != key || (k > 0 && keys[next - kEmBlock - 1] == key))) key = V;
    }
    int last = k;   // the last block whose first position is the id's: block k + 1 is one, and then LANES blocks are looked at at a time
    if (key < V) {
        last = k + 1;
        int step = 1;
        for (;;) {
            const int64_t probe = (int64_t)last + (int64_t)(lane + 1) * step;
            const bool is = probe < n_blocks && keys[probe * kEmBlock] == key;   // true for a prefix of the lanes
            const uint64_t votes = __builtin_amdgcn_ballot_w64(is) >> ((threadIdx.x & 63) / LANES * LANES);
            const int hits = __popcll(LANES == 64 ? votes : votes & ((1ull << (LANES & 63)) - 1));
            last += hits * step;
            if (hits == LANES) step *= LANES;        // the end is farther away
            else if (step > 1) step /= LANES;        // it is less than a step away
            else break;
        }
    }
    const bool many = last - k > kFewHeads;
    if (lane == 0) {
        long_block[group] = many ? k : -1;
        long_last[group] = last;
    }
    __syncthreads();
    if (key < V && !many)
        for (int64_t own = lane * VEC; own < N; own += LANES * VEC) {
            const int64_t c = vec_at<VEC, EVEN>(own, N);
            float sum[VEC];
            load_vec<float, VEC, EVEN>(tails + (int64_t)k * N + c, N - c, sum);
            add_rows<VEC, EVEN>(heads, N, c, k + 1, last + 1, sum);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] *= scale;
            store_vec<T, VEC, EVEN>(dtable + (int64_t)key * N + c, N - c, sum);
        }
    for (int g = 0; g < kPer; ++g) {
        const int b = long_block[g], end = long_last[g];
        if (b < 0) continue;
        // heads b + 1 .. end; those of whole supers in front of block `end` (whose positions need not all be the id's) come from there
        const int super0 = (b + 1 + kEmSuper - 1) / kEmSuper, super1 = end / kEmSuper;
        const bool any = super0 < super1;
        const int head1 = any ? super0 * kEmSuper : end + 1;   // heads b + 1 .. head1 - 1, then supers, then heads super1 * kEmSuper .. end
        const uint32_t id = keys[(int64_t)(b + 1) * kEmBlock];
        for (int64_t own = lane * VEC; own - lane * VEC < N; own += LANES * VEC) {
            const int64_t c = vec_at<VEC, EVEN>(own, N);
            float sum[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] = 0.0f;
            if (own < N) {
                const auto part = [&](const float *src, int from, int to) {   // this group's
                    const int each = (to - from + kPer - 1) / kPer, mine = from + group * each;
                    add_rows<VEC, EVEN>(src, N, c, mine, mine + each < to ? mine + each : to, sum);
                };
                if (group == 0) load_vec<float, VEC, EVEN>(tails + (int64_t)b * N + c, N - c, sum);
                part(heads, b + 1, head1);
                if (any) {
                    part(supers, super0, super1);
                    part(heads, super1 * kEmSuper, end + 1);
                }
            }
            groups_sum<VEC, LANES>(sum, slots);
            if (group == 0 && own < N) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] *= scale;
                store_vec<T, VEC, EVEN>(dtable + (int64_t)id * N + c, N - c, sum);
            }
        }
    }
}

template <typename T, typename Launch> hipError_t em_spread(int64_t N, bool aligned, Launch launch) {
    constexpr int kVec = kRowVec<T>;
    const auto with = [&](auto even) {
        const int64_t vectors = (N + kVec - 1) / kVec;
        using std::integral_constant;
        if (vectors <= 4) return launch(even, integral_constant<int, 4>{});
        if (vectors <= 8) return launch(even, integral_constant<int, 8>{});
        if (vectors <= 16) return launch(even, integral_constant<int, 16>{});
        if (vectors <= 32) return launch(even, integral_constant<int, 32>{});
        return launch(even, integral_constant<int, 64>{});
    };
    return aligned && N % kVec == 0 ? with(std::true_type{}) : with(std::false_type{});
}

template <typename T, typename Id>
hipError_t embedding_t(const T *table, const Id *ids, const int64_t *offsets, int64_t B, int64_t rows, int64_t V, int64_t N, float scale, T *out, hipStream_t stream) {
    return em_spread<T>(N, aligned16(table, out), [&](auto even, auto lanes) {
        constexpr bool EVEN = decltype(even)::value;
        constexpr int L = decltype(lanes)::value, kRows = kEmThreads / L * kInFlight;
        const int64_t need = (rows + kRows - 1) / kRows;
        const dim3 grid((unsigned)(need < 16384 ? need : 16384)), threads(kEmThreads);
        if (rows * N * (int64_t)sizeof(T) > kL2Bytes)
            hipLaunchKernelGGL((embedding_kernel<T, Id, EVEN, L, true>), grid, threads, 0, stream, table, ids, offsets, B, rows, V, N, scale, out);
        else
            hipLaunchKernelGGL((embedding_kernel<T, Id, EVEN, L, false>), grid, threads, 0, stream, table, ids, offsets, B, rows, V, N, scale, out);
        return hipGetLastError();
    });
}

// The workspace's parts, in 4-byte words from its start.
struct EmPlan {
    int bits, passes, tile, tiles;
    int n_blocks, n_supers;
    int64_t counts, totals, keys[2], positions[2], heads, tails, supers, words;
};
EmPlan em_plan(int64_t rows, int64_t V, int64_t N) {
    EmPlan p;
    // One tile where they fit (2000 rows: 24.4 us with a tile of 2048, 27.7 with two of 1024); up to kFewTiles tiles small ones, which put more compute units to work (20000 rows,
    // 1024, 2048 and 4096: 34.5, 39.8 and 44.0 us; 322248: 92, 87 and 92); many rows large ones, with fewer counts (2000000: 222, 198 and 184).
    p.tile = rows <= 1024 ? 1024 : rows <= 2048 ? 2048 : rows <= kFewTiles * 1024 ? 1024 : rows <= 1 << 19 ? 2048 : 4096;
    int bits = 1;
    while (((int64_t)1 << bits) < V + 1) ++bits;   // keys 0 .. V
    p.passes = (bits + kEmMostBits - 1) / kEmMostBits;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = (int)((rows + p.tile - 1) / p.tile);
    p.n_blocks = (int)((rows + kEmBlock - 1) / kEmBlock);
    p.n_supers = (int)(rows / (kEmBlock * kEmSuper));
    int64_t at = 0;
    const auto take = [&](int64_t words) { const int64_t here = at; at += (words + 3) / 4 * 4; return here; };
    p.counts = take((int64_t)p.tiles << p.bits);
    p.totals = take((int64_t)1 << p.bits);
    for (int i = 0; i < 2; ++i) { p.keys[i] = take(rows); p.positions[i] = take(rows); }
    p.heads = take(p.n_blocks * N);
    p.tails = take(p.n_blocks * N);
    p.supers = take(p.n_supers * N);
    p.words = at;
    return p;
}

template <typename T>
hipError_t embedding_backward_t(const T *dout, const void *ids, bool ids64, const int64_t *offsets, int64_t B, int64_t rows, int64_t V, int64_t N, float scale,
                                T *dtable, uint32_t *ws, hipStream_t stream) {
    const EmPlan p = em_plan(rows, V, N);
    const dim3 threads(kSortThreads);
    const bool scan = p.tiles > kFewTiles;
    uint32_t *const counts = ws + p.counts, *const totals = scan ? ws + p.totals : nullptr;
    SortSource s{ids, nullptr, nullptr, offsets, B, V, (int)rows, ids64};
    // every launch of the sort clears a share of the table
    const int64_t table_bytes = V * N * (int64_t)sizeof(T), units = (table_bytes + kClearBytes - 1) / kClearBytes;
    const int launches = p.passes * (scan ? 3 : p.tiles > 1 ? 2 : 1);
    int launch = 0;
    const auto share = [&]() {
        const Clearing c{(char *)dtable, table_bytes, units * launch / launches, units * (launch + 1) / launches};
        ++launch;
        return c;
    };
    const auto grid = [](int own, const Clearing &c) { return dim3((unsigned)(own + c.to - c.from)); };
    if (rows == 0) {
        const Clearing c{(char *)dtable, table_bytes, 0, units};
        hipLaunchKernelGGL((sort_count_kernel<true, 1024>), grid(0, c), threads, 0, stream, s, 0, 1, 0, nullptr, c);
        return hipGetLastError();
    }
    const auto pass = [&](auto first, auto tile, int number) {
        constexpr bool FIRST = decltype(first)::value;
        constexpr int TILE = decltype(tile)::value;
        uint32_t *const keys = ws + p.keys[number & 1], *const positions = ws + p.positions[number & 1];
        const int shift = number * p.bits, bins = 1 << p.bits;
        if (p.tiles > 1) {
            const Clearing c = share();
            hipLaunchKernelGGL((sort_count_kernel<FIRST, TILE>), grid(p.tiles, c), threads, 0, stream, s, shift, p.bits, p.tiles, counts, c);
        }
        if (scan) {
            const Clearing c = share();
            hipLaunchKernelGGL(sort_scan_kernel, grid((bins + 63) / 64, c), threads, 0, stream, bins, p.tiles, counts, totals, c);
        }
        const Clearing c = share();
        hipLaunchKernelGGL((sort_place_kernel<FIRST, TILE>), grid(p.tiles, c), threads, 0, stream, s, shift, p.bits, p.tiles, counts, totals, keys, positions, c);
        s.keys = keys;
        s.positions = positions;
    };
    const auto sort = [&](auto tile) {
        pass(std::true_type{}, tile, 0);
        for (int number = 1; number < p.passes; ++number) pass(std::false_type{}, tile, number);
    };
    if (p.tile == 1024) sort(std::integral_constant<int, 1024>{});
    else if (p.tile == 2048) sort(std::integral_constant<int, 2048>{});
    else sort(std::integral_constant<int, 4096>{});
    float *const heads = reinterpret_cast<float *>(ws + p.heads), *const tails = reinterpret_cast<float *>(ws + p.tails), *const supers = reinterpret_cast<float *>(ws + p.supers);
    return em_spread<T>(N, aligned16(dout, dtable), [&](auto even, auto lanes) {
        constexpr bool EVEN = decltype(even)::value;
        constexpr int L = decltype(lanes)::value, kPer = kEmThreads / L;
        const dim3 blocks((p.n_blocks + kPer - 1) / kPer), few(kEmThreads);
        hipLaunchKernelGGL((block_sums_kernel<T, EVEN, L>), blocks, few, 0, stream, dout, s.keys, s.positions, (int)rows, p.n_blocks, (uint32_t)V, N, scale, dtable, heads, tails);
        if (p.n_supers)
            hipLaunchKernelGGL((super_sums_kernel<kRowVec<T>, EVEN, L>), dim3(p.n_supers), few, 0, stream, s.keys, (uint32_t)V, N, heads, supers);
        if (p.n_blocks > 1)
            hipLaunchKernelGGL((join_blocks_kernel<T, EVEN, L>), blocks, few, 0, stream, s.keys, p.n_blocks, (uint32_t)V, N, scale, heads, tails, supers, dtable);
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
