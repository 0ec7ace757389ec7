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
#include "jfa_lds.h"
#include "jfa_mfma.h"

namespace jfa {

namespace {

typedef __attribute__((ext_vector_type(8))) float f32x8;

// A tile in LDS: kRows rows without padding, in 16-byte chunks, as the copies from memory leave them.  The chunks of a row are in another order in every
// row, chunk c at place c ^ swizzle(row), so that neither 16 rows' same chunk nor four consecutive rows' same 64 bytes meet in a bank.
template <int kChunks> __host__ __device__ constexpr int swizzle(int row) {
    return kChunks >= 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : kChunks == 8 ? (((row >> 1) & 1) << 2) | ((row >> 2) & 3) : (row >> 2) & 3;
}

// The two element types.  An operand holds 16 contraction indices, eight per lane.
// rows(): the tile's rows along the lanes, contraction along its columns, slot e of a lane in half h = lane / 32 column 8 h + e of 16.
// cols(): its columns along the lanes, contraction along its rows, slot e row (e / 4) * 8 + 4 h + e % 4 of 16: the order in which an accumulator tile
// holds its rows, so that a tile of products of rows (P) is an operand as it stands.  PERMUTED: lane l has column l with bits 2 and 3 exchanged: what is
// accumulated over such a column (the state) is, as it stands, an operand in the order of rows().
__device__ inline int exchanged(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }
template <typename T> struct Elem;

template <> struct Elem<__bf16> {
    typedef bf16x8 Operand;
    static constexpr int kRows = 64, kSplit = 2;
    __device__ static f32x16 product(Operand a, Operand b, f32x16 c) { return mfma_32x32x16(a, b, c); }
    // what a lane adds to (or exchanges bits of) every address
    template <int D> __device__ static int rows_base(int lane) { return (lane & 31) * D * 2 + ((swizzle<D / 8>(lane & 31) ^ (lane >> 5)) << 4); }
    template <int D, bool PERMUTED> __device__ static int cols_base(int lane) {
        const int half = lane >> 5, row = 4 * half + ((lane & 15) >> 2), q = PERMUTED ? ((lane & 1) << 1) | ((lane >> 1) & 1) : lane & 3;
        return row * D * 2 + (((((lane >> 4) & 1) * 2 + (q >> 1)) ^ swizzle<D / 8>(row)) << 4) + (q & 1) * 8;
    }
    template <int D> __device__ static Operand rows(const char *tile, int base, int row0, int k0) { return lds_read_b128(tile + row0 * D * 2 + (base ^ (k0 * 2))); }
    template <int D> __device__ static Operand cols(const char *tile, int base, int col0, int k0) {
        const char *const p = tile + k0 * D * 2;
        const int at = base ^ (col0 * 2);
        return concat(lds_read_tr16(p + at), lds_read_tr16(p + 8 * D * 2 + (at ^ 32)));
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
    // x rounded; what is left of it stays in x
    __device__ static Operand take(f32x8 &x) {
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            bf16x2 pair;
            pair[0] = (__bf16)x[2 * e];
            pair[1] = (__bf16)x[2 * e + 1];
            w[e] = __builtin_bit_cast(uint32_t, pair);
            asm("" : "+v"(w[e]));   // (else every second element is rounded once more to have it in a register's upper half)
            x[2 * e] -= __builtin_bit_cast(float, w[e] << 16);
            x[2 * e + 1] -= __builtin_bit_cast(float, w[e] & 0xffff0000u);
        }
        return __builtin_bit_cast(Operand, w);
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
    static constexpr int kRows = 32, kSplit = 1;
    __device__ static f32x16 product(Operand a, Operand b, f32x16 c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    template <int D> __device__ static int rows_base(int lane) { return (lane & 31) * D * 4 + ((swizzle<D / 4>(lane & 31) ^ ((lane >> 5) * 2)) << 4); }
    template <int D, bool PERMUTED> __device__ static int cols_base(int lane) {
        const int half = lane >> 5, col = PERMUTED ? exchanged(lane & 31) : lane & 31;
        return 4 * half * D * 4 + (((col >> 2) ^ swizzle<D / 4>(4 * half)) << 4) + (col & 3) * 4;
    }
    template <int D> __device__ static Operand rows(const char *tile, int base, int row0, int k0) {
        const char *const p = tile + row0 * D * 4;
        const f32x4 lo = *reinterpret_cast<const f32x4 *>(p + (base ^ (k0 * 4))), hi = *reinterpret_cast<const f32x4 *>(p + (base ^ (k0 * 4 + 16)));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    template <int D> __device__ static Operand cols(const char *tile, int base, int col0, int k0) {
        Operand r;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int row = (e >> 2) * 8 + (e & 3);
            r[e] = *reinterpret_cast<const float *>(tile + (k0 + row) * D * 4 + (base ^ (col0 * 4) ^ (swizzle<D / 4>(row) << 4)));
        }
        return r;
    }
    __device__ static Operand pack(const f32x8 &x) { return x; }
    __device__ static f32x8 widen(Operand x) { return x; }
    __device__ static Operand take(f32x8 &x) { return x; }
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
// s_waitcnt for vector memory alone: at most `left` pending (the fields of the other counters at their maximum)
template <int left> constexpr int vmem_left() { return (left & 15) | ((left >> 4) << 14) | (7 << 4) | (15 << 8); }
constexpr int kNoVmem = vmem_left<0>();
__device__ inline float power(float log2_g, int n) { return fast_exp2(log2_g * (float)n); }   // n >= 0

// Where the states between a sample's segments start, in states: a sample that begins in row r has at most as many as there are multiples of
// segment_rows in its rows, so the r / segment_rows-th is its first, `between` of them in all for each walk and head.
__device__ inline int64_t state_between(int walk, int h, int H, int between, int64_t first, int segment_rows) { return ((int64_t)walk * H + h) * between + first / segment_rows; }

}  // namespace

// A workgroup takes one (sample, head, segment) through ROLES walks that go the same way over the same tensors: one of them, or the two that
// give dk and dv, which share the tiles of q and dout.  Each walk has D / 32 waves, each of which owns 32 columns of the state and of the outputs.
// Workgroups go to the eight dies in turn.  ROLES = 1: the `sides` walks of a (sample, head, segment) follow each other on one die, whose L2 then has the tensors that
// they share (1024 x 4 heads of up to 1024 rows, D = 128, three walks: 1518 -> 1370 us, 1024 samples of 64 rows 52 -> 40; one walk after another 1500).
// KS = 2 (one walk; D = 64, and fp32 at D = 128): twice as many waves, two to a strip of 32 columns with half of the state's rows each; out is summed over
// the two halves through LDS.  Where few walks run, what a chunk takes is the issue of one wave's instructions.  fp32: the fp32 matrix instructions,
// 64 clocks for 4096 products, are what a chunk waits for: 48 of them for a wave instead of 112 (D = 128: 80 of 208); there P, too, is a sum over the waves, a
// contraction step of 16 of each (a sample of 256 rows, D = 64, 34 -> 25 us).  bf16, D = 64: 16 samples of 600 rows 28.8 -> 24.4 us, 1024 94.9 -> 78.6;
// at D = 128 the four waves fill the SIMDs: 16 samples 34.8 and 34.3 us, 1024 158 and 177.
// bf16: what is rounded in front of a product (P, the state as a factor of out, the decayed rows of C) is split into two bf16 numbers, 16 bits in
// all, so that a result's error is its own rounding; kParts = 3, exact, for the decayed rows where the state is itself a result.  One bf16 number each
// would be 1.65 times that error (root mean square), and at D = 128 save 6 % of the forward and 12 % of the backward (2048 samples of 600 rows 299 -> 280 us and
// 848 -> 738), the state's alone half of both.
// kStateOnly: the state that a segment adds to, for those with a segment after them, into `carried`.
template <typename T, int D, int ROLES, int KS, int kParts, bool kStateOnly>
__global__ __launch_bounds__(2 * D * ROLES * KS, 2) void linear_walk_kernel(LinearWalks walks, const float *__restrict__ log_decay, const int64_t *__restrict__ offsets,
                                                                       const int32_t *__restrict__ order, int B, int H, int segments, int segment_rows, int between,
                                                                       int sides, float *__restrict__ carried) {
    typedef Elem<T> E;
    typedef typename E::Operand Operand;
    constexpr int kRows = E::kRows, kSize = (int)sizeof(T), kStateTiles = D / 32, kSteps = D / 16, kSplit = E::kSplit;
    constexpr int kWalkWaves = kStateTiles * KS, kWaves = kWalkWaves * ROLES, kMine = kStateTiles / KS;   // kMine: state tiles of a wave
    constexpr int kTiles = kRows / 32, kPTiles = kTiles * (kTiles + 1) / 2;
    constexpr int kChunks = D * kSize / 16, kTileBytes = kRows * kChunks * 16, kLoads = kRows * kChunks / (64 * kWaves);   // 16-byte chunks of a row; copies of a tile per wave
    // Places of tiles.  A is free for the next chunk's once the state's product with it is done, in the middle of a chunk.  B and, of two walks, C (their B
    // and C change places) are read to the end: there are two of each, the next chunk's fetched from the start of a chunk on.  One walk's C is fetched when the
    // chunk before is done, which is in time for the products with it.  So two workgroups have room on a compute unit.
    constexpr int kPlaces = ROLES == 2 ? 6 : 4;
    // P: its tiles are shared out among a walk's waves, which leave them as operands, 16 bytes per lane; a single wave (and the fp32 kernels, whose P is
    // one tile) has it in registers.
    constexpr bool kShareP = !kStateOnly && kPTiles > 1 && kStateTiles > 1;
    constexpr int kPBytes = kShareP ? kPTiles * 2 * kSplit * 1024 : 0;
    constexpr bool kSumP = KS > 1 && kTiles == 1;
    static_assert(KS == 1 || ROLES == 1, "");
    static_assert(!kSumP || kSteps == kWalkWaves, "a step of P's contraction for each wave");
    constexpr int kHalf = kTiles == 1 ? 2 : 4;   // kilobytes of the half of out that a wave gives away
    constexpr int kXBytes = KS > 1 && !kStateOnly ? kWalkWaves * ((kSumP ? 4 : 0) + kHalf) * 1024 : 0;   // a wave's part of P, half of its part of out
    __shared__ __attribute__((aligned(16))) char lds[kPlaces * kTileBytes + ROLES * (kPBytes + kXBytes)];
    __shared__ float powers[ROLES][2][2 * kRows];

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int role = wave / kWalkWaves, walk_wave = wave % kWalkWaves, strip = walk_wave % kStateTiles, part = walk_wave / kStateTiles;
    const int col = lane & 31, half = lane >> 5;
    const int which = ROLES == 2 ? 1 : (int)(blockIdx.x / 8) % sides + (int)blockIdx.y;   // the first role's walk
    const LinearWalk &walk = walks.walk[which + role];
    const int block = ROLES == 2 ? (int)blockIdx.x : (int)(blockIdx.x / (8 * sides)) * 8 + (int)(blockIdx.x % 8);
    // Heads that share 128-byte lines are for one die, whose L2 reads a line once (600 rows x 512 x 4, D = 32: 103 -> 67 us).
    constexpr bool kSameDie = D * sizeof(T) < 128;
    const int at = kSameDie ? block / (8 * H) * 8 + block % 8 : block / H, h = kSameDie ? block / 8 % H : block % H;
    const int at_sample = at / segments, segment = at - at_sample * segments;
    if (at_sample >= B) return;
    const int b = order ? order[at_sample] : at_sample, pair = b * H + h;
    const int64_t first = offsets[b];
    const int64_t L = offsets[b + 1] - first;
    const int64_t t0 = (int64_t)segment * segment_rows;   // rows are counted in the order of the walk
    const bool last = t0 + segment_rows >= L;
    if (kStateOnly ? last || segment == segments - 1 : (t0 >= L && segment > 0)) return;
    if (segments > 1 && first / segment_rows + segment + (kStateOnly ? 1 : 0) > between) return;   // (more rows than the caller said there were)
    const int64_t left = L - t0;
    const int n = (int)(left < segment_rows ? left : segment_rows);   // rows of this segment; 0 for an empty sample
    const bool reverse = walk.reverse;
    const float lg = log2_decay(log_decay[h]);
    float *const passed = carried + state_between(walk.carried, h, H, between, first, segment_rows) * D * D;
    float *const state_out = kStateOnly ? passed + (int64_t)segment * D * D : last && walk.state_out ? walk.state_out + (int64_t)pair * D * D : nullptr;

    f32x16 S[kMine];   // tile m: rows 32 (kMine part + m) .. (dimension of B), columns 32 strip .. (dimension of C)
#pragma unroll
    for (int m = 0; m < kMine; ++m)
#pragma unroll
        for (int v = 0; v < 16; ++v) S[m][v] = 0.0f;
    if (!kStateOnly) {
        const float *from = segment > 0 ? passed + (int64_t)(segment - 1) * D * D : walk.state_in ? walk.state_in + (int64_t)pair * D * D : nullptr;
        if (from) {
            const bool transposed = segment == 0 ? walk.transposed : walk.carried_transposed;
#pragma unroll
            for (int m = 0; m < kMine; ++m)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int r = (part * kMine + m) * 32 + exchanged(acc_row(v, half)), c = strip * 32 + col;
                    S[m][v] = from[transposed ? c * D + r : r * D + c];
                }
        }
    }

    // Row t of the walk is row first + t, or first + L - 1 - t, of the tensors.  A chunk's rows are kRows rows from `low` on (where it is
    // the last and walked backwards, its first ones lie in front of the sample and are not touched): 32-bit offsets from there.
    const uint32_t row_bytes = (uint32_t)H * D * kSize;
    int64_t low = ((first + (reverse ? L - t0 - kRows : t0)) * H + h) * D;
    const int64_t low_step = (reverse ? -(int64_t)kRows : (int64_t)kRows) * H * D;
    const T *const a0 = (const T *)walks.walk[which].a, *const a1 = (const T *)walks.walk[ROLES == 2 ? 2 : which].a;
    const T *const b0 = (const T *)walks.walk[which].b, *const c0 = (const T *)walks.walk[which].c;
    // The rows from `rows` on are not there: the last one takes their place.  Whatever it is, P's mask and the decayed rows' zeros keep it out.
    auto offset_of = [&](int u, int rows) {
        const int at = (u * kWaves + wave) * 64 + lane, t = at / kChunks, c = at % kChunks ^ swizzle<kChunks>(t), there = t < rows ? t : rows - 1;
        return (uint32_t)(reverse ? kRows - 1 - there : there) * row_bytes + c * 16;
    };
    uint32_t offsets_of_all[kLoads];   // of a whole chunk
#pragma unroll
    for (int u = 0; u < kLoads; ++u) offsets_of_all[u] = offset_of(u, kRows);
    auto copy = [&](const T *tensor, int64_t from, int rows, int place) {
        const T *const base = reinterpret_cast<const T *>(uniform64((int64_t)(tensor + from)));
        char *const dst = lds + place * kTileBytes + wave * 1024;
        if (rows >= kRows) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) bd_dma16(base, offsets_of_all[u], dst + u * kWaves * 1024);
        } else {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) bd_dma16(base, offset_of(u, rows), dst + u * kWaves * 1024);
        }
    };
    const int row_base = E::template rows_base<D>(lane), col_base = E::template cols_base<D, false>(lane) ^ (strip * 32 * kSize), 
              col_base_b = E::template cols_base<D, true>(lane) ^ (part * kMine * 32 * kSize);

    // powers[0][kRows + x]: in_scale g^x, zero for negative x: P's factors.  powers[1]: with the decay after a chunk's last row, `tail`: the state's.
    const int tail = reverse ? 1 : 0;
    float (*const my_powers)[2 * kRows] = powers[role];
    for (int i = walk_wave * 64 + lane; i < 2 * 2 * kRows; i += 64 * kWalkWaves) {
        const int x = i % (2 * kRows) - kRows;
        my_powers[i / (2 * kRows)][x + kRows] = x < 0 ? 0.0f : walk.in_scale * power(lg, x + (i < 2 * kRows ? 0 : tail));
    }
    const float out_scale = walk.out_scale;
    float since[kTiles];
#pragma unroll
    for (int ti = 0; ti < kTiles; ++ti) since[ti] = power(lg, ti * 32 + col + 1 - tail);

    if (n > 0) {
        if constexpr (ROLES == 2) {
            copy(a0, low, n, 0);
            copy(a1, low, n, 1);
            copy(b0, low, n, 2);
            copy(c0, low, n, 4);
        } else {
            copy(b0, low, n, 2);
            if (!kStateOnly) copy(a0, low, n, 0);
        }
    }
    for (int r0 = 0, turn = 0; r0 < n; r0 += kRows, low += low_step, turn ^= 1) {
        const int rows = n - r0 < kRows ? n - r0 : kRows;
        const bool more = r0 + kRows < n;
        __builtin_amdgcn_s_waitcnt(kNoVmem);
        __syncthreads();   // the tiles fetched so far are there, and the last chunk's are free
        if constexpr (ROLES == 2) {
            if (more) {
                copy(b0, low + low_step, n - r0 - kRows, 2 + (turn ^ 1));
                copy(c0, low + low_step, n - r0 - kRows, 4 + (turn ^ 1));
            }
        } else {
            copy(c0, low, n - r0, 1);
            if (more) copy(b0, low + low_step, n - r0 - kRows, 2 + (turn ^ 1));
        }
        // One walk's C: its copies are the ones in front of the next B's.  (Stores have been waited for above.)
        auto c_is_there = [&]() {
            if constexpr (ROLES == 1) {
                if (more) __builtin_amdgcn_s_waitcnt(vmem_left<kLoads>());
                else __builtin_amdgcn_s_waitcnt(kNoVmem);
            }
            __syncthreads();   // P is there, too, and A is free
        };
        const char *const at = lds + role * kTileBytes;
        const char *const bt = lds + (ROLES == 2 ? 2 + 2 * role + turn : 2 + turn) * kTileBytes, *const ct = lds + (ROLES == 2 ? 4 - 2 * role + turn : 1) * kTileBytes;
        char *const pt = lds + kPlaces * kTileBytes + role * kPBytes;
        char *const px = lds + kPlaces * kTileBytes + ROLES * kPBytes, *const ox = px + (kSumP ? kWalkWaves * 4096 : 0);   // KS > 1
        Operand c[2 * kTiles];   // the chunk's rows of C, this wave's columns
        if (kStateOnly) {
            c_is_there();
#pragma unroll
            for (int k = 0; k < 2 * kTiles; ++k) c[k] = E::template cols<D>(ct, col_base, 0, k * 16);
        }
        if (!kStateOnly) {
            // P^T, tiles (rows j of B) x (columns i of A), zero above the diagonal
            Operand P[kShareP || kSumP ? 1 : kPTiles][2][kSplit];
            const float *const near = my_powers[0] + kRows + col - 4 * half;   // [-(8 g + e)]: g^(i - j)
            auto weighted = [&](f32x16 &p, int t, auto &&put) {   // t: 0, 2 on the diagonal, 1 below it; put(contraction step, part, operand)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float weight = near[(t == 1 ? 32 : 0) - ((v >> 2) * 8 + (v & 3))];
                    p[v] = t != 1 && col < acc_row(v, half) ? 0.0f : p[v] * weight;
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    f32x8 x = eight(p, k * 8);
#pragma unroll
                    for (int part = 0; part < kSplit; ++part) {
                        put(k, part, part + 1 < kSplit ? E::take(x) : E::pack(x));
                    }
                }
            };
            if constexpr (kSumP) {
                f32x16 p;
#pragma unroll
                for (int v = 0; v < 16; ++v) p[v] = 0.0f;
                const int base = row_base ^ (walk_wave * 16 * kSize);
                p = E::product(E::template rows<D>(bt, base, 0, 0), E::template rows<D>(at, base, 0, 0), p);
#pragma unroll
                for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4 *>(px + (walk_wave * 4 + g) * 1024 + lane * 16) = f32x4{p[4 * g], p[4 * g + 1], p[4 * g + 2], p[4 * g + 3]};
            } else if constexpr (kShareP) {
#pragma unroll
                for (int t = 0; t < kPTiles; ++t) {
                    if (t % kWalkWaves != walk_wave) continue;
                    // operands one step ahead of the products that use them: left alone, every read sits right in front of its product
                    Operand a[2], x[2];
                    auto read = [&](int ks) {
                        a[ks & 1] = E::template rows<D>(at, row_base, t > 0 ? 32 : 0, ks * 16);
                        x[ks & 1] = E::template rows<D>(bt, row_base, t > 1 ? 32 : 0, ks * 16);
                    };
                    f32x16 p;
#pragma unroll
                    for (int v = 0; v < 16; ++v) p[v] = 0.0f;
                    read(0);
#pragma unroll
                    for (int ks = 0; ks < kSteps; ++ks) {
                        if (ks + 1 < kSteps) read(ks + 1);
                        __builtin_amdgcn_sched_barrier(0);
                        p = E::product(x[ks & 1], a[ks & 1], p);
                    }
                    weighted(p, t, [&](int k, int part, const Operand &y) { *reinterpret_cast<Operand *>(pt + ((t * 2 + k) * kSplit + part) * 1024 + lane * 16) = y; });
                }
            } else {
                f32x16 p[kPTiles];
#pragma unroll
                for (int t = 0; t < kPTiles; ++t)
#pragma unroll
                    for (int v = 0; v < 16; ++v) p[t][v] = 0.0f;
                Operand a[2][kTiles], x[2][kTiles];
                auto read = [&](int ks) {
#pragma unroll
                    for (int ti = 0; ti < kTiles; ++ti) {
                        a[ks & 1][ti] = E::template rows<D>(at, row_base, ti * 32, ks * 16);
                        x[ks & 1][ti] = E::template rows<D>(bt, row_base, ti * 32, ks * 16);
                    }
                };
                read(0);
#pragma unroll
                for (int ks = 0; ks < kSteps; ++ks) {
                    if (ks + 1 < kSteps) read(ks + 1);
                    __builtin_amdgcn_sched_barrier(0);
                    p[0] = E::product(x[ks & 1][0], a[ks & 1][0], p[0]);
                    if constexpr (kTiles == 2) {
                        p[1] = E::product(x[ks & 1][0], a[ks & 1][1], p[1]);
                        p[2] = E::product(x[ks & 1][1], a[ks & 1][1], p[2]);
                    }
                }
#pragma unroll
                for (int t = 0; t < kPTiles; ++t) weighted(p[t], t, [&](int k, int part, const Operand &y) { P[t][k][part] = y; });
            }
            asm volatile("" ::: "memory");   // A's operands are read again: kept from above they would cost 64 registers
            // out^T = C^T P^T + g^(i + 1) S^T A^T, this wave's columns of C
            f32x16 o[kTiles];
#pragma unroll
            for (int ti = 0; ti < kTiles; ++ti)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[ti][v] = 0.0f;
            const int state_base = row_base ^ (part * (kSteps / KS) * 16 * kSize);   // from this wave's first row of the state on
            Operand a[2][kTiles];
            auto read = [&](int ks) {
#pragma unroll
                for (int ti = 0; ti < kTiles; ++ti) a[ks & 1][ti] = E::template rows<D>(at, state_base, ti * 32, ks * 16);
            };
            read(0);
#pragma unroll
            for (int ks = 0; ks < kSteps / KS; ++ks) {
                if (ks + 1 < kSteps / KS) read(ks + 1);
                __builtin_amdgcn_sched_barrier(0);
                f32x8 x = eight(S[ks >> 1], (ks & 1) * 8);
#pragma unroll
                for (int part = 0; part < kSplit; ++part) {
                    const Operand y = part + 1 < kSplit ? E::take(x) : E::pack(x);
#pragma unroll
                    for (int ti = 0; ti < kTiles; ++ti) o[ti] = E::product(y, a[ks & 1][ti], o[ti]);
                }
            }
            c_is_there();
            if (more) {
                copy(a0, low + low_step, n - r0 - kRows, 0);
                if constexpr (ROLES == 2) copy(a1, low + low_step, n - r0 - kRows, 1);
            }
#pragma unroll
            for (int k = 0; k < 2 * kTiles; ++k) c[k] = E::template cols<D>(ct, col_base, 0, k * 16);
#pragma unroll
            for (int ti = 0; ti < kTiles; ++ti)
#pragma unroll
                for (int v = 0; v < 16; ++v) o[ti][v] *= since[ti];
            if constexpr (kSumP) {
                // this wave's half of P's rows, summed over the waves, with the same rows of C; then its half of out's columns, summed over the two
                f32x8 x;
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWalkWaves; ++w) {
                    const f32x4 lo = *reinterpret_cast<const f32x4 *>(px + (w * 4 + 2 * part) * 1024 + lane * 16), hi = *reinterpret_cast<const f32x4 *>(px + (w * 4 + 2 * part + 1) * 1024 + lane * 16);
                    x += __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int row = part * 16 + (e >> 2) * 8 + (e & 3);
                    x[e] = col < row + 4 * half ? 0.0f : x[e] * near[-row];
                }
                o[0] = E::product(E::template cols<D>(ct + part * 16 * D * kSize, col_base, 0, 0), E::pack(x), o[0]);
                f32x8 mine = eight(o[0], 0), others = eight(o[0], 8);
                if (part) {
                    const f32x8 swapped = mine;
                    mine = others;
                    others = swapped;
                }
                *reinterpret_cast<f32x4 *>(ox + (walk_wave * 2) * 1024 + lane * 16) = f32x4{others[0], others[1], others[2], others[3]};
                *reinterpret_cast<f32x4 *>(ox + (walk_wave * 2 + 1) * 1024 + lane * 16) = f32x4{others[4], others[5], others[6], others[7]};
                __syncthreads();
                const int partner = strip + (1 - part) * kStateTiles;
                if (col < rows) {
                    char *const dst = reinterpret_cast<char *>((T *)walk.out + low) +
                                      ((uint32_t)(reverse ? kRows - 1 - col : col) * row_bytes + (uint32_t)(strip * 32 + part * 16 + half * 4) * kSize);
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const f32x4 y = *reinterpret_cast<const f32x4 *>(ox + (partner * 2 + g) * 1024 + lane * 16);
                        E::store4(reinterpret_cast<T *>(dst + g * 8 * kSize), f32x4{(mine[4 * g] + y[0]) * out_scale, (mine[4 * g + 1] + y[1]) * out_scale,
                                                                                   (mine[4 * g + 2] + y[2]) * out_scale, (mine[4 * g + 3] + y[3]) * out_scale});
                    }
                }
            } else {
                // (KS = 2: every second step of P's rows, and one of the two tiles of out's rows)
                const auto product_with_p = [&](int ks, const char *from) {
#pragma unroll
                    for (int half_p = 0; half_p < kSplit; ++half_p) {
                        const auto p = [&](int t) -> Operand {
                            if constexpr (kShareP) return *reinterpret_cast<const Operand *>(from + ((t * 2 + (ks & 1)) * kSplit + half_p) * 1024 + lane * 16);
                            else return P[t][ks & 1][half_p];
                        };
                        if (ks < 2) o[0] = E::product(c[ks], p(0), o[0]);
                        if constexpr (kTiles == 2) o[1] = E::product(c[ks], p(ks < 2 ? 1 : 2), o[1]);
                    }
                };
#pragma unroll
                for (int ks = 0; ks < 2 * kTiles; ++ks)
                    if (KS == 1 || (ks & 1) == part) product_with_p(ks, pt);
                char *const out = reinterpret_cast<char *>((T *)walk.out + low);
                auto store = [&](int ti, const f32x16 &o) {
                    const int r = ti * 32 + col;
                    if (r < rows) {
                        char *const dst = out + ((uint32_t)(reverse ? kRows - 1 - r : r) * row_bytes + (uint32_t)(strip * 32 + half * 4) * kSize);
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            E::store4(reinterpret_cast<T *>(dst + g * 8 * kSize), f32x4{o[4 * g] * out_scale, o[4 * g + 1] * out_scale, o[4 * g + 2] * out_scale, o[4 * g + 3] * out_scale});
                    }
                };
                if constexpr (KS > 1) {
                    f32x16 mine = part ? o[kTiles - 1] : o[0];
                    const f32x16 others = part ? o[0] : o[kTiles - 1];
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        *reinterpret_cast<f32x4 *>(ox + (walk_wave * 4 + g) * 1024 + lane * 16) = f32x4{others[4 * g], others[4 * g + 1], others[4 * g + 2], others[4 * g + 3]};
                    __syncthreads();
                    const int partner = strip + (1 - part) * kStateTiles;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 y = *reinterpret_cast<const f32x4 *>(ox + (partner * 4 + g) * 1024 + lane * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) mine[4 * g + e] += y[e];
                    }
                    store(part, mine);
                } else {
#pragma unroll
                    for (int ti = 0; ti < kTiles; ++ti) store(ti, o[ti]);
                }
            }
        }
        // S <- g^rows S + (g^(rows - 1 - i) B)^T C, unless nobody looks at it any more
        if (r0 + kRows < n || state_out) {
            const float decay = power(lg, rows);
#pragma unroll
            for (int m = 0; m < kMine; ++m)
#pragma unroll
                for (int v = 0; v < 16; ++v) S[m][v] *= decay;
            const float *const left = my_powers[1] + rows - 1 - 4 * half;   // of the chunk's row i: [kRows - i]; rows that are not there have zero
            Operand x[2][kMine];
            float weight[2][8];
            auto read = [&](int ks) {
#pragma unroll
                for (int e = 0; e < 8; ++e) weight[ks & 1][e] = left[kRows - (ks * 16 + (e >> 2) * 8 + (e & 3))];
#pragma unroll
                for (int m = 0; m < kMine; ++m) x[ks & 1][m] = E::template cols<D>(bt, col_base_b, m * 32, ks * 16);
            };
            read(0);
#pragma unroll
            for (int ks = 0; ks < kRows / 16; ++ks) {
                if (ks + 1 < kRows / 16) read(ks + 1);
                __builtin_amdgcn_sched_barrier(0);
                f32x8 y = E::widen(c[ks]);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= weight[ks & 1][e];
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    const Operand z = part + 1 < kParts ? E::take(y) : E::pack(y);
#pragma unroll
                    for (int m = 0; m < kMine; ++m) S[m] = E::product(x[ks & 1][m], z, S[m]);
                }
            }
        }
    }
    if (state_out) {
        const bool transposed = !kStateOnly && walk.transposed;
#pragma unroll
        for (int m = 0; m < kMine; ++m)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int r = (part * kMine + m) * 32 + exchanged(acc_row(v, half)), c = strip * 32 + col;
                state_out[transposed ? c * D + r : r * D + c] = S[m][v];
            }
    }
}

// carried[m] (what segment m adds) -> the state in front of segment m + 1, for every (walk, sample, head) and element.
__global__ __launch_bounds__(256) void linear_carry_kernel(LinearWalks walks, const float *__restrict__ log_decay, const int64_t *__restrict__ offsets,
                                                           int H, int D, int segments, int segment_rows, int between, float *__restrict__ carried) {
    const int blocks = D * D / 1024;   // 1024 elements, four per thread, per workgroup
    const int pair = blockIdx.x / blocks, at = (blockIdx.x - pair * blocks) * 1024 + threadIdx.x * 4;
    const LinearWalk &walk = walks.walk[blockIdx.y];
    const int b = pair / H;
    const int64_t L = offsets[b + 1] - offsets[b];
    const int64_t first = offsets[b], room = between - first / segment_rows;
    int64_t n = (L + segment_rows - 1) / segment_rows - 1;   // segments with one after them
    n = n < segments - 1 ? n : segments - 1;
    n = n < room ? n : room;
    if (n <= 0) return;
    const float decay = fast_exp2(log2_decay(log_decay[pair - b * H]) * (float)segment_rows);
    f32x4 S = {0.0f, 0.0f, 0.0f, 0.0f};
    if (walk.state_in) {
        const float *from = walk.state_in + (int64_t)pair * D * D;
        const int r = at / D, c = at % D;
#pragma unroll
        for (int e = 0; e < 4; ++e) S[e] = from[walk.transposed ? (c + e) * D + r : at + e];
    }
    f32x4 *x = reinterpret_cast<f32x4 *>(carried + state_between(walk.carried, pair - b * H, H, between, first, segment_rows) * D * D + at);
    const int64_t stride = (int64_t)D * D / 4;
    constexpr int kAhead = 32;   // states on their way at a time: a trip to memory for each 8 of them took 15 us for 63 (16 walks)
    for (int64_t m0 = 0; m0 < n; m0 += kAhead) {
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

// How a call is laid out.  A walk goes a chunk of 64 rows at a time, 3.5 us each (bf16, D = 128) where it has a compute unit to itself and 7 where two walks
// share it, by when the two have 4.5 TB/s of the memory.  So what takes longest is either all rows, W = rows * H / (2 * 256) of them for each place, or one
// long sample's walk.  A sample longer than that is cut into segments: a pass over k and v for the state that each of them adds, a scan, and the
// walks of all segments at once, at about 1.65 times W.  It pays where half the longest sample (alone on its compute unit at last) is longer than that and
// the two passes over a segment.  8 x 2 samples of up to 16000 rows (D = 128) otherwise: 250 chunks one after the other.
// Many samples of different lengths that are not cut are walked longest first: the walks that are left at the end are short ones (512 x 4 samples of up to 1024
// rows, forward 307 -> 260 us); the order is made by the attention's scheduler.
// The backward's three walks are three workgroups, side by side (see linear_walk_kernel).  At D = 64 and with many rows (W >= 1024) two: there dk and dv as one, which
// reads 6 tensors instead of 8, are faster (1024 x 8 heads of up to 1024 rows: 1390 us and three 1465; fp32, 4 heads, 1790 and 1870; but 512 samples of 256 rows,
// W = 256, 41.5 and three 39.5, 256 of 64 rows 11.0 and 7.5).  few: where all rows take no longer than the longest sample's walk.
LinearPlan linear_plan(int64_t B, int64_t rows, int64_t max_len, int H, int D, bool backward) {
    constexpr int64_t kPlaces = 2 * 256, kLeastSegment = 256, kMostSegment = 1024;
    LinearPlan p;
    const int64_t W = (int64_t)((double)rows * H / kPlaces);
    p.segments = 1;
    p.segment_rows = max_len > 0 ? max_len : 1;
    p.between = 0;
    if (max_len > rows) max_len = rows;
    if (max_len > 640 + 3.3 * W) {
        int64_t segment = (W + 63) / 64 * 64;
        segment = segment < kLeastSegment ? kLeastSegment : segment > kMostSegment ? kMostSegment : segment;
        if (segment < max_len && B * H * ((max_len + segment - 1) / segment) <= (int64_t)1 << 19) {   // (what the launches reach)
            p.segments = (int)((max_len + segment - 1) / segment);
            p.segment_rows = segment;
            p.between = (int)(rows / segment);
        }
    }
    p.few = 3 * W < max_len;
    p.apart = D != 64 || p.few || W < 1024;
    p.ordered = p.segments == 1 && B > 1 && B * H > kPlaces && max_len >= 512 && (double)max_len * B > 1.2 * rows;
    p.order_words = p.ordered ? (2 * B + 1 + kNumCounters + 63) / 64 * 64 : 0;
    p.bytes = p.order_words * 4 + (int64_t)(backward ? 2 : 1) * H * p.between * D * D * 4;
    return p;
}

template <typename T, int D, int KS, int kParts, bool kStateOnly>
static void launch_side_by_side(const LinearWalks &walks, int n, const float *log_decay, const int64_t *offsets, const int32_t *order, int64_t B, int H, const LinearPlan &p,
                                float *carried, hipStream_t stream) {
    constexpr unsigned kThreads = 2 * D * KS;
    const int64_t blocks = D * sizeof(T) < 128 ? (B * p.segments + 7) / 8 * 8 * H : (B * p.segments * H + 7) / 8 * 8;
    const bool fit = n * blocks * kThreads < (int64_t)1 << 32;   // (what a launch has room for in x)
    hipLaunchKernelGGL((linear_walk_kernel<T, D, 1, KS, kParts, kStateOnly>), dim3((unsigned)(fit ? n * blocks : blocks), fit ? 1 : n), dim3(kThreads), 0, stream, walks, log_decay,
                       offsets, order, (int)B, H, p.segments, (int)p.segment_rows, p.between, fit ? n : 1, carried);
}
template <typename T, int D, int kParts>
static void launch_walks(const LinearWalks &walks, bool backward, const float *log_decay, const int64_t *offsets, const int32_t *order, int64_t B, int H, const LinearPlan &p,
                         float *carried, hipStream_t stream) {
    constexpr int KS = D == 64 || (D == 128 && sizeof(T) == 4) ? 2 : 1;
    if (p.segments > 1) {   // walk 0, and of the two that go back, which have one state, walk 2
        const LinearWalks states{{walks.walk[0], walks.walk[2], walks.walk[2]}};
        const int n = backward ? 2 : 1;
        launch_side_by_side<T, D, KS, kParts, true>(states, n, log_decay, offsets, order, B, H, p, carried, stream);
        hipLaunchKernelGGL(linear_carry_kernel, dim3((unsigned)(B * H * (D * D / 1024)), n), dim3(256), 0, stream, states, log_decay, offsets, H, D, p.segments, (int)p.segment_rows,
                           p.between, carried);
    }
    const bool apart = backward && p.apart;
    // (bf16, D = 64, three walks of many rows: 512 samples of 256 rows 39.5 us with two waves a walk, 43 with four)
    if (D == 64 && sizeof(T) == 2 && apart && !p.few)
        launch_side_by_side<T, D, 1, kParts, false>(walks, 3, log_decay, offsets, order, B, H, p, carried, stream);
    else
        launch_side_by_side<T, D, KS, kParts, false>(walks, apart ? 3 : 1, log_decay, offsets, order, B, H, p, carried, stream);
    if constexpr (D == 64)
        if (backward && !apart)
            hipLaunchKernelGGL((linear_walk_kernel<T, D, 2, 1, kParts, false>), dim3((unsigned)(B * p.segments * H)), dim3(4 * D), 0, stream, walks, log_decay, offsets, order, (int)B,
                               H, p.segments, (int)p.segment_rows, p.between, 1, carried);
}
template <typename T, int D>
static hipError_t launch_walks(const LinearWalks &walks, bool backward, bool states, const float *log_decay, const int64_t *offsets, const int32_t *order, int64_t B, int H,
                               const LinearPlan &p, float *carried, hipStream_t stream) {
    if constexpr (sizeof(T) == 4) launch_walks<T, D, 1>(walks, backward, log_decay, offsets, order, B, H, p, carried, stream);
    else if (states) launch_walks<T, D, 3>(walks, backward, log_decay, offsets, order, B, H, p, carried, stream);
    else launch_walks<T, D, 2>(walks, backward, log_decay, offsets, order, B, H, p, carried, stream);
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_walks(const LinearWalks &walks, bool backward, bool states, const float *log_decay, const int64_t *offsets, int64_t B, int H, int D,
                               const LinearPlan &p, void *workspace, hipStream_t stream) {
    int32_t *const words = (int32_t *)workspace;
    const int32_t *order = nullptr;
    if (p.ordered) {   // [counters][order][tile_start]
        order = words + kNumCounters;
        const ScheduleJob job{offsets, nullptr, 64, words + kNumCounters, words + kNumCounters + B};
        const hipError_t e = launch_schedules(&job, 1, (int)B, words, kNumCounters, stream);
        if (e != hipSuccess) return e;
    }
    float *const carried = (float *)(words + p.order_words);
    switch (D) {
        case 32: return launch_walks<T, 32>(walks, backward, states, log_decay, offsets, order, B, H, p, carried, stream);
        case 64: return launch_walks<T, 64>(walks, backward, states, log_decay, offsets, order, B, H, p, carried, stream);
        case 128: return launch_walks<T, 128>(walks, backward, states, log_decay, offsets, order, B, H, p, carried, stream);
        default: return hipErrorInvalidValue;
    }
}

hipError_t launch_linear_walks(bool f32, const LinearWalks &walks, bool backward, bool states, const float *log_decay, const int64_t *offsets, int64_t B, int H,
                               int D, const LinearPlan &p, void *workspace, hipStream_t stream) {
    return f32 ? launch_walks<float>(walks, backward, states, log_decay, offsets, B, H, D, p, workspace, stream)
               : launch_walks<__bf16>(walks, backward, states, log_decay, offsets, B, H, D, p, workspace, stream);
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
