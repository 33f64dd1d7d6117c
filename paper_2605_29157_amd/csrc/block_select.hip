// Which blocks of a long cache a decode step reads: bounds of the keys of every block of 64, a score of every block against the
// step's queries, the list of the blocks to keep (decode_rows_bf16.hip and decode_q4_bf16.hip walk it).
//
// For a block j with smallest and largest keys lo_j, hi_j (by dimension) and a query q no key of the block has a larger product than
//     sum_i max(q_i lo_ji, q_i hi_ji) = sum_i max(q_i, 0) hi_ji + min(q_i, 0) lo_ji.
// The score is the largest of these over the rows and heads that share the list. A list has to be the same however its sums are
// ordered, so they are made in 64 bits: a product of two bf16 has 16 bits, 128 of them add 7, which leaves 30 of 53 for their range: sums are exact
// where the products that are not 0 lie within 2^30 of each other.
//
// What bounds them: bounds, the keys read once (2 D bytes a key; few blocks: one launch); scores, the bounds read once (4 D bytes
// a block, 1 / 64 of the cache's) beside 2 D additions in 64 bits a column; the choice, one workgroup a list, latency.
#include "plx_kernels.h"
#include "plx_q4.h"

namespace plx {

namespace {

// bf16 halves <-> 16-bit integers of the same order (NaN beyond the infinity of its sign); its own inverse
__device__ __forceinline__ uint32_t ordered_halves(uint32_t x) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    const s16x2 y = __builtin_bit_cast(s16x2, x);
    return x ^ (__builtin_bit_cast(uint32_t, y >> 15) & 0x7fff7fffu);
}
__device__ __forceinline__ uint32_t min_halves(uint32_t a, uint32_t b) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
    typedef short s16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(s16x2, a), __builtin_bit_cast(s16x2, b)));
}

}  // namespace

// One wave a block. A lane has 16 bytes of bf16 (8 dimensions) or 8 bytes of codes (16 dimensions, one scale) of each of its keys; all
// of them are on their way at once. PAGED: lane l looks up key l of the block and hands its place to those that read it.
template <int D, bool Q4, bool PAGED>
__global__ __launch_bounds__(256) void cache_bounds_kernel(BlockBounds p) {
    constexpr int DIMS = Q4 ? 16 : 8, LPR = D / DIMS, RPL = 64 / LPR, N = kListBlock / RPL, W = DIMS / 2;
    using Row = Q4Row<D>;
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int h = blockIdx.y, b = blockIdx.z;
    int length = p.seq_lens != nullptr ? p.seq_lens[b] : p.capacity;
    length = min(max(length, 0), p.capacity);
    const int from = p.from_lens != nullptr ? max(p.from_lens[b], 0) / kListBlock : 0;
    const int j = from + (int)blockIdx.x * 4 + w;
    if ((int)blockIdx.x * 4 + w >= p.most || j >= p.n_blocks || (int64_t)j * kListBlock >= length) return;
    const int row = lane / LPR, part = lane % LPR;
    const char *keys = p.keys + (PAGED ? 0 : (int64_t)b * p.stride[0]) + h * p.stride[1];
    int64_t mine = 0;
    if constexpr (PAGED) {  // (a table entry that is no page: page 0 or the last, as the decode kernels)
        const int key = min(j * kListBlock + lane, length - 1), page_no = key / p.page_size;
        const int64_t page = min(max(p.block_table[(int64_t)b * p.table_stride + page_no], 0), p.num_pages - 1);
        mine = page * p.stride[0] + (int64_t)(key - page_no * p.page_size) * p.stride[2];
    }
    u32x4 raw[N];
    uint32_t scale[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        int64_t at;  // (keys behind the last: that one again)
        if constexpr (PAGED)
            at = ((int64_t)__shfl((int)(mine >> 32), RPL * n + row, 64) << 32) | (uint32_t)__shfl((int)mine, RPL * n + row, 64);
        else
            at = (int64_t)min(j * kListBlock + RPL * n + row, length - 1) * p.stride[2];
        if constexpr (Q4) {
            const u32x2 codes = *(const u32x2 *)(keys + at + 8 * part);
            raw[n] = u32x4{codes[0], codes[1], 0u, 0u};
            scale[n] = *(const uint8_t *)(keys + at + Row::kKScale + part);
        } else {
            raw[n] = *(const u32x4 *)(keys + at + 16 * part);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t lo[W], hi[W];
#pragma unroll
    for (int i = 0; i < W; ++i) lo[i] = 0x7fff7fffu, hi[i] = 0x80008000u;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint32_t x[W];
        if constexpr (Q4) {
            const u32x4 a = q4_to_bf16(raw[n][0], q4_scale(scale[n])), c = q4_to_bf16(raw[n][1], q4_scale(scale[n]));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = c[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = raw[n][i];
        }
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const uint32_t y = ordered_halves(x[i]);
            lo[i] = min_halves(lo[i], y), hi[i] = max_halves(hi[i], y);
        }
    }
#pragma unroll
    for (int step = LPR; step < 64; step <<= 1)
#pragma unroll
        for (int i = 0; i < W; ++i) {
            lo[i] = min_halves(lo[i], (uint32_t)__shfl_xor((int)lo[i], step, 64));
            hi[i] = max_halves(hi[i], (uint32_t)__shfl_xor((int)hi[i], step, 64));
        }
    if (row != 0) return;
    __bf16 *out = (__bf16 *)p.bounds + ((((int64_t)b * p.Hkv + h) * p.n_blocks + j) * 2) * D + DIMS * part;
#pragma unroll
    for (int i = 0; i < W; i += 4) {
        *(u32x4 *)(out + 2 * i) = u32x4{ordered_halves(lo[i]), ordered_halves(lo[i + 1]), ordered_halves(lo[i + 2]), ordered_halves(lo[i + 3])};
        *(u32x4 *)(out + D + 2 * i) = u32x4{ordered_halves(hi[i]), ordered_halves(hi[i + 1]), ordered_halves(hi[i + 2]), ordered_halves(hi[i + 3])};
    }
}

namespace {

// Scores as 64-bit integers of the same order; a NaN is the largest score there is
__device__ __forceinline__ uint64_t score_key(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    if (x != x) return 0xfff0000000000000ull;  // (that of infinity)
    return u >> 63 ? ~u : u | (1ull << 63);
}

template <int CTRL>
__device__ __forceinline__ double moved(double x) {  // by a data-parallel-primitive pattern inside a row of 16 lanes
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// x[0 .. N) summed over pairs of lanes, half of them in each lane of a pair: upper lanes (bit) keep x[N / 2 ..)
template <int CTRL, int N>
__device__ __forceinline__ void halve(double (&x)[N], bool upper) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const double keep = upper ? x[N / 2 + i] : x[i], give = upper ? x[i] : x[N / 2 + i];
        x[i] = keep + moved<CTRL>(give);
    }
}

// The bounds of 16 blocks, from `held` on those of the last one: a lane has 8 dimensions
template <int D>
struct Bounds16 {
    static constexpr int LPB = D / 8, BPL = 64 / LPB, STEPS = 16 / BPL;  // lanes of a block; blocks of a wave at a time; times
    u32x4 lo[STEPS], hi[STEPS];
    __device__ __forceinline__ void load(const BlockSelect &p, int b, int h, int j0, int held) {
        const int lane = threadIdx.x & 63;
        const __bf16 *bounds = (const __bf16 *)p.bounds + ((int64_t)b * p.Hkv + h) * p.n_blocks * 2 * D + 8 * (lane % LPB);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int j = min(j0 + BPL * s + lane / LPB, held - 1);
            lo[s] = *(const u32x4 *)(bounds + (int64_t)j * 2 * D), hi[s] = *(const u32x4 *)(bounds + (int64_t)j * 2 * D + D);
        }
    }
};
// sum + 0 * x, x both bf16 halves: NaN once one of them is infinite or NaN, in one instruction (with bits and compares 128 lists of 2048
// blocks took 34.5 us, so 32.5)
__device__ __forceinline__ float add_zero_times(uint32_t x, float sum) {
    typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16_pair, x), bf16_pair{(__bf16)0.f, (__bf16)0.f}, sum, false);
}

// The score's key of one of these blocks, the same for the four lanes from 4 n on, which share it; its number among the 16 is returned.
// COLS columns (query rows x heads of the group) at a time.
template <int D, int COLS>
__device__ __forceinline__ int score_blocks(const BlockSelect &p, int b, int h, const Bounds16<D> &bounds, uint64_t &best) {
    constexpr int LPB = Bounds16<D>::LPB, BPL = Bounds16<D>::BPL, STEPS = Bounds16<D>::STEPS;
    const int lane = threadIdx.x & 63, part = lane % LPB;
    const int G = p.Hq / p.Hkv, n_cols = G * p.Tq;
    const auto &lo = bounds.lo, &hi = bounds.hi;
    best = 0;
    for (int x0 = 0; x0 < n_cols; x0 += COLS) {
        double sum[COLS][STEPS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            const int x = min(x0 + c, n_cols - 1), t = x / G, head = x - t * G;  // (past the last column: that again)
            const u32x4 q = *(const u32x4 *)((const __bf16 *)p.q + (((int64_t)b * p.Hq + (int64_t)h * G + head) * p.Tq + t) * D + 8 * part);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) sum[c][s] = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double q0 = (double)bf16_lo_f32(q[i]), q1 = (double)bf16_hi_f32(q[i]);
                // of negative q the smallest key counts: a byte permutation picks the bound's half and widens it to fp32 (selected
                // by masks and widened after: a third of the instructions more, 128 lists of 2048 blocks 32.8 us, so 30.9)
                const uint32_t s0 = 0x05040c0cu ^ ((uint32_t)__builtin_amdgcn_sbfe((int)q[i], 15, 1) & 0x04040000u);
                const uint32_t s1 = 0x07060c0cu ^ ((uint32_t)((int)q[i] >> 31) & 0x04040000u);
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const float y0 = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi[s][i], lo[s][i], s0));
                    const float y1 = __builtin_bit_cast(float, __builtin_amdgcn_perm(hi[s][i], lo[s][i], s1));
                    sum[c][s] = fma(q0, (double)y0, sum[c][s]);
                    sum[c][s] = fma(q1, (double)y1, sum[c][s]);
                }
            }
        }
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            double *x = sum[c];
            if constexpr (D == 128) {
                halve<0x128, 4>(sum[c], (lane & 8) != 0);                                  // row_ror:8: lane ^ 8
                double two[2] = {x[0], x[1]};
                halve<0x141, 2>(two, (lane & 4) != 0);                                     // row_half_mirror: lane ^ 7
                x[0] = two[0];
            } else {
                halve<0x141, 2>(sum[c], (lane & 4) != 0);
            }
            x[0] += moved<0x4E>(x[0]);  // quad_perm [2, 3, 0, 1]: lane ^ 2
            x[0] += moved<0xB1>(x[0]);  // quad_perm [1, 0, 3, 2]: lane ^ 1
            const uint64_t key = score_key(x[0]);
            best = key > best ? key : best;
        }
    }
    // a bound that is not finite: the highest, whichever way the queries point
    uint32_t odd = 0;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) x = add_zero_times(hi[s][i], add_zero_times(lo[s][i], x));
        odd |= x != x ? 1u << s : 0u;
    }
    const int mine = D == 128 ? (lane & 8 ? 2 : 0) + (lane & 4 ? 1 : 0) : (lane & 4 ? 1 : 0);
    if (__builtin_expect(__any(odd != 0), 0)) {
#pragma unroll
        for (int step = 1; step < LPB; step <<= 1) odd |= (uint32_t)__shfl_xor((int)odd, step, 64);
        if (odd >> mine & 1u) best = 0xfff0000000000000ull;
    }
    return BPL * mine + lane / LPB;
}

__device__ __forceinline__ int held_blocks(const BlockSelect &p, int b) {
    return p.seq_lens == nullptr ? p.n_blocks : min((int)(((int64_t)max(p.seq_lens[b], 0) + kListBlock - 1) / kListBlock), p.n_blocks);
}

// Blocks up to which one launch does it all, a workgroup reading its list's bounds alone, in one round of its waves. Two launches / one in a
// replayed graph, us, d = 128, two columns: 8 lists of 64 blocks 8.2 / 6.5, 128 8.5 / 7.4, 256 8.7 / 9.2; 128 lists 8.6 / 6.8, 9.0 / 7.7,
// 9.8 / 9.9; 512 lists 13.4 / 8.8, 17.1 / 10.9, 24.9 / 19.4 (and on a stream the host saves a launch, 2.8); 512 blocks, in two rounds:
// 8 lists 8.9 / 13.0, 128 lists 13.8 / 14.0.
constexpr int kOneLaunchBlocks = 256;
constexpr int kPickThreads = 1024, kPickWaves = kPickThreads / 64;
constexpr int kPickKeys = 4096;  // that are kept in LDS
constexpr int kDigits = 512;     // values of a digit of 9 bits

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    auto with = [](uint32_t y, auto ctrl) {
        return max(y, (uint32_t)__builtin_amdgcn_update_dpp((int)y, (int)y, decltype(ctrl)::value, 0xf, 0xf, false));
    };
    x = with(x, std::integral_constant<int, 0xB1>{});   // quad_perm [1, 0, 3, 2]
    x = with(x, std::integral_constant<int, 0x4E>{});   // quad_perm [2, 3, 0, 1]
    x = with(x, std::integral_constant<int, 0x141>{});  // row_half_mirror
    x = with(x, std::integral_constant<int, 0x140>{});  // row_mirror
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)x, 0), (uint32_t)__builtin_amdgcn_readlane((int)x, 16));
    return max(a, max((uint32_t)__builtin_amdgcn_readlane((int)x, 32), (uint32_t)__builtin_amdgcn_readlane((int)x, 48)));
}

struct PickScratch {
    uint32_t ends[2][kPickWaves];
    int hist[kDigits];
    int digit_at, digit_above, digit_count;
    int above[kPickWaves], equal[kPickWaves];
};

// The list of one (sequence, key head) that holds more blocks than are kept. Of those between the first and the recent ones the `need`
// with the largest keys, found by digits below the highest bit in which they differ; of equal ones the lowest numbers. All
// kPickThreads threads take part; keys: LDS or memory.
template <class Keys>
__device__ __forceinline__ void pick_blocks(const BlockSelect &p, int held, const Keys &keys, int32_t *out, PickScratch &lds) {
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
    const int lo = p.first, hi = held - p.recent;  // candidates
    int need = p.keep - p.first - p.recent;
    for (int i = tid; i < p.first; i += kPickThreads) out[i] = i;
    for (int i = tid; i < p.recent; i += kPickThreads) out[p.keep - p.recent + i] = hi + i;
    if (need == 0) return;  // (uniform)

    // ---- the range of the keys' upper halves ---------------------------------------------------------------
    uint32_t least = ~0u, most = 0;
    for (int i = lo + tid; i < hi; i += kPickThreads) {
        const uint32_t k = (uint32_t)(keys[i] >> 32);
        least = min(least, k), most = max(most, k);
    }
    least = ~wave_max(~least), most = wave_max(most);
    if (lane == 0) lds.ends[0][w] = least, lds.ends[1][w] = most;
    for (int i = tid; i < kDigits; i += kPickThreads) lds.hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPickWaves; ++i) least = min(least, lds.ends[0][i]), most = max(most, lds.ends[1][i]);
    const uint64_t base_key = (uint64_t)least << 32;
    // ---- the smallest key that is kept, digit by digit ------------------------------------------------------
    // Keys are looked at as key - base_key; `prefix` are the digits found, `shift` the bits below them.
    int shift = 64 - __builtin_clz((most - least) | 1u) - (most == least);
    uint64_t prefix = 0;
    while (shift > 0) {
        const int bits = min(shift, 9), below = shift - bits;
        for (int i = lo + tid; i < hi; i += kPickThreads) {
            const uint64_t k = keys[i] - base_key;
            if (shift == 64 || k >> shift == prefix) atomicAdd(&lds.hist[(k >> below) & ((1 << bits) - 1)], 1);
        }
        __syncthreads();
        if (w == 0) {  // lane l: digits 8 l .. 8 l + 7
            int own[8], sum = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) own[i] = lds.hist[8 * lane + i], lds.hist[8 * lane + i] = 0, sum += own[i];
            int above = sum;  // counts of this lane's digits and of those above them
#pragma unroll
            for (int step = 1; step < 64; step <<= 1) {
                const int up = __shfl_down(above, step, 64);
                if (lane + step < 64) above += up;
            }
            above -= sum;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                if (above < need && need <= above + own[i]) lds.digit_at = 8 * lane + i, lds.digit_above = above, lds.digit_count = own[i];
                above += own[i];
            }
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint64_t)lds.digit_at;
        need -= lds.digit_above;
        shift = below;
        if (lds.digit_count == need) break;  // every key of this digit is kept
        __syncthreads();                     // (the digit is written again)
    }
    // ---- the list, in ascending order ---------------------------------------------------------------------
    int before_above = 0, before_equal = 0;
    for (int base = lo; base < hi; base += kPickThreads) {
        const int i = base + tid;
        uint64_t k = 0;
        if (i < hi) k = keys[i] - base_key;
        const uint64_t top = shift == 64 ? 0 : k >> shift;
        const bool above = i < hi && top > prefix, equal = i < hi && top == prefix;
        const uint64_t above_mask = __ballot(above), equal_mask = __ballot(equal), mine = (1ull << lane) - 1;
        if (lane == 0) lds.above[w] = __popcll(above_mask), lds.equal[w] = __popcll(equal_mask);
        __syncthreads();
        int a = before_above, e = before_equal;
#pragma unroll
        for (int n = 0; n < kPickWaves; ++n) {
            if (n < w) a += lds.above[n], e += lds.equal[n];
            before_above += lds.above[n], before_equal += lds.equal[n];
        }
        a += __popcll(above_mask & mine), e += __popcll(equal_mask & mine);
        if (above || (equal && e < need)) out[p.first + a + min(e, need)] = i;
        __syncthreads();
    }
}

// A sequence with up to `keep` blocks keeps them all
__device__ __forceinline__ bool all_kept(const BlockSelect &p, int held, int32_t *out) {
    if (held > p.keep) return false;
    for (int i = threadIdx.x; i < p.keep; i += blockDim.x) out[i] = i < held ? i : -1;
    return true;
}

}  // namespace

// Scores alone, 64 blocks a workgroup. (32 or 64 blocks a wave, all on their way at once: 1 list set of 8 x 512 blocks 9.2 -> 11.0, 14.8
// with the pick, 128 lists x 2048 34.2 -> 35.3, 41.8.)
template <int D, int COLS>
__global__ __launch_bounds__(256) void block_score_kernel(BlockSelect p) {
    const int h = blockIdx.y, b = blockIdx.z, held = held_blocks(p, b);
    const int j0 = ((int)blockIdx.x * 4 + (threadIdx.x >> 6)) * 16;
    if (j0 >= held || held <= p.keep) return;
    Bounds16<D> bounds;
    bounds.load(p, b, h, j0, held);
    uint64_t key;
    const int j = j0 + score_blocks<D, COLS>(p, b, h, bounds, key);
    if ((threadIdx.x & 3) == 0 && j < held) p.keys[((int64_t)b * p.Hkv + h) * p.n_blocks + j] = key;
}

__global__ __launch_bounds__(kPickThreads) void block_pick_kernel(BlockSelect p) {
    __shared__ PickScratch scratch;
    __shared__ uint64_t keys[kPickKeys];
    const int h = blockIdx.x, b = blockIdx.y, held = held_blocks(p, b);
    const int64_t list = (int64_t)b * p.Hkv + h;
    int32_t *out = p.block_list + list * p.keep;
    if (all_kept(p, held, out)) return;
    const uint64_t *src = p.keys + list * p.n_blocks;
    if (held > kPickKeys) {
        pick_blocks(p, held, src, out, scratch);
    } else {
        for (int i = threadIdx.x; i < held; i += kPickThreads) keys[i] = src[i];
        __syncthreads();
        pick_blocks(p, held, keys, out, scratch);
    }
}

// Both in one launch, a workgroup a list, for few blocks. (Two workgroups a unit: with the registers of one, 512 lists of 128 blocks 13.9
// us, so 10.9.)
template <int D, int COLS>
__global__ __launch_bounds__(kPickThreads, 8) void block_select_kernel(BlockSelect p) {
    __shared__ PickScratch scratch;
    __shared__ uint64_t keys[kOneLaunchBlocks];
    static_assert(kOneLaunchBlocks <= kPickWaves * 16, "a round of the waves");
    const int h = blockIdx.x, b = blockIdx.y, held = held_blocks(p, b);
    int32_t *out = p.block_list + ((int64_t)b * p.Hkv + h) * p.keep;
    if (all_kept(p, held, out)) return;
    const int j0 = (threadIdx.x >> 6) * 16;
    if (j0 < held) {
        Bounds16<D> bounds;
        bounds.load(p, b, h, j0, held);
        uint64_t key;
        const int j = j0 + score_blocks<D, COLS>(p, b, h, bounds, key);
        if ((threadIdx.x & 3) == 0 && j < held) keys[j] = key;
    }
    __syncthreads();
    pick_blocks(p, held, keys, out, scratch);
}

template <int D, bool Q4>
static void launch_bounds_form(const BlockBounds &p, hipStream_t stream) {
    const dim3 grid((p.most + 3) / 4, p.Hkv, p.B);
    if (p.block_table != nullptr)
        hipLaunchKernelGGL((cache_bounds_kernel<D, Q4, true>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((cache_bounds_kernel<D, Q4, false>), grid, dim3(256), 0, stream, p);
}

hipError_t launch_cache_bounds(const BlockBounds &p, hipStream_t stream) {
    if (p.d == 128)
        p.q4 ? launch_bounds_form<128, true>(p, stream) : launch_bounds_form<128, false>(p, stream);
    else
        p.q4 ? launch_bounds_form<64, true>(p, stream) : launch_bounds_form<64, false>(p, stream);
    return hipGetLastError();
}

template <int D, int COLS>
static hipError_t launch_select_form(const BlockSelect &p, hipStream_t stream) {
    const dim3 lists(p.Hkv, p.B);
    if (p.n_blocks <= kOneLaunchBlocks) {
        hipLaunchKernelGGL((block_select_kernel<D, COLS>), lists, dim3(kPickThreads), 0, stream, p);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((block_score_kernel<D, COLS>), dim3((p.n_blocks + 63) / 64, p.Hkv, p.B), dim3(256), 0, stream, p);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(block_pick_kernel, lists, dim3(kPickThreads), 0, stream, p);
    return hipGetLastError();
}

template <int D>
static hipError_t launch_select_columns(const BlockSelect &p, hipStream_t stream) {
    return p.Hq / p.Hkv * p.Tq == 1 ? launch_select_form<D, 1>(p, stream) : launch_select_form<D, 2>(p, stream);
}

hipError_t launch_select_blocks(const BlockSelect &p, hipStream_t stream) {
    return p.d == 128 ? launch_select_columns<128>(p, stream) : launch_select_columns<64>(p, stream);
}

}  // namespace plx
