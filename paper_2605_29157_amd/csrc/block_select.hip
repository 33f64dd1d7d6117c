// Which blocks of a long cache a decode step reads: bounds of the keys of every block of 64, a score of every block against the
// step's queries, the list of the blocks to keep (decode_rows_bf16.hip and decode_q4_bf16.hip walk it).
//
// For a block j with smallest and largest keys lo_j, hi_j (by dimension) and a query q no key of the block has a larger product than
//     sum_i max(q_i lo_ji, q_i hi_ji) = sum_i max(q_i, 0) hi_ji + min(q_i, 0) lo_ji.
// The score is the largest of these over the rows and heads that share the list. A list has to be the same however its sums are
// ordered, so they are made in 64 bits: a product of two bf16 has 16 bits, so sums of 128 of them are exact unless they lie more than
// 2^37 apart.
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

// One wave a block. A lane has 16 bytes of bf16 (8 dimensions) or 8 bytes of codes (16 dimensions, one scale) of each of its keys.
template <int D, bool Q4>
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
    uint32_t lo[W], hi[W];
#pragma unroll
    for (int i = 0; i < W; ++i) lo[i] = 0x7fff7fffu, hi[i] = 0x80008000u;
    u32x4 raw[N];
    float scale[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        // (keys behind the last: that one again. A table entry that is no page: page 0, as the decode kernels)
        const int key = min(j * kListBlock + RPL * n + row, length - 1);
        int64_t at = (int64_t)b * p.stride[0] + (int64_t)key * p.stride[2];
        if (p.block_table != nullptr) {
            const int page_no = key / p.page_size;
            const int64_t page = min(max(p.block_table[(int64_t)b * p.table_stride + page_no], 0), p.num_pages - 1);
            at = page * p.stride[0] + (int64_t)(key - page_no * p.page_size) * p.stride[2];
        }
        const char *src = p.keys + at + h * p.stride[1];
        if constexpr (Q4) {
            const u32x2 codes = *(const u32x2 *)(src + 8 * part);
            raw[n] = u32x4{codes[0], codes[1], 0u, 0u};
            scale[n] = q4_scale(*(const uint8_t *)(src + Row::kKScale + part));
        } else {
            raw[n] = *(const u32x4 *)(src + 16 * part);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        uint32_t x[W];
        if constexpr (Q4) {
            const u32x4 a = q4_to_bf16(raw[n][0], scale[n]), c = q4_to_bf16(raw[n][1], scale[n]);
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

constexpr int kScoreBlocks = 64;  // blocks of a workgroup of the score kernel, 16 a wave

// Scores as 64-bit integers of the same order; a NaN is the largest score there is
__device__ __forceinline__ uint64_t score_key(double x) {
    const uint64_t u = __builtin_bit_cast(uint64_t, x);
    if (x != x) return 0xfff0000000000000ull;  // (that of infinity)
    return u >> 63 ? ~u : u | (1ull << 63);
}

template <int N>
__device__ __forceinline__ double lanes_sum(double x) {
#pragma unroll
    for (int step = 1; step < N; step <<= 1) x += __shfl_xor(x, step, 64);
    return x;
}

}  // namespace

// A lane has 8 dimensions of a block's bounds and of COLS columns (query rows x heads of the group) at a time.
template <int D, int COLS>
__global__ __launch_bounds__(256) void block_score_kernel(BlockSelect p) {
    constexpr int LPB = D / 8, BPL = 64 / LPB;  // lanes of a block; blocks of a wave at a time
    const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, part = lane % LPB;
    const int h = blockIdx.y, b = blockIdx.z;
    int held = p.n_blocks;
    if (p.seq_lens != nullptr) held = min((int)(((int64_t)max(p.seq_lens[b], 0) + kListBlock - 1) / kListBlock), held);
    const int j0 = ((int)blockIdx.x * 4 + w) * (kScoreBlocks / 4);
    if (j0 >= held || held <= p.keep) return;  // (all are kept)
    const int G = p.Hq / p.Hkv, n_cols = G * p.Tq;
    const __bf16 *bounds = (const __bf16 *)p.bounds + ((int64_t)b * p.Hkv + h) * p.n_blocks * 2 * D + 8 * part;
    uint64_t *keys = p.keys + ((int64_t)b * p.Hkv + h) * p.n_blocks;
    constexpr int STEPS = kScoreBlocks / 4 / BPL;
    uint64_t best[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) best[s] = 0;
    for (int x0 = 0; x0 < n_cols; x0 += COLS) {
        double up[COLS][8], down[COLS][8];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            const int x = min(x0 + c, n_cols - 1), t = x / G, head = x - t * G;  // (past the last column: that again)
            const u32x4 q = *(const u32x4 *)((const __bf16 *)p.q + (((int64_t)b * p.Hq + (int64_t)h * G + head) * p.Tq + t) * D + 8 * part);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y0 = bf16_lo_f32(q[i]), y1 = bf16_hi_f32(q[i]);
                // (a NaN stays one in both)
                up[c][2 * i] = (double)(y0 < 0.f ? 0.f : y0), down[c][2 * i] = (double)(y0 > 0.f ? 0.f : y0);
                up[c][2 * i + 1] = (double)(y1 < 0.f ? 0.f : y1), down[c][2 * i + 1] = (double)(y1 > 0.f ? 0.f : y1);
            }
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int j = min(j0 + BPL * s + lane / LPB, held - 1);
            const u32x4 lo = *(const u32x4 *)(bounds + (int64_t)j * 2 * D), hi = *(const u32x4 *)(bounds + (int64_t)j * 2 * D + D);
            double sum[COLS];
#pragma unroll
            for (int c = 0; c < COLS; ++c) sum[c] = 0.0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const double l0 = (double)bf16_lo_f32(lo[i]), l1 = (double)bf16_hi_f32(lo[i]);
                const double h0 = (double)bf16_lo_f32(hi[i]), h1 = (double)bf16_hi_f32(hi[i]);
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    sum[c] = fma(up[c][2 * i], h0, sum[c]), sum[c] = fma(down[c][2 * i], l0, sum[c]);
                    sum[c] = fma(up[c][2 * i + 1], h1, sum[c]), sum[c] = fma(down[c][2 * i + 1], l1, sum[c]);
                }
            }
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const uint64_t key = score_key(lanes_sum<LPB>(sum[c]));
                best[s] = key > best[s] ? key : best[s];
            }
        }
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int j = j0 + BPL * s + lane / LPB;
        if (part == 0 && j < held) keys[j] = best[s];
    }
}

namespace {
constexpr int kPickThreads = 512, kPickWaves = kPickThreads / 64;
}

// The list of one (sequence, key head). Of the blocks between the first and the recent ones the `need` largest keys, found by digits
// of 8 bits below the highest bit in which they differ; of equal ones the lowest numbers.
__global__ __launch_bounds__(kPickThreads) void block_pick_kernel(BlockSelect p) {
    __shared__ uint64_t ends[2][kPickWaves];
    __shared__ int hist[256];
    __shared__ int digit_at, digit_above, digit_count;
    __shared__ int wave_above[kPickWaves], wave_equal[kPickWaves];
    const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63;
    const int64_t list = (int64_t)blockIdx.y * p.Hkv + blockIdx.x;
    int32_t *out = p.block_list + list * p.keep;
    int held = p.n_blocks;
    if (p.seq_lens != nullptr) held = min((int)(((int64_t)max(p.seq_lens[blockIdx.y], 0) + kListBlock - 1) / kListBlock), held);
    if (held <= p.keep) {  // (uniform)
        for (int i = tid; i < p.keep; i += kPickThreads) out[i] = i < held ? i : -1;
        return;
    }
    const uint64_t *keys = p.keys + list * p.n_blocks;
    const int lo = p.first, hi = held - p.recent;  // candidates
    int need = p.keep - p.first - p.recent;
    for (int i = tid; i < p.first; i += kPickThreads) out[i] = i;
    for (int i = tid; i < p.recent; i += kPickThreads) out[p.keep - p.recent + i] = hi + i;
    if (need == 0) return;  // (uniform)

    // ---- the range of the keys ----------------------------------------------------------------------------
    uint64_t least = ~0ull, most = 0;
    for (int i = lo + tid; i < hi; i += kPickThreads) {
        const uint64_t k = keys[i];
        least = k < least ? k : least, most = k > most ? k : most;
    }
#pragma unroll
    for (int step = 1; step < 64; step <<= 1) {
        const uint64_t a = __shfl_xor((unsigned long long)least, step, 64), c = __shfl_xor((unsigned long long)most, step, 64);
        least = a < least ? a : least, most = c > most ? c : most;
    }
    if (lane == 0) ends[0][w] = least, ends[1][w] = most;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPickWaves; ++i) {
        least = ends[0][i] < least ? ends[0][i] : least;
        most = ends[1][i] > most ? ends[1][i] : most;
    }
    // ---- the smallest key that is kept, digit by digit ------------------------------------------------------
    // Keys are looked at as key - least; `prefix` are the digits found, `shift` the bits below them.
    int shift = most == least ? 0 : 64 - __builtin_clzll(most - least);
    uint64_t prefix = 0;
    while (shift > 0) {
        const int bits = min(shift, 8), below = shift - bits;
        for (int i = tid; i < 256; i += kPickThreads) hist[i] = 0;
        __syncthreads();
        for (int i = lo + tid; i < hi; i += kPickThreads) {
            const uint64_t k = keys[i] - least;
            if (shift == 64 || k >> shift == prefix) atomicAdd(&hist[(k >> below) & ((1 << bits) - 1)], 1);
        }
        __syncthreads();
        if (w == 0) {  // lane l: digits 4 l .. 4 l + 3
            int own[4], sum = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) own[i] = hist[4 * lane + i], sum += own[i];
            int above = sum;  // counts of this lane's digits and of those above them
#pragma unroll
            for (int step = 1; step < 64; step <<= 1) {
                const int up = __shfl_down(above, step, 64);
                if (lane + step < 64) above += up;
            }
            above -= sum;
#pragma unroll
            for (int i = 3; i >= 0; --i) {
                if (above < need && need <= above + own[i]) digit_at = 4 * lane + i, digit_above = above, digit_count = own[i];
                above += own[i];
            }
        }
        __syncthreads();
        prefix = (prefix << bits) | (uint64_t)digit_at;
        need -= digit_above;
        shift = below;
        const bool all = digit_count == need;  // every key of this digit is kept
        __syncthreads();                       // (hist and the digit are written again)
        if (all) break;
    }
    // ---- the list, in ascending order ---------------------------------------------------------------------
    int before_above = 0, before_equal = 0;
    for (int base = lo; base < hi; base += kPickThreads) {
        const int i = base + tid;
        uint64_t k = 0;
        if (i < hi) k = keys[i] - least;
        const uint64_t top = shift == 64 ? 0 : k >> shift;
        const bool above = i < hi && top > prefix, equal = i < hi && top == prefix;
        const uint64_t above_mask = __ballot(above), equal_mask = __ballot(equal), mine = (1ull << lane) - 1;
        if (lane == 0) wave_above[w] = __popcll(above_mask), wave_equal[w] = __popcll(equal_mask);
        __syncthreads();
        int a = before_above, e = before_equal;
#pragma unroll
        for (int n = 0; n < kPickWaves; ++n) {
            if (n < w) a += wave_above[n], e += wave_equal[n];
            before_above += wave_above[n], before_equal += wave_equal[n];
        }
        a += __popcll(above_mask & mine), e += __popcll(equal_mask & mine);
        if (above || (equal && e < need)) out[p.first + a + min(e, need)] = i;
        __syncthreads();
    }
}

hipError_t launch_cache_bounds(const BlockBounds &p, hipStream_t stream) {
    const dim3 grid((p.most + 3) / 4, p.Hkv, p.B);
    if (p.d == 128) {
        if (p.q4)
            hipLaunchKernelGGL((cache_bounds_kernel<128, true>), grid, dim3(256), 0, stream, p);
        else
            hipLaunchKernelGGL((cache_bounds_kernel<128, false>), grid, dim3(256), 0, stream, p);
    } else {
        if (p.q4)
            hipLaunchKernelGGL((cache_bounds_kernel<64, true>), grid, dim3(256), 0, stream, p);
        else
            hipLaunchKernelGGL((cache_bounds_kernel<64, false>), grid, dim3(256), 0, stream, p);
    }
    return hipGetLastError();
}

template <int D>
static void launch_scores(const BlockSelect &p, hipStream_t stream) {
    const dim3 grid((p.n_blocks + kScoreBlocks - 1) / kScoreBlocks, p.Hkv, p.B);
    const int cols = p.Hq / p.Hkv * p.Tq;
    if (cols == 1)
        hipLaunchKernelGGL((block_score_kernel<D, 1>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((block_score_kernel<D, 2>), grid, dim3(256), 0, stream, p);
}

hipError_t launch_select_blocks(const BlockSelect &p, hipStream_t stream) {
    p.d == 128 ? launch_scores<128>(p, stream) : launch_scores<64>(p, stream);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
    hipLaunchKernelGGL(block_pick_kernel, dim3(p.Hkv, p.B), dim3(kPickThreads), 0, stream, p);
    return hipGetLastError();
}

}  // namespace plx
