// Split-KV Parallax decode for more than 16 columns (rows x heads of a GQA group) whose key sets differ, bf16, gfx950: large
// trees of drafted nodes, several rows with a window and sinks. Same function, records and masks as
// decode_rows_bf16.hip; here the waves of a workgroup share the keys instead of the columns.
//
// What bounds it: up to 64 columns the bytes of K and V, every key fetched once for all columns (128 keys at D = 128 in 2.8 us
// with all units at work, 6.0 TB/s; 1.7 with few). With 128 columns the matrix work (8 D flop a score): 64 keys take 1.1 us of
// matrix instructions and 0.6 of vector work (exponentials: 16 clocks each), which the two waves of a SIMD overlap only in part;
// measured 1.9 with all units at work, 1.6 with few.
//
// Layout:
//   * eight waves, two per SIMD, so that the vector work of one runs under the matrix instructions of the other: up to 64 columns
//     four blocks of 16 columns and two halves of a tile of 128 keys, beyond eight blocks of 16 columns and tiles of 64. A wave
//     takes its 64 keys in one go, one test and no branch between their products, and reads its operands four fragments
//     ahead. Measured (us; 16 x up to 6000 keys, 8 key heads, 52 columns, 2 splits; 8 x 16384 keys, 4 key heads, 256
//     columns, 4 splits): 32 keys in one go 107, 188; 64 99, 177; reads ahead and no bank conflicts 96, 170; with a
//     faster merge 83, 160; q and rho waited for in front of the tile loop 67, 138 (since then reading two to four fragments
//     ahead, the conflicts and s_setprio around the products make no difference). Four waves
//     of 32 columns, which halve the reads of LDS, their steps pipelined by hand: 210 for the second (where 32 keys in one go
//     took 188; both with q and rho waited for inside the loop, not measured since);
//   * a tile with masks is first looked through for values of V that are not finite, and only then treated for them
//     (48 nodes x 2 heads, window 321, 6 sequences: 31 -> 23; 16 rows x 2, window 256, 8 sequences 31 -> 21);
//   * tiles in a ring of 128 KB of LDS, filled by direct global -> LDS loads (no registers parked), 64 - 112 KB of it on
//     their way; one barrier per tile;
//   * the reference of the exponentials is moved only when a score exceeds it by 2^6 (then the sums are rescaled): no
//     maximum across lanes, no rescaling of accumulators in most tiles. Sums of up to 2^6 times the number of
//     keys are far inside fp32.
#include "plx_lds_dma.h"
#include "plx_rows.h"

namespace plx {

namespace {
// Chunk c of a tile's row is at row * CPR + (c ^ rows_swizzle(row)). At D = 128 a row is 256 bytes, all 64 banks once: the sixteen rows of
// one chunk that a K operand reads get sixteen different chunks, the eight rows of two chunks of a transposing V read sixteen as
// well (with eight different chunks only, every second access waited for a bank).
template <int D>
__device__ __forceinline__ int rows_swizzle(int row) {
    const int low = ((row & 3) << 1) | ((row >> 2) & 1);
    return D == 128 ? low | (((row << 1) ^ row) & 8) : low;
}
template <int D>
__device__ __forceinline__ int rows_chunk_slot(int row, int chunk) { return row * (D / 8) + (chunk ^ rows_swizzle<D>(row)); }

constexpr float kWideSlack = 6.f;  // in the exponent of 2

// Fetches tiles of TILE keys, global -> LDS: each of the eight waves brings in TILE / 8 rows of K and of V, one run of 16 keys that
// follow each other in memory or half of one. A tile: K rows, then V rows, chunks swizzled as rows_chunk_slot.
template <int D, int CACHE, bool TREE, int TILE>
struct WideLoader {
    static constexpr int CPR = D / 8, RPL = 64 / CPR, ROWS = TILE / 8;  // rows per load, of this wave
    static constexpr int LOADS = ROWS / RPL;                                     // per tensor
    static_assert(ROWS == 8 || ROWS == 16, "within a run of 16 keys");
    const DecodeParams &p;
    const RowsScope<TREE, TILE> &scope;
    const RowsPages pages;
    const __bf16 *kbase, *vbase;
    uint32_t k_row_bytes, v_row_bytes, lds_base;
    int w, lane, last16, run_first, in_run;
    int run_k[2], run_v[2], run_slot;  // kRowsPagedRuns: where the runs are, lane j: of the j-th of the next 64 tiles

    __device__ __forceinline__ WideLoader(const DecodeParams &p, const RowsScope<TREE, TILE> &scope, int b, int hk, int w,
                                          int lane, const u32x4 *lds)
        : p(p), scope(scope), pages(p, b), w(w), lane(lane) {
        kbase = (const __bf16 *)p.k + (p.block_table == nullptr ? (int64_t)b * p.ksb : 0) + (int64_t)hk * p.ksh;
        vbase = (const __bf16 *)p.v + (p.block_table == nullptr ? (int64_t)b * p.vsb : 0) + (int64_t)hk * p.vsh;
        k_row_bytes = (uint32_t)p.ksl * 2u, v_row_bytes = (uint32_t)p.vsl * 2u;
        lds_base = lds_byte_address(lds);
        last16 = max(scope.Lb - 1, 0) & ~15;  // first key of the last run that exists
        run_first = ROWS * w & ~15, in_run = ROWS * w & 15;
        run_slot = 64;
    }
    __device__ __forceinline__ void lookup(int v) {
        int64_t ko, vo;
        pages.offsets(min(scope.key_of(min(v + lane, max(scope.n_virtual - 1, 0))) + run_first, last16), ko, vo);
        run_k[0] = (int)ko, run_k[1] = (int)(ko >> 32);
        run_v[0] = (int)vo, run_v[1] = (int)(vo >> 32);
        run_slot = 0;
    }
    __device__ __forceinline__ void issue(int v, int stage) {
        const uint32_t dk = lds_base + (uint32_t)((2 * stage * TILE + ROWS * w) * CPR) * 16u, dv = dk + TILE * CPR * 16u;
        const int tk = scope.key_of(v);
        int l = lane;
        asm volatile("" : "+v"(l));  // (the lane's offsets are worked out here: kept across the loop they would be spilled)
        if constexpr (CACHE != kRowsAny) {
            const int key0 = __builtin_amdgcn_readfirstlane(min(tk + run_first, last16));
            int64_t ko = (int64_t)key0 * p.ksl, vo = (int64_t)key0 * p.vsl;
            if constexpr (CACHE == kRowsPagedRuns) {
                if (__builtin_expect(run_slot == 64, 0)) lookup(v);  // (uniform)
                ko = ((int64_t)__builtin_amdgcn_readlane(run_k[1], run_slot) << 32) | (uint32_t)__builtin_amdgcn_readlane(run_k[0], run_slot);
                vo = ((int64_t)__builtin_amdgcn_readlane(run_v[1], run_slot) << 32) | (uint32_t)__builtin_amdgcn_readlane(run_v[0], run_slot);
                ++run_slot;
            }
            const __bf16 *kp = kbase + ko, *vp = vbase + vo;
            const int last = scope.Lb - 1 - key0;  // rows past the sequence end re-read its last row (masked later)
            const int row0 = in_run + l / CPR;     // of load 0 in the run
            if (__builtin_expect(last >= 15, 1)) {  // (uniform) the whole run exists
                const uint32_t k0 = __umul24((uint32_t)row0, k_row_bytes), v0 = __umul24((uint32_t)row0, v_row_bytes);
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const uint32_t chunk = 16u * (uint32_t)((l % CPR) ^ rows_swizzle<D>(run_first + row0 + RPL * i));
                    tile_load16_uniform<false>(k0 + (uint32_t)(RPL * i) * k_row_bytes + chunk, kp, dk + 1024u * i);
                    tile_load16_uniform<false>(v0 + (uint32_t)(RPL * i) * v_row_bytes + chunk, vp, dv + 1024u * i);
                }
            } else {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) {
                    const uint32_t chunk = 16u * (uint32_t)((l % CPR) ^ rows_swizzle<D>(run_first + row0 + RPL * i));
                    const uint32_t at = (uint32_t)min(row0 + RPL * i, last);
                    tile_load16_uniform<false>(__umul24(at, k_row_bytes) + chunk, kp, dk + 1024u * i);
                    tile_load16_uniform<false>(__umul24(at, v_row_bytes) + chunk, vp, dv + 1024u * i);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int row = ROWS * w + RPL * i + l / CPR, key = min(tk + row, scope.Lb - 1);
                int64_t ko = (int64_t)key * p.ksl, vo = (int64_t)key * p.vsl;
                if (p.block_table != nullptr) pages.offsets(key, ko, vo);  // (uniform)
                const int chunk = (l % CPR) ^ rows_swizzle<D>(row);
                tile_load16<64>(kbase + ko + 8 * chunk, dk + 1024u * i);
                tile_load16<64>(vbase + vo + 8 * chunk, dv + 1024u * i);
            }
        }
    }
    // Is a value in this wave's V rows of a tile not finite?
    __device__ __forceinline__ bool not_finite(const u32x4 *tileV) const {
        uint32_t bad = 0;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const u32x4 x = tileV[ROWS * w * CPR + 64 * i + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) bad |= not_finite_halves(x[e]);
        }
        return __any(bad != 0);
    }
    // Such values out of these rows
    __device__ __forceinline__ void clean(u32x4 *tileV) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            u32x4 &x = tileV[ROWS * w * CPR + 64 * i + lane];
            u32x4 y = x;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] &= ~not_finite_halves(y[e]);
            x = y;
        }
    }
};

// Work item of a workgroup: the column groups of one (split, key head, sequence) follow each other on one XCD (workgroups are
// dealt over the eight of them in turn), whose L2 they share. False: none.
__device__ __forceinline__ bool wide_item(const DecodeRowsParams &P, int &cg, int &split, int &hk, int &b) {
    const DecodeParams &p = P.d;
    const int id = blockIdx.x, j = id >> 3;
    cg = j % P.col_groups;
    const int unit = j / P.col_groups * 8 + (id & 7);
    if (unit >= p.S * p.Hkv * p.B) return false;
    split = unit % p.S;
    const int pair = unit / p.S;
    hk = pair % p.Hkv, b = pair / p.Hkv;
    return true;
}
}  // namespace

// Eight waves, two per SIMD. KH = 2: 64 columns per workgroup, wave w owns columns 16 (w % 4) .. + 15 and half w / 4 of the
// keys of a tile; KH = 1: 128 columns, wave w owns columns 16 w .. + 15 and all keys.
template <int D, bool USE_R, int CACHE, int KH, bool TREE>
__global__ __launch_bounds__(512, 2) void decode_rows_wide_kernel(DecodeRowsParams P) {
    const DecodeParams &p = P.d;
    constexpr int CPR = D / 8, KSTEPS = D / 32, NDB = D / 16;
    constexpr int TILE = 64 * KH, TILE_CHUNKS = TILE * CPR, STAGE_CHUNKS = 2 * TILE_CHUNKS;
    constexpr int STAGES = 8 * 1024 / STAGE_CHUNKS;  // 128 KB
    __shared__ u32x4 lds[STAGES * STAGE_CHUNKS];
    static_assert(2 * 4 * NDB * 64 <= STAGES * STAGE_CHUNKS, "the states of four waves");
    constexpr int CW = 8 / KH, COLS = 16 * CW;  // waves side by side over the columns
    __shared__ float head[CW][3][16];
    __shared__ TreeWords<TREE ? COLS : 0> tree_words;
    __shared__ int some_bad[2];  // of the masked tile in turn: V holds a value that is not finite

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int c = lane & 15, g = lane >> 4;
    const int cw = w % CW, kh = w / CW;
    int cg, split, hk, b;
    if (!wide_item(P, cg, split, hk, b)) return;
    if (tid < 2) some_bad[tid] = 0;  // (the ring's first barrier is in front of its use)
    const int G = p.G, S = p.S, Tq = p.Tq, n_cols = G * Tq, x0 = cg * COLS;
    // ---- this lane's column: q and rho operands, key set ----------------------------------------------------
    // They are here before the first tile is asked for: waited for inside the tile loop, they would make every
    // round wait for the tiles on their way as well (the wait counts loads, whichever they are): 1.9 us a tile of 64 keys x 128
    // columns instead of 1.6.
    u32x4 qf[KSTEPS], rf[KSTEPS];
    int col_end, col_lo;
    TreeRow col_nodes{};
    const int x = x0 + 16 * cw + c;
    const bool live = x < n_cols;
    const int t = live ? x / G : 0;
    {
        const int h = live ? x - t * G : 0;
        const int64_t row = (((int64_t)b * p.Hq + (int64_t)hk * G + h) * Tq + t) * D;
        const __bf16 *qrow = (const __bf16 *)p.q + row, *rrow = (const __bf16 *)p.r + row;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            const u32x4 z = {0u, 0u, 0u, 0u};
            qf[s] = live ? *(const u32x4 *)(qrow + 8 * (4 * s + g)) : z;
            if constexpr (USE_R) rf[s] = live ? *(const u32x4 *)(rrow + 8 * (4 * s + g)) : z;
        }
    }
    const RowsScope<TREE, TILE> scope(P, b, x0, COLS);
    scope.column(P, tree_words, x0, 16 * cw + c, t, live, col_lo, col_end, col_nodes);
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
        asm volatile("" : "+v"(qf[s]));
        if constexpr (USE_R) asm volatile("" : "+v"(rf[s]));
    }
    if constexpr (TREE) asm volatile("" : "+v"(col_nodes.first));
    const int per = (scope.n_virtual + S - 1) / S;
    const int v_lo = split * per, v_hi = min(v_lo + per, scope.n_virtual);

    using Loader = WideLoader<D, CACHE, TREE, TILE>;
    Loader loader(p, scope, b, hk, w, lane, lds);
    constexpr int AHEAD = STAGES - 1, LOADS = 2 * Loader::LOADS;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (v_lo + i < v_hi) loader.issue(v_lo + i, i);

    float m_run = kNegInf;
    f32x4 o1[NDB], o2[NDB], dsum1 = {0.f, 0.f, 0.f, 0.f}, dsum2 = dsum1;  // (four times the same sum: a product with ones)
#pragma unroll
    for (int i = 0; i < NDB; ++i) o1[i] = o2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float scale_log2 = p.scale * kLog2e;
    const bool live_wave = x0 + 16 * cw < n_cols;  // (uniform)

    // A operand of O^T += V^T P^T for 16 output dimensions: the 8 keys of this lane's B operand
    const int tr_key = 4 * g + (c >> 2), tr_half = (c & 1) * 4;
    auto v_fragment = [&](const u32x4 *tileV, int i) __attribute__((always_inline)) {
        const unsigned short *ldsV16 = (const unsigned short *)tileV;
        const int chunk = 2 * i + ((c & 3) >> 1);
        const u32x2 lo = lds_read_tr16(ldsV16 + rows_chunk_slot<D>(tr_key, chunk) * 8 + tr_half);
        const u32x2 hi = lds_read_tr16(ldsV16 + rows_chunk_slot<D>(16 + tr_key, chunk) * 8 + tr_half);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    uint32_t seen[2];  // of the two 32-key blocks of this wave's 64 keys
    // 32 keys of a tile that some column does not see completely and that holds values of V that are not finite: these reach the
    // columns that see their key; then (behind a barrier) they are taken out of the tile.
    auto spread_not_finite = [&](const u32x4 *tileV, uint32_t seen) __attribute__((always_inline)) {
        const u32x4 big = big_halves(seen);
#pragma unroll
        for (int i = 0; i < NDB; ++i) {
            u32x4 bad = v_fragment(tileV, i);
#pragma unroll
            for (int e = 0; e < 4; ++e) bad[e] = not_finite_halves(bad[e]) & kBigHalves;
            o1[i] = mfma16(bad, big, o1[i]);
        }
    };
    // 64 keys x 16 columns
    auto tile = [&](const u32x4 *tileK, bool whole) __attribute__((always_inline)) {
        constexpr int LOOK = 4, QK = 4 * KSTEPS, PV = 2 * NDB;  // fragments read ahead of their products; fragments of K, of V
        u32x4 kf[QK], vt[PV];
        auto load_k = [&](int f) { kf[f] = tileK[rows_chunk_slot<D>(16 * (f / KSTEPS) + c, 4 * (f % KSTEPS) + g)]; };
        auto load_v = [&](int f) { vt[f] = v_fragment(tileK + TILE_CHUNKS + 32 * (f / NDB) * CPR, f % NDB); };
        f32x4 s1[4], s2[4];
#pragma unroll
        for (int sub = 0; sub < 4; ++sub) s1[sub] = s2[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < LOOK; ++f) load_k(f);
#pragma unroll
        for (int f = 0; f < QK; ++f) {
            if (f + LOOK < QK)
                load_k(f + LOOK);
            else
                load_v(f + LOOK - QK);
            s1[f / KSTEPS] = mfma16(kf[f], qf[f % KSTEPS], s1[f / KSTEPS]);
            if constexpr (USE_R) s2[f / KSTEPS] = mfma16(kf[f], rf[f % KSTEPS], s2[f / KSTEPS]);
            __builtin_amdgcn_sched_barrier(0);
        }
        float factor = scale_log2;
        if (__builtin_expect(!whole, 0)) {  // (uniform)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool ok = (seen[e >> 3] >> (e & 7)) & 1u;
                s1[e >> 2][e & 3] = ok ? s1[e >> 2][e & 3] * factor : kNegInf;
                if (!ok) s2[e >> 2][e & 3] = 0.f;
            }
            factor = 1.f;
        }
        float tmax = kNegInf;
#pragma unroll
        for (int e = 0; e < 16; ++e) tmax = fmaxf(tmax, s1[e >> 2][e & 3]);
        tmax *= factor;
        if (__builtin_expect(__any(tmax > m_run + kWideSlack), 0)) {  // (rare, but for the first tile)
            tmax = rows_max(tmax);
            const float m_new = fmaxf(m_run, tmax);
            const float alpha = fast_exp2(m_run - (m_new == kNegInf ? 0.f : m_new));
            m_run = m_new;
            dsum1 *= alpha, dsum2 *= alpha;
#pragma unroll
            for (int i = 0; i < NDB; ++i) {
                o1[i] *= alpha;
                if constexpr (USE_R) o2[i] *= alpha;
            }
        }
        const float neg_m = m_run == kNegInf ? 0.f : -m_run;
        // P1 and P2 are rounded to bf16 once, as matrix operands; d1 and d2 add the rounded values, so that the
        // weights still sum to one (by the matrix instruction: four vector instructions a score less).
        u32x4 pb1[2], pb2[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 &x = s1[2 * h + (e >> 1)], &u = s2[2 * h + (e >> 1)];
                const int at = 2 * (e & 1);
                const float p0 = fast_exp2(fmaf(x[at], factor, neg_m)), p1 = fast_exp2(fmaf(x[at + 1], factor, neg_m));
                pb1[h][e] = pack_bf16(p0, p1);
                if constexpr (USE_R) pb2[h][e] = pack_bf16(p0 * u[at], p1 * u[at + 1]);
            }
            const u32x4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
            dsum1 = mfma16(ones, pb1[h], dsum1);
            if constexpr (USE_R) dsum2 = mfma16(ones, pb2[h], dsum2);
        }
#pragma unroll
        for (int f = 0; f < PV; ++f) {
            if (f + LOOK < PV) load_v(f + LOOK);
            o1[f % NDB] = mfma16(vt[f], pb1[f / NDB], o1[f % NDB]);
            if constexpr (USE_R) o2[f % NDB] = mfma16(vt[f], pb2[f / NDB], o2[f % NDB]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // Ring: at the top of a round the tiles v .. v + AHEAD - 1 are on their way; the wait leaves those behind v, the barrier
    // says that v has landed for all waves and that nobody reads tile v - 1 any more, whose stage takes tile v + AHEAD.
    int stage = 0, masked = 0;
    for (int v = v_lo; v < v_hi; ++v) {
        if (v + AHEAD <= v_hi)  // (uniform)
            tile_barrier<LOADS *(AHEAD - 1)>();
        else
            tile_barrier<0>();  // (the last tiles: all of them)
        if (v + AHEAD < v_hi) loader.issue(v + AHEAD, stage == 0 ? STAGES - 1 : stage - 1);
        u32x4 *tileK = lds + stage * STAGE_CHUNKS;
        const int tk = __builtin_amdgcn_readfirstlane(scope.key_of(v));
        const bool whole = scope.whole(tk, TILE);
        if (!whole) {  // (the same for all waves)
            if (loader.not_finite(tileK + TILE_CHUNKS) && lane == 0) some_bad[masked & 1] = 1;
#pragma unroll
            for (int h = 0; h < 2; ++h) seen[h] = scope.seen(P, col_nodes, col_lo, col_end, tk + 64 * kh + 32 * h, g);
            __syncthreads();
            const bool bad = some_bad[masked & 1] != 0;
            ++masked;
            if (tid == 0) some_bad[masked & 1] = 0;  // (read a masked tile ago; the next barrier is in front of its next use)
            if (__builtin_expect(bad, 0)) {
                if (live_wave)
#pragma unroll
                    for (int h = 0; h < 2; ++h) spread_not_finite(tileK + TILE_CHUNKS + (64 * kh + 32 * h) * CPR, seen[h]);
                __syncthreads();
                loader.clean(tileK + TILE_CHUNKS);
                __syncthreads();
            }
        }
        if (live_wave) tile(tileK + 64 * kh * CPR, whole);
        stage = stage == STAGES - 1 ? 0 : stage + 1;
    }

    // ---- the two halves of the keys (KH = 2); then the record or the output row --------------------------------
    const float e1 = dsum1[0], e2 = dsum2[0];
    float m_star = m_run, w0 = 1.f, w1 = 0.f, f1 = 0.f, f2 = 0.f;
    f32x4 *mine = (f32x4 *)lds + cw * (2 * NDB * 64) + lane;
    if constexpr (KH == 2) {
        __syncthreads();  // the ring is free (no load is in flight: the last round waited for all)
        if (kh == 1) {
            if (g == 0) head[cw][0][c] = m_run, head[cw][1][c] = e1, head[cw][2][c] = e2;
#pragma unroll
            for (int i = 0; i < NDB; ++i) {
                mine[i * 64] = o1[i];
                if constexpr (USE_R) mine[(NDB + i) * 64] = o2[i];
            }
        }
        __syncthreads();
        if (kh != 0) return;
        const float m1 = head[cw][0][c];
        f1 = head[cw][1][c], f2 = head[cw][2][c], m_star = fmaxf(m_run, m1);
        // (a reference of -inf with a sum that is not zero: scores of NaN only, which must reach the result)
        w0 = m_run == kNegInf && e1 == 0.f ? 0.f : fast_exp2(m_run - m_star);
        w1 = m1 == kNegInf && f1 == 0.f ? 0.f : fast_exp2(m1 - m_star);
    }
    if (x >= n_cols) return;
    // (a node behind the drafted ones sees nothing, also where all others see everything)
    const RowsColumn<D> column(p, b, hk, x, split, m_star, w0 * e1 + w1 * f1, w0 * e2 + w1 * f2, col_end == 0, g == 0);
#pragma unroll
    for (int i = 0; i < NDB; ++i) {
        f32x4 a1 = o1[i], a2 = o2[i];
        if constexpr (KH == 2) {
            a1 = w0 * a1 + w1 * mine[i * 64];
            if constexpr (USE_R) a2 = w0 * a2 + w1 * mine[(NDB + i) * 64];
        }
        column.store(16 * i + 4 * g, a1, a2);
    }
}

template <int D, bool USE_R, int CACHE>
static void launch_wide_columns(DecodeRowsParams P, hipStream_t stream) {
    const int n_cols = P.d.G * P.d.Tq, cols = decode_rows_columns(n_cols);
    P.col_groups = (n_cols + cols - 1) / cols;
    const int64_t units = ((int64_t)P.d.S * P.d.Hkv * P.d.B + 7) / 8 * 8;
    const dim3 grid((unsigned)(units * P.col_groups));
    auto run = [&](auto kh, auto tree) {
        hipLaunchKernelGGL((decode_rows_wide_kernel<D, USE_R, CACHE, decltype(kh)::value, decltype(tree)::value>), grid, dim3(512), 0, stream, P);
    };
    const std::integral_constant<int, 1> all_keys{};
    const std::integral_constant<int, 2> halves{};
    const std::true_type tree;
    const std::false_type chain;
    if (cols == 64)
        P.mask != nullptr ? run(halves, tree) : run(halves, chain);
    else
        P.mask != nullptr ? run(all_keys, tree) : run(all_keys, chain);
}

template <int D, bool USE_R>
static void launch_wide_cache(const DecodeRowsParams &P, hipStream_t stream) {
    const DecodeParams &p = P.d;
    const bool short_rows = p.ksl < (1 << 23) && p.vsl < (1 << 23);
    if (short_rows && p.block_table == nullptr)
        launch_wide_columns<D, USE_R, kRowsContiguous>(P, stream);
    else if (short_rows && p.page_size % 16 == 0)
        launch_wide_columns<D, USE_R, kRowsPagedRuns>(P, stream);
    else
        launch_wide_columns<D, USE_R, kRowsAny>(P, stream);
}

hipError_t launch_decode_rows_wide_bf16(const DecodeRowsParams &P, hipStream_t stream) {
    if (P.d.d == 128)
        P.d.use_r ? launch_wide_cache<128, true>(P, stream) : launch_wide_cache<128, false>(P, stream);
    else
        P.d.use_r ? launch_wide_cache<64, true>(P, stream) : launch_wide_cache<64, false>(P, stream);
    return hipGetLastError();
}

}  // namespace plx
