// Split-KV Parallax decode for several rows whose key sets differ, bf16, gfx950: drafted nodes that see the cache and
// their own ancestors (tree masks), rows with a sliding window and a few first tokens that stay visible (sinks), and rows that
// see the blocks of a list only. Here: up to 16 columns (rows x heads of a GQA group); decode_rows_wide_bf16.hip has the kernel for more.
//
// What it computes: the forward of the paper (Sec. 3.1, Algorithm 1) over the key set J of each row,
//     p = softmax_J(scale q.k),  u = rho.k,  o = sum_J p (1 + sum_J p u - u) v,   empty J: zeros,
// in one pass with the running state (m, d1, d2, O1, O2); the key range is split over workgroups whose records are
// merged as in App. C by the combine kernel of decode_bf16.hip (same record format).
//
// What bounds it: the bytes of K and V (a key costs 4 D bytes and 8 D flop per column, 32 flop a byte).
//
// Layout. As decode_bf16.hip: four waves, each with its own 32-key tiles (no barrier in the loop), K and V rows parked in
// registers one tile ahead and staged through the wave's own LDS tile, S^T = K [Q; R]^T on 16x16x32 MFMAs with the
// columns as MFMA columns, P kept in its lane; two workgroups per compute unit. What differs:
//   * the tiles walked are those of the sinks, then those from the first key any window reaches (RowsScope), or those of the
//     list's blocks: a wave looks the entries of its next 32 tiles up at once, like the pages, and goes past those that are none;
//   * tiles that every column sees completely take no masks. In the others a key that a column does not see must
//     not reach it whatever its row holds (unwritten rows, freed pages): scores are selected, not multiplied, and
//     values that are not finite are taken out of the V tile and reach the columns that do see their key
//     through a product that overflows (2^127 * 2^127), so those columns come out infinite or NaN.
#include "plx_rows.h"

namespace plx {

namespace {
constexpr int kRowsTile = 32;  // keys per wave tile
constexpr int kRowsWaves = 4;
}  // namespace

template <int D, bool USE_R, int CACHE, bool TREE, bool LIST = false>
__global__ __launch_bounds__(256, 2) void decode_rows_kernel(DecodeRowsParams P) {
    const DecodeParams &p = P.d;
    constexpr int CPR = D / 8;            // 16-byte chunks per K/V row
    constexpr int KPI = 64 / CPR;         // rows covered by one wave-wide 16-byte load
    constexpr int NLD = kRowsTile / KPI;  // loads per lane per tile and tensor
    constexpr int KSTEPS = D / 32, NDB = D / 16;
    constexpr int TILE_CHUNKS = kRowsTile * CPR;
    __shared__ u32x4 lds[kRowsWaves * 2 * TILE_CHUNKS + 48];  // tiles; at the end the states of 16 columns
    __shared__ TreeWords<TREE ? 16 : 0> tree_words;

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int c = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int G = p.G, S = p.S, Tq = p.Tq, n_cols = G * Tq;

    const RowsScope<TREE, kRowsTile, LIST> scope(P, b, 0, 16, hk);
    const int Lb = scope.Lb;
    // (splits in whole rounds of the four waves)
    const int per = ((scope.n_virtual + S - 1) / S + kRowsWaves - 1) / kRowsWaves * kRowsWaves;
    const int v_lo = split * per, v_hi = min(v_lo + per, scope.n_virtual);

    // ---- this lane's column: q and rho operands, key set ---------------------------------------------------
    u32x4 qf[KSTEPS], rf[KSTEPS];
    int col_end, col_lo;
    TreeRow col_nodes{};
    {
        const bool live = c < n_cols;
        const int t = live ? c / G : 0, h = live ? c - t * G : 0;
        const int64_t row = (((int64_t)b * p.Hq + (int64_t)hk * G + h) * Tq + t) * D;
        const __bf16 *qrow = (const __bf16 *)p.q + row, *rrow = (const __bf16 *)p.r + row;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            const u32x4 z = {0u, 0u, 0u, 0u};
            qf[s] = live ? *(const u32x4 *)(qrow + 8 * (4 * s + g)) : z;
            if constexpr (USE_R) rf[s] = live ? *(const u32x4 *)(rrow + 8 * (4 * s + g)) : z;
        }
        scope.column(P, tree_words, 0, c, t, live, col_lo, col_end, col_nodes);
    }

    const __bf16 *kbase = (const __bf16 *)p.k + (p.block_table == nullptr ? (int64_t)b * p.ksb : 0) + (int64_t)hk * p.ksh;
    const __bf16 *vbase = (const __bf16 *)p.v + (p.block_table == nullptr ? (int64_t)b * p.vsb : 0) + (int64_t)hk * p.vsh;
    u32x4 *ldsK = lds + w * (2 * TILE_CHUNKS), *ldsV = ldsK + TILE_CHUNKS;
    const unsigned short *ldsV16 = (const unsigned short *)ldsV;

    const int ld_row = lane / CPR, ld_chunk = lane % CPR;
    u32x4 kst[NLD], vst[NLD];
    const RowsPages pages(p, b);
    const int last16 = max(Lb - 1, 0) & ~15;  // first key of the last half tile that exists
    // kRowsPagedRuns: offsets of the halves of this wave's next 32 tiles, lane 2 * j + half
    constexpr bool RUNS = CACHE == kRowsPagedRuns || LIST;
    int run_k[2] = {0, 0}, run_v[2] = {0, 0}, run_slot = LIST ? 64 : 0, run_key = 0;  // LIST: and the keys
    auto lookup_runs = [&](int v) {
        const int ahead = min(v + (lane >> 1) * kRowsWaves, max(scope.n_virtual - 1, 0));
        int64_t ko, vo;
        int key = scope.key_of(ahead);
        if constexpr (LIST) run_key = key, key = max(key, 0);
        key = min(key + 16 * (lane & 1), last16);
        if constexpr (CACHE == kRowsContiguous)
            ko = (int64_t)key * p.ksl, vo = (int64_t)key * p.vsl;
        else if constexpr (CACHE == kRowsPagedRuns)
            pages.offsets(key, ko, vo);
        else
            ko = vo = 0;
        run_k[0] = (int)ko, run_k[1] = (int)(ko >> 32);
        run_v[0] = (int)vo, run_v[1] = (int)(vo >> 32);
        run_slot = 0;
    };
    const uint32_t k_row_bytes = (uint32_t)p.ksl * 2u, v_row_bytes = (uint32_t)p.vsl * 2u;
    int list_key = 0;  // LIST: of the tile that is loaded next
    auto list_tile = [&](int &v) {  // LIST: the first tile at or behind number v that there is
        for (; v < v_hi; v += kRowsWaves) {
            if (run_slot == 64) lookup_runs(v);  // (uniform)
            list_key = __builtin_amdgcn_readlane(run_key, run_slot);
            if (list_key >= 0) break;
            run_slot += 2;
        }
    };
    auto issue_loads = [&](int v) {
        const int tk0 = LIST ? list_key : scope.key_of(v);
        if constexpr (CACHE != kRowsAny) {
            if constexpr (CACHE == kRowsPagedRuns && !LIST)
                if (run_slot == 64) lookup_runs(v);  // (uniform)
            int l = lane;
            asm volatile("" : "+v"(l));  // (the lane's offsets are worked out here: kept across the loop they would be spilled)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const int key0 = __builtin_amdgcn_readfirstlane(min(tk0 + 16 * hf, last16));
                int64_t ko = (int64_t)key0 * p.ksl, vo = (int64_t)key0 * p.vsl;
                if constexpr (RUNS) {
                    auto pick = [&](const int(&x)[2]) {
                        return ((int64_t)__builtin_amdgcn_readlane(x[1], run_slot + hf) << 32) |
                               (uint32_t)__builtin_amdgcn_readlane(x[0], run_slot + hf);
                    };
                    ko = pick(run_k), vo = pick(run_v);
                }
                const char *kp = (const char *)(kbase + ko), *vp = (const char *)(vbase + vo);
                const int last = Lb - 1 - key0;  // rows past the sequence end re-read its last row (masked below)
#pragma unroll
                for (int i = 0; i < NLD / 2; ++i) {
                    const uint32_t row = (uint32_t)min(i * KPI + l / CPR, last);
                    kst[hf * (NLD / 2) + i] = *(const u32x4 *)(kp + (__umul24(row, k_row_bytes) + 16u * (uint32_t)(l % CPR)));
                    vst[hf * (NLD / 2) + i] = *(const u32x4 *)(vp + (__umul24(row, v_row_bytes) + 16u * (uint32_t)(l % CPR)));
                }
            }
            run_slot += 2;
        } else {
#pragma unroll
            for (int i = 0; i < NLD; ++i) {
                const int key = min(tk0 + i * KPI + ld_row, Lb - 1);
                int64_t ko = (int64_t)key * p.ksl, vo = (int64_t)key * p.vsl;
                if (p.block_table != nullptr) pages.offsets(key, ko, vo);  // (uniform)
                kst[i] = *(const u32x4 *)(kbase + ko + ld_chunk * 8);
                vst[i] = *(const u32x4 *)(vbase + vo + ld_chunk * 8);
            }
            if constexpr (LIST) run_slot += 2;
        }
    };

    // ---- running state (per lane: its column, partial over this lane's keys) --------------------------------
    float m_run = kNegInf, dsum1 = 0.f, dsum2 = 0.f;
    f32x4 o1[NDB], o2[NDB];
#pragma unroll
    for (int i = 0; i < NDB; ++i) o1[i] = o2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float scale_log2 = p.scale * kLog2e;
    // A operand of O^T += V^T P^T for 16 output dimensions: the 8 keys of this lane's B operand
    const int tr_key = 4 * g + (c >> 2), tr_half = (c & 1) * 4;
    auto v_fragment = [&](int i) __attribute__((always_inline)) {
        const int chunk = 2 * i + ((c & 3) >> 1);
        const u32x2 lo = lds_read_tr16(ldsV16 + lds_chunk_slot<D>(tr_key, chunk) * 8 + tr_half);
        const u32x2 hi = lds_read_tr16(ldsV16 + lds_chunk_slot<D>(16 + tr_key, chunk) * 8 + tr_half);
        return u32x4{lo[0], lo[1], hi[0], hi[1]};
    };
    // lanes exchange data through LDS inside one wave: LDS executes a wave's accesses in
    // order, the fence only stops the compiler from moving reads above the writes
    auto wave_lds_fence = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };

    int v = v_lo + w;
    if constexpr (LIST) list_tile(v);
    if (v < v_hi) {
        if constexpr (CACHE == kRowsPagedRuns && !LIST) lookup_runs(v);
        issue_loads(v);
    }
    for (int v_next; v < v_hi; v = v_next) {
        const int tk = LIST ? list_key : __builtin_amdgcn_readfirstlane(scope.key_of(v));
        v_next = v + kRowsWaves;
        const bool whole = scope.whole(tk, kRowsTile);  // (uniform) every column sees all of the keys
        bool any_bad = false;
        if (!whole) {
            uint32_t bad = 0;
#pragma unroll
            for (int i = 0; i < NLD; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) bad |= not_finite_halves(vst[i][e]);
            any_bad = __any(bad != 0);
        }
        int l = lane;
        asm volatile("" : "+v"(l));  // (as above)
#pragma unroll
        for (int i = 0; i < NLD; ++i) {
            const int slot = lds_chunk_slot<D>(i * KPI + l / CPR, l % CPR);
            ldsK[slot] = kst[i];
            ldsV[slot] = vst[i];
        }
        if constexpr (LIST) list_tile(v_next);
        if (v_next < v_hi) issue_loads(v_next);
        wave_lds_fence();
        uint32_t seen = 0xffu;
        if (!whole) {
            seen = scope.seen(P, col_nodes, col_lo, col_end, tk, g);
            if (__builtin_expect(any_bad, 0)) {
                // values that are not finite: into the columns that see their key, and out of the V tile
                const u32x4 big = big_halves(seen);
#pragma unroll
                for (int i = 0; i < NDB; ++i) {
                    u32x4 bad = v_fragment(i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) bad[e] = not_finite_halves(bad[e]) & kBigHalves;
                    o1[i] = mfma16(bad, big, o1[i]);
                }
                wave_lds_fence();
#pragma unroll
                for (int i = 0; i < NLD; ++i) {
                    u32x4 &x = ldsV[lds_chunk_slot<D>(i * KPI + ld_row, ld_chunk)];
                    u32x4 y = x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[e] &= ~not_finite_halves(y[e]);
                    x = y;
                }
                wave_lds_fence();
            }
        }
        f32x4 s1[2], s2[2];
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
            s1[sub] = s2[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) {
                const u32x4 kf = ldsK[lds_chunk_slot<D>(16 * sub + c, 4 * s + g)];
                s1[sub] = mfma16(kf, qf[s], s1[sub]);
                if constexpr (USE_R) s2[sub] = mfma16(kf, rf[s], s2[sub]);
            }
        }
        float x[8], tmax = kNegInf;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] = (seen >> e) & 1u ? s1[e >> 2][e & 3] * scale_log2 : kNegInf;
            tmax = fmaxf(tmax, x[e]);
        }
        tmax = rows_max(tmax);
        const float m_new = fmaxf(m_run, tmax), m_use = m_new == kNegInf ? 0.f : m_new;
        const float alpha = fast_exp2(m_run - m_use);  // 0 on the first tile that is seen
        m_run = m_new;
        // P1 and P2 are rounded to bf16 once, as matrix operands; d1 and d2 add the rounded values, so
        // that the weights still sum to one. LIST: what the rounding takes is multiplied too (without it the result's error is
        // 1.4 times that of its own rounding; 16 x 8 lists of 64 blocks 58.1 us, with it 59.1).
        u32x4 rest1 = {0u, 0u, 0u, 0u}, rest2 = rest1;
        auto split = [&](const float(&x)[8], u32x4 &rest, float &sum) {
            u32x4 y;
            if constexpr (LIST) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t pair = pack_bf16(x[2 * e], x[2 * e + 1]);
                    const uint32_t left = pack_bf16(x[2 * e] - bf16_lo_f32(pair), x[2 * e + 1] - bf16_hi_f32(pair));
                    sum = add_bf16_pair(left, add_bf16_pair(pair, sum)), y[e] = pair, rest[e] = left;
                }
            } else {
                y = pack8_bf16_accumulate(x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7], sum);
            }
            return y;
        };
        float p1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p1[e] = fast_exp2(x[e] - m_use);
        dsum1 *= alpha;
        const u32x4 pb1 = split(p1, rest1, dsum1);
        u32x4 pb2 = {0u, 0u, 0u, 0u};
        if constexpr (USE_R) {
            float p2[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p2[e] = (seen >> e) & 1u ? p1[e] * s2[e >> 2][e & 3] : 0.f;
            dsum2 *= alpha;
            pb2 = split(p2, rest2, dsum2);
        }
        if (!__all(alpha == 1.f)) {
#pragma unroll
            for (int i = 0; i < NDB; ++i) {
                o1[i] *= alpha;
                if constexpr (USE_R) o2[i] *= alpha;
            }
        }
#pragma unroll
        for (int i = 0; i < NDB; ++i) {
            const u32x4 vt = v_fragment(i);
            o1[i] = mfma16(vt, pb1, o1[i]);
            if constexpr (LIST) o1[i] = mfma16(vt, rest1, o1[i]);
            if constexpr (USE_R) o2[i] = mfma16(vt, pb2, o2[i]);
            if constexpr (LIST && USE_R) o2[i] = mfma16(vt, rest2, o2[i]);
        }
        wave_lds_fence();
    }

    // ---- the four waves' states (in the order of the lanes' registers: no bank conflicts), then the record or the output row ----
    constexpr int QUADS = NDB * 64;  // of four dimensions: quad 64 i + lane' is column lane' % 16, dimensions 16 i + 4 (lane' / 16) ..
    f32x4 *mrg1 = (f32x4 *)lds, *mrg2 = mrg1 + kRowsWaves * QUADS;  // [wave][quad]
    float *mrg_m = (float *)(lds + kRowsWaves * 2 * TILE_CHUNKS), *mrg_d1 = mrg_m + kRowsWaves * 16, *mrg_d2 = mrg_d1 + kRowsWaves * 16;
    static_assert(2 * kRowsWaves * QUADS <= kRowsWaves * 2 * TILE_CHUNKS, "the states of four waves");
    __syncthreads();  // every wave is done with its tiles
    {
        const float s1 = rows_sum(dsum1), s2 = rows_sum(dsum2);
        // a node behind the sequence's drafted ones sees nothing, also where all others see everything
        const bool none = col_end == 0;
        if (g == 0) {
            mrg_m[w * 16 + c] = none ? kNegInf : m_run;
            mrg_d1[w * 16 + c] = none ? 0.f : s1;
            mrg_d2[w * 16 + c] = none ? 0.f : s2;
        }
#pragma unroll
        for (int i = 0; i < NDB; ++i) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            mrg1[w * QUADS + 64 * i + lane] = none ? zero : o1[i];
            if constexpr (USE_R) mrg2[w * QUADS + 64 * i + lane] = none ? zero : o2[i];
        }
    }
    __syncthreads();
    if (c >= n_cols) return;  // (a thread's column is the same in all of its quads)
    float m_star = kNegInf, wt[kRowsWaves], d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int ww = 0; ww < kRowsWaves; ++ww) m_star = fmaxf(m_star, mrg_m[ww * 16 + c]);
#pragma unroll
    for (int ww = 0; ww < kRowsWaves; ++ww) {
        // (a reference of -inf with a sum that is not zero: scores of NaN only, which must reach the result)
        const float mw = mrg_m[ww * 16 + c], dw = mrg_d1[ww * 16 + c];
        wt[ww] = mw == kNegInf && dw == 0.f ? 0.f : fast_exp2(mw - m_star);
        d1 += wt[ww] * dw;
        d2 += wt[ww] * mrg_d2[ww * 16 + c];
    }
    const RowsColumn<D> column(p, b, hk, c, split, m_star, d1, d2, false, w == 0 && g == 0);
#pragma unroll
    for (int quad = tid; quad < QUADS; quad += 256) {
        f32x4 a1 = {0.f, 0.f, 0.f, 0.f}, a2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ww = 0; ww < kRowsWaves; ++ww) {
            a1 += wt[ww] * mrg1[ww * QUADS + quad];
            if constexpr (USE_R) a2 += wt[ww] * mrg2[ww * QUADS + quad];
        }
        column.store(16 * (quad >> 6) + 4 * g, a1, a2);
    }
}

// The records of a row, up to N of them: D / 4 lanes a row, all loads at once, no exchange between lanes. The merge of
// decode_bf16.hip, a workgroup a row, is for many records; with many rows it is bound by the workgroups' starts: 6656 rows x
// 2 records 18.3 us, 8192 x 4 23.8; here 5.0 and 6.6, 8192 x 8 11.6 (few rows: 4 us with either).
template <int D, int N>
__global__ __launch_bounds__(256) void rows_combine_kernel(DecodeParams p) {
    constexpr int DL = D / 4, REC = 2 * D + 4;
    const int64_t row = (int64_t)blockIdx.x * (256 / DL) + threadIdx.x / DL;
    if (row >= (int64_t)p.B * p.Hq * p.Tq) return;
    const int dim = 4 * (threadIdx.x % DL);
    f32x4 head[N], a1[N], a2[N];
#pragma unroll
    for (int s = 0; s < N; ++s) {  // (past the last one: that again, with no weight)
        const float *rec = p.ws + (row * p.S + min(s, p.S - 1)) * REC;
        head[s] = *(const f32x4 *)rec;
        a1[s] = *(const f32x4 *)(rec + 4 + dim);
        a2[s] = *(const f32x4 *)(rec + 4 + D + dim);
    }
    float m_star = kNegInf, d1 = 0.f, d2 = 0.f;
    f32x4 o1 = {0.f, 0.f, 0.f, 0.f}, o2 = o1;
#pragma unroll
    for (int s = 0; s < N; ++s) m_star = fmaxf(m_star, head[s][0]);
#pragma unroll
    for (int s = 0; s < N; ++s) {
        const float w = s >= p.S || head[s][0] == kNegInf ? 0.f : fast_exp2(head[s][0] - m_star);
        d1 += w * head[s][1], d2 += w * head[s][2];
        o1 += w * a1[s], o2 += w * a2[s];
    }
    f32x4 y = {0.f, 0.f, 0.f, 0.f};  // empty key set: zeros
    if (d1 != 0.f) {
        const float inv = 1.f / d1;
        y = o1 * (inv * (1.f + d2 * inv)) - o2 * inv;
    }
    *(u32x2 *)((__bf16 *)p.o + row * D + dim) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
}

template <int D>
static void launch_rows_combine(const DecodeParams &p, int64_t rows, hipStream_t stream) {
    const dim3 grid((unsigned)((rows * (D / 4) + 255) / 256));
    if (p.S <= 2)
        hipLaunchKernelGGL((rows_combine_kernel<D, 2>), grid, dim3(256), 0, stream, p);
    else if (p.S <= 4)
        hipLaunchKernelGGL((rows_combine_kernel<D, 4>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((rows_combine_kernel<D, 8>), grid, dim3(256), 0, stream, p);
}

hipError_t launch_decode_rows_combine(const DecodeParams &p, hipStream_t stream) {
    const int64_t rows = (int64_t)p.B * p.Hq * p.Tq;
    if (p.S > 8) return launch_decode_combine(p, stream);
    p.d == 128 ? launch_rows_combine<128>(p, rows, stream) : launch_rows_combine<64>(p, rows, stream);
    return hipGetLastError();
}

// Columns per workgroup: 16 with private tiles, 64 or 128 with shared ones. (Private tiles with 32 columns a wave, one
// workgroup per unit, took 26 nodes x 2 heads over 16 x 6000 keys, which the columns read twice, in 135 us.)
int decode_rows_columns(int n_cols) { return n_cols <= 16 ? 16 : n_cols <= 64 ? 64 : 128; }
int decode_rows_tile(int columns) { return columns == 64 ? 128 : 64; }

template <int D, bool USE_R, int CACHE>
static void launch_rows_form(const DecodeRowsParams &P, hipStream_t stream) {
    const dim3 grid(P.d.S, P.d.Hkv, P.d.B);
    if (P.block_list != nullptr)
        hipLaunchKernelGGL((decode_rows_kernel<D, USE_R, CACHE, false, true>), grid, dim3(256), 0, stream, P);
    else if (P.mask != nullptr)
        hipLaunchKernelGGL((decode_rows_kernel<D, USE_R, CACHE, true>), grid, dim3(256), 0, stream, P);
    else
        hipLaunchKernelGGL((decode_rows_kernel<D, USE_R, CACHE, false>), grid, dim3(256), 0, stream, P);
}

template <int D, bool USE_R>
static void launch_rows_cache(const DecodeRowsParams &P, hipStream_t stream) {
    const DecodeParams &p = P.d;
    const bool short_rows = p.ksl < (1 << 23) && p.vsl < (1 << 23);  // (24-bit products, see decode_bf16.hip)
    if (short_rows && p.block_table == nullptr)
        launch_rows_form<D, USE_R, kRowsContiguous>(P, stream);
    else if (short_rows && p.page_size % 16 == 0)
        launch_rows_form<D, USE_R, kRowsPagedRuns>(P, stream);
    else
        launch_rows_form<D, USE_R, kRowsAny>(P, stream);
}

hipError_t launch_decode_rows_bf16(const DecodeRowsParams &P, hipStream_t stream) {
    if (decode_rows_columns(P.d.G * P.d.Tq) > 16) return launch_decode_rows_wide_bf16(P, stream);
    if (P.d.d == 128)
        P.d.use_r ? launch_rows_cache<128, true>(P, stream) : launch_rows_cache<128, false>(P, stream);
    else
        P.d.use_r ? launch_rows_cache<64, true>(P, stream) : launch_rows_cache<64, false>(P, stream);
    return hipGetLastError();
}

}  // namespace plx
