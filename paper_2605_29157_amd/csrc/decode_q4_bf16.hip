// Split-KV Parallax decode over a cache held in 4 bits (plx_q4.h has the row), bf16 queries, gfx950.
//
// What it computes: the forward of the paper (Sec. 3.1, Algorithm 1) over the key set J of each row,
//     p = softmax_J(scale q.k),  u = rho.k,  o = sum_J p (1 + sum_J p u - u) v,   empty J: zeros,
// with k and v the values that the codes and scales stand for, in one pass with the running state (m, d1, d2, O1, O2); splits and
// records as in decode_bf16.hip. J: the keys a row sees behind a window and sinks, or those in the blocks of a list.
//
// What bounds it: 9 D / 8 bytes a key (144 at D = 128, where bf16 takes 512) against the same 8 D flop per column and, beside them, the
// conversion of 2 D codes.
//
// Layout. As decode_rows_bf16.hip: four waves with 32-key tiles of their own, S^T = K [Q; R]^T on 16x16x32 MFMAs, P kept in its
// lane. What differs:
//   * a lane's 16 bytes (D = 128; D = 64: 8) of a K row are its operands of all k-steps: the order of the dimensions is the
//     product's to choose, so lane (key c, g) takes dimensions D / 4 g .. of its key, and q and rho are fetched to match. Codes become
//     bf16 (one conversion for two, with their scale: exact) as they are used.
//   * V has to be turned round (a lane's operand is 8 keys of one dimension), which its scales, one for each key, do not survive in
//     4 bits: it is converted first and goes through the wave's LDS tile as bf16.
#include "plx_q4.h"
#include "plx_rows.h"

namespace plx {

namespace {
constexpr int kQ4Tile = 32;  // keys per wave tile
constexpr int kQ4Waves = 4;
}  // namespace

template <int D, bool USE_R, int CACHE, bool LIST>
__global__ __launch_bounds__(256, 2) void decode_q4_kernel(DecodeRowsParams P) {
    const DecodeParams &p = P.d;
    using Row = Q4Row<D>;
    constexpr int CPR = D / 8;             // 16-byte chunks of a bf16 V row
    constexpr int KSTEPS = D / 32, NDB = D / 16;
    constexpr int TILE_CHUNKS = kQ4Tile * CPR;
    constexpr int KW = D / 32;             // dwords of K codes a lane has of a key (KSTEPS of them)
    constexpr int VLPR = D / 32;           // lanes of a row of V codes, 16 bytes each
    constexpr int VRPL = 64 / VLPR, NV = kQ4Tile / VRPL;  // rows of a load; loads
    __shared__ u32x4 lds[kQ4Waves * TILE_CHUNKS > 2 * kQ4Waves * NDB * 64 + 48 ? kQ4Waves * TILE_CHUNKS : 2 * kQ4Waves * NDB * 64 + 48];
    __shared__ TreeWords<0> no_words;

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int c = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int G = p.G, S = p.S, Tq = p.Tq, n_cols = G * Tq;

    const RowsScope<false, kQ4Tile, LIST> scope(P, b, 0, 16, hk);
    const int Lb = scope.Lb;
    // (splits in whole rounds of the four waves)
    const int per = ((scope.n_virtual + S - 1) / S + kQ4Waves - 1) / kQ4Waves * kQ4Waves;
    const int v_lo = split * per, v_hi = min(v_lo + per, scope.n_virtual);

    // ---- this lane's column: q and rho operands, key set ---------------------------------------------------
    u32x4 qf[KSTEPS], rf[KSTEPS];
    int col_end, col_lo;
    TreeRow col_nodes{};
    {
        const bool live = c < n_cols;
        const int t = live ? c / G : 0, h = live ? c - t * G : 0;
        const int64_t row = (((int64_t)b * p.Hq + (int64_t)hk * G + h) * Tq + t) * D + D / 4 * g;
        const __bf16 *qrow = (const __bf16 *)p.q + row, *rrow = (const __bf16 *)p.r + row;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            const u32x4 z = {0u, 0u, 0u, 0u};
            qf[s] = live ? *(const u32x4 *)(qrow + 8 * s) : z;
            if constexpr (USE_R) rf[s] = live ? *(const u32x4 *)(rrow + 8 * s) : z;
        }
        scope.column(P, no_words, 0, c, t, live, col_lo, col_end, col_nodes);
    }

    const char *base = (const char *)p.k + (p.block_table == nullptr ? (int64_t)b * p.ksb : 0) + (int64_t)hk * p.ksh;
    u32x4 *ldsV = lds + w * TILE_CHUNKS;
    const unsigned short *ldsV16 = (const unsigned short *)ldsV;
    const int32_t *table = p.block_table + (int64_t)b * p.table_stride;
    auto paged_offset = [&](int key) {
        const int page_no = key / p.page_size;
        const int64_t page = min(max(table[page_no], 0), p.num_pages - 1);
        return page * p.ksb + (int64_t)(key - page_no * p.page_size) * p.ksl;
    };
    const int last16 = max(Lb - 1, 0) & ~15;  // first key of the last half tile that exists
    const uint32_t row_bytes = (uint32_t)p.ksl;

    // ---- the wave's tiles --------------------------------------------------------------------------------
    // Keys and (runs) the halves' offsets of its next 32 tiles, lane 2 * j + half
    constexpr bool AHEAD = LIST || CACHE == kRowsPagedRuns;
    int ahead_key = 0, ahead_off[2] = {0, 0}, slot = 64;
    auto look_ahead = [&](int v) {
        const int key = scope.key_of(min(v + (lane >> 1) * kQ4Waves, scope.n_virtual - 1));
        ahead_key = key;
        if constexpr (CACHE != kRowsAny) {
            const int first = min(max(key, 0) + 16 * (lane & 1), last16);
            const int64_t off = CACHE == kRowsPagedRuns ? paged_offset(first) : (int64_t)first * p.ksl;
            ahead_off[0] = (int)off, ahead_off[1] = (int)(off >> 32);
        }
        slot = 0;
    };
    // The first tile at or behind number v: its key and the addresses of its halves (CACHE kRowsAny: not these)
    auto next_tile = [&](int &v, int &key, const char *(&half)[2]) -> bool {
        for (; v < v_hi; v += kQ4Waves) {
            if constexpr (AHEAD) {
                if (slot == 64) look_ahead(v);
                key = __builtin_amdgcn_readlane(ahead_key, slot);
                if constexpr (CACHE != kRowsAny)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf)
                        half[hf] = base + (((int64_t)__builtin_amdgcn_readlane(ahead_off[1], slot + hf) << 32) |
                                           (uint32_t)__builtin_amdgcn_readlane(ahead_off[0], slot + hf));
                slot += 2;
                if (LIST && key < 0) continue;
            } else {
                key = __builtin_amdgcn_readfirstlane(scope.key_of(v));
                if constexpr (CACHE != kRowsAny)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) half[hf] = base + (int64_t)min(key + 16 * hf, last16) * p.ksl;
            }
            return true;
        }
        return false;
    };
    // row of key `key` + 16 hf + i (rows past the sequence end: its last one, masked below)
    auto row_of = [&](int key, const char *const(&half)[2], int hf, int i) -> const char * {
        if constexpr (CACHE != kRowsAny) {
            const int last = Lb - 1 - min(key + 16 * hf, last16);
            return half[hf] + __umul24((uint32_t)min(i, last), row_bytes);
        } else {
            const int k = min(key + 16 * hf + i, Lb - 1);
            return base + (p.block_table != nullptr ? paged_offset(k) : (int64_t)k * p.ksl);
        }
    };
    uint32_t k_codes[2][KW], v_codes[NV][4], k_scales[2], v_scales[NV];
    auto issue = [&](int key, const char *const(&half)[2]) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const char *row = row_of(key, half, hf, c);
            if constexpr (D == 128) {
                const u32x4 x = *(const u32x4 *)(row + 16 * g);
#pragma unroll
                for (int s = 0; s < KW; ++s) k_codes[hf][s] = x[s];
                k_scales[hf] = *(const uint16_t *)(row + Row::kKScale + 2 * g);
            } else {
                const u32x2 x = *(const u32x2 *)(row + 8 * g);
#pragma unroll
                for (int s = 0; s < KW; ++s) k_codes[hf][s] = x[s];
                k_scales[hf] = *(const uint8_t *)(row + Row::kKScale + g);
            }
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = VRPL * n + lane / VLPR;
            const char *row = NV == 2 ? row_of(key, half, n, lane / VLPR) : (i < 16 ? row_of(key, half, 0, i & 15) : row_of(key, half, 1, i & 15));
            const u32x4 x = *(const u32x4 *)(row + Row::kV + 16 * (lane % VLPR));
#pragma unroll
            for (int e = 0; e < 4; ++e) v_codes[n][e] = x[e];
            v_scales[n] = *(const uint16_t *)(row + Row::kVScale + 2 * (lane % VLPR));
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

    int v = v_lo + w, key = 0;
    const char *half[2] = {base, base};
    bool have = next_tile(v, key, half);
    if (have) issue(key, half);
    while (have) {
        const int tk = key;
        const bool whole = scope.whole(tk, kQ4Tile);  // (uniform) every column sees all of the keys
        uint32_t kc[2][KW], ks[2];
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            ks[hf] = k_scales[hf];
#pragma unroll
            for (int s = 0; s < KW; ++s) kc[hf][s] = k_codes[hf][s];
        }
        bool any_bad = false;
        if (!whole) {  // scales above 252 stand for values that are not finite, or not in bf16
            bool bad = false;
#pragma unroll
            for (int n = 0; n < NV; ++n) bad = bad || (v_scales[n] & 255u) > 252u || (v_scales[n] >> 8) > 252u;
            any_bad = __any(bad);
        }
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = VRPL * n + lane / VLPR;
            const float lo = q4_scale(v_scales[n] & 255u), hi = q4_scale(v_scales[n] >> 8);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                ldsV[lds_chunk_slot<D>(i, 4 * (lane % VLPR) + e)] = q4_to_bf16(v_codes[n][e], e < 2 ? lo : hi);
        }
        v += kQ4Waves;
        have = next_tile(v, key, half);
        if (have) issue(key, half);
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
                for (int i = 0; i < TILE_CHUNKS / 64; ++i) {
                    u32x4 &x = ldsV[64 * i + lane];
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
            const float lo = q4_scale(ks[sub] & 255u), hi = q4_scale(ks[sub] >> 8);
#pragma unroll
            for (int s = 0; s < KSTEPS; ++s) {
                const u32x4 kf = q4_to_bf16(kc[sub][s], D == 64 || s < 2 ? lo : hi);
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
        // that the weights still sum to one.
        float p1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) p1[e] = fast_exp2(x[e] - m_use);
        dsum1 *= alpha;
        const u32x4 pb1 = pack8_bf16_accumulate(p1[0], p1[1], p1[2], p1[3], p1[4], p1[5], p1[6], p1[7], dsum1);
        u32x4 pb2 = {0u, 0u, 0u, 0u};
        if constexpr (USE_R) {
            float p2[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) p2[e] = (seen >> e) & 1u ? p1[e] * s2[e >> 2][e & 3] : 0.f;
            dsum2 *= alpha;
            pb2 = pack8_bf16_accumulate(p2[0], p2[1], p2[2], p2[3], p2[4], p2[5], p2[6], p2[7], dsum2);
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
            if constexpr (USE_R) o2[i] = mfma16(vt, pb2, o2[i]);
        }
        wave_lds_fence();
    }

    // ---- the four waves' states (in the order of the lanes' registers: no bank conflicts), then the record or the output row ----
    constexpr int QUADS = NDB * 64;  // of four dimensions: quad 64 i + lane' is column lane' % 16, dimensions 16 i + 4 (lane' / 16) ..
    f32x4 *mrg1 = (f32x4 *)lds, *mrg2 = mrg1 + kQ4Waves * QUADS;  // [wave][quad]
    float *mrg_m = (float *)(lds + 2 * kQ4Waves * QUADS), *mrg_d1 = mrg_m + kQ4Waves * 16, *mrg_d2 = mrg_d1 + kQ4Waves * 16;
    __syncthreads();  // every wave is done with its tiles
    {
        const float s1 = rows_sum(dsum1), s2 = rows_sum(dsum2);
        // a row in front of the sequence sees nothing, also where all others see everything
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
    float m_star = kNegInf, wt[kQ4Waves], d1 = 0.f, d2 = 0.f;
#pragma unroll
    for (int ww = 0; ww < kQ4Waves; ++ww) m_star = fmaxf(m_star, mrg_m[ww * 16 + c]);
#pragma unroll
    for (int ww = 0; ww < kQ4Waves; ++ww) {
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
        for (int ww = 0; ww < kQ4Waves; ++ww) {
            a1 += wt[ww] * mrg1[ww * QUADS + quad];
            if constexpr (USE_R) a2 += wt[ww] * mrg2[ww * QUADS + quad];
        }
        column.store(16 * (quad >> 6) + 4 * g, a1, a2);
    }
}

template <int D, bool USE_R, int CACHE>
static void launch_q4_form(const DecodeRowsParams &P, hipStream_t stream) {
    const dim3 grid(P.d.S, P.d.Hkv, P.d.B);
    if (P.block_list != nullptr)
        hipLaunchKernelGGL((decode_q4_kernel<D, USE_R, CACHE, true>), grid, dim3(256), 0, stream, P);
    else
        hipLaunchKernelGGL((decode_q4_kernel<D, USE_R, CACHE, false>), grid, dim3(256), 0, stream, P);
}

template <int D, bool USE_R>
static void launch_q4_cache(const DecodeRowsParams &P, hipStream_t stream) {
    const DecodeParams &p = P.d;
    const bool short_rows = p.ksl < (1 << 24);  // (24-bit products of a row number below 16 and the row stride)
    if (short_rows && p.block_table == nullptr)
        launch_q4_form<D, USE_R, kRowsContiguous>(P, stream);
    else if (short_rows && p.page_size % 16 == 0)
        launch_q4_form<D, USE_R, kRowsPagedRuns>(P, stream);
    else
        launch_q4_form<D, USE_R, kRowsAny>(P, stream);
}

hipError_t launch_decode_q4(const DecodeRowsParams &P, hipStream_t stream) {
    if (P.d.d == 128)
        P.d.use_r ? launch_q4_cache<128, true>(P, stream) : launch_q4_cache<128, false>(P, stream);
    else
        P.d.use_r ? launch_q4_cache<64, true>(P, stream) : launch_q4_cache<64, false>(P, stream);
    return hipGetLastError();
}

}  // namespace plx
