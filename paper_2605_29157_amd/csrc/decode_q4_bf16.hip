// Split-KV Parallax decode over a cache held in 4 bits (plx_q4.h has the row), bf16 queries, gfx950.
//
// What it computes: the forward of the paper (Sec. 3.1, Algorithm 1) over the key set J of each row,
//     p = softmax_J(scale q.k),  u = rho.k,  o = sum_J p (1 + sum_J p u - u) v,   empty J: zeros,
// with k and v the values that the codes and scales stand for, in one pass with the running state (m, d1, d2, O1, O2); splits and
// records as in decode_bf16.hip. J: the keys a row sees behind a window and sinks, or those in the blocks of a list.
//
// What bounds it: 9 D / 8 bytes a key (144 at D = 128, where bf16 takes 512) against the same 8 D flop per column; beside them the
// conversion of 2 D codes, and LDS.
//
// Layout. Four waves with 64-key tiles of their own (no barrier in the loop), S^T = K [Q; R]^T on 16x16x32 MFMAs, P kept in its
// lane, as decode_bf16.hip. A tile comes into LDS as it is (direct loads, 1 KB each, two tiles a wave: one is worked on while the other is
// on its way), and the codes stay codes until they are operands:
//   * K: a lane's 16 bytes (D = 64: 8) of a row are its operands of all k-steps: the order of the dimensions is the product's to
//     choose, so lane (key c, g) takes dimensions D / 4 g .. of its key, and q and rho are fetched to match. Codes become bf16
//     with their scale, two in one conversion, exactly.
//   * V has to be turned round (a lane's operand is 8 keys of one dimension): the 4-bit transposing read gives a lane 16 keys of its
//     dimension at once, but a scale serves 16 dimensions of one key, so it cannot be applied there. It goes to the other side of
//     the product, P: of the 16 columns of the matrix only those of the group's heads x rows are needed, and the copies of such a
//     column hold P times the scales of one group of 16 dimensions each: 8 groups x 2 columns at D = 128 (C = 2). The product for a
//     group's dimensions is right in its own copy only, and only that is kept. With more columns (C) the groups do not fit beside each
//     other and P is multiplied 2, 4 or 8 times. A key that a column does not see has the scale 0, so nothing in its row can reach it.
// P. One rounding of it to bf16 makes the result's error 1.4 times that of its own rounding; f16 has the bits but not the range, and bf16 for
// what the rounding leaves costs as many products again. So a tile is looked at first. Where f16 holds its operands (scales within 2^8
// of each other, each column's largest weight not 2^16 below the row's, P rho.k not too large) they are f16, the scales as exponents,
// and what a product loses is at most 2^-13 of the tile's largest one in that column and group. Any other tile (values or
// products rho.k of other sizes beside each other, rows with a few heavy keys, NaN; at d = 128 also the ends of a sequence or window) takes its P in
// two bf16, with scales of any size. O1 and O2 count in the same unit either way, so the two kinds of tile mix.
// us, 16 x 32768 keys, 8 key heads, d = 128, at the best split, for 2, 4, 8, 16 columns: all tiles in f16 with references that followed the largest scale
// (and lost smaller ones) 116, 117, 120, 124; now 117, 119, 122, 131; all tiles in two bf16, as they are where scores have a standard deviation
// of 12, 142, 164, 195, 255. Ends of sequences in f16, too: d = 64, window 4096, 4 rows 22.6 us, so 21.4; at d = 128 100 x <= 500 keys 25.4 and
// 23.5, but the compiler then spills registers of the second way, and 16 x 64 listed blocks take 26.5 instead of 25.0.
// Steps before that, us for 16 x 32768 keys, 8 key heads, d = 128, and for 1 x 65536 at 8 splits (a workgroup a unit, 64 units): tiles in registers, V as bf16
// through LDS, 32 keys at a time 130 and 81; two tiles in LDS 117, 77; 64 keys at a time, no bank conflicts 116, 61 (now bound by
// LDS: 16 KB of V written at 64 bytes a cycle, and every read costs 6); scales with P instead 115, 50; scales out of their bytes by one
// instruction 111, 48.5 (the loads alone, without any arithmetic, 106).
#include "plx_lds_dma.h"
#include "plx_q4.h"
#include "plx_rows.h"

namespace plx {

namespace {
constexpr int kQ4Tile = 64;  // keys per wave tile
constexpr int kQ4Waves = 4;
// Exponents of 2. Weights are held times 2^13 and may grow by 2^2 before their reference moves, P rho.k times 2^7 (rho times 2^-6). Tiles of f16:
// scales down to 2^8 below the largest, weights whose largest is not below 2^-16, P rho.k below 2^15.
constexpr float kQ4Slack = 2.f, kWeightFloor = 16.f;
constexpr int kWeightUp = 13, kProbeDown = 6, kScaleRange = 8, kProbeMost = 15;
constexpr int kRecordDown = 8;  // in a record weights are 2^8 lower: times the largest values they are finite

// How the rows of a tile are found: 64 that follow each other in memory, counted from the start of the cache or looked up ahead
// (lists; pages of a multiple of 64), four runs of 16 (other pages of a multiple of 16), eight of 8 likewise, or row by row.
enum Q4Form { kQ4Direct, kQ4Runs64, kQ4Runs16, kQ4Runs8, kQ4Any };

// The tiles of a workgroup: those of a list's blocks, or RowsScope's
struct Q4Scope : RowsScope<false, kQ4Tile> {
    const int32_t *list;
    __device__ __forceinline__ Q4Scope(const DecodeRowsParams &P, int b, int hk) : RowsScope<false, kQ4Tile>(P, b, 0, 16), list(nullptr) {
        static_assert(kListBlock == kQ4Tile, "a tile is a block");
        if (P.block_list != nullptr) {
            list = P.block_list + ((int64_t)b * P.d.Hkv + hk) * P.n_list;
            n_virtual = Lb > 0 ? P.n_list : 0;
        }
    }
    __device__ __forceinline__ int key_of(int v) const {
        return list != nullptr ? listed_key<kQ4Tile>(list, v, Lb) : RowsScope<false, kQ4Tile>::key_of(v);
    }
};

// x of the lane whose number in its row of 16 is 4 less (or 12 more), in the banks of 4 lanes of BANKS; the others keep `old`
template <int BANKS>
__device__ __forceinline__ uint32_t from_other_quad(uint32_t old, uint32_t x) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)old, (int)x, 0x124, 0xf, BANKS, false);  // row_ror:4
}
// Bits of the 16 lanes of a row together, and the largest number of theirs
__device__ __forceinline__ uint32_t row_or(uint32_t x) {
    x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true);  // row_ror:8
    x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true);
    x |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, true);
    return x | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, true);
}
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x124, 0xf, 0xf, true));
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x122, 0xf, 0xf, true));
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x121, 0xf, 0xf, true));
}
template <int A, int B>
__device__ __forceinline__ uint32_t from_quad(uint32_t x) {  // lanes A, B, A, B of the quad
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, A | B << 2 | A << 4 | B << 6, 0xf, 0xf, true);
}
// A number cut to the 16 bits of mantissa that two bf16 hold
__device__ __forceinline__ float cut(float x) { return __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, x) & 0xffffff00u); }
// The upper bf16 of two such numbers, and what they leave
__device__ __forceinline__ void halves(float a, float b, u32x4 &upper_halves, u32x4 &rest, int i) {
    auto upper = [](float lo, float hi) {
        return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
    };
    const uint32_t big = upper(a, b);
    upper_halves[i] = big, rest[i] = upper(a - bf16_lo_f32(big), b - bf16_hi_f32(big));
}
// Group (16 dimensions) 16 / C * J + c % (16 / C) of the scales for operand J of C columns. own: the tr_b8 read's, D = 128: group c % 8,
// D = 64: scales of K (c % 8 < 4) and then of V.
template <int D, int C, int J>
__device__ __forceinline__ uint32_t operand_scales(uint32_t own) {
    if constexpr (D == 128 && C == 2) return own;
    // groups 4 h + c % 4 of V
    constexpr int H = D == 128 ? 16 / C * J / 4 : 1;
    const uint32_t x = from_other_quad<H == 0 ? 0xA : 0x5>(own, own);
    if constexpr (C == 4) return x;
    if constexpr (C == 8) return from_quad<2 * (J & 1), 2 * (J & 1) + 1>(x);
    return from_quad<J & 3, J & 3>(x);
}
}  // namespace

// C: columns (rows x heads of a group) there is room for, 2 (D = 128 only), 4, 8 or 16
template <int D, int C, bool USE_R, int FORM>
__global__ __launch_bounds__(256, 2) void decode_q4_kernel(DecodeRowsParams P) {
    const DecodeParams &p = P.d;
    using Row = Q4Row<D>;
    constexpr int KSTEPS = D / 32, NDB = D / 16;
    constexpr int REP = 16 / C, OPERANDS = NDB / REP;  // matrix columns of a column; sets of them
    static_assert(REP <= NDB, "no more copies than groups of dimensions");
    constexpr int RPC = Row::kBytes / 16;            // 16-byte chunks of a row
    constexpr int RAW = kQ4Tile * RPC;               // ... of a tile
    constexpr bool FOLLOWING = FORM < kQ4Runs8;  // a load's rows follow each other in memory
    constexpr int RUNS = FORM == kQ4Runs8 ? 8 : FORM == kQ4Runs16 ? 4 : 1;  // of rows that follow each other
    constexpr int RUN = FOLLOWING ? RAW / RUNS : RAW;                       // chunks whose loads have an address of their own
    constexpr int FULL = RUN / 64, REST = RUN % 64, LOADS = FULL + (REST != 0);  // of a run
    static_assert(REST == 0 || REST == 16, "the last load of 16 rows takes 16 lanes");
    __shared__ u32x4 lds[kQ4Waves * 2 * RAW + 48];  // two tiles a wave; at the end the states of 16 columns
    static_assert(2 * NDB * 64 <= 2 * RAW, "the states of four waves");
    __shared__ TreeWords<0> no_words;

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int c = lane & 15, g = lane >> 4;
    const int split = blockIdx.x, hk = blockIdx.y, b = blockIdx.z;
    const int G = p.G, S = p.S, Tq = p.Tq, n_cols = G * Tq;

    const Q4Scope scope(P, b, hk);
    const int Lb = scope.Lb;
    // (splits in whole rounds of the four waves)
    const int per = ((scope.n_virtual + S - 1) / S + kQ4Waves - 1) / kQ4Waves * kQ4Waves;
    const int v_lo = split * per, v_hi = min(v_lo + per, scope.n_virtual);

    // ---- this lane's column: q and rho operands, key set ---------------------------------------------------
    u32x4 qf[KSTEPS], rf[KSTEPS];
    {
        const int col = c / REP;
        const bool live = col < n_cols;
        const int t = live ? col / G : 0, h = live ? col - t * G : 0;
        const int64_t row = (((int64_t)b * p.Hq + (int64_t)hk * G + h) * Tq + t) * D + D / 4 * g;
        const __bf16 *qrow = (const __bf16 *)p.q + row, *rrow = (const __bf16 *)p.r + row;
#pragma unroll
        for (int s = 0; s < KSTEPS; ++s) {
            const u32x4 z = {0u, 0u, 0u, 0u};
            qf[s] = live ? *(const u32x4 *)(qrow + 8 * s) : z;
            if constexpr (USE_R) rf[s] = live ? *(const u32x4 *)(rrow + 8 * s) : z;
        }
    }
    TreeRow no_nodes{};
    auto key_set = [&](int column, int &lo, int &end) {  // of matrix column `column`
        const int col = column / REP;
        const bool live = col < n_cols;
        scope.column(P, no_words, 0, column, live ? col / G : 0, live, lo, end, no_nodes);
    };

    constexpr int ADDRESSES = FOLLOWING ? RUNS : 1;
    const char *base = (const char *)p.k + (p.block_table == nullptr ? (int64_t)b * p.ksb : 0) + (int64_t)hk * p.ksh;
    u32x4 *raw = lds + w * 2 * RAW;
    const int32_t *table = p.block_table + (int64_t)b * p.table_stride;
    auto offset_of = [&](int key) -> int64_t {
        if (FORM == kQ4Direct || p.block_table == nullptr) return (int64_t)key * p.ksl;
        int page_size = p.page_size;
        if constexpr (FORM == kQ4Any && C == 16) asm volatile("" : "+s"(page_size));  // (no register to keep its reciprocal in)
        const int page_no = key / page_size;
        const int64_t page = min(max(table[page_no], 0), p.num_pages - 1);
        return page * p.ksb + (int64_t)(key - page_no * page_size) * p.ksl;
    };
    const uint32_t row_bytes = (uint32_t)p.ksl;

    // ---- the wave's tiles --------------------------------------------------------------------------------
    // Keys and offsets of the runs of its next 64 / RUNS tiles, lane RUNS * j + run
    int ahead_key = 0, ahead_off[2] = {0, 0}, slot = 64;
    auto look_ahead = [&](int v) {
        const int key = scope.key_of(min(v + lane / RUNS * kQ4Waves, scope.n_virtual - 1));
        ahead_key = key;
        if constexpr (FORM != kQ4Any) {
            // (runs behind the last token: the one that it is in)
            constexpr int LENGTH = RUNS == 8 ? 8 : 16;
            const int64_t off = offset_of(min(max(key, 0) + LENGTH * (lane % RUNS), (Lb - 1) & ~(LENGTH - 1)));
            ahead_off[0] = (int)off, ahead_off[1] = (int)(off >> 32);
        }
        slot = 0;
    };
    // The first tile at or behind number v: its key and the addresses of its runs (kQ4Any: the offset of this lane's row)
    int64_t row_off = 0;
    auto next_tile = [&](int &v, int &key, const char *(&run)[ADDRESSES]) -> bool {
        for (; v < v_hi; v += kQ4Waves) {
            if constexpr (FORM != kQ4Direct) {
                if (slot == 64) look_ahead(v);
                key = __builtin_amdgcn_readlane(ahead_key, slot);
                if constexpr (FOLLOWING)
#pragma unroll
                    for (int i = 0; i < RUNS; ++i)
                        run[i] = base + (((int64_t)__builtin_amdgcn_readlane(ahead_off[1], slot + i) << 32) |
                                         (uint32_t)__builtin_amdgcn_readlane(ahead_off[0], slot + i));
                slot += RUNS;
                if (key < 0) continue;  // (an entry of a list that is passed over)
                if constexpr (FORM == kQ4Any) row_off = offset_of(min(key + lane, Lb - 1));
            } else {
                key = __builtin_amdgcn_readfirstlane(scope.key_of(v));
                run[0] = base + (int64_t)key * p.ksl;
            }
            return true;
        }
        return false;
    };
    // Chunk n of a run is chunk n % RPC of its row n / RPC; this lane's of load i is n = 64 i + lane. Many columns leave no registers for all of
    // them: 16 n where rows follow each other without a gap, else worked out for every tile
    constexpr bool KEPT = C < 8;
    uint32_t chunk_off[LOADS];
    if constexpr (FOLLOWING && KEPT)
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t n = 64 * i + lane;
            chunk_off[i] = __umul24(n / RPC, row_bytes) + 16 * (n % RPC);
        }
    // A tile's rows on their way into stage 0 or 1 (rows past the sequence end: its last one, masked below)
    const uint32_t raw_address = lds_byte_address(raw);
    auto issue = [&](int key, const char *const(&run)[ADDRESSES], int stage) {
        const uint32_t to = raw_address + 16 * RAW * stage;
        if constexpr (FOLLOWING) {
            const bool exists = key + kQ4Tile <= Lb;  // (uniform) all of it
#pragma unroll
            for (int r = 0; r < RUNS; ++r) {
                const uint32_t dst = to + 16 * RUN * r;
                if (__builtin_expect(exists && KEPT, 1)) {
#pragma unroll
                    for (int i = 0; i < FULL; ++i) tile_load16_uniform<false>(chunk_off[i], run[r], dst + 1024 * i);
                    if constexpr (REST != 0) tile_load16_uniform<true>(chunk_off[FULL], run[r], dst + 1024 * FULL);
                } else if (exists && row_bytes == Row::kBytes) {  // (uniform)
#pragma unroll
                    for (int i = 0; i < FULL; ++i) tile_load16_uniform<false>(16u * lane, run[r] + 1024 * i, dst + 1024 * i);
                    if constexpr (REST != 0) tile_load16_uniform<true>(16u * lane, run[r] + 1024 * FULL, dst + 1024 * FULL);
                } else {
                    const int last = Lb - 1 - min(key + 16 * r, (Lb - 1) & ~15);
                    int l = lane;
                    asm volatile("" : "+v"(l));  // (the offsets are worked out here: kept across the loop they would be spilled)
#pragma unroll
                    for (int i = 0; i < LOADS; ++i) {
                        const int n = 64 * i + l;
                        const uint32_t off = __umul24((uint32_t)min(n / RPC, last), row_bytes) + 16u * (n % RPC);
                        if (i < FULL)
                            tile_load16_uniform<false>(off, run[r], dst + 1024 * i);
                        else
                            tile_load16_uniform<true>(off, run[r], dst + 1024 * i);
                    }
                }
            }
        } else {
            const int last = FORM == kQ4Runs8 ? min(Lb - 1 - key, kQ4Tile - 1) : kQ4Tile - 1;
            int row0 = lane / RPC, chunk0 = lane % RPC;
            if constexpr (D == 128) asm volatile("" : "+v"(row0), "+v"(chunk0));  // (what follows from them is worked out here, as above)
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {  // (from the lane that has the offset of the row, or of its run)
                const int more = chunk0 + 64 * i % RPC, over = more >= RPC;
                const int at = row0 + 64 * i / RPC + over, chunk = more - RPC * over;
                const int row = FORM == kQ4Runs8 ? min(at, last) : at;
                const int from = FORM == kQ4Runs8 ? slot - RUNS + row / 8 : row;
                const int lo = __shfl(FORM == kQ4Runs8 ? ahead_off[0] : (int)row_off, from, 64);
                const int hi = __shfl(FORM == kQ4Runs8 ? ahead_off[1] : (int)(row_off >> 32), from, 64);
                const uint32_t in_run = FORM == kQ4Runs8 ? __umul24((uint32_t)row % 8, row_bytes) : 0u;
                tile_load16<64>(base + (((int64_t)hi << 32) | (uint32_t)lo) + in_run + 16 * chunk, to + 1024 * i);
            }
        }
    };

    // ---- running state (per lane: its column, partial over this lane's keys) --------------------------------
    float m_run = kNegInf, dsum1 = 0.f, dsum2 = 0.f;
    f32x4 o1[NDB], o2[NDB];
#pragma unroll
    for (int i = 0; i < NDB; ++i) o1[i] = o2[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    const float scale_log2 = p.scale * kLog2e;
    // (uniform) O1 and O2 count in 2^(zero - 127): a scale byte is 2^(byte - zero) to them
    int zero = 128;
    bool counted = false;
    auto recount = [&](int to) {
        const float by = __builtin_amdgcn_ldexpf(1.f, zero - to);
        zero = to;
#pragma unroll
        for (int i = 0; i < NDB; ++i) {
            o1[i] *= by;
            if constexpr (USE_R) o2[i] *= by;
        }
    };

    int v = v_lo + w, key = 0, key_next = 0, stage = 0;
    const char *run[ADDRESSES];
    bool have = next_tile(v, key, run), have_next = false;
    if (have) {
        issue(key, run, 0);
        v += kQ4Waves;
        have_next = next_tile(v, key_next, run);
        if (have_next) issue(key_next, run, 1);
    }
    // (q and rho, asked for in front of the first tiles, are waited for here: inside the loop every round would wait for them, and with
    // them for the tiles on their way)
#pragma unroll
    for (int s = 0; s < KSTEPS; ++s) {
        asm volatile("" : "+v"(qf[s]));
        if constexpr (USE_R) {
            asm volatile("" : "+v"(rf[s]));
#pragma unroll
            for (int e = 0; e < 4; ++e) {  // (exact but for what is too small to count)
                const uint32_t x = rf[s][e];
                constexpr float by = 1.f / (1 << kProbeDown);
                rf[s][e] = pack_bf16(bf16_lo_f32(x) * by, bf16_hi_f32(x) * by);
            }
        }
    }
    while (have) {
        const int tk = key;
        const bool whole = scope.whole(tk, kQ4Tile);  // (uniform) every column sees all of the keys
        if (have_next)                                // (uniform) the tile is here, the next one may not be
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(ADDRESSES * LOADS) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const char *tile = (const char *)(raw + stage * RAW);
        // This lane's places in a tile: of the K rows, and of the rows it gives the transposing reads (element i of a lane's 4-bit
        // operand is key 32 (i / 8) + 16 (i / 4 % 2) + 4 g + i % 4, of its scales, 32 keys at a time, likewise)
        int place = lane;
        if constexpr (C == 16) asm volatile("" : "+v"(place));  // (no registers to keep them in across the loop)
        const uint32_t pc = place & 15, pg = place >> 4;
        const uint32_t k_at = pc * Row::kBytes + (D == 128 ? 16 : 8) * pg, k_scale_at = pc * Row::kBytes + Row::kKScale + (D == 128 ? 2 : 1) * pg;
        const uint32_t v_at = (32 * (pc >> 3) + 16 * ((pc >> 2) & 1) + 4 * pg + (pc & 3)) * Row::kBytes + Row::kV;
        const uint32_t v_scale_at = (16 * (pc >> 3) + 4 * pg + ((pc >> 1) & 3)) * Row::kBytes + (D == 128 ? Row::kVScale : Row::kKScale);
        int key_third = 0;  // the tile behind the next one is looked for here, and asked for when this one has been read
        bool have_third = false;
        if (have_next) {
            v += kQ4Waves;
            have_third = next_tile(v, key_third, run);
        }

        // ---- S1^T = K q^T, S2^T = K rho^T -------------------------------------------------------------------
        f32x4 s1[4], s2[4];
#pragma unroll
        for (int sub = 0; sub < 4; ++sub) {
            s1[sub] = s2[sub] = f32x4{0.f, 0.f, 0.f, 0.f};
            const char *row = tile + 16 * sub * Row::kBytes;
            if constexpr (D == 128) {
                const u32x4 codes = *(const u32x4 *)(row + k_at);
                const uint32_t scales = *(const uint16_t *)(row + k_scale_at);
                const float lo = q4_scale_byte(scales, 0), hi = q4_scale_byte(scales, 1);
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s) {
                    const u32x4 kf = q4_to_bf16(codes[s], s < 2 ? lo : hi);
                    s1[sub] = mfma16(kf, qf[s], s1[sub]);
                    if constexpr (USE_R) s2[sub] = mfma16(kf, rf[s], s2[sub]);
                }
            } else {
                const u32x2 codes = *(const u32x2 *)(row + k_at);
                const float scale = q4_scale(*(const uint8_t *)(row + k_scale_at));
#pragma unroll
                for (int s = 0; s < KSTEPS; ++s) {
                    const u32x4 kf = q4_to_bf16(codes[s], scale);
                    s1[sub] = mfma16(kf, qf[s], s1[sub]);
                    if constexpr (USE_R) s2[sub] = mfma16(kf, rf[s], s2[sub]);
                }
            }
        }
        u32x2 scales[2];  // of V, 8 keys each
#pragma unroll
        for (int h = 0; h < 2; ++h) scales[h] = lds_read_tr8(tile + 32 * h * Row::kBytes + v_scale_at);
        uint32_t seen[2] = {0xffu, 0xffu};
        float factor = scale_log2;
        if (__builtin_expect(!whole, 0)) {
            int l = lane, lo, end;
            asm volatile("" : "+v"(l));  // (the key set is worked out here, see above)
            key_set(l & 15, lo, end);
#pragma unroll
            for (int h = 0; h < 2; ++h) seen[h] = scope.seen(P, no_nodes, lo, end, tk + 32 * h, l >> 4);
            asm volatile("" : "+v"(seen[0]), "+v"(seen[1]));  // (not to be worked out for every tile)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const bool ok = (seen[e >> 3] >> (e & 7)) & 1u;
                s1[e >> 2][e & 3] = ok ? s1[e >> 2][e & 3] * factor : kNegInf;
                if constexpr (USE_R) s2[e >> 2][e & 3] = ok ? s2[e >> 2][e & 3] : 0.f;
            }
            factor = 1.f;
        }
        // Any reference near the row's largest score does: it moves (and everything with it) only when a weight is 2^2 above it
        float tmax = kNegInf;
#pragma unroll
        for (int e = 0; e < 16; ++e) tmax = fmaxf(tmax, s1[e >> 2][e & 3]);
        tmax *= factor;
        if (__builtin_expect(__any(tmax > m_run + kQ4Slack), 0)) {  // (rare, but for the first tile)
            tmax = rows_max(tmax);
            const float m_new = fmaxf(m_run, tmax);
            const float alpha = fast_exp2(m_run - (m_new == kNegInf ? 0.f : m_new));
            const bool any = __any(m_run > kNegInf);  // (nothing to move in front of the first tile)
            m_run = m_new;
            if (any) {
                dsum1 *= alpha, dsum2 *= alpha;
#pragma unroll
                for (int i = 0; i < NDB; ++i) {
                    o1[i] *= alpha;
                    if constexpr (USE_R) o2[i] *= alpha;
                }
            }
        }
        float tilt = 0.f;  // of this lane's keys
        if constexpr (USE_R) {
#pragma unroll
            for (int e = 0; e < 16; ++e) tilt = fmaxf(tilt, fabsf(s2[e >> 2][e & 3]));
        }
        const float up_m = m_run == kNegInf ? 0.f : kWeightUp - m_run;
        auto weight = [&](int e) { return fast_exp2(fmaf(s1[e >> 2][e & 3], factor, up_m)); };
        // This lane's scales counted from zero - 8: 0 .. 8 if they are within reach (lower ones wrap round)
        typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
        u16x2 own[8];
        auto far_scales = [&]() {
            u16x2 widest = {0, 0};
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const uint32_t bytes = __builtin_amdgcn_perm(0u, scales[n >> 2][(n >> 1) & 1], n & 1 ? 0x0c030c02u : 0x0c010c00u);
                const uint16_t lowest = (uint16_t)(zero - kScaleRange);
                own[n] = __builtin_bit_cast(u16x2, bytes) - u16x2{lowest, lowest};
                widest = __builtin_elementwise_max(widest, own[n]);
            }
            const bool far = max(widest[0], widest[1]) > kScaleRange;
            return D == 64 ? far && (c & 4) : far;  // (the others have the scales of K)
        };
        bool wild = far_scales();
        if (__builtin_expect(whole && !counted && __any(wild), 0)) {  // (once) the largest scale of the tile's last key, and 2^2 of room
            int top = D == 128 || (c & 4) ? (int)(scales[1][1] >> 24) : 0;
            top = (int)row_max((uint32_t)top);
            top = __builtin_amdgcn_readlane(top, 48);
            recount(min(max(top + 2, 64), 190)), counted = true;
            wild = far_scales();
        }
        if (__builtin_expect(__any(tmax < m_run - kWeightFloor), 0)) {
            const float most = rows_max(tmax);  // (of the tile; -infinity: nothing to lose)
            wild |= most < m_run - kWeightFloor && most > kNegInf;
        }
        if constexpr (USE_R) wild |= tilt * fast_exp2(tmax - m_run + kWeightUp) > 1 << kProbeMost;

        // (a key that a column does not see has a weight of 0, and here a scale within reach)
        if (__builtin_expect((whole || D == 64) && !__any(wild), 1)) {
            // P1 and P2 in f16, once (in bf16 they made the result's error 1.4 times that of its own rounding); d1 and d2 add the rounded
            // values, so that the weights still sum to one and what cancels between O1 d2 and O2 does so exactly.
            uint32_t w1[8], w2[8];
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const float p0 = weight(2 * n), p1 = weight(2 * n + 1);
                w1[n] = pack_f16(p0, p1), dsum1 = add_f16_pair(w1[n], dsum1);
                if constexpr (USE_R) {
                    w2[n] = pack_f16(p0 * s2[n >> 1][2 * (n & 1)], p1 * s2[n >> 1][2 * (n & 1) + 1]);
                    dsum2 = add_f16_pair(w2[n], dsum2);
                }
                own[n] = own[n] * u16x2{1 << 10, 1 << 10} + u16x2{(15 - kScaleRange) << 10, (15 - kScaleRange) << 10};  // as f16
            }
            if constexpr (C >= 4) __builtin_amdgcn_sched_barrier(0);
            // ---- O1^T += V^T P1^T, O2^T += V^T P2^T, 16 * REP dimensions with the same operands --------------------
            auto products = [&](auto j) __attribute__((always_inline)) {
                constexpr int J = decltype(j)::value;
                u32x4 pb1[2], pb2[2];
#pragma unroll
                for (int n = 0; n < 8; ++n) {
                    const uint32_t x = operand_scales<D, C, J>(__builtin_bit_cast(uint32_t, own[n]));
                    pb1[n >> 2][n & 3] = mul_f16_pair(w1[n], x);
                    if constexpr (USE_R) pb2[n >> 2][n & 3] = mul_f16_pair(w2[n], x);
                }
#pragma unroll
                for (int n = 0; n < REP; ++n) {
                    const int i = REP * J + n;
                    const u32x2 codes = lds_read_tr4(tile + v_at + 8 * i);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const u32x4 x = q4_to_f16(codes[h]);
                        o1[i] = mfma16_f16(x, pb1[h], o1[i]);
                        if constexpr (USE_R) o2[i] = mfma16_f16(x, pb2[h], o2[i]);
                    }
                }
                if constexpr (C >= 8) __builtin_amdgcn_sched_barrier(0);
            };
            each_of<OPERANDS>(products);
        } else {
            // Any sizes: P1 and P2 are cut to 16 bits, which two bf16 hold, times their scales. Only a scale 2^90 above what O1 and O2 count in
            // is too large, and moves that. A scale of NaN (255, infinite here): infinity less itself.
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t byte = (scales[e >> 3][(e >> 2) & 1] >> (8 * (e & 3))) & 255u;
                const bool some = (row_or(seen[e >> 3]) >> (e & 7)) & 1u;  // (a column that sees the key)
                if (some && byte != 255 && (D == 128 || (c & 4))) top = max(top, byte);
            }
            if (__any((int)top > zero + 90)) {
                top = row_max(top);
                top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32, 64));
                recount(min(__builtin_amdgcn_readfirstlane((int)top), 190));
            }
            const float unit = __builtin_amdgcn_ldexpf(1.f, 127 - zero);
            u32x2 keep[2];  // bytes of the keys that are seen: bits 0 .. 3 of a half, to bytes
#pragma unroll
            for (int h = 0; h < 2; ++h) keep[h] = u32x2{((seen[h] & 15u) * 0x204081u & 0x01010101u) * 255u, ((seen[h] >> 4) * 0x204081u & 0x01010101u) * 255u};
            float p1[16], p2[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p1[e] = cut(weight(e)), dsum1 += p1[e];
                if constexpr (USE_R) p2[e] = cut(p1[e] * s2[e >> 2][e & 3]), dsum2 += p2[e];
            }
            auto products = [&](auto j) __attribute__((always_inline)) {
                constexpr int J = decltype(j)::value;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    u32x4 pb1, pb2, rest1, rest2;
#pragma unroll
                    for (int d = 0; d < 2; ++d) {
                        const uint32_t e4 = operand_scales<D, C, J>(scales[h][d]) & keep[h][d];
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const float x0 = q4_scale_byte(e4, e) * unit, x1 = q4_scale_byte(e4, e + 1) * unit;
                            const int at = 8 * h + 4 * d + e, to = 2 * d + e / 2;
                            halves(p1[at] * x0, p1[at + 1] * x1, pb1, rest1, to);
                            if constexpr (USE_R) halves(p2[at] * x0, p2[at + 1] * x1, pb2, rest2, to);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < REP; ++n) {
                        const int i = REP * J + n;
                        const u32x4 x = q4_to_bf16(lds_read_tr4(tile + v_at + 8 * i)[h], 1.f);
                        o1[i] = mfma16(x, pb1, o1[i]);
                        if constexpr (USE_R) o2[i] = mfma16(x, pb2, o2[i]);
                        o1[i] = mfma16(x, rest1, o1[i]);
                        if constexpr (USE_R) o2[i] = mfma16(x, rest2, o2[i]);
                    }
                    if constexpr (D == 128) __builtin_amdgcn_sched_barrier(0);  // (step after step: together they need more registers than there are)
                }
            };
            each_of<OPERANDS>(products);
        }

        if (have_third) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (read before it is written again)
            issue(key_third, run, stage);
        }
        key = key_next, key_next = key_third;
        have = have_next, have_next = have_third;
        stage ^= 1;
    }

    // ---- the four waves' states (in the order of the lanes' registers: no bank conflicts), then the record or the output row ----
    constexpr int QUADS = NDB * 64;  // of four dimensions: quad 64 i + lane' is matrix column lane' % 16, dimensions 16 i + 4 (lane' / 16) ..
    f32x4 *mrg1 = (f32x4 *)lds, *mrg2 = mrg1 + kQ4Waves * QUADS;  // [wave][quad]
    float *mrg_m = (float *)(lds + kQ4Waves * 2 * RAW), *mrg_d1 = mrg_m + kQ4Waves * 16, *mrg_d2 = mrg_d1 + kQ4Waves * 16;
    __syncthreads();  // every wave is done with its tiles
    int last = threadIdx.x;
    asm volatile("" : "+v"(last));  // (places of threads are worked out again: kept across the loop they would be spilled)
    {
        const int lane = last & 63, c = lane & 15, g = lane >> 4;
        constexpr int DOWN = -kWeightUp - kRecordDown;
        const float s1 = __builtin_amdgcn_ldexpf(rows_sum(dsum1), DOWN), s2 = __builtin_amdgcn_ldexpf(rows_sum(dsum2), DOWN + kProbeDown);
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o1[i][e] = __builtin_amdgcn_ldexpf(o1[i][e], zero - 127 + DOWN);
                if constexpr (USE_R) o2[i][e] = __builtin_amdgcn_ldexpf(o2[i][e], zero - 127 + DOWN + kProbeDown);
            }
        // a row in front of the sequence sees nothing, also where all others see everything
        int lo, end;
        key_set(c, lo, end);
        const bool none = end == 0;
        if (g == 0) {
            mrg_m[w * 16 + c] = none ? kNegInf : m_run + kRecordDown;
            mrg_d1[w * 16 + c] = none ? 0.f : s1;
            mrg_d2[w * 16 + c] = none ? 0.f : s2;
        }
#pragma unroll
        for (int i = 0; i < NDB; ++i) {
            const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
            if (c % REP != i % REP) continue;  // (the copies with other groups' scales)
            mrg1[w * QUADS + 64 * i + lane] = none ? zero : o1[i];
            if constexpr (USE_R) mrg2[w * QUADS + 64 * i + lane] = none ? zero : o2[i];
        }
    }
    __syncthreads();
    for (int at = last; at < NDB * 4 * C; at += 256) {
        const int i = at / (4 * C), quarter = at / C % 4, col = at % C, x = col * REP + i % REP;  // x: matrix column
        if (col >= n_cols) continue;
        float m_star = kNegInf, wt[kQ4Waves], d1 = 0.f, d2 = 0.f;
#pragma unroll
        for (int ww = 0; ww < kQ4Waves; ++ww) m_star = fmaxf(m_star, mrg_m[ww * 16 + x]);
        f32x4 a1 = {0.f, 0.f, 0.f, 0.f}, a2 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ww = 0; ww < kQ4Waves; ++ww) {
            // (a reference of -inf with a sum that is not zero: scores of NaN only, which must reach the result)
            const float mw = mrg_m[ww * 16 + x], dw = mrg_d1[ww * 16 + x];
            wt[ww] = mw == kNegInf && dw == 0.f ? 0.f : fast_exp2(mw - m_star);
            d1 += wt[ww] * dw;
            d2 += wt[ww] * mrg_d2[ww * 16 + x];
            a1 += wt[ww] * mrg1[ww * QUADS + 64 * i + 16 * quarter + x];
            if constexpr (USE_R) a2 += wt[ww] * mrg2[ww * QUADS + 64 * i + 16 * quarter + x];
        }
        const RowsColumn<D> column(p, b, hk, col, split, m_star, d1, d2, false, i == 0 && quarter == 0);
        column.store(16 * i + 4 * quarter, a1, a2);
    }
}

template <int D, int C, bool USE_R>
static void launch_q4_form(const DecodeRowsParams &P, hipStream_t stream) {
    const DecodeParams &p = P.d;
    const dim3 grid(p.S, p.Hkv, p.B);
    const bool short_rows = p.ksl < (1 << 24);  // (24-bit products of a row number below 64 and the row stride)
    // (us, pages of a multiple of 8 against row by row: 24 x <= 6000 keys 46, 50; d = 64, window 4096, 4 rows 24.3, 27.1; pages of 16 41.3,
    // 23.5, of 64 40, 21.8, none 38.7, 21.5)
    if (short_rows && p.block_table == nullptr && P.block_list == nullptr)
        hipLaunchKernelGGL((decode_q4_kernel<D, C, USE_R, kQ4Direct>), grid, dim3(256), 0, stream, P);
    else if (short_rows && (p.block_table == nullptr || p.page_size % 64 == 0))
        hipLaunchKernelGGL((decode_q4_kernel<D, C, USE_R, kQ4Runs64>), grid, dim3(256), 0, stream, P);
    else if (short_rows && p.page_size % 16 == 0)
        hipLaunchKernelGGL((decode_q4_kernel<D, C, USE_R, kQ4Runs16>), grid, dim3(256), 0, stream, P);
    else if (short_rows && p.page_size % 8 == 0)
        hipLaunchKernelGGL((decode_q4_kernel<D, C, USE_R, kQ4Runs8>), grid, dim3(256), 0, stream, P);
    else
        hipLaunchKernelGGL((decode_q4_kernel<D, C, USE_R, kQ4Any>), grid, dim3(256), 0, stream, P);
}

template <int D>
static void launch_q4_columns(const DecodeRowsParams &P, hipStream_t stream) {
    const int cols = P.d.G * P.d.Tq;
    if (!P.d.use_r) return cols <= 4 ? launch_q4_form<D, 4, false>(P, stream) : launch_q4_form<D, 16, false>(P, stream);
    if constexpr (D == 128)
        if (cols <= 2) return launch_q4_form<D, 2, true>(P, stream);
    if (cols <= 4) return launch_q4_form<D, 4, true>(P, stream);
    cols <= 8 ? launch_q4_form<D, 8, true>(P, stream) : launch_q4_form<D, 16, true>(P, stream);
}

hipError_t launch_decode_q4(const DecodeRowsParams &P, hipStream_t stream) {
    P.d.d == 128 ? launch_q4_columns<128>(P, stream) : launch_q4_columns<64>(P, stream);
    return hipGetLastError();
}

}  // namespace plx
