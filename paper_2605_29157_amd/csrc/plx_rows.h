// What the kernels for rows whose key sets differ share (decode_rows_bf16.hip: up to 16 columns, private tiles;
// decode_rows_wide_bf16.hip: more, shared tiles): which keys a workgroup walks, which of them a column sees.
#pragma once
#include "plx_device.h"
#include "plx_kernels.h"

namespace plx {

// How the rows of a tile are found; as in decode_bf16.hip: runs of 16 keys that follow each other in memory (contiguous,
// pages of a multiple of 16), or row by row.
enum RowsCache { kRowsContiguous, kRowsPagedRuns, kRowsAny };

// The dword's bf16 halves that are infinite or NaN, as a mask of whole halves
__device__ __forceinline__ uint32_t not_finite_halves(uint32_t x) {
    const uint32_t lo = (x & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (x & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
    return lo | hi;
}
constexpr uint32_t kBigHalves = 0x7f007f00u;  // two bf16 of 2^127

// The bits of an 8-key operand (bit e: k-element e) as halves of 2^127 or 0
__device__ __forceinline__ u32x4 big_halves(uint32_t seen) {
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        x[e] = kBigHalves & (((seen >> (2 * e)) & 1u ? 0xffffu : 0u) | ((seen >> (2 * e + 1)) & 1u ? 0xffff0000u : 0u));
    return x;
}

// First key of tile number v of a list's blocks, or -1: an entry that is no block of Lb tokens, or not above the one in front of it
template <int TILE>
__device__ __forceinline__ int listed_key(const int32_t *list, int v, int Lb) {
    constexpr int TILES = kListBlock / TILE;
    const int i = v / TILES, block = list[i], before = i > 0 ? list[i - 1] : -1;
    if (block < 0 || block <= before || block > (Lb - 1) / kListBlock) return -1;
    const int key = block * kListBlock + TILE * (v % TILES);
    return key < Lb ? key : -1;
}

// The keys that the columns [x0, x0 + width) of (sequence b, key head) see, columns x = row * G + head of the group, and
// the tiles of TILE keys that are walked for them: those of the sinks, then those from the first key any window
// reaches. Tile number v of this walk holds the keys from key_of(v) on; no key is in two of them.
// LIST: the tiles are those of the blocks of a list (one for each key head, hk). A tile's key is then -1 where its entry is passed over.
template <bool TREE, int TILE, bool LIST = false>
struct RowsScope {
    int Lb, n, base;          // cached tokens; drafted ones among them (TREE), behind `base` committed ones (else base = Lb - Tq)
    int lo_all, end_all;      // keys every column sees: [lo_all, end_all), and [0, sinks) below end_all
    int sinks, n_sink_tiles, first_tile, n_virtual;
    const uint64_t *masks;    // TREE: the sequence's
    const int32_t *list;      // LIST: the sequence's and key head's

    __device__ __forceinline__ RowsScope(const DecodeRowsParams &P, int b, int x0, int width, int hk = 0) {
        const DecodeParams &p = P.d;
        Lb = p.seq_lens ? p.seq_lens[b] : p.Lmax;
        Lb = min(max(Lb, 0), p.Lmax);
        n = p.Tq;
        if constexpr (TREE) n = min(P.draft_lens ? min(max(P.draft_lens[b], 0), p.Tq) : p.Tq, Lb);
        base = Lb - n;
        masks = TREE ? P.mask + (int64_t)b * P.mask_stride_b : nullptr;
        const int t_first = x0 / p.G, t_last = min(x0 + width - 1, p.G * p.Tq - 1) / p.G;
        int lo_any = 0, end_any;
        lo_all = 0;
        if constexpr (TREE) {
            end_any = t_first < n ? Lb : 0, end_all = base;
            if (p.window > 0) lo_any = min(max(base + 1 - p.window, 0), base), lo_all = min(max(base + n - p.window, 0), base);
        } else {
            end_any = max(base + t_last + 1, 0), end_all = max(base + t_first + 1, 0);
            if (p.window > 0) lo_any = max(base + t_first + 1 - p.window, 0), lo_all = max(base + t_last + 1 - p.window, 0);
        }
        sinks = p.window > 0 ? P.sinks : 0;
        n_sink_tiles = (min(sinks, end_any) + TILE - 1) / TILE;
        first_tile = max(lo_any / TILE, n_sink_tiles);
        n_virtual = n_sink_tiles + max((end_any + TILE - 1) / TILE - first_tile, 0);
        list = nullptr;
        if constexpr (LIST) {
            list = P.block_list + ((int64_t)b * p.Hkv + hk) * P.n_list;
            n_virtual = end_any > 0 ? P.n_list * (kListBlock / TILE) : 0;
        }
    }
    __device__ __forceinline__ int key_of(int v) const {
        if constexpr (LIST) {
            return listed_key<TILE>(list, v, Lb);
        }
        return TILE * (v < n_sink_tiles ? v : v - n_sink_tiles + first_tile);
    }
    // does every column see the keys [key, key + count)?
    __device__ __forceinline__ bool whole(int key, int count) const {
        return (key >= lo_all || key + count <= sinks) && key + count <= end_all;
    }
    // Keys of column x (number `at` of the workgroup's COLS from x0 on): [lo, end) and the sinks below end, of the drafted ones those
    // whose bit is set. All threads take part.
    template <int COLS>
    __device__ __forceinline__ void column(const DecodeRowsParams &P, TreeWords<COLS> &lds, int x0, int at, int t, bool live, int &lo,
                                           int &end, TreeRow &nodes) const {
        if constexpr (TREE) {
            const uint64_t *words = masks + (int64_t)t * P.mask_words;
            nodes = {lds.of[at], *words};
            if (tree_staged(P.mask_words, P.d.window, n)) {  // (uniform)
                tree_stage<COLS>(lds, masks, P.mask_words, n, base, P.d.window, sinks, threadIdx.x, blockDim.x,
                                 [&](int col) { return (x0 + col) / P.d.G; });
                nodes.first = lds.of[at][0];
            }
            end = live && t < n ? Lb : 0;
            lo = 0;
            if (P.d.window > 0) lo = min(max(base + tree_position(words, P.mask_words, n) - P.d.window + 1, 0), base);
        } else {
            end = live ? max(base + t + 1, 0) : 0;
            lo = P.d.window > 0 ? max(end - P.d.window, 0) : 0;
        }
    }
    // Bit e of the result: the column sees key first + 16 (e / 4) + e % 4 (first = key + 4 g of a 32-key block)
    __device__ __forceinline__ uint32_t seen(const DecodeRowsParams &P, const TreeRow &nodes, int lo, int end, int key, int g) const {
        uint32_t bits = 0xffffffffu, out = 0;
        if constexpr (TREE)
            if (key + 32 > base) bits = tree_bits(nodes, P.mask_words, key - base);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int at = 16 * (e >> 2) + 4 * g + (e & 3), k = key + at;
            const bool ok = k < end && (k >= lo || k < sinks) && ((bits >> at) & 1u);
            out |= ok ? 1u << e : 0u;
        }
        return out;
    }
};

// Where a workgroup's keys are
struct RowsPages {
    const DecodeParams &p;
    const int32_t *table;
    __device__ __forceinline__ RowsPages(const DecodeParams &p, int b) : p(p), table(p.block_table + (int64_t)b * p.table_stride) {}
    __device__ __forceinline__ void offsets(int key, int64_t &ko, int64_t &vo) const {  // element offsets of a key's row in the pools
        const int page_no = key / p.page_size, row = key - page_no * p.page_size;
        const int64_t page = min(max(table[page_no], 0), p.num_pages - 1);
        ko = page * p.ksb + (int64_t)row * p.ksl, vo = page * p.vsb + (int64_t)row * p.vsl;
    }
};

// Four dimensions of a finished column: of its record, or of its output row
template <int D>
struct RowsColumn {
    const DecodeParams &p;
    int64_t row;
    float d1, d2, inv, gain;
    float *rec;
    bool none, nan;
    __device__ __forceinline__ RowsColumn(const DecodeParams &p, int b, int hk, int x, int split, float m, float d1_, float d2_, bool none, bool head)
        : p(p), d1(none ? 0.f : d1_), d2(none ? 0.f : d2_), none(none) {
        const int t = x / p.G, h = x - t * p.G;
        row = ((int64_t)b * p.Hq + (int64_t)hk * p.G + h) * p.Tq + t;
        nan = d1 != d1;
        inv = d1 != 0.f ? 1.f / d1 : 0.f, gain = inv * (1.f + d2 * inv);
        rec = p.ws + (row * p.S + split) * (int64_t)(2 * D + 4);
        // (NaN: a record that the merge takes alone)
        if (!p.direct_out && head) *(f32x4 *)rec = nan ? f32x4{3.0e38f, -kNegInf, 0.f, 0.f} : f32x4{none ? kNegInf : m, d1, d2, 0.f};
    }
    __device__ __forceinline__ void store(int dim, f32x4 a1, f32x4 a2) const {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        if (none) a1 = a2 = zero;
        if (p.direct_out) {
            f32x4 y = zero;  // empty key set: zeros
            if (d1 != 0.f) y = a1 * gain - a2 * inv;
            *(u32x2 *)((__bf16 *)p.o + row * D + dim) = u32x2{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3])};
        } else {
            if (nan) a1[0] = a1[1] = a1[2] = a1[3] = __builtin_nanf("");
            *(f32x4 *)(rec + 4 + dim) = a1;
            *(f32x4 *)(rec + 4 + D + dim) = a2;
        }
    }
};

}  // namespace plx
