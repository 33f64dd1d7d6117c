// Rows of K and V to and from a cache held in 4 bits (plx_q4.h has the row).
//
// Writing: of each 16 dimensions the scale is the power of two s with 3.5 <= max |x| / s < 7, so that the largest rounds to 4 or 6
// and nothing saturates: e = exponent of (max |x| * 8 / 7, rounded down) - 2, one integer addition on the float's bits. (Normal values,
// relative error of a row: 0.110; with s <= max / 4 < 2 s, whose largest magnitudes saturate at 6, 0.118; with max / s <= 6 0.113; 32
// dimensions to a scale 0.112 - 0.115.) x / s is exact, so the one rounding is that to the code, to nearest, ties to even.
//
// What bounds them: the bytes of the rows, 4 D of bf16 and 9 D / 8 of the cache; few rows: one launch. A thread has 16 bytes
// of bf16 of each of its rows, two neighbours share a scale, and the scale bytes of eight threads are put together, so that
// a row goes out in whole dwords. Many rows: four a thread, all on their way at once, of one sequence and head, whose numbers, first token
// and count are the workgroup's. What a row costs beside its bytes decides: 172 MB through pages of 16 were written in 47 us and read back
// in 55 with divisions by T, Hkv and the page size a row (the last in 64 bits); with a workgroup's rows of one sequence 38 and 34; K and V,
// which pass once, asked for and stored as such 37 and 27; the page by a multiplication, offsets from 32-bit factors, magnitudes and codes
// from bf16 pairs, all lookups in front of the loads 36 and 27 (4.7, 6.5 TB/s; without pages 33 and 27; a copy of as much 35).
#include "plx_kernels.h"
#include "plx_q4.h"

namespace plx {

namespace {

// Rows from which a thread takes four: us, written / read, one a thread and four: d = 128 3200 rows 3.0 / 3.1 and 3.9 / 3.7, 16000
// 5.0 / 4.4 and 4.9 / 4.4, 32000 7.7 / 6.2 and 6.6 / 5.7, 262144 (172 MB) 42 / 30 and 33 / 28; fp32 131072 29 / 29 and 31 / 26. And
// tokens of a sequence from which it does, in workgroups: 33 tokens (two workgroups of 32) 8.0 / 6.4 and 8.9 / 7.2, 64 12.9 / 9.4 and 9.9 / 9.1.
constexpr int64_t kManyRows = 32000;
constexpr int kManyRuns = 2;

// Thread -> (K or V, DIMS of its dimensions) of ROWS rows: of one row in the order of (b, h, t), or of tokens that follow one another at a
// distance in one sequence and head, whose numbers are then the workgroup's
template <int D, int ROWS, int DIMS = 8>
struct Q4Place {
    static constexpr int kLanes = D / DIMS, kThreads = 2 * kLanes;  // of a tensor's row; of a row
    static constexpr int kRows = 256 / kThreads;                 // of a workgroup at a time
    static constexpr int kTokens = kRows * ROWS;                 // of a workgroup
    int part, b, h, t;
    bool is_v, any;
    __device__ __forceinline__ Q4Place(const Q4Rows &p) : part(threadIdx.x % kLanes), is_v(threadIdx.x / kLanes % 2 != 0) {
        uint32_t bh;
        if constexpr (ROWS == 1) {
            const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kThreads;
            any = row < (int64_t)p.cache.B * p.cache.Hkv * p.T;
            const uint32_t r = any ? (uint32_t)row : 0;
            bh = r / (uint32_t)p.T, t = (int)(r - bh * p.T);
        } else {
            const uint32_t runs = ((uint32_t)p.T + kTokens - 1) / kTokens;
            bh = blockIdx.x / runs, t = (int)((blockIdx.x - bh * runs) * kTokens + threadIdx.x / kThreads), any = true;
        }
        b = (int)(bh / (uint32_t)p.cache.Hkv), h = (int)(bh - b * p.cache.Hkv);
    }
    __device__ __forceinline__ int token(int i) const { return t + kRows * i; }
    __device__ __forceinline__ bool has(const Q4Rows &p, int i) const { return any && (ROWS == 1 || token(i) < p.T); }
    // Where a token's row is, in two steps so that no branch and no wait comes between the rows: its page (0 without a table, -1: no row), ..
    __device__ __forceinline__ int page_of(const Q4Rows &p, int64_t token, bool wanted) const {
        const Q4Cache &c = p.cache;
        wanted = wanted && token >= 0 && token < c.capacity;
        int page = 0;
        if (c.block_table != nullptr) {  // (uniform)
            const uint32_t n = wanted ? (uint32_t)token : 0;
            page = c.block_table[b * c.table_stride + (__umulhi(2 * n, c.page_mul) >> c.page_shift)];
            if (page >= c.num_pages) page = -1;
        }
        return wanted ? page : -1;
    }
    // .. and its byte offset, or -1. (Pages and rows are counted in 16 bytes: with factors of 32 bits it takes four multiplications, each
    // of the time of four other instructions.)
    __device__ __forceinline__ int64_t row_of(const Q4Rows &p, int64_t token, int page) const {
        const Q4Cache &c = p.cache;
        const uint32_t row16 = (uint32_t)((uint64_t)c.stride[2] >> 4), page16 = (uint32_t)((uint64_t)c.stride[0] >> 4), n = (uint32_t)token;
        int64_t at = h * c.stride[1];
        if (c.block_table == nullptr) {
            at += b * c.stride[0] + (int64_t)((uint64_t)n * row16 << 4);
        } else {
            const uint32_t page_no = __umulhi(2 * n, c.page_mul) >> c.page_shift;
            at += (int64_t)((uint64_t)(uint32_t)page * page16 + (uint64_t)(n - page_no * c.page_size) * row16) << 4;
        }
        return page < 0 ? -1 : at;
    }
    __device__ __forceinline__ int64_t element(const int64_t (&s)[3], int i, int T) const {  // (behind the last token: one in front of it)
        return b * s[0] + h * s[1] + min(t, T - 1) * s[2] + DIMS * part + (token(i) < T ? i * (kRows * s[2]) : 0);
    }
};

}  // namespace

template <int D, bool F32, int ROWS>
__global__ __launch_bounds__(256) void cache_write_q4_kernel(Q4Rows p) {
    using Row = Q4Row<D>;
    const Q4Place<D, ROWS> me(p);
    const int64_t start = p.start != nullptr ? p.start[me.b] : 0;
    const int count = p.counts != nullptr ? p.counts[me.b] : p.T;
    const void *src = me.is_v ? p.v : p.k;
    int page[ROWS];
    u32x4 raw[ROWS];
    f32x4 wide[ROWS][2];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) page[i] = me.page_of(p, start + me.token(i), me.has(p, i) && me.token(i) < count);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t e = me.element(me.is_v ? p.vs : p.ks, i, p.T);
        if constexpr (F32) {
            wide[i][0] = *(const f32x4 *)((const float *)src + e), wide[i][1] = *(const f32x4 *)((const float *)src + e + 4);
        } else {
            raw[i] = __builtin_nontemporal_load((const u32x4 *)((const __bf16 *)src + e));
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        uint32_t top = 0;  // of the magnitudes' bits, as those of a float: infinities and NaN are the largest
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = wide[i][e / 4][e % 4];  // (a cast of the element itself is compiled as one of element 0)
                top = max(top, __builtin_bit_cast(uint32_t, x) & 0x7fffffffu);
            }
        } else {
            typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
            u16x2 both = {0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) both = __builtin_elementwise_max(both, __builtin_bit_cast(u16x2, raw[i][e] & 0x7fff7fffu));
            const uint32_t halves = __builtin_bit_cast(uint32_t, both);
            top = max(halves << 16, halves & 0xffff0000u);
        }
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));  // quad_perm [1, 0, 3, 2]
        const bool bad = top >= 0x7f800000u;
        const uint32_t e = (uint32_t)min(max((int)((top + 0x200000u) >> 23) - 2, 4), 252);
        const float scale = q4_scale(e);
        uint32_t codes = 0;
        if constexpr (F32) {
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, wide[i][0][0], wide[i][0][1], scale, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, wide[i][0][2], wide[i][0][3], scale, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, wide[i][1][0], wide[i][1][1], scale, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, wide[i][1][2], wide[i][1][3], scale, 3);
        } else {
            typedef __bf16 bf16_pair __attribute__((ext_vector_type(2)));
            auto pair = [&](int e) {
                const uint32_t x = raw[i][e];  // (as above)
                return __builtin_bit_cast(bf16_pair, x);
            };
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(0), scale, 0);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(1), scale, 1);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(2), scale, 2);
            codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, pair(3), scale, 3);
        }
        uint32_t scales = (bad ? 255u : e) << (8 * (me.part / 2 & 3));  // four scales of eight lanes
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x4E, 0xf, 0xf, true);   // quad_perm [2, 3, 0, 1]
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x141, 0xf, 0xf, true);  // row_half_mirror
        const int64_t at = me.row_of(p, start + me.token(i), page[i]);
        if (at < 0) continue;
        char *row = p.cache.rows + at;
        *(uint32_t *)(row + (me.is_v ? Row::kV : 0) + 4 * me.part) = bad ? 0u : codes;
        if (me.part % 8 == 0) *(uint32_t *)(row + (me.is_v ? Row::kVScale : Row::kKScale) + me.part / 2) = scales;
        if constexpr (Row::kBytes > Row::kEnd) {
            static_assert(Row::kBytes - Row::kEnd == 8, "one store");
            if (me.is_v && me.part == 1) *(u32x2 *)(row + Row::kEnd) = u32x2{0u, 0u};
        }
    }
}

template <int D, bool F32, int ROWS>
__global__ __launch_bounds__(256) void cache_read_q4_kernel(Q4Rows p) {
    using Row = Q4Row<D>;
    constexpr int DIMS = F32 ? 4 : 8;  // 16 bytes to store: halves of a line go to memory apart (fp32, eight: 66 us)
    using Codes = std::conditional_t<F32, uint16_t, uint32_t>;
    const Q4Place<D, ROWS, DIMS> me(p);
    const int64_t start = p.start != nullptr ? p.start[me.b] : 0;
    const int64_t count = p.counts != nullptr ? p.counts[me.b] : p.cache.capacity;
    uint32_t codes[ROWS], scales[ROWS];
    int64_t to[ROWS];
    int page[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) page[i] = me.page_of(p, start + me.token(i), me.has(p, i) && start + me.token(i) < count);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int64_t at = me.row_of(p, start + me.token(i), page[i]);
        codes[i] = scales[i] = 0;
        if (at >= 0) {
            const char *row = p.cache.rows + at;
            codes[i] = *(const Codes *)(row + (me.is_v ? Row::kV : 0) + DIMS / 2 * me.part);
            scales[i] = *(const uint8_t *)(row + (me.is_v ? Row::kVScale : Row::kKScale) + me.part / (16 / DIMS));
        }
        to[i] = me.has(p, i) ? me.element(me.is_v ? p.vs : p.ks, i, p.T) : -1;
    }
    void *dst = me.is_v ? p.v : p.k;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (to[i] < 0) continue;
        const u32x4 y = q4_to_bf16(codes[i], q4_scale(scales[i]));
        if constexpr (F32)
            __builtin_nontemporal_store(f32x4{bf16_lo_f32(y[0]), bf16_hi_f32(y[0]), bf16_lo_f32(y[1]), bf16_hi_f32(y[1])},
                                        (f32x4 *)((float *)dst + to[i]));
        else
            __builtin_nontemporal_store(y, (u32x4 *)((__bf16 *)dst + to[i]));
    }
}

template <class Place>
static dim3 grid_rows_q4(const Q4Rows &p, int rows) {
    const int64_t heads = (int64_t)p.cache.B * p.cache.Hkv;
    return dim3((unsigned)(rows == 1 ? (heads * p.T + Place::kRows - 1) / Place::kRows : heads * ((p.T + Place::kTokens - 1) / Place::kTokens)));
}

template <int D, bool F32, int ROWS>
static void launch_rows_q4_form(const Q4Rows &p, bool write, hipStream_t stream) {
    using Written = Q4Place<D, ROWS>;
    using Read = Q4Place<D, ROWS, F32 ? 4 : 8>;
    if (write)
        hipLaunchKernelGGL((cache_write_q4_kernel<D, F32, ROWS>), grid_rows_q4<Written>(p, ROWS), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((cache_read_q4_kernel<D, F32, ROWS>), grid_rows_q4<Read>(p, ROWS), dim3(256), 0, stream, p);
}

template <int D, bool F32>
static void launch_rows_q4(const Q4Rows &p, bool write, hipStream_t stream) {
    if (p.T >= kManyRuns * Q4Place<D, 4>::kTokens && (int64_t)p.cache.B * p.cache.Hkv * p.T >= kManyRows)
        launch_rows_q4_form<D, F32, 4>(p, write, stream);
    else
        launch_rows_q4_form<D, F32, 1>(p, write, stream);
}

static hipError_t launch_rows_q4(const Q4Rows &p, bool write, hipStream_t stream) {
    if (p.cache.d == 128)
        p.f32 ? launch_rows_q4<128, true>(p, write, stream) : launch_rows_q4<128, false>(p, write, stream);
    else
        p.f32 ? launch_rows_q4<64, true>(p, write, stream) : launch_rows_q4<64, false>(p, write, stream);
    return hipGetLastError();
}

hipError_t launch_cache_write_q4(const Q4Rows &p, hipStream_t stream) { return launch_rows_q4(p, true, stream); }
hipError_t launch_cache_read_q4(const Q4Rows &p, hipStream_t stream) { return launch_rows_q4(p, false, stream); }

}  // namespace plx
