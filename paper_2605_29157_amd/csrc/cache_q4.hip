// Rows of K and V to and from a cache held in 4 bits (plx_q4.h has the row).
//
// Writing: of each 16 dimensions the scale is the power of two s with 3.5 <= max |x| / s < 7, so that the largest rounds to 4 or 6
// and nothing saturates: e = exponent of (max |x| * 8 / 7, rounded down) - 2, one integer addition on the float's bits. (Normal values,
// relative error of a row: 0.110; with s <= max / 4 < 2 s, whose largest magnitudes saturate at 6, 0.118; with max / s <= 6 0.113; 32
// dimensions to a scale 0.112 - 0.115.) x / s is exact, so the one rounding is that to the code, to nearest, ties to even.
//
// What bounds them: the bytes of the rows, 4 D of bf16 and 9 D / 8 of the cache; few rows: one launch. A thread has 8 dimensions (16 bytes
// of bf16) of each of its rows, two neighbours share a scale, and the scale bytes of eight threads are put together, so that
// a row goes out in whole dwords. Many rows: four a thread, all on their way at once.
#include "plx_kernels.h"
#include "plx_q4.h"

namespace plx {

namespace {

// bf16 rows from which a thread takes four: us, written / read, one a thread and four: 1600 rows of d = 128 2.9 / 3.0 and 3.9 / 3.9, 16000
// 5.0 / 5.1 and 5.0 / 5.4, 32000 7.4 / 7.5 and 7.1 / 7.4, 262144 (172 MB) 42 / 42 and 36 / 35. (fp32, which has twice the bytes
// on their way: 131072 rows 29 / 39 and 30 / 43.)
constexpr int64_t kManyRows = 32000;

// Thread -> (K or V, 8 of its dimensions) of the rows row0, row0 + step, ..
template <int D>
struct Q4Place {
    static constexpr int kLanes = D / 8, kThreads = 2 * kLanes;  // of a tensor's row; of a row
    static constexpr int kRows = 256 / kThreads;                 // of a workgroup at a time
    int part;
    bool is_v;
    __device__ __forceinline__ Q4Place() : part(threadIdx.x % kLanes), is_v(threadIdx.x / kLanes % 2 != 0) {}
};
struct Q4Token {
    int b, h, t;
    bool any;
    __device__ __forceinline__ Q4Token(const Q4Rows &p, int64_t row) {
        any = row < (int64_t)p.cache.B * p.cache.Hkv * p.T;
        const uint32_t r = any ? (uint32_t)row : 0, bh = r / (uint32_t)p.T;
        t = (int)(r - bh * p.T);
        b = (int)(bh / p.cache.Hkv), h = (int)(bh - b * p.cache.Hkv);
    }
    // byte offset of a token's row in the cache, or -1
    __device__ __forceinline__ int64_t row_of(const Q4Rows &p, int64_t token) const {
        const Q4Cache &c = p.cache;
        if (token < 0 || token >= c.capacity) return -1;
        const int64_t at = q4_token_offset(c.block_table, c.table_stride, c.page_size, c.num_pages, c.stride, b, token);
        return at < 0 ? -1 : at + h * c.stride[1];
    }
    __device__ __forceinline__ int64_t element(const int64_t (&s)[3]) const { return b * s[0] + h * s[1] + t * s[2]; }
};

}  // namespace

template <int D, bool F32, int ROWS>
__global__ __launch_bounds__(256) void cache_write_q4_kernel(Q4Rows p) {
    using Row = Q4Row<D>;
    using Place = Q4Place<D>;
    const Place me;
    const int64_t row0 = (int64_t)blockIdx.x * (Place::kRows * ROWS) + threadIdx.x / Place::kThreads;
    const void *src = me.is_v ? p.v : p.k;
    int64_t at[ROWS];
    u32x4 raw[ROWS];
    f32x4 wide[ROWS][2];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const Q4Token x(p, row0 + Place::kRows * i);
        const bool counted = x.any && (p.counts == nullptr || x.t < p.counts[x.b]);
        at[i] = counted ? x.row_of(p, (int64_t)(p.start != nullptr ? p.start[x.b] : 0) + x.t) : -1;
        const int64_t e = x.element(me.is_v ? p.vs : p.ks) + 8 * me.part;
        if constexpr (F32) {
            wide[i][0] = *(const f32x4 *)((const float *)src + e), wide[i][1] = *(const f32x4 *)((const float *)src + e + 4);
        } else {
            raw[i] = *(const u32x4 *)((const __bf16 *)src + e);
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (F32)
                x[e] = wide[i][0][e], x[4 + e] = wide[i][1][e];
            else
                x[2 * e] = bf16_lo_f32(raw[i][e]), x[2 * e + 1] = bf16_hi_f32(raw[i][e]);
        }
        uint32_t top = 0;  // of the magnitudes' bits: infinities and NaN are the largest
#pragma unroll
        for (int e = 0; e < 8; ++e) top = max(top, __builtin_bit_cast(uint32_t, x[e]) & 0x7fffffffu);
        top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, true));  // quad_perm [1, 0, 3, 2]
        const bool bad = top >= 0x7f800000u;
        const uint32_t e = (uint32_t)min(max((int)((top + 0x200000u) >> 23) - 2, 4), 252);
        const float scale = q4_scale(e);
        uint32_t codes = 0;
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
        uint32_t scales = (bad ? 255u : e) << (8 * (me.part / 2 & 3));  // four scales of eight lanes
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x4E, 0xf, 0xf, true);   // quad_perm [2, 3, 0, 1]
        scales |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)scales, 0x141, 0xf, 0xf, true);  // row_half_mirror
        if (at[i] < 0) continue;
        char *row = p.cache.rows + at[i];
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
    using Place = Q4Place<D>;
    const Place me;
    const int64_t row0 = (int64_t)blockIdx.x * (Place::kRows * ROWS) + threadIdx.x / Place::kThreads;
    uint32_t codes[ROWS], scales[ROWS];
    int64_t to[ROWS];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const Q4Token x(p, row0 + Place::kRows * i);
        const int64_t token = (int64_t)(p.start != nullptr ? p.start[x.b] : 0) + x.t;
        const int64_t at = p.counts != nullptr && token >= p.counts[x.b] ? -1 : x.row_of(p, token);
        codes[i] = scales[i] = 0;
        if (x.any && at >= 0) {
            const char *row = p.cache.rows + at;
            codes[i] = *(const uint32_t *)(row + (me.is_v ? Row::kV : 0) + 4 * me.part);
            scales[i] = *(const uint8_t *)(row + (me.is_v ? Row::kVScale : Row::kKScale) + me.part / 2);
        }
        to[i] = x.any ? x.element(me.is_v ? p.vs : p.ks) + 8 * me.part : -1;
    }
    void *dst = me.is_v ? p.v : p.k;
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (to[i] < 0) continue;
        const u32x4 y = q4_to_bf16(codes[i], q4_scale(scales[i]));
        if constexpr (F32) {
            float *out = (float *)dst + to[i];
            *(f32x4 *)out = f32x4{bf16_lo_f32(y[0]), bf16_hi_f32(y[0]), bf16_lo_f32(y[1]), bf16_hi_f32(y[1])};
            *(f32x4 *)(out + 4) = f32x4{bf16_lo_f32(y[2]), bf16_hi_f32(y[2]), bf16_lo_f32(y[3]), bf16_hi_f32(y[3])};
        } else {
            *(u32x4 *)((__bf16 *)dst + to[i]) = y;
        }
    }
}

template <int D, bool F32, int ROWS>
static void launch_rows_q4_form(const Q4Rows &p, bool write, hipStream_t stream) {
    constexpr int64_t PER = Q4Place<D>::kRows * ROWS;
    const dim3 grid((unsigned)(((int64_t)p.cache.B * p.cache.Hkv * p.T + PER - 1) / PER));
    if (write)
        hipLaunchKernelGGL((cache_write_q4_kernel<D, F32, ROWS>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((cache_read_q4_kernel<D, F32, ROWS>), grid, dim3(256), 0, stream, p);
}

template <int D, bool F32>
static void launch_rows_q4(const Q4Rows &p, bool write, hipStream_t stream) {
    if constexpr (!F32)
        if ((int64_t)p.cache.B * p.cache.Hkv * p.T >= kManyRows) return launch_rows_q4_form<D, F32, 4>(p, write, stream);
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
