// Rows of K and V to and from a cache held in 4 bits (plx_q4.h has the row).
//
// Writing: of each 16 dimensions the scale is the power of two s with 3.5 <= max |x| / s < 7, so that the largest rounds to 4 or 6
// and nothing saturates: e = exponent of (max |x| * 8 / 7, rounded down) - 2, one integer addition on the float's bits. (Normal values,
// relative error of a row: 0.110; with s <= max / 4 < 2 s, whose largest magnitudes saturate at 6, 0.118; with max / s <= 6 0.113; 32
// dimensions to a scale 0.112 - 0.115.) x / s is exact, so the one rounding is that to the code, to nearest, ties to even.
//
// What bounds them: the bytes of the rows, 4 D of bf16 and 9 D / 8 of the cache; few rows: one launch. A thread has 16 dimensions, one
// scale: no exchange between lanes.
#include "plx_kernels.h"
#include "plx_q4.h"

namespace plx {

namespace {

// Thread -> (row, K or V, 16 of its dimensions)
template <int D>
struct Q4Place {
    static constexpr int kGroups = D / 16, kThreads = 2 * kGroups;  // of a tensor's row; of a row
    int b, h, t, group;
    bool is_v, any;
    __device__ __forceinline__ Q4Place(const Q4Rows &p) {
        const int64_t row = (int64_t)blockIdx.x * (256 / kThreads) + threadIdx.x / kThreads;
        const int part = threadIdx.x % kThreads;
        is_v = part >= kGroups, group = part % kGroups;
        any = row < (int64_t)p.cache.B * p.cache.Hkv * p.T;
        const int64_t bh = row / p.T;
        t = (int)(row - bh * p.T);
        b = (int)(bh / p.cache.Hkv), h = (int)(bh - (int64_t)b * p.cache.Hkv);
    }
    // byte offset of this row in the cache, or -1
    __device__ __forceinline__ int64_t row_of(const Q4Rows &p, int64_t token) const {
        const Q4Cache &c = p.cache;
        if (token < 0 || token >= c.capacity) return -1;
        const int64_t at = q4_token_offset(c.block_table, c.table_stride, c.page_size, c.num_pages, c.stride, b, token);
        return at < 0 ? -1 : at + h * c.stride[1];
    }
    __device__ __forceinline__ int64_t element(const Q4Rows &p) const {  // of this thread's dimensions in k or v
        const int64_t(&s)[3] = is_v ? p.vs : p.ks;
        return b * s[0] + h * s[1] + t * s[2] + 16 * group;
    }
};

}  // namespace

template <int D, bool F32>
__global__ __launch_bounds__(256) void cache_write_q4_kernel(Q4Rows p) {
    using Row = Q4Row<D>;
    const Q4Place<D> me(p);
    if (!me.any || (p.counts != nullptr && me.t >= p.counts[me.b])) return;
    const int64_t at = me.row_of(p, (int64_t)(p.start != nullptr ? p.start[me.b] : 0) + me.t);
    if (at < 0) return;
    float x[16];
    const void *src = me.is_v ? p.v : p.k;
    if constexpr (F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x4 y = *(const f32x4 *)((const float *)src + me.element(p) + 4 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 y = *(const u32x4 *)((const __bf16 *)src + me.element(p) + 8 * i);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[8 * i + 2 * e] = bf16_lo_f32(y[e]), x[8 * i + 2 * e + 1] = bf16_hi_f32(y[e]);
        }
    }
    uint32_t top = 0;  // of the magnitudes' bits: infinities and NaN are the largest
#pragma unroll
    for (int i = 0; i < 16; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    const bool bad = top >= 0x7f800000u;
    const uint32_t e = (uint32_t)min(max((int)((top + 0x200000u) >> 23) - 2, 4), 252);
    const float scale = q4_scale(e);
    u32x2 codes = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 0], x[8 * i + 1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 2], x[8 * i + 3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 4], x[8 * i + 5], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[8 * i + 6], x[8 * i + 7], scale, 3);
        codes[i] = bad ? 0u : c;
    }
    char *row = p.cache.rows + at;
    *(u32x2 *)(row + (me.is_v ? Row::kV : 0) + 8 * me.group) = codes;
    *(uint8_t *)(row + (me.is_v ? Row::kVScale : Row::kKScale) + me.group) = (uint8_t)(bad ? 255u : e);
    if constexpr (Row::kBytes > Row::kEnd) {
        static_assert(Row::kBytes - Row::kEnd == 8 && Row::kEnd % 8 == 0, "one store");
        if (me.is_v && me.group == 0) *(u32x2 *)(row + Row::kEnd) = u32x2{0u, 0u};
    }
}

template <int D, bool F32>
__global__ __launch_bounds__(256) void cache_read_q4_kernel(Q4Rows p) {
    using Row = Q4Row<D>;
    const Q4Place<D> me(p);
    if (!me.any) return;
    const int64_t token = (int64_t)(p.start != nullptr ? p.start[me.b] : 0) + me.t;
    const int64_t at = p.counts != nullptr && token >= p.counts[me.b] ? -1 : me.row_of(p, token);
    u32x4 y[2] = {{0u, 0u, 0u, 0u}, {0u, 0u, 0u, 0u}};
    if (at >= 0) {
        const char *row = p.cache.rows + at;
        const u32x2 codes = *(const u32x2 *)(row + (me.is_v ? Row::kV : 0) + 8 * me.group);
        const float scale = q4_scale(*(const uint8_t *)(row + (me.is_v ? Row::kVScale : Row::kKScale) + me.group));
        y[0] = q4_to_bf16(codes[0], scale), y[1] = q4_to_bf16(codes[1], scale);
    }
    void *dst = me.is_v ? p.v : p.k;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (F32) {
            float *out = (float *)dst + me.element(p) + 8 * i;
            *(f32x4 *)out = f32x4{bf16_lo_f32(y[i][0]), bf16_hi_f32(y[i][0]), bf16_lo_f32(y[i][1]), bf16_hi_f32(y[i][1])};
            *(f32x4 *)(out + 4) = f32x4{bf16_lo_f32(y[i][2]), bf16_hi_f32(y[i][2]), bf16_lo_f32(y[i][3]), bf16_hi_f32(y[i][3])};
        } else {
            *(u32x4 *)((__bf16 *)dst + me.element(p) + 8 * i) = y[i];
        }
    }
}

template <int D, bool F32>
static void launch_rows_q4(const Q4Rows &p, bool write, hipStream_t stream) {
    constexpr int64_t PER = 256 / Q4Place<D>::kThreads;
    const dim3 grid((unsigned)(((int64_t)p.cache.B * p.cache.Hkv * p.T + PER - 1) / PER));
    if (write)
        hipLaunchKernelGGL((cache_write_q4_kernel<D, F32>), grid, dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((cache_read_q4_kernel<D, F32>), grid, dim3(256), 0, stream, p);
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
