// The row of a 4-bit cache: K and V of one token and key head (cache_q4.hip writes and reads them, decode_q4_bf16.hip and
// block_select.hip read them).
//
// Codes are e2m1 (sign, 2 bits of exponent, 1 of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6), which this chip's conversions take eight to a
// dword together with a scale 2^(e - 127), given as the float that has e as its exponent bits (e = 255: NaN). A scale serves 16
// dimensions: with K and V in one row, which is a multiple of 16 bytes, 16 cost no more than 32 would (d = 128: 128 bytes of codes
// and 16 or 8 of scales, 144 both ways; d = 64: 64 and 8 or 4, 80 both ways).
#pragma once
#include <type_traits>
#include <utility>

#include "plx_device.h"

namespace plx {

template <int D>
struct Q4Row {
    static constexpr int kV = D / 2;                 // V codes (K codes: 0)
    static constexpr int kKScale = D;                // scale bytes of K
    static constexpr int kVScale = D + D / 16;       // ... of V
    static constexpr int kEnd = D + D / 8;           // zeros from here
    static constexpr int kBytes = (kEnd + 15) / 16 * 16;
};

__device__ __forceinline__ float q4_scale(uint32_t e) { return __builtin_bit_cast(float, e << 23); }
// ... of byte n (a constant) of four: one instruction, where a mask and a shift are two (decode of 16 x 32768 keys, 8 heads, at one split
// 173 us, so 167)
__device__ __forceinline__ float q4_scale_byte(uint32_t scales, int n) {
    uint32_t y;
    const uint32_t at = 23;
#define PLX_Q4_SCALE(BYTE) \
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:" BYTE : "=v"(y) : "v"(at), "v"(scales))
    if (n == 0)
        PLX_Q4_SCALE("BYTE_0");
    else if (n == 1)
        PLX_Q4_SCALE("BYTE_1");
    else if (n == 2)
        PLX_Q4_SCALE("BYTE_2");
    else
        PLX_Q4_SCALE("BYTE_3");
#undef PLX_Q4_SCALE
    return __builtin_bit_cast(float, y);
}

// Eight codes times their scale, as bf16 (exact but for overflow, which is infinite)
__device__ __forceinline__ u32x4 q4_to_bf16(uint32_t codes, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// Eight codes as they are, in f16 (0 .. 6)
__device__ __forceinline__ u32x4 q4_to_f16(uint32_t codes) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.f, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.f, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.f, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.f, 3))};
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}
__device__ __forceinline__ float add_f16_pair(uint32_t x, float sum) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, x), f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
}
__device__ __forceinline__ uint32_t mul_f16_pair(uint32_t x, uint32_t y) {
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, x) * __builtin_bit_cast(f16x2, y));
}
__device__ __forceinline__ f32x4 mfma16_f16(u32x4 a, u32x4 b, f32x4 c) {
    typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Transposing LDS reads. Within each group of 16 lanes, lane i gets nibble i of the 8 bytes that each of the 16 lanes addresses, in the
// order of the lanes (ds_read_b64_tr_b4), or byte i % 8 of the 8 bytes that every other lane addresses, from lane i / 8 on
// (ds_read_b64_tr_b8).
__device__ __forceinline__ u32x2 lds_read_tr4(const void *generic_lds_ptr) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef i32x2 __attribute__((address_space(3))) * lds_ptr_t;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_ptr_t)generic_lds_ptr));
}
__device__ __forceinline__ u32x2 lds_read_tr8(const void *generic_lds_ptr) {
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef i32x2 __attribute__((address_space(3))) * lds_ptr_t;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_ptr_t)generic_lds_ptr));
}

// f(0), f(1), .. f(N - 1) with the numbers as types
template <int N, class F, int... I>
__device__ __forceinline__ void each_of(F &f, std::integer_sequence<int, I...>) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void each_of(F &f) {
    each_of<N>(f, std::make_integer_sequence<int, N>{});
}

}  // namespace plx
