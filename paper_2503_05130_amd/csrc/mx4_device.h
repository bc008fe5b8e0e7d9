// The microscaled 4-bit form on the device: 32 neighbours share a power of two as a
// scale, 2^(s - 127) of a byte s, and are each one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign (1-2-1 bits).
//
// A block's scale is 2^(floor(log2(largest)) - 2), at least 2^-127: floor(log2) is the exponent field of the largest
// magnitude's bits (fields 0 to 2 end at 2^-127).  x / scale is exact, rounded to the nearest (ties to the even
// code) and cut off at 6, which v_cvt_scalef32_pk_fp4 does as a whole; it takes the scale as an fp32 number
// of which it reads the exponent field alone, 0 as 2^-127 and 255 as NaN.  A block with an infinity or a NaN
// gets the scale byte 255, which makes all of its values NaN, and codes 0.
#pragma once

#include "gemm_device.h"

namespace iefwd {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Between a wave's writes to its own LDS and other lanes' reads of them (and the other way round).  The hardware keeps a wave's LDS
// accesses in order; without this the compiler may take what a lane has read before, or read it where the lane itself has written.
__device__ inline void wave_lds_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Eight neighbours of a lane, and 4 lanes (a quad) a block.
struct Eight {
    u32x4 lo, hi;      // bf16: lo alone; fp32: both
};

// The largest of v over the 4 lanes of a quad.
__device__ inline uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));      // lanes 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));   // lanes 2 3 0 1
}

// The scale byte of the quad's block.
template <bool F32>
__device__ inline uint32_t mx4_scale(const Eight &x) {
    uint32_t field;
    if constexpr (F32) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = max(top, max(x.lo[i] & 0x7fffffffu, x.hi[i] & 0x7fffffffu));
        field = quad_max(top) >> 23;
    } else {
        u16x2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x.lo[i] & 0x7fff7fffu));
        field = quad_max(max(top[0], top[1])) >> 7;
    }
    return field == 255 ? 255u : (uint32_t)max((int)field - 2, 0);
}

// (a function, since __builtin_bit_cast of a vector's element as it stands takes the vector's first)
__device__ inline bf16x2 bf16_pair(uint32_t w) { return __builtin_bit_cast(bf16x2, w); }

// The lane's eight codes, the first in the lowest 4 bits.
template <bool F32>
__device__ inline uint32_t mx4_codes(const Eight &x, uint32_t scale_byte) {
    const float s = __uint_as_float(scale_byte << 23);
    uint32_t w = 0;
    if constexpr (F32) {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.lo[0]), __uint_as_float(x.lo[1]), s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.lo[2]), __uint_as_float(x.lo[3]), s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.hi[0]), __uint_as_float(x.hi[1]), s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, __uint_as_float(x.hi[2]), __uint_as_float(x.hi[3]), s, 3);
    } else {
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x.lo[0]), s, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x.lo[1]), s, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x.lo[2]), s, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, bf16_pair(x.lo[3]), s, 3);
    }
    return scale_byte == 255 ? 0 : w;
}

// Eight codes as bf16 (exact) or fp32.
__device__ inline u32x4 mx4_bf16(uint32_t codes, uint32_t scale_byte) {
    const float s = __uint_as_float(scale_byte << 23);
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
}

// D += A B of 16 x 128 by 128 x 16 in 4 bits.  Lane l: row (column) l % 16 and the 32 of K from 32 (l / 16) on, of
// which byte B of its scale register is the scale; D as for every 16 x 16 product.
template <int B = 0>
__device__ inline f32x4 mfma_mx4(u32x4 a, u32x4 b, f32x4 d, uint32_t a_scale, uint32_t b_scale) {
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, d, 4, 4, B, (int)a_scale, B, (int)b_scale);
}

}  // namespace
}  // namespace iefwd
