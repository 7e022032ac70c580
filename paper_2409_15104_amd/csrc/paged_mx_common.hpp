// A key/value cache in pages whose values are held in 4 bits (gfx950): the format, and what the kernels on it share.
//
// A head row of 128 values is 64 bytes of codes and four scale bytes.  A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (two
// bits of exponent, one of fraction), the value of dim 2 i in the low half of byte i; the scale byte of 32 dims stands for
// 2^(byte - 127), 255 for NaN.  A group with the largest magnitude a = m 2^E, 1 <= m < 2, takes 2^(E - 2), or 2^(E - 1) where m is
// 1.75 and more: a rounded to two significant bits is 4 or 6 of it then, so that no value is cut off by more than rounding to the
// nearest code costs any value of its size.  Values are rounded to the nearest, ties to the even code.
//
// Codes are the ones the matrix cores of gfx950 have a conversion for: one instruction turns two of them into bf16 with their scale
// applied, which is exact, since such a value has two significant bits; another rounds two bf16 values to codes.  Both take the scale
// as the exponent bits of an fp32 number, whatever its other bits are, so a scale byte only has to be shifted into place.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_common.hpp"

namespace pec {

constexpr int kMxRowBytes = kHeadDim / 2;
constexpr int kMxGroups = 4;                 // of 32 dims
constexpr uint32_t kMxNan = 255;

struct PagedMx {
    unsigned char *k, *v;        // codes (page, slot, head) at page_b * page + row_b * slot + head_b * head, 64 bytes
    unsigned char *ks, *vs;      // scales (page, head, group, slot) at scale_page_b * page + scale_head_b * head + page size * group + slot
    int64_t page_b, scale_page_b;
    uint32_t row_b, head_b, scale_head_b;      // less than 2^31 bytes inside a page
    uint32_t last_page;          // pages - 1
    int32_t log_page;            // log2 of the page size
};

// fp32 bits whose exponent is byte B of `scales`
template <int B>
__device__ __forceinline__ float mx_scale(uint32_t scales) {
    return __builtin_bit_cast(float, B == 3 ? scales >> 1 : scales << (23 - 8 * B));
}
__device__ __forceinline__ float mx_scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// eight codes -> eight bf16 values, in four registers
__device__ __forceinline__ u32x4 mx_values(uint32_t codes, float scale) {
    return u32x4{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}

// The scale byte of a group whose largest magnitude has the bf16 bits `top`, without the sign.  Exponents are kept between -125 and
// 125, so that every value of a group is a normal bf16 number (what is smaller becomes 0 or 2^-126) and none overflows; a group
// with an infinity or NaN is NaN.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
    if (top >= 0x7f80u) return kMxNan;
    return (uint32_t)min(max((int)((top + 32) >> 7) - 2, 2), 252);
}
__device__ __forceinline__ uint32_t mx_codes(const u32x4& x, uint32_t byte) {      // eight bf16 values
    const float scale = mx_scale_of(byte);
    const uint32_t x0 = x[0], x1 = x[1], x2 = x[2], x3 = x[3];      // (a bit_cast of a vector's element would take the first one)
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x0), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x1), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x2), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(bf16x2, x3), scale, 3);
    return byte == kMxNan ? 0u : r;
}

// Largest magnitude, as bf16 bits, of the eight values of each of four neighbouring lanes.
__device__ __forceinline__ uint32_t mx_top_of_group(const u32x4& x) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, x[0] & 0x7fff7fffu);
#pragma unroll
    for (int e = 1; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
    int top = max((int)m[0], (int)m[1]);
    top = max(top, __builtin_amdgcn_update_dpp(0, top, 0xB1, 0xf, 0xf, true));      // the neighbour's
    top = max(top, __builtin_amdgcn_update_dpp(0, top, 0x4E, 0xf, 0xf, true));      // the other two's
    return (uint32_t)top;
}

}  // namespace pec
