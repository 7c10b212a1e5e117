// A cache held in 4 bits, the OCP microscaling format MXFP4 (gfx950 only): 32 neighbouring values of a row share a power of two, each of them is
// an E2M1 code (+-0, 0.5, 1, 1.5, 2, 3, 4, 6; bit 3 is the sign).  A slab, the block of a (page, K or V, kv head), is 16 rows of D / 2 bytes of
// codes, the even element in the low half of a byte, and behind them 16 rows of D / 32 bytes: the exponents of the powers plus 127.
#pragma once
#include "attn_common.h"

namespace tetri_dev {

// Bytes of a slab whose elements have BITS bits: 16 (bf16), 8 (E4M3 codes) or 4.
template <int D, int BITS> __host__ __device__ __forceinline__ constexpr uint32_t slab_bytes()
{
    return BITS == 4 ? kPage * (D / 2 + D / 32) : kPage * D * BITS / 8;
}
template <int D> constexpr uint32_t kFp4Slab = slab_bytes<D, 4>();
template <int D> constexpr uint32_t kFp4Codes = kPage * D / 2;

// The power of two an exponent stands for, as the conversions below take it: they look at the exponent of a 32-bit number only, 0 is 2^-127
// and 255 makes NaN of every code.
__device__ __forceinline__ float fp4_scale(uint32_t exponent) { return __builtin_bit_cast(float, exponent << 23); }

// 8 codes to 8 bf16 values; exact, since a code has two significant bits and the smallest value, 2^-128, is a subnormal bf16 number (under exponents of 253 and 254
// magnitudes of 2^128 and more become infinities).
__device__ __forceinline__ u32x4 fp4_to_bf16(uint32_t codes, float scale)
{
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
    return r;
}

// 8 values of a lane to codes (element i in bits 4i ..), and the exponent that they share with those of the three other lanes of the lane's
// quad, which has to be active as a whole.  The power is that of the largest magnitude divided by 4, so that this becomes 4 .. 6 (what is above 6 after
// rounding is 6); a block with an infinity or a NaN has the exponent 255, which stands for NaN, and codes of 0.  The product with the power's
// inverse is exact; v_cvt_scalef32_pk_fp4_f32 rounds to the nearest code, ties to even, and saturates.  (The conversion that divides by the power itself is
// wrong for 2^-127, a subnormal number.)
__device__ __forceinline__ uint32_t bf16_to_fp4(const u32x4 &v, uint32_t &exponent)
{
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
    int top = max((int)m[0], (int)m[1]);
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0xb1, 0xf, 0xf, true));      // (lane ^ 1)
    top = max(top, __builtin_amdgcn_mov_dpp(top, 0x4e, 0xf, 0xf, true));      // (lane ^ 2)
    const int field = top >> 7;                          // the exponent field of the largest magnitude
    const bool finite = field != 255;
    exponent = finite ? (uint32_t)max(field - 2, 0) : 255u;
    const float inv = __builtin_bit_cast(float, (254u - min(exponent, 253u)) << 23);       // 1 over the power (up to 2^127: the values may be subnormal)
    auto value = [&](int j) -> float { return __builtin_bit_cast(float, (j & 1) ? v[j / 2] & 0xffff0000u : v[j / 2] << 16) * inv; };
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(0), value(1), 1.0f, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(2), value(3), 1.0f, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(4), value(5), 1.0f, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, value(6), value(7), 1.0f, 3);
    return finite ? codes : 0u;
}

// Loads of codes and exponents as global-memory instructions (see global_u32x4).
__device__ __forceinline__ void load_fp4_codes(const char *p, uint32_t (&c)[4])
{
    const u32x4 x = *reinterpret_cast<global_u32x4 *>((uintptr_t)p);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = x[i];
}
__device__ __forceinline__ void load_fp4_codes(const char *p, uint32_t (&c)[2])
{
    const u32x2 x = *reinterpret_cast<__attribute__((address_space(1))) const u32x2 *>((uintptr_t)p);
    c[0] = x[0];
    c[1] = x[1];
}
__device__ __forceinline__ uint32_t load_global_byte(const char *p)
{
    return *reinterpret_cast<__attribute__((address_space(1))) const uint8_t *>((uintptr_t)p);
}

// Chunk `c` (8 values) of row `row` of a slab is stored: the codes by every lane, the exponent by the first of the four lanes of a group of 32.
template <int D> __device__ __forceinline__ void store_fp4(char *slab, int row, int c, uint32_t codes, uint32_t exponent)
{
    *reinterpret_cast<__attribute__((address_space(1))) uint32_t *>((uintptr_t)(slab + row * (D / 2) + c * 4)) = codes;
    if ((c & 3) == 0)
        *reinterpret_cast<__attribute__((address_space(1))) uint8_t *>((uintptr_t)(slab + kFp4Codes<D> + row * (D / 32) + c / 4)) = (uint8_t)exponent;
}

}  // namespace tetri_dev
