// 8-bit floating point by blocks of 128: what the quantiser's and the product's kernels share.
#pragma once

#include "mv_mx.hpp"

namespace mvf {

using mvx::f32x2;
using mvx::f32x4u;
using mvx::kMostGroups;
using mvx::kNanScale;
using mvx::power_of;
using mvx::size_valid;
using mvx::top2;
using mvx::top_of_pair;
using mvx::top_of_quad;
using mvx::u32x4;
using mvx::u32x4u;
using mvx::Values;
using mvx::values_valid;

constexpr int kBlock = 128;                   // values under one scale, and bytes of their codes

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int16_t  i16x2 __attribute__((ext_vector_type(2)));
typedef __bf16   bf16x2 __attribute__((ext_vector_type(2)));

__host__ __device__ constexpr int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

// The scale byte of a block whose largest magnitude has the bit pattern `top`: 448 = 1.75 * 2^8, so the exponent field less 8,
// and one more where the fraction is beyond .75, which the sum carries.  Magnitudes up to 448 * 2^-127 all get 2^-127.
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    const uint32_t e = (top + 0x1FFFFFu) >> 23;
    return top >= 0x7F800000u ? kNanScale : e > 8u ? e - 8u : 0u;
}

// Codes of four values whose block has this scale byte; the instruction divides by the power of two and rounds to the nearest,
// ties to even.  Nothing is beyond 448 times the power.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float power)
{
    i16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, power, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, power, true);
    return __builtin_bit_cast(uint32_t, w);
}
// Of two pairs of bf16 values.
__device__ __forceinline__ uint32_t encode4(uint32_t ab, uint32_t cd, float power)
{
    i16x2 w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, ab), power, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(bf16x2, cd), power, true);
    return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ u32x2 encode8(const uint32_t (&x)[4], uint32_t scale)
{
    if (scale == kNanScale) return u32x2{0u, 0u};
    const float p = power_of(scale);
    return u32x2{encode4(x[0], x[1], p), encode4(x[2], x[3], p)};
}
__device__ __forceinline__ u32x2 encode8(const float (&x)[8], uint32_t scale)
{
    if (scale == kNanScale) return u32x2{0u, 0u};
    const float p = power_of(scale);
    return u32x2{encode4(x[0], x[1], x[2], x[3], p), encode4(x[4], x[5], x[6], x[7], p)};
}
// The way back.  The instruction multiplies by the power of two whose exponent field its operand has, 0 for 2^-127 and 255
// for a NaN.
__device__ __forceinline__ void decode4(uint32_t w, uint32_t scale, float* x)
{
    const float p = mvx::factor_of(scale);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, p, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, p, true);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}

// The larger of the lanes' patterns among each sixteen consecutive lanes.
__device__ __forceinline__ uint32_t top_of_sixteen(uint32_t t)
{
    t = mvx::top_of_eight(t);
    return max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x140, 0xf, 0xf, false));   // lane 15 - i of sixteen
}

// Arguments that every call on codes has in common.
inline bool codes_valid(const void* codes, int64_t ld_bytes, const void* scales, int64_t ld_scales, int64_t n)
{
    return codes && scales && (reinterpret_cast<uintptr_t>(codes) & 15) == 0 && (reinterpret_cast<uintptr_t>(scales) & 3) == 0 &&
           (ld_bytes & 15) == 0 && ld_bytes >= kBlock * blocks_of(n) && (ld_scales & 3) == 0 &&
           ld_scales >= (blocks_of(n) + 3) / 4 * 4;
}
// Blocks are counted in 32 bits.
inline bool count_valid(int64_t rows, int64_t n) { return rows * blocks_of(n) <= (1ll << 29) - 512; }

// A matrix of codes.
struct Factor {
    const uint8_t* codes;
    const uint8_t* scales;
    int64_t        ld_bytes, ld_scales, rows;
};
// One that is written.
struct Held {
    uint8_t* codes;
    uint8_t* scales;
    int64_t  ld_bytes, ld_scales, rows;
};
// In mv_f8.hip; arguments checked by the caller.  The last one: columns of x and of dy and rows of dy, where asked for.
mv_status launch_encode(const Values& v, int32_t dtype, const Held& to, hipStream_t st);
mv_status launch_encode_t(const Values& v, int32_t dtype, const Held& to, hipStream_t st);
mv_status launch_encode_grad(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, int32_t dtype,
                             hipStream_t st);

}  // namespace mvf
