// Microscaled 4-bit values: what the quantiser's and the product's kernels share.
#pragma once

#include "../../include/mv.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mvx {

constexpr int      kBlock = 32;               // values under one scale
constexpr uint32_t kNanScale = 255;
constexpr int64_t  kMostGroups = 0xFFFFFF;    // workgroups of 256 threads in a launch: their threads are counted in 32 bits

typedef float    f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Vectors at any multiple of their element's size.
typedef float    f32x4u __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));

__host__ __device__ constexpr int64_t blocks_of(int64_t n) { return (n + kBlock - 1) / kBlock; }

__device__ __forceinline__ float widen(uint32_t b) { return __uint_as_float(b << 16); }

// To the nearest bf16, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Values [0, 8) of p, those at `live` and behind as zeros.
__device__ __forceinline__ void load8(const float* p, int64_t live, float (&x)[8])
{
    if (live >= 8) {
        const f32x4u a = *reinterpret_cast<const f32x4u*>(p), b = *reinterpret_cast<const f32x4u*>(p + 4);
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < live ? p[i] : 0.0f;
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, int64_t live, float (&x)[8])
{
    if (live >= 8) {
        const u32x4u a = *reinterpret_cast<const u32x4u*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(a[i] << 16);
            x[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = i < live ? widen(p[i]) : 0.0f;
    }
}
// As they are.
__device__ __forceinline__ void load8(const uint16_t* p, int64_t live, uint32_t (&x)[4])
{
    if (live >= 8) {
        const u32x4u a = *reinterpret_cast<const u32x4u*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (2 * i < live ? p[2 * i] : 0u) | (2 * i + 1 < live ? (uint32_t)p[2 * i + 1] << 16 : 0u);
    }
}
__device__ __forceinline__ void load4(const float* p, int64_t live, float (&x)[4])
{
    if (live >= 4) {
        const f32x4u v = *reinterpret_cast<const f32x4u*>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < live ? p[i] : 0.0f;
    }
}
// Stores of which a wavefront's cover one run of memory pass the caches: 8192 x 4096 bf16 quantised and read back 36.5 ->
// 29.3 us.  Where lanes leave gaps for a second store, that costs more than it saves (fp32 in 32 bytes a lane 57 -> 78 us).
__device__ __forceinline__ void store4(float* p, int64_t live, const float* x, bool past = true)
{
    if (live >= 4) {
        const f32x4u v = {x[0], x[1], x[2], x[3]};
        if (past) __builtin_nontemporal_store(v, reinterpret_cast<f32x4u*>(p));
        else *reinterpret_cast<f32x4u*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < live) p[i] = x[i];
    }
}
__device__ __forceinline__ void store8(float* p, int64_t live, const float (&x)[8])
{
    if (live >= 8) {
        const f32x4u a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        *reinterpret_cast<f32x4u*>(p) = a;
        *reinterpret_cast<f32x4u*>(p + 4) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < live) p[i] = x[i];
    }
}
__device__ __forceinline__ void store8(uint16_t* p, int64_t live, const float (&x)[8], bool past = true)
{
    if (live >= 8) {
        u32x4u a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = narrow(x[2 * i]) | narrow(x[2 * i + 1]) << 16;
        if (past) __builtin_nontemporal_store(a, reinterpret_cast<u32x4u*>(p));
        else *reinterpret_cast<u32x4u*>(p) = a;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < live) p[i] = (uint16_t)narrow(x[i]);
    }
}

// The scale byte of a block whose largest magnitude has the bit pattern `top` (patterns without their sign have the
// values' order, a NaN's is above infinity's): floor(log2) is the exponent field, less 2 for the grid's 6 = 1.5 * 2^2.
// Magnitudes below 2^-125 all get 2^-127, which is the byte 0.
__device__ __forceinline__ uint32_t scale_of(uint32_t top)
{
    const uint32_t e = top >> 23;
    return e == 255u ? kNanScale : e > 2u ? e - 2u : 0u;
}
// 2 ** (scale byte - 127); the byte 0 is 2^-127, a denormal.
__device__ __forceinline__ float power_of(uint32_t scale)
{
    return __uint_as_float(scale ? scale << 23 : 1u << 22);
}

// Codes of eight values whose block has this scale byte.  The instruction divides by the power of two, rounds to the
// nearest, ties to even, and cuts at 6: compared with the definition on 4614 values from denormals to 2^125.
__device__ __forceinline__ uint32_t encode8(const float (&x)[8], uint32_t scale)
{
    if (scale == kNanScale) return 0u;
    const float p = power_of(scale);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], p, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], p, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], p, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], p, 3);
    return w;
}
// The way back: the instruction multiplies by the power of two whose exponent field its operand has, with 0 for 2^-127 and 255
// for a NaN: compared with the definition for all scales and codes.
__device__ __forceinline__ float factor_of(uint32_t scale) { return __uint_as_float(scale << 23); }
__device__ __forceinline__ void decode8(uint32_t w, uint32_t scale, float (&x)[8])
{
    const float p = factor_of(scale);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 1);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 3);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}

// Of four values: 16 bits.
__device__ __forceinline__ uint32_t encode4(const float (&x)[4], uint32_t scale)
{
    if (scale == kNanScale) return 0u;
    const float p = power_of(scale);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], p, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], p, 1);
}
__device__ __forceinline__ void decode4(uint32_t w, uint32_t scale, float (&x)[4])
{
    const float p = factor_of(scale);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 1);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}

// The same of bf16 pairs as they are.
typedef __bf16   bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t encode8(const uint32_t (&x)[4], uint32_t scale)
{
    if (scale == kNanScale) return 0u;
    const float p = power_of(scale);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[0]), p, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[1]), p, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[2]), p, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x[3]), p, 3);
    return w;
}
// The larger patterns without their sign, of each half.
__device__ __forceinline__ uint32_t top2(uint32_t t, uint32_t x)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, t), __builtin_bit_cast(u16x2, x & 0x7FFF7FFFu)));
}
// The larger half as an fp32 pattern.
__device__ __forceinline__ uint32_t top_of_pair(uint32_t t) { return max(t & 0xFFFF0000u, t << 16); }

// The larger of the lanes' patterns among each four consecutive lanes.
__device__ __forceinline__ uint32_t top_of_quad(uint32_t t)
{
    t = max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xf, 0xf, false));   // lanes 1 0 3 2
    return max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xf, 0xf, false)); // lanes 2 3 0 1
}

// ... among each eight.
__device__ __forceinline__ uint32_t top_of_eight(uint32_t t)
{
    t = top_of_quad(t);
    return max(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x141, 0xf, 0xf, false));   // lane 7 - i of eight
}

// Arguments that every call on codes has in common.
inline bool codes_valid(const void* codes, int64_t ld_words, const void* scales, int64_t ld_scales, int64_t n)
{
    return codes && scales && (reinterpret_cast<uintptr_t>(codes) & 15) == 0 && (reinterpret_cast<uintptr_t>(scales) & 3) == 0 &&
           (ld_words & 3) == 0 && ld_words >= 4 * blocks_of(n) && (ld_scales & 3) == 0 && ld_scales >= (blocks_of(n) + 3) / 4 * 4;
}
inline bool size_valid(int64_t n) { return n >= 1 && n <= 0x7FFFFFFFll; }
// A launch's threads are counted in 32 bits, at most eight to a block.
inline bool count_valid(int64_t rows, int64_t n) { return rows * blocks_of(n) <= (1ll << 29) - 512; }
inline bool dtype_valid(int32_t t) { return t == MV_F32 || t == MV_BF16; }
inline bool values_valid(const void* p, int32_t dtype, int64_t ld, int64_t n)
{
    return p && dtype_valid(dtype) && (reinterpret_cast<uintptr_t>(p) & (dtype == MV_BF16 ? 1 : 3)) == 0 && ld >= n;
}

// A matrix of values, and codes that are written.
struct Values {
    const void* p;
    int64_t     ld, rows, n;
};
struct Held {
    uint32_t* codes;
    uint8_t*  scales;
    int64_t   ld_words, ld_scales, rows;
};
// In mv_mx.hip; arguments checked by the caller.  The last one: columns of x and of dy and rows of dy, where asked for.
mv_status launch_encode(const Values& v, int32_t dtype, const Held& to, float* resid, int64_t ld_resid, hipStream_t st);
mv_status launch_encode_t(const Values& v, int32_t dtype, const Held& to, hipStream_t st);
mv_status launch_encode_grad(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, int32_t dtype,
                             hipStream_t st);

}  // namespace mvx
