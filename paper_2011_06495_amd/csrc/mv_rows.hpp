// Kernels that work row by row (layer norm, distillation): a row's values in registers, and sums over a row's threads.
#pragma once

#include "mv_mx.hpp"

namespace mvr {

using mvx::dtype_valid;
using mvx::size_valid;
using mvx::u32x4;
using mvx::values_valid;

constexpr float kInf = __builtin_inff();
constexpr int   kNoLds = 0xC07F;        // s_waitcnt: no LDS access in flight
constexpr int   kNoLoads = 0x0F70;      // s_waitcnt: none of the vector loads in flight, the other counters as they are

// A row is LANES threads' (64, 256, 512 or 1024); thread t has chunks t, t + LANES, ... of 16 bytes.
template <typename T>
constexpr int kChunk = 16 / (int)sizeof(T);

// Rows go round a workgroup's groups of LANES threads.
template <int LANES>
constexpr int kThreadsOf = LANES < 256 ? 256 : LANES;

template <typename T>
struct Chunk;
template <>
struct Chunk<float> {
    float x[4];
    // what is not there: -infinity
    __device__ __forceinline__ void take(const u32x4& w)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(w[i]);
    }
    // To the compiler: other values from here on.
    __device__ __forceinline__ void forget() { asm("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3])); }
    __device__ __forceinline__ void none() { x[0] = x[1] = x[2] = x[3] = -kInf; }
    __device__ __forceinline__ void load_low(const float* p, int live)
    {
        if (live >= 4) mvx::load4(p, 4, x);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = i < live ? p[i] : -kInf;
    }
    __device__ __forceinline__ void load(const float* p, int64_t live) { mvx::load4(p, live, x); }
    // What a chunk that a row ends in has been loaded from ends where the row does: its first `live` values are the last ones.
    __device__ __forceinline__ void settle(int live)
    {
        const int s = live > 0 && live < 4 ? 4 - live : 0;
        if (s & 1) x[0] = x[1], x[1] = x[2], x[2] = x[3], x[3] = 0.0f;
        if (s & 2) x[0] = x[2], x[1] = x[3], x[2] = x[3] = 0.0f;
    }
    __device__ __forceinline__ void none_at_all() { x[0] = x[1] = x[2] = x[3] = 0.0f; }
    __device__ __forceinline__ void load_whole(const float* p)
    {
        const mvx::f32x4u v = *reinterpret_cast<const mvx::f32x4u*>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    }
    __device__ __forceinline__ float at(int i) const { return x[i]; }
};
template <>
struct Chunk<uint16_t> {
    uint32_t x[4];
    __device__ __forceinline__ void take(const u32x4& w)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = w[i];
    }
    __device__ __forceinline__ void forget() { asm("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3])); }
    __device__ __forceinline__ void none() { x[0] = x[1] = x[2] = x[3] = 0xFF80FF80u; }
    __device__ __forceinline__ void load_low(const uint16_t* p, int live)
    {
        if (live >= 8) mvx::load8(p, 8, x);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                x[i] = (2 * i < live ? p[2 * i] : 0xFF80u) | (2 * i + 1 < live ? (uint32_t)p[2 * i + 1] : 0xFF80u) << 16;
    }
    __device__ __forceinline__ void load(const uint16_t* p, int64_t live) { mvx::load8(p, live, x); }
    __device__ __forceinline__ void settle(int live)
    {
        const int s = live > 0 && live < 8 ? 8 - live : 0;
        if (s & 1)
            x[0] = __builtin_amdgcn_alignbit(x[1], x[0], 16), x[1] = __builtin_amdgcn_alignbit(x[2], x[1], 16),
            x[2] = __builtin_amdgcn_alignbit(x[3], x[2], 16), x[3] >>= 16;
        if (s & 2) x[0] = x[1], x[1] = x[2], x[2] = x[3], x[3] = 0;
        if (s & 4) x[0] = x[2], x[1] = x[3], x[2] = x[3] = 0;
    }
    __device__ __forceinline__ void none_at_all() { x[0] = x[1] = x[2] = x[3] = 0; }
    __device__ __forceinline__ void load_whole(const uint16_t* p)
    {
        const mvx::u32x4u v = *reinterpret_cast<const mvx::u32x4u*>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? __uint_as_float(x[i / 2] & 0xFFFF0000u) : mvx::widen(x[i / 2]); }
};

// Loads that are on their way while others are at work leave what they bring as it is: a row's last values one by one, each
// waited for, would hold everything up.  A chunk that a row ends in is the row's last values, to be settled when they are used; of
// rows with at least one chunk's.  `live`: values from `col` on.
template <typename T>
__device__ __forceinline__ void load_ahead(Chunk<T>& c, const T* row, int64_t col, int64_t live)
{
    c.none_at_all();
    if (live > 0) c.load_whole(row + col + (live < kChunk<T> ? live - kChunk<T> : 0));
}

// Chunk-sized runs of fp32 or bf16 at any address, in a type that only the call knows.
struct Any {
    const void* p;
    uint32_t    bf16;
    template <int V>
    __device__ __forceinline__ void load(int64_t at, int64_t live, float (&x)[V]) const
    {
#pragma unroll
        for (int h = 0; h < V; h += 4) {
            if (!bf16) {
                float y[4];
                mvx::load4(static_cast<const float*>(p) + at + h, live - h, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h + i] = y[i];
            } else {
                typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
                const uint16_t* q = static_cast<const uint16_t*>(p) + at + h;
                if (live - h >= 4) {
                    const u16x4u w = *reinterpret_cast<const u16x4u*>(q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h + i] = mvx::widen(w[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[h + i] = h + i < live ? mvx::widen(q[i]) : 0.0f;
                }
            }
        }
    }
};
struct AnyOut {
    void*    p;
    uint32_t bf16;
    template <int V>
    __device__ __forceinline__ void store(int64_t at, int64_t live, const float (&x)[V]) const
    {
        if (!bf16) {
#pragma unroll
            for (int h = 0; h < V; h += 4) mvx::store4(static_cast<float*>(p) + at + h, live - h, x + h, V == 4);
        } else if constexpr (V == 8) {
            mvx::store8(static_cast<uint16_t*>(p) + at, live, x);
        } else {
            typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
            uint16_t* q = static_cast<uint16_t*>(p) + at;
            if (live >= 4) {
                const u16x4u w = {(uint16_t)mvx::narrow(x[0]), (uint16_t)mvx::narrow(x[1]), (uint16_t)mvx::narrow(x[2]),
                                  (uint16_t)mvx::narrow(x[3])};
                __builtin_nontemporal_store(w, reinterpret_cast<u16x4u*>(q));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < live) q[i] = (uint16_t)mvx::narrow(x[i]);
            }
        }
    }
    __device__ __forceinline__ void put(int64_t i, float x) const
    {
        if (bf16) static_cast<uint16_t*>(p)[i] = (uint16_t)mvx::narrow(x);
        else static_cast<float*>(p)[i] = x;
    }
};

// A row's whole chunks as a buffer: an offset of the lane's own and one that all share, and no addresses in between.  What lies
// behind them reads as 0 and is not written.
struct RowOf {
    __amdgpu_buffer_rsrc_t buf;
    __device__ __forceinline__ RowOf(const void* p, int bytes)
        : buf(__builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, bytes, 0x00020000))
    {
    }
    __device__ __forceinline__ u32x4 load(uint32_t mine, uint32_t all) const
    {
        return __builtin_amdgcn_raw_buffer_load_b128(buf, mine, all, 0);
    }
    // 1024 bytes of a wavefront straight into LDS.
    __device__ __forceinline__ void load_lds(uint8_t* to, uint32_t mine, uint32_t all) const
    {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(buf, (__attribute__((address_space(3))) void*)to, 16, mine, all, 0, 0);
    }
    // Past the caches.  The whole offset is the lane's: of a store with a shared one in a scalar register the compiler (hipcc 7.2)
    // takes the data as read at once, and the next instruction may write over it; addresses have turned up in place of values.
    __device__ __forceinline__ void store(const u32x4& w, uint32_t mine, uint32_t all) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(w, buf, mine + all, 0, 2);
    }
    // V values at chunk `c` of LANES threads, fp32 or bf16.
    template <int LANES, int V>
    __device__ __forceinline__ void store(const float (&y)[V], uint32_t t, int c, bool bf16) const
    {
        if (!bf16) {
#pragma unroll
            for (int h = 0; h < V; h += 4)
                store(u32x4{__float_as_uint(y[h]), __float_as_uint(y[h + 1]), __float_as_uint(y[h + 2]), __float_as_uint(y[h + 3])},
                      t * (V * 4) + h * 4, c * (LANES * V * 4));
        } else {
            uint32_t w[V / 2];
#pragma unroll
            for (int i = 0; i < V / 2; ++i) w[i] = mvx::narrow(y[2 * i]) | mvx::narrow(y[2 * i + 1]) << 16;
            typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
            if constexpr (V == 8) store(u32x4{w[0], w[1], w[2], w[3]}, t * 16, c * (LANES * 16));
            else __builtin_amdgcn_raw_buffer_store_b64(u32x2{w[0], w[1]}, buf, t * 8 + c * (LANES * 8), 0, 2);
        }
    }
};

template <int CTRL>
__device__ __forceinline__ float moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// Over a wavefront, the same in all lanes: pairs, fours, eights and sixteens of lanes by DPP, then those four.
__device__ __forceinline__ float wave_sum(float v)
{
    v += moved<0xB1>(v);
    v += moved<0x4E>(v);
    v += moved<0x141>(v);
    v += moved<0x140>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_max(float v)                       // of what is no NaN
{
    v = fmaxf(v, moved<0xB1>(v));
    v = fmaxf(v, moved<0x4E>(v));
    v = fmaxf(v, moved<0x141>(v));
    v = fmaxf(v, moved<0x140>(v));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}

// Sums and maxima over the LANES threads of a row; all threads of the workgroup call these together.  Two calls in a row
// use different halves of the LDS, so one barrier each is enough.
template <int LANES>
struct Across {
    static constexpr int kWaves = LANES / 64;
    float (*held)[2][kWaves];           // two halves of two values a wavefront
    int   half = 0;
    __device__ __forceinline__ explicit Across(float (*lds)[2][kWaves]) : held(lds) {}
    __device__ __forceinline__ void sum2(float& a, float& b)
    {
        a = wave_sum(a), b = wave_sum(b);
        if constexpr (LANES > 64) {
            const int wave = threadIdx.x / 64;
            if ((threadIdx.x & 63) == 0) held[half][0][wave] = a, held[half][1][wave] = b;
            __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) a += held[half][0][w], b += held[half][1][w];
            half ^= 1;
        }
    }
    __device__ __forceinline__ float sum(float a)
    {
        a = wave_sum(a);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) held[half][0][threadIdx.x / 64] = a;
            __syncthreads();
            a = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) a += held[half][0][w];
            half ^= 1;
        }
        return a;
    }
    __device__ __forceinline__ float max(float a)
    {
        a = wave_max(a);
        if constexpr (LANES > 64) {
            if ((threadIdx.x & 63) == 0) held[half][0][threadIdx.x / 64] = a;
            __syncthreads();
            a = held[half][0][0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) a = fmaxf(a, held[half][0][w]);
            half ^= 1;
        }
        return a;
    }
};

inline mv_status launched() { return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE; }

}  // namespace mvr
