// What the products of 4-bit and of 8-bit matrices share: where results go, how launches are put together, and which tile a
// workgroup takes.
#pragma once

#include "mv_mx.hpp"

namespace mvx {

typedef int   i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// Where results go: fp32 or bf16, rounded once.
struct Out {
    void*    p;
    uint32_t bf16;
    __device__ __forceinline__ void put(int64_t at, float x) const
    {
        if (bf16) static_cast<uint16_t*>(p)[at] = (uint16_t)narrow(x);
        else static_cast<float*>(p)[at] = x;
    }
    // four consecutive ones of which `live` are left
    __device__ __forceinline__ void put4(int64_t at, int64_t live, const f32x4& v) const
    {
        typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
        if (live >= 4) {
            if (bf16)
                *reinterpret_cast<u16x4u*>(static_cast<uint16_t*>(p) + at) =
                    u16x4u{(uint16_t)narrow(v.x), (uint16_t)narrow(v.y), (uint16_t)narrow(v.z), (uint16_t)narrow(v.w)};
            else
                *reinterpret_cast<f32x4u*>(static_cast<float*>(p) + at) = v;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < live) put(at + e, v[e]);
        }
    }
};

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

constexpr int kNoLoads = 0x0F70;    // s_waitcnt: none of the vector loads in flight, the other counters as they are

// One or two products of a launch, the first workgroups are the first one's.  A launch from the host takes a microsecond
// longer with 400 bytes of arguments than with 8, so a single product's have room for one only.
template <typename P, bool PAIR>
struct Launch {
    P        products[PAIR ? 2 : 1];
    uint32_t firsts;
    __device__ __forceinline__ const P& product() const { return products[PAIR && blockIdx.x >= firsts ? 1 : 0]; }
    __device__ __forceinline__ uint32_t id() const { return PAIR && blockIdx.x >= firsts ? blockIdx.x - firsts : blockIdx.x; }
};

// Which tile a workgroup takes: consecutive workgroups run on eight dies with an L2 of their own, so a die gets a run of
// consecutive tiles, and those go down eight tiles of a before they go along b.
__device__ __forceinline__ void tile_of(uint32_t id, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn)
{
    const uint32_t all = tiles_m * tiles_n, each = all / 8, more = all % 8, die = id % 8;
    const uint32_t t = die * each + min(die, more) + id / 8;
    const uint32_t band = t / (8 * tiles_n), first = band * 8, high = min(8u, tiles_m - first), in = t - first * tiles_n;
    tm = first + in % high;
    tn = in / high;
}

// c = the sum of the splits: a group of `lanes` threads takes four results, each thread every lanes-th split, and their
// sums are added in order.
__device__ __forceinline__ void join_splits(uint32_t id, const float* __restrict__ parts, uint32_t splits, uint32_t lanes, int64_t m,
                                            int64_t n, int64_t split_c, int64_t quads, Out c, int64_t ld_c)
{
    __shared__ f32x4 sums[256];
    const uint32_t per = 256 / lanes, lane = threadIdx.x / per;          // a group's threads lie `per` apart
    const int64_t at = (int64_t)id * per + threadIdx.x % per;
    const int64_t i = at / quads, j = at % quads * 4;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < m) {
        const float* p = parts + i * (quads * 4) + j;
        uint32_t s = lane;
        for (; s + 3 * lanes < splits; s += 4 * lanes)
#pragma unroll
            for (uint32_t u = 0; u < 4; ++u) sum += *reinterpret_cast<const f32x4*>(p + (s + u * lanes) * split_c);
        // the last ones at once, too, not one after the other
        if (s < splits) {
            f32x4 v[3];
#pragma unroll
            for (uint32_t u = 0; u < 3; ++u) v[u] = *reinterpret_cast<const f32x4*>(p + min(s + u * lanes, splits - 1) * split_c);
#pragma unroll
            for (uint32_t u = 0; u < 3; ++u)
                if (s + u * lanes < splits) sum += v[u];
        }
    }
    if (lanes > 1) {                                                     // uniform
        sums[threadIdx.x] = sum;
        __syncthreads();
        if (lane) return;
        for (uint32_t l = 1; l < lanes; ++l) sum += sums[l * per + threadIdx.x];
    }
    if (i < m) c.put4(i * ld_c + j, n - j, sum);
}

inline int64_t quads_of(int64_t n) { return (n + 3) / 4; }

// Results of 16 MB and more, which are half of the L2s, are stored past them.  Smaller ones, and sums that are added up right
// away, are a little faster stored as usual: 1000 x 1000 by 1000 7.8 us, past the caches 8.0; 130 x 130 by 8000 14.1 : 16.3.  From
// 8 to 67 MB a product alone takes as long either way (4096 x 8192 by 8192 140.6 : 140.5).
constexpr int64_t kPastBytes = 16 << 20;

inline bool scratch_valid(const void* p, size_t have, size_t need)
{
    return need == 0 || (p && have >= need && (reinterpret_cast<uintptr_t>(p) & 15) == 0);
}
inline bool sizes_valid(int64_t m, int64_t n, int64_t k) { return size_valid(m) && size_valid(n) && size_valid(k); }

}  // namespace mvx
