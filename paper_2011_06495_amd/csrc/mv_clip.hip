// Gradient norms over many tensors, and clipping by them (mv_clip_* of include/mv.h).
//
//   norm[g] = sqrt(sum x^2) or max |x| over the tensors of group g,  coef[g] = min(1, max_norm / (norm[g] + 1e-6)),
//   dst = src * coef[g]
//
// The list of tensors is cut into chunks, sorted by group, when the handle is made.  A chunk fits a workgroup's registers,
// and a launch's workgroups hold 57 MB together, so a group is read once and written once: its workgroups
// load their chunks, leave their sums, and wait for the group's last workgroup, which adds the sums up in a fixed order.
// 16 x 11.2 M fp32 values: 304 us, 4.7 TB/s; 32 x 25.6 M bf16 760, 4.3; a copy reaches 5.5 to 5.9.
// What is missing: a group's reads and its stores overlap little, and what each group loses between its last load and its
// first store is not known.  More registers, 80 MB of chunks, did not help.
// Memory is the bound; reading a second time, even out of the last-level cache, would be a third of the time (reads from
// there reach 7.0 TB/s on this machine, from memory 6.2).
// The waits are bounded.  Workgroups start in their order, so those that wait have all started as long as nothing else
// holds the units; whoever gives up leaves its chunk to the launch behind, which finds all sums there.  A limit of half a
// millisecond keeps that cheap where something else does.
// Groups too large for that are read twice, by two launches, as a rule with one between them that adds up the group's sums: 25.6 M
// fp32 53 us (gathering 15.8, the sums 4.6, scaling 30), 5.8 TB/s of the three passes, 2^30 bf16 1.2 ms, 5.4.  Groups of up to 256 KB
// are a single workgroup's, in one launch.
//
// Squares of fp32 and bf16 values are exact in fp64 and cannot leave its range; a lane has a few fp64 sums of its own, the
// order of all additions follows from the list's sizes and types, so a norm does not depend on timing.  Maxima are those of the bit
// patterns without the sign: a NaN's pattern is above infinity's, so a NaN stays.
#include "../../include/mv.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <new>
#include <stdint.h>
#include <string.h>

namespace mvc {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// 16 bytes of a thread each.  Eight leave room for seven workgroups to a unit (66 registers a lane), 57 MB in all; sixteen
// for five and 80 MB, but no gain: 16 x 11.2 M fp32 307 : 310 us, 32 x 25.6 M bf16 760 : 773, 25.6 M bf16 to fp32 32.6 : 36.9.
constexpr int kRounds = 8;
constexpr int kChunkBytes = kThreads * kRounds * 16;
constexpr int kSmallWaves = 16, kSmallBytes = 64 * 16;                   // of the kernel for small groups: a wavefront, 16 bytes a lane
constexpr int kSmallRounds = 16, kSmallMost = kSmallWaves * kSmallRounds;   // its chunks of a group
constexpr int kMostSums = 7;        // of a thread of mv_clip_once: chunks of a group over kThreads
constexpr int kBindMost = 128;      // pairs of addresses in the arguments of one launch

// Of one tensor.  But for small groups, a group's last one is empty: the workgroup that adds up.
struct Chunk {
    const void* src;
    void*       dst;
    uint32_t    count, group;
    uint32_t    src_bf16, dst_bf16;
};
struct Tensor {
    uint32_t first, chunks;         // of the list of chunks
};
// What workgroups tell each other, each word with the number of the call it belongs to in its upper half.
struct Sum {
    uint64_t hi, lo;                // the halves of an fp64 sum
};
struct State {
    uint32_t call;                  // never 0
    uint32_t late;                  // workgroups of this call that gave up
    uint32_t fixed;                 // workgroups of the launch behind that are done with their share
    uint32_t pad;
};
struct Lists {
    const Chunk*    chunks;
    const uint32_t* group_first;    // n_groups + 1: chunks of group g are [group_first[g], group_first[g + 1])
    Sum*            sums;           // of each chunk
    uint64_t*       coefs;          // of each group
    uint32_t*       late;           // of each chunk: the last call in which it was left
    State*          state;
    uint32_t        n_chunks, n_groups;
};

// Addresses that come out of memory are not known to be global memory's otherwise; vectors lie at any multiple of their
// element's size.
#define MV_GLOBAL __attribute__((address_space(1)))
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef MV_GLOBAL uint32_t gword;
typedef MV_GLOBAL uint16_t gshort;
typedef uint32_t u32x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x2u __attribute__((ext_vector_type(2), aligned(2)));

// Stores that need not stay in a cache: 25.6 M bf16 to fp32 38.9 -> 34.4 us, 16 x 11.2 M fp32 334 -> 311.
__device__ __forceinline__ void put(MV_GLOBAL void* p, const u32x4& w) { __builtin_nontemporal_store(w, (MV_GLOBAL u32x4u*)p); }
__device__ __forceinline__ void put(MV_GLOBAL void* p, const u32x2& w) { __builtin_nontemporal_store(w, (MV_GLOBAL u32x2u*)p); }

__device__ __forceinline__ float lower(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float upper(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
// Two values to the nearest bf16, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t narrow2(float a, float b)
{
    return __builtin_bit_cast(uint16_t, (__bf16)a) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)b) << 16;
}

// A lane's share of a sum of squares or of a maximum.
template <bool MAX>
struct Share {
    double   sum[4] = {0.0, 0.0, 0.0, 0.0};
    uint32_t top = 0;
    __device__ __forceinline__ void add(int i, float x)
    {
        if constexpr (MAX) {
            top = max(top, __float_as_uint(x) & 0x7FFFFFFFu);
        } else {
            const double v = (double)x;
            sum[i & 3] = fma(v, v, sum[i & 3]);
        }
    }
    // what a lane hands on: a sum, or a maximum's bit pattern (whole numbers below 2^32 are exact in fp64)
    __device__ __forceinline__ double value() const
    {
        if constexpr (MAX) return (double)top;
        else return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
};

template <bool MAX>
__device__ __forceinline__ double joined(double a, double b)
{
    return MAX ? fmax(a, b) : a + b;
}

// The workgroup's sum or maximum, in every thread; `lds` holds a value per wavefront.
template <bool MAX, int WAVES>
__device__ __forceinline__ double of_workgroup(double v, double* lds)
{
    for (int o = 32; o >= 1; o >>= 1) v = joined<MAX>(v, __shfl_xor(v, o, 64));
    if ((threadIdx.x & 63u) == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = joined<MAX>(v, lds[w]);
    __syncthreads();
    return v;
}

template <bool MAX>
__device__ __forceinline__ float norm_of(double v)
{
    return MAX ? __uint_as_float((uint32_t)v) : (float)sqrt(v);
}

__device__ __forceinline__ float coef_of(float norm, float max_norm)
{
    const float c = max_norm / (norm + 1e-6f);
    return c >= 1.0f ? 1.0f : c;                  // NaN stays
}

// How a chunk's elements pass through registers: every store of a wavefront covers one run of memory.
enum class Kind { F32, F32toBf16, Bf16, Bf16toF32 };
__device__ __forceinline__ Kind kind_of(const Chunk& c)
{
    return c.src_bf16 ? (c.dst_bf16 ? Kind::Bf16 : Kind::Bf16toF32) : (c.dst_bf16 ? Kind::F32toBf16 : Kind::F32);
}

// A chunk in registers, ROUNDS x 16 bytes a thread of LANES: vectors of V elements, vector u of thread t being elements
// [(u LANES + t) V, + V) of it.
template <Kind K, int LANES, int ROUNDS>
struct Held {
    static constexpr bool kSrcBf16 = K == Kind::Bf16 || K == Kind::Bf16toF32, kDstBf16 = K == Kind::Bf16 || K == Kind::F32toBf16;
    static constexpr int V = K == Kind::Bf16 ? 8 : 4, kWords = kSrcBf16 ? V / 2 : V, kVectors = ROUNDS * 4 / kWords;
    uint32_t x[kVectors][kWords];

    __device__ __forceinline__ void load_vector(const void* src, int at, int u)
    {
        if constexpr (kWords == 4) {
            const u32x4u v = *(const MV_GLOBAL u32x4u*)((const gshort*)src + (kSrcBf16 ? at : 2 * at));
            x[u][0] = v.x, x[u][1] = v.y, x[u][2] = v.z, x[u][3] = v.w;
        } else {
            const u32x2u v = *(const MV_GLOBAL u32x2u*)((const gshort*)src + at);
            x[u][0] = v.x, x[u][1] = v.y;
        }
    }
    __device__ __forceinline__ void load(const void* src, int n, int t)
    {
        if (n == LANES * kVectors * V) {
#pragma unroll
            for (int u = 0; u < kVectors; ++u) load_vector(src, (u * LANES + t) * V, u);
            return;
        }
#pragma unroll
        for (int u = 0; u < kVectors; ++u) {
            const int at = (u * LANES + t) * V;
#pragma unroll
            for (int i = 0; i < kWords; ++i) x[u][i] = 0;
            if (at + V <= n) {
                load_vector(src, at, u);
            } else if constexpr (kSrcBf16) {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < n) x[u][i / 2] |= (uint32_t)((const gshort*)src)[at + i] << (16 * (i & 1));
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < n) x[u][i] = ((const gword*)src)[at + i];
            }
        }
    }
    // The raw words are all that lives on: without this the compiler keeps widened values over a wait, twice as many registers.
    __device__ __forceinline__ void settle()
    {
#pragma unroll
        for (int u = 0; u < kVectors; ++u)
#pragma unroll
            for (int i = 0; i < kWords; ++i) asm volatile("" : "+v"(x[u][i]));
    }
    __device__ __forceinline__ float value(int u, int i) const
    {
        if constexpr (kSrcBf16) return i & 1 ? upper(x[u][i / 2]) : lower(x[u][i / 2]);
        else return __uint_as_float(x[u][i]);
    }
    __device__ __forceinline__ void store(void* dst, int n, int t, float c) const
    {
#pragma unroll
        for (int u = 0; u < kVectors; ++u) {
            const int at = (u * LANES + t) * V;
            if (at >= n) break;
            float y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = value(u, i) * c;
            if (at + V <= n) {
                if constexpr (!kDstBf16) {
                    const u32x4 w = {__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
                    put((gword*)dst + at, w);
                } else if constexpr (V == 8) {
                    const u32x4 w = {narrow2(y[0], y[1]), narrow2(y[2], y[3]), narrow2(y[4], y[5]), narrow2(y[6], y[7])};
                    put((gshort*)dst + at, w);
                } else {
                    const u32x2 w = {narrow2(y[0], y[1]), narrow2(y[2], y[3])};
                    put((gshort*)dst + at, w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at + i < n) {
                        if constexpr (kDstBf16) ((gshort*)dst)[at + i] = (uint16_t)narrow2(y[i], 0.0f);
                        else ((gword*)dst)[at + i] = __float_as_uint(y[i]);
                    }
            }
        }
    }
    template <bool MAX>
    __device__ __forceinline__ void add(Share<MAX>& share) const
    {
#pragma unroll
        for (int u = 0; u < kVectors; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) share.add(i, value(u, i));
    }
};

// f(a Held of the chunk's kind)
template <int LANES, int ROUNDS, typename F>
__device__ __forceinline__ void by_kind(const Chunk& c, F f)
{
    switch (kind_of(c)) {
        case Kind::F32: { Held<Kind::F32, LANES, ROUNDS> h; f(h); break; }
        case Kind::F32toBf16: { Held<Kind::F32toBf16, LANES, ROUNDS> h; f(h); break; }
        case Kind::Bf16: { Held<Kind::Bf16, LANES, ROUNDS> h; f(h); break; }
        case Kind::Bf16toF32: { Held<Kind::Bf16toF32, LANES, ROUNDS> h; f(h); break; }
    }
}

// ---- words between workgroups ----------------------------------------------------------------------------------------

__device__ __forceinline__ uint64_t read_word(const uint64_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void write_word(uint64_t* p, uint32_t call, uint32_t v)
{
    __hip_atomic_store(p, (uint64_t)call << 32 | v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void write_sum(Sum* s, uint32_t call, double v)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    write_word(&s->hi, call, (uint32_t)(b >> 32));
    write_word(&s->lo, call, (uint32_t)b);
}
__device__ __forceinline__ double sum_of(uint64_t hi, uint64_t lo) { return __longlong_as_double((long long)(hi << 32 | (lo & 0xFFFFFFFFu))); }

// A group's value from its chunks' sums, which an earlier launch has left; the same in every workgroup that asks.  AHEAD of
// a thread's sums are in flight at once; they are added one after the other whatever it is.
template <bool MAX, int AHEAD>
__device__ __forceinline__ double group_value(const Lists& l, uint32_t first, uint32_t last, double* lds)
{
    double v = 0.0;
    for (uint32_t at = first + threadIdx.x; at < last; at += AHEAD * kThreads) {
        Sum s[AHEAD];
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k) s[k] = l.sums[min(at + k * kThreads, last - 1)];
#pragma unroll
        for (uint32_t k = 0; k < AHEAD; ++k)
            if (at + k * kThreads < last) v = joined<MAX>(v, sum_of(s[k].hi, s[k].lo));
    }
    return of_workgroup<MAX, kWaves>(v, lds);
}

// ---- a group's workgroups together ---------------------------------------------------------------------------------

// The group's last workgroup, which has no elements: the sums of all others, in the same order as group_value's.  False:
// one of them was not there in time.
template <bool MAX>
__device__ __forceinline__ bool collect(const Lists& l, uint32_t call, uint32_t first, uint32_t last, uint32_t polls, double* lds, double& value)
{
    // all of a thread's sums in flight at once: one after the other a look takes most of a microsecond
    uint64_t hi[kMostSums], lo[kMostSums];
    bool     all = false;
    for (uint32_t left = polls;; --left) {
        all = true;
#pragma unroll
        for (int k = 0; k < kMostSums; ++k) {
            const uint32_t i = first + threadIdx.x + k * kThreads;
            hi[k] = i < last ? read_word(&l.sums[i].hi) : 0;
            lo[k] = i < last ? read_word(&l.sums[i].lo) : 0;
        }
#pragma unroll
        for (int k = 0; k < kMostSums; ++k)
            all &= first + threadIdx.x + k * kThreads >= last || ((uint32_t)(hi[k] >> 32) == call && (uint32_t)(lo[k] >> 32) == call);
        if (all || left == 0) break;
        __builtin_amdgcn_s_sleep(2);
    }
    double v = 0.0;
#pragma unroll
    for (int k = 0; k < kMostSums; ++k)
        if (first + threadIdx.x + k * kThreads < last) v = joined<MAX>(v, sum_of(hi[k], lo[k]));
    if (!__syncthreads_and(all)) return false;
    value = of_workgroup<MAX, kWaves>(v, lds);
    return true;
}

template <bool MAX>
__global__ __launch_bounds__(kThreads, 7) void mv_clip_once(Lists l, float max_norm, uint32_t polls, float* __restrict__ norms,
                                                            float* __restrict__ coefs)
{
    __shared__ double lds[kWaves];
    __shared__ uint32_t told[2];
    const uint32_t at = blockIdx.x, call = l.state->call;
    const Chunk c = l.chunks[at];
    const uint32_t first = l.group_first[c.group], last = l.group_first[c.group + 1];
    auto give_up = [&] {
        if (threadIdx.x == 0) {
            l.late[at] = call;
            atomicAdd(&l.state->late, 1u);
        }
    };
    if (at + 1 == last) {
        double v;
        if (!collect<MAX>(l, call, first, last - 1, polls, lds, v)) return give_up();
        const float norm = norm_of<MAX>(v), coef = coef_of(norm, max_norm);
        if (threadIdx.x == 0) {
            write_word(&l.coefs[c.group], call, __float_as_uint(coef));
            norms[c.group] = norm;
            if (coefs) coefs[c.group] = coef;
        }
        return;
    }
    by_kind<kThreads, kRounds>(c, [&](auto& h) {
        h.load(c.src, (int)c.count, (int)threadIdx.x);
        Share<MAX> share;
        h.add(share);
        const double sum = of_workgroup<MAX, kWaves>(share.value(), lds);
        if (threadIdx.x == 0) {
            write_sum(&l.sums[at], call, sum);
            uint64_t w = 0;
            for (uint32_t left = polls;; --left) {
                w = read_word(&l.coefs[c.group]);
                if ((uint32_t)(w >> 32) == call || left == 0) break;
                __builtin_amdgcn_s_sleep(8);
            }
            told[0] = (uint32_t)(w >> 32) == call;
            told[1] = (uint32_t)w;
        }
        __syncthreads();
        if (!told[0]) return give_up();
        const float coef = __uint_as_float(told[1]);
        if (coef == 1.0f && c.src == c.dst) return;
        h.settle();
        h.store(c.dst, (int)c.count, (int)threadIdx.x, coef);
    });
}

// A chunk whose factor nobody has left: its workgroup adds up all of its group's sums.
template <bool MAX>
__device__ __forceinline__ void finish_chunk(const Lists& l, uint32_t at, const Chunk& c, float max_norm, float* __restrict__ norms,
                                             float* __restrict__ coefs, double* lds)
{
    const uint32_t first = l.group_first[c.group], last = l.group_first[c.group + 1];
    by_kind<kThreads, kRounds>(c, [&](auto& h) {
        h.load(c.src, (int)c.count, (int)threadIdx.x);               // on its way while the factor is found
        const float norm = norm_of<MAX>(group_value<MAX, 1>(l, first, last, lds));
        const float coef = coef_of(norm, max_norm);
        if (at + 1 == last && threadIdx.x == 0) {
            norms[c.group] = norm;
            if (coefs) coefs[c.group] = coef;
        }
        if (coef == 1.0f && c.src == c.dst) return;
        h.store(c.dst, (int)c.count, (int)threadIdx.x, coef);
    });
}

// Behind mv_clip_once: the chunks that were left, the norms of groups without chunks, and the next call's number.
constexpr int kFixGroups = 64;
template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_rest(Lists l, float max_norm, float* __restrict__ norms, float* __restrict__ coefs,
                                                         bool any_empty)
{
    __shared__ double lds[kWaves];
    const uint32_t late = l.state->late;
    if (any_empty && blockIdx.x == 0)
        for (uint32_t g = threadIdx.x; g < l.n_groups; g += kThreads)
            if (l.group_first[g] == l.group_first[g + 1]) {
                norms[g] = 0.0f;
                if (coefs) coefs[g] = coef_of(0.0f, max_norm);
            }
    if (late == 0) {                              // the same for all workgroups: nobody changes it then
        if (blockIdx.x == 0 && threadIdx.x == 0) l.state->call = l.state->call + 1 ? l.state->call + 1 : 1;
        return;
    }
    const uint32_t call = l.state->call;
    for (uint32_t at = blockIdx.x; at < l.n_chunks; at += kFixGroups)
        if (l.late[at] == call) finish_chunk<MAX>(l, at, l.chunks[at], max_norm, norms, coefs, lds);
    __syncthreads();
    // the last workgroup to come here
    if (threadIdx.x == 0 && atomicAdd(&l.state->fixed, 1u) == kFixGroups - 1) {
        l.state->fixed = 0;
        l.state->late = 0;
        l.state->call = call + 1 ? call + 1 : 1;
    }
}

// ---- a group a workgroup -----------------------------------------------------------------------------------------------

template <bool MAX>
__global__ __launch_bounds__(64 * kSmallWaves) void mv_clip_small(Lists l, float max_norm, float* __restrict__ norms,
                                                                  float* __restrict__ coefs, bool write)
{
    __shared__ double lds[kSmallWaves];
    const uint32_t g = blockIdx.x, first = l.group_first[g], last = l.group_first[g + 1];
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = (int)(threadIdx.x & 63u);
    // 16 bytes a lane of every chunk of this wavefront
    u32x4 x[kSmallRounds];
    Share<MAX> share;
#pragma unroll
    for (int i = 0; i < kSmallRounds; ++i) {
        const uint32_t at = first + wave + i * kSmallWaves;
        if (at >= last) break;                                           // uniform
        const Chunk c = l.chunks[at];
        by_kind<64, 1>(c, [&](auto& h) {
            h.load(c.src, (int)c.count, lane);
            x[i] = __builtin_bit_cast(u32x4, h.x);
        });
    }
#pragma unroll
    for (int i = 0; i < kSmallRounds; ++i) {
        const uint32_t at = first + wave + i * kSmallWaves;
        if (at >= last) break;
        by_kind<64, 1>(l.chunks[at], [&](auto& h) {
            __builtin_memcpy(&h.x, &x[i], sizeof h.x);
            h.add(share);
        });
    }
    const float norm = norm_of<MAX>(of_workgroup<MAX, kSmallWaves>(share.value(), lds)), coef = coef_of(norm, max_norm);
    if (threadIdx.x == 0) {
        norms[g] = norm;
        if (coefs) coefs[g] = coef;
    }
    if (!write) return;
#pragma unroll
    for (int i = 0; i < kSmallRounds; ++i) {
        const uint32_t at = first + wave + i * kSmallWaves;
        if (at >= last) break;
        const Chunk c = l.chunks[at];
        if (coef == 1.0f && c.src == c.dst) continue;
        by_kind<64, 1>(c, [&](auto& h) {
            __builtin_memcpy(&h.x, &x[i], sizeof h.x);
            h.store(c.dst, (int)c.count, lane, coef);
        });
    }
}

// ---- reading twice, and norms alone --------------------------------------------------------------------------------------

template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_gather(Lists l)
{
    __shared__ double lds[kWaves];
    const Chunk c = l.chunks[blockIdx.x];
    Share<MAX> share;
    by_kind<kThreads, kRounds>(c, [&](auto& h) {
        h.load(c.src, (int)c.count, (int)threadIdx.x);
        h.add(share);
    });
    const double v = of_workgroup<MAX, kWaves>(share.value(), lds);
    if (threadIdx.x == 0) {
        const uint64_t b = (uint64_t)__double_as_longlong(v);
        l.sums[blockIdx.x] = {b >> 32, b & 0xFFFFFFFFu};
    }
}

// One workgroup per group.  For mv_clip_scale it leaves the factor.
constexpr int kSumsAhead = 8;
template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_norm(Lists l, float max_norm, float* __restrict__ norms, float* __restrict__ coefs)
{
    __shared__ double lds[kWaves];
    const uint32_t g = blockIdx.x;
    const float norm = norm_of<MAX>(group_value<MAX, kSumsAhead>(l, l.group_first[g], l.group_first[g + 1], lds));
    if (threadIdx.x == 0) {
        const float coef = coef_of(norm, max_norm);
        norms[g] = norm;
        if (coefs) coefs[g] = coef;
        l.coefs[g] = __float_as_uint(coef);                       // of call 0: mv_clip_once waits for another's
    }
}

// The second reading: with the factor that mv_clip_norm leaves, or with every workgroup adding up its group's sums.  That saves a
// launch, but a group's work grows with its square, so it is taken only while all workgroups together read few sums.  us of a
// clip, adding up and with the launch: one fp32 group of 14.7 M values 30.0, 31.4; 20.5 M 39.9, 41.5; 24 M, 8.6 million sums, 46.9,
// 47.7; 25.5 M, 9.7 million, 51.2, 50.2; 32 M 64.5, 60.9; four of 15 M, 13.4 million, 108.6, 105.8; one of 2^30 bf16 3225, 1200.
constexpr uint64_t kSumsRead = 9000000;
template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_add_scale(Lists l, float max_norm, float* __restrict__ norms,
                                                              float* __restrict__ coefs)
{
    __shared__ double lds[kWaves];
    finish_chunk<MAX>(l, blockIdx.x, l.chunks[blockIdx.x], max_norm, norms, coefs, lds);
}
__global__ __launch_bounds__(kThreads) void mv_clip_scale(Lists l)
{
    const Chunk c = l.chunks[blockIdx.x];
    by_kind<kThreads, kRounds>(c, [&](auto& h) {
        h.load(c.src, (int)c.count, (int)threadIdx.x);
        const float coef = __uint_as_float((uint32_t)l.coefs[c.group]);
        if (coef == 1.0f && c.src == c.dst) return;
        h.store(c.dst, (int)c.count, (int)threadIdx.x, coef);
    });
}

struct Pairs {
    const void* src[kBindMost];
    void*       dst[kBindMost];
};
// A workgroup writes one tensor's new addresses into its chunks, `bytes` of src each.
__global__ __launch_bounds__(64) void mv_clip_bind_kernel(Chunk* __restrict__ chunks, const Tensor* __restrict__ tensors, int bytes, Pairs p)
{
    const Tensor t = tensors[blockIdx.x];
    for (uint32_t i = threadIdx.x; i < t.chunks; i += 64) {
        Chunk& c = chunks[t.first + i];
        const size_t at = (size_t)i * (bytes / (c.src_bf16 ? 2 : 4));
        c.src = static_cast<const char*>(p.src[blockIdx.x]) + at * (c.src_bf16 ? 2 : 4);
        c.dst = p.dst[blockIdx.x] ? static_cast<char*>(p.dst[blockIdx.x]) + at * (c.dst_bf16 ? 2 : 4) : nullptr;
    }
}

}  // namespace mvc

struct mv_clip {
    mv_clip_config cfg;
    bool           has_dst, ended, failed, owns_ws, used;
    bool           any_empty;
    bool           small;          // every group a workgroup's
    int            chunk_bytes;
    uint32_t       most_chunks;    // of a group
    uint32_t       at_once;        // workgroups of mv_clip_once that run together
    uint32_t       polls;
    int64_t        n_tensors;
    char*          ws;
    mvc::Lists     lists;
    mvc::Tensor*   tensors;
    mvc::Chunk*    chunks;
    mv_clip_tensor* list;          // the caller's list as it was given
    hipStream_t    last_stream;
};

namespace {

constexpr size_t   kAlign = 256;
// Looks of about a microsecond each.  Alone on the card nobody needs more than 96 (32 x 25.6 M bf16; 64 at 16 x 11.2 M fp32, 24 at
// 25.6 M); where another stream's work holds units, so that a group's workgroups are not all there at once, this is what they
// lose before the launch behind takes over.  Two handles on two streams, 4 x 11.2 M fp32 each, 76 us alone, together 820 us
// (with 2^16 looks 63,500).
constexpr uint32_t kPolls = 512;
constexpr uint64_t kMostChunks = 0xFFFFFF;   // a workgroup of 256 threads each: their threads are counted in 32 bits
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct DeviceGuard {
    int prev = 0;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) return;
        if (prev != dev && hipSetDevice(dev) != hipSuccess) return;
        ok = true;
    }
    ~DeviceGuard() { if (ok) (void)hipSetDevice(prev); }
};

inline size_t elem(int dtype) { return dtype == MV_BF16 ? 2 : 4; }

bool addresses_valid(const mv_clip_tensor& t, const void* src, const void* dst)
{
    if (t.numel == 0) return true;
    if (!src || (reinterpret_cast<uintptr_t>(src) & (elem(t.src_dtype) - 1))) return false;
    if (reinterpret_cast<uintptr_t>(dst) & (elem(t.dst_dtype) - 1)) return false;
    return src != dst || t.src_dtype == t.dst_dtype;
}

struct Sizes {
    uint64_t chunks;
    bool     has_dst, small;
    int      chunk_bytes;
    size_t   off_tensors, off_chunks, off_first, off_state, off_coefs, off_late, off_sums, total;
};

inline uint64_t chunks_of(const mv_clip_tensor& t, int bytes)
{
    const int64_t per = bytes / (int64_t)elem(t.src_dtype);
    return (uint64_t)((t.numel + per - 1) / per);
}

// Allocates a word per group for the time of the call.
mv_status measure(const mv_clip_config* c, const mv_clip_tensor* t, int64_t n, Sizes* s)
{
    if (!c || !t || c->struct_size != sizeof(mv_clip_config) || c->device < 0) return MV_ERR_INVALID_ARG;
    if (c->n_groups < 1 || c->n_groups > 65535 || n < 1 || n > (1 << 24)) return MV_ERR_INVALID_ARG;
    if (c->norm != MV_NORM_L2 && c->norm != MV_NORM_MAX) return MV_ERR_INVALID_ARG;
    uint64_t* pieces = new (std::nothrow) uint64_t[(size_t)c->n_groups]();      // of each group
    if (!pieces) return MV_ERR_ALLOC;
    int64_t  with = 0, without = 0;
    uint64_t large = 0, small = 0, most = 0;
    bool     fine = true;
    for (int64_t i = 0; i < n && fine; ++i) {
        fine = t[i].numel >= 0 && t[i].numel <= ((int64_t)1 << 40) && t[i].group >= 0 && t[i].group < c->n_groups &&
               (t[i].src_dtype == MV_F32 || t[i].src_dtype == MV_BF16) && (t[i].dst_dtype == MV_F32 || t[i].dst_dtype == MV_BF16) &&
               addresses_valid(t[i], t[i].src, t[i].dst);
        if (!fine) break;
        if (t[i].numel) ++(t[i].dst ? with : without);
        large += chunks_of(t[i], mvc::kChunkBytes);
        const uint64_t p = chunks_of(t[i], mvc::kSmallBytes);
        small += p;
        if (p && pieces[t[i].group] == 0) ++large;                        // the group's empty one
        pieces[t[i].group] += p;
        if (pieces[t[i].group] > most) most = pieces[t[i].group];
    }
    delete[] pieces;
    if (!fine || (with && without) || large > kMostChunks) return MV_ERR_INVALID_ARG;
    s->small = most <= (uint64_t)mvc::kSmallMost;
    s->chunk_bytes = s->small ? mvc::kSmallBytes : mvc::kChunkBytes;
    s->chunks = s->small ? small : large;
    s->has_dst = without == 0;
    const size_t chunks = (size_t)s->chunks, groups = (size_t)c->n_groups;
    s->off_tensors = 0;
    s->off_chunks = align_up((size_t)n * sizeof(mvc::Tensor));
    s->off_first = s->off_chunks + align_up(chunks * sizeof(mvc::Chunk));
    s->off_state = s->off_first + align_up((groups + 1) * sizeof(uint32_t));
    s->off_coefs = s->off_state + align_up(sizeof(mvc::State));
    s->off_late = s->off_coefs + align_up(groups * sizeof(uint64_t));
    s->off_sums = s->off_late + align_up(chunks * sizeof(uint32_t));
    s->total = s->off_sums + align_up(chunks * sizeof(mvc::Sum));
    return MV_OK;
}

// The lists as the device holds them; false: no memory.  `most`: a group's largest number of chunks.
bool lay_out(const mv_clip_config* c, const mv_clip_tensor* t, int64_t n, const Sizes& s, char* host, uint32_t* most, bool* any_empty)
{
    mvc::Tensor* tensors = reinterpret_cast<mvc::Tensor*>(host + s.off_tensors);
    mvc::Chunk*  chunks = reinterpret_cast<mvc::Chunk*>(host + s.off_chunks);
    uint32_t*    first = reinterpret_cast<uint32_t*>(host + s.off_first);
    uint32_t*    at = new (std::nothrow) uint32_t[(size_t)c->n_groups];
    if (!at) return false;
    reinterpret_cast<mvc::State*>(host + s.off_state)->call = 1;
    for (int64_t i = 0; i < n; ++i) first[t[i].group + 1] += (uint32_t)chunks_of(t[i], s.chunk_bytes);
    *most = 0;
    *any_empty = false;
    for (int32_t g = 0; g < c->n_groups; ++g) {
        if (first[g + 1] == 0) *any_empty = true;
        else if (!s.small) ++first[g + 1];
        if (first[g + 1] > *most) *most = first[g + 1];
        at[g] = first[g];
        first[g + 1] += first[g];
    }
    for (int64_t i = 0; i < n; ++i) {
        const uint32_t many = (uint32_t)chunks_of(t[i], s.chunk_bytes);
        const bool sb = t[i].src_dtype == MV_BF16, db = t[i].dst_dtype == MV_BF16;
        const int64_t per = s.chunk_bytes / (sb ? 2 : 4);
        tensors[i] = {at[t[i].group], many};
        for (uint32_t k = 0; k < many; ++k) {
            const int64_t from = k * per, left = t[i].numel - from;
            chunks[at[t[i].group]++] = {static_cast<const char*>(t[i].src) + from * (sb ? 2 : 4),
                                        t[i].dst ? static_cast<char*>(t[i].dst) + from * (db ? 2 : 4) : nullptr,
                                        (uint32_t)(left < per ? left : per), (uint32_t)t[i].group, sb, db};
        }
    }
    if (!s.small)
        for (int32_t g = 0; g < c->n_groups; ++g)
            if (first[g] < first[g + 1]) chunks[at[g]] = {nullptr, nullptr, 0, (uint32_t)g, 0, 0};
    delete[] at;
    return true;
}

mv_status usable(const mv_clip* c) { return c->ended || c->failed ? MV_ERR_STATE : MV_OK; }

mv_status done(mv_clip* c)
{
    if (hipGetLastError() == hipSuccess) return MV_OK;
    c->failed = true;
    return MV_ERR_DEVICE;
}

}  // namespace

extern "C" {

size_t mv_clip_workspace_bytes(const mv_clip_config* cfg, const mv_clip_tensor* tensors, int64_t n_tensors)
{
    Sizes s;
    return measure(cfg, tensors, n_tensors, &s) == MV_OK ? s.total : 0;
}

mv_status mv_clip_begin(const mv_clip_config* cfg, const mv_clip_tensor* tensors, int64_t n_tensors, mv_clip** out)
{
    if (!out) return MV_ERR_INVALID_ARG;
    *out = nullptr;
    Sizes s;
    if (const mv_status st = measure(cfg, tensors, n_tensors, &s); st != MV_OK) return st;
    if (cfg->workspace &&
        (cfg->workspace_bytes < s.total || (reinterpret_cast<uintptr_t>(cfg->workspace) & (kAlign - 1)) != 0))
        return MV_ERR_INVALID_ARG;
    mv_clip* c = new (std::nothrow) mv_clip;
    char* host = new (std::nothrow) char[s.total]();
    mv_clip_tensor* list = new (std::nothrow) mv_clip_tensor[(size_t)n_tensors];
    if (c) memset(static_cast<void*>(c), 0, sizeof *c);
    if (!c || !host || !list || !lay_out(cfg, tensors, n_tensors, s, host, &c->most_chunks, &c->any_empty)) {
        delete c;
        delete[] host;
        delete[] list;
        return MV_ERR_ALLOC;
    }
    memcpy(list, tensors, (size_t)n_tensors * sizeof *list);
    c->list = list;
    c->cfg = *cfg;
    c->has_dst = s.has_dst;
    c->small = s.small;
    c->chunk_bytes = s.chunk_bytes;
    c->n_tensors = n_tensors;
    c->polls = kPolls;

    DeviceGuard guard(cfg->device);
    mv_status st = guard.ok ? MV_OK : MV_ERR_DEVICE;
    int per_unit = 0, units = 0;
    if (st == MV_OK && (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_unit, mvc::mv_clip_once<false>, mvc::kThreads, 0) != hipSuccess ||
                        hipDeviceGetAttribute(&units, hipDeviceAttributeMultiprocessorCount, cfg->device) != hipSuccess)) {
        (void)hipGetLastError();
        st = MV_ERR_DEVICE;
    }
    c->at_once = (uint32_t)(per_unit * units);
    if (c->at_once > (uint32_t)(mvc::kMostSums * mvc::kThreads)) c->at_once = mvc::kMostSums * mvc::kThreads;
    if (st == MV_OK) {
        if (cfg->workspace) {
            c->ws = static_cast<char*>(cfg->workspace);
        } else {
            void* p = nullptr;
            if (hipMalloc(&p, s.total) == hipSuccess) {
                c->ws = static_cast<char*>(p);
                c->owns_ws = true;
            } else {
                (void)hipGetLastError();
                st = MV_ERR_ALLOC;
            }
        }
    }
    if (st == MV_OK && hipMemcpy(c->ws, host, s.total, hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        st = MV_ERR_DEVICE;
    }
    delete[] host;
    if (st != MV_OK) {
        if (c->owns_ws) (void)hipFree(c->ws);
        delete[] list;
        delete c;
        return st;
    }
    c->tensors = reinterpret_cast<mvc::Tensor*>(c->ws + s.off_tensors);
    c->chunks = reinterpret_cast<mvc::Chunk*>(c->ws + s.off_chunks);
    c->lists = {c->chunks,
                reinterpret_cast<const uint32_t*>(c->ws + s.off_first),
                reinterpret_cast<mvc::Sum*>(c->ws + s.off_sums),
                reinterpret_cast<uint64_t*>(c->ws + s.off_coefs),
                reinterpret_cast<uint32_t*>(c->ws + s.off_late),
                reinterpret_cast<mvc::State*>(c->ws + s.off_state),
                (uint32_t)s.chunks,
                (uint32_t)cfg->n_groups};
    *out = c;
    return MV_OK;
}

mv_status mv_clip_bind(mv_clip* c, const void* const* src, void* const* dst, void* stream)
{
    if (!c || !src || !dst) return MV_ERR_INVALID_ARG;
    if (const mv_status st = usable(c); st != MV_OK) return st;
    for (int64_t i = 0; i < c->n_tensors; ++i) {
        if (!addresses_valid(c->list[i], src[i], dst[i])) return MV_ERR_INVALID_ARG;
        if (c->list[i].numel && (dst[i] != nullptr) != c->has_dst) return MV_ERR_INVALID_ARG;
    }
    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return MV_ERR_DEVICE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    c->last_stream = st;
    c->used = true;
    for (int64_t i = 0; i < c->n_tensors; i += mvc::kBindMost) {
        const int32_t n = (int32_t)(c->n_tensors - i < mvc::kBindMost ? c->n_tensors - i : mvc::kBindMost);
        mvc::Pairs p;
        memset(&p, 0, sizeof p);
        memcpy(p.src, src + i, (size_t)n * sizeof *src);
        memcpy(p.dst, dst + i, (size_t)n * sizeof *dst);
        hipLaunchKernelGGL(mvc::mv_clip_bind_kernel, dim3((uint32_t)n), dim3(64), 0, st, c->chunks, c->tensors + i, c->chunk_bytes, p);
    }
    return done(c);
}

#define MV_CLIP_LAUNCH(KERNEL, GROUPS, THREADS, ...)                                                                   \
    do {                                                                                                               \
        if (c->cfg.norm == MV_NORM_MAX)                                                                                \
            hipLaunchKernelGGL(mvc::KERNEL<true>, dim3(GROUPS), dim3(THREADS), 0, st, c->lists, ##__VA_ARGS__);        \
        else hipLaunchKernelGGL(mvc::KERNEL<false>, dim3(GROUPS), dim3(THREADS), 0, st, c->lists, ##__VA_ARGS__);      \
    } while (0)

mv_status mv_clip_norms(mv_clip* c, float* norms, void* stream)
{
    if (!c || !norms || (reinterpret_cast<uintptr_t>(norms) & 3)) return MV_ERR_INVALID_ARG;
    if (const mv_status st = usable(c); st != MV_OK) return st;
    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return MV_ERR_DEVICE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    c->last_stream = st;
    c->used = true;
    float* none = nullptr;
    if (c->small) {
        MV_CLIP_LAUNCH(mv_clip_small, c->lists.n_groups, 64 * mvc::kSmallWaves, 0.0f, norms, none, false);
    } else {
        if (c->lists.n_chunks) MV_CLIP_LAUNCH(mv_clip_gather, c->lists.n_chunks, mvc::kThreads);
        MV_CLIP_LAUNCH(mv_clip_norm, c->lists.n_groups, mvc::kThreads, 0.0f, norms, none);
    }
    return done(c);
}

mv_status mv_clip_grads(mv_clip* c, float max_norm, float* norms, float* coefs, void* stream)
{
    if (!c || !norms || (reinterpret_cast<uintptr_t>(norms) & 3) || (reinterpret_cast<uintptr_t>(coefs) & 3))
        return MV_ERR_INVALID_ARG;
    if (!(max_norm >= 0.0f) || isinf(max_norm)) return MV_ERR_INVALID_ARG;
    if (const mv_status st = usable(c); st != MV_OK) return st;
    if (!c->has_dst) return MV_ERR_STATE;
    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return MV_ERR_DEVICE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    c->last_stream = st;
    c->used = true;
    if (c->small) {
        MV_CLIP_LAUNCH(mv_clip_small, c->lists.n_groups, 64 * mvc::kSmallWaves, max_norm, norms, coefs, true);
    } else if (c->most_chunks <= c->at_once) {
        MV_CLIP_LAUNCH(mv_clip_once, c->lists.n_chunks, mvc::kThreads, max_norm, c->polls, norms, coefs);
        MV_CLIP_LAUNCH(mv_clip_rest, mvc::kFixGroups, mvc::kThreads, max_norm, norms, coefs, c->any_empty);
    } else {
        MV_CLIP_LAUNCH(mv_clip_gather, c->lists.n_chunks, mvc::kThreads);
        const bool add = (uint64_t)c->lists.n_chunks * c->most_chunks <= mvc::kSumsRead;
        // norms of groups without chunks are its as well
        if (!add || c->any_empty) MV_CLIP_LAUNCH(mv_clip_norm, c->lists.n_groups, mvc::kThreads, max_norm, norms, coefs);
        if (add) MV_CLIP_LAUNCH(mv_clip_add_scale, c->lists.n_chunks, mvc::kThreads, max_norm, norms, coefs);
        else hipLaunchKernelGGL(mvc::mv_clip_scale, dim3(c->lists.n_chunks), dim3(mvc::kThreads), 0, st, c->lists);
    }
    return done(c);
}
#undef MV_CLIP_LAUNCH

mv_status mv_clip_set_spin_limit(mv_clip* c, uint32_t polls)
{
    if (!c) return MV_ERR_INVALID_ARG;
    if (c->ended) return MV_ERR_STATE;
    c->polls = polls;
    return MV_OK;
}

mv_status mv_clip_end(mv_clip* c)
{
    if (!c) return MV_ERR_INVALID_ARG;
    if (c->ended) return MV_ERR_STATE;
    c->ended = true;
    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return MV_ERR_DEVICE;
    mv_status rc = MV_OK;
    // calls run in their order, so the last one's stream is the one that still holds work
    if (c->used && hipStreamSynchronize(c->last_stream) != hipSuccess) rc = MV_ERR_DEVICE;
    if (c->owns_ws && c->ws && hipFree(c->ws) != hipSuccess) rc = MV_ERR_DEVICE;
    c->ws = nullptr;
    return rc;
}

void mv_clip_release(mv_clip* c)
{
    if (!c) return;
    if (!c->ended) (void)mv_clip_end(c);
    delete[] c->list;
    delete c;
}

}  // extern "C"
