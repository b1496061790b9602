// Gradient norms over many tensors, and clipping by them (mv_clip_* of include/mv.h).
//
//   norm[g] = sqrt(sum x^2) or max |x| over the tensors of group g,  coef[g] = min(1, max_norm / (norm[g] + 1e-6)),
//   dst = src * coef[g]
//
// The list of tensors is cut into chunks of at most kChunk elements, sorted by group, when the handle is made.
// Two launches: a workgroup per chunk leaves the chunk's sum (or maximum); a workgroup per chunk adds up its group's
// sums in a fixed order, which every workgroup of the group does alike, and scales its chunk.
//
// Squares of fp32 and bf16 values are exact in fp64 and cannot leave its range; a lane has a few fp64 sums of its own, the
// order of all additions follows from the sizes, so a norm does not depend on timing.  Maxima are those of the bit
// patterns without the sign: a NaN's pattern is above infinity's, so a NaN stays.
#include "../../include/mv.h"

#include <hip/hip_runtime.h>
#include <math.h>
#include <new>
#include <stdint.h>
#include <string.h>

namespace mvc {

#ifndef CHUNK
#define CHUNK 16384
#endif
#ifndef BATCH_MB
#define BATCH_MB 64
#endif
constexpr int kChunk = CHUNK;
constexpr int64_t kBatchBytes = (int64_t)BATCH_MB << 20;
constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBindMost = 128;      // pairs of addresses in the arguments of one launch

struct Tensor {
    const void* src;
    void*       dst;
    int64_t     numel;
    uint32_t    group;
    uint16_t    src_bf16, dst_bf16;
};
struct Chunk {
    uint32_t tensor, index;         // elements [index kChunk, (index + 1) kChunk) of the tensor
};
struct Lists {
    const Tensor*   tensors;
    const Chunk*    chunks;
    const uint32_t* group_first;    // n_groups + 1: chunks of group g are [group_first[g], group_first[g + 1])
    double*         partial;        // of each chunk
};

// Vectors at any multiple of their element's size.
typedef float    f32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint16_t u16x8 __attribute__((ext_vector_type(8), aligned(2)));

__device__ __forceinline__ float widen(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }

// To the nearest bf16, ties to even; NaN stays NaN.
__device__ __forceinline__ uint16_t narrow(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }

// Addresses that come out of memory are not known to be global memory's otherwise.
#define MV_GLOBAL __attribute__((address_space(1)))
typedef MV_GLOBAL float          gfloat;
typedef MV_GLOBAL uint16_t       gshort;
typedef const MV_GLOBAL float    cfloat;
typedef const MV_GLOBAL uint16_t cshort;

// V consecutive elements as fp32.
template <int V>
__device__ __forceinline__ void load(cfloat* p, float (&x)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        const f32x4 v = *reinterpret_cast<const MV_GLOBAL f32x4*>(p + i);
        x[i] = v.x, x[i + 1] = v.y, x[i + 2] = v.z, x[i + 3] = v.w;
    }
}
template <int V>
__device__ __forceinline__ void load(cshort* p, float (&x)[V])
{
    if constexpr (V == 8) {
        const u16x8 v = *reinterpret_cast<const MV_GLOBAL u16x8*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = widen(v[i]);
    } else {
        const u16x4 v = *reinterpret_cast<const MV_GLOBAL u16x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = widen(v[i]);
    }
}
template <int V>
__device__ __forceinline__ void store(gfloat* p, const float (&x)[V])
{
#pragma unroll
    for (int i = 0; i < V; i += 4) {
        f32x4 v = {x[i], x[i + 1], x[i + 2], x[i + 3]};
#ifdef NTS
        __builtin_nontemporal_store(v, reinterpret_cast<MV_GLOBAL f32x4*>(p + i));
#else
        *reinterpret_cast<MV_GLOBAL f32x4*>(p + i) = v;
#endif
    }
}
template <int V>
__device__ __forceinline__ void store(gshort* p, const float (&x)[V])
{
    if constexpr (V == 8) {
        u16x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = narrow(x[i]);
#ifdef NTS
        __builtin_nontemporal_store(v, reinterpret_cast<MV_GLOBAL u16x8*>(p));
#else
        *reinterpret_cast<MV_GLOBAL u16x8*>(p) = v;
#endif
    } else {
        u16x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = narrow(x[i]);
        *reinterpret_cast<MV_GLOBAL u16x4*>(p) = v;
    }
}
__device__ __forceinline__ float one(cfloat* p) { return *p; }
__device__ __forceinline__ float one(cshort* p) { return widen(*p); }
__device__ __forceinline__ void put(gfloat* p, float x) { *p = x; }
__device__ __forceinline__ void put(gshort* p, float x) { *p = narrow(x); }

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

// Elements [0, n) of a chunk: a thread takes V of them at a time, U times in flight.
template <int V, int U, int THREADS, bool MAX, typename S>
__device__ __forceinline__ void gather(S* src, int n, Share<MAX>& share)
{
    constexpr int kStep = THREADS * V;
    int at = (int)threadIdx.x * V;
    for (; at + (U - 1) * kStep + V <= n; at += U * kStep) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load<V>(src + at + u * kStep, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) share.add(i, x[u][i]);
    }
    for (; at + V <= n; at += kStep) {
        float x[V];
        load<V>(src + at, x);
#pragma unroll
        for (int i = 0; i < V; ++i) share.add(i, x[i]);
    }
    for (int i = 0; at + i < n; ++i) share.add(0, one(src + at + i));
}

template <int V, int U, int THREADS, typename S, typename D>
__device__ __forceinline__ void scale(S* src, D* dst, int n, float c)
{
    constexpr int kStep = THREADS * V;
    int at = (int)threadIdx.x * V;
    for (; at + (U - 1) * kStep + V <= n; at += U * kStep) {
        float x[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u) load<V>(src + at + u * kStep, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int i = 0; i < V; ++i) x[u][i] *= c;
            store<V>(dst + at + u * kStep, x[u]);
        }
    }
    for (; at + V <= n; at += kStep) {
        float x[V];
        load<V>(src + at, x);
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] *= c;
        store<V>(dst + at, x);
    }
    for (int i = 0; at + i < n; ++i) put(dst + at + i, one(src + at + i) * c);
}

__device__ __forceinline__ int chunk_count(const Tensor& t, Chunk c)
{
    const int64_t left = t.numel - (int64_t)c.index * kChunk;
    return left < kChunk ? (int)left : kChunk;
}

template <int THREADS, bool MAX>
__device__ __forceinline__ void gather_chunk(const Tensor& t, Chunk c, Share<MAX>& share)
{
    const int n = chunk_count(t, c);
    const int64_t first = (int64_t)c.index * kChunk;
    if (t.src_bf16) gather<8, 4, THREADS, MAX>((cshort*)t.src + first, n, share);
    else gather<4, 8, THREADS, MAX>((cfloat*)t.src + first, n, share);
}

template <int THREADS>
__device__ __forceinline__ void scale_chunk(const Tensor& t, Chunk k, float c)
{
    if (c == 1.0f && t.src == t.dst) return;
    const int n = chunk_count(t, k);
    const int64_t first = (int64_t)k.index * kChunk;
    if (t.src_bf16) {
        cshort* s = (cshort*)t.src + first;
        if (t.dst_bf16) scale<8, 4, THREADS>(s, (gshort*)t.dst + first, n, c);
        else scale<4, 8, THREADS>(s, (gfloat*)t.dst + first, n, c);
    } else {
        cfloat* s = (cfloat*)t.src + first;
        if (t.dst_bf16) scale<4, 8, THREADS>(s, (gshort*)t.dst + first, n, c);
        else scale<4, 8, THREADS>(s, (gfloat*)t.dst + first, n, c);
    }
}

// A group's value from its chunks', the same in every workgroup that asks.
template <bool MAX, int THREADS>
__device__ __forceinline__ double group_value(const Lists& l, uint32_t first, uint32_t last, double* lds)
{
    double v = 0.0;
    for (uint32_t i = first + threadIdx.x; i < last; i += THREADS) v = joined<MAX>(v, l.partial[i]);
    return of_workgroup<MAX, THREADS / 64>(v, lds);
}

struct Range {
    uint32_t first, count;          // of chunks
};

template <bool MAX>
__device__ __forceinline__ void gather_one(const Lists& l, uint32_t at, double* lds)
{
    const Chunk c = l.chunks[at];
    const Tensor t = l.tensors[c.tensor];
    Share<MAX> share;
    gather_chunk<kThreads, MAX>(t, c, share);
    const double v = of_workgroup<MAX, kWaves>(share.value(), lds);
    if (threadIdx.x == 0) l.partial[at] = v;
}

template <bool MAX>
__device__ __forceinline__ void scale_one(const Lists& l, uint32_t at, float max_norm, float* __restrict__ norms,
                                          float* __restrict__ coefs, double* lds)
{
    const Chunk c = l.chunks[at];
    const Tensor t = l.tensors[c.tensor];
    const uint32_t first = l.group_first[t.group], last = l.group_first[t.group + 1];
    const float norm = norm_of<MAX>(group_value<MAX, kThreads>(l, first, last, lds));
    const float coef = coef_of(norm, max_norm);
    if (at == first && threadIdx.x == 0) {
        norms[t.group] = norm;
        if (coefs) coefs[t.group] = coef;
    }
    scale_chunk<kThreads>(t, c, coef);
}

template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_gather(Lists l)
{
    __shared__ double lds[kWaves];
    gather_one<MAX>(l, blockIdx.x, lds);
}

// One launch scales a batch of groups and reads the next one, workgroups of both in turn.
template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_turn(Lists l, Range scaled, Range read, float max_norm, float* __restrict__ norms,
                                                         float* __restrict__ coefs)
{
    __shared__ double lds[kWaves];
    const uint32_t both = 2 * min(scaled.count, read.count), b = blockIdx.x;
    const uint32_t at = b < both ? b / 2 : b - both / 2;
    if (b < both ? (b & 1u) != 0 : scaled.count > read.count) scale_one<MAX>(l, scaled.first + at, max_norm, norms, coefs, lds);
    else gather_one<MAX>(l, read.first + at, lds);
}

// One workgroup per group.
template <bool MAX>
__global__ __launch_bounds__(kThreads) void mv_clip_norm(Lists l, float* __restrict__ norms)
{
    __shared__ double lds[kWaves];
    const uint32_t g = blockIdx.x;
    const double v = group_value<MAX, kThreads>(l, l.group_first[g], l.group_first[g + 1], lds);
    if (threadIdx.x == 0) norms[g] = norm_of<MAX>(v);
}

// Groups without chunks have no workgroup above.
__global__ __launch_bounds__(kThreads) void mv_clip_empty(Lists l, uint32_t n_groups, float max_norm,
                                                          float* __restrict__ norms, float* __restrict__ coefs)
{
    for (uint32_t g = blockIdx.x * kThreads + threadIdx.x; g < n_groups; g += gridDim.x * kThreads)
        if (l.group_first[g] == l.group_first[g + 1]) {
            norms[g] = 0.0f;
            if (coefs) coefs[g] = coef_of(0.0f, max_norm);
        }
}

struct Pairs {
    const void* src[kBindMost];
    void*       dst[kBindMost];
};
__global__ __launch_bounds__(kBindMost) void mv_clip_bind_kernel(Tensor* __restrict__ tensors, int64_t first, int32_t n, Pairs p)
{
    const int i = (int)threadIdx.x;
    if (i >= n) return;
    tensors[first + i].src = p.src[i];
    tensors[first + i].dst = p.dst[i];
}

}  // namespace mvc

struct mv_clip {
    mv_clip_config cfg;
    bool           has_dst, ended, failed, owns_ws;
    bool           any_empty, used;
    int64_t        n_tensors;
    uint32_t       n_chunks;
    char*          ws;
    mvc::Lists     lists;
    mvc::Tensor*   tensors;
    mv_clip_tensor* list;      // the caller's list as it was given
    uint32_t*      batch_end;  // batches of whole groups, their chunks' ends
    uint32_t       n_batches;
    hipStream_t    last_stream;
};

namespace {

constexpr size_t   kAlign = 256;
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
    bool     has_dst;
    size_t   off_tensors, off_chunks, off_first, off_partial, total;
};

bool measure(const mv_clip_config* c, const mv_clip_tensor* t, int64_t n, Sizes* s)
{
    if (!c || !t || c->struct_size != sizeof(mv_clip_config) || c->device < 0) return false;
    if (c->n_groups < 1 || c->n_groups > 65535 || n < 1 || n > (1 << 24)) return false;
    if (c->norm != MV_NORM_L2 && c->norm != MV_NORM_MAX) return false;
    int64_t with = 0, without = 0;
    s->chunks = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (t[i].numel < 0 || t[i].numel > ((int64_t)1 << 40) || t[i].group < 0 || t[i].group >= c->n_groups) return false;
        if ((t[i].src_dtype != MV_F32 && t[i].src_dtype != MV_BF16) || (t[i].dst_dtype != MV_F32 && t[i].dst_dtype != MV_BF16))
            return false;
        if (!addresses_valid(t[i], t[i].src, t[i].dst)) return false;
        if (t[i].numel) ++(t[i].dst ? with : without);
        s->chunks += (uint64_t)(t[i].numel + mvc::kChunk - 1) / mvc::kChunk;
    }
    if ((with && without) || s->chunks > kMostChunks) return false;
    s->has_dst = without == 0;
    s->off_tensors = 0;
    s->off_chunks = align_up((size_t)n * sizeof(mvc::Tensor));
    s->off_first = s->off_chunks + align_up((size_t)s->chunks * sizeof(mvc::Chunk));
    s->off_partial = s->off_first + align_up(((size_t)c->n_groups + 1) * sizeof(uint32_t));
    s->total = s->off_partial + align_up((size_t)s->chunks * sizeof(double) + 1);
    return true;
}

// The lists as the device holds them.
bool lay_out(const mv_clip_config* c, const mv_clip_tensor* t, int64_t n, const Sizes& s, char* host)
{
    mvc::Tensor* tensors = reinterpret_cast<mvc::Tensor*>(host + s.off_tensors);
    mvc::Chunk*  chunks = reinterpret_cast<mvc::Chunk*>(host + s.off_chunks);
    uint32_t*    first = reinterpret_cast<uint32_t*>(host + s.off_first);
    uint32_t*    at = new (std::nothrow) uint32_t[(size_t)c->n_groups];
    if (!at) return false;
    for (int64_t i = 0; i < n; ++i) {
        tensors[i] = {t[i].src, t[i].dst, t[i].numel, (uint32_t)t[i].group, (uint16_t)(t[i].src_dtype == MV_BF16),
                      (uint16_t)(t[i].dst_dtype == MV_BF16)};
        first[t[i].group + 1] += (uint32_t)((t[i].numel + mvc::kChunk - 1) / mvc::kChunk);
    }
    for (int32_t g = 0; g < c->n_groups; ++g) {
        at[g] = first[g];
        first[g + 1] += first[g];
    }
    for (int64_t i = 0; i < n; ++i) {
        const uint32_t many = (uint32_t)((t[i].numel + mvc::kChunk - 1) / mvc::kChunk);
        for (uint32_t k = 0; k < many; ++k) chunks[at[t[i].group]++] = {(uint32_t)i, k};
    }
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
    return measure(cfg, tensors, n_tensors, &s) ? s.total : 0;
}

mv_status mv_clip_begin(const mv_clip_config* cfg, const mv_clip_tensor* tensors, int64_t n_tensors, mv_clip** out)
{
    if (!out) return MV_ERR_INVALID_ARG;
    *out = nullptr;
    Sizes s;
    if (!measure(cfg, tensors, n_tensors, &s)) return MV_ERR_INVALID_ARG;
    if (cfg->workspace &&
        (cfg->workspace_bytes < s.total || (reinterpret_cast<uintptr_t>(cfg->workspace) & (kAlign - 1)) != 0))
        return MV_ERR_INVALID_ARG;
    mv_clip* c = new (std::nothrow) mv_clip;
    char* host = new (std::nothrow) char[s.off_partial];
    mv_clip_tensor* list = new (std::nothrow) mv_clip_tensor[(size_t)n_tensors];
    uint32_t* batch_end = new (std::nothrow) uint32_t[(size_t)cfg->n_groups];
    int64_t* group_bytes = new (std::nothrow) int64_t[(size_t)cfg->n_groups];
    if (host) memset(host, 0, s.off_partial);
    if (!c || !host || !list || !batch_end || !group_bytes || !lay_out(cfg, tensors, n_tensors, s, host)) {
        delete c;
        delete[] host;
        delete[] list;
        delete[] batch_end;
        delete[] group_bytes;
        return MV_ERR_ALLOC;
    }
    memset(static_cast<void*>(c), 0, sizeof *c);
    c->list = list;
    c->batch_end = batch_end;
    memcpy(list, tensors, (size_t)n_tensors * sizeof *list);
    c->cfg = *cfg;
    c->has_dst = s.has_dst;
    c->n_tensors = n_tensors;
    c->n_chunks = (uint32_t)s.chunks;
    const uint32_t* first = reinterpret_cast<const uint32_t*>(host + s.off_first);
    for (int32_t g = 0; g < cfg->n_groups; ++g)
        if (first[g] == first[g + 1]) c->any_empty = true;
    memset(group_bytes, 0, (size_t)cfg->n_groups * sizeof *group_bytes);
    for (int64_t i = 0; i < n_tensors; ++i) group_bytes[tensors[i].group] += tensors[i].numel * (int64_t)elem(tensors[i].src_dtype);
    int64_t bytes = 0;
    for (int32_t g = 0; g < cfg->n_groups; ++g) {
        if (bytes && bytes + group_bytes[g] > mvc::kBatchBytes) {
            if (first[g] > (c->n_batches ? batch_end[c->n_batches - 1] : 0)) batch_end[c->n_batches++] = first[g];
            bytes = 0;
        }
        bytes += group_bytes[g];
    }
    if (c->n_chunks > (c->n_batches ? batch_end[c->n_batches - 1] : 0)) batch_end[c->n_batches++] = c->n_chunks;
    delete[] group_bytes;

    DeviceGuard guard(cfg->device);
    mv_status st = guard.ok ? MV_OK : MV_ERR_DEVICE;
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
    if (st == MV_OK && (hipMemcpy(c->ws, host, s.off_partial, hipMemcpyHostToDevice) != hipSuccess)) {
        (void)hipGetLastError();
        st = MV_ERR_DEVICE;
    }
    delete[] host;
    if (st != MV_OK) {
        if (c->owns_ws) (void)hipFree(c->ws);
        delete[] list;
        delete[] batch_end;
        delete c;
        return st;
    }
    c->tensors = reinterpret_cast<mvc::Tensor*>(c->ws + s.off_tensors);
    c->lists.tensors = c->tensors;
    c->lists.chunks = reinterpret_cast<const mvc::Chunk*>(c->ws + s.off_chunks);
    c->lists.group_first = reinterpret_cast<const uint32_t*>(c->ws + s.off_first);
    c->lists.partial = reinterpret_cast<double*>(c->ws + s.off_partial);
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
        hipLaunchKernelGGL(mvc::mv_clip_bind_kernel, dim3(1), dim3(mvc::kBindMost), 0, st, c->tensors, i, n, p);
    }
    return done(c);
}

mv_status mv_clip_norms(mv_clip* c, float* norms, void* stream)
{
    if (!c || !norms || (reinterpret_cast<uintptr_t>(norms) & 3)) return MV_ERR_INVALID_ARG;
    if (const mv_status st = usable(c); st != MV_OK) return st;
    DeviceGuard guard(c->cfg.device);
    if (!guard.ok) return MV_ERR_DEVICE;
    hipStream_t st = static_cast<hipStream_t>(stream);
    c->last_stream = st;
    c->used = true;
    const bool max = c->cfg.norm == MV_NORM_MAX;
    if (c->n_chunks) {
        if (max) hipLaunchKernelGGL(mvc::mv_clip_gather<true>, dim3(c->n_chunks), dim3(mvc::kThreads), 0, st, c->lists);
        else hipLaunchKernelGGL(mvc::mv_clip_gather<false>, dim3(c->n_chunks), dim3(mvc::kThreads), 0, st, c->lists);
    }
    const dim3 grid((uint32_t)c->cfg.n_groups);
    if (max) hipLaunchKernelGGL(mvc::mv_clip_norm<true>, grid, dim3(mvc::kThreads), 0, st, c->lists, norms);
    else hipLaunchKernelGGL(mvc::mv_clip_norm<false>, grid, dim3(mvc::kThreads), 0, st, c->lists, norms);
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
    const dim3 threads(mvc::kThreads);
    mvc::Range scaled = {0, 0};
    for (uint32_t b = 0; c->n_chunks && b <= c->n_batches; ++b) {
        const uint32_t end = b < c->n_batches ? c->batch_end[b] : c->n_chunks;
        const mvc::Range read = {scaled.first + scaled.count, end - (scaled.first + scaled.count)};
        const dim3 grid(scaled.count + read.count);
        if (c->cfg.norm == MV_NORM_MAX)
            hipLaunchKernelGGL(mvc::mv_clip_turn<true>, grid, threads, 0, st, c->lists, scaled, read, max_norm, norms, coefs);
        else
            hipLaunchKernelGGL(mvc::mv_clip_turn<false>, grid, threads, 0, st, c->lists, scaled, read, max_norm, norms, coefs);
        scaled = read;
    }
    if (c->any_empty)
        hipLaunchKernelGGL(mvc::mv_clip_empty, dim3(1), threads, 0, st, c->lists, (uint32_t)c->cfg.n_groups, max_norm,
                           norms, coefs);
    return done(c);
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
    delete[] c->batch_end;
    delete c;
}

}  // extern "C"
