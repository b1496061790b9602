// Distillation from a teacher's top logits (mv_distill_loss, mv_distill_grad of include/mv.h).
//
//   q = softmax(z / T),  s = softmax(z),  p = softmax(t / T) over a row's list
//   loss  = soft T^2 sum p (log p - log q)  +  hard (-log s[label])
//   dz[v] = g ( soft T (P q[v] - p listed for v)  +  hard (s[v] - [v = label]) )
//
// Only the logits are long, so memory bounds it: z is read once and dz written once where a row fits its workgroup's
// registers, and then a row is: its maximum, its sums of exponentials, its list, and dz from the registers.  Longer rows are
// cut into ranges, a workgroup each: their maxima and sums, which a second kernel joins and makes the loss of, and dz in a third.
//
// dz has the same formula everywhere but at the listed coordinates and the label.  Those are written behind the rest of
// their row, or range, by the workgroup that wrote it: one thread for each entry, which adds up what the list has for its
// coordinate, in the list's order, where it is the first to name it.
#include "mv_rows.hpp"

namespace mvr {

constexpr int64_t kMostTop = 4096;
constexpr float   kLog2e = 1.44269504088896340736f;

struct Distill {
    const void*    z;
    int64_t        ld_z, rows, n;
    const int32_t* idx;
    int64_t        ld_idx;
    Any            t;
    int64_t        ld_t;
    uint32_t       top;                 // 0: no first term
    const int32_t* labels;              // NULL: no second term
    float          inv_t;               // 1 / T
    float          soft_loss, soft_grad, hard;      // soft T^2, soft T
    float *        loss, *stats;
    const float *  grad, *had;          // had: the stats of the call for the loss
    AnyOut         dz;
    int64_t        ld_dz;
    float*         parts;               // of ranges: largest and two sums each
    uint32_t       ranges;              // of a row
    int64_t        range;               // their length
};

__device__ __forceinline__ float power(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's list in LDS: coordinates, p, and the logits there; and what the row's terms come to.
struct List {
    int32_t* idx;
    float *  p, *z;
};
struct Terms {
    float soft, hard;                   // weights of q and s in dz: 0 where the row has no such term
    float largest, inv_a, inv_b;        // 1 / sum of exp((z - largest) / T) and of exp(z - largest)
    float g;
    int32_t label;                      // -1: none
};

__host__ __device__ constexpr size_t list_bytes(uint32_t top) { return ((size_t)top + 3) / 4 * 4 * 12; }
__device__ __forceinline__ List list_at(void* lds, uint32_t top)
{
    const uint32_t room = (top + 3) / 4 * 4;
    int32_t* idx = static_cast<int32_t*>(lds);
    return {idx, reinterpret_cast<float*>(idx + room), reinterpret_cast<float*>(idx + 2 * room)};
}

// Fetches a row's list, and the logits it names where `logits` is a row.  Returns, in all threads, the teacher's largest logit.
template <int LANES, typename T>
__device__ __forceinline__ float fetch_list(const Distill& d, const List& l, int64_t row, bool live_row, const T* logits,
                                            Across<LANES>& across)
{
    const uint32_t t = threadIdx.x % LANES, room = (d.top + 3) / 4 * 4;
    float most = -kInf;
    for (uint32_t j = t; j < room; j += LANES) {
        int32_t at = -1;
        float   v = -kInf, z = 0.0f;
        if (live_row && j < d.top) {
            at = d.idx[row * d.ld_idx + j];
            if (at < 0 || at >= d.n) at = -1;
            if (at >= 0) {
                v = d.t.at(row * d.ld_t + j);
                if (logits) z = sizeof(T) == 2 ? mvx::widen(reinterpret_cast<const uint16_t*>(logits)[at])
                                               : reinterpret_cast<const float*>(logits)[at];
            }
        }
        l.idx[j] = at, l.p[j] = v, l.z[j] = z;
        most = fmaxf(most, v);
    }
    return across.max(most);
}
// The sum of exp((t - most) / T): its log, and what the p made of it come to: 0 where there are none, else 1, or NaN.
template <int LANES>
__device__ __forceinline__ float total_p(const Distill& d, const List& l, float most, float& log_sum, Across<LANES>& across)
{
    const uint32_t t = threadIdx.x % LANES;
    float sum = 0.0f;
    for (uint32_t j = t; j < d.top; j += LANES) {
        const float v = l.p[j];
        if (v != -kInf) sum += expf((v - most) * d.inv_t);               // NaN among them, or +infinity: NaN
    }
    sum = across.sum(sum);
    log_sum = logf(sum);
    return sum == 0.0f ? 0.0f : sum * 0.0f + 1.0f;
}

// sum p (log p - log q) over the list; p replaces the teacher's logits in LDS.
template <int LANES>
__device__ __forceinline__ float soft_loss(const Distill& d, const List& l, float most, float log_sum, float largest, float log_a,
                                           Across<LANES>& across)
{
    const uint32_t t = threadIdx.x % LANES;
    float sum = 0.0f;
    for (uint32_t j = t; j < d.top; j += LANES) {
        const float v = l.p[j];
        float p = 0.0f;
        if (v != -kInf) {
            const float log_p = (v - most) * d.inv_t - log_sum;
            p = expf(log_p);
            if (p != 0.0f) sum += p * (log_p - ((l.z[j] - largest) * d.inv_t - log_a));
        }
        l.p[j] = p;
    }
    return across.sum(sum);
}

// dz where the list or the label names a coordinate of [first, last).
template <int LANES>
__device__ __forceinline__ void patch(const Distill& d, const List& l, const Terms& w, int64_t row, int64_t first, int64_t last, float label_z)
{
    typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
    const uint32_t t = threadIdx.x % LANES, room = w.soft != 0.0f ? (d.top + 3) / 4 * 4 : 0u;
    for (uint32_t j = t; j < room + 1; j += LANES) {
        const int32_t at = j < room ? l.idx[j] : w.label;                // behind the list: the label
        if (at < first || at >= last) continue;                          // none is -1
        float p = 0.0f;
        bool  named = false;                                             // by an entry before
        for (uint32_t i = 0; i < room; i += 4) {
            const i32x4 other = *reinterpret_cast<const i32x4*>(l.idx + i);
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
                if (other[e] == at) {
                    named |= i + e < j;
                    p += l.p[i + e];
                }
        }
        if (named) continue;
        const float z = (j < room ? l.z[j] : label_z) - w.largest;
        float v = 0.0f;
        if (w.soft != 0.0f) v = w.soft * (power(z * d.inv_t * kLog2e) * w.inv_a - p);
        if (w.hard != 0.0f) v += w.hard * (power(z * kLog2e) * w.inv_b - (at == w.label ? 1.0f : 0.0f));
        d.dz.put(row * d.ld_dz + at, w.g * v);
    }
}

// dz of a chunk before its patches.
template <int V>
__device__ __forceinline__ void plain_grad(const Terms& w, float scale, bool any, const float (&z)[V], float (&to)[V])
{
    const float a = w.g * w.soft * w.inv_a, b = w.g * w.hard * w.inv_b;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float x = z[i] - w.largest;
        float v = 0.0f;
        if (w.soft != 0.0f) v = a * power(x * scale);
        if (w.hard != 0.0f) v += b * power(x * kLog2e);
        to[i] = any ? v : 0.0f;
    }
}

// A row in registers: LANES threads, C chunks each.
template <typename T, int LANES, int C>
__global__ __launch_bounds__(kThreadsOf<LANES>) void mv_distill_kernel(Distill d)
{
    constexpr int V = kChunk<T>, kRows = kThreadsOf<LANES> / LANES;
    __shared__ float sums[kRows][2][2][LANES / 64];
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t t = threadIdx.x % LANES, mine = threadIdx.x / LANES;
    Across<LANES> across(sums[mine]);
    const List list = list_at(lds + mine * list_bytes(d.top), d.top);
    const float scale = d.inv_t * kLog2e;
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < d.rows; first += (int64_t)gridDim.x * kRows) {
        const int64_t row = first + mine;
        const bool live_row = row < d.rows;
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        Chunk<T> held[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (int64_t)(c * LANES + t) * V;
            held[c].load(z + col, live_row ? d.n - col : 0);
        }
        const float most = d.top ? fetch_list<LANES>(d, list, row, live_row, z, across) : -kInf;
        int32_t label = live_row && d.labels ? d.labels[row] : -1;
        if (label >= d.n) label = -1;
        const float label_z = label >= 0 ? Any{d.z, sizeof(T) == 2}.at(row * d.ld_z + label) : 0.0f;
        float largest = -kInf;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t live = live_row ? d.n - (int64_t)(c * LANES + t) * V : 0;
#pragma unroll
            for (int i = 0; i < V; ++i) largest = fmaxf(largest, i < live ? held[c].at(i) : -kInf);
        }
        largest = across.max(largest);
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t live = live_row ? d.n - (int64_t)(c * LANES + t) * V : 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x = i < live ? held[c].at(i) - largest : -kInf;
                if (d.top) a += power(x * scale);
                if (d.labels) b += power(x * kLog2e);
            }
        }
        __builtin_amdgcn_s_waitcnt(kNoLoads);                       // dz may be z: all that is read of the row is here
        across.sum2(a, b);
        if (live_row && t == 0 && d.stats) {
            d.stats[3 * row] = largest;
            d.stats[3 * row + 1] = a;
            d.stats[3 * row + 2] = b;
        }
        float log_sum = 0.0f, loss = 0.0f;
        const float total = d.top ? total_p<LANES>(d, list, most, log_sum, across) : 0.0f;
        const bool soft = total != 0.0f;
        if (d.top) {
            const float sum = soft_loss<LANES>(d, list, most, log_sum, largest, logf(a), across);
            if (soft) loss = d.soft_loss * sum;
        }
        if (label >= 0) loss += d.hard * (logf(b) - (label_z - largest));
        if (live_row && t == 0 && d.loss) d.loss[row] = loss;
        if (d.dz.p) {                                                    // uniform
            const Terms w = {total * d.soft_grad, label >= 0 ? d.hard : 0.0f, largest, 1.0f / a, 1.0f / b,
                             d.grad && live_row ? d.grad[row] : 1.0f, label};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int64_t col = (int64_t)(c * LANES + t) * V;
                float x[V], y[V];
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = held[c].at(i);
                plain_grad(w, scale, soft || label >= 0, x, y);
                if (live_row) d.dz.store(row * d.ld_dz + col, d.n - col, y);
            }
            __builtin_amdgcn_s_waitcnt(0);                               // all of a row is written before its patches
            __syncthreads();
            if (live_row) patch<LANES>(d, list, w, row, 0, d.n, label_z);
        }
        __syncthreads();                                                 // the list is read before the next row's
    }
}

// ---- long rows, in ranges ----------------------------------------------------------------------------------------------

constexpr int kRangeThreads = 512;

// Largest and sums of a range: each thread's as it goes, joined at the end.
template <typename T>
__global__ __launch_bounds__(kRangeThreads) void mv_distill_range_kernel(Distill d)
{
    constexpr int V = kChunk<T>;
    __shared__ float sums[2][2][kRangeThreads / 64];
    Across<kRangeThreads> across(sums);
    const float scale = d.inv_t * kLog2e;
    const int64_t all = d.rows * d.ranges;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
        const int64_t row = at / d.ranges, first = at % d.ranges * d.range, last = first + d.range < d.n ? first + d.range : d.n;
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        float largest = -kInf, a = 0.0f, b = 0.0f;
        for (int64_t col = first + (int64_t)threadIdx.x * V; col < last; col += kRangeThreads * V) {
            Chunk<T> c;
            c.load(z + col, last - col);
            const int64_t live = last - col;
            float x[V], top = largest;
#pragma unroll
            for (int i = 0; i < V; ++i) top = fmaxf(top, x[i] = i < live ? c.at(i) : -kInf);
            const float base = top == -kInf ? 0.0f : top, old = largest - base;          // -infinity: nothing yet
            if (top > largest) a *= power(old * scale), b *= power(old * kLog2e);
            largest = top;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (d.top) a += power((x[i] - base) * scale);
                if (d.labels) b += power((x[i] - base) * kLog2e);
            }
        }
        const float top = across.max(largest), old = largest - (top == -kInf ? 0.0f : top);
        a *= power(old * scale), b *= power(old * kLog2e);
        across.sum2(a, b);
        if (threadIdx.x == 0) {
            float* to = d.parts + 4 * at;
            to[0] = top, to[1] = a, to[2] = b;
        }
        __syncthreads();
    }
}

// A row's ranges joined, and its loss.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ __launch_bounds__(kJoinThreads) void mv_distill_join_kernel(Distill d)
{
    __shared__ float sums[2][2][kJoinThreads / 64];
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Across<kJoinThreads> across(sums);
    const List list = list_at(lds, d.top);
    const float scale = d.inv_t * kLog2e;
    for (int64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const float* part = d.parts + 4 * row * d.ranges;
        float largest = -kInf, a = 0.0f, b = 0.0f;
        for (uint32_t r = threadIdx.x; r < d.ranges; r += kJoinThreads) largest = fmaxf(largest, part[4 * r]);
        largest = across.max(largest);
        for (uint32_t r = threadIdx.x; r < d.ranges; r += kJoinThreads) {
            const float old = part[4 * r] - largest;
            a += part[4 * r + 1] * power(old * scale);
            b += part[4 * r + 2] * power(old * kLog2e);
        }
        across.sum2(a, b);
        if (threadIdx.x == 0) {
            float* to = d.stats + 3 * row;
            to[0] = largest, to[1] = a, to[2] = b;
        }
        if (!d.loss) continue;                                           // uniform
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        float log_sum = 0.0f, loss = 0.0f;
        if (d.top) {
            const float most = fetch_list<kJoinThreads>(d, list, row, true, z, across);
            const bool soft = total_p<kJoinThreads>(d, list, most, log_sum, across) != 0.0f;
            const float sum = soft_loss<kJoinThreads>(d, list, most, log_sum, largest, logf(a), across);
            if (soft) loss = d.soft_loss * sum;
        }
        const int32_t label = d.labels ? d.labels[row] : -1;
        if (label >= 0 && label < d.n) loss += d.hard * (logf(b) - (Any{d.z, sizeof(T) == 2}.at(row * d.ld_z + label) - largest));
        if (threadIdx.x == 0) d.loss[row] = loss;
        __syncthreads();
    }
}

// dz of a range, from the row's stats.
template <typename T>
__global__ __launch_bounds__(kRangeThreads) void mv_distill_grad_kernel(Distill d)
{
    constexpr int V = kChunk<T>;
    __shared__ float sums[2][2][kRangeThreads / 64];
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Across<kRangeThreads> across(sums);
    const List list = list_at(lds, d.top);
    const float scale = d.inv_t * kLog2e;
    const int64_t all = d.rows * d.ranges;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
        const int64_t row = at / d.ranges, first = at % d.ranges * d.range, last = first + d.range < d.n ? first + d.range : d.n;
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        float total = 0.0f;
        if (d.top) {
            // logits are asked for only where this range names them: others may have been written over
            const uint32_t room = (d.top + 3) / 4 * 4;
            const float most = fetch_list<kRangeThreads, T>(d, list, row, true, nullptr, across);
            for (uint32_t j = threadIdx.x; j < room; j += kRangeThreads)
                if (list.idx[j] >= first && list.idx[j] < last) list.z[j] = Any{d.z, sizeof(T) == 2}.at(row * d.ld_z + list.idx[j]);
            float log_sum;
            total = total_p<kRangeThreads>(d, list, most, log_sum, across);
            for (uint32_t j = threadIdx.x; j < d.top; j += kRangeThreads)
                list.p[j] = list.p[j] == -kInf ? 0.0f : expf((list.p[j] - most) * d.inv_t - log_sum);
        }
        int32_t label = d.labels ? d.labels[row] : -1;
        if (label >= d.n) label = -1;
        const float label_z = label >= first && label < last ? Any{d.z, sizeof(T) == 2}.at(row * d.ld_z + label) : 0.0f;
        const float* had = d.had + 3 * row;
        const Terms w = {total * d.soft_grad, label >= 0 ? d.hard : 0.0f, had[0], 1.0f / had[1], 1.0f / had[2],
                         d.grad ? d.grad[row] : 1.0f, label};
        __builtin_amdgcn_s_waitcnt(kNoLoads);                            // dz may be z: the list's and the label's are here
        __syncthreads();
        for (int64_t col = first + (int64_t)threadIdx.x * V; col < last; col += kRangeThreads * V) {
            Chunk<T> c;
            c.load(z + col, last - col);
            float x[V], y[V];
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = c.at(i);
            plain_grad(w, scale, total != 0.0f || label >= 0, x, y);
            d.dz.store(row * d.ld_dz + col, last - col, y);
        }
        __builtin_amdgcn_s_waitcnt(0);                                   // all of the range is written before its patches
        __syncthreads();
        patch<kRangeThreads>(d, list, w, row, first, last, label_z);
        __syncthreads();
    }
}

// How a row is held: LANES threads with C chunks each, or 0: not at all.
struct Lanes {
    int lanes, chunks;
};
static Lanes lanes_of(int64_t n, int32_t dtype, int64_t top)
{
    const int64_t wide = dtype == MV_BF16 ? 8 : 4, chunks = (n + wide - 1) / wide;
    for (int i = top > 1024 ? 1 : 0; i < 3; ++i)                         // four rows' lists in one workgroup's LDS: 48 KB
        for (int c = i ? 4 : 1; c <= (i == 2 ? 16 : i ? 8 : 4); c *= i ? 2 : 4)
            if (chunks <= ((int64_t)64 << (2 * i)) * c) return {64 << (2 * i), c};
    return {0, 0};
}

// Ranges of long rows: of 16,384 values or more, as few as give the card a thousand workgroups.
constexpr int64_t kRangeLeast = 16384, kRangeGroups = 1024;
struct Ranges {
    uint32_t count;
    int64_t  length;
};
static Ranges ranges_of(int64_t rows, int64_t n)
{
    int64_t count = (kRangeGroups + rows - 1) / rows, most = (n + kRangeLeast - 1) / kRangeLeast;
    if (count > most) count = most;
    const int64_t length = ((n + count - 1) / count + 7) / 8 * 8;        // ranges begin where a chunk does
    return {(uint32_t)((n + length - 1) / length), length};
}
inline uint32_t grid_of(int64_t groups, int64_t most) { return (uint32_t)(groups < most ? groups : most); }

template <typename T, int LANES, int C>
static void held(const Distill& d, hipStream_t st)
{
    constexpr int kRows = kThreadsOf<LANES> / LANES;
    hipLaunchKernelGGL((mv_distill_kernel<T, LANES, C>), dim3(grid_of((d.rows + kRows - 1) / kRows, 1 << 20)), dim3(kThreadsOf<LANES>),
                       kRows * list_bytes(d.top), st, d);
}
template <typename T>
static void grad(Distill d, hipStream_t st)
{
    const Ranges r = ranges_of(d.rows, d.n);
    d.ranges = r.count, d.range = r.length;
    hipLaunchKernelGGL(mv_distill_grad_kernel<T>, dim3(grid_of(d.rows * r.count, 1 << 20)), dim3(kRangeThreads), list_bytes(d.top), st, d);
}
template <typename T>
static void loss(Distill d, const Lanes& l, hipStream_t st)
{
    if (l.lanes == 64) return l.chunks == 1 ? held<T, 64, 1>(d, st) : held<T, 64, 4>(d, st);
    if (l.lanes == 256) return l.chunks == 4 ? held<T, 256, 4>(d, st) : held<T, 256, 8>(d, st);
    if (l.lanes == 1024) return l.chunks == 4 ? held<T, 1024, 4>(d, st) : l.chunks == 8 ? held<T, 1024, 8>(d, st) : held<T, 1024, 16>(d, st);
    const Ranges r = ranges_of(d.rows, d.n);
    d.ranges = r.count, d.range = r.length;
    hipLaunchKernelGGL(mv_distill_range_kernel<T>, dim3(grid_of(d.rows * r.count, 1 << 20)), dim3(kRangeThreads), 0, st, d);
    hipLaunchKernelGGL(mv_distill_join_kernel<T>, dim3(grid_of(d.rows, 1 << 20)), dim3(kJoinThreads), list_bytes(d.top), st, d);
    if (d.dz.p) {
        d.had = d.stats;
        grad<T>(d, st);
    }
}

// What long rows need: the ranges' parts and, where the caller keeps none, the rows' stats.
inline size_t parts_bytes(int64_t rows, int64_t n) { return (size_t)rows * ranges_of(rows, n).count * 16; }
inline size_t stats_bytes(int64_t rows) { return ((size_t)rows * 12 + 15) / 16 * 16; }

static bool fill(Distill& d, const void* logits, int32_t dtype, int64_t ld_z, int64_t rows, int64_t n, const int32_t* idx, int64_t ld_idx,
                 const void* t, int32_t t_dtype, int64_t ld_t, int64_t top, const int32_t* labels, float temperature, float soft, float hard,
                 const float* g, void* dz, int32_t dz_dtype, int64_t ld_dz)
{
    auto aligned = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; };
    if (!size_valid(rows) || !size_valid(n) || !values_valid(logits, dtype, ld_z, n) || top < 0 || top > kMostTop ||
        !(temperature >= 0x1p-60f && temperature <= 0x1p60f) || !(soft > -kInf && soft < kInf) || !(hard > -kInf && hard < kInf) ||
        !aligned(labels) || !aligned(g) || (dz && !values_valid(dz, dz_dtype, ld_dz, n)) ||
        (dz == logits && (dz_dtype != dtype || ld_dz != ld_z)))
        return false;
    const bool listed = top > 0 && soft != 0.0f;
    if (listed && (!idx || !aligned(idx) || ld_idx < top || !values_valid(t, t_dtype, ld_t, top))) return false;
    d.z = logits, d.ld_z = ld_z, d.rows = rows, d.n = n;
    d.idx = idx, d.ld_idx = ld_idx, d.t = {t, t_dtype == MV_BF16}, d.ld_t = ld_t, d.top = listed ? (uint32_t)top : 0u;
    d.labels = hard != 0.0f ? labels : nullptr;
    d.inv_t = 1.0f / temperature;
    d.soft_grad = soft * temperature, d.soft_loss = soft * temperature * temperature, d.hard = hard;
    d.grad = g, d.dz = {dz, dz_dtype == MV_BF16}, d.ld_dz = ld_dz;
    return true;
}

}  // namespace mvr

extern "C" {

size_t mv_distill_scratch_bytes(int64_t rows, int64_t n)
{
    using namespace mvr;
    // fp32 rows are the first to be too long
    return size_valid(rows) && size_valid(n) && !lanes_of(n, MV_F32, 0).lanes ? parts_bytes(rows, n) + stats_bytes(rows) : 0;
}

mv_status mv_distill_loss(const void* logits, int32_t dtype, int64_t ld_z, int64_t rows, int64_t n, const int32_t* idx, int64_t ld_idx,
                          const void* t, int32_t t_dtype, int64_t ld_t, int64_t top, const int32_t* labels, float temperature, float soft,
                          float hard, float* loss, float* stats, const float* grad, void* dz, int32_t dz_dtype, int64_t ld_dz,
                          void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvr;
    Distill d = {};
    if ((!loss && !dz) || (reinterpret_cast<uintptr_t>(loss) & 3) || (reinterpret_cast<uintptr_t>(stats) & 3) ||
        !fill(d, logits, dtype, ld_z, rows, n, idx, ld_idx, t, t_dtype, ld_t, top, labels, temperature, soft, hard, grad, dz, dz_dtype, ld_dz))
        return MV_ERR_INVALID_ARG;
    const size_t need = mv_distill_scratch_bytes(rows, n);
    if (need && (!scratch || scratch_bytes < need || (reinterpret_cast<uintptr_t>(scratch) & 15))) return MV_ERR_INVALID_ARG;
    d.loss = loss, d.stats = stats;
    const Lanes l = lanes_of(n, dtype, d.top);
    if (!l.lanes) {
        d.parts = static_cast<float*>(scratch);
        if (!stats) d.stats = reinterpret_cast<float*>(static_cast<char*>(scratch) + parts_bytes(rows, n));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == MV_BF16) mvr::loss<uint16_t>(d, l, st);
    else mvr::loss<float>(d, l, st);
    return launched();
}

mv_status mv_distill_grad(const void* logits, int32_t dtype, int64_t ld_z, int64_t rows, int64_t n, const int32_t* idx, int64_t ld_idx,
                          const void* t, int32_t t_dtype, int64_t ld_t, int64_t top, const int32_t* labels, float temperature, float soft,
                          float hard, const float* stats, const float* grad, void* dz, int32_t dz_dtype, int64_t ld_dz, void* stream)
{
    using namespace mvr;
    Distill d = {};
    if (!dz || !stats || (reinterpret_cast<uintptr_t>(stats) & 3) ||
        !fill(d, logits, dtype, ld_z, rows, n, idx, ld_idx, t, t_dtype, ld_t, top, labels, temperature, soft, hard, grad, dz, dz_dtype, ld_dz))
        return MV_ERR_INVALID_ARG;
    d.had = stats;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == MV_BF16) mvr::grad<uint16_t>(d, st);
    else mvr::grad<float>(d, st);
    return launched();
}

}  // extern "C"
