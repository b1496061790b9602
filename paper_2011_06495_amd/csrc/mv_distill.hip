// Distillation from a teacher's top logits (mv_distill_loss, mv_distill_grad of include/mv.h).
//
//   q = softmax(z / T),  s = softmax(z),  p = softmax(t / T) over a row's list
//   loss  = soft T^2 sum p (log p - log q)  +  hard (-log s[label])
//   dz[v] = g ( soft T (P q[v] - p listed for v)  +  hard (s[v] - [v = label]) )
//
// Only the logits are long, so memory bounds it, and next to it the exponentials: two for each logit, or four where both
// terms are wanted and T is not 1 (of T = 2 the second one is the first one's square).  Where dz is wanted with the loss and a
// row fits a workgroup's registers, z is read once: its maximum, its sums, and dz from the registers, which take the next row's
// logits as they become free.  Otherwise rows, or ranges of rows where there are few, stream by for their maxima and sums,
// each thread's joined at the end, and once more for dz.  Loss and dz of 4096 x 131,072 bf16, 64 listed, both terms: T = 2 430 us,
// 5.0 TB/s, T = 3 450, T = 1 418, 5.1; 2000 x 50,001 fp32 170, 4.7, the loss alone 70, 5.7; dz alone 3000 x 32,768 bf16 77, 5.1.
//
// A row's list is the first wavefront's, while the others have the logits.  dz has the same formula everywhere but at the
// listed coordinates and the label.  Those are written behind the rest by the wavefront that wrote them before, a lane for each
// entry.  Entries that name one coordinate add up, in the list's order, for the first of them; they find each other by slots
// that their coordinates have in LDS (all compared with all took 2000 x 60,000 with 256 listed 288 us, now 129).
#include "mv_rows.hpp"

#include <type_traits>

namespace mvr {

constexpr int64_t kMostTop = 4096;
constexpr float   kLog2e = 1.44269504088896340736f;

// Which exponentials the terms need: one, two, or one and its square.
enum { kOne, kTwo, kSquare };

struct Distill {
    const void*    z;
    int64_t        ld_z, rows, n;
    const int32_t* idx;
    int64_t        ld_idx;
    Any            t;
    int64_t        ld_t;
    uint32_t       top;                 // 0: no first term
    const int32_t* labels;              // NULL: no second term
    float          inv_t, scale;        // 1 / T; what an exponent of the first kind is multiplied with, for a power of 2
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
// A lane's number that nothing is made of beforehand, where registers are short.
__device__ __forceinline__ uint32_t fresh(uint32_t lane)
{
    asm volatile("" : "+v"(lane));
    return lane;
}
__device__ __forceinline__ float larger(float x, float y) { return __builtin_amdgcn_fmed3f(x, y, kInf); }    // one instruction

// The largest of a lane's logits.  Pairs of bf16 as they are: as whole numbers non-negative ones have their order, and are
// above negative ones, which have the opposite order.
template <typename T>
struct Largest;
template <>
struct Largest<float> {
    float most = -kInf;
    __device__ __forceinline__ void look(const Chunk<float>& c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) most = larger(c.x[i], most);
    }
    __device__ __forceinline__ float value() const { return most; }
};
template <>
struct Largest<uint16_t> {
    typedef int16_t  i16x2 __attribute__((ext_vector_type(2)));
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    i16x2 most = {-32768, -32768};
    u16x2 least = {0xFF80u, 0xFF80u};   // -infinity
    __device__ __forceinline__ void look(const Chunk<uint16_t>& c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            most = __builtin_elementwise_max(most, __builtin_bit_cast(i16x2, c.x[i]));
            least = __builtin_elementwise_min(least, __builtin_bit_cast(u16x2, c.x[i]));
        }
    }
    __device__ __forceinline__ float value() const
    {
        const int16_t  m = most.x > most.y ? most.x : most.y;
        const uint16_t l = least.x < least.y ? least.x : least.y;
        return mvx::widen(m >= 0 ? (uint16_t)m : l);
    }
};

// A logit's exponentials.
template <int TERMS>
struct Pair {
    float a, b;
    __device__ __forceinline__ Pair(float x, float scale)
    {
        a = power(x * scale);
        b = TERMS == kTwo ? power(x * kLog2e) : TERMS == kSquare ? a * a : 0.0f;
    }
};
template <typename T, int TERMS>
__device__ __forceinline__ void add_up(const Chunk<T>& c, float largest, float scale, float& a, float& b)
{
#pragma unroll
    for (int i = 0; i < kChunk<T>; ++i) {
        const Pair<TERMS> e(c.at(i) - largest, scale);
        a += e.a;
        if (TERMS != kOne) b += e.b;
    }
}

// ---- the list ------------------------------------------------------------------------------------------------------

// A row's list in LDS: coordinates, p (its sign set where another entry may name the same coordinate), and the logits there;
// and a slot for each entry, where entries of one coordinate meet.
struct List {
    int32_t*  idx;
    float *   p, *z;
    uint16_t* slots;
    uint32_t  many;                     // slots
};
__host__ __device__ constexpr uint32_t room_of(uint32_t top) { return (top + 3) / 4 * 4; }
__host__ __device__ constexpr uint32_t slots_of(uint32_t top) { return room_of(top) * 16 < 8192 ? room_of(top) * 16 : 8192; }
__host__ __device__ constexpr size_t   list_bytes(uint32_t top) { return (size_t)room_of(top) * 12 + slots_of(top) * 2; }
__device__ __forceinline__ List list_at(void* lds, uint32_t top)
{
    const uint32_t each = room_of(top);
    int32_t* idx = static_cast<int32_t*>(lds);
    return {idx, reinterpret_cast<float*>(idx + each), reinterpret_cast<float*>(idx + 2 * each), reinterpret_cast<uint16_t*>(idx + 3 * each),
            slots_of(top)};
}
__device__ __forceinline__ uint32_t slot_of(const List& l, int32_t at) { return __umulhi((uint32_t)at * 0x9E3779B1u, l.many); }
// The slot may hold what another lane has put there: LDS is in order within a wavefront, and the compiler does not know the place.
__device__ __forceinline__ uint16_t& slot_again(const List& l, int32_t at) { return l.slots[fresh(slot_of(l, at))]; }

// An entry of the list on its way, or the label: asked for, then taken as it has come, then its logit asked for.  What is loaded
// stays as it is until then, or it would be waited for at once.
struct Entry {
    int32_t  at;                        // -1: none
    uint32_t raw, raw16;                // the teacher's logit, in one of them
    float    t;
    uint32_t z;                         // the row's, as it is
    __device__ __forceinline__ void name(const Distill& d, int64_t row, uint32_t j)
    {
        at = -1, raw = raw16 = 0;
        if (j < d.top) {
            at = d.idx[row * d.ld_idx + j];
            if (d.t.bf16) raw16 = static_cast<const uint16_t*>(d.t.p)[row * d.ld_t + j];
            else raw = static_cast<const uint32_t*>(d.t.p)[row * d.ld_t + j];
        }
    }
    __device__ __forceinline__ void name_label(const Distill& d, int64_t row) { at = d.labels ? d.labels[row] : -1; }
    __device__ __forceinline__ void take(const Distill& d)
    {
        t = __uint_as_float(raw | raw16 << 16), z = 0;
        if (at < 0 || at >= d.n) at = -1, t = -kInf;
    }
    __device__ __forceinline__ void take_label(const Distill& d)         // a wavefront's row is one
    {
        at = __builtin_amdgcn_readfirstlane(at), z = 0;
        if (at < 0 || at >= d.n) at = -1;
    }
    // With a range of coordinates only, logits elsewhere are not looked at.
    template <typename T>
    __device__ __forceinline__ void look(const T* row, int64_t from, int64_t to)
    {
        if (at >= from && at < to) z = sizeof(T) == 2 ? (uint32_t)reinterpret_cast<const uint16_t*>(row)[at] : reinterpret_cast<const uint32_t*>(row)[at];
    }
    template <typename T>
    __device__ __forceinline__ float logit() const { return __uint_as_float(sizeof(T) == 2 ? z << 16 : z); }
    template <typename T>
    __device__ __forceinline__ void keep(const List& l, uint32_t j) const
    {
        l.idx[j] = at, l.p[j] = t, l.z[j] = logit<T>();
        if (at >= 0) l.slots[slot_of(l, at)] = (uint16_t)j;
    }
};

// What a row's terms come to, but for the sums over its logits.
struct Terms {
    float   soft;                       // P: 0 where there is no first term, else 1, or NaN
    float   cross;                      // sum p (log p - (z - largest) / T)
    float   share;                      // sum p, as rounding has it
    float   label_z;
    int32_t label;                      // -1: none
    bool    listed;                     // is the label's coordinate in the list, too
};

// A wavefront makes p of the list: `first` is its lanes' first entries, the others are fetched here.  An entry that finds
// another one in its slot marks it, and all entries of a marked slot are told apart where dz is written.
template <typename T>
__device__ __forceinline__ Terms take_list(const Distill& d, const List& l, int64_t row, const T* z, Entry first, Entry label, float largest,
                                           int64_t from, int64_t to)
{
    constexpr uint16_t kMarked = 0xFFFF;
    const uint32_t lane = fresh(threadIdx.x & 63u);
    float most = first.t;
    bool  listed = first.at == label.at;
    if (lane < d.top) first.keep<T>(l, lane);
    for (uint32_t j = lane + 64; j < d.top; j += 64) {
        Entry e;
        e.name(d, row, j);
        e.take(d);
        e.look(z, from, to);
        e.keep<T>(l, j);
        most = fmaxf(most, e.t);
        listed |= e.at == label.at;
    }
    most = wave_max(most);
    float sum = 0.0f;
    for (uint32_t j = lane; j < d.top; j += 64) {
        const float   v = l.p[j];
        const int32_t at = l.idx[j];
        if (v != -kInf) sum += expf((v - most) * d.inv_t);               // NaN among them, or +infinity: NaN
        if (at >= 0) {
            uint16_t& slot = slot_again(l, at);
            if (slot != j) slot = kMarked;
        }
    }
    sum = wave_sum(sum);
    const float log_sum = logf(sum);
    Terms w = {sum == 0.0f ? 0.0f : sum * 0.0f + 1.0f, 0.0f, 0.0f, label.logit<T>(), label.at, __ballot(listed) != 0 && label.at >= 0};
    for (uint32_t j = lane; j < d.top; j += 64) {
        const float   v = l.p[j];
        const int32_t at = l.idx[j];
        float p = 0.0f;
        if (v != -kInf) {
            const float log_p = (v - most) * d.inv_t - log_sum;
            p = expf(log_p);
            if (p != 0.0f) w.cross += p * (log_p - (l.z[j] - largest) * d.inv_t), w.share += p;
        }
        const bool met = at >= 0 && slot_again(l, at) != j;
        l.p[j] = __uint_as_float((__float_as_uint(p) & 0x7FFFFFFFu) | (met ? 0x80000000u : 0u));
    }
    w.cross = wave_sum(w.cross), w.share = wave_sum(w.share);
    return w;
}
__device__ __forceinline__ float loss_of(const Distill& d, const Terms& w, float largest, float a, float b)
{
    float loss = 0.0f;
    if (w.soft != 0.0f) loss = d.soft_loss * (w.cross + logf(a) * w.share) * w.soft;
    if (w.label >= 0) loss += d.hard * (logf(b) - (w.label_z - largest));
    return loss;
}

// dz away from the list: a e_a + b e_b.
struct Weights {
    float a, b, largest, g;
    bool  any;                          // is there a term at all
    template <int TERMS>
    __device__ __forceinline__ float of(const Pair<TERMS>& e) const
    {
        return TERMS == kOne ? a * e.a : TERMS == kTwo ? __builtin_fmaf(b, e.b, a * e.a) : __builtin_fmaf(b, e.a, a) * e.a;
    }
};
template <int TERMS>
__device__ __forceinline__ Weights weights_of(const Distill& d, float soft, int32_t label, float g, float largest, float a, float b)
{
    const float first = soft != 0.0f ? g * (soft * d.soft_grad) / a : 0.0f, second = label >= 0 ? g * d.hard / b : 0.0f;
    return {TERMS == kOne ? first + second : first, second, largest, g, soft != 0.0f || label >= 0};
}
template <typename T, int TERMS>
__device__ __forceinline__ void plain_grad(const Chunk<T>& c, const Weights& w, float scale, float (&y)[kChunk<T>])
{
#pragma unroll
    for (int i = 0; i < kChunk<T>; ++i) y[i] = w.any ? w.of(Pair<TERMS>(c.at(i) - w.largest, scale)) : 0.0f;
}

// dz at what the list and the label name among the coordinates from `from` to `to` that this wavefront wrote before: chunks go
// round THREADS threads.
template <typename T, int THREADS, int TERMS>
__device__ __forceinline__ void patch(const Distill& d, const List& l, const Weights& w, int64_t row, const Terms& terms, int64_t from,
                                      int64_t to)
{
    const uint32_t lane = fresh(threadIdx.x & 63u);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x % THREADS / 64);
    if (!w.any) return;
    auto ours = [&](int32_t at) {                                        // none is -1
        return at >= from && at < to && (uint32_t)(at - (int32_t)from) / (64 * kChunk<T>) % (THREADS / 64) == wave;
    };
    auto put = [&](int32_t at, float z, float p) {
        const float off = d.soft_grad * p + (at == terms.label ? d.hard : 0.0f);
        d.dz.put(row * d.ld_dz + at, w.of(Pair<TERMS>(z - w.largest, d.scale)) - w.g * off);
    };
    // these stores are behind the ones before without a wait: a wavefront's are in order
    for (uint32_t base = 0; base < d.top; base += 64) {
        const uint32_t j = base + lane;
        const int32_t  at = j < d.top ? l.idx[j] : -1;
        bool  write = ours(at);
        float p = write ? l.p[j] : 0.0f;
        // Entries that share their slot, one by one: the first of a coordinate has the sum in the list's order, and takes the others
        // out of the list, so that a coordinate is looked for once, however often it is named (64 rows of 5000 with 4096 entries
        // for one coordinate 0.2 ms; each of them looking for all 538).
        for (uint64_t met = __ballot(write && __float_as_uint(p) >> 31); met;) {
            const int     whose = __builtin_ctzll(met);
            const int32_t name = __builtin_amdgcn_readlane(at, whose);
            float sum = 0.0f;
            for (uint32_t i = base; i < d.top; i += 64) {
                const bool same = i + lane < d.top && l.idx[i + lane] == name;
                const float q = same ? l.p[i + lane] : 0.0f;
                uint64_t hits = __ballot(same);
                if (i == base) met &= ~hits, write &= !same;
                else if (same) l.idx[i + lane] = -1;
                for (; hits; hits &= hits - 1) sum += fabsf(lane_of(q, __builtin_ctzll(hits)));
            }
            if (lane == (uint32_t)whose) p = sum, write = true;
        }
        if (write) put(at, l.z[j], fabsf(p));
    }
    if (!terms.listed && lane == 0 && ours(terms.label)) put(terms.label, terms.label_z, 0.0f);
}

// ---- a row in registers ------------------------------------------------------------------------------------------------

// How many chunks of the next row a thread has in LDS beforehand.
__host__ __device__ constexpr int ahead_of(int lanes, int chunks) { return lanes > 64 ? chunks / 2 : 0; }
constexpr int kSixteenOps = 0x4F70;     // s_waitcnt: no more than sixteen vector loads and stores in flight

// LANES threads with up to C whole chunks each, and one that the row may end in.  With no more than a hundred registers
// beside them: whole chunks come and go through buffers, and chunks that a row does not have are 0 and left out.
//
// 1024 threads have a unit to themselves (OUT: 1 + whether dz is bf16, else 0: known at run time).  So that memory has as much to do
// while a row is summed up as while it is written, chunks whose successors come from memory are written first, and the stores
// of the others need not have ended when the next row's maximum is looked for: waits count what was issued since, which takes a
// store for each chunk, beyond the row's end as well, where the buffer drops it (4096 x 131,072 bf16 T = 2
// 451 -> 432 us, T = 3 487 -> 449).
//
// GIVEN: the gradient alone, from the stats of a call before (a variant of its own: asked at run time, loss and dz of 20,000 x 100 bf16
// took 26.2 us instead of 24.1).
template <typename T, int LANES, int C, int TERMS, bool AHEAD, int OUT, bool GIVEN>
__global__ __launch_bounds__(kThreadsOf<LANES>, C == 4 ? 6 : 4) void mv_distill_kernel(Distill d)
{
    constexpr int V = kChunk<T>, kRows = kThreadsOf<LANES> / LANES, kWaves = LANES / 64;
    __shared__ float tops[kWaves], sums[2][kWaves];
    __shared__ Terms shared;
    __shared__ float shared_g;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const uint32_t t = threadIdx.x % LANES, mine = __builtin_amdgcn_readfirstlane(threadIdx.x / LANES);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(t / 64);
    const List list = list_at(lds + mine * list_bytes(d.top), d.top);
    const int n = (int)d.n, full = n / (LANES * V), rest = n - full * (LANES * V) - (int)t * V;
    Chunk<T> held[C], tail;
    // The first chunks of the next row are fetched into LDS while this one's are summed up; each wavefront reads its own again.
    constexpr int kAhead = AHEAD ? ahead_of(LANES, C) : 0;
    __shared__ __attribute__((aligned(16))) uint8_t ahead[kAhead ? kAhead * LANES * 16 : 16];
    const bool out16 = OUT ? OUT == 2 : d.dz.bf16;
    // in one scalar comparison each time, not in sixteen masks that are kept
    auto there = [&](int c) {
        int f = full;
        asm("" : "+s"(f));
        return c < f;
    };
    auto row_at = [&](int64_t row) { return static_cast<const T*>(d.z) + row * d.ld_z; };
    auto fetch_tail = [&](const T* z) {
        if (rest > 0) tail.load_low(z + full * (LANES * V) + t * V, rest);
        else tail.none();
    };
    int64_t row = (int64_t)blockIdx.x * kRows + mine;
    const int64_t step = (int64_t)gridDim.x * kRows;
    if (row >= d.rows) return;                                           // a wavefront's own row, or the whole workgroup's
    {
        const RowOf z(row_at(row), full * (LANES * 16));
#pragma unroll
        for (int c = 0; c < C; ++c) held[c].take(z.load(t * 16, c * (LANES * 16)));
        fetch_tail(row_at(row));
    }
    Entry entry, label;
    float g = 1.0f, had[3];
    auto name = [&](int64_t of) {
        entry.name(d, of, t), label.name_label(d, of);
        if (d.grad) g = d.grad[of];
        if constexpr (GIVEN) had[0] = d.had[3 * of], had[1] = d.had[3 * of + 1], had[2] = d.had[3 * of + 2];
    };
    if (wave == 0) name(row);
    if (OUT) __builtin_amdgcn_s_waitcnt(kNoLoads);                       // or the loop would wait for all of its own each time
    for (; row < d.rows; row += step) {
        float largest;
        if constexpr (GIVEN) {
            largest = had[0];
        } else {
            Largest<T> most;
            most.look(tail);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (there(c)) most.look(held[c]);
            largest = wave_max(most.value());
        }
        if (wave == 0) {
            entry.take(d), label.take_label(d);
            entry.look(row_at(row), 0, d.n), label.look(row_at(row), 0, d.n);
        }
        const bool more = row + step < d.rows;                           // behind the last row there is nothing
        const RowOf next(row_at(more ? row + step : row), more ? full * (LANES * 16) : 0);
        if constexpr (kWaves > 1) {
            if ((t & 63u) == 0) tops[wave] = largest;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kWaves; ++w) largest = larger(tops[w], largest);
        }
        if constexpr (kAhead > 0) {
            __builtin_amdgcn_s_waitcnt(kNoLds);                          // what was read of the last ones is here
#pragma unroll
            for (int c = 0; c < kAhead; ++c) next.load_lds(ahead + (c * kWaves + wave) * 1024, t * 16, c * (LANES * 16));
        }
        float a = 0.0f, b = 0.0f;
        if constexpr (GIVEN) {
            static_assert(kWaves == 1, "sums of a wavefront's own");
            a = had[1], b = had[2];
        } else {
            add_up<T, TERMS>(tail, largest, d.scale, a, b);
#pragma unroll
            for (int c = 0; c < C; ++c)
                if (there(c)) add_up<T, TERMS>(held[c], largest, d.scale, a, b);
            a = wave_sum(a);
            if (TERMS != kOne) b = wave_sum(b);
        }
        float row_g = g;
        Terms w;
        if (wave == 0) w = take_list(d, list, row, row_at(row), entry, label, largest, 0, d.n);
        // Dz may be z: what is read of the row is in registers or LDS by now.
        if constexpr (kWaves > 1) {
            if ((t & 63u) == 0) sums[0][wave] = a, sums[1][wave] = b;
            if (t == 0) shared = w, shared_g = g;
            // the next row's chunks need not be here
            if constexpr (OUT) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            else __syncthreads();
            a = b = 0.0f;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) a += sums[0][i], b += sums[1][i];
            w = shared, row_g = shared_g;
        }
        if (TERMS == kOne && !GIVEN) b = a;
        if (t == 0 && !GIVEN) {
            if (d.loss) d.loss[row] = loss_of(d, w, largest, a, b);
            if (d.stats) {
                d.stats[3 * row] = largest;
                d.stats[3 * row + 1] = d.top ? a : 0.0f;
                d.stats[3 * row + 2] = d.labels ? b : 0.0f;
            }
        }
        const Weights weights = weights_of<TERMS>(d, w.soft, w.label, row_g, largest, a, b);
        // each chunk's registers take the next row's as soon as its own is written
        const RowOf dz(static_cast<char*>(d.dz.p) + row * d.ld_dz * (out16 ? 2 : 4), d.dz.p ? full * (LANES * V) * (out16 ? 2 : 4) : 0);
        if (d.dz.p) {
            float y[V];
            plain_grad<T, TERMS>(tail, weights, d.scale, y);
            d.dz.store(row * d.ld_dz + full * (LANES * V) + t * V, rest, y);
        }
        if (more) fetch_tail(row_at(row + step));
#pragma unroll
        for (int i = 0; i < C; ++i) {
            const int c = OUT ? (i + kAhead) % C : i;
            if (i == C / 2 && wave == 0 && more) name(row + step);
            if (OUT && i == C - kAhead) __builtin_amdgcn_s_waitcnt(kSixteenOps);     // a store and a load a chunk: the ones into LDS are here
            float y[V] = {};
            if (there(c)) {
                held[c].forget();                                        // what was made of it for the sums is not kept
                plain_grad<T, TERMS>(held[c], weights, d.scale, y);
                if (!OUT) dz.store<LANES>(y, t, c, out16);
            }
            if (OUT) dz.store<LANES>(y, t, c, out16);
            if (c < kAhead) held[c].take(*reinterpret_cast<const u32x4*>(ahead + (c * kWaves + wave) * 1024 + (t & 63u) * 16));
            else held[c].take(next.load(t * 16, c * (LANES * 16)));
        }
        if (d.dz.p) patch<T, LANES, TERMS>(d, list, weights, row, w, 0, d.n);
    }
}

// ---- rows that stream by ---------------------------------------------------------------------------------------------

constexpr int kRangeThreads = 512;      // of a range
template <typename T>
constexpr int kAhead = sizeof(T) == 2 ? 2 : 4;                           // chunks of a turn

// A thread's largest and sums of [first, last) of a row: each turn's largest first, what was added up before scaled down to it.
template <typename T, int THREADS, int TERMS>
__device__ __forceinline__ void stream(const T* z, int64_t first, int64_t last, float scale, float& largest, float& a, float& b)
{
    constexpr int V = kChunk<T>, G = kAhead<T>;
    constexpr int64_t kTurn = (int64_t)THREADS * V * G;
    largest = -kInf, a = b = 0.0f;
    for (int64_t at = first; at < last; at += kTurn) {
        Chunk<T> c[G];
        const T* p = z + at + threadIdx.x * V;
        if (at + kTurn <= last) {
#pragma unroll
            for (int g = 0; g < G; ++g) c[g].load(p + g * (THREADS * V), V);
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t live = last - at - threadIdx.x * V - g * (THREADS * V);
                c[g].load_low(p + g * (THREADS * V), live < 0 ? 0 : live < V ? (int)live : V);
            }
        }
        Largest<T> most;
#pragma unroll
        for (int g = 0; g < G; ++g) most.look(c[g]);
        const float top = most.value();
        if (top > largest) {                                             // from -infinity: of nothing
            const float down = largest - top;
            a *= power(down * scale);
            if (TERMS != kOne) b *= power(down * kLog2e);
            largest = top;
        }
        const float base = largest == -kInf ? 0.0f : largest;
#pragma unroll
        for (int g = 0; g < G; ++g) add_up<T, TERMS>(c[g], base, scale, a, b);
    }
}
// Joined over the workgroup; sums of nothing but -infinity are 0.
template <int THREADS, int TERMS>
__device__ __forceinline__ void join(Across<THREADS>& across, float scale, float& largest, float& a, float& b)
{
    const float top = across.max(largest), down = largest - (top == -kInf ? 0.0f : top);
    a *= power(down * scale);
    if (TERMS != kOne) b *= power(down * kLog2e);
    across.sum2(a, b);
    if (TERMS == kOne) b = a;
    largest = top;
}

// The loss of whole rows, a workgroup each.
template <typename T, int THREADS, int TERMS>
__global__ __launch_bounds__(THREADS) void mv_distill_loss_kernel(Distill d)
{
    __shared__ float sums[2][2][THREADS / 64];
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    Across<THREADS> across(sums);
    const List list = list_at(lds, d.top);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    for (int64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        Entry entry, label;
        if (wave == 0 && d.loss) {
            entry.name(d, row, threadIdx.x), label.name_label(d, row);
            entry.take(d), label.take_label(d);
            entry.look(z, 0, d.n), label.look(z, 0, d.n);
        }
        float largest, a, b;
        stream<T, THREADS, TERMS>(z, 0, d.n, d.scale, largest, a, b);
        join<THREADS, TERMS>(across, d.scale, largest, a, b);
        // a row of nothing but -infinity has no sums
        if (largest == -kInf) a = b = __builtin_nanf("");
        if (wave == 0) {
            if (d.loss) {
                const Terms w = take_list(d, list, row, z, entry, label, largest, 0, d.n);
                if (threadIdx.x == 0) d.loss[row] = loss_of(d, w, largest, a, b);
            }
            if (threadIdx.x == 0 && d.stats) {
                d.stats[3 * row] = largest;
                d.stats[3 * row + 1] = d.top ? a : 0.0f;
                d.stats[3 * row + 2] = d.labels ? b : 0.0f;
            }
        }
    }
}

// Largest and sums of a range.
template <typename T, int TERMS>
__global__ __launch_bounds__(kRangeThreads) void mv_distill_range_kernel(Distill d)
{
    __shared__ float sums[2][2][kRangeThreads / 64];
    Across<kRangeThreads> across(sums);
    const int64_t all = d.rows * d.ranges;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
        const int64_t row = at / d.ranges, first = at % d.ranges * d.range, last = first + d.range < d.n ? first + d.range : d.n;
        float largest, a, b;
        stream<T, kRangeThreads, TERMS>(static_cast<const T*>(d.z) + row * d.ld_z, first, last, d.scale, largest, a, b);
        join<kRangeThreads, TERMS>(across, d.scale, largest, a, b);
        if (threadIdx.x == 0) {
            float* to = d.parts + 4 * at;
            to[0] = largest, to[1] = a, to[2] = b;
        }
    }
}

// A row's ranges joined, and its loss: a wavefront each.
template <typename T, int TERMS>
__global__ __launch_bounds__(64) void mv_distill_join_kernel(Distill d)
{
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const List list = list_at(lds, d.top);
    for (int64_t row = blockIdx.x; row < d.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        Entry entry, label;
        if (d.loss) {
            entry.name(d, row, threadIdx.x), label.name_label(d, row);
            entry.take(d), label.take_label(d);
            entry.look(z, 0, d.n), label.look(z, 0, d.n);
        }
        const float* part = d.parts + 4 * row * d.ranges;
        float largest = -kInf, a = 0.0f, b = 0.0f;
        for (uint32_t r = threadIdx.x; r < d.ranges; r += 64) largest = fmaxf(largest, part[4 * r]);
        largest = wave_max(largest);
        for (uint32_t r = threadIdx.x; r < d.ranges; r += 64) {
            const float down = part[4 * r] - largest;                    // of nothing but -infinity: NaN
            a += part[4 * r + 1] * power(down * d.scale);
            b += part[4 * r + 2] * power(down * (TERMS == kOne ? d.scale : kLog2e));
        }
        a = wave_sum(a), b = wave_sum(b);
        if (d.loss) {
            const Terms w = take_list(d, list, row, z, entry, label, largest, 0, d.n);
            if (threadIdx.x == 0) d.loss[row] = loss_of(d, w, largest, a, b);
        }
        if (threadIdx.x == 0 && d.stats) {
            d.stats[3 * row] = largest;
            d.stats[3 * row + 1] = d.top ? a : 0.0f;
            d.stats[3 * row + 2] = d.labels ? b : 0.0f;
        }
    }
}

// dz of a range, from the row's stats.
template <typename T, int THREADS, int TERMS>
__global__ __launch_bounds__(THREADS) void mv_distill_grad_kernel(Distill d)
{
    constexpr int V = kChunk<T>, G = kAhead<T>;
    constexpr int64_t kTurn = (int64_t)THREADS * V * G;
    __shared__ Terms shared;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const List list = list_at(lds, d.top);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int64_t all = d.rows * d.ranges;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x) {
        const int64_t row = at / d.ranges, first = at % d.ranges * d.range, last = first + d.range < d.n ? first + d.range : d.n;
        const T* z = static_cast<const T*>(d.z) + row * d.ld_z;
        const float* had = d.had + 3 * row;
        const float largest = had[0];
        if (wave == 0) {
            Entry entry, label;                                          // logits elsewhere may have been written over
            entry.name(d, row, threadIdx.x), label.name_label(d, row);
            entry.take(d), label.take_label(d);
            entry.look(z, first, last), label.look(z, first, last);
            const Terms w = take_list(d, list, row, z, entry, label, largest, first, last);
            if (threadIdx.x == 0) shared = w;
            __builtin_amdgcn_s_waitcnt(kNoLoads);                        // dz may be z: the list's logits are here
        }
        __syncthreads();
        const Terms   terms = shared;
        const Weights w = weights_of<TERMS>(d, terms.soft, terms.label, d.grad ? d.grad[row] : 1.0f, largest, had[1], had[2]);
        for (int64_t col = first; col < last; col += kTurn) {
            Chunk<T> c[G];
            int live[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int64_t left = last - col - threadIdx.x * V - g * (THREADS * V);
                live[g] = left < 0 ? 0 : left < V ? (int)left : V;
                c[g].load(z + col + threadIdx.x * V + g * (THREADS * V), live[g]);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float y[V];
                plain_grad<T, TERMS>(c[g], w, d.scale, y);
                d.dz.store(row * d.ld_dz + col + threadIdx.x * V + g * (THREADS * V), live[g], y);
            }
        }
        patch<T, THREADS, TERMS>(d, list, w, row, terms, first, last);
        __syncthreads();                                                 // the list and the terms are read before the next ones
    }
}

// How a row is held: LANES threads with C chunks each, or 0: not at all.
struct Lanes {
    int lanes, chunks;
};
static Lanes lanes_of(int64_t rows, int64_t n, int32_t dtype, int64_t top)
{
    // A few long rows are cut into ranges, for a workgroup each in three launches: 1 x 131,072 bf16 23 -> 15 us, 48 rows 25 -> 18, of
    // 72,000 1 16 -> 15 and 48 17 -> 16; but 128 rows 29 -> 28 and 18 -> 22, of 33,000 1 12.5 -> 14.
    if (rows <= 48 && n > 65536) return {0, 0};
    const int64_t wide = dtype == MV_BF16 ? 8 : 4, chunks = n / wide;
    // A wavefront's rows need no barriers, and four times as many are at once on a unit: 8192 x 2500 bf16 26 us, with 256 threads 50; fp32
    // 42 (53); 4096 x 8192 bf16 30 (35); but 1000 x 8192 13.5 (12.3).  Four rows' lists share a workgroup's LDS.
    if (chunks < 64 * 4 && top <= 1024) return {64, 4};
    if (chunks < 64 * 17 && top <= 1024 && rows >= 1000) return {64, 16};
    for (int lanes : {256, 512, 1024})
        if (chunks < (int64_t)lanes * 17) return {lanes, 16};            // the tail is one more
    return {0, 0};
}

// Ranges of rows: of 16,384 values or more, as few as give the card a thousand workgroups.
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

template <typename T, int LANES, int C, int TERMS, bool GIVEN = false>
static void held(const Distill& d, hipStream_t st)
{
    constexpr int kRows = kThreadsOf<LANES> / LANES;
    // as many as run at once: sixteen wavefronts to a unit, of the smallest rows twenty-four (20,000 x 100 bf16 30 -> 26 us)
    const dim3   grid(grid_of((d.rows + kRows - 1) / kRows, C == 4 ? 1536 : 256 * 1024 / kThreadsOf<LANES>)), group(kThreadsOf<LANES>);
    const size_t lists = kRows * list_bytes(d.top);
    auto launch = [&](auto ahead, auto out) {
        hipLaunchKernelGGL((mv_distill_kernel<T, LANES, C, TERMS, decltype(ahead)::value, decltype(out)::value, GIVEN>), grid, group, lists,
                           st, d);
    };
    const std::integral_constant<int, 0> any{};
    if constexpr (LANES < 1024) {
        launch(std::true_type{}, any);
    } else {
        // the longest lists need the LDS that the next row would have: 160 KB less what the kernel's own variables take
        if (ahead_of(LANES, C) * LANES * 16 + lists > 159 * 1024) launch(std::false_type{}, any);
        else if (d.dz.bf16) launch(std::true_type{}, std::integral_constant<int, 2>{});
        else launch(std::true_type{}, std::integral_constant<int, 1>{});
    }
}
// Threads of a row, or range, that streams by: as few as have a few chunks each, for many short ones are at once on a unit then, and
// a list's way is long (6 us).  us with 64, 256 and 512.  The loss alone: 8192 x 5000 bf16 23, 28, 40; fp32 35, 34, 50; 8192 x
// 12,000 bf16 47, 42, 60; 8192 x 30,000 101, 90, 102; 3000 x 32,768 43, 41, 40; 4000 x 30,000 fp32 88, 86, 82; 100 x 2500 fp32 12, 9, 9.  Dz: 8192 x
// 5000 bf16 48, 53, 67; 8192 x 2500 fp32 52, 45, 69; 8192 x 12,000 bf16 98, 86, 101; fp32 198, 168, 152; 3000 x 32,768 bf16 86, 82, 77.
template <typename F>
static void with_threads(int64_t rows, int64_t chunks, int64_t most256, F launch)
{
    if (chunks <= 640 && rows >= 1000) launch(std::integral_constant<int, 64>{});
    else if (chunks <= most256) launch(std::integral_constant<int, 256>{});
    else launch(std::integral_constant<int, 512>{});
}
template <typename T, int TERMS>
static void grad(Distill d, const Lanes& l, hipStream_t st)
{
    // The shortest rows in registers, as for the loss: 8192 x 1000 bf16 13.8 us, streaming by 55.
    if (l.chunks == 4) return held<T, 64, 4, TERMS, true>(d, st);
    const Ranges r = ranges_of(d.rows, d.n);
    d.ranges = r.count, d.range = r.length;
    with_threads(d.rows * r.count, d.range / kChunk<T>, 2048, [&](auto threads) {
        constexpr int kThreads = decltype(threads)::value;
        hipLaunchKernelGGL((mv_distill_grad_kernel<T, kThreads, TERMS>), dim3(grid_of(d.rows * r.count, 1 << 20)), dim3(kThreads),
                           list_bytes(d.top), st, d);
    });
}
template <typename T, int TERMS>
static void loss(Distill d, const Lanes& l, hipStream_t st)
{
    if (l.chunks == 4) return held<T, 64, 4, TERMS>(d, st);
    if (d.dz.p && l.lanes == 64) return held<T, 64, 16, TERMS>(d, st);
    if (d.dz.p && l.lanes == 256) return held<T, 256, 16, TERMS>(d, st);
    if (d.dz.p && l.lanes == 512) return held<T, 512, 16, TERMS>(d, st);
    if (d.dz.p && l.lanes == 1024) return held<T, 1024, 16, TERMS>(d, st);
    const Ranges r = ranges_of(d.rows, d.n);
    d.ranges = r.count, d.range = r.length;
    if (r.count == 1 || !d.parts) {
        with_threads(d.rows, d.n / kChunk<T>, 4000, [&](auto threads) {
            constexpr int kThreads = decltype(threads)::value;
            hipLaunchKernelGGL((mv_distill_loss_kernel<T, kThreads, TERMS>), dim3(grid_of(d.rows, 1 << 20)), dim3(kThreads), list_bytes(d.top), st,
                               d);
        });
    } else {
        hipLaunchKernelGGL((mv_distill_range_kernel<T, TERMS>), dim3(grid_of(d.rows * r.count, 1 << 20)), dim3(kRangeThreads), 0, st, d);
        hipLaunchKernelGGL((mv_distill_join_kernel<T, TERMS>), dim3(grid_of(d.rows, 1 << 20)), dim3(64), list_bytes(d.top), st, d);
    }
    if (d.dz.p) {
        d.had = d.stats;
        grad<T, TERMS>(d, l, st);
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
    d.scale = d.top ? d.inv_t * kLog2e : kLog2e;                         // without a first term: of the second
    d.soft_grad = soft * temperature, d.soft_loss = soft * temperature * temperature, d.hard = hard;
    d.grad = g, d.dz = {dz, dz_dtype == MV_BF16}, d.ld_dz = ld_dz;
    return true;
}

template <typename F>
static mv_status with_terms(const Distill& d, float temperature, F launch)
{
    if (!d.top || !d.labels || temperature == 1.0f) launch(std::integral_constant<int, kOne>{});
    else if (temperature == 2.0f) launch(std::integral_constant<int, kSquare>{});
    else launch(std::integral_constant<int, kTwo>{});
    return launched();
}

}  // namespace mvr

extern "C" {

size_t mv_distill_scratch_bytes(int64_t rows, int64_t n)
{
    using namespace mvr;
    if (!size_valid(rows) || !size_valid(n)) return 0;
    // what is cut into ranges, and what no type's rows of are held
    return ranges_of(rows, n).count > 1 || !lanes_of(rows, n, MV_F32, 0).lanes ? parts_bytes(rows, n) + stats_bytes(rows) : 0;
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
    const Lanes l = lanes_of(rows, n, dtype, d.top);
    if (need) {
        d.parts = static_cast<float*>(scratch);
        if (!stats && !l.lanes) d.stats = reinterpret_cast<float*>(static_cast<char*>(scratch) + parts_bytes(rows, n));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_terms(d, temperature, [&](auto terms) {
        if (dtype == MV_BF16) mvr::loss<uint16_t, decltype(terms)::value>(d, l, st);
        else mvr::loss<float, decltype(terms)::value>(d, l, st);
    });
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
    const Lanes l = lanes_of(rows, n, dtype, d.top);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return with_terms(d, temperature, [&](auto terms) {
        if (dtype == MV_BF16) mvr::grad<uint16_t, decltype(terms)::value>(d, l, st);
        else mvr::grad<float, decltype(terms)::value>(d, l, st);
    });
}

}  // extern "C"
