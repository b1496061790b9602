// Products of microscaled 4-bit matrices (mv_mx_product, mv_mx_linear, mv_mx_linear_grad of include/mv.h).
//
//   c[i][j] = sum_k a[i][k] b[j][k],  both factors in blocks of 32 along k
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of each factor times four blocks: lane l holds row l % 16 of a
// block, 16 bytes of codes, and the block's scale in one byte of a register; which blocks of k the four groups of lanes
// hold does not matter as long as both factors agree.  So a group takes four consecutive blocks of each 16: 64
// consecutive bytes of codes for four instructions, and their four scales in one word.
#include "mv_mx.hpp"

#include <type_traits>

namespace mvx {

typedef int   i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Factor {
    const uint32_t* codes;
    const uint8_t*  scales;
    int64_t         ld_words, ld_scales, rows;
};

// c += a b over one instruction's blocks, scale byte S of each word.
template <int S>
__device__ __forceinline__ f32x4 mfma(const u32x4& a, uint32_t a_scale, const u32x4& b, uint32_t b_scale, f32x4 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, S, (int)a_scale, S, (int)b_scale);
}

// Four consecutive blocks of a row, as far as there are any: what lies behind reads as zeros of scale 1.
struct Four {
    u32x4    codes[4];
    uint32_t scales;
};
__device__ __forceinline__ void load_four(const Factor& f, int64_t row, int64_t block, int64_t blocks, Four& v)
{
    const uint32_t* p = f.codes + row * f.ld_words + block * 4;
    const int64_t live = blocks - block;
#pragma unroll
    for (int s = 0; s < 4; ++s) v.codes[s] = s < live ? *reinterpret_cast<const u32x4*>(p + 4 * s) : u32x4{0u, 0u, 0u, 0u};
    uint32_t w = live > 0 ? *reinterpret_cast<const uint32_t*>(f.scales + row * f.ld_scales + block) : 0x7F7F7F7Fu;
    if (live > 0 && live < 4) {
        const uint32_t keep = (1u << (8 * (uint32_t)live)) - 1u;
        w = (w & keep) | (0x7F7F7F7Fu & ~keep);
    }
    v.scales = w;
}

// Four consecutive results of a row of which `live` are left.
typedef uint16_t u16x4u __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store4(float* p, int64_t live, const f32x4& v)
{
    if (live >= 4) {
        *reinterpret_cast<f32x4u*>(p) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < live) p[e] = v[e];
    }
}
__device__ __forceinline__ void store4(uint16_t* p, int64_t live, const f32x4& v)
{
    const u16x4u w = {(uint16_t)narrow(v.x), (uint16_t)narrow(v.y), (uint16_t)narrow(v.z), (uint16_t)narrow(v.w)};
    if (live >= 4) {
        *reinterpret_cast<u16x4u*>(p) = w;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < live) p[e] = w[e];
    }
}

__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)narrow(x); }

constexpr int kTile = 64;           // rows of each factor that a wavefront takes
constexpr int kProductThreads = 256;

template <typename T>
__global__ __launch_bounds__(kProductThreads) void mv_mx_product_kernel(Factor a, Factor b, int64_t blocks, int64_t tiles_n,
                                                                        T* __restrict__ c, int64_t ld_c)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64, in = lane & 15u, group = lane / 16;
    const int64_t i0 = (int64_t)blockIdx.x / tiles_n * (2 * kTile) + wave / 2 * kTile;
    const int64_t j0 = (int64_t)blockIdx.x % tiles_n * (2 * kTile) + wave % 2 * kTile;
    f32x4 acc[4][4] = {};
    for (int64_t k = 0; k < blocks; k += 16) {
        Four x[4], y[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t i = i0 + 16 * t + in, j = j0 + 16 * t + in;
            load_four(a, i < a.rows ? i : a.rows - 1, k + 4 * group, blocks, x[t]);
            load_four(b, j < b.rows ? j : b.rows - 1, k + 4 * group, blocks, y[t]);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                acc[t][u] = mfma<0>(y[u].codes[0], y[u].scales, x[t].codes[0], x[t].scales, acc[t][u]);
                acc[t][u] = mfma<1>(y[u].codes[1], y[u].scales, x[t].codes[1], x[t].scales, acc[t][u]);
                acc[t][u] = mfma<2>(y[u].codes[2], y[u].scales, x[t].codes[2], x[t].scales, acc[t][u]);
                acc[t][u] = mfma<3>(y[u].codes[3], y[u].scales, x[t].codes[3], x[t].scales, acc[t][u]);
            }
    }
    // a lane has four consecutive columns j of row i
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t i = i0 + 16 * t + in;
        if (i >= a.rows) continue;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t j = j0 + 16 * u + 4 * group;
            store4(c + i * ld_c + j, b.rows - j, acc[t][u]);
        }
    }
}

// ---- tiles through LDS ---------------------------------------------------------------------------------------------
//
// A workgroup of WM x WN wavefronts takes 32 MT WM x 32 NT WN results, 32 MT x 32 NT a wavefront, in steps of eight blocks (256 values,
// 128 bytes a row).  The rows of both factors go from memory straight into LDS, each row's 16-byte blocks in the order
// block ^ (row % 8): what eight lanes of neighbouring rows read together lies in different banks, and what eight lanes
// write together is one whole line of memory.  Two buffers: the next step's loads are in flight during this one's
// products.  Loads beyond the last row or block return zeros by the buffer's bounds.  The scales of two steps, 16 bytes a row,
// go through registers, where those behind the last block become 1, into LDS of their own.
//
// A lane of the 32 x 32 x 64 instruction holds half of a row's eight blocks: blocks 4 (lane / 32) + s of step s, whose
// scales are one word.

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int kStepBlocks = 8;
constexpr int kScalePitch = 20;     // bytes between the rows' scales in LDS: 16 and a word against bank conflicts

constexpr int kNoLoads = 0x0F70;    // s_waitcnt: none of the vector loads in flight, the other counters as they are

template <int S>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, uint32_t a_scale, const u32x4& b, uint32_t b_scale, f32x16 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, S, (int)a_scale, S, (int)b_scale);
}

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

// A wavefront's share of one instruction's blocks: rows of a and of b.
template <int MT, int NT>
struct Rows {
    u32x4 x[MT], y[NT];
};

template <int MT, int NT, int WM, int WN, typename T>
__global__ __launch_bounds__(64 * WM * WN, 2) void mv_mx_product_tile_kernel(Factor a, Factor b, uint32_t blocks, uint32_t tiles_m,
                                                                             uint32_t tiles_n, uint32_t steps_each,
                                                                             T* __restrict__ c, int64_t ld_c, int64_t split_c)
{
    constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    constexpr int kM = 32 * MT * WM, kN = 32 * NT * WN, kRows = kM + kN;
    typedef uint8_t Codes[kRows * 128];
    // two variables, not an array of two: reads of one need not wait for the loads into the other
    __shared__ __attribute__((aligned(1024))) Codes even, odd;
    __shared__ uint8_t scales[2][kRows * kScalePitch];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t / 64);
    uint32_t tm, tn;
    tile_of(blockIdx.x, tiles_m, tiles_n, tm, tn);
    const int64_t i0 = (int64_t)tm * kM, j0 = (int64_t)tn * kN;
    const uint32_t steps = (blocks + kStepBlocks - 1) / kStepBlocks;
    const uint32_t step0 = blockIdx.y * steps_each, count = min(steps_each, steps - step0);       // at least one
    const uint32_t end = min(blocks, (step0 + count) * kStepBlocks);       // an odd count's last step is one of zeros

    // what this wavefront loads: rows [wave kM / kWaves, ...) of a and as many of b, eight rows an instruction
    const uint32_t a_pitch = (uint32_t)a.ld_words * 4u, b_pitch = (uint32_t)b.ld_words * 4u;
    const int64_t a_rows = a.rows - i0 < kM ? a.rows - i0 : kM, b_rows = b.rows - j0 < kN ? b.rows - j0 : kN;
    const __amdgpu_buffer_rsrc_t a_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint32_t*>(a.codes + i0 * a.ld_words), 0, (int)((uint32_t)(a_rows - 1) * a_pitch + blocks * 16u), 0x00020000);
    const __amdgpu_buffer_rsrc_t b_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint32_t*>(b.codes + j0 * b.ld_words), 0, (int)((uint32_t)(b_rows - 1) * b_pitch + blocks * 16u), 0x00020000);
    const uint32_t my_block = (lane & 7u) ^ (lane >> 3);
    const uint32_t a_at = (wave * (kM / kWaves) + (lane >> 3)) * a_pitch + my_block * 16u;
    const uint32_t b_at = (wave * (kN / kWaves) + (lane >> 3)) * b_pitch + my_block * 16u;
    auto load_codes = [&](uint32_t k, Codes& to) {
        const uint32_t step = step0 + k;
        // The whole offset is the lane's own, for the bounds to hold: below 2^30 + 2^21, and beyond every buffer where the
        // row has no such block.
        const bool live = step * kStepBlocks + my_block < end;
        const uint32_t av = live ? a_at + step * 128u : 0x80000000u, bv = live ? b_at + step * 128u : 0x80000000u;
#pragma unroll
        for (int i = 0; i < kM / kWaves / 8; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                a_buf, (__attribute__((address_space(3))) void*)(to + (wave * (kM / kWaves) + i * 8) * 128), 16,
                av + i * 8 * a_pitch, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kN / kWaves / 8; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                b_buf, (__attribute__((address_space(3))) void*)(to + (kM + wave * (kN / kWaves) + i * 8) * 128), 16,
                bv + i * 8 * b_pitch, 0, 0, 0);
    };
    // the scales' rows
    constexpr int kScaleRows = (kRows + kThreads - 1) / kThreads;
    const uint8_t* scale_row[kScaleRows];
#pragma unroll
    for (int i = 0; i < kScaleRows; ++i) {
        const uint32_t r = t + kThreads * i;
        const int64_t at = r < kM ? i0 + r : j0 + (r - kM);
        scale_row[i] = r < kM ? a.scales + (at < a.rows ? at : a.rows - 1) * a.ld_scales
                              : b.scales + (at < b.rows ? at : b.rows - 1) * b.ld_scales;
    }
    const uint32_t last_word = (end - 1) / 4 * 4;
    uint32_t next[kScaleRows][4];
    auto fetch_scales = [&](uint32_t k) {
#pragma unroll
        for (int i = 0; i < kScaleRows; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w)
                next[i][w] = *reinterpret_cast<const uint32_t*>(scale_row[i] + min((step0 + k) * kStepBlocks + 4 * w, last_word));
    };
    auto keep_scales = [&](uint32_t pair) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int live = (int)end - (int)((step0 + 2 * pair) * kStepBlocks + 4 * w);
            const uint32_t real = live >= 4 ? 0xFFFFFFFFu : live > 0 ? (1u << (8 * live)) - 1u : 0u;
#pragma unroll
            for (int i = 0; i < kScaleRows; ++i)
                if (kRows % kThreads == 0 || t + kThreads * i < kRows)
                    *reinterpret_cast<uint32_t*>(&scales[pair & 1u][(t + kThreads * i) * kScalePitch + 4 * w]) =
                        (next[i][w] & real) | (0x7F7F7F7Fu & ~real);
        }
    };

    const uint32_t in = lane & 31u, half = lane >> 5;
    const uint32_t a_row = wave / WN * (32 * MT) + in, b_row = kM + wave % WN * (32 * NT) + in;
    f32x16 acc[MT][NT] = {};
    Rows<MT, NT> one, two;
    uint32_t as[MT], bs[NT], as_next[MT], bs_next[NT];
    auto read_rows = [&](const Codes& from, uint32_t s, Rows<MT, NT>& r) {
        const uint32_t slot = ((4 * half + s) ^ (lane & 7u)) * 16;
#pragma unroll
        for (int i = 0; i < MT; ++i) r.x[i] = *reinterpret_cast<const u32x4*>(from + (a_row + 32 * i) * 128 + slot);
#pragma unroll
        for (int i = 0; i < NT; ++i) r.y[i] = *reinterpret_cast<const u32x4*>(from + (b_row + 32 * i) * 128 + slot);
    };
    auto read_scales = [&](uint32_t k) {
        const uint8_t* sc = scales[k >> 1 & 1u] + (k & 1u) * 8 + half * 4;
#pragma unroll
        for (int i = 0; i < MT; ++i) as_next[i] = *reinterpret_cast<const uint32_t*>(sc + (a_row + 32 * i) * kScalePitch);
#pragma unroll
        for (int i = 0; i < NT; ++i) bs_next[i] = *reinterpret_cast<const uint32_t*>(sc + (b_row + 32 * i) * kScalePitch);
    };
    auto products = [&](auto s, const Rows<MT, NT>& r) {
        constexpr int S = decltype(s)::value;
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int j = 0; j < NT; ++j) acc[i][j] = mfma32<S>(r.y[j], bs[j], r.x[i], as[i], acc[i][j]);
    };
    // The first three quarters of a step whose first rows are in `one` and its scales in the next ones already.
    auto most_of_step = [&](const Codes& now) {
#pragma unroll
        for (int i = 0; i < MT; ++i) as[i] = as_next[i];
#pragma unroll
        for (int i = 0; i < NT; ++i) bs[i] = bs_next[i];
        read_rows(now, 1, two);
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 0>{}, one);
        __builtin_amdgcn_sched_barrier(0);
        read_rows(now, 2, one);
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 1>{}, two);
        __builtin_amdgcn_sched_barrier(0);
        read_rows(now, 3, two);
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 2>{}, one);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto all_here = [&] {
        __builtin_amdgcn_s_waitcnt(kNoLoads);
        __syncthreads();
    };
    auto last_of_step = [&] {
        __builtin_amdgcn_sched_barrier(0);
        products(std::integral_constant<int, 3>{}, two);
        __builtin_amdgcn_sched_barrier(0);
    };
    load_codes(0, even);
    fetch_scales(0);
    keep_scales(0);
    all_here();
    load_codes(1, odd);
    read_rows(even, 0, one);
    read_scales(0);
    // Two steps a turn.  Before a step's last products come the next one's first rows, so those products cover the way
    // from LDS, and the loads into this step's buffer begin as soon as all wavefronts have read it.  The turn has no
    // branches, or the compiler moves products past them and runs out of registers: behind the last step zeros are loaded.
    for (uint32_t k = 0; k < count; k += 2) {
        most_of_step(even);
        all_here();
        read_rows(odd, 0, one);
        read_scales(k + 1);
        fetch_scales(k + 2);
        load_codes(k + 2, even);
        last_of_step();
        most_of_step(odd);
        keep_scales(k / 2 + 1);
        all_here();
        read_rows(even, 0, one);
        read_scales(k + 2);
        load_codes(k + 3, odd);
        last_of_step();
    }
    __builtin_amdgcn_s_waitcnt(kNoLoads);

    // a lane has, of row i, four times four consecutive columns
    T* out = c + blockIdx.y * split_c;
    const int64_t col0 = j0 + wave % WN * (32 * NT) + 4 * half;
    const bool whole = j0 + kN <= b.rows;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int64_t row = i0 + a_row + 32 * i;
        if (row >= a.rows) continue;
        T* to = out + row * ld_c + col0;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (whole) store4(to + 32 * j + 8 * q, 4, v);
                else store4(to + 32 * j + 8 * q, b.rows - (col0 + 32 * j + 8 * q), v);
            }
    }
}

// c = the sum of the splits, in their order.
template <typename T>
__global__ __launch_bounds__(256) void mv_mx_product_join_kernel(const float* __restrict__ parts, int splits, int64_t m, int64_t n,
                                                                 int64_t split_c, int64_t quads, T* __restrict__ c, int64_t ld_c)
{
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t i = at / quads, j = at % quads * 4;
    if (i >= m) return;
    const float* p = parts + i * (quads * 4) + j;
    f32x4 sum = *reinterpret_cast<const f32x4*>(p);
    for (int s = 1; s < splits; ++s) sum += *reinterpret_cast<const f32x4*>(p + s * split_c);
    store4(c + i * ld_c + j, n - j, sum);
}

// ---- few rows of one factor ------------------------------------------------------------------------------------------
//
// Up to 16 rows of one factor ("few") against many of the other ("many"), whose codes are the bytes to read.  A workgroup
// takes 16 NT of the many rows and all of k, its wavefronts turns of 16 blocks; what they have is added up through LDS in
// the wavefronts' order.  Lane l of an instruction holds row l % 16 and block 4 s + l / 16 of the turn, s = 0 .. 3: the
// four lanes of a row read 64 bytes in a row; the scales of a lane's four blocks are picked from the row's 16.
// The few rows' codes and scales are in LDS: copied there, or quantised by every workgroup for itself, a lane a block,
// while the first turn's codes are on their way.

constexpr int kTurn = 16;           // blocks
constexpr int kFewWaves = 8;
template <typename X>
struct Few {                        // X: uint32_t: codes; uint16_t or float: bf16 or fp32 values
    const X*       rows;
    int64_t        ld;
    const uint8_t* scales;          // of codes
    int64_t        ld_scales;
    uint32_t       count;
};

// Byte g of each of a turn's four words of scales: those of blocks 4 s + g.
__device__ __forceinline__ uint32_t pick_scales(const u32x4& w, uint32_t g)
{
    const uint32_t two = (g | (4u + g) << 8) | 0x0C0C0000u;              // byte g of the second and of the first argument
    return __builtin_amdgcn_perm(w.y, w.x, two) | __builtin_amdgcn_perm(w.w, w.z, two) << 16;
}

// A block of the few rows on its way: fetched, and then made codes and scale of.
template <typename X>
struct Block;
template <>
struct Block<uint32_t> {
    u32x4    w;
    uint32_t scale;
    __device__ __forceinline__ void fetch(const Few<uint32_t>& f, uint32_t row, uint32_t block, int64_t)
    {
        w = *reinterpret_cast<const u32x4*>(f.rows + row * f.ld + 4 * (int64_t)block);
        scale = f.scales[row * f.ld_scales + block];
    }
    __device__ __forceinline__ void finish(u32x4& codes, uint32_t& s) const { codes = w, s = scale; }
};
template <>
struct Block<float> {
    float x[4][8];
    __device__ __forceinline__ void fetch(const Few<float>& f, uint32_t row, uint32_t block, int64_t k)
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) load8(f.rows + row * f.ld + (int64_t)block * kBlock + 8 * q, k - (int64_t)block * kBlock - 8 * q, x[q]);
    }
    __device__ __forceinline__ void finish(u32x4& codes, uint32_t& s) const
    {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[q][i]) & 0x7FFFFFFFu);
        s = scale_of(top);
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[q] = encode8(x[q], s);
    }
};
template <>
struct Block<uint16_t> {
    uint32_t x[4][4];
    __device__ __forceinline__ void fetch(const Few<uint16_t>& f, uint32_t row, uint32_t block, int64_t k)
    {
        const uint16_t* p = f.rows + row * f.ld + (int64_t)block * kBlock;
        const int64_t live = k - (int64_t)block * kBlock;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (live >= kBlock) {
                const u32x4u v = *reinterpret_cast<const u32x4u*>(p + 8 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[q][i] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int at = 8 * q + 2 * i;
                    x[q][i] = (at < live ? p[at] : 0u) | (at + 1 < live ? (uint32_t)p[at + 1] << 16 : 0u);
                }
            }
    }
    __device__ __forceinline__ void finish(u32x4& codes, uint32_t& s) const
    {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = top2(top, x[q][i]);
        s = scale_of(top_of_pair(top));
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[q] = encode8(x[q], s);
    }
};

// LDS of the few rows: `count` rows of `turns` x 16 blocks, rows 16 bytes longer against bank conflicts, then one byte
// of scale each, the four of a lane and turn in one word.
__host__ __device__ constexpr uint32_t few_pitch(uint32_t turns) { return turns * (kTurn * 16) + 16; }
// Behind them the many rows' scales, rows 16 bytes longer too.
__host__ __device__ constexpr uint32_t many_pitch(uint32_t turns) { return turns * kTurn + 16; }
__host__ __device__ constexpr uint32_t few_bytes(uint32_t count, uint32_t turns, uint32_t many)
{
    return count * (few_pitch(turns) + turns * kTurn) + many * many_pitch(turns);
}

// c[many][few] or c[few][many]: element (j, i) lies at j * step_many + i * step_few.
template <int NT, typename X, typename T>
__global__ __launch_bounds__(64 * kFewWaves) void mv_mx_product_few_kernel(Factor many, Few<X> few, uint32_t blocks, int64_t k,
                                                                           T* __restrict__ c, int64_t step_many, int64_t step_few)
{
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    const uint32_t in = lane & 15u, g = lane / 16;
    const int64_t j0 = (int64_t)blockIdx.x * (16 * NT);
    extern __shared__ __attribute__((aligned(16))) uint8_t held[];
    const uint32_t turns = (blocks + kTurn - 1) / kTurn, row_blocks = turns * kTurn, pitch = few_pitch(turns);
    uint8_t* held_scales = held + few.count * pitch;
    uint8_t* many_scales = held_scales + few.count * row_blocks;

    // Loads come back in their order, so what LDS gets is asked for first: the thread's first block of the few rows ...
    Block<X> mine;
    const uint32_t few_blocks = few.count * row_blocks;
    auto fetch = [&](uint32_t at) {
        const uint32_t row = at / row_blocks, block = at - row * row_blocks;
        if (at < few_blocks && block < blocks) mine.fetch(few, row, block, k);
    };
    auto hold = [&](uint32_t at) {
        const uint32_t row = at / row_blocks, block = at - row * row_blocks;
        u32x4 codes = {0u, 0u, 0u, 0u};
        uint32_t scale = 127;
        if (block < blocks) mine.finish(codes, scale);
        *reinterpret_cast<u32x4*>(held + row * pitch + block * 16) = codes;
        // block 4 s + g of a turn is byte s of word g
        held_scales[row * row_blocks + (block & ~15u) + (block & 3u) * 4 + (block >> 2 & 3u)] = (uint8_t)scale;
    };
    fetch(threadIdx.x);
    // ... and the many rows' scales, a word a thread; those behind the last block are 1
    const uint32_t row_words = row_blocks / 4, last_word = (blocks - 1) / 4;
    for (uint32_t at = threadIdx.x; at < 16 * NT * row_words; at += blockDim.x) {
        const uint32_t r = at / row_words, word = at - r * row_words;
        const int64_t j = j0 + r < many.rows ? j0 + r : many.rows - 1;
        uint32_t w = word <= last_word ? *reinterpret_cast<const uint32_t*>(many.scales + j * many.ld_scales + 4 * word) : 0x7F7F7F7Fu;
        const uint32_t live = blocks - 4 * word;
        if (word == last_word && live < 4) w = (w & ((1u << (8 * live)) - 1u)) | (0x7F7F7F7Fu & ~((1u << (8 * live)) - 1u));
        *reinterpret_cast<uint32_t*>(many_scales + r * many_pitch(turns) + 4 * word) = w;
    }
    // then the first turn's codes; what lies behind the last block is some block's, and meets zeros of the few rows
    const uint32_t* rows[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t j = j0 + 16 * t + in, row = j < many.rows ? j : many.rows - 1;
        rows[t] = many.codes + row * many.ld_words;
    }
    u32x4 codes[NT][4];
    auto load = [&](uint32_t block) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                codes[t][s] = *reinterpret_cast<const u32x4*>(rows[t] + 4 * (int64_t)min(block + 4 * s + g, blocks - 1));
    };
    uint32_t block = wave * kTurn;
    load(block);
    for (uint32_t at = threadIdx.x; at < few_blocks; at += blockDim.x) {
        if (at >= blockDim.x) fetch(at);
        hold(at);
    }
    __syncthreads();
    f32x4 acc[NT] = {};
    const uint32_t few_row = min(in, few.count - 1);
    while (block < blocks) {
        u32x4 x[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) x[s] = *reinterpret_cast<const u32x4*>(held + few_row * pitch + (block + 4 * s + g) * 16);
        const uint32_t xs = *reinterpret_cast<const uint32_t*>(held_scales + few_row * row_blocks + block + 4 * g);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const uint32_t ws =
                pick_scales(*reinterpret_cast<const u32x4*>(many_scales + (16 * t + in) * many_pitch(turns) + block), g);
            acc[t] = mfma<0>(codes[t][0], ws, x[0], xs, acc[t]);
            acc[t] = mfma<1>(codes[t][1], ws, x[1], xs, acc[t]);
            acc[t] = mfma<2>(codes[t][2], ws, x[2], xs, acc[t]);
            acc[t] = mfma<3>(codes[t][3], ws, x[3], xs, acc[t]);
        }
        block += waves * kTurn;
        if (block < blocks) load(block);
    }
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(held);                         // wavefront, tile, lane
#pragma unroll
    for (int t = 0; t < NT; ++t) sums[(wave * NT + t) * 64 + lane] = acc[t];
    __syncthreads();
    for (uint32_t at = threadIdx.x; at < NT * 64; at += blockDim.x) {
        f32x4 v = sums[at];
        for (uint32_t w = 1; w < waves; ++w) v += sums[w * NT * 64 + at];
        const uint32_t i = at & 15u;
        const int64_t j = j0 + at / 64 * 16 + (at >> 4 & 3u) * 4;
        if (i >= few.count) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (j + e < many.rows) put(c + (j + e) * step_many + i * step_few, v[e]);
    }
}

// How a product is cut: tiles of 64 `mt` rows of each factor (0: the kernel without LDS), and the steps of k over `splits`.
struct Cut {
    int      mt;
    int64_t  tiles_m, tiles_n;
    uint32_t splits, steps_each;
};
static Cut cut_of(int64_t m, int64_t n, int64_t k)
{
    auto tiles = [](int64_t rows, int mt) { return (rows + 64 * mt - 1) / (64 * mt); };
    Cut c = {4, tiles(m, 4), tiles(n, 4), 1, 0};
    const int64_t steps = (blocks_of(k) + kStepBlocks - 1) / kStepBlocks;
    if (c.tiles_m * c.tiles_n < 192) {
        c = {2, tiles(m, 2), tiles(n, 2), 1, 0};
        const int64_t most = 512 / (c.tiles_m * c.tiles_n);
        int64_t splits = most < steps / 4 ? most : steps / 4;
        if (splits > 16) splits = 16;
        if (splits > 1) c.splits = (uint32_t)splits;
    }
    c.steps_each = (uint32_t)((steps + c.splits - 1) / c.splits);
    c.splits = (uint32_t)((steps + c.steps_each - 1) / c.steps_each);
    return c;
}
inline int64_t quads_of(int64_t n) { return (n + 3) / 4; }
inline size_t parts_bytes(int64_t m, int64_t n, int64_t k)
{
    const Cut c = cut_of(m, n, k);
    return c.splits > 1 ? (size_t)c.splits * (size_t)m * (size_t)quads_of(n) * 16 : 0;
}

template <typename T>
static mv_status launch_product_of(const Factor& a, const Factor& b, int64_t k, T* c, int64_t ld_c, float* parts, hipStream_t st)
{
    const Cut cut = cut_of(a.rows, b.rows, k);
    const dim3 threads(256);
    if (cut.tiles_m * cut.tiles_n * cut.splits > kMostGroups) return MV_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)(cut.tiles_m * cut.tiles_n), cut.splits);
    const uint32_t blocks = (uint32_t)blocks_of(k), tm = (uint32_t)cut.tiles_m, tn = (uint32_t)cut.tiles_n;
    if (cut.mt == 4) {
        hipLaunchKernelGGL((mv_mx_product_tile_kernel<4, 2, 2, 4, T>), grid, dim3(512), 0, st, a, b, blocks, tm, tn, cut.steps_each, c, ld_c, 0);
    } else if (cut.splits == 1) {
        hipLaunchKernelGGL((mv_mx_product_tile_kernel<2, 2, 2, 2, T>), grid, threads, 0, st, a, b, blocks, tm, tn, cut.steps_each, c, ld_c, 0);
    } else {
        const int64_t quads = quads_of(b.rows), split_c = a.rows * quads * 4;
        hipLaunchKernelGGL((mv_mx_product_tile_kernel<2, 2, 2, 2, float>), grid, threads, 0, st, a, b, blocks, tm, tn, cut.steps_each, parts,
                           quads * 4, split_c);
        hipLaunchKernelGGL(mv_mx_product_join_kernel<T>, dim3((uint32_t)((a.rows * quads + 255) / 256)), threads, 0, st, parts,
                           (int)cut.splits, a.rows, b.rows, split_c, quads, c, ld_c);
    }
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

constexpr int64_t kFewRows = 16;
constexpr uint32_t kFewLds = 144 * 1024;
// Workgroups of the kernel for few rows read all of k: so many of its rows, or so short rows, and it is the faster one.
// Workgroups of 16 rows as long as all of them run at once, three to a unit; beyond that 32 rows, which share what a
// workgroup spends on the few rows.  Four bf16 rows against 8192 x 8192: 13.0 us with 16 and 13.4 with 32; 12,000 x 8192
// 15.9 and 17.5; 14,000 x 8192 19.5 and 18.0; 16,384 x 6000 18.8 and 14.7; 16,384 x 8192 28 and 19.9.
inline int few_tiles(int64_t many) { return many > 12288 ? 2 : 1; }
inline bool few_fits(int64_t few, int64_t many, int64_t k)
{
    const int64_t turns = (blocks_of(k) + kTurn - 1) / kTurn;
    return few <= kFewRows && (many >= 512 || k <= 8192) && turns < 4096 && few_bytes((uint32_t)few, (uint32_t)turns, 16u * (uint32_t)few_tiles(many)) <= kFewLds;
}

template <int NT, typename X, typename T>
static void launch_few_of(const Factor& many, const Few<X>& few, int64_t k, T* c, int64_t step_many, int64_t step_few, hipStream_t st)
{
    const uint32_t blocks = (uint32_t)blocks_of(k), turns = (blocks + kTurn - 1) / kTurn;
    const uint32_t waves = turns < kFewWaves ? turns : kFewWaves;
    const uint32_t room = few_bytes(few.count, turns, 16 * NT), sums = waves * NT * 1024;
    hipLaunchKernelGGL((mv_mx_product_few_kernel<NT, X, T>), dim3((uint32_t)((many.rows + 16 * NT - 1) / (16 * NT))),
                       dim3(64 * waves), room > sums ? room : sums, st, many, few, blocks, k, c, step_many, step_few);
}
template <typename X, typename T>
static mv_status launch_few(const Factor& many, const Few<X>& few, int64_t k, T* c, int64_t step_many, int64_t step_few, hipStream_t st)
{
    if (many.rows / 16 > kMostGroups / 2) return MV_ERR_INVALID_ARG;
    if (few_tiles(many.rows) == 2) launch_few_of<2>(many, few, k, c, step_many, step_few, st);
    else launch_few_of<1>(many, few, k, c, step_many, step_few, st);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}
template <typename T>
static mv_status launch_few_codes(const Factor& a, const Factor& b, int64_t k, T* c, int64_t ld_c, hipStream_t st)
{
    if (few_fits(a.rows, b.rows, k))
        return launch_few(b, Few<uint32_t>{a.codes, a.ld_words, a.scales, a.ld_scales, (uint32_t)a.rows}, k, c, 1, ld_c, st);
    return launch_few(a, Few<uint32_t>{b.codes, b.ld_words, b.scales, b.ld_scales, (uint32_t)b.rows}, k, c, ld_c, 1, st);
}

static mv_status launch_product(const Factor& a, const Factor& b, int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* parts,
                                hipStream_t st)
{
    if (few_fits(a.rows, b.rows, k) || few_fits(b.rows, a.rows, k))
        return c_dtype == MV_BF16 ? launch_few_codes(a, b, k, static_cast<uint16_t*>(c), ld_c, st)
                                  : launch_few_codes(a, b, k, static_cast<float*>(c), ld_c, st);
    // byte offsets inside a tile's rows are 32 bits
    if (a.ld_words * 4 > (1 << 22) || b.ld_words * 4 > (1 << 22)) {
        const int64_t tiles_m = (a.rows + 2 * kTile - 1) / (2 * kTile), tiles_n = (b.rows + 2 * kTile - 1) / (2 * kTile);
        if (tiles_m * tiles_n > kMostGroups) return MV_ERR_INVALID_ARG;
        const dim3 grid((uint32_t)(tiles_m * tiles_n)), threads(kProductThreads);
        if (c_dtype == MV_BF16)
            hipLaunchKernelGGL(mv_mx_product_kernel<uint16_t>, grid, threads, 0, st, a, b, blocks_of(k), tiles_n,
                               static_cast<uint16_t*>(c), ld_c);
        else
            hipLaunchKernelGGL(mv_mx_product_kernel<float>, grid, threads, 0, st, a, b, blocks_of(k), tiles_n, static_cast<float*>(c),
                               ld_c);
        return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
    }
    return c_dtype == MV_BF16 ? launch_product_of(a, b, k, static_cast<uint16_t*>(c), ld_c, static_cast<float*>(parts), st)
                              : launch_product_of(a, b, k, static_cast<float*>(c), ld_c, static_cast<float*>(parts), st);
}

inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }
inline size_t code_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)blocks_of(n) * 16); }
inline size_t scale_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)((blocks_of(n) + 3) / 4 * 4)); }

// A matrix of codes in the scratch, `at` moves behind it.
struct Held {
    uint32_t* codes;
    uint8_t*  scales;
    int64_t   ld_words, ld_scales, rows;
    Factor factor() const { return {codes, scales, ld_words, ld_scales, rows}; }
};
static Held carve(char*& at, int64_t rows, int64_t n)
{
    Held h = {reinterpret_cast<uint32_t*>(at), reinterpret_cast<uint8_t*>(at + code_bytes(rows, n)), 4 * blocks_of(n),
              (blocks_of(n) + 3) / 4 * 4, rows};
    at += code_bytes(rows, n) + scale_bytes(rows, n);
    return h;
}

inline bool scratch_valid(const void* p, size_t have, size_t need)
{
    return need == 0 || (p && have >= need && (reinterpret_cast<uintptr_t>(p) & 15) == 0);
}

}  // namespace mvx

extern "C" {

size_t mv_mx_product_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    return size_valid(m) && size_valid(n) && size_valid(k) ? parts_bytes(m, n, k) : 0;
}

mv_status mv_mx_product(const uint32_t* a_codes, int64_t ld_aw, const uint8_t* a_scales, int64_t ld_as,
                        const uint32_t* b_codes, int64_t ld_bw, const uint8_t* b_scales, int64_t ld_bs, int64_t m, int64_t n,
                        int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k) || !codes_valid(a_codes, ld_aw, a_scales, ld_as, k) ||
        !codes_valid(b_codes, ld_bw, b_scales, ld_bs, k) || !values_valid(c, c_dtype, ld_c, n) ||
        !scratch_valid(scratch, scratch_bytes, mv_mx_product_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    return launch_product({a_codes, a_scales, ld_aw, ld_as, m}, {b_codes, b_scales, ld_bw, ld_bs, n}, k, c, c_dtype, ld_c,
                          scratch, static_cast<hipStream_t>(stream));
}

size_t mv_mx_linear_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k)) return 0;
    return code_bytes(m, k) + scale_bytes(m, k) + parts_bytes(m, n, k);
}

mv_status mv_mx_linear(const void* x, int32_t x_dtype, int64_t ld_x, const uint32_t* w_codes, int64_t ld_words,
                       const uint8_t* w_scales, int64_t ld_scales, int64_t m, int64_t n, int64_t k, void* y, int32_t y_dtype,
                       int64_t ld_y, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k) || !values_valid(x, x_dtype, ld_x, k) ||
        !codes_valid(w_codes, ld_words, w_scales, ld_scales, k) || !values_valid(y, y_dtype, ld_y, n) ||
        !scratch_valid(scratch, scratch_bytes, mv_mx_linear_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (few_fits(m, n, k)) {
        const Factor w = {w_codes, w_scales, ld_words, ld_scales, n};
        if (x_dtype == MV_BF16) {
            const Few<uint16_t> f = {static_cast<const uint16_t*>(x), ld_x, nullptr, 0, (uint32_t)m};
            return y_dtype == MV_BF16 ? launch_few(w, f, k, static_cast<uint16_t*>(y), 1, ld_y, st)
                                      : launch_few(w, f, k, static_cast<float*>(y), 1, ld_y, st);
        }
        const Few<float> f = {static_cast<const float*>(x), ld_x, nullptr, 0, (uint32_t)m};
        return y_dtype == MV_BF16 ? launch_few(w, f, k, static_cast<uint16_t*>(y), 1, ld_y, st)
                                  : launch_few(w, f, k, static_cast<float*>(y), 1, ld_y, st);
    }
    char* at = static_cast<char*>(scratch);
    const Held q = carve(at, m, k);
    if (const mv_status rc = launch_encode(x, x_dtype, ld_x, m, k, q.codes, q.ld_words, q.scales, q.ld_scales, nullptr, 0, st))
        return rc;
    return launch_product(q.factor(), {w_codes, w_scales, ld_words, ld_scales, n}, k, y, y_dtype, ld_y, at, st);
}

size_t mv_mx_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k)) return 0;
    const size_t dx = code_bytes(m, n) + scale_bytes(m, n), dw = code_bytes(n, m) + scale_bytes(n, m) + code_bytes(k, m) + scale_bytes(k, m);
    const size_t dx_parts = parts_bytes(m, k, n), dw_parts = parts_bytes(n, k, m);
    return dx + dw + (dx_parts > dw_parts ? dx_parts : dw_parts);
}

mv_status mv_mx_linear_grad(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype,
                            const uint32_t* wt_codes, int64_t ld_words, const uint8_t* wt_scales, int64_t ld_scales,
                            int64_t m, int64_t n, int64_t k, void* dx, int32_t dx_dtype, int64_t ld_dx, void* dw,
                            int32_t dw_dtype, int64_t ld_dw, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k) || !values_valid(dy, dtype, ld_dy, n) || (!dx && !dw) ||
        !scratch_valid(scratch, scratch_bytes, mv_mx_linear_grad_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    if (dx && (!codes_valid(wt_codes, ld_words, wt_scales, ld_scales, n) || !values_valid(dx, dx_dtype, ld_dx, k)))
        return MV_ERR_INVALID_ARG;
    if (dw && (!values_valid(x, dtype, ld_x, k) || !values_valid(dw, dw_dtype, ld_dw, k))) return MV_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* at = static_cast<char*>(scratch);
    // the two products' parts take one place, behind all codes
    char* parts = at + code_bytes(m, n) + scale_bytes(m, n) + code_bytes(n, m) + scale_bytes(n, m) + code_bytes(k, m) + scale_bytes(k, m);
    if (dx) {
        const Held q = carve(at, m, n);
        if (const mv_status rc = launch_encode(dy, dtype, ld_dy, m, n, q.codes, q.ld_words, q.scales, q.ld_scales, nullptr, 0, st))
            return rc;
        if (const mv_status rc = launch_product(q.factor(), {wt_codes, wt_scales, ld_words, ld_scales, k}, n, dx, dx_dtype, ld_dx, parts, st))
            return rc;
    }
    if (dw) {
        const Held p = carve(at, n, m), q = carve(at, k, m);
        if (const mv_status rc = launch_encode_t(dy, dtype, ld_dy, m, n, p.codes, p.ld_words, p.scales, p.ld_scales, st)) return rc;
        if (const mv_status rc = launch_encode_t(x, dtype, ld_x, m, k, q.codes, q.ld_words, q.scales, q.ld_scales, st)) return rc;
        return launch_product(p.factor(), q.factor(), m, dw, dw_dtype, ld_dw, parts, st);
    }
    return MV_OK;
}

}  // extern "C"
