// Products of microscaled 4-bit matrices (mv_mx_product, mv_mx_linear, mv_mx_linear_grad of include/mv.h).
//
//   c[i][j] = sum_k a[i][k] b[j][k],  both factors in blocks of 32 along k
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of each factor times four blocks: lane l holds row l % 16 of a
// block, 16 bytes of codes, and the block's scale in one byte of a register; which blocks of k the four groups of lanes
// hold does not matter as long as both factors agree.  So a group takes four consecutive blocks of each 16: 64
// consecutive bytes of codes for four instructions, and their four scales in one word.
#include "mv_mx.hpp"
#include "mv_product.hpp"

#include <type_traits>

namespace mvx {

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

constexpr int kTile = 64;           // rows of each factor that a wavefront takes
constexpr int kProductThreads = 256;

__global__ __launch_bounds__(kProductThreads) void mv_mx_product_kernel(Factor a, Factor b, int64_t blocks, int64_t tiles_n, Out c,
                                                                        int64_t ld_c)
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
            c.put4(i * ld_c + j, b.rows - j, acc[t][u]);
        }
    }
}

// ---- tiles through LDS ---------------------------------------------------------------------------------------------
//
// A workgroup of WM x WN wavefronts takes 32 MT WM x 32 NT WN results, 32 MT x 32 NT a wavefront, in steps of eight
// blocks (256 values, 128 bytes a row).  The rows of both factors go from memory straight into LDS, each row's
// 16-byte blocks in the order block ^ (row % 8): what eight lanes of neighbouring rows read together lies in
// different banks, and what eight lanes write together is one whole line of memory.  Two buffers: the next step's
// loads are in flight during this one's products.  With few steps, one buffer, and the unit's other workgroups fill
// the waiting.  Loads beyond the last row or block return zeros by the buffer's bounds.  The scales of two steps, 16
// bytes a row, go through registers, where those behind the last block become 1, into LDS of their own.
//
// A lane of the 32 x 32 x 64 instruction holds half of a row's eight blocks: blocks 4 (lane / 32) + s of step s, whose
// scales are one word.
// 4096 x 8192 by 8192, bf16 results: 139 us on a cool card to 150, 4.0 to 3.7 PFLOP/s.  The instructions alone, out of
// registers, reach 8.4 on small numbers and 6.2 to 6.7 on random codes, where power bounds them; the rest is the codes' way
// into LDS beside them (without it 111), the reads from there and the end, where 67 MB leave.  With 512 values of k the results are all: 4900 x 512 by 4608 to fp32 26 us with the launch
// that quantises (4), a fill of those 90 MB 15.5.

constexpr int kStepBlocks = 8;
constexpr int kScalePitch = 20;     // bytes between the rows' scales in LDS: 16 and a word against bank conflicts

template <int S>
__device__ __forceinline__ f32x16 mfma32(const u32x4& a, uint32_t a_scale, const u32x4& b, uint32_t b_scale, f32x16 c)
{
    const i32x8 x = {(int)a.x, (int)a.y, (int)a.z, (int)a.w, 0, 0, 0, 0}, y = {(int)b.x, (int)b.y, (int)b.z, (int)b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, S, (int)a_scale, S, (int)b_scale);
}

// One product and how it is cut: tiles_m x tiles_n tiles, `splits` runs of steps_each steps each.  With several splits c is
// fp32 and holds their sums one after the other, split_c apart.
struct Product {
    Factor   a, b;
    uint32_t blocks, tiles_m, tiles_n, steps_each, splits;
    Out      c;
    int64_t  ld_c, split_c;
    uint32_t past;                  // store past the caches
};

// A wavefront's share of one instruction's blocks: rows of a and of b.
template <int MT, int NT>
struct Rows {
    u32x4 x[MT], y[NT];
};

template <int MT, int NT, int WM, int WN, int BUFFERS, bool PAIR>
__global__ __launch_bounds__(64 * WM * WN, BUFFERS == 1 ? 3 : 2) void mv_mx_product_tile_kernel(Launch<Product, PAIR> l)
{
    constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    constexpr int kM = 32 * MT * WM, kN = 32 * NT * WN, kRows = kM + kN;
    typedef uint8_t Codes[kRows * 128];
    __shared__ __attribute__((aligned(1024))) Codes even;
    __shared__ uint8_t scales[BUFFERS][kRows * kScalePitch];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t / 64);
    const Product& p = l.product();
    const Factor a = p.a, b = p.b;
    const uint32_t blocks = p.blocks, steps_each = p.steps_each, id = l.id();
    const uint32_t split = id / (p.tiles_m * p.tiles_n);
    uint32_t tm, tn;
    tile_of(id - split * (p.tiles_m * p.tiles_n), p.tiles_m, p.tiles_n, tm, tn);
    const int64_t i0 = (int64_t)tm * kM, j0 = (int64_t)tn * kN;
    const uint32_t steps = (blocks + kStepBlocks - 1) / kStepBlocks;
    const uint32_t step0 = split * steps_each, count = min(steps_each, steps - step0);       // at least one
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
        // The whole offset is the lane's own, for the bounds to hold: beyond every buffer where the row has no such block.
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
    // A thread has one row's scales, of a the first wavefronts, of b the others: one load for two steps, which reads zeros
    // where the rows end, and the next row's behind a row's last block.
    static_assert(kThreads == kRows, "a row a thread");
    const bool of_a = wave < kM / 64;
    const uint32_t sc_pitch = (uint32_t)(of_a ? a.ld_scales : b.ld_scales), sc_rows = (uint32_t)(of_a ? a_rows : b_rows);
    const __amdgpu_buffer_rsrc_t sc_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(of_a ? a.scales + i0 * a.ld_scales : b.scales + j0 * b.ld_scales), 0,
        (int)((sc_rows - 1) * sc_pitch + (blocks + 3) / 4 * 4), 0x00020000);
    const uint32_t sc_at = (t - (of_a ? 0u : (uint32_t)kM)) * sc_pitch;
    u32x4 next;
    auto fetch_scales = [&](uint32_t k) {
        next = __builtin_amdgcn_raw_buffer_load_b128(sc_buf, sc_at + (step0 + k) * kStepBlocks, 0, 0);
    };
    auto keep_scales = [&](uint32_t pair) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int live = (int)end - (int)((step0 + 2 * pair) * kStepBlocks + 4 * w);
            const uint32_t real = live >= 4 ? 0xFFFFFFFFu : live > 0 ? (1u << (8 * live)) - 1u : 0u;
            *reinterpret_cast<uint32_t*>(&scales[pair % BUFFERS][t * kScalePitch + 4 * w]) = (next[w] & real) | (0x7F7F7F7Fu & ~real);
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
        const uint8_t* sc = scales[k / 2 % BUFFERS] + (k & 1u) * 8 + half * 4;
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
    if constexpr (BUFFERS == 1) {
        for (uint32_t k = 0; k < count; ++k) {
            load_codes(k, even);
            if (k % 2 == 0) {
                fetch_scales(k);
                keep_scales(k / 2);
            }
            all_here();
            read_rows(even, 0, one);
            read_scales(k);
            most_of_step(even);
            last_of_step();
            __syncthreads();
        }
    } else {
        // two variables, not an array of two: reads of one need not wait for the loads into the other
        __shared__ __attribute__((aligned(1024))) Codes odd;
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
    }

    // A lane has, of 32 rows, four times four consecutive columns.  32 rows of the wavefront's 64 columns at a time go
    // through its part of LDS, 16-byte units in the order unit ^ (row % 16), and out in whole runs of a row.
    static_assert(NT == 2 && kWaves * 8192 <= sizeof(Codes), "a wavefront's 32 x 64 results");
    float* mine = reinterpret_cast<float*>(even + wave * 8192);
    const int64_t col0 = j0 + wave % WN * 64, out = split * p.split_c;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<f32x4*>(mine + in * 64 + ((8 * j + 2 * q + half) ^ (in & 15u)) * 4) =
                    f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        const int64_t row0 = i0 + wave / WN * (32 * MT) + 32 * i;
        if (p.c.bf16) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t r = 8 * u + lane / 8, unit = lane % 8 * 2;
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + r * 64 + (unit ^ (r & 15u)) * 4);
                const f32x4 y = *reinterpret_cast<const f32x4*>(mine + r * 64 + ((unit + 1) ^ (r & 15u)) * 4);
                const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                const int64_t col = col0 + 4 * unit;
                if (row0 + r < a.rows) store8(static_cast<uint16_t*>(p.c.p) + out + (row0 + r) * p.ld_c + col, b.rows - col, v, p.past);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t r = 4 * u + lane / 16, unit = lane % 16;
                const f32x4 x = *reinterpret_cast<const f32x4*>(mine + r * 64 + (unit ^ (r & 15u)) * 4);
                const float v[4] = {x.x, x.y, x.z, x.w};
                const int64_t col = col0 + 4 * unit;
                if (row0 + r < a.rows) store4(static_cast<float*>(p.c.p) + out + (row0 + r) * p.ld_c + col, b.rows - col, v, p.past);
            }
        }
    }
}

__global__ __launch_bounds__(256) void mv_mx_product_join_kernel(const float* __restrict__ parts, uint32_t splits, uint32_t lanes,
                                                                 int64_t m, int64_t n, int64_t split_c, int64_t quads, Out c,
                                                                 int64_t ld_c)
{
    join_splits(blockIdx.x, parts, splits, lanes, m, n, split_c, quads, c, ld_c);
}

// ---- few rows of one factor ------------------------------------------------------------------------------------------
//
// Up to 16 rows of one factor ("few"; up to 64 where they are values) against many of the other ("many"), whose
// codes are the bytes to read.  A workgroup takes 16 NT of the many rows and all of k, its wavefronts turns of 16
// blocks; what they have is added up through LDS in the wavefronts' order.  Lane l of an instruction holds row l %
// 16 and block 4 s + l / 16 of the turn, s = 0 .. 3: the four lanes of a row read 64 bytes in a row; the scales of a
// lane's four blocks are picked from the row's 16. The few rows' codes and scales are in LDS: copied there, or
// quantised by every workgroup for itself, a lane a block, while the first turn's codes are on their way.
// Loads in flight are what it lives on: codes of two turns are asked for before the first are needed, behind what LDS gets.
// 5 x 8192 bf16 by 16,384: 18.0 us for 71.5 MB, 4.0 TB/s (one turn, and the scales one word after the other, 19.8); 4 x 8192 by
// 8192 10.4 (12.6).  1 x 2048 by 1000 3.9, which is a launch.

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
        const float* p = f.rows + row * f.ld + (int64_t)block * kBlock;
        const int64_t live = k - (int64_t)block * kBlock;
        if (live >= kBlock) {
#pragma unroll
            for (int q = 0; q < 4; ++q) load8(p + 8 * q, 8, x[q]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) load8(p + 8 * q, live - 8 * q, x[q]);
        }
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
        if (live >= kBlock) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const u32x4u v = *reinterpret_cast<const u32x4u*>(p + 8 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[q][i] = v[i];
            }
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
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
template <typename X>
struct FewProduct {
    Factor   many;
    Few<X>   few;
    uint32_t blocks;
    int64_t  k;
    Out      c;
    int64_t  step_many, step_few;
};

// A workgroup: 16 MT few rows, 16 NT of the many.
template <int MT, int NT, typename X, bool PAIR>
__global__ __launch_bounds__(64 * kFewWaves) void mv_mx_product_few_kernel(Launch<FewProduct<X>, PAIR> l)
{
    const FewProduct<X>& p = l.product();
    const uint32_t id = l.id();
    const Factor many = p.many;
    const Few<X> few = p.few;
    const uint32_t blocks = p.blocks;
    const int64_t k = p.k, j0 = (int64_t)id * (16 * NT);
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    const uint32_t in = lane & 15u, g = lane / 16;
    extern __shared__ __attribute__((aligned(16))) uint8_t held[];
    const uint32_t turns = (blocks + kTurn - 1) / kTurn, row_blocks = turns * kTurn, pitch = few_pitch(turns);
    uint8_t* held_scales = held + few.count * pitch;
    uint8_t* many_scales = held_scales + few.count * row_blocks;

    // Loads come back in their order, so all that goes into LDS is asked for first, several pieces of a thread at once: the
    // few rows' blocks ...
    constexpr uint32_t kFirst = 2;
    Block<X> mine[kFirst];
    const uint32_t few_blocks = few.count * row_blocks;
    auto fetch = [&](uint32_t at, Block<X>& b) {
        const uint32_t row = at / row_blocks, block = at - row * row_blocks;
        if (at < few_blocks && block < blocks) b.fetch(few, row, block, k);
    };
    auto hold = [&](uint32_t at, const Block<X>& b) {
        if (at >= few_blocks) return;
        const uint32_t row = at / row_blocks, block = at - row * row_blocks;
        u32x4 codes = {0u, 0u, 0u, 0u};
        uint32_t scale = 127;
        if (block < blocks) b.finish(codes, scale);
        *reinterpret_cast<u32x4*>(held + row * pitch + block * 16) = codes;
        // block 4 s + g of a turn is byte s of word g
        held_scales[row * row_blocks + (block & ~15u) + (block & 3u) * 4 + (block >> 2 & 3u)] = (uint8_t)scale;
    };
    // ... and the many rows' scales, a turn's 16; those behind the last block are 1
    const uint32_t many_turns = 16 * NT * turns, last_word = (blocks - 1) / 4;
    auto fetch_scales = [&](uint32_t at, u32x4& w) {
        const uint32_t r = at / turns, word = (at - r * turns) * 4;
        const int64_t j = j0 + r < many.rows ? j0 + r : many.rows - 1;
        const uint32_t* from = reinterpret_cast<const uint32_t*>(many.scales + j * many.ld_scales) + word;
        if (at >= many_turns) return;
        if (word + 3 <= last_word) {
            w = *reinterpret_cast<const u32x4u*>(from);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 4; ++i) w[i] = word + i <= last_word ? from[i] : 0u;
        }
    };
    auto hold_scales = [&](uint32_t at, u32x4 w) {
        if (at >= many_turns) return;
        const uint32_t r = at / turns, word = (at - r * turns) * 4;
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const int live = (int)blocks - 4 * (int)(word + i);
            const uint32_t real = live >= 4 ? 0xFFFFFFFFu : live > 0 ? (1u << (8 * live)) - 1u : 0u;
            w[i] = (w[i] & real) | (0x7F7F7F7Fu & ~real);
        }
        *reinterpret_cast<u32x4*>(many_scales + r * many_pitch(turns) + 4 * word) = w;
    };
    u32x4 my_scales;
#pragma unroll
    for (uint32_t i = 0; i < kFirst; ++i) fetch(threadIdx.x + i * blockDim.x, mine[i]);
    fetch_scales(threadIdx.x, my_scales);
    // then codes, of two turns; what lies behind the last block is some block's, and meets zeros of the few rows
    const uint32_t* rows[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t j = j0 + 16 * t + in, row = j < many.rows ? j : many.rows - 1;
        rows[t] = many.codes + row * many.ld_words;
    }
    typedef u32x4 Codes[NT][4];
    Codes one, two;
    auto load = [&](uint32_t block, Codes& codes) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int s = 0; s < 4; ++s)
                codes[t][s] = *reinterpret_cast<const u32x4*>(rows[t] + 4 * (int64_t)min(block + 4 * s + g, blocks - 1));
    };
    const uint32_t step = waves * kTurn;
    uint32_t block = wave * kTurn;
    load(block, one);
#pragma unroll
    for (uint32_t i = 0; i < kFirst; ++i) hold(threadIdx.x + i * blockDim.x, mine[i]);
    hold_scales(threadIdx.x, my_scales);
    if (block + step < blocks) load(block + step, two);
    for (uint32_t at = threadIdx.x + kFirst * blockDim.x; at < few_blocks; at += kFirst * blockDim.x) {
#pragma unroll
        for (uint32_t i = 0; i < kFirst; ++i) fetch(at + i * blockDim.x, mine[i]);
#pragma unroll
        for (uint32_t i = 0; i < kFirst; ++i) hold(at + i * blockDim.x, mine[i]);
    }
    for (uint32_t at = threadIdx.x + blockDim.x; at < many_turns; at += blockDim.x) {
        fetch_scales(at, my_scales);
        hold_scales(at, my_scales);
    }
    __syncthreads();
    f32x4 acc[MT][NT] = {};
    auto turn = [&](const Codes& codes) {
        uint32_t ws[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
            ws[t] = pick_scales(*reinterpret_cast<const u32x4*>(many_scales + (16 * t + in) * many_pitch(turns) + block), g);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const uint32_t row = min(16 * i + in, few.count - 1);
            u32x4 x[4];
#pragma unroll
            for (int s = 0; s < 4; ++s) x[s] = *reinterpret_cast<const u32x4*>(held + row * pitch + (block + 4 * s + g) * 16);
            const uint32_t xs = *reinterpret_cast<const uint32_t*>(held_scales + row * row_blocks + block + 4 * g);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                acc[i][t] = mfma<0>(codes[t][0], ws[t], x[0], xs, acc[i][t]);
                acc[i][t] = mfma<1>(codes[t][1], ws[t], x[1], xs, acc[i][t]);
                acc[i][t] = mfma<2>(codes[t][2], ws[t], x[2], xs, acc[i][t]);
                acc[i][t] = mfma<3>(codes[t][3], ws[t], x[3], xs, acc[i][t]);
            }
        }
    };
    while (block < blocks) {
        turn(one);
        if (block + 2 * step < blocks) load(block + 2 * step, one);
        block += step;
        if (block >= blocks) break;
        turn(two);
        if (block + 2 * step < blocks) load(block + 2 * step, two);
        block += step;
    }
    __syncthreads();
    f32x4* sums = reinterpret_cast<f32x4*>(held);                         // wavefront, tile, lane
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t) sums[((wave * MT + i) * NT + t) * 64 + lane] = acc[i][t];
    __syncthreads();
    for (uint32_t at = threadIdx.x; at < MT * NT * 64; at += blockDim.x) {
        f32x4 v = sums[at];
        for (uint32_t w = 1; w < waves; ++w) v += sums[w * MT * NT * 64 + at];
        const uint32_t i = at / (64 * NT) * 16 + (at & 15u);
        const int64_t j = j0 + at / 64 % NT * 16 + (at >> 4 & 3u) * 4, to = j * p.step_many + i * p.step_few;
        if (i >= few.count) continue;
        if (p.step_many == 1) {
            if (j < many.rows) p.c.put4(to, many.rows - j, v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < many.rows) p.c.put(to + e * p.step_many, v[e]);
        }
    }
}

constexpr int64_t  kFewRows = 16, kFewValues = 64;
constexpr uint32_t kFewLds = 144 * 1024;

// Whether and how the kernel for few rows takes a product.  Up to 16 rows of codes it always is the faster one.  Of values it
// takes up to 64, as long as each unit quantises them once, and saves the launch that quantises them: bf16, 64 rows with
// 4096 x 1024 7.4 us (two launches 9.0), 20 rows with 4000 x 2048 6.0 (11.1), 5 with 16,384 x 8192 18.1 (18.6), 1 with 8192 x
// 8192 9.4 (11.3); but 16,000 x 256, a thousand workgroups, 16.8 (7.9), and 200 rows in four tiles with 1000 x 1000 11.6 (9.2).
// What all workgroups quantise together is bounded, too, fp32 at a third of bf16: 16 rows bf16 with 16,384 x 4096, 33 M values,
// 14.9 us (13.8), 12 with 12,000 x 8192, 74 M, 21.9 (17.0); fp32 8 with 4096 x 4096, 8 M, 8.5 (6.5, but a launch costs the host
// 3 more), 4 with 8192 x 8192, 17 M, 15.4 (11.5), 16 with 14,000 x 8192, 57 M, 44 (20).
constexpr int64_t kQuantisedBf16 = 36000000, kQuantisedF32 = 12000000;
struct FewCut {
    int      mt, nt;                // 0: it does not
    uint32_t groups, lds, waves;
};
static FewCut few_cut(int64_t few, int64_t many, int64_t k, int64_t quantised)     // most values to quantise; 0: codes
{
    const bool values = quantised > 0;
    if (few > (values ? kFewValues : kFewRows)) return FewCut{};
    const int64_t turns = (blocks_of(k) + kTurn - 1) / kTurn;
    FewCut c = {};
    c.mt = few <= 16 ? 1 : few <= 32 ? 2 : 4;
    // Workgroups of 16 rows as long as all of them run at once, three to a unit; beyond that 32 rows, which share what a
    // workgroup spends on the few rows.  bf16 us with 16 and with 32: four rows against 8192 x 8192 10.5, 10.4; 10,000 x 8192
    // 13.0, 15.5; 12,000 x 8192 13.9, 15.8; 14,000 x 8192 16.6, 16.5; 16,384 x 8192 17.4, 17.6; 16,384 x 6000 16.8, 15.9; five
    // fp32 rows 16,384 x 8192 30, 24; sixteen bf16 rows 16,384 x 4096 18.3, 14.7.
    c.nt = c.mt == 1 && many > 12288 ? 2 : 1;
    const int64_t groups = (many + 16 * c.nt - 1) / (16 * c.nt);
    if (turns >= 4096 || groups > kMostGroups / 4 || (values && groups * few * k > quantised)) return FewCut{};
    c.groups = (uint32_t)groups;
    // a wavefront for each turn, or for each 64 blocks of the few rows
    const int64_t waves = few > 4 ? few * turns / 4 + 1 : turns;
    c.waves = (uint32_t)(waves < kFewWaves ? waves : kFewWaves);
    const uint32_t sums = c.waves * c.mt * c.nt * 1024;
    c.lds = few_bytes((uint32_t)few, (uint32_t)turns, 16u * c.nt);
    if (c.lds < sums) c.lds = sums;
    if (few <= kFewRows ? (many < 512 && k > 8192) || c.lds > kFewLds : c.groups > 256 || c.lds > kFewLds) return FewCut{};
    return c;
}

template <typename X>
static FewProduct<X> few_product(const Factor& many, const Few<X>& few, int64_t k, const Out& c, int64_t step_many,
                                 int64_t step_few)
{
    return {many, few, (uint32_t)blocks_of(k), k, c, step_many, step_few};
}
// One product, or two whose cuts have the same mt and nt.
template <int MT, int NT, typename X>
static void launch_few_of(const FewProduct<X>* p, const FewCut* cut, int n, hipStream_t st)
{
    const dim3 threads(64 * (n == 2 && cut[1].waves > cut[0].waves ? cut[1].waves : cut[0].waves));
    const uint32_t lds = n == 2 && cut[1].lds > cut[0].lds ? cut[1].lds : cut[0].lds;
    if constexpr (std::is_same_v<X, uint32_t>) {
        if (n == 2) {
            hipLaunchKernelGGL((mv_mx_product_few_kernel<MT, NT, X, true>), dim3(cut[0].groups + cut[1].groups), threads, lds, st,
                               Launch<FewProduct<X>, true>{{p[0], p[1]}, cut[0].groups});
            return;
        }
    }
    hipLaunchKernelGGL((mv_mx_product_few_kernel<MT, NT, X, false>), dim3(cut[0].groups), threads, lds, st,
                       Launch<FewProduct<X>, false>{{p[0]}, cut[0].groups});
}
template <typename X>
static mv_status launch_few(const FewProduct<X>* p, const FewCut* cut, int n, hipStream_t st)
{
    if (cut[0].nt == 2) launch_few_of<1, 2>(p, cut, n, st);
    else if (cut[0].mt == 1) launch_few_of<1, 1>(p, cut, n, st);
    else if constexpr (!std::is_same_v<X, uint32_t>) {                   // codes: up to 16 rows only
        if (cut[0].mt == 2) launch_few_of<2, 1>(p, cut, n, st);
        else launch_few_of<4, 1>(p, cut, n, st);
    }
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

// How a product is cut for the kernel with tiles of 64 mt rows of each factor.
struct Cut {
    int      mt;
    int64_t  tiles_m, tiles_n;
    uint32_t splits, steps_each;
    int64_t  groups() const { return tiles_m * tiles_n * splits; }
};
// How many runs the steps are split into, where `beside` tiles of another product share the launch.
static constexpr int64_t splits_of(int64_t tiles, int64_t steps, int64_t results, int64_t beside)
{
    int64_t splits = 512 / tiles < steps / 4 ? 512 / tiles : steps / 4;
    // many splits only of small results: all of them are written and read again
    if (splits > 16 && splits * results > (4 << 20)) splits = 16;
    // never more than alone, which is what the scratch has room for
    if (beside && splits > 512 / (tiles + beside)) splits = 512 / (tiles + beside);
    return splits > 1 ? splits : 1;
}
static_assert(splits_of(4, 512, 200 * 200, 0) == 16 && splits_of(4, 512, 200 * 200, 4) == 16, "the limit of 16 holds in company, too");
static Cut cut_of(int64_t m, int64_t n, int64_t k, int mt, int64_t beside = 0)
{
    auto tiles = [mt](int64_t rows) { return (rows + 64 * mt - 1) / (64 * mt); };
    Cut c = {mt, tiles(m), tiles(n), 1, 0};
    const int64_t steps = (blocks_of(k) + kStepBlocks - 1) / kStepBlocks;
    if (mt == 2) c.splits = (uint32_t)splits_of(c.tiles_m * c.tiles_n, steps, m * n, beside);
    c.steps_each = (uint32_t)((steps + c.splits - 1) / c.splits);
    c.splits = (uint32_t)((steps + c.steps_each - 1) / c.steps_each);
    return c;
}
// Up to four steps and more tiles of 128 x 128 than units: one buffer and three workgroups a unit, of which one loads or
// stores while another multiplies.  bf16, with the launch that quantises, before -> with: 4900 x 256 by 4608 24.8 -> 17.0 us,
// x 512 25.4 -> 20.8, x 1024 32.3 -> 27.6, x 2048 44.5 here; 4096 x 1024 by 8192 35.5 : 35.6, x 2048 56.0 : 60.2; 2500 x 512 by
// 2500, 400 tiles, 12.5 -> 11.8; 2000 x 512 by 2000, 256 tiles, 10.1 : 10.4.
constexpr int64_t kFewSteps = 4, kUnits = 256;
inline bool few_steps(int64_t k) { return blocks_of(k) <= kFewSteps * kStepBlocks; }
static bool large(int64_t m, int64_t n) { return ((m + 255) / 256) * ((n + 255) / 256) >= 192; }
inline size_t parts_bytes(int64_t m, int64_t n, int64_t k)
{
    const uint32_t splits = cut_of(m, n, k, 2).splits;
    return splits > 1 ? up256((size_t)splits * (size_t)m * (size_t)quads_of(n) * 16) : 0;
}

// A product that is asked for: c = a b^T, m rows and n rows of k values.
struct Wanted {
    Factor  a, b;
    int64_t k;
    Out     c;
    int64_t ld_c;
    void*   parts;                  // room for parts_bytes
};
static Product product_of(const Wanted& w, const Cut& cut)
{
    const int64_t quads = quads_of(w.b.rows);
    const bool split = cut.splits > 1;
    return {w.a, w.b, (uint32_t)blocks_of(w.k), (uint32_t)cut.tiles_m, (uint32_t)cut.tiles_n, cut.steps_each, cut.splits,
            split ? Out{w.parts, 0} : w.c, split ? quads * 4 : w.ld_c, w.a.rows * quads * 4,
            w.a.rows * w.b.rows * (split ? 4 * (int64_t)cut.splits : w.c.bf16 ? 2 : 4) >= kPastBytes};
}
static void launch_join(const Wanted& w, const Cut& cut, hipStream_t st)
{
    if (cut.splits == 1) return;
    const int64_t quads = quads_of(w.b.rows), all = w.a.rows * quads;
    const uint32_t lanes = cut.splits > 16 ? 16 : 1, per = 256 / lanes;
    hipLaunchKernelGGL(mv_mx_product_join_kernel, dim3((uint32_t)((all + per - 1) / per)), dim3(256), 0, st,
                       static_cast<const float*>(w.parts), cut.splits, lanes, w.a.rows, w.b.rows, all * 4, quads, w.c, w.ld_c);
}
// The kernel without LDS, for rows so long that a tile's byte offsets leave 32 bits.
static mv_status launch_plain(const Wanted& w, hipStream_t st)
{
    const int64_t tiles_m = (w.a.rows + 2 * kTile - 1) / (2 * kTile), tiles_n = (w.b.rows + 2 * kTile - 1) / (2 * kTile);
    if (tiles_m * tiles_n > kMostGroups) return MV_ERR_INVALID_ARG;
    hipLaunchKernelGGL(mv_mx_product_kernel, dim3((uint32_t)(tiles_m * tiles_n)), dim3(kProductThreads), 0, st, w.a, w.b,
                       blocks_of(w.k), tiles_n, w.c, w.ld_c);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

// The kernel for few rows on codes: which factor's rows are the few ones.
static FewCut few_codes_cut(const Wanted& w, bool& few_a)
{
    few_a = w.a.rows <= w.b.rows;
    FewCut c = few_a ? few_cut(w.a.rows, w.b.rows, w.k, 0) : few_cut(w.b.rows, w.a.rows, w.k, 0);
    if (!c.mt) {
        few_a = !few_a;
        c = few_a ? few_cut(w.a.rows, w.b.rows, w.k, 0) : few_cut(w.b.rows, w.a.rows, w.k, 0);
    }
    return c;
}
static FewProduct<uint32_t> few_codes(const Wanted& w, bool few_a)
{
    const Factor& few = few_a ? w.a : w.b;
    return few_product(few_a ? w.b : w.a, Few<uint32_t>{few.codes, few.ld_words, few.scales, few.ld_scales, (uint32_t)few.rows}, w.k, w.c,
                       few_a ? 1 : w.ld_c, few_a ? w.ld_c : 1);
}
// Whether a tile's byte offsets fit 32 bits: those of rows that there are stay below 2^31, where the loads of blocks that there
// are not begin, and those of all rows of a tile below 2^32.
static bool offsets_fit(const Factor& f, int64_t blocks, int mt)
{
    const int64_t pitch = f.ld_words * 4, rows = f.rows < 64 * mt ? f.rows : 64 * mt;
    return pitch <= ((int64_t)1 << (mt == 4 ? 23 : 24)) && (rows - 1) * pitch + blocks * 16 <= ((int64_t)1 << 31) - 256 &&
           f.ld_scales <= (1 << 22);
}
static bool offsets_fit(const Wanted& w, int mt) { return offsets_fit(w.a, blocks_of(w.k), mt) && offsets_fit(w.b, blocks_of(w.k), mt); }

template <bool PAIR>
static void launch_tiles(const Launch<Product, PAIR>& l, int mt, bool one_buffer, uint32_t groups, hipStream_t st)
{
    const dim3 grid(groups), threads(mt == 4 ? 512 : 256);
    if (mt == 4) hipLaunchKernelGGL((mv_mx_product_tile_kernel<4, 2, 2, 4, 2, PAIR>), grid, threads, 0, st, l);
    else if (one_buffer) hipLaunchKernelGGL((mv_mx_product_tile_kernel<2, 2, 2, 2, 1, PAIR>), grid, threads, 0, st, l);
    else hipLaunchKernelGGL((mv_mx_product_tile_kernel<2, 2, 2, 2, 2, PAIR>), grid, threads, 0, st, l);
}

// Up to two products (n: how many) in as few launches as their sizes allow.
static mv_status launch_products(const Wanted* w, int n, hipStream_t st)
{
    FewCut few[2] = {};
    bool few_a[2] = {};
    FewProduct<uint32_t> fp[2];
    for (int i = 0; i < n; ++i) {
        few[i] = few_codes_cut(w[i], few_a[i]);
        if (few[i].mt) fp[i] = few_codes(w[i], few_a[i]);
    }
    if (n == 2 && few[0].mt && few[0].mt == few[1].mt && few[0].nt == few[1].nt) return launch_few(fp, few, 2, st);
    Cut  cut[2] = {};
    bool tiled[2] = {};
    for (int i = 0; i < n; ++i) {
        tiled[i] = !few[i].mt && offsets_fit(w[i], 2);
        if (tiled[i]) {
            cut[i] = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, large(w[i].a.rows, w[i].b.rows) && offsets_fit(w[i], 4) ? 4 : 2);
            if (cut[i].groups() > kMostGroups / 2) return MV_ERR_INVALID_ARG;
        }
    }
    const bool both = tiled[0] && tiled[1];
    bool       one_buffer = true;
    int64_t    all = 0;
    for (int i = 0; i < n; ++i)
        if (tiled[i]) {
            const Cut c = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, 2);
            one_buffer &= few_steps(w[i].k);
            all += c.tiles_m * c.tiles_n;
        }
    one_buffer &= all > kUnits && all <= kMostGroups;
    // with one buffer: the smaller tiles; in one launch: those for both, and each other's tiles to fill the units with
    if (one_buffer || (both && (cut[0].mt == 2 || cut[1].mt == 2))) {
        int64_t tiles[2] = {};
        for (int i = 0; i < n; ++i)
            if (tiled[i]) tiles[i] = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, 2, 512).groups();
        for (int i = 0; i < n; ++i)
            if (tiled[i]) cut[i] = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, 2, tiles[1 - i]);
        if (cut[0].groups() + cut[1].groups() > kMostGroups) return MV_ERR_INVALID_ARG;
    }
    for (int i = 0; i < n; ++i) {
        if (few[i].mt) {
            if (const mv_status rc = launch_few(fp + i, few + i, 1, st)) return rc;
        } else if (!tiled[i]) {
            if (const mv_status rc = launch_plain(w[i], st)) return rc;
        } else if (!both || i == 0) {
            const Product  p = product_of(w[i], cut[i]);
            const uint32_t firsts = (uint32_t)cut[i].groups();
            if (both) {
                const Launch<Product, true> l = {{p, product_of(w[1], cut[1])}, firsts};
                launch_tiles(l, cut[i].mt, one_buffer, firsts + (uint32_t)cut[1].groups(), st);
            } else {
                launch_tiles(Launch<Product, false>{{p}, firsts}, cut[i].mt, one_buffer, firsts, st);
            }
            launch_join(w[i], cut[i], st);
            if (both) launch_join(w[1], cut[1], st);
            if (hipGetLastError() != hipSuccess) return MV_ERR_DEVICE;
        }
    }
    return MV_OK;
}

// A matrix of codes in the scratch, `at` moves behind it.
// Its rows of codes are whole lines of 128 bytes: the columns' codes come in runs of 64.
inline int64_t line_words(int64_t n) { return (4 * blocks_of(n) + 31) / 32 * 32; }
inline size_t code_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)line_words(n) * 4); }
inline size_t scale_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)((blocks_of(n) + 3) / 4 * 4)); }
inline size_t held_bytes(int64_t rows, int64_t n) { return code_bytes(rows, n) + scale_bytes(rows, n); }
static Held carve(char*& at, int64_t rows, int64_t n)
{
    Held h = {reinterpret_cast<uint32_t*>(at), reinterpret_cast<uint8_t*>(at + code_bytes(rows, n)), line_words(n),
              (blocks_of(n) + 3) / 4 * 4, rows};
    at += held_bytes(rows, n);
    return h;
}
static Factor factor_of(const Held& h) { return {h.codes, h.scales, h.ld_words, h.ld_scales, h.rows}; }

template <typename X>
static mv_status launch_few_values(const FewCut& cut, const void* x, int64_t ld_x, int64_t m, const Factor& w, int64_t k, const Out& y,
                                   int64_t ld_y, hipStream_t st)
{
    const FewProduct<X> p = few_product(w, Few<X>{static_cast<const X*>(x), ld_x, nullptr, 0, (uint32_t)m}, k, y, 1, ld_y);
    return launch_few(&p, &cut, 1, st);
}

}  // namespace mvx

extern "C" {

size_t mv_mx_product_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    return sizes_valid(m, n, k) ? parts_bytes(m, n, k) : 0;
}

mv_status mv_mx_product(const uint32_t* a_codes, int64_t ld_aw, const uint8_t* a_scales, int64_t ld_as,
                        const uint32_t* b_codes, int64_t ld_bw, const uint8_t* b_scales, int64_t ld_bs, int64_t m, int64_t n,
                        int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!sizes_valid(m, n, k) || !codes_valid(a_codes, ld_aw, a_scales, ld_as, k) ||
        !codes_valid(b_codes, ld_bw, b_scales, ld_bs, k) || !values_valid(c, c_dtype, ld_c, n) ||
        !scratch_valid(scratch, scratch_bytes, parts_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    const Wanted w = {{a_codes, a_scales, ld_aw, ld_as, m}, {b_codes, b_scales, ld_bw, ld_bs, n}, k, {c, c_dtype == MV_BF16}, ld_c, scratch};
    return launch_products(&w, 1, static_cast<hipStream_t>(stream));
}

size_t mv_mx_linear_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    return sizes_valid(m, n, k) ? held_bytes(m, k) + parts_bytes(m, n, k) : 0;
}

mv_status mv_mx_linear(const void* x, int32_t x_dtype, int64_t ld_x, const uint32_t* w_codes, int64_t ld_words,
                       const uint8_t* w_scales, int64_t ld_scales, int64_t m, int64_t n, int64_t k, void* y, int32_t y_dtype,
                       int64_t ld_y, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!sizes_valid(m, n, k) || !values_valid(x, x_dtype, ld_x, k) || !codes_valid(w_codes, ld_words, w_scales, ld_scales, k) ||
        !values_valid(y, y_dtype, ld_y, n) || !scratch_valid(scratch, scratch_bytes, mv_mx_linear_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Factor w = {w_codes, w_scales, ld_words, ld_scales, n};
    const Out out = {y, y_dtype == MV_BF16};
    const FewCut cut = few_cut(m, n, k, x_dtype == MV_BF16 ? kQuantisedBf16 : kQuantisedF32);
    if (cut.mt)
        return x_dtype == MV_BF16 ? launch_few_values<uint16_t>(cut, x, ld_x, m, w, k, out, ld_y, st)
                                  : launch_few_values<float>(cut, x, ld_x, m, w, k, out, ld_y, st);
    char* at = static_cast<char*>(scratch);
    const Held q = carve(at, m, k);
    if (const mv_status rc = launch_encode({x, ld_x, m, k}, x_dtype, q, nullptr, 0, st)) return rc;
    const Wanted p = {factor_of(q), w, k, out, ld_y, at};
    return launch_products(&p, 1, st);
}

size_t mv_mx_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    if (!sizes_valid(m, n, k)) return 0;
    return held_bytes(m, n) + held_bytes(n, m) + held_bytes(k, m) + parts_bytes(m, k, n) + parts_bytes(n, k, m);
}

mv_status mv_mx_linear_grad(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype,
                            const uint32_t* wt_codes, int64_t ld_words, const uint8_t* wt_scales, int64_t ld_scales,
                            int64_t m, int64_t n, int64_t k, void* dx, int32_t dx_dtype, int64_t ld_dx, void* dw,
                            int32_t dw_dtype, int64_t ld_dw, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvx;
    if (!sizes_valid(m, n, k) || !values_valid(dy, dtype, ld_dy, n) || (!dx && !dw) ||
        !scratch_valid(scratch, scratch_bytes, mv_mx_linear_grad_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    if (dx && (!codes_valid(wt_codes, ld_words, wt_scales, ld_scales, n) || !values_valid(dx, dx_dtype, ld_dx, k)))
        return MV_ERR_INVALID_ARG;
    if (dw && (!values_valid(x, dtype, ld_x, k) || !values_valid(dw, dw_dtype, ld_dw, k))) return MV_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* at = static_cast<char*>(scratch);
    const Held dy_r = carve(at, m, n), dy_t = carve(at, n, m), x_t = carve(at, k, m);
    if (const mv_status rc = launch_encode_grad({x, ld_x, m, k}, dw ? &x_t : nullptr, {dy, ld_dy, m, n}, dw ? &dy_t : nullptr,
                                                dx ? &dy_r : nullptr, dtype, st))
        return rc;
    // dw first: its sums are the long ones, as a rule
    Wanted w[2];
    int    many = 0;
    if (dw) w[many++] = {factor_of(dy_t), factor_of(x_t), m, {dw, dw_dtype == MV_BF16}, ld_dw, at};
    if (dx)
        w[many++] = {factor_of(dy_r), {wt_codes, wt_scales, ld_words, ld_scales, k}, n, {dx, dx_dtype == MV_BF16}, ld_dx,
                     at + parts_bytes(n, k, m)};
    return launch_products(w, many, st);
}

}  // extern "C"
