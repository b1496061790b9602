// Products of 8-bit matrices with a scale for each block of 128 (mv_f8_product, mv_f8_linear, mv_f8_linear_grad of
// include/mv.h).
//
//   c[i][j] = sum_k a[i][k] b[j][k],  both factors in blocks of 128 along k
//
// There are two ways to multiply.  v_mfma_scale_f32_32x32x64_f8f6f4 takes codes and scales as they are: all bytes that it takes of
// a row have one scale, so which of them its lanes hold does not matter as long as both factors agree, and the power of
// two costs no instruction of its own.  But it adds each eight neighbouring products, before they join the fp32 sum, on a
// grid 2^-13 below the largest of them, cut towards zero (measured with single products): at worst 7 * 2^-13 of the sum of the
// magnitudes.  Normal values come out within 2^-12.7 of it where k is 8, 2^-15.2 at 128, 2^-17.4 at 768 and 2^-18.5 at 8192, rms
// 2^-17.1, 2^-18.9, 2^-20.2 and 2^-21.9 (the products' eight bits lie on the grid but for those below 2^-6 of the largest).  That
// is far below the rounding of a typical bf16 result, and results in bf16 are formed so: of 4096 x 8192 by 8192 with random signs,
// whose magnitudes' sum is some 70 times a typical result, 1.2 to 1.6 % are the other neighbour of the exact value, and the error
// against 64 bits is 0.0016576 where rounding alone makes 0.0016575; with products of one sign 0.06 %.  Results that nearly vanish
// keep that share of the magnitudes, not of themselves; who needs those asks for fp32.  For fp32 results codes become bf16 values,
// which holds each and its power of two exactly (down to multiples of 2^-133), and v_mfma_f32_32x32x16_bf16 adds those to within
// 2^-23: half the rate, and two values an instruction to convert.  Few rows, whose products are not what they wait for, always
// take that way, but for small ones beside another product.
#include "mv_f8.hpp"
#include "mv_product.hpp"

#include <type_traits>

namespace mvf {

using mvx::f32x16;
using mvx::f32x4;
using mvx::i32x8;
using mvx::Launch;
using mvx::Out;
using mvx::kNoLoads;
using mvx::kPastBytes;
using mvx::quads_of;
using mvx::scratch_valid;
using mvx::sizes_valid;
using mvx::up256;

struct Half {                       // 32 bytes of a row
    u32x4 lo, hi;
};
__device__ __forceinline__ i32x8 whole(const Half& h)
{
    return i32x8{(int)h.lo.x, (int)h.lo.y, (int)h.lo.z, (int)h.lo.w, (int)h.hi.x, (int)h.hi.y, (int)h.hi.z, (int)h.hi.w};
}
// c += a b over one instruction's bytes, with byte SA, or SB, of a word of scales; the two zeros say that both factors are of
// this kind.
template <int SA, int SB>
__device__ __forceinline__ f32x16 mfma32(const Half& a, uint32_t a_scale, const Half& b, uint32_t b_scale, f32x16 c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(a), whole(b), c, 0, 0, SA, (int)a_scale, SB, (int)b_scale);
}

// The same 32 values as bf16, with their scale.
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
struct Wide {
    bf16x8 v[4];
};
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi, float factor)
{
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, factor, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, factor, true);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, factor, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, factor, true);
    return bf16x8{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
// The scale is the lowest byte of the word.
__device__ __forceinline__ Wide widen(const Half& h, uint32_t scale)
{
    const float f = mvx::factor_of(scale & 0xFFu);
    return Wide{{widen(h.lo.x, h.lo.y, f), widen(h.lo.z, h.lo.w, f), widen(h.hi.x, h.hi.y, f), widen(h.hi.z, h.hi.w, f)}};
}
__device__ __forceinline__ f32x4 mfma(const Wide& a, const Wide& b, f32x4 c)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[q], b.v[q], c, 0, 0, 0);
    return c;
}

// ---- straight from memory --------------------------------------------------------------------------------------------
//
// For rows so far apart that a tile's byte offsets leave 32 bits.
constexpr int kTile = 64;           // rows of each factor that a wavefront takes
constexpr int kProductThreads = 256;

__global__ __launch_bounds__(kProductThreads) void mv_f8_product_kernel(Factor a, Factor b, int64_t blocks, int64_t tiles_n, Out c,
                                                                        int64_t ld_c)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64, in = lane & 15u, group = lane / 16;
    const int64_t i0 = (int64_t)blockIdx.x / tiles_n * (2 * kTile) + wave / 2 * kTile;
    const int64_t j0 = (int64_t)blockIdx.x % tiles_n * (2 * kTile) + wave % 2 * kTile;
    auto load = [&](const Factor& f, int64_t row, int64_t k, Half& v, uint32_t& scale) {
        row = row < f.rows ? row : f.rows - 1;
        const uint8_t* p = f.codes + row * f.ld_bytes + k * kBlock + group * 16;
        v.lo = *reinterpret_cast<const u32x4*>(p);
        v.hi = *reinterpret_cast<const u32x4*>(p + 64);
        scale = f.scales[row * f.ld_scales + k];
    };
    f32x4 acc[4][4] = {};
    for (int64_t k = 0; k < blocks; ++k) {
        Half x[4], y[4];
        uint32_t xs[4], ys[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            load(a, i0 + 16 * t + in, k, x[t], xs[t]);
            load(b, j0 + 16 * t + in, k, y[t], ys[t]);
        }
        Wide yw[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) yw[u] = widen(y[u], ys[u]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const Wide xw = widen(x[t], xs[t]);
#pragma unroll
            for (int u = 0; u < 4; ++u) acc[t][u] = mfma(yw[u], xw, acc[t][u]);
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
// A workgroup of WM x WN wavefronts takes 32 MT WM x 32 NT WN results, 32 MT x 32 NT a wavefront, in steps of one block, 128
// bytes a row.  The rows of both factors go from memory straight into LDS, each row's 16-byte units in the order
// unit ^ (row / 2 % 8): what sixteen lanes of neighbouring rows read together lies in different banks, and what eight
// lanes write together is one whole line of memory.  Two buffers: the next step's loads are in flight during this one's
// products.  With few steps, one buffer, and the unit's other workgroups fill the waiting.  Loads beyond the last row or block
// return zeros by the buffer's bounds.  The scales of two steps, two bytes a row, go through registers, where those
// behind the last block become 0, into LDS of their own.
//
// A lane of the 32 x 32 x 64 instruction holds 32 of the 64 bytes that a half step takes of its row.
//
// The matrix units bound it: 4096 x 8192 by 8192 to bf16 216 us, 2.5 PFLOP/s, as much as the card's power leaves for such values
// in a long product (the instruction alone 3.6, on zeros 4.8); to fp32 440, 1.25 (the bf16 instruction alone 1.8, on zeros 2.45;
// the conversions, full rate, run beside it).

// One product and how it is cut: tiles_m x tiles_n tiles, `splits` runs of steps_each steps each.  With several splits c is
// fp32 and holds their sums one after the other, split_c apart.
struct Product {
    Factor   a, b;
    uint32_t blocks, tiles_m, tiles_n, steps_each, splits;
    Out      c;
    int64_t  ld_c, split_c;
    uint32_t past;                  // store past the caches
};

template <int MT, int NT, int WM, int WN, int BUFFERS, bool WIDE, bool PAIR>
__global__ __launch_bounds__(64 * WM * WN, BUFFERS == 1 ? 3 : 2) void mv_f8_product_tile_kernel(Launch<Product, PAIR> l)
{
    constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    constexpr int kM = 32 * MT * WM, kN = 32 * NT * WN, kRows = kM + kN;
    typedef uint8_t Codes[kRows * kBlock];
    __shared__ __attribute__((aligned(1024))) Codes even;
    __shared__ __attribute__((aligned(4))) uint16_t scales[2][kRows];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = __builtin_amdgcn_readfirstlane(t / 64);
    const Product& p = l.product();
    const Factor a = p.a, b = p.b;
    const uint32_t blocks = p.blocks, steps_each = p.steps_each, id = l.id();
    const uint32_t split = id / (p.tiles_m * p.tiles_n);
    uint32_t tm, tn;
    mvx::tile_of(id - split * (p.tiles_m * p.tiles_n), p.tiles_m, p.tiles_n, tm, tn);
    const int64_t i0 = (int64_t)tm * kM, j0 = (int64_t)tn * kN;
    const uint32_t step0 = split * steps_each, count = min(steps_each, blocks - step0);       // at least one
    const uint32_t end = step0 + count;                                    // an odd count's last step is one of zeros

    // what this wavefront loads: rows [wave kM / kWaves, ...) of a and as many of b, eight rows an instruction
    const uint32_t a_pitch = (uint32_t)a.ld_bytes, b_pitch = (uint32_t)b.ld_bytes;
    const int64_t a_rows = a.rows - i0 < kM ? a.rows - i0 : kM, b_rows = b.rows - j0 < kN ? b.rows - j0 : kN;
    const __amdgpu_buffer_rsrc_t a_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(a.codes + i0 * a.ld_bytes), 0, (int)((uint32_t)(a_rows - 1) * a_pitch + blocks * kBlock), 0x00020000);
    const __amdgpu_buffer_rsrc_t b_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(b.codes + j0 * b.ld_bytes), 0, (int)((uint32_t)(b_rows - 1) * b_pitch + blocks * kBlock), 0x00020000);
    static_assert(kM / kWaves % 16 == 0 && kN / kWaves % 16 == 0, "rows from a multiple of 16 on");
    const uint32_t row_in = lane >> 3, unit = (lane & 7u) ^ (row_in >> 1);       // of every second eight rows unit ^ 4
    uint32_t other = unit & 4u ? 0u - 64u : 64u;
    uint32_t a_at = (wave * (kM / kWaves) + row_in) * a_pitch + unit * 16, b_at = (wave * (kN / kWaves) + row_in) * b_pitch + unit * 16;
    auto load_codes = [&](uint32_t k, Codes& to) {
        const uint32_t step = step0 + k;
        // The whole offset is the lane's own, for the bounds to hold: beyond every buffer where there is no such block.  It is
        // made anew each time: eight registers that are kept for it are eight too many.
        const uint32_t at = step * kBlock;
        const bool live = step < end;
        asm volatile("" : "+v"(a_at), "+v"(b_at), "+v"(other));
#pragma unroll
        for (int i = 0; i < kM / kWaves / 8; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                a_buf, (__attribute__((address_space(3))) void*)(to + (wave * (kM / kWaves) + i * 8) * kBlock), 16,
                live ? (i % 2 ? a_at + other : a_at) + (i * 8 * a_pitch + at) : 0x80000000u, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kN / kWaves / 8; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                b_buf, (__attribute__((address_space(3))) void*)(to + (kM + wave * (kN / kWaves) + i * 8) * kBlock), 16,
                live ? (i % 2 ? b_at + other : b_at) + (i * 8 * b_pitch + at) : 0x80000000u, 0, 0, 0);
    };
    // A thread has one row's scales, of a the first wavefronts, of b the others: one load for two steps, which reads zeros
    // where the rows end, and what lies behind a row's last block.
    static_assert(kThreads == kRows, "a row a thread");
    const bool of_a = wave < kM / 64;
    const uint32_t sc_pitch = (uint32_t)(of_a ? a.ld_scales : b.ld_scales), sc_rows = (uint32_t)(of_a ? a_rows : b_rows);
    const __amdgpu_buffer_rsrc_t sc_buf = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(of_a ? a.scales + i0 * a.ld_scales : b.scales + j0 * b.ld_scales), 0,
        (int)((sc_rows - 1) * sc_pitch + (blocks + 3) / 4 * 4), 0x00020000);
    const uint32_t sc_at = (t - (of_a ? 0u : (uint32_t)kM)) * sc_pitch;
    uint32_t next;
    auto fetch_scales = [&](uint32_t k) { next = __builtin_amdgcn_raw_buffer_load_b16(sc_buf, sc_at + step0 + k, 0, 0); };
    auto keep_scales = [&](uint32_t k) {
        const int live = (int)end - (int)(step0 + k);
        // rows 32 apart side by side
        scales[k / 2 % 2][(t & ~63u) + (t & 31u) * 2 + (t >> 5 & 1u)] = (uint16_t)(next & (live >= 2 ? 0xFFFFu : live == 1 ? 0xFFu : 0u));
    };

    const uint32_t in = lane & 31u, half = lane >> 5;
    const uint32_t a_row = wave / WN * (32 * MT) + in, b_row = kM + wave % WN * (32 * NT) + in;
    f32x16 acc[MT][NT] = {};
    Half x[MT], y[2][NT];
    uint32_t as[MT / 2], bs[NT / 2], next_as[MT / 2], next_bs[NT / 2];     // two rows' scales of two steps in each
    // bytes of half step s: units 4 s + half and two more
    const uint32_t turn = lane >> 1 & 7u;
    auto read = [&](const Codes& from, uint32_t row, uint32_t s, Half& h) {
        h.lo = *reinterpret_cast<const u32x4*>(from + row * kBlock + ((4 * s + half) ^ turn) * 16);
        h.hi = *reinterpret_cast<const u32x4*>(from + row * kBlock + ((4 * s + 2 + half) ^ turn) * 16);
    };
    auto read_y = [&](const Codes& from, uint32_t s, Half (&to)[NT]) {
#pragma unroll
        for (int j = 0; j < NT; ++j) read(from, b_row + 32 * j, s, to[j]);
    };
    auto read_scales = [&](uint32_t k, uint32_t (&a_to)[MT / 2], uint32_t (&b_to)[NT / 2]) {
        typedef uint32_t __attribute__((may_alias)) pair;
        const pair* sc = reinterpret_cast<const pair*>(scales[k / 2 % 2]);
#pragma unroll
        for (int i = 0; i < MT / 2; ++i) a_to[i] = sc[((a_row & ~63u) >> 1) + 32 * i + in];
#pragma unroll
        for (int j = 0; j < NT / 2; ++j) b_to[j] = sc[((b_row & ~63u) >> 1) + 32 * j + in];
    };
    // The products of half a step, whose rows are here; each row's next half is asked for right behind its last product.
    auto products = [&](auto step, const Half (&with)[NT], const Codes& then, uint32_t then_s) {
        constexpr int S = decltype(step)::value;
        if constexpr (WIDE) {
            Wide yw[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) yw[j] = widen(with[j], bs[j / 2] >> (8 * S + 16 * (j % 2)));
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const Wide xw = widen(x[i], as[i / 2] >> (8 * S + 16 * (i % 2)));
                read(then, a_row + 32 * i, then_s, x[i]);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(yw[j].v[q], xw.v[q], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            static_assert(NT == 2 && MT % 2 == 0, "pairs of rows");
#pragma unroll
            for (int i = 0; i < MT; i += 2) {
                acc[i][0] = mfma32<S, S>(with[0], bs[0], x[i], as[i / 2], acc[i][0]);
                acc[i][1] = mfma32<2 + S, S>(with[1], bs[0], x[i], as[i / 2], acc[i][1]);
                read(then, a_row + 32 * i, then_s, x[i]);
                __builtin_amdgcn_sched_barrier(0);
                acc[i + 1][0] = mfma32<S, 2 + S>(with[0], bs[0], x[i + 1], as[i / 2], acc[i + 1][0]);
                acc[i + 1][1] = mfma32<2 + S, 2 + S>(with[1], bs[0], x[i + 1], as[i / 2], acc[i + 1][1]);
                read(then, a_row + 32 * i + 32, then_s, x[i + 1]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    auto all_here = [&] {
        __builtin_amdgcn_s_waitcnt(kNoLoads);
        __syncthreads();
    };
    const std::integral_constant<int, 0> first{};
    const std::integral_constant<int, 1> second{};
    if constexpr (BUFFERS == 1) {
        for (uint32_t k = 0; k < count; ++k) {
            load_codes(k, even);
            if (k % 2 == 0) {
                fetch_scales(k);
                keep_scales(k);
            }
            all_here();
            read_scales(k, as, bs);
            if (k % 2) {
#pragma unroll
                for (int i = 0; i < MT / 2; ++i) as[i] >>= 8;
#pragma unroll
                for (int j = 0; j < NT / 2; ++j) bs[j] >>= 8;
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) read(even, a_row + 32 * i, 0, x[i]);
            read_y(even, 0, y[0]);
            read_y(even, 1, y[1]);
            products(first, y[0], even, 1);
            products(first, y[1], even, 0);
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
#pragma unroll
        for (int i = 0; i < MT; ++i) read(even, a_row + 32 * i, 0, x[i]);
        read_y(even, 0, y[0]);
        read_scales(0, as, bs);
        // Two steps a turn.  In the middle of a step all wavefronts have read its buffer, so there the next loads into it
        // begin, and the second half's products cover the way of the next step's first rows from LDS.  The turn has no branches:
        // behind the last step zeros are loaded.
        for (uint32_t k = 0; k < count; k += 2) {
            read_y(even, 1, y[1]);
            products(first, y[0], even, 1);
            all_here();
            fetch_scales(k + 2);
            load_codes(k + 2, even);
            read_y(odd, 0, y[0]);
            products(first, y[1], odd, 0);
            read_y(odd, 1, y[1]);
            products(second, y[0], odd, 1);
            keep_scales(k + 2);
            all_here();
            load_codes(k + 3, odd);
            read_y(even, 0, y[0]);
            read_scales(k + 2, next_as, next_bs);
            products(second, y[1], even, 0);
#pragma unroll
            for (int i = 0; i < MT / 2; ++i) as[i] = next_as[i];
#pragma unroll
            for (int j = 0; j < NT / 2; ++j) bs[j] = next_bs[j];
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
                const f32x4 v0 = *reinterpret_cast<const f32x4*>(mine + r * 64 + (unit ^ (r & 15u)) * 4);
                const f32x4 v1 = *reinterpret_cast<const f32x4*>(mine + r * 64 + ((unit + 1) ^ (r & 15u)) * 4);
                const float v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
                const int64_t col = col0 + 4 * unit;
                if (row0 + r < a.rows) mvx::store8(static_cast<uint16_t*>(p.c.p) + out + (row0 + r) * p.ld_c + col, b.rows - col, v, p.past);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t r = 4 * u + lane / 16, unit = lane % 16;
                const f32x4 w = *reinterpret_cast<const f32x4*>(mine + r * 64 + (unit ^ (r & 15u)) * 4);
                const float v[4] = {w.x, w.y, w.z, w.w};
                const int64_t col = col0 + 4 * unit;
                if (row0 + r < a.rows) mvx::store4(static_cast<float*>(p.c.p) + out + (row0 + r) * p.ld_c + col, b.rows - col, v, p.past);
            }
        }
    }
}

// A product's splits, to be added up.
struct Splits {
    const float* parts;
    uint32_t     count, lanes;
    int64_t      m, n, split_c, quads;
    Out          c;
    int64_t      ld_c;
    int64_t      groups() const { return (m * quads + 256 / lanes - 1) / (256 / lanes); }
};
template <bool PAIR>
__global__ __launch_bounds__(256) void mv_f8_product_join_kernel(Launch<Splits, PAIR> l)
{
    const Splits& p = l.product();
    mvx::join_splits(l.id(), p.parts, p.count, p.lanes, p.m, p.n, p.split_c, p.quads, p.c, p.ld_c);
}

// ---- few rows of one factor ------------------------------------------------------------------------------------------
//
// Up to 16 rows of one factor ("few"; up to 64 where they are values) against many of the other ("many"), whose
// codes are the bytes to read.  A workgroup takes 16 of the many rows and all of k, its wavefronts turns of four
// blocks; what they have is added up through LDS in the wavefronts' order.  Lane l of an instruction holds row l % 16
// and the 16-byte units l / 16 and l / 16 + 4 of the block, so the four lanes of a row read 64 bytes in a row.  The four
// scales of a row and turn are one word.  The few rows' codes are read as the many's are, out of the caches; values are
// quantised by every workgroup for itself, four lanes a block, into LDS, while the first turn's codes are on their way.
// Loads in flight are what it lives on, and those of many wavefronts with one turn each are worth more than two turns each of
// the half of them: 5 x 8192 bf16 by 16,384 31.6 us (two turns 37.7, and 32 of the many rows to a workgroup 41.0).

constexpr int kTurn = 4;            // blocks
constexpr int kFewWaves = 8;
template <typename X>
struct Few {                        // X: uint8_t: codes; uint16_t or float: bf16 or fp32 values
    const X*       rows;
    int64_t        ld;
    const uint8_t* scales;          // of codes
    int64_t        ld_scales;
    uint32_t       count;
};

// A quarter of a block of the few rows on its way, 32 values: fetched, and then made codes and scale of, the four quarters of a
// block by four consecutive lanes.
template <typename X>
struct Quarter;
template <>
struct Quarter<float> {
    float x[4][8];
    __device__ __forceinline__ void fetch(const Few<float>& f, uint32_t row, uint32_t block, uint32_t q, int64_t k)
    {
        const int64_t at = (int64_t)block * kBlock + q * 32;
        const float* p = f.rows + row * f.ld + at;
#pragma unroll
        for (int i = 0; i < 4; ++i) mvx::load8(p + 8 * i, k - at - 8 * i, x[i]);
    }
    __device__ __forceinline__ void finish(u32x4 (&codes)[2], uint32_t& s) const
    {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[q][i]) & 0x7FFFFFFFu);
        s = scale_of(top_of_quad(top));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x2 w = encode8(x[q], s);
            codes[q / 2][q % 2 * 2] = w.x, codes[q / 2][q % 2 * 2 + 1] = w.y;
        }
    }
};
template <>
struct Quarter<uint16_t> {
    uint32_t x[4][4];
    __device__ __forceinline__ void fetch(const Few<uint16_t>& f, uint32_t row, uint32_t block, uint32_t q, int64_t k)
    {
        const int64_t at = (int64_t)block * kBlock + q * 32;
        const uint16_t* p = f.rows + row * f.ld + at;
#pragma unroll
        for (int i = 0; i < 4; ++i) mvx::load8(p + 8 * i, k - at - 8 * i, x[i]);
    }
    __device__ __forceinline__ void finish(u32x4 (&codes)[2], uint32_t& s) const
    {
        uint32_t top = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) top = top2(top, x[q][i]);
        s = scale_of(top_of_quad(top_of_pair(top)));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const u32x2 w = encode8(x[q], s);
            codes[q / 2][q % 2 * 2] = w.x, codes[q / 2][q % 2 * 2 + 1] = w.y;
        }
    }
};

// LDS of the few rows' values: `count` rows of `turns` x 4 blocks of codes, rows 16 bytes longer against bank conflicts, then a
// word of scales for each row and turn.
__host__ __device__ constexpr uint32_t few_pitch(uint32_t turns) { return turns * (kTurn * kBlock) + 16; }
__host__ __device__ constexpr uint32_t few_bytes(uint32_t count, uint32_t turns) { return count * (few_pitch(turns) + turns * kTurn); }

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

// A lane's codes and scales of a turn of a row.  Of its last turn's blocks that there are not the last one is read again: loads
// that may be left out leave open how many are on their way, and a wait for earlier ones becomes one for all.
struct Turn {
    Half     codes[kTurn];
    uint32_t scales;
    __device__ __forceinline__ void load(const uint8_t* row, const uint8_t* row_scales, uint32_t block, uint32_t blocks)
    {
        scales = *reinterpret_cast<const uint32_t*>(row_scales + block);
#pragma unroll
        for (uint32_t b = 0; b < kTurn; ++b) {
            const uint8_t* p = row + (int64_t)min(block + b, blocks - 1) * kBlock;
            codes[b].lo = *reinterpret_cast<const u32x4*>(p);
            codes[b].hi = *reinterpret_cast<const u32x4*>(p + 64);
        }
    }
};
// Its products with the same of the few rows, a block at a time, and those of the last turn as far as there are any.
template <int S = 0>
__device__ __forceinline__ void add(const Turn& a, const uint8_t* p, uint32_t scales, int live, f32x4& c)
{
    if constexpr (S < kTurn) {
        if (S == 0 || live > S) {
            const Half x = {*reinterpret_cast<const u32x4*>(p + S * kBlock), *reinterpret_cast<const u32x4*>(p + S * kBlock + 64)};
            c = mfma(widen(a.codes[S], a.scales >> (8 * S)), widen(x, scales >> (8 * S)), c);
            add<S + 1>(a, p, scales, live, c);
        }
    }
}

// A workgroup: 16 MT few rows, 16 of the many.
template <int MT, typename X, bool PAIR>
__global__ __launch_bounds__(64 * kFewWaves, MT == 1 ? 4 : 2) void mv_f8_product_few_kernel(Launch<FewProduct<X>, PAIR> l)
{
    constexpr bool kCodes = std::is_same_v<X, uint8_t>;
    static_assert(!kCodes || MT == 1, "codes: up to 16 rows");
    const FewProduct<X>& p = l.product();
    const uint32_t id = l.id();
    const Factor many = p.many;
    const Few<X> few = p.few;
    const uint32_t blocks = p.blocks;
    const int64_t k = p.k, j0 = (int64_t)id * 16;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = blockDim.x / 64;
    const uint32_t in = lane & 15u, g = lane / 16;
    extern __shared__ __attribute__((aligned(16))) uint8_t held[];
    const uint32_t turns = (blocks + kTurn - 1) / kTurn, row_blocks = turns * kTurn, pitch = few_pitch(turns);
    uint8_t* held_scales = held + few.count * pitch;

    const int64_t row = j0 + in < many.rows ? j0 + in : many.rows - 1;
    const uint8_t *codes = many.codes + row * many.ld_bytes + g * 16, *scales = many.scales + row * many.ld_scales;
    uint32_t block = wave * kTurn;
    Turn now;
    f32x4 acc[MT] = {};
    if constexpr (kCodes) {
        const int64_t few_row = min(in, few.count - 1);
        const uint8_t *few_codes = few.rows + few_row * few.ld + g * 16, *few_scales = few.scales + few_row * few.ld_scales;
        for (; block < blocks; block += waves * kTurn) {
            const int live = (int)(blocks - block);
            now.load(codes, scales, block, blocks);
            add(now, few_codes + (int64_t)block * kBlock, *reinterpret_cast<const uint32_t*>(few_scales + block), live, acc[0]);
        }
    } else {
        // Loads come back in their order, so what goes into LDS is asked for first.
        Quarter<X> mine;
        const uint32_t quarters = few.count * row_blocks * 4;
        auto fetch = [&](uint32_t at) {
            const uint32_t r = at / (4 * row_blocks), b = at / 4 - r * row_blocks;
            if (at < quarters && b < blocks) mine.fetch(few, r, b, at % 4, k);
        };
        auto hold = [&](uint32_t at) {
            const uint32_t r = at / (4 * row_blocks), b = at / 4 - r * row_blocks, q = at % 4;
            if (at >= quarters || b >= blocks) return;                   // all four lanes of a block
            u32x4 made[2];
            uint32_t scale;
            mine.finish(made, scale);
            *reinterpret_cast<u32x4*>(held + r * pitch + b * kBlock + q * 32) = made[0];
            *reinterpret_cast<u32x4*>(held + r * pitch + b * kBlock + q * 32 + 16) = made[1];
            if (q == 0) held_scales[r * row_blocks + b] = (uint8_t)scale;
        };
        fetch(threadIdx.x);
        now.load(codes, scales, min(block, (blocks - 1) / kTurn * kTurn), blocks);
        hold(threadIdx.x);
        for (uint32_t at = threadIdx.x + blockDim.x; at < quarters; at += blockDim.x) {
            fetch(at);
            hold(at);
        }
        __syncthreads();
        while (block < blocks) {
            const int live = (int)(blocks - block);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const uint32_t r = min(16 * i + in, few.count - 1);
                const uint32_t few_word = *reinterpret_cast<const uint32_t*>(held_scales + r * row_blocks + block);
                add(now, held + r * pitch + block * kBlock + g * 16, few_word, live, acc[i]);
            }
            block += waves * kTurn;
            if (block < blocks) now.load(codes, scales, block, blocks);
        }
        __syncthreads();
    }
    f32x4* sums = reinterpret_cast<f32x4*>(held);                         // wavefront, tile, lane
#pragma unroll
    for (int i = 0; i < MT; ++i) sums[(wave * MT + i) * 64 + lane] = acc[i];
    __syncthreads();
    for (uint32_t at = threadIdx.x; at < MT * 64; at += blockDim.x) {
        f32x4 v = sums[at];
        for (uint32_t w = 1; w < waves; ++w) v += sums[w * MT * 64 + at];
        const uint32_t i = at / 64 * 16 + (at & 15u);
        const int64_t j = j0 + (at >> 4 & 3u) * 4, to = j * p.step_many + i * p.step_few;
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

// Whether and how the kernel for few rows takes a product: up to 16 rows of codes (with 32 it is faster for some sizes and slower
// for others: 32 x 4096 by 4096 12.2 us, in tiles 13.8, 8192 by 8192 29.7, in tiles 21.5), and up to 64 of values where
// quantising them in every workgroup costs less than a launch that does it once, which is where all of them together have few.
// bf16 us in one launch, and in two: 2 x 4096 by 4096, 2 million values to all workgroups, 6.7 (9.1); 32 x 2048 by 2048, 8 M, 8.4
// (11.9); 1 x 8192 by 16,384, 8 M, 26.7 (27.9); 3 x 8192 by 8192, 13 M, 16.3 (16.1); 16 x 4096 by 4096, 17 M, 10.0 (9.1); 5 x
// 8192 by 16,384, 42 M, 36.2 (32.2); beyond 16 rows 64 x 1024 by 4096, 17 M, 9.3 (11.8).  fp32: 8 x 2048 by 4096, 4 M, 7.6 (9.0);
// 1 x 8192 by 8192, 4 M, 16.4 (15.5); 2 x 8192 by 8192, 8 M, 17.8 (15.9); 20 x 2048 by 4000, 10 M, 10.8 (13.4).
constexpr int64_t kQuantisedBf16 = 12000000, kQuantisedF32 = 5000000;
struct FewCut {
    int      mt;                    // 0: it does not
    uint32_t groups, lds, waves;
};
static FewCut few_cut(int64_t few, int64_t many, int64_t k, int64_t quantised)     // most values to quantise; 0: codes
{
    const bool values = quantised > 0;
    if (few > (values ? kFewValues : kFewRows)) return FewCut{};
    if (values && few > 16) quantised *= 2;
    const int64_t turns = (blocks_of(k) + kTurn - 1) / kTurn;
    FewCut c = {};
    c.mt = few <= 16 ? 1 : few <= 32 ? 2 : 4;
    const int64_t groups = (many + 15) / 16;
    if (groups > kMostGroups / 4 || (values && (turns >= 4096 || groups * few * k > quantised))) return FewCut{};
    c.groups = (uint32_t)groups;
    // a wavefront for each turn, or for each 16 blocks of the few rows' values
    const int64_t waves = values && few > 4 ? few * turns / 4 + 1 : turns;
    c.waves = (uint32_t)(waves < kFewWaves ? waves : kFewWaves);
    const int64_t sums = c.waves * c.mt * 1024, lds = values ? few_bytes(1, (uint32_t)turns) * few : 0;
    if (lds > kFewLds || (values && few > 16 && c.groups > 256)) return FewCut{};
    c.lds = (uint32_t)(lds < sums ? sums : lds);
    return c;
}

template <typename X>
static FewProduct<X> few_product(const Factor& many, const Few<X>& few, int64_t k, const Out& c, int64_t step_many,
                                 int64_t step_few)
{
    return {many, few, (uint32_t)blocks_of(k), k, c, step_many, step_few};
}
// One product, or two of codes.
template <int MT, typename X>
static void launch_few_of(const FewProduct<X>* p, const FewCut* cut, int n, hipStream_t st)
{
    const dim3 threads(64 * (n == 2 && cut[1].waves > cut[0].waves ? cut[1].waves : cut[0].waves));
    const uint32_t lds = n == 2 ? threads.x * 16 : cut[0].lds;
    if constexpr (std::is_same_v<X, uint8_t>) {
        if (n == 2) {
            hipLaunchKernelGGL((mv_f8_product_few_kernel<MT, X, true>), dim3(cut[0].groups + cut[1].groups), threads, lds, st,
                               Launch<FewProduct<X>, true>{{p[0], p[1]}, cut[0].groups});
            return;
        }
    }
    hipLaunchKernelGGL((mv_f8_product_few_kernel<MT, X, false>), dim3(cut[0].groups), threads, lds, st,
                       Launch<FewProduct<X>, false>{{p[0]}, cut[0].groups});
}
template <typename X>
static mv_status launch_few(const FewProduct<X>* p, const FewCut* cut, int n, hipStream_t st)
{
    if (cut[0].mt == 1) launch_few_of<1>(p, cut, n, st);
    else if constexpr (!std::is_same_v<X, uint8_t>) {                   // codes: up to 16 rows only
        if (cut[0].mt == 2) launch_few_of<2>(p, cut, n, st);
        else launch_few_of<4>(p, cut, n, st);
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
// How many runs the steps are split into, of four steps at least (1000 x 300 by 600 in one 9.3 us, of two 10.7; 2000 x 500 by 1024 of four
// 12.8, of two 13.7).  With another product in the launch (`share`: the steps that each of two workgroups to a
// unit has of both) never more than alone, which is what the scratch has room for; one where it is not much longer than the
// share, because the other product's workgroups fill the units meanwhile; and no more than pay for writing and reading the
// sums, a microsecond a step against 4 TB/s.  us with as many splits as fit beside the other's tiles, with runs of the share's
// length, and so: 300 x 2000 by 4000 45.6, 34.0, 34.0; 8000 x 300 by 300 47.0, 34.7, 34.1; 4900 x 4608 by 512 82.8, 88.0, 82.4; 3000 x 512 by
// 2048 38.9, 42.2, 38.7 (by now 33.0, 27.8, 78.0 and 34.0).
static constexpr int64_t splits_of(int64_t tiles, int64_t steps, int64_t results, int64_t share)
{
    int64_t splits = 512 / tiles < steps / 3 ? 512 / tiles : steps / 3;
    // many splits only of small results: all of them are written and read again
    if (splits > 16 && splits * results > (4 << 20)) splits = 16;
    if (share) {
        const int64_t run = share > 4 ? share : 4;
        if (splits > (steps + run - 1) / run) splits = (steps + run - 1) / run;
        if (steps <= 2 * share) splits = 1;
        while (splits > 1 && splits * splits * results > steps * 500000) --splits;
    }
    return splits > 1 ? splits : 1;
}
static_assert(splits_of(4, 512, 200 * 200, 0) == 16 && splits_of(4, 512, 200 * 200, 4) == 16, "the limit of 16 holds in company, too");
static Cut cut_of(int64_t m, int64_t n, int64_t k, int mt, int64_t share = 0)
{
    auto tiles = [mt](int64_t rows) { return (rows + 64 * mt - 1) / (64 * mt); };
    Cut c = {mt, tiles(m), tiles(n), 1, 0};
    const int64_t steps = blocks_of(k);
    if (mt == 2) c.splits = (uint32_t)splits_of(c.tiles_m * c.tiles_n, steps, m * n, share);
    c.steps_each = (uint32_t)((steps + c.splits - 1) / c.splits);
    // runs begin at even steps, as pairs of scales do: a pair that begins with a row's last byte would leave the last row's buffer
    if (c.splits > 1) c.steps_each += c.steps_each % 2;
    c.splits = (uint32_t)((steps + c.steps_each - 1) / c.steps_each);
    return c;
}
// Results in bf16: tiles of 256 x 256, one to a unit, where those of 128 x 128 are more than the 512 that run at once, of up to four
// steps from 192 on.  us without and with: 2048 x 4352 by 4096 67.8, 59.4; 2816 x 3584 by 8192 127, 105; 4096 x 8192 by 8192
// 310, 238; but 2048 x 4096 by 4096, 128 of them, 50.1, 57.6; 4096 x 4096 by 512 20.9, 18.6, but 2560 x 3700 by 512 14.4, 17.6.
//
// Else, with up to four steps and more tiles than units: one buffer and three workgroups a unit, of which one loads or stores
// while another multiplies.  us with two buffers and with one: 2304 x 2304 by 512 14.4, 12.3, in fp32 16.4, 15.7; 8192 x 8192 by
// 512 fp32 112, 104; but 4096 x 4096 by 768 fp32 41.0, 43.7.
constexpr int64_t kFewSteps = 4, kUnits = 256;
inline bool few_steps(int64_t k) { return blocks_of(k) <= kFewSteps; }
static bool large(int64_t m, int64_t n, int64_t k) { return ((m + 255) / 256) * ((n + 255) / 256) >= (few_steps(k) ? 192 : 129); }
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
// Of one product or two, in one launch (1000 x 1000 by 1000, both gradients: 22.8 us, joined one after the other 24.8).
static void launch_joins(const Wanted* w, const Cut* cut, int n, hipStream_t st)
{
    Splits s[2];
    int    many = 0;
    for (int i = 0; i < n; ++i) {
        if (cut[i].splits == 1) continue;
        const int64_t rows = w[i].a.rows, quads = quads_of(w[i].b.rows);
        s[many++] = {static_cast<const float*>(w[i].parts), cut[i].splits, cut[i].splits > 16 ? 16u : 1u, rows, w[i].b.rows,
                     rows * quads * 4, quads, w[i].c, w[i].ld_c};
    }
    if (!many) return;
    const uint32_t firsts = (uint32_t)s[0].groups();
    if (many == 2)
        hipLaunchKernelGGL((mv_f8_product_join_kernel<true>), dim3(firsts + (uint32_t)s[1].groups()), dim3(256), 0, st,
                           Launch<Splits, true>{{s[0], s[1]}, firsts});
    else
        hipLaunchKernelGGL((mv_f8_product_join_kernel<false>), dim3(firsts), dim3(256), 0, st, Launch<Splits, false>{{s[0]}, firsts});
}
// The kernel without LDS, for rows so long that a tile's byte offsets leave 32 bits.
static mv_status launch_plain(const Wanted& w, hipStream_t st)
{
    const int64_t tiles_m = (w.a.rows + 2 * kTile - 1) / (2 * kTile), tiles_n = (w.b.rows + 2 * kTile - 1) / (2 * kTile);
    if (tiles_m * tiles_n > kMostGroups) return MV_ERR_INVALID_ARG;
    hipLaunchKernelGGL(mv_f8_product_kernel, dim3((uint32_t)(tiles_m * tiles_n)), dim3(kProductThreads), 0, st, w.a, w.b,
                       blocks_of(w.k), tiles_n, w.c, w.ld_c);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

// Whether a tile's byte offsets fit 32 bits: those of rows that there are stay below 2^31, where the loads of blocks that there
// are not begin, and those of all rows of a tile below 2^32.
static bool offsets_fit(const Factor& f, int64_t blocks, int mt)
{
    const int64_t pitch = f.ld_bytes, rows = f.rows < 64 * mt ? f.rows : 64 * mt;
    return pitch <= ((int64_t)1 << (mt == 4 ? 23 : 24)) && (rows - 1) * pitch + blocks * kBlock <= ((int64_t)1 << 31) - 256 &&
           f.ld_scales <= (1 << 22);
}
static bool offsets_fit(const Wanted& w, int mt) { return offsets_fit(w.a, blocks_of(w.k), mt) && offsets_fit(w.b, blocks_of(w.k), mt); }

// The kernel for few rows has a workgroup for 16 of the many rows and all of k. Where those are few and k is long, the tiles,
// which split it over the units, are faster, if a tile's offsets fit. us of few rows and of tiles, fp32 results, codes: 16 x 16 by
// 10,300 11.9, 10.1, by 131,072 126, 12; 5 x 300 by 10,300 9.7, 10.3, by 12,288 11.4, 10.2; 16 x 1000 by 16,384 18.9, 11.5; 1 x
// 1000 by 16,500 12.1, 11.5; 1 x 1 by 16,384 6.5, 9.6, by 32,768 10.2, 9.6; 3 x 5 by 16,384 9.3, 9.5, by 2,000,000 773, 50; 16 x
// 2048 by 32,768 34.8, 22.1; 16 x 4096 37.9, 35.3. Values, with the launch that quantises them: 16 x 16 by 10,300 fp32 14.6, 12.9;
// 5 x 16 bf16 11.4, 12.5, by 12,288 12.0, 12.4, by 14,000 13.2, 12.4; 1 x 1000 by 16,384 fp32 13.3, 13.1; 1 x 2048 by 16,384 14.2,
// 17.3, by 32,768 24.2, 23.2.
static bool long_sum(int64_t few, int64_t many, int64_t k)
{
    const int64_t from = many > 1024 || few * many < 8 ? 32768 : few > 4 ? 10240 : 16384;
    return few <= kFewRows && many <= 2048 && k > from;
}
// The kernel for few rows on codes: which factor's rows are the few ones; `split`: not taken because the tiles' splits are faster.
static FewCut few_codes_cut(const Wanted& w, bool& few_a, bool& split)
{
    few_a = w.a.rows <= w.b.rows;
    FewCut c = few_a ? few_cut(w.a.rows, w.b.rows, w.k, 0) : few_cut(w.b.rows, w.a.rows, w.k, 0);
    if (!c.mt) {
        few_a = !few_a;
        c = few_a ? few_cut(w.a.rows, w.b.rows, w.k, 0) : few_cut(w.b.rows, w.a.rows, w.k, 0);
    }
    split = c.mt && long_sum(few_a ? w.a.rows : w.b.rows, few_a ? w.b.rows : w.a.rows, w.k) && offsets_fit(w, 2);
    return split ? FewCut{} : c;
}
static FewProduct<uint8_t> few_codes(const Wanted& w, bool few_a)
{
    const Factor& few = few_a ? w.a : w.b;
    return few_product(few_a ? w.b : w.a, Few<uint8_t>{few.codes, few.ld_bytes, few.scales, few.ld_scales, (uint32_t)few.rows}, w.k, w.c,
                       few_a ? 1 : w.ld_c, few_a ? w.ld_c : 1);
}
template <bool PAIR>
static void launch_tiles(const Launch<Product, PAIR>& l, int mt, bool one_buffer, bool wide, uint32_t groups, hipStream_t st)
{
    const dim3 grid(groups), threads(mt == 4 ? 512 : 256);
#define MV_F8_TILES(...) hipLaunchKernelGGL((mv_f8_product_tile_kernel<__VA_ARGS__, PAIR>), grid, threads, 0, st, l)
    if (mt == 4) MV_F8_TILES(4, 2, 2, 4, 2, false);
    else if (one_buffer && wide) MV_F8_TILES(2, 2, 2, 2, 1, true);
    else if (one_buffer) MV_F8_TILES(2, 2, 2, 2, 1, false);
    else if (wide) MV_F8_TILES(2, 2, 2, 2, 2, true);
    else MV_F8_TILES(2, 2, 2, 2, 2, false);
#undef MV_F8_TILES
}

// A product of few rows with fewer bytes of codes than this goes into the other one's launch of tiles: 500 x 10 by 300, both
// gradients, 13.1 us, in two launches 16.4; 12 x 3000 by 1000, 3 million, 17.7 (18.9); 1000 x 10 by 4000, 4 million, 21.4 (20.2).
constexpr int64_t kFewBeside = 3 << 20;
// Up to two products (n: how many) in as few launches as their sizes allow.
static mv_status launch_products(const Wanted* w, int n, hipStream_t st)
{
    FewCut few[2] = {};
    bool few_a[2] = {}, split[2] = {};
    FewProduct<uint8_t> fp[2];
    for (int i = 0; i < n; ++i) {
        few[i] = few_codes_cut(w[i], few_a[i], split[i]);
        if (few[i].mt) fp[i] = few_codes(w[i], few_a[i]);
        // by bf16 products like few rows' others, so not in a launch that forms bf16 results from 8-bit ones, unless it is small
        if (n == 2 && split[i] && w[i].c.bf16 && (few_a[i] ? w[i].b.rows : w[i].a.rows) * w[i].k > kFewBeside) {
            if (const mv_status rc = launch_products(w, 1, st)) return rc;
            return launch_products(w + 1, 1, st);
        }
    }
    if (n == 2 && few[0].mt && few[1].mt) return launch_few(fp, few, 2, st);
    if (n == 2 && (few[0].mt || few[1].mt)) {
        const int f = few[0].mt ? 0 : 1;
        if (w[0].c.bf16 == w[1].c.bf16 && (few_a[f] ? w[f].b.rows : w[f].a.rows) * w[f].k <= kFewBeside) few[f].mt = 0;
    }
    Cut  cut[2] = {};
    bool tiled[2] = {};
    for (int i = 0; i < n; ++i) {
        tiled[i] = !few[i].mt && offsets_fit(w[i], 2);
        if (tiled[i]) {
            const bool larger = w[i].c.bf16 && large(w[i].a.rows, w[i].b.rows, w[i].k) && offsets_fit(w[i], 4);
            cut[i] = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, larger ? 4 : 2);
            if (cut[i].groups() > kMostGroups / 2) return MV_ERR_INVALID_ARG;
        }
    }
    if (n == 2 && !(tiled[0] && tiled[1] && w[0].c.bf16 == w[1].c.bf16)) {
        if (const mv_status rc = launch_products(w, 1, st)) return rc;
        return launch_products(w + 1, 1, st);
    }
    if (few[0].mt) return launch_few(fp, few, 1, st);
    if (!tiled[0]) return launch_plain(w[0], st);
    bool    one_buffer = true;
    int64_t all = 0, work = 0;
    for (int i = 0; i < n; ++i) {
        const Cut c = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, 2);
        one_buffer &= few_steps(w[i].k);
        all += c.tiles_m * c.tiles_n;
        work += c.tiles_m * c.tiles_n * blocks_of(w[i].k);
    }
    one_buffer &= all > kUnits && all <= kMostGroups && (cut[0].mt == 2 || (n == 2 && cut[1].mt == 2));
    // with one buffer: the smaller tiles; in one launch: those for both
    if (one_buffer || (n == 2 && (cut[0].mt == 2 || cut[1].mt == 2))) {
        const int64_t share = n == 1 ? 0 : (work + 2 * kUnits - 1) / (2 * kUnits);
        for (int i = 0; i < n; ++i) cut[i] = cut_of(w[i].a.rows, w[i].b.rows, w[i].k, 2, share);
        if (cut[0].groups() + cut[1].groups() > kMostGroups) return MV_ERR_INVALID_ARG;
    }
    const Product  p = product_of(w[0], cut[0]);
    const uint32_t firsts = (uint32_t)cut[0].groups();
    const bool     wide = !w[0].c.bf16 || (n == 1 && split[0]);
    if (n == 2) {
        const Launch<Product, true> l = {{p, product_of(w[1], cut[1])}, firsts};
        launch_tiles(l, cut[0].mt, one_buffer, wide, firsts + (uint32_t)cut[1].groups(), st);
    } else {
        launch_tiles(Launch<Product, false>{{p}, firsts}, cut[0].mt, one_buffer, wide, firsts, st);
    }
    launch_joins(w, cut, n, st);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

// A matrix of codes in the scratch, `at` moves behind it.
inline size_t code_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)blocks_of(n) * kBlock); }
inline size_t scale_bytes(int64_t rows, int64_t n) { return up256((size_t)rows * (size_t)((blocks_of(n) + 3) / 4 * 4)); }
inline size_t held_bytes(int64_t rows, int64_t n) { return code_bytes(rows, n) + scale_bytes(rows, n); }
static Held carve(char*& at, int64_t rows, int64_t n)
{
    Held h = {reinterpret_cast<uint8_t*>(at), reinterpret_cast<uint8_t*>(at + code_bytes(rows, n)), blocks_of(n) * kBlock,
              (blocks_of(n) + 3) / 4 * 4, rows};
    at += held_bytes(rows, n);
    return h;
}
static Factor factor_of(const Held& h) { return {h.codes, h.scales, h.ld_bytes, h.ld_scales, h.rows}; }

template <typename X>
static mv_status launch_few_values(const FewCut& cut, const void* x, int64_t ld_x, int64_t m, const Factor& w, int64_t k, const Out& y,
                                   int64_t ld_y, hipStream_t st)
{
    const FewProduct<X> p = few_product(w, Few<X>{static_cast<const X*>(x), ld_x, nullptr, 0, (uint32_t)m}, k, y, 1, ld_y);
    return launch_few(&p, &cut, 1, st);
}

}  // namespace mvf

extern "C" {

size_t mv_f8_product_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvf;
    return sizes_valid(m, n, k) ? parts_bytes(m, n, k) : 0;
}

mv_status mv_f8_product(const uint8_t* a_codes, int64_t ld_ab, const uint8_t* a_scales, int64_t ld_as,
                        const uint8_t* b_codes, int64_t ld_bb, const uint8_t* b_scales, int64_t ld_bs, int64_t m, int64_t n,
                        int64_t k, void* c, int32_t c_dtype, int64_t ld_c, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvf;
    if (!sizes_valid(m, n, k) || !codes_valid(a_codes, ld_ab, a_scales, ld_as, k) ||
        !codes_valid(b_codes, ld_bb, b_scales, ld_bs, k) || !values_valid(c, c_dtype, ld_c, n) ||
        !scratch_valid(scratch, scratch_bytes, parts_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    const Wanted w = {{a_codes, a_scales, ld_ab, ld_as, m}, {b_codes, b_scales, ld_bb, ld_bs, n}, k, {c, c_dtype == MV_BF16}, ld_c, scratch};
    return launch_products(&w, 1, static_cast<hipStream_t>(stream));
}

size_t mv_f8_linear_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvf;
    return sizes_valid(m, n, k) ? held_bytes(m, k) + parts_bytes(m, n, k) : 0;
}

mv_status mv_f8_linear(const void* x, int32_t x_dtype, int64_t ld_x, const uint8_t* w_codes, int64_t ld_bytes,
                       const uint8_t* w_scales, int64_t ld_scales, int64_t m, int64_t n, int64_t k, void* y, int32_t y_dtype,
                       int64_t ld_y, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvf;
    if (!sizes_valid(m, n, k) || !values_valid(x, x_dtype, ld_x, k) || !codes_valid(w_codes, ld_bytes, w_scales, ld_scales, k) ||
        !values_valid(y, y_dtype, ld_y, n) || !scratch_valid(scratch, scratch_bytes, mv_f8_linear_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Factor w = {w_codes, w_scales, ld_bytes, ld_scales, n};
    const Out out = {y, y_dtype == MV_BF16};
    const FewCut cut = few_cut(m, n, k, x_dtype == MV_BF16 ? kQuantisedBf16 : kQuantisedF32);
    char* at = static_cast<char*>(scratch);
    const Held q = carve(at, m, k);
    const Wanted p = {factor_of(q), w, k, out, ld_y, at};
    if (cut.mt && !(long_sum(m, n, k) && offsets_fit(p, 2)))
        return x_dtype == MV_BF16 ? launch_few_values<uint16_t>(cut, x, ld_x, m, w, k, out, ld_y, st)
                                  : launch_few_values<float>(cut, x, ld_x, m, w, k, out, ld_y, st);
    if (const mv_status rc = launch_encode({x, ld_x, m, k}, x_dtype, q, st)) return rc;
    return launch_products(&p, 1, st);
}

size_t mv_f8_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvf;
    if (!sizes_valid(m, n, k)) return 0;
    return held_bytes(m, n) + held_bytes(n, m) + held_bytes(k, m) + parts_bytes(m, k, n) + parts_bytes(n, k, m);
}

mv_status mv_f8_linear_grad(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype,
                            const uint8_t* wt_codes, int64_t ld_bytes, const uint8_t* wt_scales, int64_t ld_scales,
                            int64_t m, int64_t n, int64_t k, void* dx, int32_t dx_dtype, int64_t ld_dx, void* dw,
                            int32_t dw_dtype, int64_t ld_dw, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvf;
    if (!sizes_valid(m, n, k) || !values_valid(dy, dtype, ld_dy, n) || (!dx && !dw) ||
        !scratch_valid(scratch, scratch_bytes, mv_f8_linear_grad_scratch_bytes(m, n, k)))
        return MV_ERR_INVALID_ARG;
    if (dx && (!codes_valid(wt_codes, ld_bytes, wt_scales, ld_scales, n) || !values_valid(dx, dx_dtype, ld_dx, k)))
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
        w[many++] = {factor_of(dy_r), {wt_codes, wt_scales, ld_bytes, ld_scales, k}, n, {dx, dx_dtype == MV_BF16}, ld_dx,
                     at + parts_bytes(n, k, m)};
    return launch_products(w, many, st);
}

}  // extern "C"
