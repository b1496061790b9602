// Microscaled 4-bit floating point (mv_mx_* of include/mv.h): quantising rows or columns, reading back, and the
// receiver's sum over the workers.
//
// All of these read and write each value once and compute a few instructions on it: HBM bounds them, launches where they
// are short.  A lane takes 16 bytes of values, so a wavefront's loads and stores cover one run of memory: four lanes a
// block of 32 bf16 values, eight lanes one of fp32; the block's largest magnitude is two or three DPP moves away.
// 16 x 11.2 M fp32 to codes and residual 247 us, 6.2 TB/s; 4096 x 8192 bf16 to codes 20 us, 4.2 TB/s (in a loop with a
// product whose 67 MB of results are still on their way to memory); the mean of 16 x 11.2 M 31 us, 4.5 TB/s; 8192 x 4096
// codes back to bf16 13 us, 6.5 TB/s, the codes out of the last-level cache.
#include "mv_mx.hpp"

namespace mvx {

constexpr int kThreads = 256;

// (row, block of the row) of a block of all rows one after the other.  There are fewer than 2^31 of them in a launch.
struct Place {
    uint32_t row, block;
};
// Block `first` + `more`, with a division for the whole workgroup and, where a row may end in between, one of small numbers.
__device__ __forceinline__ Place place_of(uint32_t first, uint32_t more, uint32_t row_blocks)
{
    const uint32_t row = first / row_blocks;
    Place p = {row, first - row * row_blocks + more};
    if (p.block >= row_blocks) {
        const uint32_t rows = row_blocks > more ? 1u : p.block / row_blocks;
        p.row += rows;
        p.block -= rows * row_blocks;
    }
    return p;
}

// Lanes of a block, and blocks of a workgroup.
template <typename T>
constexpr int kBlockLanes = sizeof(T) == 2 ? 4 : 8;
constexpr int kBf16Blocks = 2;      // of four lanes, in quantising rows
template <typename T>
constexpr int kGroupBlocks = kThreads / kBlockLanes<T> * (sizeof(T) == 2 ? kBf16Blocks : 1);

// A matrix of values and where its codes go.
template <typename T>
struct Encode {
    const T*  vals;
    int64_t   ld_vals, rows, n;
    uint32_t* codes;
    int64_t   ld_words;
    uint8_t*  scales;
    int64_t   ld_scales;
};

template <bool RESID>
__device__ __forceinline__ void encode_rows(const Encode<float>& e, uint32_t at_group, float* resid, int64_t ld_resid)
{
    const uint32_t mine = threadIdx.x % 8;
    const Place p = place_of(at_group * kGroupBlocks<float>, threadIdx.x / 8, (uint32_t)blocks_of(e.n));
    if (p.row >= e.rows) return;                       // all lanes of a block
    const int64_t at = (int64_t)p.block * kBlock + mine * 4;
    float x[4];
    load4(e.vals + p.row * e.ld_vals + at, e.n - at, x);
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    const uint32_t scale = scale_of(top_of_eight(top)), w = encode4(x, scale);
    const uint32_t next = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0xB1, 0xf, 0xf, false);   // the neighbour's
    if ((mine & 1u) == 0) e.codes[p.row * e.ld_words + at / 8] = w | next << 16;
    if (mine == 0) e.scales[p.row * e.ld_scales + p.block] = (uint8_t)scale;
    if constexpr (RESID) {
        float held[4];
        decode4(w, scale, held);
#pragma unroll
        for (int i = 0; i < 4; ++i) held[i] = x[i] - held[i];
        store4(resid + p.row * ld_resid + at, e.n - at, held);
    }
}

// bf16 values stay pairs as they are; two blocks of a group of lanes are in flight together (8192 x 4096 and back 29.3 -> 27.7
// us; with four 28.3; fp32 values, of which a block alone is as many bytes, gain nothing).
template <bool RESID>
__device__ __forceinline__ void encode_rows(const Encode<uint16_t>& e, uint32_t at_group, float* resid, int64_t ld_resid)
{
    const uint32_t mine = threadIdx.x % 4;
    Place p[kBf16Blocks];
    uint32_t x[kBf16Blocks][4];
#pragma unroll
    for (int u = 0; u < kBf16Blocks; ++u) {
        p[u] = place_of(at_group * kGroupBlocks<uint16_t>, u * (kThreads / 4) + threadIdx.x / 4, (uint32_t)blocks_of(e.n));
        const int64_t at = (int64_t)p[u].block * kBlock + mine * 8;
        load8(e.vals + p[u].row * e.ld_vals + at, p[u].row < e.rows ? e.n - at : 0, x[u]);
    }
#pragma unroll
    for (int u = 0; u < kBf16Blocks; ++u) {
        if (p[u].row >= e.rows) break;
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) top = top2(top, x[u][i]);
        const uint32_t scale = scale_of(top_of_quad(top_of_pair(top))), w = encode8(x[u], scale);
        e.codes[p[u].row * e.ld_words + p[u].block * 4 + mine] = w;
        if (mine == 0) e.scales[p[u].row * e.ld_scales + p[u].block] = (uint8_t)scale;
        if constexpr (RESID) {
            const int64_t at = (int64_t)p[u].block * kBlock + mine * 8;
            float held[8];
            decode8(w, scale, held);
#pragma unroll
            for (int i = 0; i < 8; ++i) held[i] = widen(x[u][i / 2] >> (16 * (i & 1))) - held[i];
            store8(resid + p[u].row * ld_resid + at, e.n - at, held);
        }
    }
}

template <typename T, bool RESID>
__global__ __launch_bounds__(kThreads) void mv_mx_encode_kernel(Encode<T> e, float* resid, int64_t ld_resid)
{
    encode_rows<RESID>(e, blockIdx.x, resid, ld_resid);
}

// Columns: a wavefront takes 32 rows of 16 bytes of columns in each group of four lanes; lane r of a group has rows
// 8 r .. 8 r + 8, of each column a word of codes, and the block's largest magnitude is two DPP moves away again.  The
// codes of kTileBlocks wavefronts, one below the other, go out through LDS in runs of 16 kTileBlocks bytes a column.
// Memory is the bound: 8192 x 4096 bf16 18 us, 4.7 TB/s.  Whole lines, by eight wavefronts, change nothing (bf16 17.9 : 17.9,
// fp32 35.3 : 33.9, but 300 x 1000 5.9 : 6.3 and 3.8 : 4.5).
constexpr int kTileBlocks = 4;
template <typename T>
constexpr int kLaneCols = 16 / (int)sizeof(T);
template <typename T>
__device__ __forceinline__ void load_cols(const T* p, int64_t live, float (&x)[kLaneCols<T>])
{
    if constexpr (sizeof(T) == 2) load8(p, live, x);
    else load4(p, live, x);
}
template <typename T>
constexpr int kTileCols = 16 * kLaneCols<T>;
template <typename T>
struct Columns {                    // of a workgroup: codes and scales on their way out
    uint32_t words[kTileCols<T>][4 * kTileBlocks];
    alignas(4) uint8_t scales[kTileCols<T>][kTileBlocks];
};
template <typename T>
inline int64_t column_tiles(int64_t n) { return (n + kTileCols<T> - 1) / kTileCols<T>; }
template <typename T>
inline int64_t column_groups(int64_t rows, int64_t n)
{
    return column_tiles<T>(n) * ((blocks_of(rows) + kTileBlocks - 1) / kTileBlocks);
}

template <typename T>
__device__ __forceinline__ void encode_columns(const Encode<T>& e, uint32_t at_group, Columns<T>& out)
{
    constexpr int kCols = kLaneCols<T>;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64, group = lane / 4, r = lane & 3u;
    const uint32_t tiles = (uint32_t)((e.n + kTileCols<T> - 1) / kTileCols<T>), tile = at_group % tiles, strip = at_group / tiles;
    const int64_t col = (int64_t)tile * kTileCols<T> + group * kCols, row = ((int64_t)strip * kTileBlocks + wave) * kBlock + 8 * r;
    float x[8][kCols];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t live = row + i < e.rows ? e.n - col : 0;
        load_cols(e.vals + (row + i) * e.ld_vals + col, live, x[i]);
    }
#pragma unroll
    for (int j = 0; j < kCols; ++j) {
        float y[8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = x[i][j];
            top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
        }
        const uint32_t scale = scale_of(top_of_quad(top));
        out.words[group * kCols + j][4 * wave + r] = encode8(y, scale);
        if (r == 0) out.scales[group * kCols + j][wave] = (uint8_t)scale;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileCols<T> / 64; ++i) {
        const uint32_t c = i * 64 + threadIdx.x / kTileBlocks, b = threadIdx.x % kTileBlocks;
        const int64_t to = (int64_t)tile * kTileCols<T> + c, to_block = (int64_t)strip * kTileBlocks + b;
        if (to < e.n && to_block < blocks_of(e.rows)) {
            *reinterpret_cast<u32x4*>(e.codes + to * e.ld_words + to_block * 4) = *reinterpret_cast<const u32x4*>(&out.words[c][4 * b]);
            // four scales in one store where there are four
            const bool whole = ((int64_t)strip + 1) * kTileBlocks <= blocks_of(e.rows);
            if (!whole) e.scales[to * e.ld_scales + to_block] = out.scales[c][b];
            else if (b == 0)
                *reinterpret_cast<uint32_t*>(e.scales + to * e.ld_scales + to_block) = *reinterpret_cast<const uint32_t*>(out.scales[c]);
        }
    }
}

template <typename T>
__global__ __launch_bounds__(64 * kTileBlocks) void mv_mx_encode_t_kernel(Encode<T> e)
{
    __shared__ __attribute__((aligned(16))) Columns<T> out;
    encode_columns<T>(e, blockIdx.x, out);
}

// What a layer's gradients need, in one launch: columns of x, columns of dy, rows of dy; none of a kind: no workgroups.
// x 4900 x 4608 and dy 4900 x 512, bf16: 66 MB in 17 us, or 27 right behind a product whose 100 MB are still being stored.
template <typename T>
__global__ __launch_bounds__(kThreads) void mv_mx_encode_grad_kernel(Encode<T> x_t, uint32_t x_t_groups, Encode<T> dy_t,
                                                                     uint32_t dy_t_groups, Encode<T> dy)
{
    static_assert(kThreads == 64 * kTileBlocks, "one size of workgroup");
    __shared__ __attribute__((aligned(16))) Columns<T> out;
    const uint32_t b = blockIdx.x;
    if (b < x_t_groups) encode_columns<T>(x_t, b, out);
    else if (b < x_t_groups + dy_t_groups) encode_columns<T>(dy_t, b - x_t_groups, out);
    else encode_rows<false>(dy, b - x_t_groups - dy_t_groups, nullptr, 0);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mv_mx_decode_kernel(const uint32_t* __restrict__ codes, int64_t ld_words,
                                                                const uint8_t* __restrict__ scales, int64_t ld_scales,
                                                                int64_t rows, int64_t n, T* __restrict__ out, int64_t ld_out)
{
    constexpr int kLanes = kBlockLanes<T>, V = kBlock / kLanes;
    const uint32_t mine = threadIdx.x % kLanes;
    const Place p = place_of(blockIdx.x * (kThreads / kLanes), threadIdx.x / kLanes, (uint32_t)blocks_of(n));
    if (p.row >= rows) return;
    const int64_t at = (int64_t)p.block * kBlock + mine * V;
    const uint32_t w = codes[p.row * ld_words + at / 8], scale = scales[p.row * ld_scales + p.block];
    float x[V];
    if constexpr (V == 8) {
        decode8(w, scale, x);
        store8(out + p.row * ld_out + at, n - at, x);
    } else {
        decode4(w >> (16 * (mine & 1u)), scale, x);
        store4(out + p.row * ld_out + at, n - at, x);
    }
}

// A lane adds up eight values over the rows.
__global__ __launch_bounds__(kThreads) void mv_mx_aggregate_kernel(const uint32_t* __restrict__ codes, int64_t ld_words,
                                                                   const uint8_t* __restrict__ scales, int64_t ld_scales,
                                                                   int64_t rows, int64_t n, const float* __restrict__ weights,
                                                                   float mean, float* __restrict__ agg)
{
    const int64_t word = (int64_t)blockIdx.x * kThreads + threadIdx.x, at = word * 8;
    if (at >= n) return;
    float sum[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int kAhead = 8;
    for (int64_t r0 = 0; r0 < rows; r0 += kAhead) {
        uint32_t w[kAhead], s[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int64_t r = r0 + i < rows ? r0 + i : rows - 1;
            w[i] = codes[r * ld_words + word];
            s[i] = scales[r * ld_scales + word / 4];
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (r0 + i >= rows) break;
            float x[8];
            decode8(w[i], s[i], x);
            if (weights) {
                const float f = weights[r0 + i];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= f;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sum[j] += x[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] *= mean;
    store8(agg + at, n - at, sum);
}

template <typename T>
static Encode<T> encode_of(const Values& v, const Held& to)
{
    return {static_cast<const T*>(v.p), v.ld, v.rows, v.n, to.codes, to.ld_words, to.scales, to.ld_scales};
}
static int64_t groups_of(int64_t rows, int64_t n, int64_t per) { return (rows * blocks_of(n) + per - 1) / per; }
static int64_t row_groups(const Values& v, int32_t dtype)
{
    return groups_of(v.rows, v.n, dtype == MV_BF16 ? kGroupBlocks<uint16_t> : kGroupBlocks<float>);
}

mv_status launch_encode(const Values& v, int32_t dtype, const Held& to, float* resid, int64_t ld_resid, hipStream_t st)
{
    if (!count_valid(v.rows, v.n)) return MV_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)row_groups(v, dtype)), threads(kThreads);
#define MV_MX_ENCODE(T, R) hipLaunchKernelGGL((mv_mx_encode_kernel<T, R>), grid, threads, 0, st, encode_of<T>(v, to), resid, ld_resid)
    if (dtype == MV_BF16) {
        if (resid) MV_MX_ENCODE(uint16_t, true);
        else MV_MX_ENCODE(uint16_t, false);
    } else {
        if (resid) MV_MX_ENCODE(float, true);
        else MV_MX_ENCODE(float, false);
    }
#undef MV_MX_ENCODE
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

template <typename T>
static mv_status launch_encode_t_of(const Values& v, const Held& to, hipStream_t st)
{
    const int64_t groups = column_groups<T>(v.rows, v.n);
    if (groups > kMostGroups) return MV_ERR_INVALID_ARG;
    hipLaunchKernelGGL(mv_mx_encode_t_kernel<T>, dim3((uint32_t)groups), dim3(64 * kTileBlocks), 0, st, encode_of<T>(v, to));
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}
mv_status launch_encode_t(const Values& v, int32_t dtype, const Held& to, hipStream_t st)
{
    return dtype == MV_BF16 ? launch_encode_t_of<uint16_t>(v, to, st) : launch_encode_t_of<float>(v, to, st);
}

template <typename T>
static mv_status launch_encode_grad_of(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, hipStream_t st)
{
    const int64_t a = x_t ? column_groups<T>(x.rows, x.n) : 0, b = dy_t ? column_groups<T>(dy.rows, dy.n) : 0;
    const int64_t c = dy_r ? row_groups(dy, sizeof(T) == 2 ? MV_BF16 : MV_F32) : 0;
    if ((dy_r && !count_valid(dy.rows, dy.n)) || a + b + c > kMostGroups) return MV_ERR_INVALID_ARG;
    const Encode<T> none = {};
    hipLaunchKernelGGL(mv_mx_encode_grad_kernel<T>, dim3((uint32_t)(a + b + c)), dim3(kThreads), 0, st,
                       x_t ? encode_of<T>(x, *x_t) : none, (uint32_t)a, dy_t ? encode_of<T>(dy, *dy_t) : none, (uint32_t)b,
                       dy_r ? encode_of<T>(dy, *dy_r) : none);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}
mv_status launch_encode_grad(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, int32_t dtype,
                             hipStream_t st)
{
    return dtype == MV_BF16 ? launch_encode_grad_of<uint16_t>(x, x_t, dy, dy_t, dy_r, st)
                            : launch_encode_grad_of<float>(x, x_t, dy, dy_t, dy_r, st);
}

}  // namespace mvx

extern "C" {

int64_t mv_mx_row_words(int64_t n) { return mvx::size_valid(n) ? 4 * mvx::blocks_of(n) : 0; }
int64_t mv_mx_row_scales(int64_t n) { return mvx::size_valid(n) ? (mvx::blocks_of(n) + 3) / 4 * 4 : 0; }

mv_status mv_mx_encode(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint32_t* codes,
                       int64_t ld_words, uint8_t* scales, int64_t ld_scales, float* resid, int64_t ld_resid, void* stream)
{
    using namespace mvx;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(vals, dtype, ld_vals, n) ||
        !codes_valid(codes, ld_words, scales, ld_scales, n))
        return MV_ERR_INVALID_ARG;
    if (resid && (!values_valid(resid, MV_F32, ld_resid, n) || (vals == resid && (dtype != MV_F32 || ld_vals != ld_resid))))
        return MV_ERR_INVALID_ARG;
    return launch_encode({vals, ld_vals, rows, n}, dtype, {codes, scales, ld_words, ld_scales, rows}, resid, ld_resid,
                         static_cast<hipStream_t>(stream));
}

mv_status mv_mx_encode_t(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint32_t* codes,
                         int64_t ld_words, uint8_t* scales, int64_t ld_scales, void* stream)
{
    using namespace mvx;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(vals, dtype, ld_vals, n) ||
        !codes_valid(codes, ld_words, scales, ld_scales, rows))
        return MV_ERR_INVALID_ARG;
    return launch_encode_t({vals, ld_vals, rows, n}, dtype, {codes, scales, ld_words, ld_scales, n}, static_cast<hipStream_t>(stream));
}

mv_status mv_mx_decode(const uint32_t* codes, int64_t ld_words, const uint8_t* scales, int64_t ld_scales, int64_t rows,
                       int64_t n, void* out, int32_t dtype, int64_t ld_out, void* stream)
{
    using namespace mvx;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(out, dtype, ld_out, n) ||
        !codes_valid(codes, ld_words, scales, ld_scales, n))
        return MV_ERR_INVALID_ARG;
    if (!count_valid(rows, n)) return MV_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)groups_of(rows, n, kThreads / (dtype == MV_BF16 ? kBlockLanes<uint16_t> : kBlockLanes<float>))), threads(kThreads);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == MV_BF16)
        hipLaunchKernelGGL(mv_mx_decode_kernel<uint16_t>, grid, threads, 0, st, codes, ld_words, scales, ld_scales, rows, n,
                           static_cast<uint16_t*>(out), ld_out);
    else
        hipLaunchKernelGGL(mv_mx_decode_kernel<float>, grid, threads, 0, st, codes, ld_words, scales, ld_scales, rows, n,
                           static_cast<float*>(out), ld_out);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

mv_status mv_mx_aggregate(const uint32_t* codes, int64_t ld_words, const uint8_t* scales, int64_t ld_scales, int64_t rows,
                          int64_t n, const float* weights, float* agg, void* stream)
{
    using namespace mvx;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(agg, MV_F32, n, n) ||
        !codes_valid(codes, ld_words, scales, ld_scales, n) || (reinterpret_cast<uintptr_t>(weights) & 3))
        return MV_ERR_INVALID_ARG;
    const int64_t groups = ((n + 7) / 8 + kThreads - 1) / kThreads;
    hipLaunchKernelGGL(mv_mx_aggregate_kernel, dim3((uint32_t)groups), dim3(kThreads), 0, static_cast<hipStream_t>(stream), codes,
                       ld_words, scales, ld_scales, rows, n, weights, weights ? 1.0f : 1.0f / (float)rows, agg);
    return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE;
}

}  // extern "C"
