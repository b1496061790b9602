// 8-bit floating point by blocks of 128 (mv_f8_encode, _encode_t, _decode of include/mv.h).
//
// As with 4 bits each value is read and written once and a few instructions are spent on it: HBM bounds these kernels,
// launches where they are short.  A block is sixteen lanes', eight values each, and its largest magnitude four DPP moves away.
// 16,384 x 8192 rows bf16 70 us, 5.8 TB/s, fp32 119, 5.6; columns 95 and 157, 4.2 and 4.3: their codes go out as single lines
// of 128 bytes, a row apart.  Read back to bf16 66 us, to fp32 112, both 6.0.
#include "mv_f8.hpp"

namespace mvf {

constexpr int kThreads = 256;
constexpr int kLanes = 16;                    // of a block
constexpr int kGroupBlocks = kThreads / kLanes * 2;

// (row, block of the row) of block `first` + `more` of all rows one after the other: a division for the whole workgroup and,
// where a row may end in between, one of small numbers.
struct Place {
    uint32_t row, block;
};
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

// A matrix of values and where its codes go.
template <typename T>
struct Encode {
    const T* vals;
    int64_t  ld_vals, rows, n;
    uint8_t* codes;
    int64_t  ld_bytes;
    uint8_t* scales;
    int64_t  ld_scales;
};

// A lane's values of a block: bf16 eight consecutive ones, as they are; fp32 four and four that lie 64 behind, so that sixteen
// lanes read and write whole runs.
template <typename T>
struct Mine;
template <>
struct Mine<uint16_t> {
    uint32_t x[4];
    __device__ __forceinline__ void load(const uint16_t* p, int64_t live, uint32_t lane) { mvx::load8(p + 8 * lane, live - 8 * lane, x); }
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) t = top2(t, x[i]);
        return top_of_pair(t);
    }
    __device__ __forceinline__ void store(uint8_t* p, uint32_t scale, uint32_t lane) const
    {
        *reinterpret_cast<u32x2*>(p + 8 * lane) = encode8(x, scale);
    }
};
template <>
struct Mine<float> {
    float x[2][4];
    __device__ __forceinline__ void load(const float* p, int64_t live, uint32_t lane)
    {
        mvx::load4(p + 4 * lane, live - 4 * lane, x[0]);
        mvx::load4(p + 64 + 4 * lane, live - 64 - 4 * lane, x[1]);
    }
    __device__ __forceinline__ uint32_t top() const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(x[i / 4][i % 4]) & 0x7FFFFFFFu);
        return t;
    }
    __device__ __forceinline__ void store(uint8_t* p, uint32_t scale, uint32_t lane) const
    {
        const float power = power_of(scale);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<uint32_t*>(p + 64 * h + 4 * lane) =
                scale == kNanScale ? 0u : encode4(x[h][0], x[h][1], x[h][2], x[h][3], power);
    }
};

template <typename T>
__device__ __forceinline__ void encode_rows(const Encode<T>& e, uint32_t at_group)
{
    const uint32_t lane = threadIdx.x % kLanes;
    Place   p[2];
    Mine<T> mine[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        p[u] = place_of(at_group * kGroupBlocks, u * (kThreads / kLanes) + threadIdx.x / kLanes, (uint32_t)blocks_of(e.n));
        const int64_t at = (int64_t)p[u].block * kBlock;
        mine[u].load(e.vals + p[u].row * e.ld_vals + at, p[u].row < e.rows ? e.n - at : 0, lane);
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        if (p[u].row >= e.rows) break;                 // all lanes of a block
        const uint32_t scale = scale_of(top_of_sixteen(mine[u].top()));
        mine[u].store(e.codes + p[u].row * e.ld_bytes + (int64_t)p[u].block * kBlock, scale, lane);
        if (lane == 0) e.scales[p[u].row * e.ld_scales + p[u].block] = (uint8_t)scale;
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mv_f8_encode_kernel(Encode<T> e)
{
    encode_rows(e, blockIdx.x);
}

// Columns: four wavefronts take 128 rows, one block, of 16 bytes of columns in each group of four lanes; lane r of a group has
// rows 8 r .. 8 r + 8 of its wavefront's 32, of each column two words of codes.  A column's largest magnitude is two DPP moves
// and a look at the four wavefronts' away; its codes go out through LDS as the 128 bytes that they are, their 16-byte units in
// the order unit ^ (group % 8) against bank conflicts.  bf16 values stay in pairs until they are codes (4096 x 8192 25.0 -> 21.5 us).
template <typename T>
constexpr int kLaneCols = 16 / (int)sizeof(T);
template <typename T>
constexpr int kTileCols = 16 * kLaneCols<T>;
// A lane's 8 rows of 16 bytes: bf16 two columns to a word, as they are.  Four words of largest magnitudes, of a column each or
// of two.
template <typename T>
struct Strip;
template <>
struct Strip<uint16_t> {
    static constexpr int kOf = 2;   // columns of a word
    uint32_t x[8][4];
    __device__ __forceinline__ void load(int i, const uint16_t* p) { load(i, p, 8); }
    __device__ __forceinline__ void load(int i, const uint16_t* p, int64_t live) { mvx::load8(p, live, x[i]); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return top2(a, b); }
    static __device__ __forceinline__ uint32_t top_of(uint32_t t, uint32_t h) { return h ? t & 0xFFFF0000u : t << 16; }
    __device__ __forceinline__ uint32_t top(int w) const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = top2(t, x[i][w]);
        t = top2(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0xB1, 0xf, 0xf, false));
        return top2(t, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)t, 0x4E, 0xf, 0xf, false));
    }
    // of column h of word w
    __device__ __forceinline__ u32x2 codes(int w, uint32_t h, uint32_t scale) const
    {
        uint32_t y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(x[2 * i + 1][w], x[2 * i][w], h ? 0x07060302u : 0x05040100u);
        return encode8(y, scale);
    }
};
template <>
struct Strip<float> {
    static constexpr int kOf = 1;
    float x[8][4];
    __device__ __forceinline__ void load(int i, const float* p) { load(i, p, 4); }
    __device__ __forceinline__ void load(int i, const float* p, int64_t live) { mvx::load4(p, live, x[i]); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t top_of(uint32_t t, uint32_t) { return t; }
    __device__ __forceinline__ uint32_t top(int w) const
    {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) t = max(t, __float_as_uint(x[i][w]) & 0x7FFFFFFFu);
        return top_of_quad(t);
    }
    __device__ __forceinline__ u32x2 codes(int w, uint32_t, uint32_t scale) const
    {
        const float y[8] = {x[0][w], x[1][w], x[2][w], x[3][w], x[4][w], x[5][w], x[6][w], x[7][w]};
        return encode8(y, scale);
    }
};
template <typename T>
struct Columns {                    // of a workgroup: largest magnitudes, and codes on their way out
    uint32_t tops[4][64];
    uint8_t  codes[kTileCols<T> * kBlock];
    __device__ __forceinline__ uint32_t top(uint32_t w) const
    {
        return Strip<T>::larger(Strip<T>::larger(tops[0][w], tops[1][w]), Strip<T>::larger(tops[2][w], tops[3][w]));
    }
};
template <typename T>
inline int64_t column_groups(int64_t rows, int64_t n)
{
    return (n + kTileCols<T> - 1) / kTileCols<T> * blocks_of(rows);
}

template <typename T>
__device__ __forceinline__ void encode_columns(const Encode<T>& e, uint32_t at_group, Columns<T>& out)
{
    constexpr int kCols = kLaneCols<T>;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x / 64, group = lane / 4, r = lane & 3u;
    const uint32_t tiles = (uint32_t)((e.n + kTileCols<T> - 1) / kTileCols<T>), tile = at_group % tiles, block = at_group / tiles;
    const int64_t col = (int64_t)tile * kTileCols<T> + group * kCols, row = (int64_t)block * kBlock + 32 * wave + 8 * r;
    Strip<T> x;
    const T* p = e.vals + row * e.ld_vals + col;
    if ((int64_t)(block + 1) * kBlock <= e.rows && (int64_t)(tile + 1) * kTileCols<T> <= e.n) {      // the same for all
#pragma unroll
        for (int i = 0; i < 8; ++i) x.load(i, p + i * e.ld_vals);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.load(i, p + i * e.ld_vals, row + i < e.rows ? e.n - col : 0);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t top = x.top(w);
        if (r == 0) out.tops[wave][group * 4 + w] = top;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t top = out.top(group * 4 + w), unit = 2 * wave + r / 2;
#pragma unroll
        for (uint32_t h = 0; h < Strip<T>::kOf; ++h) {
            const uint32_t c = group * kCols + w * Strip<T>::kOf + h;
            *reinterpret_cast<u32x2*>(out.codes + c * kBlock + (unit ^ (group & 7u)) * 16 + (r & 1u) * 8) =
                x.codes(w, h, scale_of(Strip<T>::top_of(top, h)));
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kTileCols<T> / 32; ++i) {
        const uint32_t c = i * 32 + threadIdx.x / 8, unit = threadIdx.x % 8;
        const int64_t to = (int64_t)tile * kTileCols<T> + c;
        if (to < e.n) {
            *reinterpret_cast<u32x4*>(e.codes + to * e.ld_bytes + (int64_t)block * kBlock + unit * 16) =
                *reinterpret_cast<const u32x4*>(out.codes + c * kBlock + (unit ^ (c / kCols & 7u)) * 16);
            if (unit == 0)
                e.scales[to * e.ld_scales + block] = (uint8_t)scale_of(Strip<T>::top_of(out.top(c / Strip<T>::kOf), c % Strip<T>::kOf));
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mv_f8_encode_t_kernel(Encode<T> e)
{
    __shared__ __attribute__((aligned(16))) Columns<T> out;
    encode_columns<T>(e, blockIdx.x, out);
}

// What a layer's gradients need, in one launch: columns of x, columns of dy, rows of dy; none of a kind: no workgroups.
template <typename T>
__global__ __launch_bounds__(kThreads) void mv_f8_encode_grad_kernel(Encode<T> x_t, uint32_t x_t_groups, Encode<T> dy_t,
                                                                     uint32_t dy_t_groups, Encode<T> dy)
{
    __shared__ __attribute__((aligned(16))) Columns<T> out;
    const uint32_t b = blockIdx.x;
    if (b < x_t_groups) encode_columns<T>(x_t, b, out);
    else if (b < x_t_groups + dy_t_groups) encode_columns<T>(dy_t, b - x_t_groups, out);
    else encode_rows<T>(dy, b - x_t_groups - dy_t_groups);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void mv_f8_decode_kernel(const uint8_t* __restrict__ codes, int64_t ld_bytes,
                                                                const uint8_t* __restrict__ scales, int64_t ld_scales,
                                                                int64_t rows, int64_t n, T* __restrict__ out, int64_t ld_out)
{
    const uint32_t lane = threadIdx.x % kLanes;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const Place p = place_of(blockIdx.x * kGroupBlocks, u * (kThreads / kLanes) + threadIdx.x / kLanes, (uint32_t)blocks_of(n));
        if (p.row >= rows) break;
        const int64_t at = (int64_t)p.block * kBlock;
        const uint8_t* from = codes + p.row * ld_bytes + at;
        T* to = out + p.row * ld_out + at;
        const uint32_t scale = scales[p.row * ld_scales + p.block];
        float x[8];
        if constexpr (sizeof(T) == 2) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(from + 8 * lane);
            decode4(w.x, scale, x);
            decode4(w.y, scale, x + 4);
            mvx::store8(to + 8 * lane, n - at - 8 * lane, x);
        } else {
            decode4(*reinterpret_cast<const uint32_t*>(from + 4 * lane), scale, x);
            decode4(*reinterpret_cast<const uint32_t*>(from + 64 + 4 * lane), scale, x + 4);
            mvx::store4(to + 4 * lane, n - at - 4 * lane, x);
            mvx::store4(to + 64 + 4 * lane, n - at - 64 - 4 * lane, x + 4);
        }
    }
}

template <typename T>
static Encode<T> encode_of(const Values& v, const Held& to)
{
    return {static_cast<const T*>(v.p), v.ld, v.rows, v.n, to.codes, to.ld_bytes, to.scales, to.ld_scales};
}
static int64_t groups_of(int64_t rows, int64_t n, int64_t per) { return (rows * blocks_of(n) + per - 1) / per; }
static mv_status done() { return hipGetLastError() == hipSuccess ? MV_OK : MV_ERR_DEVICE; }

mv_status launch_encode(const Values& v, int32_t dtype, const Held& to, hipStream_t st)
{
    if (!count_valid(v.rows, v.n)) return MV_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)groups_of(v.rows, v.n, kGroupBlocks)), threads(kThreads);
    if (dtype == MV_BF16) hipLaunchKernelGGL(mv_f8_encode_kernel<uint16_t>, grid, threads, 0, st, encode_of<uint16_t>(v, to));
    else hipLaunchKernelGGL(mv_f8_encode_kernel<float>, grid, threads, 0, st, encode_of<float>(v, to));
    return done();
}

template <typename T>
static mv_status launch_encode_t_of(const Values& v, const Held& to, hipStream_t st)
{
    const int64_t groups = column_groups<T>(v.rows, v.n);
    if (groups > kMostGroups) return MV_ERR_INVALID_ARG;
    hipLaunchKernelGGL(mv_f8_encode_t_kernel<T>, dim3((uint32_t)groups), dim3(kThreads), 0, st, encode_of<T>(v, to));
    return done();
}
mv_status launch_encode_t(const Values& v, int32_t dtype, const Held& to, hipStream_t st)
{
    return dtype == MV_BF16 ? launch_encode_t_of<uint16_t>(v, to, st) : launch_encode_t_of<float>(v, to, st);
}

template <typename T>
static mv_status launch_encode_grad_of(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, hipStream_t st)
{
    const int64_t a = x_t ? column_groups<T>(x.rows, x.n) : 0, b = dy_t ? column_groups<T>(dy.rows, dy.n) : 0;
    const int64_t c = dy_r ? groups_of(dy.rows, dy.n, kGroupBlocks) : 0;
    if ((dy_r && !count_valid(dy.rows, dy.n)) || a + b + c > kMostGroups) return MV_ERR_INVALID_ARG;
    const Encode<T> none = {};
    hipLaunchKernelGGL(mv_f8_encode_grad_kernel<T>, dim3((uint32_t)(a + b + c)), dim3(kThreads), 0, st,
                       x_t ? encode_of<T>(x, *x_t) : none, (uint32_t)a, dy_t ? encode_of<T>(dy, *dy_t) : none, (uint32_t)b,
                       dy_r ? encode_of<T>(dy, *dy_r) : none);
    return done();
}
mv_status launch_encode_grad(const Values& x, const Held* x_t, const Values& dy, const Held* dy_t, const Held* dy_r, int32_t dtype,
                             hipStream_t st)
{
    return dtype == MV_BF16 ? launch_encode_grad_of<uint16_t>(x, x_t, dy, dy_t, dy_r, st)
                            : launch_encode_grad_of<float>(x, x_t, dy, dy_t, dy_r, st);
}

}  // namespace mvf

extern "C" {

int64_t mv_f8_row_bytes(int64_t n) { return mvf::size_valid(n) ? mvf::kBlock * mvf::blocks_of(n) : 0; }
int64_t mv_f8_row_scales(int64_t n) { return mvf::size_valid(n) ? (mvf::blocks_of(n) + 3) / 4 * 4 : 0; }

mv_status mv_f8_encode(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint8_t* codes, int64_t ld_bytes,
                       uint8_t* scales, int64_t ld_scales, void* stream)
{
    using namespace mvf;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(vals, dtype, ld_vals, n) ||
        !codes_valid(codes, ld_bytes, scales, ld_scales, n))
        return MV_ERR_INVALID_ARG;
    return launch_encode({vals, ld_vals, rows, n}, dtype, {codes, scales, ld_bytes, ld_scales, rows}, static_cast<hipStream_t>(stream));
}

mv_status mv_f8_encode_t(const void* vals, int32_t dtype, int64_t ld_vals, int64_t rows, int64_t n, uint8_t* codes, int64_t ld_bytes,
                         uint8_t* scales, int64_t ld_scales, void* stream)
{
    using namespace mvf;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(vals, dtype, ld_vals, n) ||
        !codes_valid(codes, ld_bytes, scales, ld_scales, rows))
        return MV_ERR_INVALID_ARG;
    return launch_encode_t({vals, ld_vals, rows, n}, dtype, {codes, scales, ld_bytes, ld_scales, n}, static_cast<hipStream_t>(stream));
}

mv_status mv_f8_decode(const uint8_t* codes, int64_t ld_bytes, const uint8_t* scales, int64_t ld_scales, int64_t rows, int64_t n,
                       void* out, int32_t dtype, int64_t ld_out, void* stream)
{
    using namespace mvf;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(out, dtype, ld_out, n) ||
        !codes_valid(codes, ld_bytes, scales, ld_scales, n))
        return MV_ERR_INVALID_ARG;
    if (!count_valid(rows, n)) return MV_ERR_INVALID_ARG;
    const dim3 grid((uint32_t)groups_of(rows, n, kGroupBlocks)), threads(kThreads);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == MV_BF16)
        hipLaunchKernelGGL(mv_f8_decode_kernel<uint16_t>, grid, threads, 0, st, codes, ld_bytes, scales, ld_scales, rows, n,
                           static_cast<uint16_t*>(out), ld_out);
    else
        hipLaunchKernelGGL(mv_f8_decode_kernel<float>, grid, threads, 0, st, codes, ld_bytes, scales, ld_scales, rows, n,
                           static_cast<float*>(out), ld_out);
    return done();
}

}  // extern "C"
