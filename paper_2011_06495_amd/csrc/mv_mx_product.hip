// Products of microscaled 4-bit matrices (mv_mx_product, mv_mx_linear, mv_mx_linear_grad of include/mv.h).
//
//   c[i][j] = sum_k a[i][k] b[j][k],  both factors in blocks of 32 along k
//
// One v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 rows of each factor times four blocks: lane l holds row l % 16 of a
// block, 16 bytes of codes, and the block's scale in one byte of a register; which blocks of k the four groups of lanes
// hold does not matter as long as both factors agree.  So a group takes four consecutive blocks of each 16: 64
// consecutive bytes of codes for four instructions, and their four scales in one word.
#include "mv_mx.hpp"

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
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < b.rows) {
                    if constexpr (sizeof(T) == 2) c[i * ld_c + j + e] = (T)narrow(acc[t][u][e]);
                    else c[i * ld_c + j + e] = acc[t][u][e];
                }
        }
    }
}

static mv_status launch_product(const Factor& a, const Factor& b, int64_t k, void* c, int32_t c_dtype, int64_t ld_c, hipStream_t st)
{
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
    return 0;
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
                          static_cast<hipStream_t>(stream));
}

size_t mv_mx_linear_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k)) return 0;
    return code_bytes(m, k) + scale_bytes(m, k);
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
    char* at = static_cast<char*>(scratch);
    const Held q = carve(at, m, k);
    if (const mv_status rc = launch_encode(x, x_dtype, ld_x, m, k, q.codes, q.ld_words, q.scales, q.ld_scales, nullptr, 0, st))
        return rc;
    return launch_product(q.factor(), {w_codes, w_scales, ld_words, ld_scales, n}, k, y, y_dtype, ld_y, st);
}

size_t mv_mx_linear_grad_scratch_bytes(int64_t m, int64_t n, int64_t k)
{
    using namespace mvx;
    if (!size_valid(m) || !size_valid(n) || !size_valid(k)) return 0;
    return code_bytes(m, n) + scale_bytes(m, n) + code_bytes(n, m) + scale_bytes(n, m) + code_bytes(k, m) + scale_bytes(k, m);
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
    if (dx) {
        const Held q = carve(at, m, n);
        if (const mv_status rc = launch_encode(dy, dtype, ld_dy, m, n, q.codes, q.ld_words, q.scales, q.ld_scales, nullptr, 0, st))
            return rc;
        if (const mv_status rc = launch_product(q.factor(), {wt_codes, wt_scales, ld_words, ld_scales, k}, n, dx, dx_dtype, ld_dx, st))
            return rc;
    }
    if (dw) {
        const Held p = carve(at, n, m), q = carve(at, k, m);
        if (const mv_status rc = launch_encode_t(dy, dtype, ld_dy, m, n, p.codes, p.ld_words, p.scales, p.ld_scales, st)) return rc;
        if (const mv_status rc = launch_encode_t(x, dtype, ld_x, m, k, q.codes, q.ld_words, q.scales, q.ld_scales, st)) return rc;
        return launch_product(p.factor(), q.factor(), m, dw, dw_dtype, ld_dw, st);
    }
    return MV_OK;
}

}  // extern "C"
