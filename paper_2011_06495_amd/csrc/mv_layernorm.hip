// Layer norm and its gradients (mv_layernorm_forward, mv_layernorm_backward of include/mv.h).
//
//   h = (x - mean) rstd,  y = h gamma + beta
//   d = dy gamma,  dx = rstd (d - mean(d) - h mean(d h)),  dgamma = sum over rows of dy h,  dbeta = sum over rows of dy
//
// Memory bounds both: a row is read once, into registers, and written once.  A workgroup takes row after row, with gamma and
// beta (for the gradients: gamma, and the sums for dgamma and dbeta) of its threads' columns in registers, and the next row
// on its way meanwhile.  16,384 x 8192 bf16 forward 98 us, 5.5 TB/s, fp32 199, 5.4; backward 152 and 298, 5.3 and 5.4, the
// join of the workgroups' sums (4 to 5 us) among them.  Rows beyond the registers are read again: 4096 x 30,000 bf16 forward 184 us, 2.7 of
// what one read and one write would be, fp32 335, 2.9; backward (8192 x 16,384) 279 and 498, 2.9 and 3.2.
//
// The mean is formed first and the squares are those of the differences from it; what the mean's own rounding left over,
// the differences' mean, is taken off them and out of the variance, so rows far from zero keep their digits.
#include "mv_rows.hpp"

namespace mvr {

struct Forward {
    const void* x;
    int64_t     ld_x, rows, n;
    Any         gamma, beta;            // p NULL: 1 and 0
    float       eps;
    AnyOut      y;
    int64_t     ld_y;
    float *     mean, *rstd;
};

// A thread's columns of the weights; `other` where there are none.
template <typename T, int LANES, int C>
__device__ __forceinline__ void load_weights(const Any& from, int64_t n, uint32_t t, float other, float (&to)[C][kChunk<T>])
{
    constexpr int V = kChunk<T>;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t col = (int64_t)(c * LANES + t) * V;
        if (from.p) from.load(col, n - col, to[c]);
        else
#pragma unroll
            for (int i = 0; i < V; ++i) to[c][i] = other;
    }
}

// Squares that have left fp32 would make a reciprocal of 0 and so results of beta, which look as if they were some.
__device__ __forceinline__ float rstd_of(float var, float eps)
{
    const float v = (var < 0.0f ? 0.0f : var) + eps;
    return v < kInf ? 1.0f / sqrtf(v) : __builtin_nanf("");
}

// AHEAD: the next row by load_ahead.  Of bf16, whose rows may end in a chunk of up to seven values, 32,768 x 2047 77 -> 61 us, whole
// chunks 32,768 x 4096 107 -> 102; those of 1024 threads, 8192 x 16,384 99 -> 109, and fp32 rows, 32,768 x 1536 78 -> 94, come as others do
// (that is of whole chunks; those that end inside one, x 1023 58 us, x 2047 112, have 4.6 and 4.8 TB/s).
template <typename T, int LANES, int C, bool AHEAD>
__global__ __launch_bounds__(kThreadsOf<LANES>) void mv_layernorm_kernel(Forward f)
{
    constexpr int V = kChunk<T>, kRows = kThreadsOf<LANES> / LANES;
    __shared__ float lds[2][2][LANES / 64];
    Across<LANES> across(lds);
    const uint32_t t = threadIdx.x % LANES;
    const T* x = static_cast<const T*>(f.x);
    const float share = 1.0f / (float)f.n;
    float gamma[C][V], beta[C][V];
    load_weights<T, LANES, C>(f.gamma, f.n, t, 1.0f, gamma);
    load_weights<T, LANES, C>(f.beta, f.n, t, 0.0f, beta);
    Chunk<T> next[C];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (int64_t)(c * LANES + t) * V;
            if constexpr (AHEAD) load_ahead(next[c], x + row * f.ld_x, col, row < f.rows ? f.n - col : 0);
            else next[c].load(x + row * f.ld_x + col, row < f.rows ? f.n - col : 0);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t step = (int64_t)gridDim.x * kRows;
    fetch(row);
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < f.rows; first += step, row += step) {
        Chunk<T> v[C];
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            v[c] = next[c];
            if (AHEAD) v[c].settle((int)f.n - (c * LANES + (int)t) * V);
#pragma unroll
            for (int i = 0; i < V; ++i) sum += v[c].at(i);
        }
        fetch(row + step);
        const float mean = across.sum(sum) * share;
        float more = 0.0f, squares = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t live = f.n - (int64_t)(c * LANES + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float off = i < live ? v[c].at(i) - mean : 0.0f;
                more += off;
                squares = __builtin_fmaf(off, off, squares);
            }
        }
        across.sum2(more, squares);
        more *= share;
        const float rstd = rstd_of(squares * share - more * more, f.eps);
        if (row >= f.rows) continue;
        // the next row is waited for here, or it would be together with these stores
        __builtin_amdgcn_s_waitcnt(kNoLoads);
        if (t == 0) {
            if (f.mean) f.mean[row] = mean + more;
            if (f.rstd) f.rstd[row] = rstd;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (int64_t)(c * LANES + t) * V;
            float y[V];
            v[c].forget();                               // as they came: their differences would take twice the registers
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(((v[c].at(i) - mean) - more) * rstd, gamma[c][i], beta[c][i]);
            f.y.store(row * f.ld_y + col, f.n - col, y);
        }
    }
}

// Rows beyond the registers: read three times, the second and third time out of a cache as far as that goes.
constexpr int kLongThreads = 1024;
template <typename T>
__global__ __launch_bounds__(kLongThreads) void mv_layernorm_long_kernel(Forward f)
{
    constexpr int V = kChunk<T>;
    __shared__ float lds[2][2][kLongThreads / 64];
    Across<kLongThreads> across(lds);
    const T* x = static_cast<const T*>(f.x);
    const float share = 1.0f / (float)f.n;
    for (int64_t row = blockIdx.x; row < f.rows; row += gridDim.x) {
        const T* p = x + row * f.ld_x;
        float sum = 0.0f, mean = 0.0f, more = 0.0f, squares = 0.0f, rstd = 0.0f;
        for (int pass = 0; pass < 3; ++pass) {
            for (int64_t col = (int64_t)threadIdx.x * V; col < f.n; col += kLongThreads * V) {
                Chunk<T> c;
                c.load(p + col, f.n - col);
                const int64_t live = f.n - col;
                if (pass == 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i) sum += c.at(i);
                } else if (pass == 1) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const float v = i < live ? c.at(i) - mean : 0.0f;
                        more += v;
                        squares = __builtin_fmaf(v, v, squares);
                    }
                } else {
                    float gamma[V], beta[V], y[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) gamma[i] = 1.0f, beta[i] = 0.0f;
                    if (f.gamma.p) f.gamma.load(col, live, gamma);
                    if (f.beta.p) f.beta.load(col, live, beta);
#pragma unroll
                    for (int i = 0; i < V; ++i) y[i] = __builtin_fmaf(((c.at(i) - mean) - more) * rstd, gamma[i], beta[i]);
                    f.y.store(row * f.ld_y + col, live, y);
                }
            }
            if (pass == 0) mean = across.sum(sum) * share;
            if (pass == 1) {
                across.sum2(more, squares);
                more *= share;
                rstd = rstd_of(squares * share - more * more, f.eps);
            }
        }
        if (threadIdx.x == 0) {
            if (f.mean) f.mean[row] = mean + more;
            if (f.rstd) f.rstd[row] = rstd;
        }
    }
}

// ---- gradients -----------------------------------------------------------------------------------------------------

struct Backward {
    const void * x, *dy;
    int64_t      ld_x, ld_dy, rows, n;
    Any          gamma;
    const float *mean, *rstd;
    AnyOut       dx;                    // p NULL: not wanted
    int64_t      ld_dx;
    float*       parts;                 // a row of dgamma's and one of dbeta's for each workgroup, `pitch` apart; NULL: not wanted
    int64_t      pitch;
    float*       sums;                  // of long rows: mean(d) and mean(d h)
};

// AHEAD: as there.  bf16 32,768 x 2047 203 -> 100 us, x 1100 126 -> 71, 16,384 x 8192 162 -> 150; fp32 32,768 x 1100 112 -> 92, but x 4096
// 296 -> 309: of fp32 rows up to 2048 only.
template <typename T, int LANES, int C, bool AHEAD>
__global__ __launch_bounds__(kThreadsOf<LANES>) void mv_layernorm_grad_kernel(Backward b)
{
    constexpr int V = kChunk<T>, kRows = kThreadsOf<LANES> / LANES;
    __shared__ float lds[2][2][LANES / 64];
    Across<LANES> across(lds);
    const uint32_t t = threadIdx.x % LANES;
    const T *x = static_cast<const T*>(b.x), *dy = static_cast<const T*>(b.dy);
    const float share = 1.0f / (float)b.n;
    float gamma[C][V], dgamma[C][V] = {}, dbeta[C][V] = {};
    load_weights<T, LANES, C>(b.gamma, b.n, t, 1.0f, gamma);
    Chunk<T> next_x[C], next_dy[C];
    float    next_mean = 0.0f, next_rstd = 0.0f;
    auto fetch = [&](int64_t row) {
        if constexpr (AHEAD) next_mean = b.mean[row < b.rows ? row : b.rows - 1], next_rstd = b.rstd[row < b.rows ? row : b.rows - 1];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (int64_t)(c * LANES + t) * V, live = row < b.rows ? b.n - col : 0;
            if constexpr (AHEAD) {
                load_ahead(next_x[c], x + row * b.ld_x, col, live);
                load_ahead(next_dy[c], dy + row * b.ld_dy, col, live);
            } else {
                next_x[c].load(x + row * b.ld_x + col, live);
                next_dy[c].load(dy + row * b.ld_dy + col, live);
            }
        }
    };
    int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / LANES;
    const int64_t step = (int64_t)gridDim.x * kRows;
    fetch(row);
    for (int64_t first = (int64_t)blockIdx.x * kRows; first < b.rows; first += step, row += step) {
        const bool  live_row = row < b.rows;
        const float mean = live_row ? AHEAD ? next_mean : b.mean[row] : 0.0f, rstd = live_row ? AHEAD ? next_rstd : b.rstd[row] : 0.0f;
        Chunk<T> vx[C], vdy[C];
        float along = 0.0f, both = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            vx[c] = next_x[c], vdy[c] = next_dy[c];
            const int live = live_row ? (int)b.n - (c * LANES + (int)t) * V : 0;
            if (AHEAD) vx[c].settle(live), vdy[c].settle(live);
        }
        fetch(row + step);
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < V; ++i) {                // dy is 0 where a row has ended
                const float g = vdy[c].at(i), h = (vx[c].at(i) - mean) * rstd, d = g * gamma[c][i];
                dgamma[c][i] = __builtin_fmaf(g, h, dgamma[c][i]);
                dbeta[c][i] += g;
                along += d;
                both = __builtin_fmaf(d, h, both);
            }
        if (!b.dx.p) continue;                                           // uniform
        across.sum2(along, both);
        along *= share, both *= share;
        if (!live_row) continue;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int64_t col = (int64_t)(c * LANES + t) * V;
            float dx[V];
            vx[c].forget(), vdy[c].forget();             // as they came: h and d would take four times the registers
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float h = (vx[c].at(i) - mean) * rstd, d = vdy[c].at(i) * gamma[c][i];
                dx[i] = rstd * __builtin_fmaf(-h, both, d - along);
            }
            b.dx.store(row * b.ld_dx + col, b.n - col, dx);
        }
    }
    if (!b.parts) return;
    // the workgroup's rows of threads one after the other
    if constexpr (kRows > 1) {
        __shared__ float shared[2][C * LANES * V];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (threadIdx.x / LANES == r) {
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        float *g = &shared[0][(c * V + i) * LANES + t], *s = &shared[1][(c * V + i) * LANES + t];
                        if (r) dgamma[c][i] += *g, dbeta[c][i] += *s;
                        if (r < kRows - 1) *g = dgamma[c][i], *s = dbeta[c][i];
                    }
            }
            __syncthreads();
        }
        if (threadIdx.x / LANES != kRows - 1) return;
    }
    float* to = b.parts + (int64_t)blockIdx.x * 2 * b.pitch;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int64_t col = (int64_t)(c * LANES + t) * V;
#pragma unroll
        for (int h4 = 0; h4 < V; h4 += 4) {
            mvx::store4(to + col + h4, b.n - col - h4, &dgamma[c][h4], false);
            mvx::store4(to + b.pitch + col + h4, b.n - col - h4, &dbeta[c][h4], false);
        }
    }
}

// Rows beyond the registers: their two means first ...
template <typename T>
__global__ __launch_bounds__(kLongThreads) void mv_layernorm_grad_sums_kernel(Backward b)
{
    constexpr int V = kChunk<T>;
    __shared__ float lds[2][2][kLongThreads / 64];
    Across<kLongThreads> across(lds);
    const float share = 1.0f / (float)b.n;
    for (int64_t row = blockIdx.x; row < b.rows; row += gridDim.x) {
        const T *x = static_cast<const T*>(b.x) + row * b.ld_x, *dy = static_cast<const T*>(b.dy) + row * b.ld_dy;
        const float mean = b.mean[row], rstd = b.rstd[row];
        float along = 0.0f, both = 0.0f;
        for (int64_t col = (int64_t)threadIdx.x * V; col < b.n; col += kLongThreads * V) {
            Chunk<T> cx, cy;
            cx.load(x + col, b.n - col);
            cy.load(dy + col, b.n - col);
            float gamma[V];
#pragma unroll
            for (int i = 0; i < V; ++i) gamma[i] = 1.0f;
            if (b.gamma.p) b.gamma.load(col, b.n - col, gamma);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = i < b.n - col ? cy.at(i) * gamma[i] : 0.0f, h = i < b.n - col ? (cx.at(i) - mean) * rstd : 0.0f;
                along += d;
                both = __builtin_fmaf(d, h, both);
            }
        }
        across.sum2(along, both);
        if (threadIdx.x == 0) b.sums[2 * row] = along * share, b.sums[2 * row + 1] = both * share;
    }
}
// ... then columns: a workgroup takes 256 chunks of them and every gridDim.y-th row.
constexpr int kColumnThreads = 256;
template <typename T>
__global__ __launch_bounds__(kColumnThreads) void mv_layernorm_grad_columns_kernel(Backward b)
{
    constexpr int V = kChunk<T>;
    const int64_t col = ((int64_t)blockIdx.x * kColumnThreads + threadIdx.x) * V, live = b.n - col;
    if (live <= 0) return;
    const T *x = static_cast<const T*>(b.x) + col, *dy = static_cast<const T*>(b.dy) + col;
    float gamma[V], dgamma[V] = {}, dbeta[V] = {};
#pragma unroll
    for (int i = 0; i < V; ++i) gamma[i] = 1.0f;
    if (b.gamma.p) b.gamma.load(col, live, gamma);
    for (int64_t row = blockIdx.y; row < b.rows; row += gridDim.y) {
        Chunk<T> cx, cy;
        cx.load(x + row * b.ld_x, live);
        cy.load(dy + row * b.ld_dy, live);
        const float mean = b.mean[row], rstd = b.rstd[row];
        float dx[V];
        const float along = b.dx.p ? b.sums[2 * row] : 0.0f, both = b.dx.p ? b.sums[2 * row + 1] : 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float g = cy.at(i), h = (cx.at(i) - mean) * rstd;
            dgamma[i] = __builtin_fmaf(g, h, dgamma[i]);
            dbeta[i] += g;
            dx[i] = rstd * __builtin_fmaf(-h, both, g * gamma[i] - along);
        }
        if (b.dx.p) b.dx.store(row * b.ld_dx + col, live, dx);
    }
    if (!b.parts) return;
    float* to = b.parts + (int64_t)blockIdx.y * 2 * b.pitch;
#pragma unroll
    for (int h4 = 0; h4 < V; h4 += 4) {
        mvx::store4(to + col + h4, live - h4, &dgamma[h4], false);
        mvx::store4(to + b.pitch + col + h4, live - h4, &dbeta[h4], false);
    }
}

// dgamma and dbeta: the parts' columns added up, sixteen threads every sixteenth part of four columns, and theirs in order.
__global__ __launch_bounds__(256) void mv_layernorm_join_kernel(const float* __restrict__ parts, uint32_t count, int64_t n, int64_t pitch,
                                                                float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __shared__ f32x4 held[16][16];
    const uint32_t lane = threadIdx.x % 16, part = threadIdx.x / 16;
    for (int64_t first = (int64_t)blockIdx.x * 64; first < 2 * pitch; first += (int64_t)gridDim.x * 64) {
        const int64_t col = first + lane * 4;                            // of the two rows of a part, one behind the other
        f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
        if (col < 2 * pitch) {
            const float* from = parts + col;
            uint32_t p = part;
            for (; p + 112 < count; p += 128)
#pragma unroll
                for (uint32_t u = 0; u < 8; ++u) sum += *reinterpret_cast<const f32x4*>(from + (int64_t)(p + 16 * u) * 2 * pitch);
            // the rest at once, too: one after the other they would take as long as eight times as many (1000 x 1024 bf16 12.4 us, now 10.9)
            if (p < count) {
                f32x4 v[7];
#pragma unroll
                for (uint32_t u = 0; u < 7; ++u) v[u] = *reinterpret_cast<const f32x4*>(from + (int64_t)min(p + 16 * u, count - 1) * 2 * pitch);
#pragma unroll
                for (uint32_t u = 0; u < 7; ++u)
                    if (p + 16 * u < count) sum += v[u];
            }
        }
        held[part][lane] = sum;
        __syncthreads();
        if (part == 0 && col < 2 * pitch) {
#pragma unroll
            for (int p = 1; p < 16; ++p) sum += held[p][lane];
            const bool bias = col >= pitch;
            const int64_t at = bias ? col - pitch : col;
            float* to = bias ? dbeta : dgamma;
            if (to)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (at + i < n) to[at + i] = sum[i];
        }
        __syncthreads();
    }
}

// How a row is held: LANES threads with up to `values` of its values each, or 0: not at all.  Forward, sixteen values a thread are
// as fast as eight, or faster (bf16 16,384 x 8192 98 us, by twice the threads 144).  With the sums for the weights eight
// are (16,384 x 4096 83, with sixteen 90), and rows beyond 8192 do not fit: 1024 threads with sixteen values each leave
// registers (8192 x 16,384 bf16 369 us, fp32 861; read twice from memory 276 and 499).
struct Held {
    int lanes, values;
};
static Held held_of(int64_t n, bool grad)
{
    if (n <= 64 * 16) return {64, n <= 64 * 8 ? 8 : 16};
    for (int lanes : {256, 512, 1024})
        for (int values : {8, 16})
            if (n <= lanes * values && (values == 8 || !grad)) return {lanes, values};
    return {0, 0};
}

template <typename T, int LANES, int C>
static void forward_of(const Forward& f, hipStream_t st)
{
    constexpr int kRows = kThreadsOf<LANES> / LANES;
    const int64_t groups = (f.rows + kRows - 1) / kRows, most = 2048 * 256 / kThreadsOf<LANES>;
    const dim3 grid((uint32_t)(groups < most ? groups : most)), threads(kThreadsOf<LANES>);
    constexpr bool kShort = LANES == 64 && C * kChunk<T> == 8;           // perhaps no chunk long
    if constexpr (sizeof(T) == 2) {
        if (kShort ? f.n >= kChunk<T> : LANES < 1024 || f.n % kChunk<T> != 0) {
            hipLaunchKernelGGL((mv_layernorm_kernel<T, LANES, C, true>), grid, threads, 0, st, f);
            return;
        }
    }
    if constexpr (sizeof(T) == 4 || kShort || LANES == 1024)
        hipLaunchKernelGGL((mv_layernorm_kernel<T, LANES, C, false>), grid, threads, 0, st, f);
}
template <typename T>
static void forward(const Forward& f, const Held& h, hipStream_t st)
{
    constexpr int C = 8 / kChunk<T>;
    switch (h.lanes + h.values) {
    case 64 + 8: return forward_of<T, 64, C>(f, st);
    case 64 + 16: return forward_of<T, 64, 2 * C>(f, st);
    case 256 + 8: return forward_of<T, 256, C>(f, st);
    case 256 + 16: return forward_of<T, 256, 2 * C>(f, st);
    case 512 + 8: return forward_of<T, 512, C>(f, st);
    case 512 + 16: return forward_of<T, 512, 2 * C>(f, st);
    case 1024 + 8: return forward_of<T, 1024, C>(f, st);
    case 1024 + 16: return forward_of<T, 1024, 2 * C>(f, st);
    }
    hipLaunchKernelGGL(mv_layernorm_long_kernel<T>, dim3((uint32_t)(f.rows < 512 ? f.rows : 512)), dim3(kLongThreads), 0, st, f);
}

// Workgroups of the gradients' kernel, each with a part of the weights' sums to be joined: what runs at once, and at least two rows
// each where that leaves 256.  us with 256, 512, 768: bf16 32,768 x 2048 184, 104, 82; 16,384 x 4096 103, 83, 96; 16,384 x 8192
// 164, 169, 176; 300 x 8192 15, 19, 19; fp32 32,768 x 2048 208, 145, 152; 16,384 x 768 42, 38, 45; 2000 x 512 10.8, 12.0, 11.9.
constexpr int64_t kMostParts = 768, kLeastParts = 256;
inline int64_t pitch_of(int64_t n) { return (n + 3) / 4 * 4; }
static int64_t parts_of(int64_t rows, const Held& h, bool bf16)
{
    const int64_t groups = h.lanes == 64 ? (rows + 3) / 4 : rows, most = h.lanes == 1024 ? 256 : h.lanes == 256 && bf16 ? kMostParts : 512;
    int64_t parts = groups / 2 < kLeastParts ? kLeastParts : groups / 2;
    if (parts > most) parts = most;
    return parts < groups ? parts : groups;
}
// Of rows beyond the registers: tiles of columns, and workgroups that share the rows of each.
static int64_t tiles_of(int64_t n, int chunk) { return (n + kColumnThreads * chunk - 1) / (kColumnThreads * chunk); }
static int64_t deep_of(int64_t rows, int64_t n, int chunk)
{
    const int64_t most = tiles_of(n, chunk) < 64 ? 64 : 8;
    return rows < most ? rows : most;
}
// Room for the parts of either type's rows (bf16's are never fewer), and of shorter rows: what is enough for a program's longest ones
// is enough for all of them, though longer ones may have fewer parts.
inline size_t parts_bytes(int64_t rows, int64_t n)
{
    size_t most = 0;
    for (int64_t top : {(int64_t)1024, (int64_t)2048, (int64_t)4096, (int64_t)8192, (int64_t)63 * kColumnThreads * kChunk<uint16_t>, n}) {
        const int64_t at = top < n ? top : n;
        const Held    h = held_of(at, true);
        const int64_t parts = h.lanes ? parts_of(rows, h, true) : deep_of(rows, at, kChunk<uint16_t>);
        const size_t  bytes = (size_t)parts * 2 * (size_t)pitch_of(at) * 4;
        if (bytes > most) most = bytes;
    }
    return most;
}

template <typename T, int LANES, int C>
static uint32_t backward_of(const Backward& b, const Held& h, hipStream_t st)
{
    const uint32_t grid = (uint32_t)parts_of(b.rows, h, sizeof(T) == 2);
    constexpr bool kShort = LANES == 64 && C * kChunk<T> == 8, kNever = LANES > 256 && sizeof(T) == 4, kAlways = !kShort && !kNever;
    if constexpr (!kNever) {
        if (kAlways || b.n >= kChunk<T>) {
            hipLaunchKernelGGL((mv_layernorm_grad_kernel<T, LANES, C, true>), dim3(grid), dim3(kThreadsOf<LANES>), 0, st, b);
            return grid;
        }
    }
    if constexpr (!kAlways)
        hipLaunchKernelGGL((mv_layernorm_grad_kernel<T, LANES, C, false>), dim3(grid), dim3(kThreadsOf<LANES>), 0, st, b);
    return grid;
}
template <typename T>
static uint32_t backward(const Backward& b, const Held& h, hipStream_t st)               // returns how many parts there are
{
    constexpr int C = 8 / kChunk<T>;
    switch (h.lanes + h.values) {
    case 64 + 8: return backward_of<T, 64, C>(b, h, st);
    case 64 + 16: return backward_of<T, 64, 2 * C>(b, h, st);
    case 256 + 8: return backward_of<T, 256, C>(b, h, st);
    case 512 + 8: return backward_of<T, 512, C>(b, h, st);
    case 1024 + 8: return backward_of<T, 1024, C>(b, h, st);
    }
    if (b.dx.p)
        hipLaunchKernelGGL(mv_layernorm_grad_sums_kernel<T>, dim3((uint32_t)(b.rows < 512 ? b.rows : 512)), dim3(kLongThreads), 0, st, b);
    const uint32_t deep = (uint32_t)deep_of(b.rows, b.n, kChunk<T>);
    hipLaunchKernelGGL(mv_layernorm_grad_columns_kernel<T>, dim3((uint32_t)tiles_of(b.n, kChunk<T>), deep), dim3(kColumnThreads), 0, st, b);
    return deep;
}

inline bool weights_valid(const void* p, int32_t dtype) { return !p || values_valid(p, dtype, 1, 1); }
inline bool floats_valid(const float* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }

}  // namespace mvr

extern "C" {

mv_status mv_layernorm_forward(const void* x, int32_t x_dtype, int64_t ld_x, int64_t rows, int64_t n, const void* gamma, const void* beta,
                               int32_t weight_dtype, float eps, void* y, int32_t y_dtype, int64_t ld_y, float* mean, float* rstd,
                               void* stream)
{
    using namespace mvr;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(x, x_dtype, ld_x, n) || !values_valid(y, y_dtype, ld_y, n) ||
        !dtype_valid(weight_dtype) || !weights_valid(gamma, weight_dtype) || !weights_valid(beta, weight_dtype) || !floats_valid(mean) ||
        !floats_valid(rstd) || !(eps >= 0.0f && eps < kInf) || (x == y && (x_dtype != y_dtype || ld_x != ld_y)))
        return MV_ERR_INVALID_ARG;
    const uint32_t bf16 = weight_dtype == MV_BF16;
    const Forward f = {x, ld_x, rows, n, {gamma, bf16}, {beta, bf16}, eps, {y, y_dtype == MV_BF16}, ld_y, mean, rstd};
    const Held h = held_of(n, false);
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (x_dtype == MV_BF16) forward<uint16_t>(f, h, st);
    else forward<float>(f, h, st);
    return launched();
}

size_t mv_layernorm_scratch_bytes(int64_t rows, int64_t n)
{
    using namespace mvr;
    return size_valid(rows) && size_valid(n) ? (size_t)rows * 8 + 16 + parts_bytes(rows, n) : 0;
}

mv_status mv_layernorm_backward(const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, int32_t dtype, int64_t rows, int64_t n,
                                const void* gamma, int32_t weight_dtype, const float* mean, const float* rstd, void* dx, int32_t dx_dtype,
                                int64_t ld_dx, float* dgamma, float* dbeta, void* scratch, size_t scratch_bytes, void* stream)
{
    using namespace mvr;
    if (!size_valid(rows) || !size_valid(n) || !values_valid(x, dtype, ld_x, n) || !values_valid(dy, dtype, ld_dy, n) ||
        !dtype_valid(weight_dtype) || !weights_valid(gamma, weight_dtype) || !mean || !rstd || !floats_valid(mean) || !floats_valid(rstd) ||
        (!dx && !dgamma && !dbeta) || (dx && !values_valid(dx, dx_dtype, ld_dx, n)) || !floats_valid(dgamma) || !floats_valid(dbeta) ||
        !scratch || (reinterpret_cast<uintptr_t>(scratch) & 15) || scratch_bytes < mv_layernorm_scratch_bytes(rows, n) ||
        (dx && dx == x && (dx_dtype != dtype || ld_dx != ld_x)) || (dx && dx == dy && (dx_dtype != dtype || ld_dx != ld_dy)))
        return MV_ERR_INVALID_ARG;
    const size_t sums = ((size_t)rows * 8 + 15) / 16 * 16;
    float* parts = dgamma || dbeta ? reinterpret_cast<float*>(static_cast<char*>(scratch) + sums) : nullptr;
    const Backward b = {x, dy, ld_x, ld_dy, rows, n, {gamma, weight_dtype == MV_BF16}, mean, rstd, {dx, dx_dtype == MV_BF16}, ld_dx,
                        parts, pitch_of(n), static_cast<float*>(scratch)};
    const Held h = held_of(n, true);
    hipStream_t st = static_cast<hipStream_t>(stream);
    const uint32_t count = dtype == MV_BF16 ? backward<uint16_t>(b, h, st) : backward<float>(b, h, st);
    if (parts) {
        const int64_t groups = (2 * b.pitch + 63) / 64;
        hipLaunchKernelGGL(mv_layernorm_join_kernel, dim3((uint32_t)(groups < 65536 ? groups : 65536)), dim3(256), 0, st, parts, count, n,
                           b.pitch, dgamma, dbeta);
    }
    return launched();
}

}  // extern "C"
