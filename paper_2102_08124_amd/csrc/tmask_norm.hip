// tmask_layer_norm, tmask_bias_gelu and their gradients: what a training step does between the products with the compressed
// operands.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/tmask.h"
#include "tmask_host.hpp"
#include "tmask_rows.hpp"
#include "tmask_rows_host.hpp"

namespace tmask {

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *y, *total;
    float *mean, *rstd;
    size_t ld_x, ld_residual, ld_y, ld_total;
    uint32_t rows, cols;
    uint32_t param_f32;
    float eps, per_col;                   // 1 / cols
};

struct NormGradArgs {
    const void *dy, *x, *weight, *dtotal;
    const float *mean, *rstd;
    void *dx;
    void *dweight, *dbias;
    float *partial;                       // strips x {dweight, dbias} x pitch
    size_t ld_dy, ld_x, ld_dtotal, ld_dx;
    uint32_t rows, cols;
    uint32_t param_f32;
    uint32_t strips, pitch;               // strips = 1: the sums go straight to dweight and dbias
    uint32_t apart;                       // workgroups beyond the strips, which add up the columns: the strips then do not
    float per_col;
};

struct GeluArgs {
    const void *dy, *x, *bias;            // dy: gradients
    void *out, *dbias;
    float *partial;                       // strips x pitch
    size_t ld_dy, ld_x, ld_out;
    uint32_t rows, cols, chunks;          // chunks of a row, the last of them perhaps cut
    uint32_t param_f32;
    uint32_t lanes_log2;                  // lanes of a workgroup that share a row
    uint32_t groups, strips, pitch;       // workgroups beside each other, and below
};

struct ColumnArgs {
    const float *partial;                 // strips x sums x pitch
    void *out[2];
    uint32_t cols, strips, sums, pitch;
    uint32_t param_f32;
};

__device__ __forceinline__ float load_param(const void *p, uint32_t f32, size_t i) { return f32 ? load_one<kF32>(p, i) : load_one<kBF16>(p, i); }

__device__ __forceinline__ void store_param(void *p, uint32_t f32, size_t i, float v)
{
    if (f32)
        store_one<kF32>(p, i, v);
    else
        store_one<kBF16>(p, i, v);
}

// N parameters from column c on, of which `left` exist
template <int N>
__device__ __forceinline__ void load_params(const void *p, uint32_t f32, uint32_t c, uint32_t left, float (&v)[N])
{
    if (f32) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            if ((uint32_t)e < left) {
                float four[4];
                unpack<kF32>(load_chunk<kF32>(p, c + e, left - e), four);
#pragma unroll
                for (int i = 0; i < 4; i++)
                    v[e + i] = four[i];
            }
    } else if constexpr (N % 8 == 0) {
#pragma unroll
        for (int e = 0; e < N; e += 8)
            if ((uint32_t)e < left) {
                float eight[8];
                unpack<kBF16>(load_chunk<kBF16>(p, c + e, left - e), eight);
#pragma unroll
                for (int i = 0; i < 8; i++)
                    v[e + i] = eight[i];
            }
    } else {
#pragma unroll
        for (int e = 0; e < N; e++)
            if ((uint32_t)e < left)
                v[e] = load_one<kBF16>(p, c + e);
    }
}

template <int N>
__device__ __forceinline__ void store_params(void *p, uint32_t f32, uint32_t c, uint32_t left, const float (&v)[N])
{
    if (f32) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            if ((uint32_t)e < left)
                store_chunk<kF32>(p, c + e, left - e, pack<kF32>({v[e], v[e + 1], v[e + 2], v[e + 3]}));
    } else if constexpr (N == 8) {
        store_chunk<kBF16>(p, c, left, pack<kBF16>(v));
    } else {
#pragma unroll
        for (int e = 0; e < N; e++)
            if ((uint32_t)e < left)
                store_one<kBF16>(p, c + e, v[e]);
    }
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// N sums to 16-byte aligned memory
template <int N>
__device__ __forceinline__ void store_sums(float *p, const float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; e += 4)
        *(f32x4 *)(p + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
}

template <int N>
__device__ __forceinline__ void load_sums(const float *p, float (&v)[N])
{
#pragma unroll
    for (int e = 0; e < N; e += 4) {
        const f32x4 four = *(const f32x4 *)(p + e);
#pragma unroll
        for (int i = 0; i < 4; i++)
            v[e + i] = four[i];
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Layer norm of rows that stay in registers: LANES lanes (a part of a wavefront, or a workgroup of several) with E elements each,
// in chunks of 16 bytes that alternate between the lanes.  The mean first, then the mean of the squared differences
// from it: both from registers, so that a large mean costs no digits and nothing is read twice.  Bound by memory: 8192 rows of 1024 bf16
// with a residual and its sum take 12.5 us (67 MB, 5.4 TB/s, part of it from the memory-side cache), 13731 rows 24 (112 MB, 4.7); one row 3.2 us, a launch.
// More lanes with fewer elements each need a barrier for a row and were slower (13731 x 1024: 26 us).
// ---------------------------------------------------------------------------------------------------------------------
template <int LANES>
constexpr int kNormThreads = LANES <= 256 ? 256 : LANES;

template <int LANES, int T>
__device__ __forceinline__ float row_sum(float v, float *red)
{
    v = lanes_reduce<Sum, LANES < 64 ? LANES : 64>(v);
    if constexpr (LANES > 64) {
        constexpr uint32_t kWaves = LANES / 64;                                 // of a row
        const uint32_t first = threadIdx.x / LANES * kWaves;
        if ((threadIdx.x & 63) == 0)
            red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[first];
#pragma unroll
        for (uint32_t w = 1; w < kWaves; w++)
            v += red[first + w];
    }
    return v;
}

// The thread's row, of those from `first` on: the same for a wavefront if a row has one or more.
template <int LANES>
__device__ __forceinline__ uint32_t row_index(uint32_t first)
{
    const uint32_t r = first + threadIdx.x / LANES;
    return LANES >= 64 ? (uint32_t)__builtin_amdgcn_readfirstlane((int)r) : r;
}

template <int DT, int LANES, int E>
__global__ void __launch_bounds__(kNormThreads<LANES>) norm_kernel(const NormArgs p)
{
    constexpr int T = kNormThreads<LANES>, N = kElems<DT>, C = E / N, kRows = T / LANES;
    __shared__ float red[2][LANES > 64 ? T / 64 : 1];
    const uint32_t lane = threadIdx.x % LANES;
    uint32_t left[C];
#pragma unroll
    for (int i = 0; i < C; i++) {
        const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
        left[i] = c >= p.cols ? 0u : p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
    }
    u32x4 raw[C], more[C];
    auto fetch = [&](uint32_t r) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
            raw[i] = more[i] = u32x4{0u, 0u, 0u, 0u};
            if (left[i] && r < p.rows) {
                raw[i] = fetch_chunk<DT>(row_of<DT>(p.x, r, p.ld_x), c, left[i], p.cols);
                if (p.residual)
                    more[i] = fetch_chunk<DT>(row_of<DT>(p.residual, r, p.ld_residual), c, left[i], p.cols);
            }
        }
    };
    const uint32_t first = row_index<LANES>(blockIdx.x * kRows), step = gridDim.x * kRows;
    fetch(first);                                                               // on the way while the parameters are read
    float w[E], b[E];
#pragma unroll
    for (int i = 0; i < C; i++) {
        const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
        float v[N];
#pragma unroll
        for (int e = 0; e < N; e++)
            v[e] = 1.f;
        if (p.weight && left[i])
            load_params<N>(p.weight, p.param_f32, c, left[i], v);
#pragma unroll
        for (int e = 0; e < N; e++) {
            w[i * N + e] = v[e];
            v[e] = 0.f;
        }
        if (p.bias && left[i])
            load_params<N>(p.bias, p.param_f32, c, left[i], v);
#pragma unroll
        for (int e = 0; e < N; e++)
            b[i * N + e] = v[e];
    }
    const bool whole = p.cols == (uint32_t)(LANES * E);
    uint32_t r = first;
    for (uint32_t r0 = blockIdx.x * kRows; r0 < p.rows; r0 += step, r += step) {  // the same number of rounds for all: barriers are inside
        const bool exists = r < p.rows;
        float t[E], s = 0.f;
#pragma unroll
        for (int i = 0; i < C; i++) {
            float v[N], u[N];
            unpack<DT>(settle<DT>(raw[i], left[i], p.cols), v);
            unpack<DT>(settle<DT>(more[i], left[i], p.cols), u);
#pragma unroll
            for (int e = 0; e < N; e++) {
                v[e] += u[e];
                t[i * N + e] = v[e];
                s += v[e];
            }
            if (p.total && left[i] && exists)
                store_chunk<DT>(row_of<DT>(p.total, r, p.ld_total), (lane + (uint32_t)(i * LANES)) * N, left[i], pack<DT>(v));
        }
        const float mean = row_sum<LANES, T>(s, red[0]) * p.per_col;
        s = 0.f;
#pragma unroll
        for (int i = 0; i < C; i++)
#pragma unroll
            for (int e = 0; e < N; e++) {
                const float d = whole || (uint32_t)e < left[i] ? t[i * N + e] - mean : 0.f;
                t[i * N + e] = d;
                s += d * d;
            }
        const float rstd = 1.f / sqrtf(row_sum<LANES, T>(s, red[1]) * p.per_col + p.eps);
#pragma unroll
        for (int i = 0; i < C; i++) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; e++)
                v[e] = t[i * N + e] * rstd * w[i * N + e] + b[i * N + e];
            if (left[i] && exists)
                store_chunk<DT>(row_of<DT>(p.y, r, p.ld_y), (lane + (uint32_t)(i * LANES)) * N, left[i], pack<DT>(v));
        }
        if (p.mean && lane == 0 && exists) {
            p.mean[r] = mean;
            p.rstd[r] = rstd;
        }
        fetch(r + step);
    }
}

// Rows that no workgroup holds: three passes, the second and third through the caches, with one chunk of a thread in flight.  Bound by those loads'
// latency: 4000 rows of 20480 bf16 with a residual and its sum 192 us, of which 131 are what has to be moved.
constexpr int kLongThreads = 1024;

template <int DT>
__global__ void __launch_bounds__(kLongThreads) norm_long_kernel(const NormArgs p)
{
    constexpr int N = kElems<DT>;
    __shared__ float red[2][kLongThreads / 64];
    for (uint32_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        auto each = [&](auto f) {
            for (uint32_t c = threadIdx.x * N; c < p.cols; c += kLongThreads * N) {
                const uint32_t left = p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
                float v[N], u[N];
                unpack<DT>(load_chunk<DT>(row_of<DT>(p.x, r, p.ld_x), c, left), v);
                if (p.residual) {
                    unpack<DT>(load_chunk<DT>(row_of<DT>(p.residual, r, p.ld_residual), c, left), u);
#pragma unroll
                    for (int e = 0; e < N; e++)
                        v[e] += u[e];
                }
                f(c, left, v);
            }
        };
        float s = 0.f;
        each([&](uint32_t, uint32_t, float (&v)[N]) {
#pragma unroll
            for (int e = 0; e < N; e++)
                s += v[e];
        });
        const float mean = row_sum<kLongThreads, kLongThreads>(s, red[0]) * p.per_col;
        s = 0.f;
        each([&](uint32_t, uint32_t left, float (&v)[N]) {
#pragma unroll
            for (int e = 0; e < N; e++)
                s += (uint32_t)e < left ? (v[e] - mean) * (v[e] - mean) : 0.f;
        });
        const float rstd = 1.f / sqrtf(row_sum<kLongThreads, kLongThreads>(s, red[1]) * p.per_col + p.eps);
        each([&](uint32_t c, uint32_t left, float (&v)[N]) {
            float w[N], b[N];
#pragma unroll
            for (int e = 0; e < N; e++) {
                w[e] = 1.f;
                b[e] = 0.f;
            }
            if (p.weight)
                load_params<N>(p.weight, p.param_f32, c, left, w);
            if (p.bias)
                load_params<N>(p.bias, p.param_f32, c, left, b);
            if (p.total)
                store_chunk<DT>(row_of<DT>(p.total, r, p.ld_total), c, left, pack<DT>(v));
#pragma unroll
            for (int e = 0; e < N; e++)
                v[e] = (v[e] - mean) * rstd * w[e] + b[e];
            store_chunk<DT>(row_of<DT>(p.y, r, p.ld_y), c, left, pack<DT>(v));
        });
        if (p.mean && threadIdx.x == 0) {
            p.mean[r] = mean;
            p.rstd[r] = rstd;
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Its gradients, with rows held the same way.  A workgroup, one on a compute unit, goes through every strips-th group of rows and keeps
// the sums over them of dy h and dy in registers, a column in the same lane all the time; at its end the lanes and wavefronts that share
// a column add up in LDS, and the strips' sums are added up by columns_kernel.  Rows are loaded one ahead.  A short batch needs one launch:
// see norm_grad_columns.  Bound by memory where rows are many (8192 x 1024 bf16 with dtotal: 13.5 us and 2 for the sums, 4.4 TB/s of what
// has to be moved; 30000 x 1024 49 us, 5.0), by the rounds' latencies where they are few (1003 x 2051 fp32 10.5 us).  Twice the strips with
// half the threads move twice the sums (1000 x 4096 bf16, in two launches: 22 us, like this 13).
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kGradThreads = 1024;
constexpr uint32_t kGradStrips = 256;

// `v` over the lanes of a wavefront with the same number modulo LANES
template <int LANES>
__device__ __forceinline__ float across_rows(float v)
{
    if constexpr (LANES <= 8)
        v += dpp<0x128>(v);                         // rows of 16 rotated by 8
    if constexpr (LANES <= 16) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (LANES <= 32) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}

// The column sums of a short batch by workgroups of their own, in the same launch: A lanes a row, as few as make a line of 128 bytes
// and take half of the chip, and all rows.  They read dy and x once more, through the caches, and nothing has to be handed over or waited for.
constexpr uint32_t kApartGroups = kGradStrips / 2;
constexpr int64_t kApartRows = 1024;

template <int DT>
constexpr uint32_t apart_lanes(uint32_t cols)
{
    uint32_t a = 8;
    while (cols > kApartGroups * a * kElems<DT>)
        a *= 2;
    return a;
}

template <int DT, int A>
__device__ __forceinline__ void norm_grad_columns(const NormGradArgs &p, uint32_t group)
{
    constexpr int N = kElems<DT>, W = kGradThreads / 64, kAhead = 2, kWidth = A * N;
    constexpr uint32_t kHigh = kGradThreads / A;
    __shared__ __attribute__((aligned(16))) float sums[W][2][kWidth];
    const uint32_t c = (group * A + threadIdx.x % A) * N, left = c >= p.cols ? 0u : p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
    float dw[N], db[N];
#pragma unroll
    for (int e = 0; e < N; e++)
        dw[e] = db[e] = 0.f;
    if (left)
        for (uint32_t r0 = threadIdx.x / A; r0 < p.rows; r0 += kAhead * kHigh) {
            u32x4 dy[kAhead], x[kAhead];
            float mean[kAhead], rstd[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                const uint32_t r = r0 + (uint32_t)i * kHigh;
                dy[i] = x[i] = u32x4{0u, 0u, 0u, 0u};
                mean[i] = rstd[i] = 0.f;
                if (r < p.rows) {
                    dy[i] = fetch_chunk<DT>(row_of<DT>(p.dy, r, p.ld_dy), c, left, p.cols);
                    x[i] = fetch_chunk<DT>(row_of<DT>(p.x, r, p.ld_x), c, left, p.cols);
                    mean[i] = p.mean[r];
                    rstd[i] = p.rstd[r];
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; i++) {
                float v[N], u[N];
                unpack<DT>(settle<DT>(dy[i], left, p.cols), v);
                unpack<DT>(settle<DT>(x[i], left, p.cols), u);
#pragma unroll
                for (int e = 0; e < N; e++) {
                    dw[e] += v[e] * ((u[e] - mean[i]) * rstd[i]);
                    db[e] += v[e];
                }
            }
        }
#pragma unroll
    for (int e = 0; e < N; e++) {
        dw[e] = across_rows<A>(dw[e]);
        db[e] = across_rows<A>(db[e]);
    }
    if (threadIdx.x % 64u < A) {
        store_sums(&sums[threadIdx.x / 64u][0][threadIdx.x % 64u * N], dw);
        store_sums(&sums[threadIdx.x / 64u][1][threadIdx.x % 64u * N], db);
    }
    __syncthreads();
    if (threadIdx.x < 2u * kWidth) {
        const uint32_t which = threadIdx.x / kWidth, at = threadIdx.x % kWidth, col = group * kWidth + at;
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < W; i++)
            s += sums[i][which][at];
        void *const out = which ? p.dbias : p.dweight;
        if (out && col < p.cols)
            store_param(out, p.param_f32, col, s);
    }
}

// SUMS: with the column sums.
template <int DT, int LANES, int E, bool SUMS>
__device__ __forceinline__ void norm_grad_rows(const NormGradArgs p)
{
    constexpr bool KEEP = E <= 8;                                               // weights, column sums and the next row's loads in registers
    constexpr int T = kGradThreads, N = kElems<DT>, C = E / N, kRows = T / LANES, W = T / 64, kCols = LANES * E;
    constexpr int kShared = LANES < 64 ? W : kRows;                             // sets of column sums that the workgroup adds up
    constexpr bool MORE = DT == kBF16 || LANES < 1024;                          // dtotal ahead too: 128 registers do not hold it besides
    __shared__ float red[2][2 * W];
    // Rows twice as wide as the registers take with all that: the sums lie in LDS, each thread's in its own places (4000 rows of 16000 fp32 with
    // dtotal 209 us, 4.9 TB/s; with sums that spill to scratch memory 385), and the weights are read again for each row.
    __shared__ __attribute__((aligned(16))) float kept[2][KEEP || !SUMS ? 4 : kCols];
    const uint32_t lane = threadIdx.x % LANES;
    // Of a row's chunks the first half is there for every lane: narrower rows have another shape (but for the narrowest).
    constexpr int kThere = LANES > 8 ? C / 2 : 0;
    uint32_t left[C];
#pragma unroll
    for (int i = 0; i < C; i++) {
        const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
        left[i] = i < kThere ? (uint32_t)N : c >= p.cols ? 0u : p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
    }
    struct Row {
        u32x4 dy[C], x[C], more[C];
        float mean, rstd;
    } next;
    auto fetch = [&](uint32_t r, Row &row) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
            row.dy[i] = row.x[i] = row.more[i] = u32x4{0u, 0u, 0u, 0u};
            if (left[i] && r < p.rows) {
                row.dy[i] = fetch_chunk<DT>(row_of<DT>(p.dy, r, p.ld_dy), c, left[i], p.cols);
                row.x[i] = fetch_chunk<DT>(row_of<DT>(p.x, r, p.ld_x), c, left[i], p.cols);
                if (MORE && p.dtotal)
                    row.more[i] = fetch_chunk<DT>(row_of<DT>(p.dtotal, r, p.ld_dtotal), c, left[i], p.cols);
            }
        }
        row.mean = r < p.rows ? p.mean[r] : 0.f;
        row.rstd = r < p.rows ? p.rstd[r] : 0.f;
    };
    const uint32_t step = p.strips * kRows;
    uint32_t r = row_index<LANES>(blockIdx.x * kRows), turn = 0;
    if constexpr (KEEP)
        fetch(r, next);
    constexpr int kHeld = KEEP ? C : 1;
    float w[kHeld][N], dw[kHeld][N], db[kHeld][N];
    auto weights = [&](int i, float (&v)[N]) {
#pragma unroll
        for (int e = 0; e < N; e++)
            v[e] = 1.f;
        if (p.weight && left[i])
            load_params<N>(p.weight, p.param_f32, (lane + (uint32_t)(i * LANES)) * N, left[i], v);
    };
#pragma unroll
    for (int i = 0; i < C; i++) {
        constexpr float none[N] = {};
        if constexpr (KEEP) {
            weights(i, w[i]);
#pragma unroll
            for (int e = 0; e < N; e++)
                dw[i][e] = db[i][e] = 0.f;
        } else if constexpr (SUMS) {
            store_sums(&kept[0][(lane + (uint32_t)(i * LANES)) * N], none);
            store_sums(&kept[1][(lane + (uint32_t)(i * LANES)) * N], none);
        }
    }
    // the same number of rounds for the whole workgroup: barriers are inside
    for (uint32_t r0 = blockIdx.x * kRows; r0 < p.rows; r0 += step, r += step, turn ^= 1) {
        if constexpr (!KEEP)
            fetch(r, next);
        const Row row = next;
        if (KEEP && r0 + step < p.rows)
            fetch(r + step, next);
        const bool exists = r < p.rows;
        u32x4 more[C];
#pragma unroll
        for (int i = 0; i < C; i++) {
            more[i] = row.more[i];
            if (!MORE && p.dtotal && left[i] && exists)
                more[i] = fetch_chunk<DT>(row_of<DT>(p.dtotal, r, p.ld_dtotal), (lane + (uint32_t)(i * LANES)) * N, left[i], p.cols);
        }
        float d[E], h[E], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < C; i++) {
            float v[N], u[N];
            unpack<DT>(settle<DT>(row.dy[i], left[i], p.cols), v);
            unpack<DT>(settle<DT>(row.x[i], left[i], p.cols), u);
            const int at = KEEP ? i : 0;
            if constexpr (!KEEP)
                weights(i, w[0]);
            if constexpr (SUMS && !KEEP) {
                load_sums(&kept[0][(lane + (uint32_t)(i * LANES)) * N], dw[0]);
                load_sums(&kept[1][(lane + (uint32_t)(i * LANES)) * N], db[0]);
            }
#pragma unroll
            for (int e = 0; e < N; e++) {
                const int k = i * N + e;
                // dy is 0 in columns and rows that do not exist
                h[k] = (u[e] - row.mean) * row.rstd;
                if constexpr (SUMS) {
                    dw[at][e] += v[e] * h[k];
                    db[at][e] += v[e];
                }
                d[k] = v[e] * w[at][e];
                s1 += d[k];
            }
            // Not h of columns that do not exist, where the mean times rstd may be beyond all numbers, and 0 times that is none.
            if (p.cols % N) {
#pragma unroll
                for (int e = 0; e < N; e++)
                    if ((uint32_t)e < left[i])
                        s2 += d[i * N + e] * h[i * N + e];
            } else if (left[i]) {
#pragma unroll
                for (int e = 0; e < N; e++)
                    s2 += d[i * N + e] * h[i * N + e];
            }
            if constexpr (SUMS && !KEEP) {
                store_sums(&kept[0][(lane + (uint32_t)(i * LANES)) * N], dw[0]);
                store_sums(&kept[1][(lane + (uint32_t)(i * LANES)) * N], db[0]);
            }
        }
        s1 = lanes_reduce<Sum, LANES < 64 ? LANES : 64>(s1);
        s2 = lanes_reduce<Sum, LANES < 64 ? LANES : 64>(s2);
        if constexpr (LANES > 64) {
            constexpr uint32_t kWaves = LANES / 64;                             // of a row
            const uint32_t wave = threadIdx.x >> 6, first = wave / kWaves * kWaves;
            if ((threadIdx.x & 63) == 0) {
                red[turn][wave] = s1;
                red[turn][W + wave] = s2;
            }
            __syncthreads();
            s1 = red[turn][first];
            s2 = red[turn][W + first];
#pragma unroll
            for (uint32_t k = 1; k < kWaves; k++) {
                s1 += red[turn][first + k];
                s2 += red[turn][W + first + k];
            }
        }
        s1 *= p.per_col;
        s2 *= p.per_col;
#pragma unroll
        for (int i = 0; i < C; i++) {
            float v[N];
            unpack<DT>(settle<DT>(more[i], left[i], p.cols), v);
#pragma unroll
            for (int e = 0; e < N; e++)
                v[e] += row.rstd * (d[i * N + e] - s1 - h[i * N + e] * s2);
            if (left[i] && exists)
                store_chunk<DT>(row_of<DT>(p.dx, r, p.ld_dx), (lane + (uint32_t)(i * LANES)) * N, left[i], pack<DT>(v));
        }
    }
    if (!SUMS || (!p.dweight && !p.dbias))
        return;
    if constexpr (SUMS && kRows == 1) {
#pragma unroll
        for (int i = 0; i < C; i++) {
            const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
            const int at = KEEP ? i : 0;
            if constexpr (!KEEP) {
                load_sums(&kept[0][c], dw[0]);
                load_sums(&kept[1][c], db[0]);
            }
            if (left[i] && p.strips > 1) {
                store_sums(p.partial + (size_t)blockIdx.x * 2 * p.pitch + c, dw[at]);
                store_sums(p.partial + ((size_t)blockIdx.x * 2 + 1) * p.pitch + c, db[at]);
            } else if (left[i]) {
                if (p.dweight)
                    store_params(p.dweight, p.param_f32, c, left[i], dw[at]);
                if (p.dbias)
                    store_params(p.dbias, p.param_f32, c, left[i], db[at]);
            }
        }
    } else if constexpr (SUMS) {
        __shared__ __attribute__((aligned(16))) float sums[kShared][2][kCols];
        const uint32_t set = LANES < 64 ? threadIdx.x >> 6 : threadIdx.x / LANES;
#pragma unroll
        for (int i = 0; i < C; i++) {
#pragma unroll
            for (int e = 0; e < N; e++) {
                dw[i][e] = across_rows<LANES>(dw[i][e]);
                db[i][e] = across_rows<LANES>(db[i][e]);
            }
            if (LANES >= 64 || (threadIdx.x & 63) < (uint32_t)LANES) {
                const uint32_t c = (lane + (uint32_t)(i * LANES)) * N;
                store_sums(&sums[set][0][c], dw[i]);
                store_sums(&sums[set][1][c], db[i]);
            }
        }
        __syncthreads();
        for (uint32_t k = threadIdx.x; k < 2u * kCols; k += T) {
            const uint32_t which = k / kCols, c = k % kCols;
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < kShared; i++)
                s += sums[i][which][c];
            if (c < p.cols && p.strips > 1) {
                p.partial[((size_t)blockIdx.x * 2 + which) * p.pitch + c] = s;
            } else if (c < p.cols) {
                void *const out = which ? p.dbias : p.dweight;
                if (out)
                    store_param(out, p.param_f32, c, s);
            }
        }
    }
}

template <int DT, int LANES, int E>
__global__ void __launch_bounds__(kGradThreads) norm_grad_kernel(const NormGradArgs p)
{
    norm_grad_rows<DT, LANES, E, true>(p);
}

template <int DT, int LANES, int E>
__global__ void __launch_bounds__(kGradThreads) norm_short_grad_kernel(const NormGradArgs p)
{
    if (blockIdx.x < p.strips)
        norm_grad_rows<DT, LANES, E, false>(p);
    else
        norm_grad_columns<DT, (int)apart_lanes<DT>(LANES * E)>(p, blockIdx.x - p.strips);
}

// Rows that no workgroup holds: the sums over rows first (dx may lie over dy or x), a column a thread, then dx in two passes.  4000 rows of 20480 bf16
// with dtotal 266 us (112 for the sums, by loads of one element, and 149), of which 131 are what has to be moved.
template <int DT>
__global__ void __launch_bounds__(kThreads) norm_long_columns_kernel(const NormGradArgs p)
{
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= p.cols)
        return;
    float dw = 0.f, db = 0.f;
    for (uint32_t r = blockIdx.y; r < p.rows; r += p.strips) {
        const float dy = load_one<DT>(p.dy, r * p.ld_dy + c);
        db += dy;
        dw += dy * ((load_one<DT>(p.x, r * p.ld_x + c) - p.mean[r]) * p.rstd[r]);
    }
    float *const out = p.partial + (size_t)blockIdx.y * 2u * p.pitch + c;
    out[0] = dw;
    out[p.pitch] = db;
}

template <int DT>
__global__ void __launch_bounds__(kLongThreads) norm_long_grad_kernel(const NormGradArgs p)
{
    constexpr int N = kElems<DT>;
    __shared__ float red[2][2 * kLongThreads / 64];
    uint32_t turn = 0;
    for (uint32_t r = blockIdx.x; r < p.rows; r += gridDim.x, turn ^= 1) {
        const float mean = p.mean[r], rstd = p.rstd[r];
        auto each = [&](auto f) {
            for (uint32_t c = threadIdx.x * N; c < p.cols; c += kLongThreads * N) {
                const uint32_t left = p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
                float d[N], h[N], w[N];
                unpack<DT>(load_chunk<DT>(row_of<DT>(p.dy, r, p.ld_dy), c, left), d);
                unpack<DT>(load_chunk<DT>(row_of<DT>(p.x, r, p.ld_x), c, left), h);
#pragma unroll
                for (int e = 0; e < N; e++)
                    w[e] = 1.f;
                if (p.weight)
                    load_params<N>(p.weight, p.param_f32, c, left, w);
#pragma unroll
                for (int e = 0; e < N; e++) {
                    d[e] *= w[e];
                    h[e] = (uint32_t)e < left ? (h[e] - mean) * rstd : 0.f;
                }
                f(c, left, d, h);
            }
        };
        float s1 = 0.f, s2 = 0.f;
        each([&](uint32_t, uint32_t, float (&d)[N], float (&h)[N]) {
#pragma unroll
            for (int e = 0; e < N; e++) {
                s1 += d[e];                                                     // d and h are 0 beyond the row
                s2 += d[e] * h[e];
            }
        });
        group_reduce<Sum, Sum, kLongThreads / 64>(s1, s2, red[turn]);
        s1 *= p.per_col;
        s2 *= p.per_col;
        each([&](uint32_t c, uint32_t left, float (&d)[N], float (&h)[N]) {
            float v[N];
#pragma unroll
            for (int e = 0; e < N; e++)
                v[e] = 0.f;
            if (p.dtotal)
                unpack<DT>(load_chunk<DT>(row_of<DT>(p.dtotal, r, p.ld_dtotal), c, left), v);
#pragma unroll
            for (int e = 0; e < N; e++)
                v[e] += rstd * (d[e] - s1 - h[e] * s2);
            store_chunk<DT>(row_of<DT>(p.dx, r, p.ld_dx), c, left, pack<DT>(v));
        });
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// GELU.  With E(a) = exp(-a^2 / 2), the share Phi(u) = (1 + erf(u / sqrt 2)) / 2 that passes is E(u) R(t) for u < 0 and one minus that of -u for
// u > 0, t = 1 / (1 + 0.33 |u|): R is a polynomial of degree 5 without constant term, fitted by linear programming for the least difference of E R
// from the share; it is off by at most 9.2e-8 (the least of all such is 6.6e-8, which the roundings of v_rcp, v_exp and the products hide).  That is for
// bf16, whose rounding is 2e4 times as much.  For fp32 such an R serves from |u| = 1.25 on, where the share's roundings are small, held to
// 1.3e-5 of its own size in the tail and to 1.4e-8 of 1; below, the share is 1/2 + u times a polynomial of degree 5 in u^2, off by 3.6e-9 (y of 0 < u < 1 is off by 1.2e-7 of its
// value, with R alone by 4.2e-7, with an erf by 1.4e-7; the derivative by 1.4e-7, 2.5e-7 and 1.5e-7).  The derivative Phi(u) + u E(u) / sqrt(2 pi) has the same
// exponential.  The form with tanh is the share 1 / (1 + exp(-2 s)).
//
// Bound by memory at size, with the vector ALU not far behind: 8192 x 4096 bf16 28.8 us (134 MB, 4.7 TB/s; 16 instructions an element, of which two
// transcendentals that take four times as long), gradients 43.7 us (201 MB, 4.6 TB/s; 21 instructions).  A library erf instead took 57 us.
// ---------------------------------------------------------------------------------------------------------------------
template <int DT, int FORM, bool GRAD>
__device__ __forceinline__ float gelu(float u)
{
    if constexpr (FORM == TMASK_GELU_ERF && DT == kBF16) {
        const float a = fabsf(u), t = __builtin_amdgcn_rcpf(fmaf(0.33f, a, 1.f));
        const float exponential = __builtin_amdgcn_exp2f(u * u * -0.72134752f);
        float q = fmaf(-0.11074109f, t, 0.37948442f);
        q = fmaf(q, t, -0.09645796f);
        q = fmaf(q, t, 0.20633404f);
        q = fmaf(q, t, 0.12138055f);
        q *= t * exponential;
        if constexpr (GRAD)
            return fmaf(u * 0.39894228f, exponential, u < 0.f ? q : 1.f - q);
        return fmaf(-fabsf(fminf(u, 100.f)), q, fmaxf(u, 0.f));   // u q below 0, u - u q above; q is 0 long before 100, and so +Inf stays; -Inf times 0 is NaN
    } else if constexpr (FORM == TMASK_GELU_ERF) {
        const float a = fabsf(u), u2 = u * u, s = __builtin_amdgcn_rcpf(fmaf(0.4f, a, 1.f));
        const float exponential = __builtin_amdgcn_exp2f(u2 * -0.72134752f);
        float far = fmaf(-0.09980094f, s, 0.17087775f);
        far = fmaf(far, s, 0.10440618f);
        far = fmaf(far, s, 0.16429004f);
        far = fmaf(far, s, 0.15929432f);
        far *= s * exponential;
        float near = fmaf(-6.6448616e-06f, u2, 0.00011032746f);
        near = fmaf(near, u2, -0.0011827096f);
        near = fmaf(near, u2, 0.0099715004f);
        near = fmaf(near, u2, -0.06648999f);
        near = fmaf(near, u2, 0.39894226f);
        const float share = a < 1.25f ? fmaf(u, near, 0.5f) : u < 0.f ? far : 1.f - far;
        return GRAD ? fmaf(u * 0.39894228f, exponential, share) : u * share;
    } else {
        const float u2 = fminf(u * u, 1e4f);                  // the share is 0 or 1 long before; the square stays finite
        if constexpr (GRAD) {
            // From |u|: the smaller of share and 1 - share is e t, to its own size (with share - share^2 the derivative was off by 2e-6 near u = 3.5).
            const float e = __builtin_amdgcn_exp2f(-2.3022082f * fabsf(u) * fmaf(0.044715f, u2, 1.f));
            const float t = __builtin_amdgcn_rcpf(1.f + e), less = e * t;
            return fmaf(u * (less * t) * 1.5957691f, fmaf(0.134145f, u2, 1.f), u < 0.f ? less : t);
        }
        return u * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-2.3022082f * u * fmaf(0.044715f, u2, 1.f)));
    }
}

// Workgroups of 256 threads (1024 for gradients, to have fewer strips) as 2^lanes_log2 lanes of a chunk each by the rest of the
// rows; a thread keeps its columns (and their bias and, for gradients, their sums) and takes kGeluRows rows at a time.
constexpr int kGeluRows = 4;

template <bool GRAD>
constexpr int kGeluThreads = GRAD ? kGradThreads : kThreads;

template <int DT, int FORM, bool GRAD>
__global__ void __launch_bounds__(kGeluThreads<GRAD>) gelu_kernel(const GeluArgs p)
{
    constexpr int N = kElems<DT>, T = kGeluThreads<GRAD>;
    const uint32_t lanes = 1u << p.lanes_log2, high = T >> p.lanes_log2;
    const uint32_t group = blockIdx.x % p.groups, strip = blockIdx.x / p.groups;
    const uint32_t chunk = group * lanes + (threadIdx.x & (lanes - 1u)), y = threadIdx.x >> p.lanes_log2;
    const uint32_t c = chunk * N, left = chunk >= p.chunks ? 0u : p.cols - c < (uint32_t)N ? p.cols - c : (uint32_t)N;
    // Addresses are stepped from row to row: a 64-bit product for each load took a quarter of the kernel's instructions' time.
    const uint32_t step = p.strips * high;
    uint32_t r0 = strip * high + y;
    const unsigned char *px = (const unsigned char *)p.x + (r0 * p.ld_x + c) * kSize<DT>, *pd = (const unsigned char *)p.dy + (r0 * p.ld_dy + c) * kSize<DT>;
    unsigned char *po = (unsigned char *)p.out + (r0 * p.ld_out + c) * kSize<DT>;
    const size_t next_x = step * p.ld_x * kSize<DT>, next_d = step * p.ld_dy * kSize<DT>, next_o = step * p.ld_out * kSize<DT>;
    // the chunk at a row's end: see fetch_chunk
    const uint32_t whole = p.cols >= (uint32_t)N ? (uint32_t)N : left, back = left && left < whole ? (whole - left) * kSize<DT> : 0u;
    px -= back;
    pd -= back;
    u32x4 x[kGeluRows], d[kGeluRows];
    auto fetch = [&]() {                                                        // the rows r0, r0 + step, ...
#pragma unroll
        for (int i = 0; i < kGeluRows; i++) {
            x[i] = d[i] = u32x4{0u, 0u, 0u, 0u};
            if (left && r0 + (uint32_t)i * step < p.rows) {
                x[i] = load_chunk<DT>(px, 0, whole);
                if constexpr (GRAD)
                    d[i] = load_chunk<DT>(pd, 0, whole);
            }
            px += next_x;
            if constexpr (GRAD)
                pd += next_d;
        }
    };
    fetch();                                                                    // on the way while the bias is read
    float b[N], sum[N];
#pragma unroll
    for (int e = 0; e < N; e++)
        b[e] = sum[e] = 0.f;
    if (p.bias && left)
        load_params<N>(p.bias, p.param_f32, c, left, b);
    if (left)
        while (r0 < p.rows) {
#pragma unroll
            for (int i = 0; i < kGeluRows; i++) {
                if (r0 + (uint32_t)i * step < p.rows) {
                    float v[N], u[N];
                    unpack<DT>(settle<DT>(x[i], left, p.cols), v);
                    unpack<DT>(settle<DT>(d[i], left, p.cols), u);
#pragma unroll
                    for (int e = 0; e < N; e++) {
                        v[e] = gelu<DT, FORM, GRAD>(v[e] + b[e]);
                        if constexpr (GRAD) {
                            v[e] *= u[e];
                            sum[e] += v[e];                                     // 0 beyond the row, where dy is 0 and x and bias are
                        }
                    }
                    store_chunk<DT>(po, 0, left, pack<DT>(v));
                }
                po += next_o;
            }
            r0 += kGeluRows * step;
            if (r0 < p.rows)
                fetch();
        }
    if constexpr (GRAD) {
        if (!p.dbias)
            return;
        __shared__ __attribute__((aligned(16))) float sums[T * N];               // [y][lane][element]
        store_sums(sums + threadIdx.x * N, sum);
        __syncthreads();
        const uint32_t width = lanes * N;                                       // columns of the workgroup
        uint32_t sets = high;
        if (width < T) {                                                        // all threads take part first
            sets = T / width;
            float s = 0.f;
            for (uint32_t i = threadIdx.x; i < T * N; i += T)
                s += sums[i];
            __syncthreads();
            sums[threadIdx.x] = s;
            __syncthreads();
        }
        for (uint32_t i = threadIdx.x; i < width; i += T) {
            const uint32_t col = group * width + i;
            float s = 0.f;
            for (uint32_t k = 0; k < sets; k++)
                s += sums[k * width + i];
            if (col < p.cols) {
                if (p.strips > 1)
                    p.partial[(size_t)strip * p.pitch + col] = s;
                else
                    store_param(p.dbias, p.param_f32, col, s);
            }
        }
    }
}

// Adds up the strips' sums: 8 lanes take 32 neighbouring columns (a line of 128 bytes), 32 of these groups every 32nd strip.  Latency:
// 3 to 4 us, whatever the size up to 256 strips of 4096 columns.  There are kGradStrips at most: norm_strips and gelu_tile give no more.
__global__ void __launch_bounds__(kThreads) columns_kernel(const ColumnArgs p)
{
    void *const out = p.out[blockIdx.y];
    if (!out)
        return;
    __shared__ float sums[32][33];
    const uint32_t x = threadIdx.x % 8u, y = threadIdx.x / 8u, c = blockIdx.x * 32u + x * 4u;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (c < p.cols && p.strips) {                                               // the pitch is a multiple of eight
        const float *const from = p.partial + (size_t)blockIdx.y * p.pitch + c;
        const size_t row = (size_t)p.sums * p.pitch;
        constexpr int kAll = kGradStrips / 32;                                  // all there can be, in flight together
        f32x4 v[kAll];
#pragma unroll
        for (int i = 0; i < kAll; i++) {
            const uint32_t k = y + (uint32_t)i * 32u;
            v[i] = *(const f32x4 *)(from + (k < p.strips ? k : 0u) * row);
        }
#pragma unroll
        for (int i = 0; i < kAll; i++)
            if (y + (uint32_t)i * 32u < p.strips)
                s += v[i];
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        sums[y][x * 4 + e] = s[e];
    __syncthreads();
    // 8 lanes a column
    float t = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < 4; k++)
        t += sums[x * 4 + k][y];
    t = lanes_reduce<Sum, 8>(t);
    if (x == 0 && blockIdx.x * 32u + y < p.cols)
        store_param(out, p.param_f32, blockIdx.x * 32u + y, t);
}

// ---------------------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------------------
// How a row is held, by its width.
struct NormShape {
    uint32_t cols, rows, threads;                                               // the widest row; rows of a workgroup at a time
    void (*kernel[2])(const NormArgs);
};

struct NormGradShape {
    uint32_t cols, rows;
    uint32_t apart[2];                                                          // lanes that add up a short batch's columns
    void (*kernel[2])(const NormGradArgs), (*few[2])(const NormGradArgs);
};

#define NORM_SHAPE(LANES, E) {LANES * E, kNormThreads<LANES> / LANES, kNormThreads<LANES>, {norm_kernel<kF32, LANES, E>, norm_kernel<kBF16, LANES, E>}}
static const NormShape kNormShapes[] = {NORM_SHAPE(8, 8), NORM_SHAPE(16, 8), NORM_SHAPE(32, 8), NORM_SHAPE(64, 8), NORM_SHAPE(64, 16),
                                        NORM_SHAPE(256, 8), NORM_SHAPE(256, 16), NORM_SHAPE(512, 16), NORM_SHAPE(1024, 16)};
#undef NORM_SHAPE

#define GRAD_SHAPE(LANES, E)                                                                                                      \
    {LANES * E, kGradThreads / LANES, {apart_lanes<kF32>(LANES * E), apart_lanes<kBF16>(LANES * E)},                              \
     {norm_grad_kernel<kF32, LANES, E>, norm_grad_kernel<kBF16, LANES, E>},                                                       \
     {norm_short_grad_kernel<kF32, LANES, E>, norm_short_grad_kernel<kBF16, LANES, E>}}
static const NormGradShape kNormGradShapes[] = {GRAD_SHAPE(8, 8), GRAD_SHAPE(16, 8), GRAD_SHAPE(32, 8), GRAD_SHAPE(64, 8), GRAD_SHAPE(128, 8),
                                                GRAD_SHAPE(256, 8), GRAD_SHAPE(512, 8), GRAD_SHAPE(1024, 8), GRAD_SHAPE(1024, 16)};
#undef GRAD_SHAPE

// the narrowest that holds the row, none for rows that no workgroup holds
template <typename Shape, size_t n>
static const Shape *shape_for(const Shape (&shapes)[n], int64_t cols)
{
    for (const Shape &s : shapes)
        if (cols <= s.cols)
            return &s;
    return nullptr;
}

static uint32_t at_most(uint64_t v, uint32_t most) { return (uint32_t)(v < most ? v : most); }

// whether two tensors of a call may share memory
static bool overlaps(const void *a, int64_t ld_a, const void *b, int64_t ld_b, int64_t rows, int64_t cols, size_t size)
{
    const uintptr_t pa = (uintptr_t)a, pb = (uintptr_t)b;
    return pa < pb + (size_t)((rows - 1) * ld_b + cols) * size && pb < pa + (size_t)((rows - 1) * ld_a + cols) * size;
}

// Column sums by workgroups of their own (in parentheses: in a second launch), us: 1024 columns of bf16, 200 rows 3.9 (6.4), 600 4.9 (6.7), 1000 6.2 (6.9), 1200
// 7.6 (7.1), 1500 9.5 (7.3), of fp32 600 4.6 (6.8), 1000 7.7 (7.3); 4096 columns of bf16, 1000 rows 9.6 (12.0), 1500 13.1 (13.4); 2051 of fp32, 1003 rows 10.5 (11.1),
// 1500 14.9 (12.8); 12000 of bf16, 200 rows 7.6 (15.2), 1000 22 (30), 1500 31 (40).  One limit for all widths gives away a little on both sides of it.  Not where
// a workgroup would write what another reads.
static bool columns_apart(const tmask_norm_grad_desc &d, size_t size, size_t psize)
{
    if (d.rows > kApartRows)
        return false;
    for (void *const sums : {d.dweight, d.dbias})
        if (sums && ((d.weight && overlaps(sums, 0, d.weight, 0, 1, d.cols, psize)) || sums == d.mean || sums == d.rstd))
            return false;
    return !overlaps(d.dx, d.ld_dx, d.dy, d.ld_dy, d.rows, d.cols, size) && !overlaps(d.dx, d.ld_dx, d.x, d.ld_x, d.rows, d.cols, size);
}

static uint32_t pitch_of(int64_t cols) { return (uint32_t)((cols + 7) & ~7ll); }      // whole chunks of either type

constexpr uint32_t kLongStrips = 64;                                            // of rows that no workgroup holds
static_assert(kLongStrips <= kGradStrips && kGradStrips % 32 == 0, "what columns_kernel adds up");

static uint32_t norm_strips(int64_t rows, int64_t cols)
{
    const NormGradShape *const s = shape_for(kNormGradShapes, cols);
    if (!s)
        return at_most(rows, kLongStrips);
    // Two rounds of one workgroup cost less than a second launch (16 rows of 1024 bf16: 5.1 us, with it 7.2; four rounds 7.5 and 7.3).
    const uint64_t rounds = (rows + s->rows - 1) / s->rows;
    if (rounds <= 2)
        return at_most(rounds, 1);
    if (rounds <= kGradStrips)
        return (uint32_t)rounds;
    // As many rounds for each, where that saves a quarter of the strips (and their sums): 2200 rows of 1024 bf16 on 138 strips 8.4 us, on 256 8.6; 3500 on 219 9.4,
    // on 256 9.3.
    const uint64_t each = (rounds + kGradStrips - 1) / kGradStrips, even = (rounds + each - 1) / each;
    return even <= kGradStrips * 3 / 4 ? (uint32_t)even : kGradStrips;
}

// The tile of GELU's kernels: lanes that waste little at the end of a row, but rather many, since short pieces of rows cut more lines.  `price` is what a place
// costs with 8 ... 256 lanes, set between rows that begin anywhere, where 8 lanes cost 1.8 and 2.2 times as much as 256, and whole lines, where it is 1.1 (gradients
// 1.2).  By 8, 16, 32, 64, 128 and 256 lanes, us: 30000 rows of 1400 fp32 103, 89, 80, 75, 71 (taken), 85, bf16 57, 47, 44, 39 (taken), 46, 38; of 1024 fp32 56, 51, 48, 48, 50,
// 52 (taken), gradients 93, 80, 76, 75, 75, 75 (taken); 8000 rows of 320 fp32 5.3, 5.2 (taken), 5.3, 6.0, 5.9, 5.8, bf16 4.2 (taken), 4.4, 5.7, 5.4, 5.0, 5.2.
static void gelu_tile(int64_t rows, int64_t cols, tmask_dtype dt, bool grad, GeluArgs *p)
{
    const uint32_t n = dt == TMASK_F32 ? 4 : 8;
    p->chunks = (uint32_t)((cols + n - 1) / n);
    static const uint64_t price[9] = {0, 0, 0, 150, 135, 118, 106, 102, 100};
    uint32_t best = 8;
    uint64_t least = ~0ull;
    for (uint32_t l = 8; l >= 3 && (l == 8 || p->chunks < 1u << 20); l--) {
        const uint64_t cost = (((uint64_t)p->chunks + (1u << l) - 1) >> l << l) * price[l];
        if (cost < least) {
            least = cost;
            best = l;
        }
    }
    const auto lanes = [&](uint32_t log2) {
        p->lanes_log2 = log2;
        p->groups = (p->chunks + (1u << log2) - 1) >> log2;
        return (rows + ((int64_t)(grad ? kGradThreads : kThreads) >> log2) - 1) / ((int64_t)(grad ? kGradThreads : kThreads) >> log2);
    };
    p->pitch = pitch_of(cols);
    // Gradients of a short batch: workgroups beside each other alone, few lanes to a row and so all rows in a workgroup, and no second launch.
    // Up to 16 elements a thread, as few as there can be: 20 rows of 4096 bf16 4.2 us (two launches 7.1), 200 4.9 (7.6), 400 7.0 (8.2), with 32
    // elements 8.9.  Four lanes (half a line each) in two rounds at most and on half of the chip: 900 rows of 1001 fp32 in four rounds
    // 9.3 (7.2), 200 of 4096 fp32 by 256 workgroups of them 6.0, by 128 of eight lanes 4.9.
    if (grad && rows > 0 && p->chunks < 1u << 20)
        for (uint32_t rounds = 1; rounds * n <= 16; rounds++)
            for (uint32_t l = best; l >= (rounds <= 2 ? 2u : 3u); l--)
                if (lanes(l) <= rounds && p->groups <= (l == 2 ? kGradStrips / 2 : kGradStrips)) {
                    p->strips = 1;
                    return;
                }
    // (Of the gradients' workgroups a compute unit holds one: one more than there are units doubles the time.)
    const uint64_t rounds = lanes(best), all = grad ? kGradStrips : 2048, most = p->groups < all ? all / p->groups : 1;
    const uint64_t each = rounds <= most ? 1 : grad ? (rounds + most - 1) / most : 0;
    p->strips = (uint32_t)(each ? (rounds + each - 1) / each : most);
}

// columns such that a launch over them stays below 2^32 threads
static bool norm_sizes(int64_t rows, int64_t cols) { return valid_sizes(rows, cols) && cols <= 1ll << 28; }

static int check_head(int64_t rows, int64_t cols, tmask_dtype dt, tmask_dtype param_dt)
{
    if (!known(dt) || !known(param_dt))
        return fail(TMASK_ERR_DTYPE, "unknown dtype %d or parameter dtype %d", (int)dt, (int)param_dt);
    if (!norm_sizes(rows, cols))
        return fail(TMASK_ERR_SHAPE, "rows=%lld (below 2^31) cols=%lld (up to 2^28)", (long long)rows, (long long)cols);
    return TMASK_OK;
}

static void sum_columns(const float *partial, void *out0, void *out1, int64_t cols, uint32_t strips, uint32_t sums, tmask_dtype param_dt, hipStream_t stream)
{
    const ColumnArgs c{partial, {out0, out1}, (uint32_t)cols, strips, sums, pitch_of(cols), param_dt == TMASK_F32};
    hipLaunchKernelGGL(columns_kernel, dim3((uint32_t)((cols + 31) / 32), sums), dim3(kThreads), 0, stream, c);
}

}  // namespace tmask

using namespace tmask;

extern "C" int tmask_layer_norm(const tmask_norm_desc *desc, tmask_dtype dt, tmask_dtype param_dt, float eps, void *hip_stream)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_norm_desc &d = *desc;
    TMASK_TRY(check_head(d.rows, d.cols, dt, param_dt));
    if (!(eps >= 0.f) || std::isinf(eps))
        return fail(TMASK_ERR_SHAPE, "eps=%g must be finite and not negative", (double)eps);
    if (d.rows == 0)
        return TMASK_OK;
    const size_t size = size_of(dt), psize = size_of(param_dt);
    TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size, true));
    TMASK_TRY(check_rows("residual", d.residual, d.ld_residual, d.rows, d.cols, size, d.total != nullptr));
    TMASK_TRY(check_rows("y", d.y, d.ld_y, d.rows, d.cols, size, true));
    TMASK_TRY(check_rows("total", d.total, d.ld_total, d.rows, d.cols, size, false));
    TMASK_TRY(check_vector("weight", d.weight, psize, false));
    TMASK_TRY(check_vector("bias", d.bias, psize, false));
    TMASK_TRY(check_vector("mean", d.mean, 4, d.rstd != nullptr));
    TMASK_TRY(check_vector("rstd", d.rstd, 4, d.mean != nullptr));
    NormArgs p{d.x, d.residual, d.weight, d.bias, d.y, d.total, d.mean, d.rstd, (size_t)d.ld_x, (size_t)d.ld_residual,
               (size_t)d.ld_y, (size_t)d.ld_total, (uint32_t)d.rows, (uint32_t)d.cols, param_dt == TMASK_F32, eps, (float)(1.0 / (double)d.cols)};
    hipStream_t stream = (hipStream_t)hip_stream;
    if (const NormShape *const shape = shape_for(kNormShapes, d.cols))
        hipLaunchKernelGGL(shape->kernel[dt], dim3(at_most((d.rows + shape->rows - 1) / shape->rows, 524288 / shape->threads)), dim3(shape->threads), 0,
                           stream, p);
    else
        hipLaunchKernelGGL(dt == TMASK_F32 ? norm_long_kernel<kF32> : norm_long_kernel<kBF16>, dim3(at_most(d.rows, 512)), dim3(kLongThreads), 0, stream, p);
    return launched("layer norm launch");
}

// Strips' sums of one vector, in floats: at least what norm_strips gives for up to so many rows and columns.
static size_t norm_sums(int64_t rows, int64_t cols)
{
    const NormGradShape *const s = shape_for(kNormGradShapes, cols);
    if (!s) {
        const size_t held = norm_sums(rows, kNormGradShapes[sizeof kNormGradShapes / sizeof *kNormGradShapes - 1].cols);
        const size_t own = (size_t)at_most(rows, kLongStrips) * pitch_of(cols);
        return held > own ? held : own;
    }
    const uint64_t rounds = (rows + s->rows - 1) / s->rows;
    return (size_t)at_most(rounds, rounds <= 2 ? 1 : kGradStrips) * pitch_of(cols);
}

extern "C" size_t tmask_layer_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    return norm_sizes(rows, cols) ? 2u * norm_sums(rows, cols) * 4u : 0;
}

extern "C" int tmask_layer_norm_backward(const tmask_norm_grad_desc *desc, tmask_dtype dt, tmask_dtype param_dt, void *workspace,
                                         size_t workspace_bytes, void *hip_stream)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_norm_grad_desc &d = *desc;
    TMASK_TRY(check_head(d.rows, d.cols, dt, param_dt));
    const size_t size = size_of(dt), psize = size_of(param_dt);
    TMASK_TRY(check_vector("dweight", d.dweight, psize, false));
    TMASK_TRY(check_vector("dbias", d.dbias, psize, false));
    const bool sums = d.dweight || d.dbias;
    if (d.rows == 0 && !sums)
        return TMASK_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    const uint32_t strips = norm_strips(d.rows, d.cols);
    NormGradArgs p{d.dy, d.x, d.weight, d.dtotal, d.mean, d.rstd, d.dx, d.dweight, d.dbias, (float *)workspace, (size_t)d.ld_dy, (size_t)d.ld_x,
                   (size_t)d.ld_dtotal, (size_t)d.ld_dx, (uint32_t)d.rows, (uint32_t)d.cols, param_dt == TMASK_F32, strips, pitch_of(d.cols), 0,
                   (float)(1.0 / (double)d.cols)};
    const NormGradShape *const shape = shape_for(kNormGradShapes, d.cols);
    if (d.rows > 0) {
        TMASK_TRY(check_rows("dy", d.dy, d.ld_dy, d.rows, d.cols, size, true));
        TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size, true));
        TMASK_TRY(check_rows("dtotal", d.dtotal, d.ld_dtotal, d.rows, d.cols, size, false));
        TMASK_TRY(check_rows("dx", d.dx, d.ld_dx, d.rows, d.cols, size, true));
        TMASK_TRY(check_vector("mean", d.mean, 4, true));
        TMASK_TRY(check_vector("rstd", d.rstd, 4, true));
        TMASK_TRY(check_vector("weight", d.weight, psize, false));
        if (sums)
            TMASK_TRY(check_workspace(workspace, workspace_bytes, tmask_layer_norm_workspace_bytes(d.rows, d.cols)));
        if (shape) {
            if (sums && columns_apart(d, size, psize)) {
                const uint32_t width = shape->apart[dt] * (uint32_t)(16 / size);
                p.apart = ((uint32_t)d.cols + width - 1) / width;
                p.strips = at_most((d.rows + shape->rows - 1) / shape->rows, kGradStrips - p.apart);
            }
            hipLaunchKernelGGL(p.apart ? shape->few[dt] : shape->kernel[dt], dim3(p.strips + p.apart), dim3(kGradThreads), 0, stream, p);
        } else {
            if (sums)
                hipLaunchKernelGGL(dt == TMASK_F32 ? norm_long_columns_kernel<kF32> : norm_long_columns_kernel<kBF16>,
                                   dim3((p.cols + kThreads - 1) / kThreads, strips), dim3(kThreads), 0, stream, p);
            hipLaunchKernelGGL(dt == TMASK_F32 ? norm_long_grad_kernel<kF32> : norm_long_grad_kernel<kBF16>, dim3(at_most(d.rows, 512)),
                               dim3(kLongThreads), 0, stream, p);
        }
    }
    if (sums && !p.apart && (strips != 1 || !shape))
        sum_columns(p.partial, d.dweight, d.dbias, d.cols, strips, 2, param_dt, stream);
    return launched("layer norm gradient launch");
}

static int check_form(tmask_gelu_form form)
{
    return form == TMASK_GELU_ERF || form == TMASK_GELU_TANH ? TMASK_OK : fail(TMASK_ERR_DTYPE, "unknown form of GELU %d", (int)form);
}

#define GELU_KERNELS(DT, GRAD) {gelu_kernel<DT, TMASK_GELU_ERF, GRAD>, gelu_kernel<DT, TMASK_GELU_TANH, GRAD>}

extern "C" int tmask_bias_gelu(const tmask_gelu_desc *desc, tmask_dtype dt, tmask_dtype param_dt, tmask_gelu_form form, void *hip_stream)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_gelu_desc &d = *desc;
    TMASK_TRY(check_head(d.rows, d.cols, dt, param_dt));
    TMASK_TRY(check_form(form));
    if (d.rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size_of(dt), true));
    TMASK_TRY(check_rows("y", d.y, d.ld_y, d.rows, d.cols, size_of(dt), true));
    TMASK_TRY(check_vector("bias", d.bias, size_of(param_dt), false));
    GeluArgs p{nullptr, d.x, d.bias, d.y, nullptr, nullptr, 0, (size_t)d.ld_x, (size_t)d.ld_y, (uint32_t)d.rows, (uint32_t)d.cols, 0,
               param_dt == TMASK_F32, 0, 0, 0, 0};
    gelu_tile(d.rows, d.cols, dt, false, &p);
    static void (*const kernels[2][2])(const GeluArgs) = {GELU_KERNELS(kF32, false), GELU_KERNELS(kBF16, false)};
    hipLaunchKernelGGL(kernels[dt][form], dim3(p.groups * p.strips), dim3(kThreads), 0, (hipStream_t)hip_stream, p);
    return launched("GELU launch");
}

// At least what gelu_tile needs for up to so many rows and columns of either type: one strip, or strips of four rows and more and, with
// the workgroups beside each other, at most kGradStrips workgroups of at most 256 chunks.
extern "C" size_t tmask_bias_gelu_workspace_bytes(int64_t rows, int64_t cols)
{
    if (!norm_sizes(rows, cols) || rows == 0)
        return 0;
    constexpr uint64_t kMost = (uint64_t)kGradStrips * 256u * kElems<kBF16>;
    const uint64_t pitch = pitch_of(cols), strips = ((uint64_t)rows + kGradThreads / 256 - 1) / (kGradThreads / 256), all = strips * pitch;
    return (size_t)(all < kMost ? all : kMost > pitch ? kMost : pitch) * 4u;
}

extern "C" int tmask_bias_gelu_backward(const tmask_gelu_grad_desc *desc, tmask_dtype dt, tmask_dtype param_dt, tmask_gelu_form form,
                                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_gelu_grad_desc &d = *desc;
    TMASK_TRY(check_head(d.rows, d.cols, dt, param_dt));
    TMASK_TRY(check_form(form));
    TMASK_TRY(check_vector("dbias", d.dbias, size_of(param_dt), false));
    if (d.rows == 0 && !d.dbias)
        return TMASK_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    GeluArgs p{d.dy, d.x, d.bias, d.dx, d.dbias, (float *)workspace, (size_t)d.ld_dy, (size_t)d.ld_x, (size_t)d.ld_dx, (uint32_t)d.rows,
               (uint32_t)d.cols, 0, param_dt == TMASK_F32, 0, 0, 0, 0};
    gelu_tile(d.rows, d.cols, dt, true, &p);
    if (d.rows > 0) {
        TMASK_TRY(check_rows("dy", d.dy, d.ld_dy, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_rows("dx", d.dx, d.ld_dx, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_vector("bias", d.bias, size_of(param_dt), false));
        if (d.dbias)
            TMASK_TRY(check_workspace(workspace, workspace_bytes, tmask_bias_gelu_workspace_bytes(d.rows, d.cols)));
        static void (*const kernels[2][2])(const GeluArgs) = {GELU_KERNELS(kF32, true), GELU_KERNELS(kBF16, true)};
        hipLaunchKernelGGL(kernels[dt][form], dim3(p.groups * p.strips), dim3(kGradThreads), 0, stream, p);
    }
    if (d.dbias && p.strips != 1)
        sum_columns(p.partial, d.dbias, nullptr, d.cols, p.strips, 1, param_dt, stream);
    return launched("GELU gradient launch");
}
