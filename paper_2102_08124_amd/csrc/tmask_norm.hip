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

// sum over the workgroup, in every thread; `red` has a place for each wavefront and may be used again at once
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float *red)
{
    v = lanes_reduce<Sum, 64>(v);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; w++)
        v += red[w];
    __syncthreads();
    return v;
}

struct NormArgs {
    const void *x, *residual, *weight, *bias;
    void *y, *total;
    float *mean, *rstd;
    size_t ld_x, ld_residual, ld_y, ld_total;
    uint32_t rows, cols;
    float eps;
};

struct NormGradArgs {
    const void *dy, *x, *weight, *dtotal;
    const float *mean, *rstd;
    void *dx;
    float *partial;                       // strips x {dweight, dbias} x cols
    size_t ld_dy, ld_x, ld_dtotal, ld_dx;
    uint32_t rows, cols, strips;
};

struct GeluArgs {
    const void *dy, *x, *bias;            // dy: gradients
    void *out;
    float *partial;                       // strips x cols
    size_t ld_dy, ld_x, ld_out;
    uint32_t rows, cols, strips;
};

struct ColumnArgs {
    const float *partial;                 // strips x (sums x cols)
    void *out[2];
    uint32_t cols, strips, sums;
};

template <int DT, int PDT>
__global__ void __launch_bounds__(kThreads) norm_kernel(const NormArgs p)
{
    __shared__ float red[kThreads / 64];
    for (uint32_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const size_t x0 = r * p.ld_x, r0 = r * p.ld_residual;
        auto total = [&](uint32_t c) {
            const float v = load_one<DT>(p.x, x0 + c);
            return p.residual ? v + load_one<DT>(p.residual, r0 + c) : v;
        };
        float s = 0.f;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads)
            s += total(c);
        const float mean = group_sum<kThreads / 64>(s, red) / (float)p.cols;
        s = 0.f;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads) {
            const float d = total(c) - mean;
            s += d * d;
        }
        const float rstd = 1.f / sqrtf(group_sum<kThreads / 64>(s, red) / (float)p.cols + p.eps);
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads) {
            const float t = total(c);
            const float w = p.weight ? load_one<PDT>(p.weight, c) : 1.f, b = p.bias ? load_one<PDT>(p.bias, c) : 0.f;
            if (p.total)
                store_one<DT>(p.total, r * p.ld_total + c, t);
            store_one<DT>(p.y, r * p.ld_y + c, (t - mean) * rstd * w + b);
        }
        if (p.mean && threadIdx.x == 0) {
            p.mean[r] = mean;
            p.rstd[r] = rstd;
        }
    }
}

template <int DT, int PDT>
__global__ void __launch_bounds__(kThreads) norm_grad_kernel(const NormGradArgs p)
{
    __shared__ float red[kThreads / 64];
    for (uint32_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const float mean = p.mean[r], rstd = p.rstd[r];
        float s1 = 0.f, s2 = 0.f;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads) {
            const float d = load_one<DT>(p.dy, r * p.ld_dy + c) * (p.weight ? load_one<PDT>(p.weight, c) : 1.f);
            s1 += d;
            s2 += d * ((load_one<DT>(p.x, r * p.ld_x + c) - mean) * rstd);
        }
        s1 = group_sum<kThreads / 64>(s1, red) / (float)p.cols;
        s2 = group_sum<kThreads / 64>(s2, red) / (float)p.cols;
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads) {
            const float d = load_one<DT>(p.dy, r * p.ld_dy + c) * (p.weight ? load_one<PDT>(p.weight, c) : 1.f);
            float v = rstd * (d - s1 - (load_one<DT>(p.x, r * p.ld_x + c) - mean) * rstd * s2);
            if (p.dtotal)
                v += load_one<DT>(p.dtotal, r * p.ld_dtotal + c);
            store_one<DT>(p.dx, r * p.ld_dx + c, v);
        }
    }
}

template <int DT>
__global__ void __launch_bounds__(kThreads) norm_columns_kernel(const NormGradArgs p)
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
    float *const out = p.partial + (size_t)blockIdx.y * 2u * p.cols + c;
    out[0] = dw;
    out[p.cols] = db;
}

// u / 2 * (1 + erf(u / sqrt 2)) and its form with tanh, or the derivative
template <int FORM, bool GRAD>
__device__ __forceinline__ float gelu(float u)
{
    if constexpr (FORM == TMASK_GELU_ERF) {
        const float share = 0.5f * (1.f + erff(u * 0.70710678f));
        return GRAD ? share + u * (0.39894228f * __expf(-0.5f * u * u)) : u * share;
    } else {
        const float u2 = fminf(u * u, 1e4f);                  // tanh is 1 long before; the square stays finite
        const float t = tanhf(0.79788456f * u * (1.f + 0.044715f * u2));
        const float share = 0.5f * (1.f + t);
        return GRAD ? share + u * (0.5f * (1.f - t * t) * 0.79788456f * (1.f + 0.134145f * u2)) : u * share;
    }
}

template <int DT, int PDT, int FORM, bool GRAD>
__global__ void __launch_bounds__(kThreads) gelu_kernel(const GeluArgs p)
{
    for (uint32_t r = blockIdx.x; r < p.rows; r += gridDim.x)
        for (uint32_t c = threadIdx.x; c < p.cols; c += kThreads) {
            const float u = load_one<DT>(p.x, r * p.ld_x + c) + (p.bias ? load_one<PDT>(p.bias, c) : 0.f);
            float v = gelu<FORM, GRAD>(u);
            if constexpr (GRAD)
                v *= load_one<DT>(p.dy, r * p.ld_dy + c);
            store_one<DT>(p.out, r * p.ld_out + c, v);
        }
}

template <int DT, int PDT, int FORM>
__global__ void __launch_bounds__(kThreads) gelu_columns_kernel(const GeluArgs p)
{
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= p.cols)
        return;
    const float b = p.bias ? load_one<PDT>(p.bias, c) : 0.f;
    float s = 0.f;
    for (uint32_t r = blockIdx.y; r < p.rows; r += p.strips)
        s += load_one<DT>(p.dy, r * p.ld_dy + c) * gelu<FORM, true>(load_one<DT>(p.x, r * p.ld_x + c) + b);
    p.partial[(size_t)blockIdx.y * p.cols + c] = s;
}

template <int PDT>
__global__ void __launch_bounds__(kThreads) columns_kernel(const ColumnArgs p)
{
    const uint32_t c = blockIdx.x * kThreads + threadIdx.x;
    void *const out = p.out[blockIdx.y];
    if (c >= p.cols || !out)
        return;
    float s = 0.f;
    for (uint32_t k = 0; k < p.strips; k++)
        s += p.partial[((size_t)k * p.sums + blockIdx.y) * p.cols + c];
    store_one<PDT>(out, c, s);
}

constexpr uint32_t kMaxStrips = 512;

static uint32_t strips_of(int64_t rows) { return (uint32_t)(rows < (int64_t)kMaxStrips ? rows : kMaxStrips); }

static int check_head(int64_t rows, int64_t cols, tmask_dtype dt, tmask_dtype param_dt)
{
    if (!known(dt) || !known(param_dt))
        return fail(TMASK_ERR_DTYPE, "unknown dtype %d or parameter dtype %d", (int)dt, (int)param_dt);
    if (!valid_sizes(rows, cols))
        return fail(TMASK_ERR_SHAPE, "rows=%lld cols=%lld", (long long)rows, (long long)cols);
    return TMASK_OK;
}

static uint32_t row_grid(int64_t rows) { return (uint32_t)(rows < 65536 ? rows : 65536); }

static void sum_columns(const ColumnArgs &c, tmask_dtype param_dt, hipStream_t stream)
{
    const dim3 grid((c.cols + kThreads - 1) / kThreads, c.sums);
    hipLaunchKernelGGL(param_dt == TMASK_F32 ? columns_kernel<kF32> : columns_kernel<kBF16>, grid, dim3(kThreads), 0, stream, c);
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
               (size_t)d.ld_y, (size_t)d.ld_total, (uint32_t)d.rows, (uint32_t)d.cols, eps};
    static void (*const kernels[2][2])(const NormArgs) = {{norm_kernel<kF32, kF32>, norm_kernel<kF32, kBF16>},
                                                          {norm_kernel<kBF16, kF32>, norm_kernel<kBF16, kBF16>}};
    hipLaunchKernelGGL(kernels[dt][param_dt], dim3(row_grid(d.rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, p);
    return launched("layer norm launch");
}

extern "C" size_t tmask_layer_norm_workspace_bytes(int64_t rows, int64_t cols)
{
    return valid_sizes(rows, cols) ? (size_t)strips_of(rows) * 2u * (size_t)cols * 4u : 0;
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
    NormGradArgs p{d.dy, d.x, d.weight, d.dtotal, d.mean, d.rstd, d.dx, (float *)workspace, (size_t)d.ld_dy, (size_t)d.ld_x,
                   (size_t)d.ld_dtotal, (size_t)d.ld_dx, (uint32_t)d.rows, (uint32_t)d.cols, strips_of(d.rows)};
    if (d.rows > 0) {
        TMASK_TRY(check_rows("dy", d.dy, d.ld_dy, d.rows, d.cols, size, true));
        TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size, true));
        TMASK_TRY(check_rows("dtotal", d.dtotal, d.ld_dtotal, d.rows, d.cols, size, false));
        TMASK_TRY(check_rows("dx", d.dx, d.ld_dx, d.rows, d.cols, size, true));
        TMASK_TRY(check_vector("mean", d.mean, 4, true));
        TMASK_TRY(check_vector("rstd", d.rstd, 4, true));
        TMASK_TRY(check_vector("weight", d.weight, psize, false));
        if (sums) {
            TMASK_TRY(check_workspace(workspace, workspace_bytes, tmask_layer_norm_workspace_bytes(d.rows, d.cols)));
            // first, since dx may lie over dy or x
            hipLaunchKernelGGL(dt == TMASK_F32 ? norm_columns_kernel<kF32> : norm_columns_kernel<kBF16>,
                               dim3((p.cols + kThreads - 1) / kThreads, p.strips), dim3(kThreads), 0, stream, p);
        }
        static void (*const kernels[2][2])(const NormGradArgs) = {{norm_grad_kernel<kF32, kF32>, norm_grad_kernel<kF32, kBF16>},
                                                                  {norm_grad_kernel<kBF16, kF32>, norm_grad_kernel<kBF16, kBF16>}};
        hipLaunchKernelGGL(kernels[dt][param_dt], dim3(row_grid(d.rows)), dim3(kThreads), 0, stream, p);
    }
    if (sums)
        sum_columns(ColumnArgs{p.partial, {d.dweight, d.dbias}, p.cols, p.strips, 2}, param_dt, stream);
    return launched("layer norm gradient launch");
}

static int check_form(tmask_gelu_form form)
{
    return form == TMASK_GELU_ERF || form == TMASK_GELU_TANH ? TMASK_OK : fail(TMASK_ERR_DTYPE, "unknown form of GELU %d", (int)form);
}

#define GELU_KERNELS(DT, PDT, GRAD) {gelu_kernel<DT, PDT, TMASK_GELU_ERF, GRAD>, gelu_kernel<DT, PDT, TMASK_GELU_TANH, GRAD>}
#define GELU_COLUMNS(DT, PDT) {gelu_columns_kernel<DT, PDT, TMASK_GELU_ERF>, gelu_columns_kernel<DT, PDT, TMASK_GELU_TANH>}

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
    GeluArgs p{nullptr, d.x, d.bias, d.y, nullptr, 0, (size_t)d.ld_x, (size_t)d.ld_y, (uint32_t)d.rows, (uint32_t)d.cols, 0};
    static void (*const kernels[2][2][2])(const GeluArgs) = {{GELU_KERNELS(kF32, kF32, false), GELU_KERNELS(kF32, kBF16, false)},
                                                             {GELU_KERNELS(kBF16, kF32, false), GELU_KERNELS(kBF16, kBF16, false)}};
    hipLaunchKernelGGL(kernels[dt][param_dt][form], dim3(row_grid(d.rows)), dim3(kThreads), 0, (hipStream_t)hip_stream, p);
    return launched("GELU launch");
}

extern "C" size_t tmask_bias_gelu_workspace_bytes(int64_t rows, int64_t cols)
{
    return valid_sizes(rows, cols) ? (size_t)strips_of(rows) * (size_t)cols * 4u : 0;
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
    GeluArgs p{d.dy, d.x, d.bias, d.dx, (float *)workspace, (size_t)d.ld_dy, (size_t)d.ld_x, (size_t)d.ld_dx, (uint32_t)d.rows,
               (uint32_t)d.cols, strips_of(d.rows)};
    if (d.rows > 0) {
        TMASK_TRY(check_rows("dy", d.dy, d.ld_dy, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_rows("x", d.x, d.ld_x, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_rows("dx", d.dx, d.ld_dx, d.rows, d.cols, size_of(dt), true));
        TMASK_TRY(check_vector("bias", d.bias, size_of(param_dt), false));
        if (d.dbias) {
            TMASK_TRY(check_workspace(workspace, workspace_bytes, tmask_bias_gelu_workspace_bytes(d.rows, d.cols)));
            static void (*const columns[2][2][2])(const GeluArgs) = {{GELU_COLUMNS(kF32, kF32), GELU_COLUMNS(kF32, kBF16)},
                                                                     {GELU_COLUMNS(kBF16, kF32), GELU_COLUMNS(kBF16, kBF16)}};
            hipLaunchKernelGGL(columns[dt][param_dt][form], dim3((p.cols + kThreads - 1) / kThreads, p.strips), dim3(kThreads), 0, stream, p);
        }
        static void (*const kernels[2][2][2])(const GeluArgs) = {{GELU_KERNELS(kF32, kF32, true), GELU_KERNELS(kF32, kBF16, true)},
                                                                 {GELU_KERNELS(kBF16, kF32, true), GELU_KERNELS(kBF16, kBF16, true)}};
        hipLaunchKernelGGL(kernels[dt][param_dt][form], dim3(row_grid(d.rows)), dim3(kThreads), 0, stream, p);
    }
    if (d.dbias)
        sum_columns(ColumnArgs{p.partial, {d.dbias, nullptr}, p.cols, p.strips, 1}, param_dt, stream);
    return launched("GELU gradient launch");
}
