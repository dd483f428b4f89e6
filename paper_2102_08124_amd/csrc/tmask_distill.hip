// tmask_distill and tmask_distill_backward: the loss of a pruned model against its dense teacher's top logits, and its gradient.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/tmask.h"
#include "tmask_host.hpp"
#include "tmask_rows.hpp"
#include "tmask_rows_host.hpp"

namespace tmask {

constexpr int kMaxEntries = 1024;         // of a row's list

struct DistillArgs {
    const void *logits, *teacher, *index;
    const float *row_weight;
    float *loss, *row_max, *row_sum;
    void *dlogits;
    size_t ld_logits, ld_teacher, ld_index, ld_dlogits;
    uint32_t rows, vocab, k;
    float temperature;
};

// A row's list in LDS: columns (-1: no entry), teacher's probabilities, student's logits.
struct List {
    int32_t at[kMaxEntries];
    float p[kMaxEntries];
    float z[kMaxEntries];
};

// Fills `list`; the result, the same in every thread: whether the row has an entry.  log_p_shift: log p_j = (t_j - its maximum) / T
// - log_p_shift.  p holds (t_j - maximum) / T until the caller has used it: see list_softmax.
template <int DT, int TDT, int IDX>
__device__ __forceinline__ bool read_list(const DistillArgs &a, uint32_t r, List &list, float *red, float &log_sum, float &t_max)
{
    float m = -INFINITY, some = 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += kThreads) {
        const int64_t at = IDX == 32 ? (int64_t)((const int32_t *)a.index)[r * a.ld_index + j] : ((const int64_t *)a.index)[r * a.ld_index + j];
        const float t = load_one<TDT>(a.teacher, r * a.ld_teacher + j);
        const bool counts = at >= 0 && at < (int64_t)a.vocab && t != -INFINITY;
        list.at[j] = counts ? (int32_t)at : -1;
        list.p[j] = t;
        list.z[j] = counts ? load_one<DT>(a.logits, r * a.ld_logits + (size_t)at) : 0.f;
        if (counts) {
            m = fmaxf(m, t);
            some = 1.f;
        }
    }
    t_max = group_max<kThreads / 64>(m, red);
    some = group_max<kThreads / 64>(some, red);
    float s = 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += kThreads)
        if (list.at[j] >= 0)
            s += expf((list.p[j] - t_max) / a.temperature);
    log_sum = logf(group_sum<kThreads / 64>(s, red));
    return some > 0.f;
}

// what the entries take from column `at`: the sum of their probabilities
__device__ __forceinline__ float share_of(const List &list, uint32_t k, int32_t at)
{
    float s = 0.f;
    for (uint32_t j = 0; j < k; j++)
        if (list.at[j] == at)
            s += list.p[j];
    return s;
}

template <int DT>
__device__ __forceinline__ void write_gradient(const DistillArgs &a, uint32_t r, List &list, bool some, float z_max, float z_sum, float t_max, float t_log_sum)
{
    const float w = (a.row_weight ? a.row_weight[r] : 1.f) * a.temperature;
    const size_t z0 = r * a.ld_logits, d0 = r * a.ld_dlogits;
    const bool none = !some || w == 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += kThreads)
        if (list.at[j] >= 0)
            list.p[j] = expf((list.p[j] - t_max) / a.temperature - t_log_sum);
    __syncthreads();
    for (uint32_t v = threadIdx.x; v < a.vocab; v += kThreads)
        store_one<DT>(a.dlogits, d0 + v, none ? 0.f : w * (expf((load_one<DT>(a.logits, z0 + v) - z_max) / a.temperature) / z_sum));
    __syncthreads();
    for (uint32_t j = threadIdx.x; j < a.k && !none; j += kThreads)
        if (list.at[j] >= 0)
            store_one<DT>(a.dlogits, d0 + (uint32_t)list.at[j],
                          w * (expf((list.z[j] - z_max) / a.temperature) / z_sum - share_of(list, a.k, list.at[j])));
    __syncthreads();
}

template <int DT, int TDT, int IDX>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillArgs a)
{
    __shared__ float red[kThreads / 64];
    __shared__ List list;
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        float t_log_sum, t_max;
        const bool some = read_list<DT, TDT, IDX>(a, r, list, red, t_log_sum, t_max);
        const size_t z0 = r * a.ld_logits;
        float m = -INFINITY;
        for (uint32_t v = threadIdx.x; v < a.vocab; v += kThreads)
            m = fmaxf(m, load_one<DT>(a.logits, z0 + v));
        const float z_max = group_max<kThreads / 64>(m, red);
        float s = 0.f;
        for (uint32_t v = threadIdx.x; v < a.vocab; v += kThreads)
            s += expf((load_one<DT>(a.logits, z0 + v) - z_max) / a.temperature);
        const float z_sum = group_sum<kThreads / 64>(s, red), z_log_sum = logf(z_sum);
        float loss = 0.f;
        for (uint32_t j = threadIdx.x; j < a.k; j += kThreads)
            if (list.at[j] >= 0) {
                const float log_p = (list.p[j] - t_max) / a.temperature - t_log_sum, log_q = (list.z[j] - z_max) / a.temperature - z_log_sum;
                loss += log_q == -INFINITY ? INFINITY : expf(log_p) * (log_p - log_q);
            }
        loss = group_sum<kThreads / 64>(loss, red);
        if (threadIdx.x == 0) {
            a.loss[r] = some ? a.temperature * a.temperature * loss : 0.f;
            if (a.row_max) {
                a.row_max[r] = z_max;
                a.row_sum[r] = z_sum;
            }
        }
        if (a.dlogits)
            write_gradient<DT>(a, r, list, some, z_max, z_sum, t_max, t_log_sum);
    }
}

template <int DT, int TDT, int IDX>
__global__ void __launch_bounds__(kThreads) distill_grad_kernel(const DistillArgs a)
{
    __shared__ float red[kThreads / 64];
    __shared__ List list;
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        float t_log_sum, t_max;
        const bool some = read_list<DT, TDT, IDX>(a, r, list, red, t_log_sum, t_max);
        write_gradient<DT>(a, r, list, some, a.row_max[r], a.row_sum[r], t_max, t_log_sum);
    }
}

// Everything but the outputs; `args` is complete when the result is TMASK_OK and rows > 0.
static int check_distill(const tmask_distill_desc *desc, tmask_dtype dt, tmask_dtype teacher_dt, int index_bits, float temperature,
                         DistillArgs *args)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_distill_desc &d = *desc;
    if (!known(dt) || !known(teacher_dt) || (index_bits != 32 && index_bits != 64))
        return fail(TMASK_ERR_DTYPE, "unknown dtype %d, teacher's dtype %d or index of %d bits", (int)dt, (int)teacher_dt, index_bits);
    if (!valid_sizes(d.rows, d.vocab) || d.k < 0 || d.k > kMaxEntries)
        return fail(TMASK_ERR_SHAPE, "rows=%lld vocab=%lld k=%lld (at most %d)", (long long)d.rows, (long long)d.vocab, (long long)d.k, kMaxEntries);
    if (!(temperature > 0.f) || std::isinf(temperature))
        return fail(TMASK_ERR_SHAPE, "temperature=%g must be finite and positive", (double)temperature);
    if (d.rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_rows("logits", d.logits, d.ld_logits, d.rows, d.vocab, size_of(dt), true));
    TMASK_TRY(check_rows("teacher", d.teacher, d.ld_teacher, d.rows, d.k, size_of(teacher_dt), d.k > 0));
    TMASK_TRY(check_rows("index", d.index, d.ld_index, d.rows, d.k, (size_t)index_bits / 8, d.k > 0));
    TMASK_TRY(check_vector("row_weight", d.row_weight, 4, false));
    TMASK_TRY(check_rows("dlogits", d.dlogits, d.ld_dlogits, d.rows, d.vocab, size_of(dt), false));
    *args = DistillArgs{d.logits, d.teacher, d.index, d.row_weight, d.loss, d.row_max, d.row_sum, d.dlogits, (size_t)d.ld_logits,
                        (size_t)d.ld_teacher, (size_t)d.ld_index, (size_t)d.ld_dlogits, (uint32_t)d.rows, (uint32_t)d.vocab, (uint32_t)d.k, temperature};
    return TMASK_OK;
}

}  // namespace tmask

using namespace tmask;

#define KERNELS(NAME)                                                              \
    {{{NAME<kF32, kF32, 32>, NAME<kF32, kF32, 64>}, {NAME<kF32, kBF16, 32>, NAME<kF32, kBF16, 64>}}, \
     {{NAME<kBF16, kF32, 32>, NAME<kBF16, kF32, 64>}, {NAME<kBF16, kBF16, 32>, NAME<kBF16, kBF16, 64>}}}

extern "C" size_t tmask_distill_workspace_bytes(int64_t rows, int64_t vocab)
{
    (void)rows;
    (void)vocab;
    return 0;
}

extern "C" int tmask_distill(const tmask_distill_desc *desc, tmask_dtype dt, tmask_dtype teacher_dt, int index_bits, float temperature,
                             void *workspace, size_t workspace_bytes, void *hip_stream)
{
    (void)workspace;
    (void)workspace_bytes;
    DistillArgs a;
    TMASK_TRY(check_distill(desc, dt, teacher_dt, index_bits, temperature, &a));
    if (desc->rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_vector("loss", desc->loss, 4, true));
    TMASK_TRY(check_vector("row_max", desc->row_max, 4, desc->row_sum != nullptr));
    TMASK_TRY(check_vector("row_sum", desc->row_sum, 4, desc->row_max != nullptr));
    static void (*const kernels[2][2][2])(const DistillArgs) = KERNELS(distill_kernel);
    hipLaunchKernelGGL(kernels[dt][teacher_dt][index_bits == 64], dim3(a.rows < 65536 ? a.rows : 65536), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return launched("distillation launch");
}

extern "C" int tmask_distill_backward(const tmask_distill_desc *desc, tmask_dtype dt, tmask_dtype teacher_dt, int index_bits, float temperature,
                                      void *hip_stream)
{
    DistillArgs a;
    TMASK_TRY(check_distill(desc, dt, teacher_dt, index_bits, temperature, &a));
    if (desc->rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_vector("row_max", desc->row_max, 4, true));
    TMASK_TRY(check_vector("row_sum", desc->row_sum, 4, true));
    TMASK_TRY(check_rows("dlogits", desc->dlogits, desc->ld_dlogits, desc->rows, desc->vocab, size_of(dt), true));
    static void (*const kernels[2][2][2])(const DistillArgs) = KERNELS(distill_grad_kernel);
    hipLaunchKernelGGL(kernels[dt][teacher_dt][index_bits == 64], dim3(a.rows < 65536 ? a.rows : 65536), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return launched("distillation gradient launch");
}
