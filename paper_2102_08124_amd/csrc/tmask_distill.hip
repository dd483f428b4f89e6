// tmask_distill and tmask_distill_backward: the loss of a pruned model against its dense teacher's top logits, and its gradient.
//
// With p the teacher's distribution over a row's list, q the student's over the vocabulary, both at temperature T:
//     loss = T^2 sum_j p_j (log p_j - log q_at(j))        dz_v = w T (q_v - sum of p_j with at(j) = v)
// Exponentials are of differences from the row's maximum, times log2(e) / T, by the hardware's 2^x; the differences are taken first, so
// that logits of any size (masks of the type's lowest value) neither overflow nor cancel.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/tmask.h"
#include "tmask_host.hpp"
#include "tmask_rows.hpp"
#include "tmask_rows_host.hpp"

namespace tmask {

constexpr uint32_t kMaxEntries = 1024;    // of a row's list
constexpr uint32_t kMaxParts = 64;        // of a row: a lane of a wavefront has one each
constexpr uint32_t kSlice = 256;          // threads of the kernels that work on a part of a row

struct DistillArgs {
    const void *logits, *teacher, *index;
    const float *row_weight;
    float *loss, *row_max, *row_sum;
    void *dlogits;
    float *part_stats;                    // rows x parts x {maximum, sum}
    float *list_logits;                   // rows x k: the student's logits of the entries
    size_t ld_logits, ld_teacher, ld_index, ld_dlogits;
    uint32_t rows, vocab, k;
    uint32_t parts, part_chunks;
    uint32_t teacher_f32, index64;
    uint32_t hash_shift;
    float temperature, per_t2;            // T, log2(e) / T
};

// A row's list in LDS, k numbers each: columns (-1: no entry), the teacher's logits (later: its probabilities), the student's logits.
// table: the columns hashed, to see whether one is there twice.
struct List {
    int32_t *at;
    float *t, *z;
    int32_t *table, *repeats;
};

__device__ __forceinline__ List list_in(void *lds, const DistillArgs &a)
{
    List l;
    l.repeats = (int32_t *)lds;
    l.at = l.repeats + 4;
    l.t = (float *)l.at + a.k;
    l.z = l.t + a.k;
    l.table = (int32_t *)l.z + a.k;
    return l;
}

// of LDS; `table`: with room for it
static size_t list_bytes(const DistillArgs &a, bool table) { return 4u * (4u + 3u * a.k + (a.k && table ? 1u << (32u - a.hash_shift) : 0u)); }

// exp(x / T) for x <= 0
__device__ __forceinline__ float exp_of(const DistillArgs &a, float x) { return __builtin_amdgcn_exp2f(x * a.per_t2); }

// entries that a thread of T reads at a time: all there can be, or four
template <uint32_t T>
constexpr int kEntries = T * 4u > kMaxEntries ? (int)(kMaxEntries / T) : 4;

// Entry j of row r as it lies in memory: nothing is computed from it here, so that a thread's loads are all in flight at once.
struct Entry {
    uint32_t t, lo, hi;
};

__device__ __forceinline__ Entry entry_at(const DistillArgs &a, uint32_t r, uint32_t j)
{
    const size_t i = r * a.ld_index + j, k = r * a.ld_teacher + j;
    Entry e;
    e.hi = 0;
    if (a.index64) {
        const u32x2 at = *(const u32x2 *)((const uint64_t *)a.index + i);
        e.lo = at.x;
        e.hi = at.y;
    } else {
        e.lo = ((const uint32_t *)a.index)[i];
    }
    if (a.teacher_f32)
        e.t = ((const uint32_t *)a.teacher)[k];
    else
        e.t = ((const uint16_t *)a.teacher)[k];
    return e;
}

__device__ __forceinline__ float logit_of(const DistillArgs &a, const Entry &e) { return __uint_as_float(a.teacher_f32 ? e.t : e.t << 16); }

// its column, -1 if it does not count (below 2^31 with the upper half 0, so one unsigned comparison sees negative indexes too)
__device__ __forceinline__ int32_t column_of(const DistillArgs &a, const Entry &e)
{
    return e.hi == 0 && e.lo < a.vocab && logit_of(a, e) != -INFINITY ? (int32_t)e.lo : -1;
}

// Notes whether `at` has been entered before.  The table has at least twice as many places as the list has entries, so the search
// ends.
__device__ __forceinline__ void enter(const DistillArgs &a, const List &l, int32_t at)
{
    const uint32_t mask = (1u << (32u - a.hash_shift)) - 1u;
    uint32_t h = ((uint32_t)at * 2654435769u) >> a.hash_shift;
    for (;;) {
        const int32_t was = atomicCAS(&l.table[h], -1, at);
        if (was == -1)
            return;
        if (was == at) {
            *l.repeats = 1;
            return;
        }
        h = (h + 1u) & mask;
    }
}

template <uint32_t T>
struct Entries {
    Entry e[kEntries<T>];
};

// the thread's entries from j0 on
template <uint32_t T>
__device__ __forceinline__ Entries<T> fetch_entries(const DistillArgs &a, uint32_t r, uint32_t j0)
{
    Entries<T> some;
#pragma unroll
    for (int i = 0; i < kEntries<T>; i++)
        if (j0 + (uint32_t)i * T < a.k)
            some.e[i] = entry_at(a, r, j0 + (uint32_t)i * T);
    return some;
}

// Reads row r's list into LDS; `first`: the thread's first entries; logit(at, j): the student's logit of entry j, loaded, and
// as_logit made fp32; noted(at): whether repeats of that column matter; meanwhile(): what else there is to do while the logits arrive.
// Loads come back in their order, so entries are asked for before the row, their logits behind it.  The result is the
// thread's largest logit of an entry (+Inf for NaN), -Inf if it has none.
template <uint32_t T, typename Logit, typename AsLogit, typename Noted, typename Meanwhile>
__device__ __forceinline__ float read_list(const DistillArgs &a, uint32_t r, const List &l, const Entries<T> &first, Logit logit, AsLogit as_logit,
                                           Noted noted, Meanwhile meanwhile)
{
    float t_max = -INFINITY;
    auto take = [&](uint32_t j0, const Entries<T> &some, auto &&then) {
        decltype(logit(0, 0u)) z[kEntries<T>];
        int32_t at[kEntries<T>];
#pragma unroll
        for (int i = 0; i < kEntries<T>; i++) {
            at[i] = j0 + (uint32_t)i * T < a.k ? column_of(a, some.e[i]) : -1;
            if (at[i] >= 0)
                z[i] = logit(at[i], j0 + (uint32_t)i * T);
        }
#pragma unroll
        for (int i = 0; i < kEntries<T>; i++) {
            const uint32_t j = j0 + (uint32_t)i * T;
            if (j < a.k)
                l.at[j] = at[i];
            if (at[i] >= 0) {
                const float t = logit_of(a, some.e[i]);
                l.t[j] = t;
                t_max = fmaxf(t_max, t != t ? INFINITY : t);
                if (noted(at[i]))
                    enter(a, l, at[i]);
            }
        }
        then();
#pragma unroll
        for (int i = 0; i < kEntries<T>; i++)
            if (at[i] >= 0)
                l.z[j0 + (uint32_t)i * T] = as_logit(z[i]);
    };
    take(threadIdx.x, first, meanwhile);
    if constexpr (T * kEntries<T> < kMaxEntries)
        for (uint32_t j0 = threadIdx.x + kEntries<T> * T; j0 < a.k; j0 += kEntries<T> * T)
            take(j0, fetch_entries<T>(a, r, j0), [] {});
    return t_max;
}

template <uint32_t T>
__device__ __forceinline__ void clear_table(const DistillArgs &a, const List &l)
{
    for (uint32_t i = threadIdx.x; i < 1u << (32u - a.hash_shift); i += T)
        l.table[i] = -1;
    if (threadIdx.x == 0)
        *l.repeats = 0;
}

// What the entries take from column `at`: the sum of their probabilities, in the list's order.  In a row with a repeat every entry adds up so, k LDS
// reads each, in a fixed order and without atomics: a teacher's largest logits hold none, and a list that does costs k^2 (4096 rows of 32000 bf16 with one
// repeat each 105 us at k = 64, 167 at 256, 1110 at 1000, without 102, 146 and 232; 8000 rows of 500 24 and 152 at k = 64 and 250, without 15 and 19).
__device__ __forceinline__ float share_of(const DistillArgs &a, const List &l, int32_t at)
{
    float s = 0.f;
    for (uint32_t j = 0; j < a.k; j++)
        s += l.at[j] == at ? l.t[j] : 0.f;
    return s;
}

// Running maximum and sum of exponentials of one lane: sum is relative to the maximum, or to 0 where that is -Inf (then it is 0, or
// NaN if there was one).
struct Running {
    float max, sum;
};

// G chunks more, at a price of one exponential for the sum so far.  The empty statement keeps the compiler from holding
// the unpacked elements of a row, twice its registers, until the gradient.
template <int DT, int G, int ALL>
__device__ __forceinline__ void add_chunks(const DistillArgs &a, Running &run, u32x4 (&raw)[ALL])
{
    constexpr int N = kElems<DT>;
    float v[N], m = run.max, s = 0.f;
#pragma unroll
    for (int i = 0; i < G; i++) {
        unpack<DT>(raw[i], v);
#pragma unroll
        for (int e = 0; e < N; e++)
            m = fmaxf(m, v[e]);
        asm volatile("" : "+v"(raw[i]));
    }
    const float to = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < G; i++) {
        unpack<DT>(raw[i], v);
#pragma unroll
        for (int e = 0; e < N; e++)
            s += exp_of(a, v[e] - to);
        asm volatile("" : "+v"(raw[i]));
    }
    run.sum = run.sum * (run.max == -INFINITY ? 1.f : exp_of(a, run.max - to)) + s;
    run.max = m;
}

// What `run` counts relative to the maximum of all; all -Inf: NaN, as the formula has it.
__device__ __forceinline__ float relative(const DistillArgs &a, Running run, float max)
{
    return run.max == -INFINITY && max != -INFINITY ? run.sum : run.sum * exp_of(a, run.max - max);
}

// A row as its chunks lie: from the first multiple of 16 bytes on, so that loads are aligned (and stores, if the gradient's rows lie
// alike: 1003 rows of 50021 bf16 take 52 us with chunks from the row's first element on, 42 like this).  The elements before and behind, up
// to a chunk less one each, are taken one by one by the first threads of the workgroup that has that end of the row.
struct RowShape {
    uint32_t head, full, tail;
};

template <int DT>
__device__ __forceinline__ RowShape shape_of(const DistillArgs &a, uint32_t r)
{
    constexpr uint32_t N = kElems<DT>;
    const uint64_t from = (uint64_t)(uintptr_t)a.logits / kSize<DT> + r * (uint64_t)a.ld_logits;
    RowShape s;
    s.head = (uint32_t)(0 - from) % N;
    s.head = s.head < a.vocab ? s.head : a.vocab;
    s.full = (a.vocab - s.head) / N;
    s.tail = (a.vocab - s.head) % N;
    return s;
}

// The single element of this thread, of `head` at the row's start and `tail` at its end.
struct Edge {
    bool there;
    uint32_t at;
};

__device__ __forceinline__ Edge edge_of(const DistillArgs &a, uint32_t head, uint32_t tail)
{
    return {threadIdx.x < head + tail, threadIdx.x < head ? threadIdx.x : a.vocab - (head + tail) + threadIdx.x};
}

__device__ __forceinline__ Running start(const DistillArgs &a, Edge edge, float z)
{
    if (!edge.there)
        return {-INFINITY, 0.f};
    const float m = fmaxf(-INFINITY, z);
    return {m, exp_of(a, z - (m == -INFINITY ? 0.f : m))};
}

template <int DT>
__device__ __forceinline__ u32x4 no_chunk()
{
    constexpr uint32_t kNone = DT == kF32 ? 0xFF800000u : 0xFF80FF80u;          // -Inf
    return u32x4{kNone, kNone, kNone, kNone};
}

// the gradient of a chunk without the teacher's part
template <int DT>
__device__ __forceinline__ u32x4 pull(const DistillArgs &a, u32x4 raw, float z_max, float g_q)
{
    constexpr int N = kElems<DT>;
    float v[N];
    unpack<DT>(raw, v);
#pragma unroll
    for (int e = 0; e < N; e++)
        v[e] = exp_of(a, v[e] - z_max) * g_q;
    return pack<DT>(v);
}

// Turns the logits of a thread's entries into probabilities; the result is what they add to the loss, in units of 4 T.  Everything is a quarter of its size, and
// logarithms are taken times T: so no difference of finite logits and no sum of their shares of it overflows, where the type's lowest value minus the
// maximum, times 1 / T, or shared out by shares that add up to 1 and a rounding more, would be infinite, and 0 times that NaN.
template <uint32_t T, bool LOSS = true>
__device__ __forceinline__ float take_entries(const DistillArgs &a, const List &list, float t_max, float t_sum, float z_max, float z_sum)
{
    const float part = 1.f / t_sum, scale = 0.25f * a.temperature;
    const float t_log = LOSS ? scale * logf(t_sum) : 0.f, z_log = LOSS ? scale * logf(z_sum) : 0.f, t_top = 0.25f * t_max, z_top = 0.25f * z_max;
    float loss = 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += T)
        if (list.at[j] >= 0) {
            const float t = list.t[j], p = exp_of(a, t - t_max) * part;
            if constexpr (LOSS) {
                const float log_q = fmaf(list.z[j], 0.25f, -z_top) - z_log;
                loss += log_q == -INFINITY ? INFINITY : p * ((fmaf(t, 0.25f, -t_top) - t_log) - log_q);
            }
            list.t[j] = p;
        }
    return loss;
}

template <uint32_t T>
__device__ __forceinline__ float entries_sum(const DistillArgs &a, const List &list, float t_max)
{
    float sum = 0.f;
    for (uint32_t j = threadIdx.x; j < a.k; j += T)
        if (list.at[j] >= 0)
            sum += exp_of(a, list.t[j] - t_max);
    return sum;
}

// The row's results, by thread 0, from the wavefronts' parts of the loss.
template <int W>
__device__ __forceinline__ void write_row(const DistillArgs &a, uint32_t r, const float *parts, bool some, float z_max, float z_sum)
{
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < W; w++)
        sum += parts[w];
    a.loss[r] = some ? a.temperature * 4.f * sum : 0.f;
    if (a.row_max) {
        a.row_max[r] = z_max;
        a.row_sum[r] = z_sum;
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// A row in the registers of one workgroup: T threads with P chunks each.  The logits are read once, added up as they arrive, and the
// gradient is taken from the registers.  Bound by memory: 4096 rows of 32000 bf16, loss and gradient, 102 us (524 MB, 5.1 TB/s,
// a device copy's rate; the vector ALU is busy for half of that time).  Logits and gradient pass with streaming loads and stores (with plain
// ones 119 us); but the gradient of short rows, whose lines the list's columns soon touch again, with plain stores (8000 rows of 900 fp32 18.3 us,
// streaming 19.6).
//
// The gradient's columns that the list names are written again, with what the teacher takes from them, when the rest has been
// written: k of the vocabulary's columns, and the barrier between orders the two (the counters see 4 % more bytes written).
// ---------------------------------------------------------------------------------------------------------------------
// LONGER: what the workgroup does not hold is read twice, the second time from the memory-side cache, which has room for that of a row for
// each compute unit (4000 rows of 120000 fp32 767 us, 5.0 TB/s; in parts, with two passes over all rows, 1011).
template <int DT, int T, int P, bool LONGER>
__device__ __forceinline__ void distill_row(const DistillArgs a)
{
    constexpr int W = T / 64, G = 4;
    constexpr int kAtOnce = P <= 12 ? G / 2 : 0;                                // a group's second half only if the row has it: short rows' arithmetic counts
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *const red = (float *)lds;                                            // 2 x 2 W numbers, and W
    const List list = list_in(red + 5 * W, a);
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const size_t z0 = r * a.ld_logits;
        const RowShape row = shape_of<DT>(a, r);
        const Edge edge = edge_of(a, row.head, row.tail);
        const Entries<T> first = fetch_entries<T>(a, r, threadIdx.x);
        const uint32_t edge_bits = edge.there ? load_bits<DT>(a.logits, z0 + edge.at) : 0u;
        u32x4 raw[P / G][G];
        const float g = a.dlogits ? (a.row_weight ? a.row_weight[r] : 1.f) * a.temperature : 0.f;
#pragma unroll
        for (int i = 0; i < P; i++) {
            const uint32_t c = threadIdx.x + (uint32_t)(i * T);
            raw[i / G][i % G] = no_chunk<DT>();
            if (c < row.full)
                raw[i / G][i % G] = load_whole<DT, true>((const unsigned char *)a.logits + (z0 + row.head) * kSize<DT> + (size_t)(i * T) * 16u,
                                                         threadIdx.x * 16u);
        }
        auto behind = [&](uint32_t c0, u32x4 (&some)[G]) {                      // chunks that are not held
#pragma unroll
            for (int i = 0; i < G; i++) {
                some[i] = no_chunk<DT>();
                if (c0 + threadIdx.x + (uint32_t)(i * T) < row.full)
                    some[i] = load_whole<DT>((const unsigned char *)a.logits + (z0 + row.head) * kSize<DT> + (size_t)(c0 + (uint32_t)(i * T)) * 16u,
                                             threadIdx.x * 16u);
            }
        };
        if (a.k && a.dlogits) {
            clear_table<T>(a, list);
            __syncthreads();
        }
        const float single = from_bits<DT>(edge_bits);
        Running run;
        float t_max = read_list<T>(a, r, list, first, [&](int32_t at, uint32_t) { return load_bits<DT>(a.logits, z0 + (uint32_t)at); }, from_bits<DT>,
                                   [&](int32_t) { return a.dlogits != nullptr; },
                                   [&] {
                                       run = start(a, edge, single);
#pragma unroll
                                       for (int i = 0; i < P / G; i++)
                                           if ((uint32_t)((i * G + kAtOnce) * T) < row.full)
                                               add_chunks<DT, G>(a, run, raw[i]);
                                           else if (kAtOnce && (uint32_t)(i * G * T) < row.full)
                                               add_chunks<DT, G / 2>(a, run, raw[i]);
                                       if constexpr (LONGER)
                                           for (uint32_t c0 = T * P; c0 < row.full; c0 += G * T) {
                                               u32x4 some[G];
                                               behind(c0, some);
                                               add_chunks<DT, G>(a, run, some);
                                           }
                                   });
        float z_max = run.max;
        group_reduce<Max, Max, W>(t_max, z_max, red);
        float t_sum = entries_sum<T>(a, list, t_max), z_sum = relative(a, run, z_max);
        group_reduce<Sum, Sum, W>(t_sum, z_sum, red + 2 * W);

        const bool some = t_max != -INFINITY;
        const float loss = lanes_reduce<Sum, 64>(take_entries<T>(a, list, t_max, t_sum, z_max, z_sum));
        if ((threadIdx.x & 63) == 0)
            red[4 * W + (threadIdx.x >> 6)] = loss;

        const float g_q = g / z_sum;
        const bool none = !some || g == 0.f;
        const size_t d0 = r * a.ld_dlogits;
        if (a.dlogits) {
            uint32_t me = threadIdx.x;                                          // so that neither the loads' addresses nor their masks are kept until here
            asm volatile("" : "+v"(me));
#pragma unroll
            for (int i = 0; i < P; i++) {
                if (me + (uint32_t)(i * T) < row.full)
                    store_whole<DT, (T * P > 256)>((unsigned char *)a.dlogits + (d0 + row.head) * kSize<DT> + (size_t)(i * T) * 16u, me * 16u,
                                          none ? u32x4{0u, 0u, 0u, 0u} : pull<DT>(a, raw[i / G][i % G], z_max, g_q));
            }
            if constexpr (LONGER)
                for (uint32_t c0 = T * P; c0 < row.full; c0 += G * T) {
                    u32x4 some[G];
                    behind(c0, some);
#pragma unroll
                    for (int i = 0; i < G; i++)
                        if (c0 + me + (uint32_t)(i * T) < row.full)
                            store_whole<DT, true>((unsigned char *)a.dlogits + (d0 + row.head) * kSize<DT> + (size_t)(c0 + (uint32_t)(i * T)) * 16u, me * 16u,
                                                  none ? u32x4{0u, 0u, 0u, 0u} : pull<DT>(a, some[i], z_max, g_q));
                }
            if (edge.there)
                store_one<DT>(a.dlogits, d0 + edge.at, none ? 0.f : exp_of(a, single - z_max) * g_q);
        }
        __syncthreads();
        if (threadIdx.x == 0)
            write_row<W>(a, r, red + 4 * W, some, z_max, z_sum);
        if (a.dlogits && !none) {
            const bool repeats = *list.repeats != 0;
            for (uint32_t j = threadIdx.x; j < a.k; j += T) {
                const int32_t at = list.at[j];
                if (at >= 0)
                    store_one<DT>(a.dlogits, d0 + (uint32_t)at, exp_of(a, list.z[j] - z_max) * g_q - g * (repeats ? share_of(a, list, at) : list.t[j]));
            }
        }
        if (r + gridDim.x < a.rows)
            __syncthreads();                                                    // the list and `red` are used again
    }
}

template <int DT, int T, int P>
__global__ void __launch_bounds__(T) distill_row_kernel(const DistillArgs a)
{
    distill_row<DT, T, P, false>(a);
}

constexpr int kLong = 1024;

template <int DT>
__global__ void __launch_bounds__(kLong) distill_long_kernel(const DistillArgs a)
{
    distill_row<DT, kLong, 12, true>(a);
}

// ---------------------------------------------------------------------------------------------------------------------
// Few long rows: parts of rows.  The first launch takes the maximum and the sum of each part and the
// student's logits of the entries in it; the second joins them and does the rest, part by part, from logits that the caches may
// still hold.  48 rows of 131072 fp32, loss and gradient: 7 and 10 us (25 MB read, then 25 read from the caches and 25 written).
// A gradient alone has its statistics and needs the second launch only: 1003 rows of 50021 bf16 43 us (4.6 TB/s).  Its 256 threads are
// too many for short rows, a part each: 8000 rows of 500 bf16 41 us, 4000 of 2304 fp32 28, where loss and gradient in one call take 14 and 17.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kAhead = 8;                 // chunks that a thread has in flight

struct Part {
    uint32_t r, part;
    uint32_t begin, end;                  // chunks
    uint32_t first, behind;               // columns, with the elements before and behind the chunks at the row's ends
    RowShape row;
    Edge edge;
};

template <int DT>
__device__ __forceinline__ Part part_of(const DistillArgs &a, uint64_t id)
{
    constexpr uint32_t N = kElems<DT>;
    Part p;
    p.r = (uint32_t)(id / a.parts);
    p.part = (uint32_t)(id % a.parts);
    p.row = shape_of<DT>(a, p.r);
    const bool last = p.part + 1u == a.parts;
    p.begin = p.part * a.part_chunks;
    p.end = last ? p.row.full : p.begin + a.part_chunks;
    p.first = p.part ? p.row.head + p.begin * N : 0u;
    p.behind = last ? a.vocab : p.row.head + p.end * N;
    p.edge = edge_of(a, p.part ? 0u : p.row.head, last ? p.row.tail : 0u);
    return p;
}

__device__ __forceinline__ bool in_part(const Part &p, int32_t at) { return at >= 0 && (uint32_t)at >= p.first && (uint32_t)at < p.behind; }

template <int DT, bool STREAM>
__device__ __forceinline__ void fetch(const DistillArgs &a, const Part &p, uint32_t c0, u32x4 (&raw)[kAhead])
{
#pragma unroll
    for (int i = 0; i < kAhead; i++) {
        const uint32_t c = c0 + threadIdx.x + (uint32_t)i * kSlice;
        raw[i] = no_chunk<DT>();
        if (c < p.end)
            raw[i] = load_whole<DT, STREAM>((const unsigned char *)a.logits + (p.r * a.ld_logits + p.row.head) * kSize<DT> +
                                                (size_t)(c0 + (uint32_t)i * kSlice) * 16u, threadIdx.x * 16u);
    }
}

// adds up the chunks c0 ... that the workgroup fetched: by four of a thread, and not those behind the part
template <int DT>
__device__ __forceinline__ void add_fetched(const DistillArgs &a, const Part &p, uint32_t c0, Running &run, u32x4 (&raw)[kAhead])
{
    constexpr int G = 4;
#pragma unroll
    for (int i = 0; i < kAhead; i += G)
        if (c0 + (uint32_t)i * kSlice < p.end) {
            u32x4 some[G] = {raw[i], raw[i + 1], raw[i + 2], raw[i + 3]};
            add_chunks<DT, G>(a, run, some);
        }
}

template <int DT>
__global__ void __launch_bounds__(kSlice, 8) distill_part_kernel(const DistillArgs a)
{
    constexpr int W = kSlice / 64;
    __shared__ float red[4 * W];
    for (uint64_t id = blockIdx.x; id < (uint64_t)a.rows * a.parts; id += gridDim.x) {
        const Part p = part_of<DT>(a, id);
        const size_t z0 = p.r * a.ld_logits;
        Running run = start(a, p.edge, p.edge.there ? load_one<DT>(a.logits, z0 + p.edge.at) : 0.f);
        for (uint32_t c0 = p.begin; c0 < p.end; c0 += kAhead * kSlice) {
            u32x4 raw[kAhead];
            fetch<DT, false>(a, p, c0, raw);
            add_fetched<DT>(a, p, c0, run, raw);
        }
        float all = run.max, unused = 0.f;
        group_reduce<Max, Max, W>(all, unused, red);
        float sum = run.max == -INFINITY ? run.sum : relative(a, run, all);
        group_reduce<Sum, Sum, W>(sum, unused, red + 2 * W);
        if (threadIdx.x == 0) {
            a.part_stats[2 * id] = all;
            a.part_stats[2 * id + 1] = sum;
        }
        for (uint32_t j = threadIdx.x; j < a.k; j += kSlice) {
            const size_t i = p.r * a.ld_index + j;
            const int64_t at = a.index64 ? ((const int64_t *)a.index)[i] : (int64_t)((const int32_t *)a.index)[i];
            if (at < (int64_t)a.vocab && in_part(p, at < 0 ? -1 : (int32_t)at))
                a.list_logits[(size_t)p.r * a.k + j] = load_one<DT>(a.logits, z0 + (size_t)at);
        }
        if (id + gridDim.x < (uint64_t)a.rows * a.parts)
            __syncthreads();
    }
}

// The loss alone of rows that are added up without being held, so that a compute unit has seven workgroups' loads in flight.
template <int DT>
__global__ void __launch_bounds__(kSlice) distill_loss_kernel(const DistillArgs a)
{
    constexpr int W = kSlice / 64;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *const red = (float *)lds;
    const List list = list_in(red + 5 * W, a);
    for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const Part p = part_of<DT>(a, r);                                       // the whole row
        const size_t z0 = r * a.ld_logits;
        const Entries<kSlice> first = fetch_entries<kSlice>(a, r, threadIdx.x);
        const uint32_t edge_bits = p.edge.there ? load_bits<DT>(a.logits, z0 + p.edge.at) : 0u;
        Running run;
        float t_max = read_list<kSlice>(a, r, list, first, [&](int32_t at, uint32_t) { return load_bits<DT>(a.logits, z0 + (uint32_t)at); }, from_bits<DT>,
                                        [](int32_t) { return false; },
                                        [&] {
                                            run = start(a, p.edge, from_bits<DT>(edge_bits));
                                            for (uint32_t c0 = p.begin; c0 < p.end; c0 += kAhead * kSlice) {
                                                u32x4 raw[kAhead];
                                                fetch<DT, true>(a, p, c0, raw);
                                                add_fetched<DT>(a, p, c0, run, raw);
                                            }
                                        });
        float z_max = run.max;
        group_reduce<Max, Max, W>(t_max, z_max, red);
        float t_sum = entries_sum<kSlice>(a, list, t_max), z_sum = relative(a, run, z_max);
        group_reduce<Sum, Sum, W>(t_sum, z_sum, red + 2 * W);
        const float loss = lanes_reduce<Sum, 64>(take_entries<kSlice>(a, list, t_max, t_sum, z_max, z_sum));
        if ((threadIdx.x & 63) == 0)
            red[4 * W + (threadIdx.x >> 6)] = loss;
        __syncthreads();
        if (threadIdx.x == 0)
            write_row<W>(a, r, red + 4 * W, t_max != -INFINITY, z_max, z_sum);
        if (r + gridDim.x < a.rows)
            __syncthreads();
    }
}

// JOIN: after distill_part_kernel, with the loss; otherwise the gradient from the row's statistics.
template <int DT, bool JOIN>
__global__ void __launch_bounds__(kSlice) distill_slice_kernel(const DistillArgs a)
{
    constexpr int W = kSlice / 64;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    float *const red = (float *)lds;
    const List list = list_in(red + 5 * W, a);
    for (uint64_t id = blockIdx.x; id < (uint64_t)a.rows * a.parts; id += gridDim.x) {
        const Part p = part_of<DT>(a, id);
        if (JOIN && !a.dlogits && p.part)                                       // the loss alone is joined by one workgroup a row
            continue;
        const size_t z0 = p.r * a.ld_logits;
        const Entries<kSlice> first = fetch_entries<kSlice>(a, p.r, threadIdx.x);
        const uint32_t edge_bits = a.dlogits && p.edge.there ? load_bits<DT>(a.logits, z0 + p.edge.at) : 0u;
        u32x4 raw[kAhead];
        if (a.dlogits)
            fetch<DT, true>(a, p, p.begin, raw);
        const float g = a.dlogits ? (a.row_weight ? a.row_weight[p.r] : 1.f) * a.temperature : 0.f;
        float z_max, z_sum;
        if constexpr (JOIN) {
            const uint32_t lane = threadIdx.x & 63;
            float m = -INFINITY, s = 0.f;
            if (lane < a.parts) {
                m = a.part_stats[2 * ((uint64_t)p.r * a.parts + lane)];
                s = a.part_stats[2 * ((uint64_t)p.r * a.parts + lane) + 1];
            }
            z_max = lanes_reduce<Max, 64>(m);
            z_sum = lanes_reduce<Sum, 64>(lane < a.parts ? relative(a, Running{m, s}, z_max) : 0.f);
        } else {
            z_max = a.row_max[p.r];
            z_sum = a.row_sum[p.r];
        }
        float t_max = -INFINITY, t_sum = 0.f, unused = 0.f;
        if (a.k) {
            if (a.dlogits) {
                clear_table<kSlice>(a, list);
                __syncthreads();
            }
            t_max = read_list<kSlice>(a, p.r, list, first,
                                      [&](int32_t at, uint32_t j) {
                                          if constexpr (JOIN)
                                              return __float_as_uint(a.list_logits[(size_t)p.r * a.k + j]);
                                          else
                                              return load_bits<DT>(a.logits, z0 + (uint32_t)(in_part(p, at) ? at : 0));
                                      },
                                      [](uint32_t bits) { return JOIN ? __uint_as_float(bits) : from_bits<DT>(bits); },
                                      [&](int32_t at) { return a.dlogits && in_part(p, at); }, [] {});
        }
        group_reduce<Max, Max, W>(t_max, unused, red);
        t_sum = entries_sum<kSlice>(a, list, t_max);
        group_reduce<Sum, Sum, W>(t_sum, unused, red + 2 * W);
        const bool some = t_max != -INFINITY;
        const float loss = take_entries<kSlice, JOIN>(a, list, t_max, t_sum, z_max, z_sum);
        if constexpr (JOIN) {
            const float sum = lanes_reduce<Sum, 64>(loss);
            if ((threadIdx.x & 63) == 0)
                red[4 * W + (threadIdx.x >> 6)] = sum;
        }
        __syncthreads();
        if (JOIN && p.part == 0 && threadIdx.x == 0)
            write_row<W>(a, p.r, red + 4 * W, some, z_max, z_sum);
        if (a.dlogits) {
            const float g_q = g / z_sum;
            const bool none = !some || g == 0.f;
            const size_t d0 = p.r * a.ld_dlogits;
            auto taken = [&](u32x4 chunk) { return none ? u32x4{0u, 0u, 0u, 0u} : pull<DT>(a, chunk, z_max, g_q); };
            for (uint32_t c0 = p.begin; c0 < p.end;) {
#pragma unroll
                for (int i = 0; i < kAhead; i++) {
                    const uint32_t c = c0 + threadIdx.x + (uint32_t)i * kSlice;
                    if (c < p.end)
                        store_whole<DT, true>((unsigned char *)a.dlogits + (d0 + p.row.head) * kSize<DT> + (size_t)(c0 + (uint32_t)i * kSlice) * 16u,
                                              threadIdx.x * 16u, taken(raw[i]));
                }
                c0 += kAhead * kSlice;
                if (c0 < p.end)
                    fetch<DT, true>(a, p, c0, raw);
            }
            if (p.edge.there)
                store_one<DT>(a.dlogits, d0 + p.edge.at, none ? 0.f : exp_of(a, from_bits<DT>(edge_bits) - z_max) * g_q);
            __syncthreads();
            const bool repeats = a.k && *list.repeats != 0;
            for (uint32_t j = threadIdx.x; j < a.k && !none; j += kSlice) {
                const int32_t at = list.at[j];
                if (in_part(p, at))
                    store_one<DT>(a.dlogits, d0 + (uint32_t)at, exp_of(a, list.z[j] - z_max) * g_q - g * (repeats ? share_of(a, list, at) : list.t[j]));
            }
        }
        if (id + gridDim.x < (uint64_t)a.rows * a.parts)
            __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------------------------------
struct RowKernel {
    uint32_t threads, chunks;                                                   // that the workgroup holds
    int64_t above;                                                              // for calls of more rows than this
    void (*kernel[2])(const DistillArgs);
};

#define ROW_KERNEL(T, P, ABOVE) {T, T * P, ABOVE, {distill_row_kernel<kF32, T, P>, distill_row_kernel<kBF16, T, P>}}
// Short rows are bound by a row's chain of latencies (entries, their logits, two sums, the columns that the list names): 8000 rows of 500 bf16 take 14 us, of which
// 2.9 are what so many empty workgroups take, with the vector ALU busy for 36 %.
// A compute unit holds several of the smaller workgroups, which overlap one row's loads with another's arithmetic: with many rows they win
// (2048 rows of 15000 bf16: 256 threads with 8 chunks each 31 us, 1024 with 4 58).  Up to a row for each of 256 compute units nothing
// overlaps, and a row is done soonest by many threads (64 rows of 8000 bf16: 64 threads with 16 chunks 10.1 us, 1024 with 4 6.8).  In between
// the chip takes so many wavefronts of a row at once: 4000 rows of 2304 fp32 by 256 threads 24.4 us, by 64 17.7, but 400 rows 6.6 and 7.4; 2000 of
// 9000 bf16 by 256 threads 23.1, by 128 20.1, 400 of 10000 9.2 and 10.7; 300 of 2304 bf16 by 64 threads 7.1, by 256 6.6, 800 7.5 and 8.0.
// Long rows: two workgroups on a compute unit, as long as their registers last (4000 rows of 80000 bf16 by 256 threads with 40 chunks 243 us, by 512 with
// 32, alone on their unit, 294; with 44, which spill, 329), then one of many wavefronts (of 120000, 1024 threads with 16 chunks 403, 512 with 32 426; of
// 80000 fp32, 512 with 44 chunks 482, by distill_long_kernel 472).
// The first that holds the row and is for so many.
static const RowKernel kManyRows[] = {ROW_KERNEL(64, 4, 0), ROW_KERNEL(64, 8, 640), ROW_KERNEL(64, 12, 1536), ROW_KERNEL(128, 8, 1536), ROW_KERNEL(256, 4, 0),
                                      ROW_KERNEL(128, 12, 640), ROW_KERNEL(256, 8, 0), ROW_KERNEL(256, 16, 0), ROW_KERNEL(512, 16, 0), ROW_KERNEL(256, 40, 0),
                                      ROW_KERNEL(1024, 12, 0), ROW_KERNEL(1024, 16, 0)};
static const RowKernel kFewRows[] = {ROW_KERNEL(64, 4, 0), ROW_KERNEL(256, 4, 0), ROW_KERNEL(1024, 4, 0), ROW_KERNEL(1024, 8, 0)};
constexpr int64_t kFew = 256;
constexpr uint32_t kFewHeld = 1024 * 8;
// Without a gradient longer rows need not be held (3000 rows of 64000 fp32: 148 us held, 117 not; of 4000, 1000 chunks, 14.7 both).
constexpr uint32_t kLossHeld = 1024;
#undef ROW_KERNEL
constexpr uint32_t kHeld = 1024 * 16;      // longer rows: distill_long_kernel

// How a call is cut: parts = 0 is a row per workgroup.
struct Cut {
    uint32_t parts, part_chunks;
};

static Cut cut_rows(int64_t rows, uint32_t chunks, uint32_t least, uint32_t most)
{
    // Four workgroups on each of 256 compute units, which is what their registers leave room for, and not one more (48 rows of 131072
    // fp32 in 22 parts 19.8 us, in 21 17.0); parts of `least` ... `most` chunks.
    uint64_t parts = 1024 / rows;
    const uint64_t upper = (chunks + least - 1) / least, lower = (chunks + (uint64_t)most - 1) / most;
    parts = parts > upper ? upper : parts;
    parts = parts < lower ? lower : parts;
    parts = parts > kMaxParts ? kMaxParts : parts < 1 ? 1 : parts;
    uint32_t size = (uint32_t)((chunks + parts - 1) / parts);
    size = size ? size : 1;
    return {chunks ? (chunks + size - 1) / size : 1, size};
}

static uint32_t chunks_of(int64_t vocab, tmask_dtype dt) { return (uint32_t)(vocab / (dt == TMASK_F32 ? 4 : 8)); }   // of a row at most

// Rows of so many chunks are cut in parts if there are fewer than this.  A second launch costs 3 us; a row in one workgroup longer, the longer it is and
// the fewer compute units have one (us, row / parts: 16 rows of 32000 bf16 8.4 / 10.0, of 64000 11.9 / 10.1; 64 rows of 64000 12.6 / 15.4, of
// 131072 21.1 / 15.0; 128 of 89000 17.1 / 18.1, of 131072 fp32 32.1 / 35.6; 256 57.7 / 69.4).
static int64_t cut_below(uint32_t chunks) { return chunks <= 4096 ? 0 : chunks <= kFewHeld ? 64 : 128; }

constexpr uint32_t kLeast = 512, kMost = kAhead * kSlice;                       // chunks of a part

static Cut cut_loss(int64_t rows, int64_t vocab, tmask_dtype dt)
{
    const uint32_t chunks = chunks_of(vocab, dt);
    return rows < cut_below(chunks) ? cut_rows(rows, chunks, kLeast, kMost) : Cut{0, 0};
}

static uint32_t grid_of(uint64_t workgroups) { return (uint32_t)(workgroups < (1u << 20) ? workgroups : 1u << 20); }

// Everything but the outputs; `args` is complete when the result is TMASK_OK and rows > 0.
static int check_distill(const tmask_distill_desc *desc, tmask_dtype dt, tmask_dtype teacher_dt, int index_bits, float temperature,
                         DistillArgs *args)
{
    if (!desc)
        return fail(TMASK_ERR_NULL, "descriptor is NULL");
    const tmask_distill_desc &d = *desc;
    if (!known(dt) || !known(teacher_dt) || (index_bits != 32 && index_bits != 64))
        return fail(TMASK_ERR_DTYPE, "unknown dtype %d, teacher's dtype %d or index of %d bits", (int)dt, (int)teacher_dt, index_bits);
    if (!valid_sizes(d.rows, d.vocab) || d.k < 0 || d.k > (int64_t)kMaxEntries)
        return fail(TMASK_ERR_SHAPE, "rows=%lld vocab=%lld k=%lld (at most %u)", (long long)d.rows, (long long)d.vocab, (long long)d.k, kMaxEntries);
    if (!(temperature >= 1e-18f && temperature <= 1e18f))                       // its square and its reciprocal are numbers
        return fail(TMASK_ERR_SHAPE, "temperature=%g must lie between 1e-18 and 1e18", (double)temperature);
    if (d.rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_rows("logits", d.logits, d.ld_logits, d.rows, d.vocab, size_of(dt), true));
    TMASK_TRY(check_rows("teacher", d.teacher, d.ld_teacher, d.rows, d.k, size_of(teacher_dt), d.k > 0));
    TMASK_TRY(check_rows("index", d.index, d.ld_index, d.rows, d.k, (size_t)index_bits / 8, d.k > 0));
    TMASK_TRY(check_vector("row_weight", d.row_weight, 4, false));
    TMASK_TRY(check_rows("dlogits", d.dlogits, d.ld_dlogits, d.rows, d.vocab, size_of(dt), false));
    DistillArgs &a = *args;
    a.logits = d.logits; a.teacher = d.teacher; a.index = d.index; a.row_weight = d.row_weight;
    a.loss = d.loss; a.row_max = d.row_max; a.row_sum = d.row_sum; a.dlogits = d.dlogits;
    a.part_stats = a.list_logits = nullptr;
    a.ld_logits = (size_t)d.ld_logits; a.ld_teacher = (size_t)d.ld_teacher; a.ld_index = (size_t)d.ld_index; a.ld_dlogits = (size_t)d.ld_dlogits;
    a.rows = (uint32_t)d.rows; a.vocab = (uint32_t)d.vocab; a.k = (uint32_t)d.k;
    a.parts = a.part_chunks = 0;
    a.teacher_f32 = teacher_dt == TMASK_F32; a.index64 = index_bits == 64;
    a.hash_shift = 31;
    while (a.hash_shift > 0 && (1u << (32u - a.hash_shift)) < 2u * a.k)
        a.hash_shift--;
    a.temperature = temperature; a.per_t2 = (float)(1.4426950408889634 / (double)temperature);
    return TMASK_OK;
}

}  // namespace tmask

using namespace tmask;

// Rows that are cut in parts need room for the statistics of every part and for a list's logits.  The size is a bound for all calls of up to so many
// rows, of either type: as many rows as are cut at all, of fp32's chunks, with the parts that cut_rows may give them.
extern "C" size_t tmask_distill_workspace_bytes(int64_t rows, int64_t vocab)
{
    if (!valid_sizes(rows, vocab))
        return 0;
    const uint32_t chunks = chunks_of(vocab, TMASK_F32);
    const uint64_t below = (uint64_t)cut_below(chunks), cut = below == 0 ? 0 : (uint64_t)rows < below ? (uint64_t)rows : below - 1;
    const uint64_t lower = (chunks + (uint64_t)kMost - 1) / kMost, most = cut * kMaxParts, parts = cut * lower > 1024 ? cut * lower : 1024;
    return (size_t)(cut * kMaxEntries + 2u * (parts < most ? parts : most)) * 4u;
}

extern "C" int tmask_distill(const tmask_distill_desc *desc, tmask_dtype dt, tmask_dtype teacher_dt, int index_bits, float temperature,
                             void *workspace, size_t workspace_bytes, void *hip_stream)
{
    DistillArgs a;
    TMASK_TRY(check_distill(desc, dt, teacher_dt, index_bits, temperature, &a));
    if (desc->rows == 0)
        return TMASK_OK;
    TMASK_TRY(check_vector("loss", desc->loss, 4, true));
    TMASK_TRY(check_vector("row_max", desc->row_max, 4, desc->row_sum != nullptr));
    TMASK_TRY(check_vector("row_sum", desc->row_sum, 4, desc->row_max != nullptr));
    hipStream_t stream = (hipStream_t)hip_stream;
    const Cut cut = cut_loss(desc->rows, desc->vocab, dt);
    const size_t list = list_bytes(a, a.dlogits != nullptr);                     // the loss alone does not mind repeats
    const bool bf16 = dt == TMASK_BF16;
    if (cut.parts == 0 && !a.dlogits && desc->rows > kFew && chunks_of(desc->vocab, dt) > kLossHeld) {
        a.parts = 1;
        a.part_chunks = chunks_of(desc->vocab, dt);
        hipLaunchKernelGGL(bf16 ? distill_loss_kernel<kBF16> : distill_loss_kernel<kF32>, dim3(grid_of(a.rows)), dim3(kSlice), 20 * (kSlice / 64) + list,
                           stream, a);
    } else if (cut.parts == 0) {
        const uint32_t chunks = chunks_of(desc->vocab, dt);
        if (chunks > kHeld) {
            hipLaunchKernelGGL(bf16 ? distill_long_kernel<kBF16> : distill_long_kernel<kF32>, dim3(grid_of(a.rows)), dim3(kLong), 20 * (kLong / 64) + list,
                               stream, a);
        } else {
            const RowKernel *k = desc->rows <= kFew && chunks <= kFewHeld ? kFewRows : kManyRows;
            while (k->chunks < chunks || desc->rows <= k->above)
                k++;
            hipLaunchKernelGGL(k->kernel[bf16], dim3(grid_of(a.rows)), dim3(k->threads), 20 * (k->threads / 64) + list, stream, a);
        }
    } else {
        TMASK_TRY(check_workspace(workspace, workspace_bytes, tmask_distill_workspace_bytes(desc->rows, desc->vocab)));
        a.parts = cut.parts;
        a.part_chunks = cut.part_chunks;
        a.part_stats = (float *)workspace;
        a.list_logits = a.part_stats + (size_t)a.rows * a.parts * 2u;
        const uint32_t grid = grid_of((uint64_t)a.rows * a.parts);
        hipLaunchKernelGGL(bf16 ? distill_part_kernel<kBF16> : distill_part_kernel<kF32>, dim3(grid), dim3(kSlice), 0, stream, a);
        hipLaunchKernelGGL((bf16 ? distill_slice_kernel<kBF16, true> : distill_slice_kernel<kF32, true>), dim3(grid), dim3(kSlice),
                           20 * (kSlice / 64) + list, stream, a);
    }
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
    const Cut cut = cut_rows(desc->rows, chunks_of(desc->vocab, dt), kLeast, kMost);
    a.parts = cut.parts;
    a.part_chunks = cut.part_chunks;
    hipLaunchKernelGGL((dt == TMASK_BF16 ? distill_slice_kernel<kBF16, false> : distill_slice_kernel<kF32, false>),
                       dim3(grid_of((uint64_t)a.rows * a.parts)), dim3(kSlice), 20 * (kSlice / 64) + list_bytes(a, true), (hipStream_t)hip_stream, a);
    return launched("distillation gradient launch");
}
