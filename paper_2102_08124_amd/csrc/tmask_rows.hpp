// What the row kernels (layer norm, bias + GELU, distillation) share: rows in chunks of 16 bytes, sums over lanes and workgroups.
#pragma once
#include <type_traits>

#include "tmask_device.hpp"

namespace tmask {

// A chunk may begin at any element: 16-byte loads and stores work at any address, at somewhat less speed than at multiples of 16.
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));

template <int DT>
constexpr int kElems = DT == kF32 ? 4 : 8;          // of a chunk

template <int DT>
constexpr int kSize = DT == kF32 ? 4 : 2;           // bytes of an element

// element i of an array of type DT, as fp32
template <int DT>
__device__ __forceinline__ float load_one(const void *p, size_t i)
{
    if constexpr (DT == kF32)
        return ((const float *)p)[i];
    else
        return __uint_as_float((uint32_t)((const uint16_t *)p)[i] << 16);
}

// the same in two steps: a loop of loads, and what is computed from them
template <int DT>
__device__ __forceinline__ uint32_t load_bits(const void *p, size_t i)
{
    if constexpr (DT == kF32)
        return ((const uint32_t *)p)[i];
    else
        return ((const uint16_t *)p)[i];
}

template <int DT>
__device__ __forceinline__ float from_bits(uint32_t bits)
{
    return __uint_as_float(DT == kF32 ? bits : bits << 16);
}

// rounded to nearest even
template <int DT>
__device__ __forceinline__ void store_one(void *p, size_t i, float v)
{
    if constexpr (DT == kF32)
        ((float *)p)[i] = v;
    else
        ((__bf16 *)p)[i] = (__bf16)v;
}

// row r of a matrix
template <int DT>
__device__ __forceinline__ const unsigned char *row_of(const void *p, size_t r, size_t ld)
{
    return (const unsigned char *)p + r * ld * kSize<DT>;
}

template <int DT>
__device__ __forceinline__ unsigned char *row_of(void *p, size_t r, size_t ld)
{
    return (unsigned char *)p + r * ld * kSize<DT>;
}

// elements c ... of a row, of which `left` belong to it (at least one); the others are 0.  A row's bytes stay below 2^32: where its address
// is the same for a wavefront it stays in scalar registers.
template <int DT>
__device__ __forceinline__ u32x4 load_chunk(const void *row, uint32_t c, uint32_t left)
{
    const unsigned char *const a = (const unsigned char *)row + (uint32_t)(c * kSize<DT>);
    if (left >= (uint32_t)kElems<DT>) {
        if constexpr (DT == kF32)
            return *(const u32x4_at4 *)a;
        else
            return *(const u32x4_at2 *)a;
    }
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        if constexpr (DT == kF32) {
            v[e] = (uint32_t)e < left ? ((const uint32_t *)a)[e] : 0u;
        } else {
            const uint32_t lo = 2u * e < left ? ((const uint16_t *)a)[2 * e] : 0u, hi = 2u * e + 1u < left ? ((const uint16_t *)a)[2 * e + 1] : 0u;
            v[e] = lo | hi << 16;
        }
    }
    return v;
}

// The same for a row of `cols` elements, in two steps: the load, a single one if the row has a chunk's elements at all (the one at
// the row's end, which ends with what is wanted), and what moves the wanted elements to the front and leaves 0 behind them.  Where a row of
// a wavefront's lanes fetches element by element and composes, everything that is in flight waits for it (the gradients of a layer norm of 13731
// rows of 4476 bf16 took 175 us that way, of 4480 93).
template <int DT>
__device__ __forceinline__ u32x4 fetch_chunk(const void *row, uint32_t c, uint32_t left, uint32_t cols)
{
    constexpr uint32_t N = kElems<DT>;
    return load_chunk<DT>(row, left < N && cols >= N ? c - (N - left) : c, cols >= N ? N : left);
}

template <int DT>
__device__ __forceinline__ u32x4 settle(u32x4 raw, uint32_t left, uint32_t cols)
{
    constexpr uint32_t N = kElems<DT>;
    if (cols % N && cols > N && left < N) {                                     // the first two are the same for all
        const uint32_t s = N - left;
        if constexpr (DT == kBF16)
            if (s & 1u)
                raw = u32x4{raw.x >> 16 | raw.y << 16, raw.y >> 16 | raw.z << 16, raw.z >> 16 | raw.w << 16, raw.w >> 16};
        if (s & N / 4)
            raw = u32x4{raw.y, raw.z, raw.w, 0u};
        if (s & N / 2)
            raw = u32x4{raw.z, raw.w, 0u, 0u};
    }
    return raw;
}

// A whole chunk at `offset` bytes from an address that is the same for the wavefront, which then is held in scalar registers.
// STREAM: with the non-temporal hint, for what is read or written once and does not fit the caches.
template <int DT, bool STREAM = false>
__device__ __forceinline__ u32x4 load_whole(const unsigned char *p, uint32_t offset)
{
    typedef std::conditional_t<DT == kF32, u32x4_at4, u32x4_at2> chunk;
    const chunk *const a = (const chunk *)(p + offset);
    if constexpr (STREAM)
        return __builtin_nontemporal_load(a);
    else
        return *a;
}

template <int DT, bool STREAM = false>
__device__ __forceinline__ void store_whole(unsigned char *p, uint32_t offset, u32x4 raw)
{
    typedef std::conditional_t<DT == kF32, u32x4_at4, u32x4_at2> chunk;
    chunk *const a = (chunk *)(p + offset);
    if constexpr (STREAM)
        __builtin_nontemporal_store(raw, a);
    else
        *a = raw;
}

template <int DT>
__device__ __forceinline__ void unpack(u32x4 raw, float (&v)[kElems<DT>])
{
#pragma unroll
    for (int e = 0; e < 4; e++)
        if constexpr (DT == kF32) {
            v[e] = __uint_as_float(raw[e]);
        } else {
            v[2 * e] = __uint_as_float(raw[e] << 16);
            v[2 * e + 1] = __uint_as_float(raw[e] & 0xFFFF0000u);
        }
}

// rounded to nearest even, by the hardware's packed conversion
template <int DT>
__device__ __forceinline__ u32x4 pack(const float (&v)[kElems<DT>])
{
    u32x4 raw;
#pragma unroll
    for (int e = 0; e < 4; e++)
        if constexpr (DT == kF32) {
            raw[e] = __float_as_uint(v[e]);
        } else {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            raw[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{v[2 * e], v[2 * e + 1]}, bf16x2));
        }
    return raw;
}

template <int DT>
__device__ __forceinline__ void store_chunk(void *row, uint32_t c, uint32_t left, u32x4 raw)
{
    unsigned char *const a = (unsigned char *)row + (uint32_t)(c * kSize<DT>);
    if (left >= (uint32_t)kElems<DT>) {
        if constexpr (DT == kF32)
            *(u32x4_at4 *)a = raw;
        else
            *(u32x4_at2 *)a = raw;
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
        if constexpr (DT == kF32) {
            if ((uint32_t)e < left)
                ((uint32_t *)a)[e] = raw[e];
        } else {
            if (2u * e < left)
                ((uint16_t *)a)[2 * e] = (uint16_t)raw[e];
            if (2u * e + 1u < left)
                ((uint16_t *)a)[2 * e + 1] = (uint16_t)(raw[e] >> 16);
        }
}

// ---------------------------------------------------------------------------------------------------------------------
// Sums and maxima over LANES neighbouring lanes, in every one of them and with the same bits: each step adds a lane's number to
// that of its mirror image in a group twice as large, by DPP up to 16 lanes and by the half-exchanges of gfx950 above.
// ---------------------------------------------------------------------------------------------------------------------
struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};

template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}

template <typename Op, int LANES>
__device__ __forceinline__ float lanes_reduce(float v)
{
    static_assert(LANES == 8 || LANES == 16 || LANES == 32 || LANES == 64, "lanes");
    v = Op::of(v, dpp<0xB1>(v));                    // quad: neighbours
    v = Op::of(v, dpp<0x4E>(v));                    // quad: pairs
    v = Op::of(v, dpp<0x141>(v));                   // half rows of 8 mirrored
    if constexpr (LANES >= 16)
        v = Op::of(v, dpp<0x140>(v));               // rows of 16 mirrored
    if constexpr (LANES >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    if constexpr (LANES >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = Op::of(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    return v;
}

// Two numbers over a workgroup of WAVES wavefronts, in every thread.  `red`: 2 WAVES numbers of LDS that nothing else uses between
// the barrier before this call and the one after the next: calls in a row take turns with two such places.
template <typename OpA, typename OpB, int WAVES>
__device__ __forceinline__ void group_reduce(float &a, float &b, float *red)
{
    a = lanes_reduce<OpA, 64>(a);
    b = lanes_reduce<OpB, 64>(b);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6] = a;
            red[WAVES + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = red[0];
        b = red[WAVES];
#pragma unroll
        for (int w = 1; w < WAVES; w++) {
            a = OpA::of(a, red[w]);
            b = OpB::of(b, red[WAVES + w]);
        }
    }
}

}  // namespace tmask
