// Device helpers of the operators on rows of 32- and 16-bit floating-point
// elements (norm_kernels.hip, logprob_kernels.hip, clip_kernels.hip).
#pragma once

#include <stdint.h>
#include <hip/hip_runtime.h>

namespace miconv {

// Workgroups of one launch, at most: a grid holds below 2^32 threads.
constexpr long long kMaxBlocks = 1LL << 21;

// 16 bytes of elements.  Rows may begin at any element, so a vector is loaded
// and stored with its element's alignment: the memory instructions of gfx950
// take a 16-byte access at any such address in one instruction.
template <class T>
struct Pack {
    static constexpr int N = 16 / (int)sizeof(T);
    typedef T V __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef V At __attribute__((aligned(sizeof(T))));  // as it lies in memory
};

// The N elements at p of which the first `left` (>= 1) are in the row; the
// others are `fill`.
template <class T, bool STREAM = false>
__device__ __forceinline__ typename Pack<T>::V load_pack(const T *p, long long left, T fill)
{
    typename Pack<T>::V v;
    if (left >= Pack<T>::N) {
        const auto *at = (const typename Pack<T>::At *)p;
        v = STREAM ? __builtin_nontemporal_load(at) : *at;
    } else {
#pragma unroll
        for (int i = 0; i < Pack<T>::N; i++)
            v[i] = i < left ? p[i] : fill;
    }
    return v;
}

template <class T>
__device__ __forceinline__ void store_pack(T *p, long long left, typename Pack<T>::V v)
{
    if (left >= Pack<T>::N) {
        __builtin_nontemporal_store(v, (typename Pack<T>::At *)p);
    } else {
#pragma unroll
        for (int i = 0; i < Pack<T>::N; i++)
            if (i < left)
                p[i] = v[i];
    }
}

// Sum (or maximum) over the `width` threads of a group, in a fixed order; every
// thread of the group gets it.  width is a power of two up to the 64 lanes of a
// wave, or the whole workgroup, whose waves then meet in `lds` (one value a
// wave; the caller takes another part of it for the next reduction, so that one
// barrier is enough).
struct Add {
    __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Max {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};

// Within a wave without LDS: lanes of 4, 8 and 16 exchange by DPP (quad_perm,
// row_half_mirror, row_mirror: after each step its two partners hold their
// halves' results), rows of 16 and halves of 32 by swaps.
template <int CTRL>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(
        __builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}

template <class Op>
__device__ __forceinline__ float wave_reduce(float v, int width, Op op)
{
    if (width > 1)
        v = op(v, dpp<0xb1>(v));
    if (width > 2)
        v = op(v, dpp<0x4e>(v));
    if (width > 4)
        v = op(v, dpp<0x141>(v));
    if (width > 8)
        v = op(v, dpp<0x140>(v));
    if (width > 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if (width > 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}

template <class Op>
__device__ __forceinline__ float group_reduce(float v, int width, float *lds, Op op)
{
    v = wave_reduce(v, width, op);
    if (width > 64) {
        const int waves = width >> 6;
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
        for (int i = 1; i < waves; i++)
            v = op(v, lds[i]);
    }
    return v;
}

}  // namespace miconv
