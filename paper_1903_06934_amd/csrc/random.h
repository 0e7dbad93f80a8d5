// The random numbers of include/mistep.h on the device.
#pragma once

#include <stdint.h>
#include <hip/hip_runtime.h>

#include "step.h"

namespace miconv {

// Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", 2011) of the counter {g, step, layer}: ten rounds of two 32 x 32 -> 64 bit products,
// whose low words change places with the other two words.  Both halves of a product are
// one instruction, at a quarter of the rate of others: some 20 of these and 60 others for
// eight elements, which is half of what a CU can do while the memory moves 16-bit
// elements in and out.
__device__ __forceinline__ void philox(uint32_t key0, uint32_t key1, uint32_t step, uint32_t layer,
                                       unsigned long long g, uint32_t (&w)[4])
{
    uint32_t a = (uint32_t)g, b = (uint32_t)(g >> 32), c = step, d = layer;
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const unsigned long long p = (unsigned long long)0xD2511F53u * a;
        const unsigned long long q = (unsigned long long)0xCD9E8D57u * c;
        a = (uint32_t)(q >> 32) ^ b ^ key0;
        c = (uint32_t)(p >> 32) ^ d ^ key1;
        b = (uint32_t)q;
        d = (uint32_t)p;
        key0 += 0x9E3779B9u;
        key1 += 0xBB67AE85u;
    }
    w[0] = a;
    w[1] = b;
    w[2] = c;
    w[3] = d;
}

// What a kernel holds of its Drop.
struct Dropper {
    uint32_t below, key0, key1, step, layer;
    float scale;

    __device__ __forceinline__ explicit Dropper(const Drop &d)
        : below(d.below), key0(d.key0), key1(d.key1), step(d.step), layer(d.layer), scale(d.scale)
    {
        if (d.step_at && below)
            step += (uint32_t)*d.step_at;
    }

    __device__ __forceinline__ void group(unsigned long long g, uint32_t (&w)[4]) const
    {
        philox(key0, key1, step, layer, g, w);
    }

    // Whether the element is kept whose bits are word's high half (odd), or its low one.
    __device__ __forceinline__ bool kept(uint32_t word, int odd) const
    {
        return (odd ? word >> 16 : word & 0xffff) >= below;
    }

    // The words of elements e .. e + N - 1 (N 4 or 8), which may lie in two groups.
    template <int N>
    __device__ __forceinline__ void words(long long e, uint32_t (&out)[N / 2]) const
    {
        uint32_t w[8];
        const int o = (int)(e & 7);
        {
            uint32_t g[4];
            group((unsigned long long)e >> 3, g);
#pragma unroll
            for (int i = 0; i < 4; i++)
                w[i] = g[i];
        }
        if (N == 8 && o == 0) {
#pragma unroll
            for (int i = 0; i < N / 2; i++)
                out[i] = w[i];
            return;
        }
#pragma unroll
        for (int i = 4; i < 8; i++)
            w[i] = 0;
        if (o + N > 8) {
            uint32_t g[4];
            group(((unsigned long long)e >> 3) + 1, g);
#pragma unroll
            for (int i = 0; i < 4; i++)
                w[4 + i] = g[i];
        }
        shifted<N>(w, o, out);
    }

    // The same for packs of eight that lie side by side in a wave, of which every lane calls
    // it: a pack's second group is the next lane's first, and the last lane's, the same for
    // all, is the scalar unit's.  For kernels with waves enough to hide that one's latency
    // (forward 16009 x 4369 bf16 144 us, with two groups a lane 173; backward, two waves a
    // SIMD, 246 and 227), of 16-bit elements (9000 x 2049 fp32 64.2 and 64.1, 9000 x 4096 fp32
    // 106.5 and 104.1).
    __device__ __forceinline__ void words_of_wave(long long e, uint32_t (&out)[4]) const
    {
        group((unsigned long long)e >> 3, out);
        const unsigned low = __builtin_amdgcn_readfirstlane((unsigned)e);
        const unsigned high =
            __builtin_amdgcn_readfirstlane((unsigned)((unsigned long long)e >> 32));
        if (low % 8 == 0)
            return;
        uint32_t s[4], w[8];
        group((((unsigned long long)high << 32 | low) >> 3) + 64, s);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            w[i] = out[i];
            // wave_shl:1; the last lane keeps s.
            w[4 + i] = __builtin_amdgcn_update_dpp((int)s[i], (int)w[i], 0x130, 0xf, 0xf, false);
        }
        shifted<8>(w, (int)(low & 7), out);
    }

    // The N half words from the o-th (below 8) of w on.
    template <int N>
    static __device__ __forceinline__ void shifted(uint32_t (&w)[8], int o, uint32_t (&out)[N / 2])
    {
        if (o & 4)
#pragma unroll
            for (int i = 0; i < 6; i++)
                w[i] = w[i + 2];
        if (o & 2)
#pragma unroll
            for (int i = 0; i < 5; i++)
                w[i] = w[i + 1];
        if (o & 1)
#pragma unroll
            for (int i = 0; i < N / 2; i++)
                w[i] = w[i] >> 16 | w[i + 1] << 16;
#pragma unroll
        for (int i = 0; i < N / 2; i++)
            out[i] = w[i];
    }

    // Whether element e is kept.
    __device__ __forceinline__ bool one(long long e) const
    {
        uint32_t g[4];
        group((unsigned long long)e >> 3, g);
        const int h = (int)(e & 7);
        const uint32_t w = h & 4 ? (h & 2 ? g[3] : g[2]) : (h & 2 ? g[1] : g[0]);
        return kept(w, h & 1);
    }
};

}  // namespace miconv
