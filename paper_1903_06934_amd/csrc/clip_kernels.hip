// The global norm of a list of gradients and their clipping (include/mitrain.h).
// Memory-bound: every gradient is read for the norm, then read and written for
// its clipping.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

// The tensors of one launch go by value with its arguments, which hold below
// 4 KiB: so no table of them has to reach the device.
#ifndef FS
#define FS 4
#endif
#ifndef FC
#define FC 4
#endif
#ifndef CH
#define CH 16384
#endif
#ifndef MP
#define MP 1024
#endif
constexpr int kTensors = 112;
constexpr int kChunk = CH;     // elements of a tensor that a workgroup takes at once
constexpr int kMaxParts = MP;   // workgroups, and partial sums, of a launch

struct TensorList {
    const void *in[kTensors];
    void *out[kTensors];
    long long count[kTensors];
    unsigned first[kTensors + 1];  // chunks before tensor i
    unsigned char type[kTensors];
    int n;
};

static_assert(sizeof(TensorList) <= 3840, "kernel arguments");

// The tensor of chunk c.
__device__ __forceinline__ int tensor_of(const TensorList &l, unsigned c)
{
    int lo = 0, hi = l.n;  // first[lo] <= c < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (l.first[mid] <= c)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// Sum over a workgroup of 256 threads, in a fixed order.
__device__ __forceinline__ double block_sum(double v, double *lds)
{
    for (int o = 1; o < 64; o <<= 1)
        v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return lds[0] + lds[1] + (lds[2] + lds[3]);
}

// F packs of the n elements at p in flight, a pack a thread and step.
template <class T, int F, class Use>
__device__ __forceinline__ void each_pack(const T *p, int n, Use use)
{
    constexpr int N = Pack<T>::N;
    for (int i = threadIdx.x * N; i < n; i += F * 256 * N) {
        typename Pack<T>::V raw[F];
#pragma unroll
        for (int f = 0; f < F; f++) {
            const int at = i + f * 256 * N;
            raw[f] = typename Pack<T>::V{};
            if (at < n)
                raw[f] = load_pack<T>(p + at, n - at, (T)0.f);
        }
#pragma unroll
        for (int f = 0; f < F; f++)
            use(raw[f], i + f * 256 * N);
    }
}

template <class T>
__device__ __forceinline__ double chunk_squares(const T *p, int n)
{
    constexpr int N = Pack<T>::N;
    double s[4] = {0, 0, 0, 0};
    each_pack<T, FS>(p, n, [&](typename Pack<T>::V v, int) {
#pragma unroll
        for (int j = 0; j < N; j++) {
            const double d = (double)(float)v[j];
            s[j & 3] = fma(d, d, s[j & 3]);
        }
    });
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(256) void squares(TensorList l, double *parts)
{
    __shared__ double lds[4];
    double s = 0;
    for (unsigned c = blockIdx.x; c < l.first[l.n]; c += gridDim.x) {
        const int i = tensor_of(l, c);
        const long long at = (long long)(c - l.first[i]) * kChunk;
        const int n = (int)min((long long)kChunk, l.count[i] - at);
        if (l.type[i] == 0)
            s += chunk_squares((const float *)l.in[i] + at, n);
        else if (l.type[i] == 1)
            s += chunk_squares((const __bf16 *)l.in[i] + at, n);
        else
            s += chunk_squares((const _Float16 *)l.in[i] + at, n);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0)
        parts[blockIdx.x] = s;
}

// The norm from the partial sums; every workgroup of 256 threads computes the
// same one.
__device__ __forceinline__ double norm_of(const double *parts, int n, double *lds)
{
    double s = 0;
    for (int i = threadIdx.x; i < n; i += 256)
        s += parts[i];
    return sqrt(block_sum(s, lds));
}

__global__ __launch_bounds__(256) void norm_only(const double *parts, int n, float *norm)
{
    __shared__ double lds[4];
    const double v = norm_of(parts, n, lds);
    if (threadIdx.x == 0)
        *norm = (float)v;
}

template <class T>
__device__ __forceinline__ void chunk_scale(const T *p, T *out, int n, float f)
{
    constexpr int N = Pack<T>::N;
    each_pack<T, FC>(p, n, [&](typename Pack<T>::V raw, int i) {
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++)
            v[j] = (T)((float)raw[j] * f);
        if (i < n)
            store_pack<T>(out + i, n - i, v);
    });
}

__global__ __launch_bounds__(256) void clip(TensorList l, const double *parts, int nparts,
                                            float max_norm, float *norm)
{
    __shared__ double lds[4];
    const double v = norm_of(parts, nparts, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0)
        *norm = (float)v;
    const float f = v <= (double)max_norm ? 1.f : (float)((double)max_norm / v);
    // The chunks that the norm read last come first: the caches still hold them.
    const unsigned chunks = l.first[l.n];
    for (unsigned b = blockIdx.x; b < chunks; b += gridDim.x) {
        const unsigned c = chunks - 1 - b;
        const int i = tensor_of(l, c);
        const long long at = (long long)(c - l.first[i]) * kChunk;
        const int n = (int)min((long long)kChunk, l.count[i] - at);
        if (f == 1.f && l.out[i] == l.in[i])
            continue;  // in place, nothing to clip: as it is
        if (l.type[i] == 0)
            chunk_scale((const float *)l.in[i] + at, (float *)l.out[i] + at, n, f);
        else if (l.type[i] == 1)
            chunk_scale((const __bf16 *)l.in[i] + at, (__bf16 *)l.out[i] + at, n, f);
        else
            chunk_scale((const _Float16 *)l.in[i] + at, (_Float16 *)l.out[i] + at, n, f);
    }
}

// Fills l with the tensors from `from` on, at most kTensors and 2^31 chunks; the
// first tensor not in it.  Empty ones are left out.
int fill(TensorList &l, int from, int n, const void *const *grads, void *const *out,
         const long long *count, const int *types)
{
    l.n = 0;
    unsigned long long chunks = 0;
    int i = from;
    for (; i < n && l.n < kTensors; i++) {
        if (!count[i])
            continue;
        const unsigned long long c = (unsigned long long)((count[i] + kChunk - 1) / kChunk);
        l.in[l.n] = grads[i];
        l.out[l.n] = out ? out[i] : nullptr;
        l.count[l.n] = count[i];
        l.type[l.n] = (unsigned char)types[i];
        l.first[l.n++] = (unsigned)chunks;
        chunks += c;
    }
    l.first[l.n] = (unsigned)chunks;
    return i;
}

int blocks_of(const TensorList &l)
{
    return (int)std::min<unsigned>(l.first[l.n], kMaxParts);
}

}  // namespace

size_t clip_ws(int n, const long long *count, const int *types)
{
    (void)types;
    int some = 0;
    for (int i = 0; i < n; i++)
        some += count[i] > 0;
    return (size_t)(some + kTensors - 1) / kTensors * kMaxParts * sizeof(double);
}

hipError_t launch_clip(int n, const void *const *grads, const long long *count, const int *types,
                       float max_norm, void *const *out, float *norm, double *ws,
                       hipStream_t stream)
{
    TensorList l;
    int nparts = 0;
    for (int i = 0; i < n;) {
        i = fill(l, i, n, grads, out, count, types);
        if (!l.n)
            break;
        squares<<<blocks_of(l), 256, 0, stream>>>(l, ws + nparts);
        nparts += blocks_of(l);
    }
    if (!out || !nparts) {
        if (norm)
            norm_only<<<1, 256, 0, stream>>>(ws, nparts, norm);
        return hipGetLastError();
    }
    for (int i = 0; i < n;) {
        i = fill(l, i, n, grads, out, count, types);
        if (!l.n)
            break;
        clip<<<blocks_of(l), 256, 0, stream>>>(l, ws, nparts, max_norm, norm);
        norm = nullptr;
    }
    return hipGetLastError();
}

}  // namespace miconv
