// The global norm of a list of gradients and their clipping (include/mitrain.h).
//
// norm = sqrt(sum g^2) over all tensors, then g min(1, max_norm / norm): two
// passes, as the factor needs every gradient.  Bound by memory: the first reads
// them (61 M fp32 gradients: 43 us, 5.7 TB/s), the second reads and writes them
// (75 us, 6.5 TB/s, as the caches hold a part of what the first has read).  The
// squares are summed in 64 bits (they overflow 32 from 2e19 on, and the
// instructions are hidden behind the loads); every workgroup of the second pass
// adds the first one's 1024 partial sums itself, in one order, which saves a
// launch between the two.
// The figures at the rules below are of whole calls replayed from a graph on
// three inputs in turn, both sides of a rule in one run.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

// Few tensors go by value with a launch's arguments, which hold below 4 KiB, so
// no table of them has to reach the device before; more of them are first
// written to a table in the workspace, kTensors a launch.
constexpr int kTensors = 112;
constexpr int kMaxParts = 1024;  // workgroups, and partial sums (2048: 123 -> 124 us)

struct TensorList {
    GradEntry e[kTensors];
};

static_assert(sizeof(TensorList) <= 3584, "kernel arguments");

// Tensors scaled in place, or not at all, need half the arguments: their chunks
// before each are counted here (280 small tensors: 20 us a call on the host, with
// kTensors a launch 23; 1000 tensors 47 and 62).
constexpr int kInPlace = 2 * kTensors;

struct InPlaceList {
    struct {
        const void *p;
        unsigned long long count_type;  // count * 4 + type
    } e[kInPlace];
};

static_assert(sizeof(InPlaceList) <= 3584, "kernel arguments");

__global__ __launch_bounds__(256) void write_table_in_place(InPlaceList l, int n, unsigned first,
                                                            GradEntry *table)
{
    __shared__ unsigned waves[4];
    const int t = threadIdx.x, lane = t & 63;
    const void *p = nullptr;
    long long count = 0;
    int type = 0;
    if (t < n) {
        p = l.e[t].p;
        count = (long long)(l.e[t].count_type >> 2);
        type = (int)(l.e[t].count_type & 3);
    }
    const long long most = kGradChunk / (type ? 2 : 4);
    const unsigned own = (unsigned)((count + most - 1) / most);
    unsigned sum = own;
    for (int o = 1; o < 64; o <<= 1) {
        const unsigned v = __shfl_up(sum, o);
        sum += lane >= o ? v : 0;
    }
    if (lane == 63)
        waves[t >> 6] = sum;
    __syncthreads();
    for (int i = 0; i < t >> 6; i++)
        first += waves[i];
    if (t < n)
        table[t] = GradEntry{p, (void *)p, count, first + sum - own, type};
}

__global__ __launch_bounds__(kTensors) void write_table(TensorList l, int n, GradEntry *table)
{
    if ((int)threadIdx.x < n)
        table[threadIdx.x] = l.e[threadIdx.x];
}

// The last of n entries that begins at chunk c or before it.  In the table by
// the lanes of a wave, 64 at a time; among the arguments (scalar loads) by
// halves.
__device__ __forceinline__ int entry_of(const GradEntry *e, int n, unsigned c, bool table)
{
    int lo = 0, hi = n;
    if (table) {
        const int lane = threadIdx.x & 63;
        while (hi - lo > 1) {
            const int step = (hi - lo + 63) / 64, at = lo + lane * step;
            const bool before = at < hi && e[at].first <= c;
            const int k = __popcll(__ballot(before)) - 1;
            lo += k * step;
            hi = min(hi, lo + step);
        }
        return __builtin_amdgcn_readfirstlane(lo);
    }
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (e[mid].first <= c)
            lo = mid;
        else
            hi = mid;
    }
    return lo;
}

// A workgroup's chunks: those of its share of all of them.
struct Share {
    unsigned first, end;
};

__device__ __forceinline__ Share share_of(unsigned chunks)
{
    return Share{(unsigned)((unsigned long long)chunks * blockIdx.x / gridDim.x),
                 (unsigned)((unsigned long long)chunks * (blockIdx.x + 1) / gridDim.x)};
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

// F packs of the n elements at p in flight, a pack a thread and step.  LAST: the
// last time that they are read (clipping 75 M gradients of which the caches
// hold a part, 288 tensors: 84 us instead of 91).
template <class T, int F, bool LAST, class Use>
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
                raw[f] = load_pack<T, LAST>(p + at, n - at, (T)0.f);
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
    each_pack<T, 4, false>(p, n, [&](typename Pack<T>::V v, int) {
#pragma unroll
        for (int j = 0; j < N; j++) {
            const double d = (double)(float)v[j];
            s[j & 3] = fma(d, d, s[j & 3]);
        }
    });
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// The share's chunks in order.
__device__ __forceinline__ void add_squares(const GradEntry *e, int n, unsigned chunks,
                                            double *parts, bool table)
{
    __shared__ double lds[4];
    const Share w = share_of(chunks);
    double s = 0;
    int i = entry_of(e, n, w.first, table);
    for (unsigned c = w.first; c < w.end; c++) {
        while (i + 1 < n && e[i + 1].first <= c)
            i++;
        const int most = kGradChunk >> (e[i].type == 0 ? 2 : 1);  // elements of a chunk
        const long long at = (long long)(c - e[i].first) * most;
        const int k = (int)min((long long)most, e[i].count - at);
        if (e[i].type == 0)
            s += chunk_squares((const float *)e[i].in + at, k);
        else if (e[i].type == 1)
            s += chunk_squares((const __bf16 *)e[i].in + at, k);
        else
            s += chunk_squares((const _Float16 *)e[i].in + at, k);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0)
        parts[blockIdx.x] = s;
}

__global__ __launch_bounds__(256) void squares_few(TensorList l, int n, unsigned chunks,
                                                   double *parts)
{
    add_squares(l.e, n, chunks, parts, false);
}

__global__ __launch_bounds__(256) void squares_table(const GradEntry *table, int n,
                                                     unsigned chunks, double *parts)
{
    add_squares(table, n, chunks, parts, true);
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

// g f 2^shift.
template <class T>
__device__ __forceinline__ void chunk_scale(const T *p, T *out, int n, float f, int shift)
{
    constexpr int N = Pack<T>::N;
    each_pack<T, 4, true>(p, n, [&](typename Pack<T>::V raw, int i) {
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++)
            v[j] = (T)ldexpf((float)raw[j] * f, shift);
        if (i < n)
            store_pack<T>(out + i, n - i, v);
    });
}

// The share's chunks in reverse: a workgroup of the same index has read them, the
// last ones most recently, and its caches hold them still.
__device__ __forceinline__ void scale_share(const GradEntry *e, int n, unsigned chunks,
                                            const double *parts, int nparts, float max_norm,
                                            float *norm, bool table)
{
    __shared__ double lds[4];
    const double v = norm_of(parts, nparts, lds);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0)
        *norm = (float)v;
    // The factor in 32 bits; one below their normal numbers (large gradients and a
    // small max_norm) is shifted into them, and its product with g back.
    const double factor = v <= (double)max_norm ? 1. : (double)max_norm / v;
    const int shift = factor < 0x1p-126 && factor > 0. ? ilogb(factor) + 126 : 0;
    const float f = (float)ldexp(factor, -shift);
    const Share w = share_of(chunks);
    if (w.first == w.end)
        return;
    int i = entry_of(e, n, w.end - 1, table);
    for (unsigned c = w.end; c-- > w.first;) {
        while (e[i].first > c)
            i--;
        if (f == 1.f && e[i].out == e[i].in)
            continue;  // in place, nothing to clip: as it is
        const int most = kGradChunk >> (e[i].type == 0 ? 2 : 1);  // elements of a chunk
        const long long at = (long long)(c - e[i].first) * most;
        const int k = (int)min((long long)most, e[i].count - at);
        if (e[i].type == 0)
            chunk_scale((const float *)e[i].in + at, (float *)e[i].out + at, k, f, shift);
        else if (e[i].type == 1)
            chunk_scale((const __bf16 *)e[i].in + at, (__bf16 *)e[i].out + at, k, f, shift);
        else
            chunk_scale((const _Float16 *)e[i].in + at, (_Float16 *)e[i].out + at, k, f, shift);
    }
}

__global__ __launch_bounds__(256) void clip_few(TensorList l, int n, unsigned chunks,
                                                const double *parts, int nparts, float max_norm,
                                                float *norm)
{
    scale_share(l.e, n, chunks, parts, nparts, max_norm, norm, false);
}

__global__ __launch_bounds__(256) void clip_table(const GradEntry *table, int n, unsigned chunks,
                                                  const double *parts, int nparts, float max_norm,
                                                  float *norm)
{
    scale_share(table, n, chunks, parts, nparts, max_norm, norm, true);
}

TensorList list_of(const GradEntry *e, int n)
{
    TensorList l;
    std::copy(e, e + n, l.e);
    return l;
}

// Workgroups: their shares differ by a chunk at most, so that few more chunks than
// kMaxParts are two for each of half as many (36 tensors of 9.4 M bf16: 15.7 us,
// in 1024 shares 18.2).
int blocks_of(unsigned chunks)
{
    const unsigned rounds = (chunks + kMaxParts - 1) / kMaxParts;
    return rounds ? (int)((chunks + rounds - 1) / rounds) : 0;
}

}  // namespace

size_t clip_ws(int n)
{
    return kMaxParts * sizeof(double) + (n > kTensors ? (size_t)n * sizeof(GradEntry) : 0);
}

hipError_t launch_clip(const GradEntry *e, int n, unsigned chunks, float max_norm, bool scale,
                       float *norm, void *ws, hipStream_t stream)
{
    double *parts = (double *)ws;
    GradEntry *table = (GradEntry *)(parts + kMaxParts);
    const int blocks = blocks_of(chunks);
    if (!n) {
        if (norm)
            norm_only<<<1, 256, 0, stream>>>(parts, 0, norm);
        return hipGetLastError();
    }
    if (n <= kTensors) {
        const TensorList l = list_of(e, n);
        squares_few<<<blocks, 256, 0, stream>>>(l, n, chunks, parts);
        if (scale)
            clip_few<<<blocks, 256, 0, stream>>>(l, n, chunks, parts, blocks, max_norm, norm);
    } else {
        const bool in_place = std::all_of(e, e + n, [](const GradEntry &g) {
            return !g.out || g.out == g.in;
        });
        for (int i = 0; i < n && in_place; i += kInPlace) {
            const int k = std::min(kInPlace, n - i);
            InPlaceList l;
            for (int j = 0; j < k; j++)
                l.e[j] = {e[i + j].in, (unsigned long long)e[i + j].count * 4 + e[i + j].type};
            write_table_in_place<<<1, 256, 0, stream>>>(l, k, e[i].first, table + i);
        }
        for (int i = 0; i < n && !in_place; i += kTensors) {
            const int k = std::min(kTensors, n - i);
            write_table<<<1, kTensors, 0, stream>>>(list_of(e + i, k), k, table + i);
        }
        squares_table<<<blocks, 256, 0, stream>>>(table, n, chunks, parts);
        if (scale)
            clip_table<<<blocks, 256, 0, stream>>>(table, n, chunks, parts, blocks, max_norm,
                                                   norm);
    }
    if (!scale)
        norm_only<<<1, 256, 0, stream>>>(parts, blocks, norm);
    return hipGetLastError();
}

}  // namespace miconv
