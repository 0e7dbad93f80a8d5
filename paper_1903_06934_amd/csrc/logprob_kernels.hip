// Log probabilities of given tokens, entropy and the likeliest tokens of rows
// of logits, and their gradient (include/mitrain.h).
//
// Forward, one pass over the row: every thread keeps a running maximum m of its
// logits, sum e and sum (z - m) e with e = exp(scale (z - m)); a larger maximum
// scales both sums.  From the joined sums, lse = scale m + ln sum e and the
// entropy = ln sum e - scale (sum (z - m) e) / sum e, without a second pass.  The
// top comes from the same pass: the k-th largest of the threads' (groups')
// maxima bounds the k-th largest logit from below, so only the packs of the few
// threads that reach it are looked at again.
//
// Bound by memory in large calls (4096 x 32000 bf16: 46 us, 5.7 TB/s; of about
// 11 instructions an element the exponential takes the time of four), by
// latencies in small ones (128 x 1000 fp32 with 5 alternatives: 5.4 us, one
// row a workgroup).  Backward, every element is read and written once and its
// probability computed from the row's two statistics: 4096 x 32000 bf16 in
// 90 us, 5.8 TB/s.
// The figures at the rules below are of whole calls replayed from a graph on
// three inputs in turn, both sides of a rule in one run: launches and their gaps
// (1.6 us and more) are in them.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

// The hardware's 2^x: results below 2^-126 may be 0, beside sums of at least 1
// forward and as probabilities backward.
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// ----------------------------------------------------------- one pass of a row
// A part of a softmax's sums about its running maximum m (of the unscaled
// logits, NaN aside): s = sum e, t = sum (z - m) e with e = exp(scale (z - m)).
// m is -inf, and s = t = 0, while every logit was -inf; a NaN or +inf leaves s
// NaN.
struct Soft {
    float m, s, t;
};

// (z - m) with banned logits at a finite value, so that their e = 0 makes 0.
__device__ __forceinline__ float shifted(float z, float m) { return fmaxf(z - m, -1e30f); }

// p about the maximum m >= p.m.
__device__ __forceinline__ Soft about(Soft p, float m, float c)
{
    if (m == -kInf)
        return p;  // sums of zeros, or NaN
    const float u = shifted(p.m, m), e = exp2_(u * c);
    return Soft{m, p.s * e, (p.t + u * p.s) * e};
}


// The lanes' parts joined: first the maximum, then each part about it.
__device__ __forceinline__ Soft wave_merge(Soft p, float c)
{
    const float m = wave_reduce(p.m, 64, Max());
    p = about(p, m, c);
    return Soft{m, wave_reduce(p.s, 64, Add()), wave_reduce(p.t, 64, Add())};
}

// F packs' logits.  A maximum of nothing but -inf and NaN so far is taken as 0.
template <class T, int F>
__device__ __forceinline__ void add_packs(Soft &p, const typename Pack<T>::V (&raw)[F], float c)
{
    constexpr int N = Pack<T>::N;
    float m = p.m;
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < N; j++)
            m = fmaxf(m, (float)raw[i][j]);
    if (m > p.m)
        p = about(p, m, c);
    const float base = m == -kInf ? 0.f : m;
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < F; i++)
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float u = (float)raw[i][j] - base, e = exp2_(u * c);
            s += e;
            t += fmaxf(u, -1e30f) * e;
        }
    p.s += s;
    p.t += t;
}

// --------------------------------------------------------------------- the top
// Order of the logits: unsigned, rising with the value; the zeros are equal and
// a NaN counts as -inf.  A token's key is its order and then its index, falling.
__device__ __forceinline__ float ranked(float z) { return z == z ? z + 0.f : -kInf; }
__device__ __forceinline__ uint32_t order(float z)
{
    const uint32_t u = __float_as_uint(z);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unorder(uint32_t o)
{
    return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t key(float z, uint32_t index)
{
    return (uint64_t)order(ranked(z)) << 32 | (0xffffffffu - index);
}

// A row (or piece) is worked on by a team of SIZE threads: a workgroup, or for
// short rows a wave, four of which share a workgroup and never meet.
template <int SIZE>
struct Team {
    static constexpr int kSize = SIZE;
    static constexpr int kWaves = SIZE / 64;
    static constexpr int kKeys = SIZE < 128 ? 256 : 1024;    // tokens at or above the bound in LDS

    struct Shared {
        alignas(16) float group[SIZE < 128 ? 64 : 128];
        Soft soft[kWaves];
        float bound;
        int count, nactive;
        unsigned short active[SIZE];
        int wave[kWaves];
        uint64_t keys[kKeys];
    };

    static __device__ __forceinline__ int thread() { return SIZE == 64 ? threadIdx.x & 63 : threadIdx.x; }

    static __device__ __forceinline__ void sync()
    {
        if constexpr (SIZE == 64) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }

    static __device__ __forceinline__ Soft join(Shared &sh, Soft p, float c)
    {
        p = wave_merge(p, c);
        if constexpr (SIZE > 64) {
            if ((threadIdx.x & 63) == 0)
                sh.soft[threadIdx.x >> 6] = p;
            __syncthreads();
            const int lane = threadIdx.x & 63;
            p = lane < kWaves ? sh.soft[lane] : Soft{-kInf, 0.f, 0.f};
            p = wave_merge(p, c);
        }
        return p;
    }

    static __device__ __forceinline__ int sum(Shared &sh, int v)
    {
        for (int o = 1; o < 64; o <<= 1)
            v += __shfl_xor(v, o);
        if constexpr (SIZE > 64) {
            __syncthreads();
            if ((threadIdx.x & 63) == 0)
                sh.wave[threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0;
            for (int i = 0; i < kWaves; i++)
                v += sh.wave[i];
        }
        return v;
    }
};

// A lower bound of the k-th largest logit: the k-th largest of the maxima of 64
// groups of threads, or 128 where a workgroup looks for more than 32 (so at least
// k elements reach it, and few more where large logits lie anywhere: about
// -G ln(1 - k / G) of G groups).  mine: the thread's maximum.
template <class Tm>
__device__ __forceinline__ float top_bound(typename Tm::Shared &sh, float mine, int k)
{
    const int t = Tm::thread();
    const int groups = Tm::kSize > 64 && k > 32 ? 128 : 64, per = Tm::kSize / groups;
    const float gm = wave_reduce(mine, per, Max());
    if (t % per == 0)
        sh.group[t / per] = gm;
    if (t == 0)
        sh.count = sh.nactive = 0;
    Tm::sync();
    if (t < 64) {
        // The largest that k of them reach.
        float bound = -kInf;
        for (int g = t; g < groups; g += 64) {
            const float own = sh.group[g];
            int reach = 0;
#pragma unroll 8
            for (int i = 0; i < groups; i += 4) {
                const float4 o = *(const float4 *)&sh.group[i];
                reach += (o.x >= own) + (o.y >= own) + (o.z >= own) + (o.w >= own);
            }
            if (reach >= k)
                bound = fmaxf(bound, own);
        }
        bound = wave_reduce(bound, 64, Max());
        if (t == 0)
            sh.bound = bound;
    }
    Tm::sync();
    return sh.bound;
}

// Ranks n keys in LDS and hands rank and key of the first k to put.
template <class Put>
__device__ __forceinline__ void put_ranked(const uint64_t *keys, int n, int k, int thread, int size,
                                           Put put)
{
    for (int i = thread; i < n; i += size) {
        const uint64_t mine = keys[i];
        int above = 0;
#pragma unroll 4
        for (int j = 0; j < n; j++)
            above += keys[j] > mine;
        if (above < k)
            put(above, mine);
    }
}

// Of n keys in LDS, those that can be among the first k: a bound as above from
// the keys dealt out to the groups, where the first one let many through (a row
// with elements in few groups).  Ranking them all takes n^2 steps: 2 x 130 bf16
// with 20 alternatives 14.0 us, so 8.2.  They stay in LDS; returns their number.
template <class Tm, int SIZE>
__device__ __forceinline__ int fewer_keys(typename Tm::Shared &sh, int n, int k)
{
    constexpr int PER = Tm::kKeys / SIZE < 1 ? 1 : Tm::kKeys / SIZE;  // keys a thread, at most
    const int t = Tm::thread();
    uint64_t own[PER], most = 0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        own[i] = t + i * SIZE < n ? sh.keys[t + i * SIZE] : 0;
        most = own[i] > most ? own[i] : most;
    }
    Tm::sync();  // all have read sh.count, which top_bound clears
    const float bound = top_bound<Tm>(sh, most ? unorder((uint32_t)(most >> 32)) : -kInf, k);
#pragma unroll
    for (int i = 0; i < PER; i++)
        if (own[i] && unorder((uint32_t)(own[i] >> 32)) >= bound)
            sh.keys[atomicAdd(&sh.count, 1)] = own[i];
    Tm::sync();
    return sh.count;
}

// Elements of z[0, n) above v.
template <class T, class Tm, int SIZE>
__device__ int count_above(typename Tm::Shared &sh, const T *z, int n, float v)
{
    constexpr int N = Pack<T>::N;
    int c = 0;
    for (int i = Tm::thread() * N; i < n; i += SIZE * N) {
        const auto raw = load_pack<T>(z + i, n - i, (T)-kInf);
#pragma unroll
        for (int j = 0; j < N; j++)
            c += (float)raw[j] > v;
    }
    return Tm::sum(sh, c);
}

// The keys of the top k of z[0, n) (and of some more, kKeys at most) where too
// many elements reach the bound: by bisection a larger one that few enough lie
// above, or, where equal elements stand in the way, the elements above them and
// of them the first.  Returns the keys' number.
template <class T, class Tm, int SIZE>
__device__ __noinline__ int top_by_value(typename Tm::Shared &sh, const T *z, int n,
                                         uint32_t first, int k, float bound, float most)
{
    constexpr int N = Pack<T>::N;
    uint32_t lo = order(ranked(bound)), hi = order(ranked(most));
    int above = count_above<T, Tm, SIZE>(sh, z, n, bound);
    bool equal_ones = above < k;  // elements equal to the bound are in the top
    while (!equal_ones && above > Tm::kKeys) {
        // k or more lie above lo, fewer above hi.
        if (hi - lo == 1) {
            lo = hi;
            equal_ones = true;
            break;
        }
        const uint32_t mid = lo + (hi - lo) / 2;
        const int c = count_above<T, Tm, SIZE>(sh, z, n, unorder(mid));
        if (c < k) {
            hi = mid;
        } else {
            lo = mid;
            above = c;
        }
    }
    const float v = unorder(lo);
    const int t = Tm::thread();
    Tm::sync();
    if (t == 0)
        sh.count = 0;
    Tm::sync();
    for (int i = t * N; i < n; i += SIZE * N) {
        const auto raw = load_pack<T>(z + i, n - i, (T)-kInf);
#pragma unroll
        for (int j = 0; j < N; j++)
            if ((float)raw[j] > v)
                sh.keys[atomicAdd(&sh.count, 1)] = key((float)raw[j], first + i + j);
    }
    Tm::sync();
    int have = sh.count;
    if (!equal_ones)
        return have;
    for (int base = 0; base < n && have < k; base += SIZE) {
        const int i = base + t;
        const bool equal = i < n && ranked((float)z[i]) == v;
        const uint64_t ballot = __ballot(equal);
        const int lane = t & 63, wave = t >> 6;
        Tm::sync();
        if (lane == 0)
            sh.wave[wave] = __popcll(ballot);
        Tm::sync();
        int at = have + __popcll(ballot & ((1ull << lane) - 1));
        for (int w = 0; w < Tm::kWaves; w++) {
            at += w < wave ? sh.wave[w] : 0;
            have += sh.wave[w];
        }
        if (equal && at < k)
            sh.keys[at] = key(v, first + i);
    }
    Tm::sync();
    return k;
}

// The sums' results.  none: the row bans every token (lse alone does not tell: a
// row of the type's lowest value times a scale above 1 is beyond 32 bits too).
struct Done {
    float lse, entropy, log_s;
    bool none;
};

__device__ __forceinline__ Done finish(Soft p, float scale)
{
    if (p.m == -kInf && p.s == 0.f)
        return Done{-kInf, 0.f, 0.f, true};
    const float log_s = logf(p.s);
    return Done{p.m * scale + log_s, log_s - scale * (p.t / p.s), log_s, false};
}

__device__ __forceinline__ float log_prob(float z, Soft p, Done d, float scale)
{
    if (d.none)
        return -kInf;
    const float u = z - p.m;  // beyond 32 bits where the scaled one need not be
    return (u == -kInf && z > -kInf ? z * scale - p.m * scale : u * scale) - d.log_s;
}

// The logit of a row's given token.
template <class T>
__device__ __forceinline__ float logit_of(const LogprobArgs &a, long long row, long long token)
{
    return token >= 0 && token < a.vocab
               ? (float)((const T *)a.logits.p)[row * a.logits.ld + token]
               : 0.f;
}

__device__ __forceinline__ void write_row(const LogprobArgs &a, long long row, long long token,
                                          float z, Soft p, Done d)
{
    if (a.lse)
        a.lse[row] = d.lse;
    if (a.entropy)
        a.entropy[row] = d.entropy;
    if (a.stats) {
        a.stats[2 * row] = p.m;
        a.stats[2 * row + 1] = d.log_s;
    }
    if (a.logp) {
        float lp = 0.f;
        if (token >= a.vocab)
            lp = __builtin_nanf("");
        else if (token >= 0)
            lp = log_prob(z, p, d, a.scale);
        a.logp[row] = lp;
    }
}

__device__ __forceinline__ void put_top(const LogprobArgs &a, long long row, int rank, uint64_t k,
                                        Soft p, Done d)
{
    a.top_index[row * a.top + rank] = 0xffffffffu - (uint32_t)k;
    a.top_logp[row * a.top + rank] = log_prob(unorder((uint32_t)(k >> 32)), p, d, a.scale);
}

// A team a row, or a piece of it: then the piece's sums and its top go to ws,
// as parts[row][split] and keys[row][split][top].
template <class T, int SIZE>
__global__ __launch_bounds__(SIZE < 256 ? 256 : SIZE) void logprob_rows(LogprobArgs a, int piece,
                                                                        int splits, bool through,
                                                                        Soft *parts, uint64_t *keys)
{
    using Tm = Team<SIZE>;
    // Two packs in flight a thread: more lengthen the short rows (8000 x 1000 bf16
    // 8.0 us, with 4 and 8 packs 9.4 and 12.7) and gain little on the long ones
    // (4096 x 32000 49.8, 49.6 and 49.3; with one 53.1).
    constexpr int N = Pack<T>::N, F = 2, TEAMS = SIZE < 256 ? 256 / SIZE : 1;
    __shared__ typename Tm::Shared shared[TEAMS];
    const int team = TEAMS > 1 ? threadIdx.x / SIZE : 0;
    typename Tm::Shared &sh = shared[team];
    const long long item = (long long)blockIdx.x * TEAMS + team;
    const long long row = splits == 1 ? item : item / splits;
    if (row >= a.rows)
        return;
    const int split = (int)(item - row * splits), t = Tm::thread();
    const int first = split * piece, n = (int)min((long long)piece, a.vocab - first);
    const T *z = (const T *)a.logits.p + row * a.logits.ld + first;
    const float c = a.scale * kLog2e;
    const long long token = splits == 1 && a.logp ? a.targets[row] : -1;
    typename Pack<T>::V raw[F];
    const auto load = [&](int i) {
#pragma unroll
        for (int f = 0; f < F; f++) {
            const int at = i + f * SIZE * N;
            raw[f] = typename Pack<T>::V((T)-kInf);
            if (at < n)
                raw[f] = through ? load_pack<T, true>(z + at, n - at, (T)-kInf)
                                 : load_pack<T>(z + at, n - at, (T)-kInf);
        }
    };
    Soft p{-kInf, 0.f, 0.f};
    for (int i = t * N; i < n; i += F * SIZE * N) {
        load(i);
        add_packs<T, F>(p, raw, c);
    }
    const float zt = logit_of<T>(a, row, token);
    const float mine = p.m;
    p = Tm::join(sh, p, c);
    const Done d = finish(p, a.scale);
    if (t == 0) {
        if (splits == 1)
            write_row(a, row, token, zt, p, d);
        else
            parts[item] = p;
    }
    if (!a.top)
        return;
    const int k = min(a.top, n);
    const float bound = top_bound<Tm>(sh, mine, k);
    const auto collect = [&](typename Pack<T>::V v, int i) {
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float f = ranked((float)v[j]);
            if (f >= bound && i + j < n) {
                const int at = atomicAdd(&sh.count, 1);
                if (at < Tm::kKeys)
                    sh.keys[at] = key(f, first + i + j);
            }
        }
    };
    const int rounds = (n + SIZE * N - 1) / (SIZE * N);  // packs of a thread
    if (rounds <= F) {  // in its registers still, if it has any
        if (t * N < n && mine >= bound)
#pragma unroll
            for (int f = 0; f < F; f++)
                collect(raw[f], (t + f * SIZE) * N);
    } else {
        // The packs of the threads that reach the bound, dealt out to all.
        if (mine >= bound)
            sh.active[atomicAdd(&sh.nactive, 1)] = t;
        Tm::sync();
        const int items = sh.nactive * rounds;
        for (int i = t; i < items; i += SIZE) {
            if (*(volatile int *)&sh.count > Tm::kKeys)
                break;
            const int at = (sh.active[i / rounds] + i % rounds * SIZE) * N;
            if (at < n)
                collect(load_pack<T>(z + at, n - at, (T)0.f), at);
        }
    }
    Tm::sync();
    int found = sh.count;
    if (found > Tm::kKeys)
        found = top_by_value<T, Tm, SIZE>(sh, z, n, first, k, bound, p.m);
    if (found > 2 * k + 8)
        found = fewer_keys<Tm, SIZE>(sh, found, k);
    if (splits == 1)
        put_ranked(sh.keys, found, k, t, SIZE,
                   [&](int rank, uint64_t ky) { put_top(a, row, rank, ky, p, d); });
    else
        put_ranked(sh.keys, found, k, t, SIZE,
                   [&](int rank, uint64_t ky) { keys[item * a.top + rank] = ky; });
}

// Joins the pieces (two at least, at most kPieces) of a row.  Each has sorted
// keys; all but the last have `top` of them.  A bound as above: the top-th of
// the first q keys of each piece, q the fewest that make `top` of them.
constexpr int kPieces = 64;

template <class T>
__global__ __launch_bounds__(256) void logprob_join(LogprobArgs a, int piece, int splits,
                                                    const Soft *parts, const uint64_t *keys)
{
    __shared__ uint64_t heads[256], found[kPieces * 64];
    __shared__ uint64_t bound;
    __shared__ int count;
    const long long row = blockIdx.x;
    const int lane = threadIdx.x & 63, top = a.top;
    const float c = a.scale * kLog2e;
    const long long token = a.logp ? a.targets[row] : -1;
    Soft p{-kInf, 0.f, 0.f};
    if (lane < splits)
        p = parts[row * splits + lane];
    const int last = (int)min((long long)top, a.vocab - (long long)(splits - 1) * piece);
    const int q = (top + splits - 2) / (splits - 1);
    const int nheads = (splits - 1) * q + min(q, last);
    const uint64_t *list = keys + row * splits * top;
    // heads[i]: key i % q of piece i / q.  q (splits - 1) < top + splits, so all
    // of them are fewer than 64 + 2 * 64.
    if ((int)threadIdx.x < nheads)
        heads[threadIdx.x] = list[threadIdx.x / max(q, 1) * top + threadIdx.x % max(q, 1)];
    if (threadIdx.x == 0)
        count = 0;
    const float zt = logit_of<T>(a, row, token);
    p = wave_merge(p, c);
    const Done d = finish(p, a.scale);
    if (threadIdx.x == 0)
        write_row(a, row, token, zt, p, d);
    if (!top)
        return;
    __syncthreads();
    put_ranked(heads, nheads, top, threadIdx.x, 256, [&](int rank, uint64_t k) {
        if (rank == top - 1)
            bound = k;
    });
    __syncthreads();
    const int n = (splits - 1) * top + last;
    for (int i = threadIdx.x; i < n; i += 256) {
        const uint64_t k = list[i];
        if (k >= bound)
            found[atomicAdd(&count, 1)] = k;
    }
    __syncthreads();
    put_ranked(found, count, top, threadIdx.x, 256,
               [&](int rank, uint64_t k) { put_top(a, row, rank, k, p, d); });
}

// -------------------------------------------------------------------- backward
// Groups of tpr threads (a power of two up to 256) take NV packs each: of a row
// each, or, as a workgroup, of the piece blockIdx.x of row blockIdx.y.  NV = 2
// (4096 x 32000 bf16: 96 us; with 1, 3, 4 and 8 packs 105, 104, 96 and 105).
// An element in place is read before its thread writes it, and by no other.
template <class T, int NV>
__global__ __launch_bounds__(256) void logprob_back(LogprobBwdArgs a, int tpr)
{
    constexpr int N = Pack<T>::N;
    const int t = threadIdx.x & (tpr - 1), vocab = (int)a.vocab;
    const long long row = tpr == 256 ? blockIdx.y : blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
    if (row >= a.rows)
        return;
    const int first = tpr == 256 ? blockIdx.x * (256 * N * NV) : 0;
    const T *z = (const T *)a.logits.p + row * a.logits.ld;
    T *dz = (T *)a.dlogits.p + row * a.dlogits.ld;
    typename Pack<T>::V raw[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = first + (t + i * tpr) * N;
        raw[i] = typename Pack<T>::V{};
        if (c < vocab)
            raw[i] = load_pack<T>(z + c, vocab - c, (T)0.f);
    }
    const float peak = a.stats[2 * row], log_s = a.stats[2 * row + 1], scale = a.scale;
    const long long target = a.dlogp ? a.targets[row] : -1;
    float dl = target >= 0 ? a.dlogp[row] * scale : 0.f;
    if (target >= vocab)
        dl = __builtin_nanf("");
    const float de = a.dentropy ? a.dentropy[row] * scale : 0.f;
    const float ent = a.dentropy ? a.entropy[row] : 0.f;
    const bool none = peak == -kInf && log_s == 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = first + (t + i * tpr) * N;
        if (c >= vocab)
            continue;
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float lp = fmaf((float)raw[i][j] - peak, scale, -log_s);
            const float p = exp2_(lp * kLog2e);
            float f = -p * dl;
            if (a.dentropy)
                f -= de * p * (fmaxf(lp, -1e30f) + ent);
            if (c + j == target)
                f += dl;
            if (none)
                f = target >= vocab ? dl : 0.f;
            v[j] = (T)f;
        }
        store_pack<T>(dz + c, vocab - c, v);
    }
}

// ----------------------------------------------------------------- launch rules
int pack_of(int xtype) { return xtype == 0 ? 4 : 8; }

// Pieces of a row, and the threads of a team.
// Pieces: with a quarter of the CUs' number of rows or fewer, as many as fill
// the CUs, of at least 4096 elements, up to kPieces (4 x 131072 bf16 with 20
// alternatives: 13.3 us, whole rows 17.0; in two pieces 100 rows take 24.9,
// whole 18.4: joining them costs 5).
// A wave a row up to 16 packs a lane (8000 x 1000 bf16 with 5 alternatives:
// 13.4 us, by workgroups 25.9; 8000 x 4000: 21 and 30), but with fewer rows than
// two a CU up to two (100 x 4000 bf16: by waves 5.9, by workgroups 5.0; 128 x 1000
// fp32 with 5, four packs: 6.9 and 6.4); a workgroup of 1024 threads from 12 packs
// a thread on (200 x 131072 bf16 with 20: 19.1 us, with 256 threads 34.6; 2000 x
// 40000 fp32, 10 packs: 57.3 and 55.1).
struct Cut {
    int piece, splits, team;
};

Cut cut(int xtype, long long rows, long long vocab)
{
    const int n = pack_of(xtype);
    const long long want = std::max(1LL, (long long)num_cus() / std::max(1LL, rows));
    const long long most = std::min((long long)kPieces, std::max(1LL, vocab / 4096));
    long long splits = std::min(want, most), piece = vocab;
    if (splits < 4) {
        splits = 1;
    } else {
        piece = ((vocab + splits - 1) / splits + n * 256 - 1) / (n * 256) * (n * 256);
        splits = (vocab + piece - 1) / piece;
    }
    int team = 256;
    if (splits == 1 && vocab <= 64LL * n * (rows >= 2LL * num_cus() ? 16 : 2))
        team = 64;
    else if (splits == 1 && vocab >= 1024LL * n * 12)
        team = 1024;
    return Cut{(int)piece, (int)splits, team};
}

size_t parts_bytes(long long rows, int splits)
{
    return ((size_t)rows * splits * sizeof(Soft) + 15) / 16 * 16;
}

template <class T>
hipError_t forward(int xtype, const LogprobArgs &a, hipStream_t stream)
{
    const Cut s = cut(xtype, a.rows, a.vocab);
    Soft *parts = (Soft *)a.ws;
    uint64_t *keys = (uint64_t *)((char *)a.ws + parts_bytes(a.rows, s.splits));
    const long long teams = s.team < 256 ? 256 / s.team : 1;
    // Loads that leave nothing in the caches, for logits larger than the
    // last-level one holds beside the rest (4096 x 32000 bf16: 49.8 us instead of
    // 54.5; 500 x 8191 bf16: 7.4 with them, 5.9 without).
    const bool through = a.rows * a.vocab * (long long)sizeof(T) > 100LL << 20;
    const long long most = s.splits > 1 ? a.rows : kMaxBlocks * teams;  // rows of a launch
    for (long long first = 0; first < a.rows; first += most) {
        LogprobArgs c = a;
        c.rows = std::min(most, a.rows - first);
        c.logits.p = (const T *)a.logits.p + first * a.logits.ld;
        c.targets = a.targets ? a.targets + first : nullptr;
        c.logp = a.logp ? a.logp + first : nullptr;
        c.lse = a.lse ? a.lse + first : nullptr;
        c.entropy = a.entropy ? a.entropy + first : nullptr;
        c.stats = a.stats ? a.stats + 2 * first : nullptr;
        c.top_logp = a.top ? a.top_logp + first * a.top : nullptr;
        c.top_index = a.top ? a.top_index + first * a.top : nullptr;
        const unsigned grid = (unsigned)((c.rows * s.splits + teams - 1) / teams);
        if (s.team == 64)
            logprob_rows<T, 64><<<grid, 256, 0, stream>>>(c, s.piece, s.splits, through, parts,
                                                               keys);
        else if (s.team == 256)
            logprob_rows<T, 256><<<grid, 256, 0, stream>>>(c, s.piece, s.splits, through, parts,
                                                           keys);
        else
            logprob_rows<T, 1024><<<grid, 1024, 0, stream>>>(c, s.piece, s.splits, through, parts,
                                                             keys);
        if (s.splits > 1)
            logprob_join<T><<<(unsigned)c.rows, 256, 0, stream>>>(c, s.piece, s.splits, parts,
                                                                  keys);
    }
    return hipGetLastError();
}

template <class T>
hipError_t backward(const LogprobBwdArgs &a, hipStream_t stream)
{
    constexpr int N = Pack<T>::N, NV = 2;
    const long long packs = (a.vocab + N - 1) / N;
    int tpr = 1;
    while (tpr < 256 && (long long)tpr * NV < packs)
        tpr *= 2;
    // A vocabulary below 2^29 makes at most 2^18 pieces (fp32, 2048 elements each);
    // rows of a launch by the grid's limits.
    const long long pieces = tpr == 256 ? (packs + 256 * NV - 1) / (256 * NV) : 1;
    const long long most =
        tpr == 256 ? std::min(65535LL, std::max(1LL, 4 * kMaxBlocks / pieces)) : kMaxBlocks;
    for (long long first = 0; first < a.rows; first += most) {
        LogprobBwdArgs c = a;
        c.rows = std::min(most, a.rows - first);
        c.logits.p = (const T *)a.logits.p + first * a.logits.ld;
        c.dlogits.p = (const T *)a.dlogits.p + first * a.dlogits.ld;
        c.targets = a.targets ? a.targets + first : nullptr;
        c.stats = a.stats + 2 * first;
        c.dlogp = a.dlogp ? a.dlogp + first : nullptr;
        c.entropy = a.entropy ? a.entropy + first : nullptr;
        c.dentropy = a.dentropy ? a.dentropy + first : nullptr;
        const dim3 grid = tpr == 256 ? dim3((unsigned)pieces, (unsigned)c.rows)
                                     : dim3((unsigned)((c.rows * tpr + 255) / 256));
        logprob_back<T, NV><<<grid, 256, 0, stream>>>(c, tpr);
    }
    return hipGetLastError();
}

}  // namespace

size_t logprob_ws(int xtype, long long rows, long long vocab, int top)
{
    const Cut s = cut(xtype, rows, vocab);
    if (s.splits == 1)
        return 0;
    return parts_bytes(rows, s.splits) + (size_t)rows * s.splits * top * sizeof(uint64_t);
}

hipError_t launch_logprob_fwd(int xtype, const LogprobArgs &a, hipStream_t stream)
{
    if (!a.rows)
        return hipSuccess;
    return xtype == 0   ? forward<float>(xtype, a, stream)
           : xtype == 1 ? forward<__bf16>(xtype, a, stream)
                        : forward<_Float16>(xtype, a, stream);
}

hipError_t launch_logprob_bwd(int xtype, const LogprobBwdArgs &a, hipStream_t stream)
{
    if (!a.rows)
        return hipSuccess;
    return xtype == 0   ? backward<float>(a, stream)
           : xtype == 1 ? backward<__bf16>(a, stream)
                        : backward<_Float16>(a, stream);
}

}  // namespace miconv
