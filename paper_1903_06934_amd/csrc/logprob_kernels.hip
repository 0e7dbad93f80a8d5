// Log probabilities of given tokens, entropy and the likeliest tokens of rows
// of logits, and their gradient (include/mitrain.h).  Memory-bound: the logits
// are read once forward; backward they are read once and written once.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

constexpr int kGroups = 128;      // thread groups whose maxima bound the top (>= MITRAIN_TOP_MAX)
constexpr int kCandidates = 1024; // tokens at or above that bound held in LDS
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

__device__ __forceinline__ Soft merge(Soft a, Soft b, float c)
{
    const float m = fmaxf(a.m, b.m);
    if (m == -kInf)
        return Soft{m, a.s + b.s, a.t + b.t};  // zeros, or NaN
    const float ua = shifted(a.m, m), ub = shifted(b.m, m);
    const float ea = exp2_(ua * c), eb = exp2_(ub * c);
    return Soft{m, a.s * ea + b.s * eb, (a.t + ua * a.s) * ea + (b.t + ub * b.s) * eb};
}

// A finite maximum of nothing but -inf and NaN so far is taken as 0.
template <class T>
__device__ __forceinline__ void add_pack(Soft &p, typename Pack<T>::V raw, float c)
{
    constexpr int N = Pack<T>::N;
    float m = p.m;
#pragma unroll
    for (int j = 0; j < N; j++)
        m = fmaxf(m, (float)raw[j]);
    const float base = m == -kInf ? 0.f : m;
    if (m > p.m) {
        const float u = shifted(p.m, m), e = exp2_(u * c);
        p.t = (p.t + u * p.s) * e;
        p.s *= e;
        p.m = m;
    }
#pragma unroll
    for (int j = 0; j < N; j++) {
        const float u = (float)raw[j] - base, e = exp2_(u * c);
        p.s += e;
        p.t += fmaxf(u, -1e30f) * e;
    }
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

struct TopShared {
    float group[kGroups];
    float bound;
    int count;
    int wave[17];
    uint64_t keys[kCandidates];
};

// The bound: the k-th largest of kGroups group maxima (at least k elements
// reach it).
__device__ __forceinline__ float top_bound(TopShared &sh, int k)
{
    __syncthreads();
    if (threadIdx.x < kGroups) {
        const float mine = sh.group[threadIdx.x];
        int above = 0;
        for (int i = 0; i < kGroups; i++) {
            const float o = sh.group[i];
            above += o > mine || (o == mine && i < (int)threadIdx.x);
        }
        if (above == k - 1)
            sh.bound = mine;
    }
    if (threadIdx.x == 0)
        sh.count = 0;
    __syncthreads();
    return sh.bound;
}

// Ranks the n <= kCandidates keys and hands key and rank of the first k to put.
template <class Put>
__device__ __forceinline__ void put_ranked(const TopShared &sh, int n, int k, Put put)
{
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const uint64_t mine = sh.keys[i];
        int above = 0;
        for (int j = 0; j < n; j++)
            above += sh.keys[j] > mine;
        if (above < k)
            put(above, mine);
    }
}

// Sum over the workgroup.
__device__ __forceinline__ int block_count(TopShared &sh, int v)
{
    for (int o = 1; o < 64; o <<= 1)
        v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        sh.wave[threadIdx.x >> 6] = v;
    __syncthreads();
    int n = 0;
    for (int i = 0; i < (int)blockDim.x / 64; i++)
        n += sh.wave[i];
    return n;
}

// Elements of z[0, n) above v.
template <class T>
__device__ int count_above(TopShared &sh, const T *z, int n, float v)
{
    constexpr int N = Pack<T>::N;
    int c = 0;
    for (int i = threadIdx.x * N; i < n; i += blockDim.x * N) {
        const auto raw = load_pack<T>(z + i, n - i, (T)-kInf);
#pragma unroll
        for (int j = 0; j < N; j++)
            c += (float)raw[j] > v;
    }
    return block_count(sh, c);
}

// The keys of the top k of z[0, n) where too many elements reach the bound
// (equal logits, or large ones in few threads): the k-th largest value by
// bisection, then the elements above it, and of those equal to it the first.
// Returns their number, k.
template <class T>
__device__ int top_by_value(TopShared &sh, const T *z, int n, uint32_t first, int k, float bound,
                            float most)
{
    constexpr int N = Pack<T>::N;
    uint32_t lo = order(ranked(bound)), hi = order(ranked(most));
    if (count_above(sh, z, n, bound) < k) {
        hi = lo;
    } else {
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (count_above(sh, z, n, unorder(mid)) < k)
                hi = mid;
            else
                lo = mid;
        }
    }
    const float v = unorder(hi);  // fewer than k elements lie above it, k reach it
    __syncthreads();
    if (threadIdx.x == 0)
        sh.count = 0;
    __syncthreads();
    for (int i = threadIdx.x * N; i < n; i += blockDim.x * N) {
        const auto raw = load_pack<T>(z + i, n - i, (T)-kInf);
#pragma unroll
        for (int j = 0; j < N; j++)
            if ((float)raw[j] > v)
                sh.keys[atomicAdd(&sh.count, 1)] = key((float)raw[j], first + i + j);
    }
    __syncthreads();
    int have = sh.count;
    for (int base = 0; base < n && have < k; base += blockDim.x) {
        const int i = base + threadIdx.x;
        const bool equal = i < n && ranked((float)z[i]) == v;
        const uint64_t ballot = __ballot(equal);
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();
        if (lane == 0)
            sh.wave[wave] = __popcll(ballot);
        __syncthreads();
        int at = have + __popcll(ballot & ((1ull << lane) - 1));
        for (int w = 0; w < (int)blockDim.x / 64; w++) {
            at += w < wave ? sh.wave[w] : 0;
            have += sh.wave[w];
        }
        if (equal && at < k)
            sh.keys[at] = key(v, first + i);
    }
    __syncthreads();
    return k;
}

// The sums' results.
struct Done {
    float lse, entropy, log_s;
};

__device__ __forceinline__ Done finish(Soft p, float scale)
{
    if (p.m == -kInf && p.s == 0.f)
        return Done{-kInf, 0.f, 0.f};
    const float log_s = logf(p.s);
    return Done{p.m * scale + log_s, log_s - scale * (p.t / p.s), log_s};
}

__device__ __forceinline__ float log_prob(float z, Soft p, Done d, float scale)
{
    if (d.lse == -kInf)
        return -kInf;
    return (z - p.m) * scale - d.log_s;
}

template <class T>
__device__ __forceinline__ void write_row(const LogprobArgs &a, long long row, Soft p, Done d)
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
        const long long t = a.targets[row];
        float lp = 0.f;
        if (t >= a.vocab)
            lp = __builtin_nanf("");
        else if (t >= 0)
            lp = log_prob((float)((const T *)a.logits.p)[row * a.logits.ld + t], p, d, a.scale);
        a.logp[row] = lp;
    }
}

__device__ __forceinline__ void put_top(const LogprobArgs &a, long long row, int rank, uint64_t k,
                                        Soft p, Done d)
{
    a.top_index[row * a.top + rank] = 0xffffffffu - (uint32_t)k;
    a.top_logp[row * a.top + rank] = log_prob(unorder((uint32_t)(k >> 32)), p, d, a.scale);
}

// One workgroup a row, or a piece of it: then the piece's sums and its top go
// to ws, as parts[row][split] and keys[row][split][top].
template <class T>
__global__ __launch_bounds__(1024) void logprob_rows(LogprobArgs a, int piece, int splits,
                                                     Soft *parts, uint64_t *keys)
{
    constexpr int N = Pack<T>::N;
    __shared__ Soft waves[16];
    __shared__ TopShared sh;
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const int first = split * piece, n = (int)min((long long)piece, a.vocab - first);
    const T *z = (const T *)a.logits.p + row * a.logits.ld + first;
    const float c = a.scale * kLog2e;
    Soft p{-kInf, 0.f, 0.f};
    for (int i = threadIdx.x * N; i < n; i += blockDim.x * N)
        add_pack<T>(p, load_pack<T>(z + i, n - i, (T)-kInf), c);
    const float mine = p.m;
    for (int o = 1; o < 64; o <<= 1) {
        const Soft u{__shfl_xor(p.m, o), __shfl_xor(p.s, o), __shfl_xor(p.t, o)};
        p = (threadIdx.x & o) ? merge(u, p, c) : merge(p, u, c);
    }
    if ((threadIdx.x & 63) == 0)
        waves[threadIdx.x >> 6] = p;
    __syncthreads();
    p = waves[0];
    for (int i = 1; i < (int)blockDim.x / 64; i++)
        p = merge(p, waves[i], c);
    const Done d = finish(p, a.scale);
    if (threadIdx.x == 0) {
        if (splits == 1)
            write_row<T>(a, row, p, d);
        else
            parts[row * splits + split] = p;
    }
    if (!a.top)
        return;
    // A group's maximum: of blockDim / kGroups neighbouring threads.
    const int per = blockDim.x / kGroups;
    const float gm = wave_reduce(mine, per, Max());
    if (threadIdx.x % per == 0)
        sh.group[threadIdx.x / per] = gm;
    const int k = min(a.top, n);
    const float bound = top_bound(sh, k);
    if (mine >= bound) {
        for (int i = threadIdx.x * N; i < n; i += blockDim.x * N) {
            if (*(volatile int *)&sh.count > kCandidates)
                break;
            const auto raw = load_pack<T>(z + i, n - i, (T)0.f);
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float f = ranked((float)raw[j]);
                if (i + j < n && f >= bound) {
                    const int at = atomicAdd(&sh.count, 1);
                    if (at < kCandidates)
                        sh.keys[at] = key(f, first + i + j);
                }
            }
        }
    }
    __syncthreads();
    int found = sh.count;
    if (found > kCandidates)
        found = top_by_value<T>(sh, z, n, first, k, bound, p.m);
    if (splits == 1)
        put_ranked(sh, found, k, [&](int rank, uint64_t ky) { put_top(a, row, rank, ky, p, d); });
    else
        put_ranked(sh, found, k, [&](int rank, uint64_t ky) {
            keys[(row * splits + split) * a.top + rank] = ky;
        });
}

// Joins the pieces of a row.
template <class T>
__global__ __launch_bounds__(256) void logprob_join(LogprobArgs a, int piece, int splits,
                                                    const Soft *parts, const uint64_t *keys)
{
    const long long row = blockIdx.x;
    const float c = a.scale * kLog2e;
    Soft p = parts[row * splits];
    for (int i = 1; i < splits; i++)
        p = merge(p, parts[row * splits + i], c);
    const Done d = finish(p, a.scale);
    if (threadIdx.x == 0)
        write_row<T>(a, row, p, d);
    if (!a.top)
        return;
    // A key's rank: the keys above it in its piece's list, which is sorted,
    // and in each other one.
    for (int i = threadIdx.x; i < splits * a.top; i += 256) {
        const int split = i / a.top, at = i - split * a.top;
        if (at >= min((long long)piece, a.vocab - (long long)split * piece))
            continue;
        const uint64_t mine = keys[(row * splits + split) * a.top + at];
        int above = at;
        for (int s = 0; s < splits && above < a.top; s++) {
            if (s == split)
                continue;
            const int len = (int)min((long long)a.top,
                                     min((long long)piece, a.vocab - (long long)s * piece));
            const uint64_t *list = keys + (row * splits + s) * a.top;
            int lo = 0, hi = len;  // list[lo - 1] > mine > list[hi]
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (list[mid] > mine)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            above += lo;
        }
        if (above < a.top)
            put_top(a, row, above, mine, p, d);
    }
}

// -------------------------------------------------------------------- backward
// Groups of tpr threads (a power of two up to 256) take `per` packs each of a
// row's piece.
template <class T, int NV>
__global__ __launch_bounds__(256) void logprob_back(LogprobBwdArgs a, int tpr, int pieces)
{
    constexpr int N = Pack<T>::N;
    const int t = threadIdx.x & (tpr - 1);
    const long long item = (long long)blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
    const long long row = item / pieces;
    if (row >= a.rows)
        return;
    const long long first = (item - row * pieces) * tpr * N * NV;
    const float peak = a.stats[2 * row], log_s = a.stats[2 * row + 1], scale = a.scale;
    const long long target = a.dlogp ? a.targets[row] : -1;
    float dl = target >= 0 ? a.dlogp[row] * scale : 0.f;
    if (target >= a.vocab)
        dl = __builtin_nanf("");
    const float de = a.dentropy ? a.dentropy[row] * scale : 0.f;
    const float ent = a.dentropy ? a.entropy[row] : 0.f;
    const bool none = peak == -kInf && log_s == 0.f;
    const T *z = (const T *)a.logits.p + row * a.logits.ld;
    T *dz = (T *)a.dlogits.p + row * a.dlogits.ld;
    typename Pack<T>::V raw[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const long long c = first + (t + i * tpr) * N;
        raw[i] = typename Pack<T>::V{};
        if (c < a.vocab)
            raw[i] = load_pack<T>(z + c, a.vocab - c, (T)0.f);
    }
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const long long c = first + (t + i * tpr) * N;
        if (c >= a.vocab)
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
                f = target >= a.vocab ? dl : 0.f;
            v[j] = (T)f;
        }
        store_pack<T>(dz + c, a.vocab - c, v);
    }
}

// ----------------------------------------------------------------- launch rules
int pack_of(int xtype) { return xtype == 0 ? 4 : 8; }

int block_of(int n_pack, long long n)
{
    return n >= 1024LL * n_pack * 4 ? 1024 : n >= 512LL * n_pack * 2 ? 512 : 256;
}

// Pieces of a row: one workgroup a row where the rows fill the CUs; else pieces
// of at least 4096 elements, up to 64.
struct Cut {
    int piece, splits;
};

Cut cut(int xtype, long long rows, long long vocab)
{
    const long long want = std::max(1LL, (long long)num_cus() / std::max(1LL, rows));
    const long long most = std::min(64LL, std::max(1LL, vocab / 4096));
    const long long splits = std::min(want, most);
    const int n = pack_of(xtype) * 256;
    const long long piece =
        splits == 1 ? vocab : ((vocab + splits - 1) / splits + n - 1) / n * n;
    return Cut{(int)piece, (int)((vocab + piece - 1) / piece)};
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
    const int block = block_of(pack_of(xtype), s.piece);
    if (s.splits > 1) {
        logprob_rows<T><<<(unsigned)(a.rows * s.splits), block, 0, stream>>>(a, s.piece, s.splits,
                                                                             parts, keys);
        logprob_join<T><<<(unsigned)a.rows, 256, 0, stream>>>(a, s.piece, s.splits, parts, keys);
        return hipGetLastError();
    }
    for (long long first = 0; first < a.rows; first += kMaxBlocks) {
        LogprobArgs c = a;  // the rows of this launch
        c.rows = std::min(kMaxBlocks, a.rows - first);
        c.logits.p = (const T *)a.logits.p + first * a.logits.ld;
        c.targets = a.targets ? a.targets + first : nullptr;
        c.logp = a.logp ? a.logp + first : nullptr;
        c.lse = a.lse ? a.lse + first : nullptr;
        c.entropy = a.entropy ? a.entropy + first : nullptr;
        c.stats = a.stats ? a.stats + 2 * first : nullptr;
        c.top_logp = a.top ? a.top_logp + first * a.top : nullptr;
        c.top_index = a.top ? a.top_index + first * a.top : nullptr;
        logprob_rows<T><<<(unsigned)c.rows, block, 0, stream>>>(c, s.piece, 1, nullptr, nullptr);
    }
    return hipGetLastError();
}

template <class T>
hipError_t backward(const LogprobBwdArgs &a, hipStream_t stream)
{
    constexpr int N = Pack<T>::N, NV = 4;
    const long long packs = (a.vocab + N - 1) / N;
    int tpr = 1;
    while (tpr < 256 && (long long)tpr * NV < packs)
        tpr *= 2;
    const long long pieces = (packs + tpr * NV - 1) / (tpr * NV);
    const long long groups = 256 / tpr;
    // Rows of one launch: its workgroups stay below kMaxBlocks.
    const long long most = std::max(1LL, kMaxBlocks * groups / pieces);
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
        const long long blocks = (c.rows * pieces + groups - 1) / groups;
        logprob_back<T, NV><<<(unsigned)blocks, 256, 0, stream>>>(c, tpr, (int)pieces);
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
