// The losses of fine-tuning and their gradients (include/mistep.h): the clipped
// policy loss of sampled tokens, and the loss of pairs of sequences.
//
// Tokens are taken by chunks, whatever the sequences' lengths; of a chunk's
// sequences each has a team of threads.  A sequence that reaches over several
// chunks leaves its piece of each in the workspace: `tail` of the chunk it begins
// in, `head` of those that it continues in, and a later launch adds the pieces in
// the order of the chunks, so that no result depends on which workgroup ran first.
// Calls of few tokens run as one workgroup, in one launch.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "step.h"

namespace miconv {

namespace {

constexpr int kBlock = 256, kChunk = 2048;         // of the calls of many tokens
constexpr int kOneBlock = 1024, kOneChunk = 8192;  // of those of few
constexpr int kMaxGroups = 2048;                   // workgroups of a launch, and partial sums
constexpr int kJoinGroups = 1024;                  // of a launch over the sequences

typedef Pack<float>::V F4;

__device__ __forceinline__ double wave_sum(double v)
{
    for (int o = 1; o < 64; o <<= 1)
        v += __shfl_xor(v, o);
    return v;
}

__device__ __forceinline__ int wave_sum(int v)
{
    for (int o = 1; o < 64; o <<= 1)
        v += __shfl_xor(v, o);
    return v;
}

// Sums over a workgroup; lds holds one value a wave.
template <int BLOCK, class V>
__device__ __forceinline__ V block_sum(V v, V *lds)
{
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0)
        lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int i = 1; i < BLOCK / 64; i++)
        v += lds[i];
    __syncthreads();
    return v;
}

// How many of n numbers that do not fall are at most v; by a whole wave.
__device__ __forceinline__ int count_up_to(const long long *p, int n, long long v)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = n;  // those before lo are, those from hi on are not
    while (lo < hi) {
        const int step = (int)(((long long)hi - lo + 63) / 64);
        const long long at = lo + (long long)lane * step;
        const int k = __popcll(__ballot(at < hi && p[at] <= v));
        if (!k)
            break;
        hi = (int)min((long long)hi, lo + (long long)k * step);
        lo = (int)(lo + (long long)(k - 1) * step + 1);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

struct Starts {
    const long long *p;
    int tokens;
    __device__ __forceinline__ int operator()(long long i) const
    {
        return (int)min(max(p[i], 0LL), (long long)tokens);
    }
};

// The sequences first <= s < last that have tokens in the chunk [begin, end), and
// the threads of each one's team: about as many as it has tokens there.
struct Here {
    int first, last, width;
};

__device__ __forceinline__ Here sequences_here(const long long *starts, int seqs, int begin, int end)
{
    Here h;
    h.first = count_up_to(starts + 1, seqs, begin);
    h.last = count_up_to(starts, seqs, (long long)end - 1);
    h.width = 64;
    while (h.width > 1 && (long long)h.width / 2 * (h.last - h.first) >= end - begin)
        h.width /= 2;
    return h;
}

// Bytes of the mask for four tokens, of which left (>= 1) are there, one bit each.
__device__ __forceinline__ unsigned load_mask(const unsigned char *mask, int at, int left)
{
    if (!mask)
        return left >= 4 ? 15u : (1u << left) - 1;
    unsigned bits = 0;
    if (left >= 4) {
        typedef uint32_t At __attribute__((aligned(1)));
        const uint32_t v = *(const At *)(mask + at);
#pragma unroll
        for (int j = 0; j < 4; j++)
            bits |= (unsigned)((v >> 8 * j & 255) != 0) << j;
    } else {
        for (int j = 0; j < left; j++)
            bits |= (unsigned)(mask[at + j] != 0) << j;
    }
    return bits;
}

__device__ __forceinline__ F4 load_four(const float *p, int at, int left)
{
    return load_pack<float>(p + at, left, 0.f);
}

// A workgroup's chunks of all of them.
__device__ __forceinline__ int first_chunk(int chunks, unsigned group)
{
    return (int)((long long)chunks * group / gridDim.x);
}

// ------------------------------------------------------------- counts of tokens
// What the counts of a policy loss are written to and read from.
struct Counts {
    int *seq;   // [seqs] tokens that count, of sequences within a chunk; later of all
    int *head, *tail;  // [chunks]
    int *group;        // [kMaxGroups] of each workgroup's chunks
    int *some;         // [kJoinGroups] sequences that have any
    double *part;      // [kMaxGroups][6]
};

__global__ __launch_bounds__(kBlock) void policy_count(PolicyArgs a, Counts c, int chunks)
{
    __shared__ unsigned char bits[kChunk];
    __shared__ int red[kBlock / 64];
    const bool by_seq = a.mean == 1;
    const Starts starts{a.starts, a.tokens};
    int all = 0;
    for (int k = first_chunk(chunks, blockIdx.x); k < first_chunk(chunks, blockIdx.x + 1); k++) {
        const int begin = k * kChunk, end = begin + min(kChunk, a.tokens - begin);
        const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
        for (int t = threadIdx.x * 4; t < end - begin; t += kBlock * 4) {
            const unsigned m = load_mask(a.mask, begin + t, end - begin - t);
#pragma unroll
            for (int j = 0; j < 4; j++) {
                const int at = begin + t + j;
                const bool in = m >> j & 1;
                all += in && at >= from && at < to;
                if (by_seq)
                    bits[t + j] = in;
            }
        }
        if (!by_seq)
            continue;
        __syncthreads();
        const Here h = sequences_here(a.starts, a.seqs, begin, end);
        const int lane = threadIdx.x & (h.width - 1);
        for (long long s = h.first + threadIdx.x / h.width; s < h.last; s += kBlock / h.width) {
            const int s0 = starts(s), s1 = starts(s + 1);
            int n = 0;
            for (int t = max(s0, begin) + lane; t < min(s1, end); t += h.width)
                n += bits[t - begin];
            for (int o = 1; o < h.width; o <<= 1)
                n += __shfl_xor(n, o);
            if (lane == 0)
                *(s0 < begin ? c.head + k : s1 > end ? c.tail + k : c.seq + s) = n;
        }
        __syncthreads();
    }
    all = block_sum<kBlock>(all, red);
    if (threadIdx.x == 0)
        c.group[blockIdx.x] = all;
}

// The sum of a sequence's pieces (of the tokens begin <= t < end) that chunks left;
// by a whole wave.
template <class V>
__device__ __forceinline__ V join_pieces(const V *seq, const V *head, const V *tail, long long s,
                                         int begin, int end)
{
    if (begin >= end)
        return V(0);
    const int from = begin / kChunk, to = (end - 1) / kChunk;
    if (from == to)
        return seq[s];
    V v = V(0);
    for (int k = from + (threadIdx.x & 63); k <= to; k += 64)
        v += k == from ? tail[k] : head[k];
    return wave_sum(v);
}

// A wave a sequence: its tokens that count, and how many sequences have any.
__global__ __launch_bounds__(kBlock) void policy_join(PolicyArgs a, Counts c)
{
    __shared__ int red[kBlock / 64];
    const Starts starts{a.starts, a.tokens};
    int some = 0;
    if (a.mask) {
        for (long long s = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6); s < a.seqs;
             s += gridDim.x * (kBlock / 64)) {
            const int n = join_pieces(c.seq, c.head, c.tail, s, starts(s), starts(s + 1));
            if ((threadIdx.x & 63) == 0) {
                c.seq[s] = n;
                some += n > 0;
            }
        }
    } else {
        for (long long s = (long long)blockIdx.x * kBlock + threadIdx.x; s < a.seqs;
             s += (long long)gridDim.x * kBlock)
            some += starts(s + 1) > starts(s);
    }
    some = block_sum<kBlock>(some, red);
    if (threadIdx.x == 0)
        c.some[blockIdx.x] = some;
}

// ------------------------------------------------------------------ policy loss
// exp(x) - 1 - x, and exp(x) - 1; near 0 by the exponential's series, where the
// difference would lose what matters.
__device__ __forceinline__ float low_kl(float x, float *expm1)
{
    float v;
    if (fabsf(x) < 1.f) {
        float p = 1.f / 479001600.f;  // 1 / 12!
        p = fmaf(p, x, 1.f / 39916800.f);
        p = fmaf(p, x, 1.f / 3628800.f);
        p = fmaf(p, x, 1.f / 362880.f);
        p = fmaf(p, x, 1.f / 40320.f);
        p = fmaf(p, x, 1.f / 5040.f);
        p = fmaf(p, x, 1.f / 720.f);
        p = fmaf(p, x, 1.f / 120.f);
        p = fmaf(p, x, 1.f / 24.f);
        p = fmaf(p, x, 1.f / 6.f);
        p = fmaf(p, x, 0.5f);
        v = x * x * p;
        *expm1 = x + v;
    } else {
        *expm1 = expf(x) - 1.f;
        v = *expm1 - x;
    }
    return v;
}

struct Token {
    float loss, surrogate, kl, ratio, slope;
    bool clipped;
};

__device__ __forceinline__ Token token_loss(const PolicyArgs &a, float lp, float lo, float lr,
                                            float h, float adv)
{
    Token k;
    const double d = (double)lp - (double)lo;  // in 64 bits: whether the token is clipped
    k.ratio = expf((float)d);
    float bound = k.ratio;
    k.clipped = false;
    if (adv > 0.f && d > a.log_high) {
        k.clipped = true;
        bound = a.high;
    } else if (adv < 0.f && d < a.log_low) {
        k.clipped = true;
        bound = a.low;
    } else if (adv < 0.f && d > a.log_dual) {
        k.clipped = true;
        bound = a.dual;
    }
    k.surrogate = -adv * bound;
    k.slope = k.clipped ? 0.f : k.surrogate;
    k.loss = k.surrogate;
    k.kl = 0.f;
    if (a.ref_logp) {
        const float x = lr - lp;
        float slope;
        if (a.kl == 0) {
            k.kl = -x;
            slope = 1.f;
        } else if (a.kl == 1) {
            k.kl = 0.5f * x * x;
            slope = -x;
        } else {
            k.kl = low_kl(x, &slope);
            slope = -slope;
        }
        if (a.kl_weight != 0.f) {
            k.loss += a.kl_weight * k.kl;
            k.slope += a.kl_weight * slope;
        }
    }
    if (a.entropy && a.entropy_weight != 0.f)
        k.loss -= a.entropy_weight * h;
    return k;
}

// The chunk's tokens a thread holds: two packs of four.
constexpr int kPacks = 2;

struct Tokens {
    F4 lp[kPacks], lo[kPacks], lr[kPacks], h[kPacks], adv[kPacks];
    unsigned mask[kPacks];  // of four: there, and not masked
};

template <int BLOCK>
__device__ __forceinline__ void load_tokens(const PolicyArgs &a, int begin, int end, Tokens &k)
{
#pragma unroll
    for (int i = 0; i < kPacks; i++) {
        const int at = begin + ((int)threadIdx.x + i * BLOCK) * 4, left = end - at;
        k.mask[i] = 0;
        k.lp[i] = k.lo[i] = k.lr[i] = k.h[i] = k.adv[i] = F4{};
        if (left <= 0)
            continue;
        k.mask[i] = load_mask(a.mask, at, left);
        k.lp[i] = load_four(a.logp, at, left);
        k.lo[i] = load_four(a.old_logp, at, left);
        if (a.ref_logp)
            k.lr[i] = load_four(a.ref_logp, at, left);
        if (a.entropy)
            k.h[i] = load_four(a.entropy, at, left);
        if (!a.by_sequence)
            k.adv[i] = load_four(a.advantages, at, left);
    }
}

// The tokens' losses (times their weights within their sequences) to sum, their
// gradients to memory.  weight, adv: of each token of the chunk in LDS, or null:
// the tokens from <= t < to have weight 1.  u: what all weights are multiplied by.
template <int BLOCK>
__device__ __forceinline__ void chunk_losses(const PolicyArgs &a, const Tokens &k, int begin,
                                             int end, const float *weight, const float *adv,
                                             int from, int to, double u, double (&sum)[6])
{
    const float factor = (float)(u * a.scale);
#pragma unroll
    for (int i = 0; i < kPacks; i++) {
        const int at = begin + ((int)threadIdx.x + i * BLOCK) * 4, left = end - at;
        if (left <= 0)
            continue;
        F4 g = F4{}, gh = F4{};
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int t = at + j;
            if (!(k.mask[i] >> j & 1))
                continue;
            const float w = weight ? weight[t - begin] : t >= from && t < to ? 1.f : 0.f;
            if (w == 0.f)
                continue;
            const Token r = token_loss(a, k.lp[i][j], k.lo[i][j], k.lr[i][j], k.h[i][j],
                                       a.by_sequence ? adv[t - begin] : k.adv[i][j]);
            sum[0] += (double)w * r.loss;
            sum[1] += (double)w * r.surrogate;
            sum[2] += (double)w * r.kl;
            if (a.entropy)
                sum[3] += (double)w * k.h[i][j];
            sum[4] += (double)w * r.ratio;
            sum[5] += r.clipped ? w : 0.f;
            g[j] = r.slope * (w * factor);
            gh[j] = -a.entropy_weight * (w * factor);
        }
        if (a.dlogp)
            store_pack<float>(a.dlogp + at, left, g);
        if (a.dentropy)
            store_pack<float>(a.dentropy + at, left, gh);
    }
}

// Sequence s's weight (1 / its tokens that count, or 1) and advantage to its tokens
// of the chunk; `width` threads.
__device__ __forceinline__ void fill_tokens(const PolicyArgs &a, long long s, int n, int first,
                                            int last, int begin, int lane, int width,
                                            float *weight, float *adv)
{
    const float w = a.mean == 1 ? (n > 0 ? 1.f / (float)n : 0.f) : 1.f;
    const float v = a.by_sequence ? a.advantages[s] : 0.f;
    for (int t = first + lane; t < last; t += width) {
        weight[t - begin] = w;
        adv[t - begin] = v;
    }
}

// Few tokens: all of the call in one workgroup.  SEQS: the sequences matter.
template <bool SEQS>
__global__ __launch_bounds__(kOneBlock) void policy_one(PolicyArgs a)
{
    constexpr int WAVES = kOneBlock / 64;
    __shared__ float weight[SEQS ? kOneChunk : 1], adv[SEQS ? kOneChunk : 1];
    __shared__ double red[6][WAVES];
    __shared__ int counts[2][WAVES];
    const Starts starts{a.starts, a.tokens};
    Tokens k;
    load_tokens<kOneBlock>(a, 0, a.tokens, k);
    const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
    int all = 0;
#pragma unroll
    for (int i = 0; i < kPacks; i++)
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int t = ((int)threadIdx.x + i * kOneBlock) * 4 + j;
            const bool in = k.mask[i] >> j & 1;
            all += in && t >= from && t < to;
            if (SEQS && t < a.tokens) {
                weight[t] = 0.f;
                adv[t] = in ? 1.f : 0.f;  // until the advantages are written
            }
        }
    double u = 1.0 / a.count;
    if (a.mean == 0) {
        all = block_sum<kOneBlock>(all, counts[0]);
        u = 1.0 / max(all, 1);
    }
    if (SEQS) {
        int width = 64, some = 0;
        while (width > 1 && (long long)width / 2 * a.seqs >= a.tokens)
            width /= 2;
        const int lane = threadIdx.x & (width - 1);
        __syncthreads();
        for (int s = threadIdx.x / width; s < a.seqs; s += kOneBlock / width) {
            const int s0 = starts(s), s1 = starts(s + 1);
            int n = 0;
            if (a.mean == 1) {
                for (int t = s0 + lane; t < s1; t += width)
                    n += adv[t] != 0.f;
                for (int o = 1; o < width; o <<= 1)
                    n += __shfl_xor(n, o);
                some += lane == 0 && n > 0;
            }
            fill_tokens(a, s, n, s0, s1, 0, lane, width, weight, adv);
        }
        if (a.mean == 1) {
            some = block_sum<kOneBlock>(some, counts[1]);
            u = 1.0 / max(some, 1);
        }
        __syncthreads();
    }
    double sum[6] = {0, 0, 0, 0, 0, 0};
    chunk_losses<kOneBlock>(a, k, 0, a.tokens, SEQS ? weight : nullptr, adv, from, to, u, sum);
#pragma unroll
    for (int i = 0; i < 6; i++) {
        sum[i] = wave_sum(sum[i]);
        if ((threadIdx.x & 63) == 0)
            red[i][threadIdx.x >> 6] = sum[i];
    }
    __syncthreads();
    if (threadIdx.x < 6) {
        double v = 0;
        for (int i = 0; i < WAVES; i++)
            v += red[threadIdx.x][i];
        a.stats[threadIdx.x] = (float)(v * u);
    }
}

// The sum of n (at most a few thousand) counts, by a whole workgroup.
template <int BLOCK>
__device__ __forceinline__ long long sum_counts(const int *p, int n, double *lds)
{
    double v = 0;  // whole numbers below 2^53
    for (int i = threadIdx.x; i < n; i += BLOCK)
        v += p[i];
    return (long long)block_sum<BLOCK>(v, lds);
}

// What all weights are multiplied by.
__device__ __forceinline__ double weight_of_all(const PolicyArgs &a, const Counts &c, int groups,
                                                int joins, int from, int to, double *lds)
{
    if (a.mean == 2)
        return 1.0 / a.count;
    long long n;
    if (a.mean == 1)
        n = sum_counts<kBlock>(c.some, joins, lds);
    else
        n = a.mask ? sum_counts<kBlock>(c.group, groups, lds) : to - from;
    return 1.0 / (double)max(n, 1LL);
}

template <bool SEQS>
__global__ __launch_bounds__(kBlock) void policy_main(PolicyArgs a, Counts c, int chunks, int joins)
{
    __shared__ float weight[SEQS ? kChunk : 1], adv[SEQS ? kChunk : 1];
    __shared__ double red[kBlock / 64];
    const Starts starts{a.starts, a.tokens};
    const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
    const double u = weight_of_all(a, c, gridDim.x, joins, from, to, red);
    double sum[6] = {0, 0, 0, 0, 0, 0};
    for (int k = first_chunk(chunks, blockIdx.x); k < first_chunk(chunks, blockIdx.x + 1); k++) {
        const int begin = k * kChunk, end = begin + min(kChunk, a.tokens - begin);
        Tokens tokens;
        load_tokens<kBlock>(a, begin, end, tokens);
        if (SEQS) {
            const Here h = sequences_here(a.starts, a.seqs, begin, end);
            for (int t = threadIdx.x; t < end - begin; t += kBlock)
                weight[t] = 0.f;
            __syncthreads();
            const int lane = threadIdx.x & (h.width - 1);
            for (long long s = h.first + threadIdx.x / h.width; s < h.last;
                 s += kBlock / h.width) {
                const int s0 = starts(s), s1 = starts(s + 1);
                const int n = a.mean != 1 ? 0 : a.mask ? c.seq[s] : s1 - s0;
                fill_tokens(a, s, n, max(s0, begin), min(s1, end), begin, lane, h.width, weight,
                            adv);
            }
            __syncthreads();
        }
        chunk_losses<kBlock>(a, tokens, begin, end, SEQS ? weight : nullptr, adv, from, to, u, sum);
        if (SEQS)
            __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 6; i++) {
        const double v = block_sum<kBlock>(sum[i], red);
        if (threadIdx.x == 0)
            c.part[blockIdx.x * 6 + i] = v * u;
    }
}

// Wave i adds the workgroups' sums of the i-th result.
template <int N>
__device__ __forceinline__ void add_parts(const double *part, int groups, double u, float *stats)
{
    const int i = threadIdx.x >> 6;
    if (i >= N)
        return;
    double v = 0;
    for (int g = threadIdx.x & 63; g < groups; g += 64)
        v += part[g * N + i];
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0)
        stats[i] = (float)(v * u);
}

__global__ __launch_bounds__(6 * 64) void policy_stats(const double *part, int groups, float *stats)
{
    add_parts<6>(part, groups, 1.0, stats);
}

// -------------------------------------------------------------- preference loss
struct Pairs {
    double *seq, *head, *tail;    // sums of log ratios: [2 pairs], [chunks], [chunks]
    int *count, *chead, *ctail;   // tokens that count, likewise
    double *slope;                // [pairs] of the loss in x
    double *part;                 // [kJoinGroups][5]
    int *some;                    // [kJoinGroups] pairs that have a token
};

struct Pair {
    double stats[5], slope;
};

__device__ __forceinline__ double reward(const PreferenceArgs &a, double sum, int n)
{
    return a.beta * (a.length_mean ? sum / max(n, 1) : sum);
}

__device__ __forceinline__ Pair pair_loss(const PreferenceArgs &a, double r0, double r1)
{
    Pair p;
    const double gap = r0 - r1, x = gap - a.margin;
    double loss;
    if (a.form == 1) {
        loss = x < 1.0 ? 1.0 - x : x >= 1.0 ? 0.0 : x;  // NaN stays
        p.slope = x < 1.0 ? -1.0 : x >= 1.0 ? 0.0 : x;
    } else if (a.form == 2) {
        const double v = (x - 0.5) / a.beta;
        loss = v * v;
        p.slope = 2.0 * v / a.beta;
    } else {
        const double e = a.smoothing, z = exp(-fabs(x)), l = log1p(z);
        // -ln s(x) = l + max(-x, 0), -ln s(-x) = l + max(x, 0)
        loss = (e < 1.0 ? (1.0 - e) * (l + (x < 0 ? -x : 0.0)) : 0.0) +
               (e > 0.0 ? e * (l + (x > 0 ? x : 0.0)) : 0.0);
        const double up = (x < 0 ? 1.0 : z) / (1.0 + z), down = (x < 0 ? z : 1.0) / (1.0 + z);
        p.slope = e * down - (1.0 - e) * up;
    }
    p.stats[0] = loss;
    p.stats[1] = gap;
    p.stats[2] = gap > 0;
    p.stats[3] = r0;
    p.stats[4] = r1;
    return p;
}

// A token's gradient in a sequence of n tokens that count.
__device__ __forceinline__ float pair_gradient(const PreferenceArgs &a, double slope, bool second,
                                               int n, double u)
{
    const double v = slope * a.beta * a.scale * u / (a.length_mean ? max(n, 1) : 1);
    return (float)(second ? -v : v);
}

// Four tokens' log ratios, 0 where they do not count.
__device__ __forceinline__ F4 load_ratios(const PreferenceArgs &a, int at, int left, unsigned *mask)
{
    *mask = load_mask(a.mask, at, left);
    const F4 lp = load_four(a.logp, at, left);
    F4 lr = F4{};
    if (a.ref_logp)
        lr = load_four(a.ref_logp, at, left);
    F4 v;
#pragma unroll
    for (int j = 0; j < 4; j++)
        v[j] = *mask >> j & 1 ? lp[j] - lr[j] : 0.f;
    return v;
}

// The chunk's ratios and masks to LDS.
template <int BLOCK>
__device__ __forceinline__ void stage_ratios(const PreferenceArgs &a, int begin, int end, float *v,
                                             unsigned char *bits)
{
#pragma unroll
    for (int i = 0; i < kPacks; i++) {
        const int t = ((int)threadIdx.x + i * BLOCK) * 4, left = end - begin - t;
        if (left <= 0)
            continue;
        unsigned m;
        const F4 r = load_ratios(a, begin + t, left, &m);
#pragma unroll
        for (int j = 0; j < 4; j++) {
            v[t + j] = r[j];
            bits[t + j] = m >> j & 1;
        }
    }
}

// The sum of a sequence's ratios of the chunk, and of its tokens; `width` threads.
__device__ __forceinline__ double team_sum(const float *v, const unsigned char *bits, int first,
                                           int last, int lane, int width, int *n)
{
    double s = 0;
    int c = 0;
    for (int t = first + lane; t < last; t += width) {
        s += v[t];
        c += bits[t];
    }
    for (int o = 1; o < width; o <<= 1) {
        s += __shfl_xor(s, o);
        c += __shfl_xor(c, o);
    }
    *n = c;
    return s;
}

__global__ __launch_bounds__(kBlock) void preference_sums(PreferenceArgs a, Pairs p, int chunks)
{
    __shared__ float v[kChunk];
    __shared__ unsigned char bits[kChunk];
    const Starts starts{a.starts, a.tokens};
    for (int k = first_chunk(chunks, blockIdx.x); k < first_chunk(chunks, blockIdx.x + 1); k++) {
        const int begin = k * kChunk, end = begin + min(kChunk, a.tokens - begin);
        stage_ratios<kBlock>(a, begin, end, v, bits);
        const Here h = sequences_here(a.starts, 2 * a.pairs, begin, end);
        __syncthreads();
        const int lane = threadIdx.x & (h.width - 1);
        for (long long s = h.first + threadIdx.x / h.width; s < h.last; s += kBlock / h.width) {
            const int s0 = starts(s), s1 = starts(s + 1);
            int n;
            const double sum = team_sum(v, bits, max(s0, begin) - begin, min(s1, end) - begin,
                                        lane, h.width, &n);
            if (lane == 0) {
                *(s0 < begin ? p.head + k : s1 > end ? p.tail + k : p.seq + s) = sum;
                *(s0 < begin ? p.chead + k : s1 > end ? p.ctail + k : p.count + s) = n;
            }
        }
        __syncthreads();
    }
}

// A wave a pair.
__global__ __launch_bounds__(kBlock) void preference_pairs(PreferenceArgs a, Pairs p)
{
    __shared__ double red[kBlock / 64];
    const Starts starts{a.starts, a.tokens};
    const int lane = threadIdx.x & 63;
    double sum[5] = {0, 0, 0, 0, 0}, some = 0;
    for (long long i = blockIdx.x * (kBlock / 64) + (threadIdx.x >> 6); i < a.pairs;
         i += gridDim.x * (kBlock / 64)) {
        double r[2];
        int n[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const long long s = i + (long long)k * a.pairs;
            const int s0 = starts(s), s1 = starts(s + 1);
            n[k] = join_pieces(p.count, p.chead, p.ctail, s, s0, s1);
            r[k] = reward(a, join_pieces(p.seq, p.head, p.tail, s, s0, s1), n[k]);
            if (lane == 0) {
                p.count[s] = n[k];
                if (a.rewards)
                    a.rewards[s] = (float)r[k];
            }
        }
        if (lane == 0) {
            const Pair q = pair_loss(a, r[0], r[1]);
            p.slope[i] = q.slope;
            if (n[0] + n[1] > 0) {
                some += 1;
#pragma unroll
                for (int k = 0; k < 5; k++)
                    sum[k] += q.stats[k];
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 5; k++) {
        const double v = block_sum<kBlock>(sum[k], red);
        if (threadIdx.x == 0)
            p.part[blockIdx.x * 5 + k] = v;
    }
    some = block_sum<kBlock>(some, red);
    if (threadIdx.x == 0)
        p.some[blockIdx.x] = (int)some;
}

// The chunk's gradients from LDS to memory.
template <int BLOCK>
__device__ __forceinline__ void store_gradients(const PreferenceArgs &a, int begin, int end,
                                                const float *v)
{
#pragma unroll
    for (int i = 0; i < kPacks; i++) {
        const int t = ((int)threadIdx.x + i * BLOCK) * 4, left = end - begin - t;
        if (left <= 0)
            continue;
        const unsigned m = load_mask(a.mask, begin + t, left);
        F4 g;
#pragma unroll
        for (int j = 0; j < 4; j++)
            g[j] = m >> j & 1 ? v[t + j] : 0.f;
        store_pack<float>(a.dlogp + begin + t, left, g);
    }
}

// The gradients; the first workgroup adds the results too.
__global__ __launch_bounds__(5 * 64) void preference_fill(PreferenceArgs a, Pairs p, int chunks,
                                                          int joins)
{
    constexpr int BLOCK = 5 * 64;
    __shared__ float v[kChunk];
    __shared__ double red[BLOCK / 64];
    const Starts starts{a.starts, a.tokens};
    const double u = 1.0 / (double)max(sum_counts<BLOCK>(p.some, joins, red), 1LL);
    if (blockIdx.x == 0)
        add_parts<5>(p.part, joins, u, a.stats);
    if (!a.dlogp)
        return;
    for (int k = first_chunk(chunks, blockIdx.x); k < first_chunk(chunks, blockIdx.x + 1); k++) {
        const int begin = k * kChunk, end = begin + min(kChunk, a.tokens - begin);
        const Here h = sequences_here(a.starts, 2 * a.pairs, begin, end);
        for (int t = threadIdx.x; t < end - begin; t += BLOCK)
            v[t] = 0.f;
        __syncthreads();
        const int lane = threadIdx.x & (h.width - 1);
        for (long long s = h.first + threadIdx.x / h.width; s < h.last; s += BLOCK / h.width) {
            const int first = max(starts(s), begin) - begin, last = min(starts(s + 1), end) - begin;
            const bool second = s >= a.pairs;
            const float g = pair_gradient(a, p.slope[second ? s - a.pairs : s], second, p.count[s], u);
            for (int t = first + lane; t < last; t += h.width)
                v[t] = g;
        }
        __syncthreads();
        store_gradients<BLOCK>(a, begin, end, v);
        __syncthreads();
    }
}

constexpr int kOnePairs = 1024;

__global__ __launch_bounds__(kOneBlock) void preference_one(PreferenceArgs a)
{
    constexpr int WAVES = kOneBlock / 64;
    __shared__ float v[kOneChunk];
    __shared__ unsigned char bits[kOneChunk];
    __shared__ double sums[2 * kOnePairs];  // of ratios; then a pair's slope
    __shared__ int count[2 * kOnePairs];
    __shared__ double red[WAVES];
    const Starts starts{a.starts, a.tokens};
    const int seqs = 2 * a.pairs;
    stage_ratios<kOneBlock>(a, 0, a.tokens, v, bits);
    int width = 64;
    while (width > 1 && (long long)width / 2 * seqs >= a.tokens)
        width /= 2;
    const int lane = threadIdx.x & (width - 1);
    __syncthreads();
    for (int s = threadIdx.x / width; s < seqs; s += kOneBlock / width) {
        int n;
        const double sum = team_sum(v, bits, starts(s), starts(s + 1), lane, width, &n);
        if (lane == 0) {
            sums[s] = sum;
            count[s] = n;
        }
    }
    __syncthreads();
    double sum[5] = {0, 0, 0, 0, 0}, some = 0;
    const int i = threadIdx.x;
    if (i < a.pairs) {
        const int n0 = count[i], n1 = count[a.pairs + i];
        const double r0 = reward(a, sums[i], n0), r1 = reward(a, sums[a.pairs + i], n1);
        if (a.rewards) {
            a.rewards[i] = (float)r0;
            a.rewards[a.pairs + i] = (float)r1;
        }
        const Pair q = pair_loss(a, r0, r1);
        sums[i] = q.slope;
        if (n0 + n1 > 0) {
            some = 1;
#pragma unroll
            for (int k = 0; k < 5; k++)
                sum[k] = q.stats[k];
        }
    }
    const double u = 1.0 / max(block_sum<kOneBlock>(some, red), 1.0);
#pragma unroll
    for (int k = 0; k < 5; k++) {
        const double s = block_sum<kOneBlock>(sum[k], red);
        if (threadIdx.x == 0)
            a.stats[k] = (float)(s * u);
    }
    if (!a.dlogp)
        return;
    for (int t = threadIdx.x; t < a.tokens; t += kOneBlock)
        v[t] = 0.f;
    __syncthreads();
    for (int s = threadIdx.x / width; s < seqs; s += kOneBlock / width) {
        const bool second = s >= a.pairs;
        const float g = pair_gradient(a, sums[second ? s - a.pairs : s], second, count[s], u);
        const int last = starts(s + 1);
        for (int t = starts(s) + lane; t < last; t += width)
            v[t] = g;
    }
    __syncthreads();
    store_gradients<kOneBlock>(a, 0, a.tokens, v);
}

// ---------------------------------------------------------------- launch rules
static_assert(kPacks * 4 * kBlock == kChunk && kPacks * 4 * kOneBlock == kOneChunk, "chunks");
static_assert(kPacks * 4 * 5 * 64 >= kChunk, "chunks of preference_fill");

int chunks_of(long long tokens) { return (int)std::max(1LL, (tokens + kChunk - 1) / kChunk); }

int join_groups(long long waves)
{
    return (int)std::min((waves + kBlock / 64 - 1) / (kBlock / 64), (long long)kJoinGroups);
}

// One workgroup.
bool policy_is_small(long long tokens, long long seqs)
{
    return tokens <= kOneChunk && seqs <= kOneChunk;
}

bool preference_is_small(long long tokens, long long pairs)
{
    return tokens <= kOneChunk && pairs <= kOnePairs;
}

// Arrays one after the other in the workspace, of 16 bytes' alignment.
struct Arena {
    char *p;
    size_t used = 0;

    template <class V>
    V *take(long long n)
    {
        V *at = (V *)(p + used);
        used += ((size_t)n * sizeof(V) + 15) / 16 * 16;
        return at;
    }
};

size_t layout(Counts &c, void *ws, long long tokens, long long seqs)
{
    Arena a{(char *)ws};
    const int chunks = chunks_of(tokens);
    c.part = a.take<double>(6 * std::min(chunks, kMaxGroups));
    c.seq = a.take<int>(seqs);
    c.head = a.take<int>(chunks);
    c.tail = a.take<int>(chunks);
    c.group = a.take<int>(kMaxGroups);
    c.some = a.take<int>(kJoinGroups);
    return a.used;
}

size_t layout(Pairs &p, void *ws, long long tokens, long long pairs)
{
    Arena a{(char *)ws};
    const int chunks = chunks_of(tokens);
    p.seq = a.take<double>(2 * pairs);
    p.head = a.take<double>(chunks);
    p.tail = a.take<double>(chunks);
    p.slope = a.take<double>(pairs);
    p.part = a.take<double>(5 * kJoinGroups);
    p.count = a.take<int>(2 * pairs);
    p.chead = a.take<int>(chunks);
    p.ctail = a.take<int>(chunks);
    p.some = a.take<int>(kJoinGroups);
    return a.used;
}

}  // namespace

size_t policy_ws(long long tokens, long long seqs)
{
    Counts c;
    return policy_is_small(tokens, seqs) ? 0 : layout(c, nullptr, tokens, seqs);
}

hipError_t launch_policy(const PolicyArgs &a, hipStream_t stream)
{
    const bool seqs = a.by_sequence || a.mean == 1;
    if (policy_is_small(a.tokens, a.seqs)) {
        if (seqs)
            policy_one<true><<<1, kOneBlock, 0, stream>>>(a);
        else
            policy_one<false><<<1, kOneBlock, 0, stream>>>(a);
        return hipGetLastError();
    }
    Counts c;
    layout(c, a.ws, a.tokens, a.seqs);
    const int chunks = chunks_of(a.tokens), groups = std::min(chunks, kMaxGroups);
    int joins = 0;
    if (a.mask && a.mean != 2)
        policy_count<<<groups, kBlock, 0, stream>>>(a, c, chunks);
    if (a.mean == 1) {
        joins = std::max(1, a.mask ? join_groups(a.seqs) : join_groups((a.seqs + 63LL) / 64));
        policy_join<<<joins, kBlock, 0, stream>>>(a, c);
    }
    if (seqs)
        policy_main<true><<<groups, kBlock, 0, stream>>>(a, c, chunks, joins);
    else
        policy_main<false><<<groups, kBlock, 0, stream>>>(a, c, chunks, joins);
    policy_stats<<<1, 6 * 64, 0, stream>>>(c.part, groups, a.stats);
    return hipGetLastError();
}

size_t preference_ws(long long tokens, long long pairs)
{
    Pairs p;
    return preference_is_small(tokens, pairs) ? 0 : layout(p, nullptr, tokens, pairs);
}

hipError_t launch_preference(const PreferenceArgs &a, hipStream_t stream)
{
    if (preference_is_small(a.tokens, a.pairs)) {
        preference_one<<<1, kOneBlock, 0, stream>>>(a);
        return hipGetLastError();
    }
    Pairs p;
    layout(p, a.ws, a.tokens, a.pairs);
    const int chunks = chunks_of(a.tokens), groups = std::min(chunks, kMaxGroups);
    const int joins = std::max(1, join_groups(a.pairs));
    preference_sums<<<groups, kBlock, 0, stream>>>(a, p, chunks);
    preference_pairs<<<joins, kBlock, 0, stream>>>(a, p);
    preference_fill<<<a.dlogp ? groups : 1, 5 * 64, 0, stream>>>(a, p, chunks, joins);
    return hipGetLastError();
}

}  // namespace miconv
