// The losses of fine-tuning and their gradients (include/mistep.h): the clipped
// policy loss of sampled tokens, and the loss of pairs of sequences.
//
// Tokens are taken by chunks, whatever the sequences' lengths, four or eight of them
// side by side a thread.  Where sequences begin in a chunk is marked in LDS by a thread a
// sequence; a scan over the chunk then tells each token where its sequence begins
// (what belongs to the sequence lies there), or sums the sequences' tokens.  A
// sequence that reaches over several chunks leaves its piece of each in the
// workspace: `tail` of the chunk it begins in, `head` of those that it continues in,
// and the next launch adds the pieces in the order of the chunks, so that no result
// depends on which workgroup ran first.  Calls of few tokens run as one workgroup,
// in one launch.
//
// A weight needs its sequence's (or the call's) number of tokens that count, and a
// pair's loss the sums of both its sequences, before the first gradient: that is what
// the launches are for.  Over the tokens there are two, which read the mask twice and
// everything else once; the others are over sequences (unless these are few), or join
// partial sums.  2 000 003 tokens move 50 MB for a policy, in 25.3 us, and 26 MB for
// pairs, in 20.5: the launches over the tokens run at 2 to 4 TB/s (a thread has one pack
// or two, and waits for them once), launches and their gaps take the rest.  Up to some
// 100 000 tokens there is nothing but latency: 3 to 4 us a launch (20 000 to 100 000
// tokens in 10 to 16 us), 5 to 11 for one workgroup's chain of loads, scans, exponentials
// and sums.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "step.h"

namespace miconv {

namespace {

// A workgroup's share of the tokens, a chunk: BLOCK threads, PACKS packs of EACH tokens a
// thread, the packs t + h BLOCK of thread t; 64 packs side by side are a wave's.
template <int B, int P, int E>
struct Tile {
    static constexpr int BLOCK = B, PACKS = P, EACH = E, ALL = B * P, SIZE = ALL * E;

    // Of the thread's h-th pack among all.  Computed where it is used: what follows from it,
    // held from chunk to chunk, would take the registers of the tokens (policy_main: up to
    // ten spilled, 2 000 003 tokens 26.0 us for 24.9).
    static __device__ __forceinline__ int rank(int h)
    {
        int t = (int)threadIdx.x;
        asm volatile("" : "+v"(t));
        return h * B + t;
    }
};

// Calls of many tokens.  The scans over a chunk cost as much for eight tokens a thread as
// for four, but eight tokens of a policy at once take too many registers (2 000 003
// tokens: pairs 20.6 us, by packs of four 21.7; policy 26.0 by packs of eight, 24.8 by two
// of four).
constexpr int kChunk = 2048;
typedef Tile<256, 1, 8> Wide;
typedef Tile<256, 2, 4> Narrow;
static_assert(Wide::SIZE == kChunk && Narrow::SIZE == kChunk, "one chunk for all launches");
// Calls of few, in one workgroup: up to 4096 tokens, and up to 8192 (4000 tokens: policy
// 5.2 us, pairs 7.7, by the larger 6.3 and 9.2; 8000 tokens 10.9 and 9.5, by chunks 13.8 and
// 11.2).
typedef Tile<1024, 1, 4> SmallPolicy;
typedef Tile<512, 1, 8> SmallPairs;
typedef Tile<1024, 1, 8> Small;
constexpr int kMaxGroups = 1024;  // workgroups of a launch over the chunks, and partial sums
constexpr int kJoinGroups = 1024;  // of a launch over the sequences
constexpr int kOwn = 256;  // sequences or pairs that a workgroup over the tokens joins itself
static_assert(kOwn <= Wide::BLOCK && kOwn <= Narrow::BLOCK, "a thread each");

typedef Pack<float>::V F4;

// ------------------------------------------------------------------- reductions
// Of a wave without LDS, as wave_reduce in rows.h; every lane gets the sum.
template <int CTRL>
__device__ __forceinline__ double dpp64(double v)
{
    const uint2 u = __builtin_bit_cast(uint2, v);
    uint2 r;
    r.x = __builtin_amdgcn_mov_dpp((int)u.x, CTRL, 0xf, 0xf, true);
    r.y = __builtin_amdgcn_mov_dpp((int)u.y, CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, r);
}

__device__ __forceinline__ double wave_sum(double v)
{
    v += dpp64<0xb1>(v);
    v += dpp64<0x4e>(v);
    v += dpp64<0x141>(v);
    v += dpp64<0x140>(v);
    uint2 u = __builtin_bit_cast(uint2, v);
    auto x = __builtin_amdgcn_permlane16_swap(u.x, u.x, false, false);
    auto y = __builtin_amdgcn_permlane16_swap(u.y, u.y, false, false);
    v = __builtin_bit_cast(double, uint2{x[0], y[0]}) + __builtin_bit_cast(double, uint2{x[1], y[1]});
    u = __builtin_bit_cast(uint2, v);
    x = __builtin_amdgcn_permlane32_swap(u.x, u.x, false, false);
    y = __builtin_amdgcn_permlane32_swap(u.y, u.y, false, false);
    return __builtin_bit_cast(double, uint2{x[0], y[0]}) + __builtin_bit_cast(double, uint2{x[1], y[1]});
}

__device__ __forceinline__ int wave_sum(int v)
{
    v += __builtin_amdgcn_mov_dpp(v, 0xb1, 0xf, 0xf, true);
    v += __builtin_amdgcn_mov_dpp(v, 0x4e, 0xf, 0xf, true);
    v += __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, true);
    v += __builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, true);
    auto x = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
    v = (int)(x[0] + x[1]);
    x = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
    return (int)(x[0] + x[1]);
}

// The sums of N values over a workgroup, in each thread; lds: N a wave.
template <int BLOCK, int N, class V>
__device__ __forceinline__ void block_sums(V (&v)[N], V (*lds)[N])
{
#pragma unroll
    for (int i = 0; i < N; i++) {
        v[i] = wave_sum(v[i]);
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
        v[i] = lds[0][i];
        for (int w = 1; w < BLOCK / 64; w++)
            v[i] += lds[w][i];
    }
}

// The sums of N values over a workgroup, each to one thread's f(i, sum).  some: whether
// the thread's may be other than 0.
template <int BLOCK, int N, class V, class F>
__device__ __forceinline__ void block_totals(V (&v)[N], V (*lds)[N], F f, bool some = true)
{
    const bool any = __ballot(some) != 0;
#pragma unroll
    for (int i = 0; i < N; i++) {
        if (any)
            v[i] = wave_sum(v[i]);
        if ((threadIdx.x & 63) == 0)
            lds[threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
    if (threadIdx.x < N) {
        V s = lds[0][threadIdx.x];
#pragma unroll
        for (int w = 1; w < BLOCK / 64; w++)
            s += lds[w][threadIdx.x];
        f((int)threadIdx.x, s);
    }
}

// The sum of n numbers (1 at least), by each wave; the loads of eight rounds are issued
// together.
template <class V>
__device__ __forceinline__ V sum_of(const V *p, int n)
{
    V v = V(0);
    for (int i = threadIdx.x & 63; i < n; i += 8 * 64) {
        V part[8];
#pragma unroll
        for (int k = 0; k < 8; k++)
            part[k] = p[min(i + 64 * k, n - 1)];
#pragma unroll
        for (int k = 0; k < 8; k++)
            v += i + 64 * k < n ? part[k] : V(0);
    }
    return wave_sum(v);
}

// -------------------------------------------------------------------- sequences
struct Starts {
    const long long *p;
    int tokens;

    __device__ __forceinline__ int cut(uint32_t low, int high) const
    {
        return high < 0 ? 0 : high ? tokens : (int)min(low, (uint32_t)tokens);
    }
    __device__ __forceinline__ int operator()(long long i) const
    {
        const long long v = p[i];
        return cut((uint32_t)v, (int)(v >> 32));
    }
    // Where sequence s begins and ends.
    __device__ __forceinline__ void of(long long s, int &s0, int &s1) const
    {
        typedef int V __attribute__((ext_vector_type(4)));
        typedef V At __attribute__((aligned(8)));
        const V v = *(const At *)(p + s);
        s0 = cut((uint32_t)v[0], v[1]);
        s1 = cut((uint32_t)v[2], v[3]);
    }
};

// Of the n numbers at p, which do not fall, those up to v are counted, 64 of them at a
// time by the lanes of a wave: those before lo are, those from hi on are not.
struct Search {
    const long long *p;
    long long v;
    int lo, hi;

    __device__ __forceinline__ bool open() const { return lo < hi; }
    __device__ __forceinline__ int step() const { return (int)(((long long)hi - lo + 63) / 64); }
    __device__ __forceinline__ bool probe() const
    {
        const long long at = lo + (long long)(threadIdx.x & 63) * step();
        return at < hi && p[at] <= v;
    }
    __device__ __forceinline__ void narrow(int k)
    {
        const int s = step();
        if (!k) {
            hi = lo;
            return;
        }
        hi = (int)min((long long)hi, lo + (long long)k * s);
        lo = (int)(lo + (long long)(k - 1) * s + 1);
    }
};

// The sequences that have tokens in the chunk begin <= t < end, for all threads of a
// workgroup to go through.  Each thread looks at LOOK of them, loaded at once and before
// the chunk's tokens, so that these latencies overlap; if there are more, they are
// searched for the chunk's first and last before (2 000 003 tokens: 1024 pairs with LOOK 8
// 20.6 us, with 4 and a search 22.0; 1024 sequences of a policy 29.6 and 24.8, as 8 take
// the registers of a fourth workgroup a CU).
constexpr int kPolicyLook = 4, kPairsLook = 8;

template <int BLOCK, int LOOK>
struct Sequences {
    Starts starts;
    int begin, end, first, last;
    int s0[LOOK], s1[LOOK];

    __device__ __forceinline__ Sequences(const Starts &st, int seqs, int begin_, int end_)
        : starts(st), begin(begin_), end(end_), first(0), last(seqs)
    {
        if (seqs > LOOK * BLOCK) {
            Search a{starts.p + 1, begin, 0, seqs}, b{starts.p, (long long)end - 1, 0, seqs};
            while (a.open() || b.open()) {
                const bool pa = a.open() && a.probe(), pb = b.open() && b.probe();
                const int ka = __popcll(__ballot(pa)), kb = __popcll(__ballot(pb));
                if (a.open())
                    a.narrow(ka);
                if (b.open())
                    b.narrow(kb);
            }
            first = a.lo;
            last = b.lo;
        }
        look((long long)first + threadIdx.x);
    }
    __device__ __forceinline__ void look(long long at)
    {
        // A place past the last is looked at all the same (starts has one entry more than
        // there are sequences), so that no load waits behind a branch.
        const long long most = max(last - 1, 0);
#pragma unroll
        for (int i = 0; i < LOOK; i++)
            if (last > 0)
                starts.of(min(at + i * BLOCK, most), s0[i], s1[i]);
    }
    // f(s, s0, s1), in one thread, for each sequence s, the tokens s0 <= t < s1.
    template <class F>
    __device__ __forceinline__ void each(F f)
    {
        long long at = (long long)first + threadIdx.x;
        visit(at, f);
        if (last - first <= LOOK * BLOCK)
            return;
        for (at += LOOK * BLOCK; at < last; at += LOOK * BLOCK) {
            look(at);
            visit(at, f);
        }
        look((long long)first + threadIdx.x);  // for the next time
    }
    template <class F>
    __device__ __forceinline__ void visit(long long at, F f)
    {
#pragma unroll
        for (int i = 0; i < LOOK; i++)
            if (at + i * BLOCK < last && s0[i] < s1[i] && s0[i] < end && s1[i] > begin)
                f(at + i * BLOCK, s0[i], s1[i]);
    }
};

__device__ __forceinline__ int from_lane(int v, int lane) { return __shfl(v, lane); }

// What chunks left of a sequence.
template <class V>
struct Pieces {
    V *seq;          // [seqs] of those within a chunk
    V *head, *tail;  // [chunks]

    __device__ __forceinline__ V *place(long long s, int s0, int s1, int chunk, int begin, int end)
    {
        return s0 < begin ? head + chunk : s1 > end ? tail + chunk : seq + s;
    }
};

// The sum of the pieces of a sequence (of the tokens s0 <= t < s1), for the sequence s that
// each group of `lanes` lanes (a power of two) has, else 0; in all its lanes.  Those of up
// to kFew chunks a lane are added by their group, of loads that are all issued at once,
// the others by the wave, one by one.
constexpr int kFew = 4;

template <class V>
__device__ __forceinline__ V join(bool has, const Pieces<V> &p, long long s, int s0, int s1,
                                  int lanes)
{
    const int lane = threadIdx.x & 63, own = lane & (lanes - 1);
    has = has && s0 < s1;
    const int from = has ? s0 / kChunk : 0, to = has ? (s1 - 1) / kChunk : 0, n = to - from;
    const bool few = n < kFew * lanes;
    V part[kFew], v{};
    part[0] = *(own ? p.head + min(from + own, to) : n ? p.tail + from : p.seq + (has ? s : 0));
#pragma unroll
    for (int i = 1; i < kFew; i++)
        part[i] = p.head[min(from + own + i * lanes, to)];
    if (has && few && own <= n) {
        v = part[0];
#pragma unroll
        for (int i = 1; i < kFew; i++)
            if (own + i * lanes <= n)
                v += part[i];
    }
    for (int o = 1; o < lanes; o <<= 1)
        v += from_lane(v, lane ^ o);
    unsigned long long many = __ballot(has && !few && !own);
    while (many) {
        const int at = __builtin_ctzll(many);
        many &= many - 1;
        const int f = __shfl(from, at), t = __shfl(to, at);
        V sum{};
#pragma unroll 4
        for (int k = f + lane; k <= t; k += 64)
            sum += k == f ? p.tail[k] : p.head[k];
        sum = wave_sum(sum);
        if ((lane ^ at) < lanes)
            v = sum;
    }
    return v;
}

// ----------------------------------------------------------------------- tokens
// A pack of a thread's tokens of the chunk: t0 + j for j < left.
struct Mine {
    int t0, left;
    unsigned mask;  // a bit each: there, and not masked
};

// A bit for each of four bytes: whether it is not 0.
__device__ __forceinline__ unsigned bits_of(uint32_t v)
{
    v |= v >> 4;
    v |= v >> 2;
    v = (v | v >> 1) & 0x01010101u;
    return (v | v >> 7 | v >> 14 | v >> 21) & 15;
}

// rank: of the pack in the chunk.
template <class S>
__device__ __forceinline__ Mine my_tokens(const unsigned char *mask, int begin, int end, int rank)
{
    Mine m;
    // Past the end the first token may be beyond 32 bits: it is not used.
    m.left = end - begin - rank * S::EACH;
    m.t0 = m.left > 0 ? begin + rank * S::EACH : begin;
    m.mask = (1u << min(max(m.left, 0), S::EACH)) - 1;
    if (mask && m.left > 0) {
        if (m.left >= S::EACH) {
            typedef uint32_t V __attribute__((ext_vector_type(S::EACH / 4)));
            typedef V At __attribute__((aligned(1)));
            // Four bytes, or eight.
            const V v = *(const At *)(mask + m.t0);
            m.mask = bits_of(v[0]);
            if constexpr (S::EACH == 8)
                m.mask |= bits_of(v[1]) << 4;
        } else {
            m.mask = 0;
            for (int j = 0; j < m.left; j++)
                m.mask |= (unsigned)(mask[m.t0 + j] != 0) << j;
        }
    }
    return m;
}

// Those of the pack's tokens that lie in from <= t < to.
template <class S>
__device__ __forceinline__ unsigned inside(const Mine &m, int from, int to)
{
    // Tokens past the end are not in the mask.
    const unsigned before = (1u << min(max(from - m.t0, 0), S::EACH)) - 1;
    return ((1u << min(max(to - m.t0, 0), S::EACH)) - 1) & ~before;
}

template <int E>
__device__ __forceinline__ void load_floats(const float *p, const Mine &m, float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        F4 f = F4{};
        if (m.left > i)
            f = load_pack<float>(p + m.t0 + i, m.left - i, 0.f);
#pragma unroll
        for (int j = 0; j < 4; j++)
            v[i + j] = f[j];
    }
}

template <int E>
__device__ __forceinline__ void store_floats(float *p, const Mine &m, const float (&v)[E])
{
#pragma unroll
    for (int i = 0; i < E; i += 4)
        if (m.left > i)
            store_pack<float>(p + m.t0 + i, m.left - i, F4{v[i], v[i + 1], v[i + 2], v[i + 3]});
}

// How many tokens of the chunk before each count: by pack, and a bit each.
template <class S>
struct CountTable {
    static constexpr int ALL = S::ALL;
    int before[ALL];
    unsigned char bits[ALL];
    int waves[ALL / 64];

    // To be called by all threads; the caller's barrier follows.
    __device__ __forceinline__ void scan(int h, unsigned counted)
    {
        const int rank = S::rank(h);
        int v = 0, n = 0;
#pragma unroll
        for (int j = 0; j < S::EACH; j++) {
            const unsigned long long b = __ballot(counted >> j & 1);
            v += __builtin_amdgcn_mbcnt_hi((unsigned)(b >> 32),
                                           __builtin_amdgcn_mbcnt_lo((unsigned)b, 0));
            n += __popcll(b);
        }
        before[rank] = v;
        bits[rank] = (unsigned char)counted;
        if ((threadIdx.x & 63) == 0)
            waves[rank >> 6] = n;
    }
    // Of the chunk's tokens before its at-th (at most all).
    __device__ __forceinline__ int up_to(int at) const
    {
        const int i = at / S::EACH;
        int v = 0;
        for (int w = 0; w < i / 64; w++)
            v += waves[w];
        return i < ALL ? v + before[i] + __popc(bits[i] & ((1u << at % S::EACH) - 1)) : v;
    }
};

// Marks in LDS where sequences begin: a byte each of the chunk's tokens.
template <class S>
struct Marks {
    static constexpr int ALL = S::ALL, SIZE = S::SIZE;
    alignas(8) unsigned char at[SIZE];
    int waves[ALL / 64];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int h = 0; h < S::PACKS; h++)
            for (int i = 0; i < S::EACH; i += 4)
                *(uint32_t *)(at + S::rank(h) * S::EACH + i) = 0;
    }
    __device__ __forceinline__ unsigned mine(int h) const
    {
        unsigned bits = 0;
#pragma unroll
        for (int i = 0; i < S::EACH; i += 4) {
            const uint32_t b = *(const uint32_t *)(at + S::rank(h) * S::EACH + i);
            bits |= ((b | b >> 7 | b >> 14 | b >> 21) & 15) << i;  // of bytes that are 0 or 1
        }
        return bits;
    }
    // Where the sequence of each of the thread's tokens begins in the chunk, -1 where
    // none has begun.  One barrier.
    __device__ __forceinline__ void places(int (&place)[S::PACKS][S::EACH])
    {
        const int lane = threadIdx.x & 63;
        unsigned marks[S::PACKS];
        int last[S::PACKS];
        bool within[S::PACKS];
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            const int rank = S::rank(h);
            marks[h] = mine(h);
            const int own = rank * S::EACH + 31 - __builtin_clz(marks[h] | 1);
            const unsigned long long any = __ballot(marks[h] != 0);
            const unsigned long long before = any & ((1ULL << lane) - 1);
            within[h] = before != 0;
            last[h] = __shfl(own, before ? 63 - __builtin_clzll(before) : 0);
            if (lane == (any ? 63 - __builtin_clzll(any) : 0))
                waves[rank >> 6] = any ? own : -1;
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            const int rank = S::rank(h);
            if (!within[h]) {
                last[h] = -1;
                for (int w = (rank >> 6) - 1; w >= 0 && last[h] < 0; w--)
                    last[h] = waves[w];
            }
#pragma unroll
            for (int j = 0; j < S::EACH; j++) {
                last[h] = marks[h] >> j & 1 ? rank * S::EACH + j : last[h];
                place[h][j] = last[h];
            }
        }
    }
};

__device__ __forceinline__ int end_of_chunk(int begin, int tokens)
{
    return begin + min(kChunk, tokens - begin);
}

// ------------------------------------------------------------------ policy loss
// What a call of many tokens keeps between its launches.
struct Counts {
    double *part;     // [5][groups] each workgroup's sums
    Pieces<int> n;    // tokens that count; seq later of all sequences
    int *group;       // [kMaxGroups] tokens that count of each workgroup's chunks
    int *some;        // [kJoinGroups] sequences that have any
};

// Which tokens count: of each sequence (mean 1) as its pieces, or of the workgroup's
// chunks.  Reads the mask alone (2 000 003 tokens: 4.6 us, 1024 sequences); not launched
// where there is none, or where the caller gives the number.
__global__ __launch_bounds__(Narrow::BLOCK) void policy_count(PolicyArgs a, Counts c, int chunks)
{
    typedef Narrow S;
    __shared__ CountTable<S> table;
    __shared__ int red[S::BLOCK / 64][1];
    const Starts starts{a.starts, a.tokens};
    int all[1] = {0};
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int begin = k * S::SIZE, end = end_of_chunk(begin, a.tokens);
        Mine m[S::PACKS];
        if (a.mean == 1) {
            Sequences<S::BLOCK, kPolicyLook> q(starts, a.seqs, begin, end);
#pragma unroll
            for (int h = 0; h < S::PACKS; h++) {
                m[h] = my_tokens<S>(a.mask, begin, end, S::rank(h));
                table.scan(h, m[h].mask);
            }
            __syncthreads();
            q.each([&](long long s, int s0, int s1) {
                *c.n.place(s, s0, s1, k, begin, end) =
                    table.up_to(min(s1, end) - begin) - table.up_to(max(s0, begin) - begin);
            });
            __syncthreads();
        } else {
            const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
#pragma unroll
            for (int h = 0; h < S::PACKS; h++) {
                m[h] = my_tokens<S>(a.mask, begin, end, S::rank(h));
                all[0] += __popc(m[h].mask & inside<S>(m[h], from, to));
            }
        }
    }
    if (a.mean == 1)
        return;
    block_totals<S::BLOCK>(all, red, [&](int, int v) { c.group[blockIdx.x] = v; });
}

// The tokens that count of the sequence s that a group of lanes has, else 0.
__device__ __forceinline__ int sequence_tokens(const PolicyArgs &a, const Counts &c,
                                               const Starts &starts, long long s, bool has,
                                               int lanes)
{
    int s0 = 0, s1 = 0;
    if (has)
        starts.of(s, s0, s1);
    return a.mask ? join(has, c.n, s, s0, s1, lanes) : max(s1 - s0, 0);
}

// Each sequence's tokens that count, and how many sequences have any (2.4 us for 1024:
// the latency of starts, then of their pieces).
constexpr int kJoinBlock = 256;

__global__ __launch_bounds__(kJoinBlock) void policy_join(PolicyArgs a, Counts c, int lanes)
{
    __shared__ int red[kJoinBlock / 64][1];
    const Starts starts{a.starts, a.tokens};
    const int each = kJoinBlock / lanes;
    const bool leads = (threadIdx.x & (lanes - 1)) == 0;
    int some[1] = {0};
    for (long long first = (long long)blockIdx.x * each; first < a.seqs;
         first += (long long)gridDim.x * each) {
        const long long s = first + threadIdx.x / lanes;
        const bool has = s < a.seqs;
        const int n = sequence_tokens(a, c, starts, s, has, lanes);
        if (a.mask && has && leads)
            c.n.seq[s] = n;
        some[0] += leads && n > 0;
    }
    block_totals<kJoinBlock>(some, red, [&](int, int v) { c.some[blockIdx.x] = v; });
}

// exp(x): 2^h (1 + l ln 2) with h + l = x log2(e), h its rounding to 32 bits and l what
// that leaves, so that large |x| lose nothing.  Results below 2^-126 are 0; those from
// 2^128 on are infinite, without the factor: infinity times an l of 0 or below is none.
__device__ __forceinline__ float exp_of(float x)
{
    constexpr float log2e = 0x1.715476p+0f, rest = 0x1.4ae0bep-26f;  // log2(e) = their sum
    const float h = x * log2e;
    float l = fmaf(x, log2e, -h);
    l = fmaf(x, rest, l);
    const float e = __builtin_amdgcn_exp2f(h);
    return fabsf(h) < 128.f ? fmaf(e, l * 0x1.62e43p-1f, e) : e;
}

// exp(x) - 1 - x, and exp(x) - 1; near 0 by the exponential's series, where the
// difference would lose what matters.
__device__ __forceinline__ float low_kl(float x, float *expm1)
{
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
    float v = x * x * p;
    *expm1 = x + v;
    if (!(fabsf(x) < 1.f)) {
        *expm1 = exp_of(x) - 1.f;
        v = *expm1 - fminf(x, 0x1.fffffep+127f);  // infinite at infinity
    }
    return v;
}

// The same in all lanes: held once for the wave, in no lane's register.
__device__ __forceinline__ float uniform(float v)
{
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

__device__ __forceinline__ double uniform(double v)
{
    const uint2 u = __builtin_bit_cast(uint2, v);
    return __builtin_bit_cast(double, uint2{(unsigned)__builtin_amdgcn_readfirstlane((int)u.x),
                                            (unsigned)__builtin_amdgcn_readfirstlane((int)u.y)});
}

// The borders of the clip in 32 bits, and the ratio at them.
struct Borders {
    float low, high, dual, at_low, at_high, at_dual;
    float near;  // how near to a border 32 bits do not tell on which side a log ratio is

    __device__ __forceinline__ explicit Borders(const PolicyArgs &a)
        : low(uniform((float)a.log_low)), high(uniform((float)a.log_high)),
          dual(uniform((float)a.log_dual)), at_low(a.low), at_high(a.high), at_dual(a.dual)
    {
        const auto size = [](float v) { return __builtin_isfinite(v) ? fabsf(v) : 0.f; };
        near = uniform(fmaxf(fmaxf(size(low), size(high)), size(dual)) * 0x1p-22f);
    }
};

// A token's terms and the slope of its loss in logp.  With d = logp - old and r = e^d the
// surrogate is -a r up to the clip, and its slope is itself; past it -a times the border,
// without slope.  The divergence's x is ref - logp: its slopes in logp are 1, -x and
// 1 - e^x of -x, x^2 / 2 and e^x - 1 - x.
struct Token {
    float surrogate, kl, ratio, slope;
    bool clipped;
};

// The reference's part: none, the low form, or the others.
enum class Ref { none, low, other };

template <Ref REF>
__device__ __forceinline__ Token token_loss(const PolicyArgs &a, const Borders &b, float lp,
                                            float lo, float lr, float adv)
{
    Token k;
    const float d = lp - lo;  // off by 2^-24 of it
    k.ratio = exp_of(d);
    // Above: clipped there for a gain, by the dual clip for a loss; below for a loss.
    const bool gain = adv > 0.f;
    const float b_high = b.high, b_dual = b.dual, b_low = b.low, at_high = b.at_high,
                at_dual = b.at_dual;  // a choice of values, not of addresses
    const float top = gain ? b_high : b_dual, bottom = gain ? -__builtin_inff() : b_low;
    bool above = d > top, below = d < bottom;
    if (fabsf(d - top) <= b.near || fabsf(d - bottom) <= b.near) {
        const double e = (double)lp - (double)lo;
        above = gain ? e > a.log_high : e > a.log_dual;
        below = !gain && e < a.log_low;
    }
    float r = above ? (gain ? at_high : at_dual) : k.ratio;
    r = below ? b.at_low : r;
    // No advantage gives nothing, however large the ratio; NaN stays.
    r = adv == 0.f && r == __builtin_inff() ? 0.f : r;
    k.clipped = (above || below) && fabsf(adv) > 0.f;
    k.surrogate = -adv * r;
    k.slope = k.clipped ? 0.f : k.surrogate;
    k.kl = 0.f;
    if constexpr (REF != Ref::none) {
        const float x = lr - lp;
        float slope;
        if (REF == Ref::low) {
            k.kl = low_kl(x, &slope);
            slope = -slope;
        } else if (a.kl == 0) {
            k.kl = -x;
            slope = 1.f;
        } else {
            k.kl = 0.5f * x * x;
            slope = -x;
        }
        k.slope = a.kl_weight != 0.f ? fmaf(a.kl_weight, slope, k.slope) : k.slope;
    }
    return k;
}

template <int E>
struct Tokens {
    float lp[E], lo[E], lr[E], h[E], adv[E];
};

template <Ref REF, int E>
__device__ __forceinline__ void load_tokens(const PolicyArgs &a, const Mine &m, Tokens<E> &k)
{
#pragma unroll
    for (int j = 0; j < E; j++)
        k.h[j] = 0.f;
    load_floats(a.logp, m, k.lp);
    load_floats(a.old_logp, m, k.lo);
    if (REF != Ref::none)
        load_floats(a.ref_logp, m, k.lr);
    if (a.entropy)
        load_floats(a.entropy, m, k.h);
    if (!a.by_sequence)
        load_floats(a.advantages, m, k.adv);
}

// A pack's weights within their sequences: 1 unless WEIGHTS, 0 of tokens that do not count.
// counted: those that do; weights, place: theirs, and where they lie.
template <bool WEIGHTS, int E>
__device__ __forceinline__ void token_weights(unsigned counted, const double *weights,
                                              const int (&place)[E], double (&w)[E])
{
#pragma unroll
    for (int j = 0; j < E; j++) {
        w[j] = WEIGHTS ? weights[place[j]] : 1.0;
        w[j] = counted >> j & 1 ? w[j] : 0.0;
    }
}

// The tokens' entropies, times their weights, to sum, and their gradients to memory; before
// the rest, so that their registers are free for it.  factor: what a gradient's weight is
// multiplied by.
template <int E>
__device__ __forceinline__ void token_entropies(const PolicyArgs &a, const Mine &m,
                                                const Tokens<E> &k, const double (&w)[E],
                                                unsigned counted, double factor, double (&sum)[5])
{
    float g[E];
#pragma unroll
    for (int j = 0; j < E; j++) {
        sum[2] = fma((double)(counted >> j & 1 ? k.h[j] : 0.f), w[j], sum[2]);
        g[j] = (float)(-(double)a.entropy_weight * factor * w[j]);
    }
    if (a.dentropy)
        store_floats(a.dentropy, m, g);
}

// The tokens' surrogates, divergences, ratios and clips, times their weights, to sum, and
// their gradients to memory.  A token's terms are of 32 bits, as its log probabilities are;
// weights, products and sums of 64 (2 000 003 tokens 24.9 us, with all of them in 32 bits up
// to a thread's sum 24.4), and a gradient is rounded once.
template <Ref REF, int E>
__device__ __forceinline__ void token_losses(const PolicyArgs &a, const Borders &borders,
                                             const Mine &m, const Tokens<E> &k, const double (&w)[E],
                                             unsigned counted, double factor, double (&sum)[5])
{
    float g[E];
#pragma unroll
    for (int j = 0; j < E; j++) {
        // A token that does not count is one of nothing but zeros, with no weight.
        const bool in = counted >> j & 1;
        const auto only = [in](float v) { return in ? v : 0.f; };
        const Token r = token_loss<REF>(a, borders, only(k.lp[j]), only(k.lo[j]),
                                        REF == Ref::none ? 0.f : only(k.lr[j]), only(k.adv[j]));
        sum[0] = fma((double)r.surrogate, w[j], sum[0]);
        if (REF != Ref::none)
            sum[1] = fma((double)r.kl, w[j], sum[1]);
        sum[3] = fma((double)r.ratio, w[j], sum[3]);
        sum[4] += r.clipped ? w[j] : 0.0;
        g[j] = (float)((double)r.slope * (w[j] * factor));
        __builtin_amdgcn_sched_barrier(0);  // a token at a time: fewer registers, more waves
    }
    if (a.dlogp)
        store_floats(a.dlogp, m, g);
}

// A thread's packs.
template <class S, bool WEIGHTS, Ref REF>
__device__ __forceinline__ void all_losses(const PolicyArgs &a, const Borders &borders,
                                           const Mine (&m)[S::PACKS],
                                           const Tokens<S::EACH> (&k)[S::PACKS], int from, int to,
                                           const double *weights,
                                           const int (&place)[S::PACKS][S::EACH], double factor,
                                           double (&sum)[5])
{
    double w[S::EACH];
#pragma unroll
    for (int h = 0; h < S::PACKS; h++) {
        const unsigned counted = m[h].mask & inside<S>(m[h], from, to);
        token_weights<WEIGHTS>(counted, weights, place[h], w);
        if (a.entropy)
            token_entropies(a, m[h], k[h], w, counted, factor, sum);
        token_losses<REF>(a, borders, m[h], k[h], w, counted, factor, sum);
    }
}

// The results from the sums over all tokens (times their weights): the loss is
// linear in them.
__device__ __forceinline__ float policy_result(const PolicyArgs &a, const double *sum, int i)
{
    if (i)
        return (float)sum[i - 1];
    double v = sum[0];
    if (a.ref_logp && a.kl_weight != 0.f)
        v += (double)a.kl_weight * sum[1];
    if (a.entropy && a.entropy_weight != 0.f)
        v -= (double)a.entropy_weight * sum[2];
    return (float)v;
}

// What sequences give their tokens, where these begin in the chunk.
template <int SIZE>
struct OfSequences {
    double weight[SIZE];
    float adv[SIZE];

    // Of sequence s with n tokens that count.
    __device__ __forceinline__ void set(const PolicyArgs &a, int at, long long s, int n)
    {
        const float v = a.by_sequence ? a.advantages[s] : 0.f;  // awaited with n
        weight[at] = a.mean == 1 ? 1.0 / max(n, 1) : 1.0;
        adv[at] = v;
    }
};

// Where the tokens' weights lie, and their advantages from there.
template <class S>
__device__ __forceinline__ void from_sequences(const PolicyArgs &a, Marks<S> &marks,
                                               const OfSequences<S::SIZE> &seq,
                                               Tokens<S::EACH> (&k)[S::PACKS],
                                               int (&place)[S::PACKS][S::EACH])
{
    marks.places(place);
#pragma unroll
    for (int h = 0; h < S::PACKS; h++)
#pragma unroll
        for (int j = 0; j < S::EACH; j++) {
            place[h][j] = max(place[h][j], 0);
            if (a.by_sequence)
                k[h].adv[j] = seq.adv[place[h][j]];
        }
}

// Few tokens: all of the call in one workgroup (4000 tokens 5.2 us, all of it latency).
// SEQS: the sequences matter.
template <class S, bool SEQS, Ref REF>
__global__ __launch_bounds__(S::BLOCK) void policy_one(PolicyArgs a)
{
    constexpr int WAVES = S::BLOCK / 64;
    __shared__ Marks<std::conditional_t<SEQS, S, Tile<64, 1, 4>>> marks;
    __shared__ CountTable<std::conditional_t<SEQS, S, Tile<64, 1, 4>>> table;
    __shared__ OfSequences<SEQS ? S::SIZE : 1> seq;
    __shared__ double red[WAVES][5], total[5];
    __shared__ int counts[WAVES][1];
    const Starts starts{a.starts, a.tokens};
    const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
    Sequences<S::BLOCK, kPolicyLook> q(starts, SEQS ? a.seqs : 0, 0, a.tokens);
    Mine m[S::PACKS];
    Tokens<S::EACH> k[S::PACKS];
    int place[S::PACKS][S::EACH];
#pragma unroll
    for (int h = 0; h < S::PACKS; h++) {
        m[h] = my_tokens<S>(a.mask, 0, a.tokens, S::rank(h));
        load_tokens<REF>(a, m[h], k[h]);
#pragma unroll
        for (int j = 0; j < S::EACH; j++)
            place[h][j] = 0;
    }
    int n[1] = {0};  // tokens that count, or sequences that have any
#pragma unroll
    for (int h = 0; h < S::PACKS; h++)
        n[0] += __popc(m[h].mask & inside<S>(m[h], from, to));
    const bool counted = n[0] > 0;
    double u = 1.0 / a.count;
    if constexpr (SEQS) {
        marks.clear();
#pragma unroll
        for (int h = 0; h < S::PACKS; h++)
            table.scan(h, m[h].mask);
        __syncthreads();
        if (a.mean == 1)
            n[0] = 0;
        q.each([&](long long s, int s0, int s1) {
            const int c = table.up_to(s1) - table.up_to(s0);
            if (a.mean == 1)
                n[0] += c > 0;
            marks.at[s0] = 1;
            seq.set(a, s0, s, c);
        });
    }
    if (a.mean != 2) {
        block_sums<S::BLOCK>(n, counts);
        u = 1.0 / max(n[0], 1);
    }
    if constexpr (SEQS) {
        __syncthreads();
        from_sequences(a, marks, seq, k, place);
    }
    const Borders borders(a);
    double sum[5] = {0, 0, 0, 0, 0};
    all_losses<S, SEQS, REF>(a, borders, m, k, from, to, seq.weight, place, uniform(u * a.scale),
                             sum);
    block_totals<S::BLOCK>(sum, red, [&](int i, double v) { total[i] = v * u; }, counted);
    __syncthreads();
    if (threadIdx.x < 6)
        a.stats[threadIdx.x] = policy_result(a, total, (int)threadIdx.x);
}

// The losses and gradients of a workgroup's chunks (2 000 003 tokens, 1024 sequences: 15.6
// us for 34 MB read and 16 written, 3.2 TB/s).  Some 160 vector instructions a token, of it
// two exponentials; by 128 registers, none spilled, four workgroups a CU hide their loads
// behind each other's arithmetic.
// OWN: all sequences are joined here, by `lanes` lanes each.
template <bool SEQS, bool OWN, Ref REF>
__global__ __launch_bounds__(Narrow::BLOCK, 4) void policy_main(PolicyArgs a, Counts c, int chunks,
                                                             int joins, int lanes)
{
    typedef Narrow S;
    __shared__ int n_of[OWN ? S::BLOCK : 1], some[S::BLOCK / 64][1];
    __shared__ Marks<std::conditional_t<SEQS, S, Tile<64, 1, 4>>> marks;
    __shared__ OfSequences<SEQS ? S::SIZE : 1> seq;
    __shared__ double red[S::BLOCK / 64][5], of_all;
    const Starts starts{a.starts, a.tokens};
    const Borders borders(a);
    double u = 0.0, sum[5] = {0, 0, 0, 0, 0};
    const int from = a.starts ? starts(0) : 0, to = a.starts ? starts(a.seqs) : a.tokens;
    if constexpr (OWN) {
        const int s = threadIdx.x / lanes;
        const bool has = s < a.seqs, leads = (threadIdx.x & (lanes - 1)) == 0;
        int n[1];
        n[0] = sequence_tokens(a, c, starts, s, has, lanes);
        if (leads)
            n_of[s] = n[0];
        n[0] = leads && n[0] > 0;
        block_sums<S::BLOCK>(n, some);
        if (threadIdx.x == 0)
            of_all = 1.0 / max(n[0], 1);
    } else if (threadIdx.x < 64) {  // what all weights are multiplied by
        double n = a.count;
        if (a.mean == 1)
            n = max(sum_of(c.some, joins), 1);
        else if (a.mean == 0)
            n = max(a.mask ? sum_of(c.group, (int)gridDim.x) : to - from, 1);
        of_all = 1.0 / n;
    }
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int begin = k * S::SIZE, end = end_of_chunk(begin, a.tokens);
        Sequences<S::BLOCK, kPolicyLook> q(starts, SEQS ? a.seqs : 0, begin, end);
        Mine m[S::PACKS];
        Tokens<S::EACH> tokens[S::PACKS];
        int place[S::PACKS][S::EACH];
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            m[h] = my_tokens<S>(a.mask, begin, end, S::rank(h));
            load_tokens<REF>(a, m[h], tokens[h]);
#pragma unroll
            for (int j = 0; j < S::EACH; j++)
                place[h][j] = 0;
        }
        if constexpr (SEQS) {
            marks.clear();
            __syncthreads();
            q.each([&](long long s, int s0, int s1) {
                const int at = max(s0, begin) - begin;
                int n = s1 - s0;
                if constexpr (OWN)
                    n = n_of[s];
                else if (a.mean == 1 && a.mask)
                    n = c.n.seq[s];
                marks.at[at] = 1;
                seq.set(a, at, s, n);
            });
        }
        if (SEQS || k == (int)blockIdx.x)
            __syncthreads();
        u = uniform(of_all);
        if constexpr (SEQS)
            from_sequences(a, marks, seq, tokens, place);
        all_losses<S, SEQS, REF>(a, borders, m, tokens, from, to, seq.weight, place,
                                 uniform(u * a.scale), sum);
        if (SEQS)
            __syncthreads();
    }
    block_totals<S::BLOCK>(sum, red, [&](int i, double v) {
        c.part[(size_t)i * gridDim.x + blockIdx.x] = v * u;
    });
}

// A wave a sum of the workgroups' (2.0 to 3.7 us).
__global__ __launch_bounds__(5 * 64) void policy_stats(PolicyArgs a, const double *part, int groups)
{
    __shared__ double sum[5];
    const int i = threadIdx.x >> 6;
    const double v = sum_of(part + (size_t)i * groups, groups);
    if ((threadIdx.x & 63) == 0)
        sum[i] = v;
    __syncthreads();
    if (threadIdx.x < 6)
        a.stats[threadIdx.x] = policy_result(a, sum, (int)threadIdx.x);
}

// -------------------------------------------------------------- preference loss
// A sum of log ratios, and of how many tokens.
struct Piece {
    double sum;
    long long n;
    __device__ __forceinline__ Piece &operator+=(const Piece &o)
    {
        sum += o.sum;
        n += o.n;
        return *this;
    }
};

__device__ __forceinline__ Piece wave_sum(const Piece &p)
{
    return Piece{wave_sum(p.sum), wave_sum((int)p.n)};
}

__device__ __forceinline__ Piece from_lane(const Piece &p, int lane)
{
    return Piece{__shfl(p.sum, lane), __shfl((int)p.n, lane)};
}

// What a call of many tokens keeps between its launches.
struct Pairs {
    Pieces<Piece> sum;  // log ratios and tokens that count; seq later of all sequences
    double *slope;      // [pairs] of the loss in x
    double *part;       // [5][joins]
    int *some;          // [kJoinGroups] pairs that have a token
};

struct Pair {
    double stats[5], slope;
};

__device__ __forceinline__ double reward(const PreferenceArgs &a, double sum, int n)
{
    return a.beta * (a.length_mean ? sum / max(n, 1) : sum);
}

// With r0 and r1 the rewards of the preferred and the other, and x = r0 - r1 - margin: the
// loss and its slope in x, in 64 bits (there are few pairs).  -(1 - e) ln s(x) - e ln s(-x)
// with s the logistic function, of z = e^-|x| that cannot overflow; max(0, 1 - x);
// ((x - 1/2) / beta)^2.
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

// A token's gradient in a sequence of n tokens that count, but for the pairs' number.
__device__ __forceinline__ double pair_gradient(const PreferenceArgs &a, double slope, bool second,
                                               int n)
{
    const double v = slope * a.beta * a.scale / (a.length_mean ? max(n, 1) : 1);
    return second ? -v : v;
}

// The tokens' log ratios in 64 bits (2 000 003 tokens of 1024 pairs 20.7 us, rounded to 32
// before they are added 20.5), 0 where they do not count.
template <int E>
__device__ __forceinline__ void load_ratios(const PreferenceArgs &a, const Mine &m, double (&v)[E])
{
    float lp[E], lr[E];
    load_floats(a.logp, m, lp);
    if (a.ref_logp)
        load_floats(a.ref_logp, m, lr);
#pragma unroll
    for (int j = 0; j < E; j++) {
        v[j] = a.ref_logp ? (double)lp[j] - (double)lr[j] : (double)lp[j];
        v[j] = m.mask >> j & 1 ? v[j] : 0.0;
    }
}

// The sums of the chunk's sequences, each at its last token, of the threads' values
// and the marks where sequences begin.
template <class S>
struct Sums {
    static constexpr int ALL = S::ALL;
    double at[S::SIZE];
    double tail[ALL / 64];             // since the wave's last mark
    unsigned long long marked[ALL / 64];

    // One barrier; the caller's follows.
    __device__ __forceinline__ void scan(const Marks<S> &marks,
                                         const double (&v)[S::PACKS][S::EACH])
    {
        const int lane = threadIdx.x & 63;
        double run[S::PACKS][S::EACH], before[S::PACKS];
        unsigned mine[S::PACKS];
        bool within[S::PACKS];
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            const int rank = S::rank(h);
            mine[h] = marks.mine(h);
            double s = 0;
#pragma unroll
            for (int j = 0; j < S::EACH; j++) {
                s = mine[h] >> j & 1 ? v[h][j] : s + v[h][j];
                run[h][j] = s;
            }
            // A lane takes those before it up to the last that has a mark.
            const unsigned long long any = __ballot(mine[h] != 0);
            const unsigned long long here = any & (~0ULL >> (63 - lane));
            const int last = here ? 63 - __builtin_clzll(here) : -1;
            double t = s;
            for (int o = 1; o < 64; o <<= 1) {
                const double q = __shfl_up(t, o);
                if (lane >= o && lane - o >= last && last != lane)
                    t += q;
            }
            if (lane == 63) {
                tail[rank >> 6] = t;
                marked[rank >> 6] = any;
            }
            // What comes before the pack in its first token's sequence.
            before[h] = __shfl_up(t, 1);
            if (lane == 0)
                before[h] = 0;
            within[h] = any & ((1ULL << lane) - 1);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            const int rank = S::rank(h);
            if (!within[h])  // from the waves before, the nearest first
                for (int w = (rank >> 6) - 1; w >= 0; w--) {
                    before[h] += tail[w];
                    if (marked[w])
                        break;
                }
            const bool next = rank + 1 == ALL || marks.at[min(rank + 1, ALL - 1) * S::EACH];
#pragma unroll
            for (int j = 0; j < S::EACH; j++) {
                const bool ends = j + 1 < S::EACH ? mine[h] >> (j + 1) & 1 : next;
                if (ends)
                    at[rank * S::EACH + j] =
                        mine[h] & ((2u << j) - 1) ? run[h][j] : before[h] + run[h][j];
            }
        }
    }
};

// Marks where a sequence begins and ends in the chunk, so that its sum stops there
// whatever follows.
template <class M>
__device__ __forceinline__ void mark_sequence(M &marks, int first, int end)
{
    marks.at[first] = 1;
    if (end < M::SIZE)
        marks.at[end] = 1;
}

// The sums of log ratios and the counts of each sequence, or its pieces: a segmented scan
// over the chunk in 64 bits, at whose places the sequences' threads look (2 000 003
// tokens: 9.4 us for 18 MB, 76 vector instructions a token).
__global__ __launch_bounds__(Wide::BLOCK) void preference_sums(PreferenceArgs a, Pairs p,
                                                                int chunks)
{
    typedef Wide S;
    __shared__ Marks<S> marks;
    __shared__ CountTable<S> table;
    __shared__ Sums<S> sums;
    const Starts starts{a.starts, a.tokens};
    for (int k = blockIdx.x; k < chunks; k += gridDim.x) {
        const int begin = k * S::SIZE, end = end_of_chunk(begin, a.tokens);
        Sequences<S::BLOCK, kPairsLook> q(starts, 2 * a.pairs, begin, end);
        double v[S::PACKS][S::EACH];
#pragma unroll
        for (int h = 0; h < S::PACKS; h++) {
            const Mine m = my_tokens<S>(a.mask, begin, end, S::rank(h));
            load_ratios(a, m, v[h]);
            table.scan(h, m.mask);
        }
        marks.clear();
        __syncthreads();
        q.each([&](long long, int s0, int s1) {
            mark_sequence(marks, max(s0, begin) - begin, min(s1, end) - begin);
        });
        __syncthreads();
        sums.scan(marks, v);
        __syncthreads();
        q.each([&](long long s, int s0, int s1) {
            const int b = max(s0, begin) - begin, e = min(s1, end) - begin;
            *p.sum.place(s, s0, s1, k, begin, end) =
                Piece{sums.at[e - 1], table.up_to(e) - table.up_to(b)};
        });
        __syncthreads();
    }
}

// What a group of lanes gets of its pair.
struct Joined {
    Piece v[2];  // of both sequences
    double r[2];
    Pair q;
    bool some;  // has a token
};

__device__ __forceinline__ Joined join_pair(const PreferenceArgs &a, const Pairs &p,
                                            const Starts &starts, long long i, bool has, int lanes)
{
    Joined o;
    int s0[2], s1[2];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        s0[k] = s1[k] = 0;
        if (has)
            starts.of(i + (long long)k * a.pairs, s0[k], s1[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; k++)
        o.v[k] = join(has, p.sum, i + (long long)k * a.pairs, s0[k], s1[k], lanes);
#pragma unroll
    for (int k = 0; k < 2; k++)
        o.r[k] = reward(a, o.v[k].sum, (int)o.v[k].n);
    o.q = pair_loss(a, o.r[0], o.r[1]);
    o.some = o.v[0].n + o.v[1].n > 0;
    return o;
}

// A thread a pair: its rewards and loss (4.0 us for 1024, the latency of starts, pieces, an
// exponential and a logarithm in 64 bits).
__global__ __launch_bounds__(kJoinBlock) void preference_pairs(PreferenceArgs a, Pairs p, int lanes)
{
    __shared__ double red[kJoinBlock / 64][6];
    const Starts starts{a.starts, a.tokens};
    double sum[6] = {0, 0, 0, 0, 0, 0};  // the results, and how many pairs they are of
    const int each = kJoinBlock / lanes;
    const bool leads = (threadIdx.x & (lanes - 1)) == 0;
    for (long long first = (long long)blockIdx.x * each; first < a.pairs;
         first += (long long)gridDim.x * each) {
        const long long i = first + threadIdx.x / lanes;
        const bool has = i < a.pairs;
        const Joined o = join_pair(a, p, starts, i, has, lanes);
        if (!has || !leads)
            continue;
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const long long s = i + (long long)k * a.pairs;
            p.sum.seq[s] = o.v[k];
            if (a.rewards)
                a.rewards[s] = (float)o.r[k];
        }
        p.slope[i] = o.q.slope;
        if (o.some) {
#pragma unroll
            for (int k = 0; k < 5; k++)
                sum[k] += o.q.stats[k];
            sum[5] += 1;
        }
    }
    block_totals<kJoinBlock>(sum, red, [&](int i, double v) {
        if (i < 5)
            p.part[(size_t)i * gridDim.x + blockIdx.x] = v;
        else
            p.some[blockIdx.x] = (int)v;
    });
}

// The tokens' gradients from what lies where their sequences begin.
template <class S>
__device__ __forceinline__ void store_gradients(const PreferenceArgs &a, const Mine (&m)[S::PACKS],
                                                int from, int to, Marks<S> &marks,
                                                const double *seq, double u)
{
    int place[S::PACKS][S::EACH];
    marks.places(place);
#pragma unroll
    for (int h = 0; h < S::PACKS; h++) {
        const unsigned counted = m[h].mask & inside<S>(m[h], from, to);
        float g[S::EACH];
#pragma unroll
        for (int j = 0; j < S::EACH; j++) {
            const float v = (float)(seq[max(place[h][j], 0)] * u);
            g[j] = counted >> j & 1 ? v : 0.f;
        }
        store_floats(a.dlogp, m[h], g);
    }
}

// The gradients; the workgroup behind those of the chunks adds the results (2 000 003
// tokens: 6.4 us for 2 MB of mask and 8 MB written).
// OWN: all pairs are joined here, by `lanes` lanes each.
template <bool OWN>
__global__ __launch_bounds__(Wide::BLOCK) void preference_fill(PreferenceArgs a, Pairs p,
                                                                int chunks, int joins, int lanes)
{
    typedef Wide S;
    __shared__ double slope_of[OWN ? S::BLOCK : 1], red[S::BLOCK / 64][5];
    __shared__ int n_of[2][OWN ? S::BLOCK : 1], some[S::BLOCK / 64][1];
    __shared__ Marks<S> marks;
    __shared__ double seq[S::SIZE];
    const Starts starts{a.starts, a.tokens};
    __shared__ double of_all;
    const unsigned groups = gridDim.x - 1;
    if constexpr (OWN) {
        const int i = threadIdx.x / lanes;
        const bool has = i < a.pairs, leads = (threadIdx.x & (lanes - 1)) == 0;
        const Joined o = join_pair(a, p, starts, i, has, lanes);
        const bool counts = has && leads && o.some;
        if (leads) {
            slope_of[i] = o.q.slope;
            n_of[0][i] = (int)o.v[0].n;
            n_of[1][i] = (int)o.v[1].n;
        }
        int n[1] = {counts};
        block_sums<S::BLOCK>(n, some);
        const double u = 1.0 / max(n[0], 1);
        if (threadIdx.x == 0)
            of_all = u;
        if (blockIdx.x == groups) {
            if (a.rewards && has && leads)
#pragma unroll
                for (int k = 0; k < 2; k++)
                    a.rewards[i + (long long)k * a.pairs] = (float)o.r[k];
            double sum[5];
#pragma unroll
            for (int k = 0; k < 5; k++)
                sum[k] = counts ? o.q.stats[k] : 0.0;
            block_totals<S::BLOCK>(sum, red, [&](int k, double v) { a.stats[k] = (float)(v * u); });
            return;
        }
    } else {
        if (threadIdx.x < 64)
            of_all = 1.0 / max(sum_of(p.some, joins), 1);  // what all pairs are multiplied by
        if (blockIdx.x == groups) {
            const double u = 1.0 / max(sum_of(p.some, joins), 1);
            for (int i = threadIdx.x >> 6; i < 5; i += S::BLOCK / 64) {
                const double v = sum_of(p.part + (size_t)i * joins, joins);
                if ((threadIdx.x & 63) == 0)
                    a.stats[i] = (float)(v * u);
            }
            return;
        }
    }
    const int from = starts(0), to = starts(2LL * a.pairs);
    for (int k = blockIdx.x; k < chunks; k += groups) {
        const int begin = k * S::SIZE, end = end_of_chunk(begin, a.tokens);
        Sequences<S::BLOCK, kPairsLook> q(starts, 2 * a.pairs, begin, end);
        Mine m[S::PACKS];
#pragma unroll
        for (int h = 0; h < S::PACKS; h++)
            m[h] = my_tokens<S>(a.mask, begin, end, S::rank(h));
        marks.clear();
        __syncthreads();
        q.each([&](long long s, int s0, int) {
            const bool second = s >= a.pairs;
            const int at = max(s0, begin) - begin;
            const long long i = second ? s - a.pairs : s;
            double slope;
            int n;
            if constexpr (OWN) {
                slope = slope_of[i];
                n = n_of[second][i];
            } else {
                slope = p.slope[i];
                n = (int)p.sum.seq[s].n;
            }
            marks.at[at] = 1;
            seq[at] = pair_gradient(a, slope, second, n);
        });
        __syncthreads();
        store_gradients(a, m, from, to, marks, seq, of_all);
        __syncthreads();
    }
}

// Few tokens and pairs: all of the call in one workgroup (4001 tokens of 4 pairs 6.9 us, all
// of it latency).
template <class S>
__global__ __launch_bounds__(S::BLOCK) void preference_one(PreferenceArgs a)
{
    __shared__ Marks<S> marks;
    __shared__ CountTable<S> table;
    __shared__ Sums<S> sums;
    __shared__ double seq[S::SIZE];
    __shared__ double red[S::BLOCK / 64][6];
    __shared__ int counts[S::BLOCK / 64];
    const Starts starts{a.starts, a.tokens};
    Mine m[S::PACKS];
    double v[S::PACKS][S::EACH];
#pragma unroll
    for (int h = 0; h < S::PACKS; h++) {
        m[h] = my_tokens<S>(a.mask, 0, a.tokens, S::rank(h));
        load_ratios(a, m[h], v[h]);
        table.scan(h, m[h].mask);
    }
    const int from = starts(0), to = starts(2LL * a.pairs);
    // A thread a pair.
    const int i = threadIdx.x;
    const bool has = i < a.pairs;
    int s0[2], s1[2], n[2];
#pragma unroll
    for (int k = 0; k < 2; k++) {
        s0[k] = s1[k] = 0;
        if (has)
            starts.of(i + k * a.pairs, s0[k], s1[k]);
    }
    marks.clear();
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; k++)
        if (s0[k] < s1[k])
            mark_sequence(marks, s0[k], s1[k]);
    __syncthreads();
    sums.scan(marks, v);
    __syncthreads();
    double sum[6] = {0, 0, 0, 0, 0, 0}, slope = 0;
    if (has) {
        double r[2];
#pragma unroll
        for (int k = 0; k < 2; k++) {
            const bool some = s0[k] < s1[k];
            n[k] = some ? table.up_to(s1[k]) - table.up_to(s0[k]) : 0;
            r[k] = reward(a, some ? sums.at[s1[k] - 1] : 0.0, n[k]);
            if (a.rewards)
                a.rewards[i + k * a.pairs] = (float)r[k];
        }
        const Pair q = pair_loss(a, r[0], r[1]);
        slope = q.slope;
        if (n[0] + n[1] > 0) {
#pragma unroll
            for (int k = 0; k < 5; k++)
                sum[k] = q.stats[k];
            sum[5] = 1;
        }
    }
    // How many pairs have a token.
    const int given = __popcll(__ballot(sum[5] > 0));
    if ((threadIdx.x & 63) == 0)
        counts[threadIdx.x >> 6] = given;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < S::BLOCK / 64; w++)
        all += counts[w];
    const double u = 1.0 / max(all, 1);
    block_totals<S::BLOCK>(sum, red, [&](int k, double v) {
        if (k < 5)
            a.stats[k] = (float)(v * u);
    }, has);
    if (!a.dlogp)
        return;
#pragma unroll
    for (int k = 0; k < 2; k++)
        if (s0[k] < s1[k])
            seq[s0[k]] = pair_gradient(a, slope, k == 1, n[k]);
    __syncthreads();
    // Marks at the ends of sequences are the next one's beginning, or of tokens that
    // are in none.
    store_gradients(a, m, from, to, marks, seq, u);
}

// ---------------------------------------------------------------- launch rules
int chunks_of(long long tokens) { return (int)std::max(1LL, (tokens + kChunk - 1) / kChunk); }

// Lanes for a sequence: some two for each of its chunks, on an average, up to a wave (2 199
// 573 tokens of 58 pairs: 24.1 us, with one lane 60.4; 1 015 210 of 174 16.2 and 20.7).
int join_lanes(int chunks, long long seqs)
{
    int lanes = 1;
    while (lanes < 64 && lanes * seqs <= 2LL * chunks)
        lanes *= 2;
    return lanes;
}

// `lanes` lanes a sequence or pair.
int join_groups(long long n, int lanes)
{
    const long long all = n * lanes;
    return (int)std::max(1LL, std::min((all + kJoinBlock - 1) / kJoinBlock, (long long)kJoinGroups));
}

// So few sequences or pairs that every workgroup of the launch over the tokens joins all of
// them itself, which saves a launch: lanes for each, else 0; at least half of what a launch
// of their own would give them (158 508 tokens of 199 pairs 11.4 us, with that launch 13.7; 42
// 011 of a policy's 45 sequences 14.0 and 15.9; 2 468 375 of 79 pairs, by two lanes instead
// of 16, 34.6 and 24.2).
int own_lanes(long long n, int lanes)
{
    int own = 64;
    while (own * n > kOwn)
        own /= 2;
    return 2 * own < lanes ? 0 : own;
}

// One workgroup.
bool policy_is_small(long long tokens, long long seqs)
{
    return tokens <= Small::SIZE && seqs <= Small::SIZE;
}

// A thread a pair.
bool preference_is_small(long long tokens, long long pairs)
{
    return tokens <= Small::SIZE && pairs <= Small::BLOCK;
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
    c.part = a.take<double>(5 * std::min(chunks, kMaxGroups));
    c.n.seq = a.take<int>(seqs);
    c.n.head = a.take<int>(chunks);
    c.n.tail = a.take<int>(chunks);
    c.group = a.take<int>(kMaxGroups);
    c.some = a.take<int>(kJoinGroups);
    return a.used;
}

size_t layout(Pairs &p, void *ws, long long tokens, long long pairs)
{
    Arena a{(char *)ws};
    const int chunks = chunks_of(tokens);
    p.sum.seq = a.take<Piece>(2 * pairs);
    p.sum.head = a.take<Piece>(chunks);
    p.sum.tail = a.take<Piece>(chunks);
    p.slope = a.take<double>(pairs);
    p.part = a.take<double>(5 * kJoinGroups);
    p.some = a.take<int>(kJoinGroups);
    return a.used;
}

template <bool SEQS, bool OWN, Ref REF>
void policy_tokens(const PolicyArgs &a, const Counts *c, int groups, int joins, int lanes,
                   hipStream_t stream)
{
    if (c)
        policy_main<SEQS, OWN, REF>
            <<<groups, Narrow::BLOCK, 0, stream>>>(a, *c, chunks_of(a.tokens), joins, lanes);
    else if (a.tokens <= SmallPolicy::SIZE)
        policy_one<SmallPolicy, SEQS, REF><<<1, SmallPolicy::BLOCK, 0, stream>>>(a);
    else
        policy_one<Small, SEQS, REF><<<1, Small::BLOCK, 0, stream>>>(a);
}

// The launch over the tokens: by chunks, or (c null) of one workgroup.
template <bool SEQS, bool OWN>
void policy_tokens(const PolicyArgs &a, const Counts *c, int groups, int joins, int lanes,
                   hipStream_t stream)
{
    if (!a.ref_logp)
        policy_tokens<SEQS, OWN, Ref::none>(a, c, groups, joins, lanes, stream);
    else if (a.kl == 2)
        policy_tokens<SEQS, OWN, Ref::low>(a, c, groups, joins, lanes, stream);
    else
        policy_tokens<SEQS, OWN, Ref::other>(a, c, groups, joins, lanes, stream);
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
        (seqs ? policy_tokens<true, false>
              : policy_tokens<false, false>)(a, nullptr, 0, 0, 0, stream);
        return hipGetLastError();
    }
    Counts c;
    layout(c, a.ws, a.tokens, a.seqs);
    const int chunks = chunks_of(a.tokens), groups = std::min(chunks, kMaxGroups);
    const int lanes = a.mask ? join_lanes(chunks, a.seqs) : 1, joins = join_groups(a.seqs, lanes);
    const int own = a.mean == 1 ? own_lanes(a.seqs, lanes) : 0;
    if (a.mask && a.mean != 2)
        policy_count<<<groups, Narrow::BLOCK, 0, stream>>>(a, c, chunks);
    if (a.mean == 1 && !own)
        policy_join<<<joins, kJoinBlock, 0, stream>>>(a, c, lanes);
    (own    ? policy_tokens<true, true>
     : seqs ? policy_tokens<true, false>
            : policy_tokens<false, false>)(a, &c, groups, joins, own, stream);
    policy_stats<<<1, 5 * 64, 0, stream>>>(a, c.part, groups);
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
        if (a.tokens <= SmallPairs::SIZE && a.pairs <= SmallPairs::BLOCK)
            preference_one<SmallPairs><<<1, SmallPairs::BLOCK, 0, stream>>>(a);
        else
            preference_one<Small><<<1, Small::BLOCK, 0, stream>>>(a);
        return hipGetLastError();
    }
    Pairs p;
    layout(p, a.ws, a.tokens, a.pairs);
    const int chunks = chunks_of(a.tokens), groups = std::min(chunks, kMaxGroups);
    const int lanes = join_lanes(chunks, 2LL * a.pairs), joins = join_groups(a.pairs, lanes);
    preference_sums<<<groups, Wide::BLOCK, 0, stream>>>(a, p, chunks);
    const int own = own_lanes(a.pairs, lanes);
    if (!own)
        preference_pairs<<<joins, kJoinBlock, 0, stream>>>(a, p, lanes);
    const int n = (a.dlogp ? groups : 0) + 1;
    if (own)
        preference_fill<true><<<n, Wide::BLOCK, 0, stream>>>(a, p, chunks, joins, own);
    else
        preference_fill<false><<<n, Wide::BLOCK, 0, stream>>>(a, p, chunks, joins, own);
    return hipGetLastError();
}

}  // namespace miconv
