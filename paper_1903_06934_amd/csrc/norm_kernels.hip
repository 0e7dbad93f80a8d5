// Layer norm of rows, forward and backward (include/mitrain.h).
//
// Bound by memory: a row is read once and held in registers between its
// statistics and its result (16384 x 4096 bf16: forward 47 us, 5.7 TB/s; backward
// 80 us with the sums of dw and db, 5.0 TB/s, against the 5.3 of a large copy).
// Backward, about 17 instructions an element take nearly half of the time that
// the memory does, and the two overlap but in part.  Rows longer than
// what a workgroup is given to hold (32768 elements forward, 8192 backward), and
// long rows of which there are few, go by pieces and are read twice (32 x 100352
// fp32 backward: 15 us).  Calls of few rows are bound by
// launches and latencies (4 x 2048 bf16 forward: 3.4 us of kernel).
// The figures at the rules below are of whole calls replayed from a graph on
// three inputs in turn, both sides of a rule in one run: launches and their gaps
// (1.6 us and more) are in them.
#include <algorithm>
#include <initializer_list>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

// A pack that the row's end cuts short holds the elements that are left in
// halves: of 8 places the first four a half pack's (if four are left at least),
// the next two a quarter's, the seventh a single one.  Each is one load or store
// of whole registers; element by element two of 16 bits would meet in a register,
// for which the loads have to be waited for where they are issued, and all loads
// before them (16009 x 4369 f16 backward 129 us, element by element 188; forward
// 86 and 101).
// place: the element of place j in a pack of which `left` (>= 1) are left, or -1.
template <int N>
__device__ __forceinline__ int place(int j, int left)
{
    if (left >= N)
        return j;
#pragma unroll
    for (int h = N / 2, at = 0, from = 0; h; h /= 2) {
        if (j < at + h)
            return (left & h) ? from + j - at : -1;
        at += h;
        from += left & h;
    }
    return -1;
}

// Register parts of a pack, and as they lie in memory.
template <class T, int H>
struct Part {
    typedef T V __attribute__((ext_vector_type(H)));
    typedef V At __attribute__((aligned(sizeof(T))));
};

// The elements at p of which `left` (>= 1) are in the row, the others 0.
template <class T, bool STREAM = false>
__device__ __forceinline__ typename Pack<T>::V load_places(const T *p, int left)
{
    constexpr int N = Pack<T>::N;
    if (left >= N) {
        const auto *at = (const typename Pack<T>::At *)p;
        return STREAM ? __builtin_nontemporal_load(at) : *at;
    }
    uint32_t r[4] = {0, 0, 0, 0};
    if (left & (N / 2)) {
        const auto v = __builtin_bit_cast(uint2, *(const typename Part<T, N / 2>::At *)p);
        r[0] = v.x;
        r[1] = v.y;
        p += N / 2;
    }
    if constexpr (N == 8) {
        if (left & 2) {
            r[2] = __builtin_bit_cast(uint32_t, *(const typename Part<T, 2>::At *)p);
            p += 2;
        }
        if (left & 1)
            r[3] = __builtin_bit_cast(uint16_t, *p);
    } else if (left & 1) {
        r[2] = __builtin_bit_cast(uint32_t, *p);
    }
    return __builtin_bit_cast(typename Pack<T>::V, r);
}

template <class T>
__device__ __forceinline__ void store_places(T *p, int left, typename Pack<T>::V v)
{
    constexpr int N = Pack<T>::N;
    if (left >= N) {
        __builtin_nontemporal_store(v, (typename Pack<T>::At *)p);
        return;
    }
    if (left & (N / 2)) {
        if constexpr (N == 8)
            *(typename Part<T, 4>::At *)p = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        else
            *(typename Part<T, 2>::At *)p = __builtin_shufflevector(v, v, 0, 1);
        p += N / 2;
    }
    if constexpr (N == 8)
        if (left & 2) {
            *(typename Part<T, 2>::At *)p = __builtin_shufflevector(v, v, 4, 5);
            p += 2;
        }
    if (left & 1)
        *p = v[N - 2];
}

// The N weights at column c of a row of cols (`none` without weights).
template <int N, class TW>
__device__ __forceinline__ void load_weights(const TW *w, long long c, long long cols, float none,
                                             float *f)
{
#pragma unroll
    for (int j = 0; j < N; j++)
        f[j] = none;
    if (!w || c >= cols)
        return;
    if (c + N <= cols) {
        constexpr int K = Pack<TW>::N < N ? Pack<TW>::N : N;
#pragma unroll
        for (int i = 0; i < N; i += K) {
            typedef TW V __attribute__((ext_vector_type(K), aligned(sizeof(TW))));
            const V v = *(const V *)(w + c + i);
#pragma unroll
            for (int j = 0; j < K; j++)
                f[i + j] = (float)v[j];
        }
    } else {
        const int left = (int)(cols - c);
        const TW *p = w + c;
        int at = 0;
#pragma unroll
        for (int h = N / 2; h; at += h, h /= 2)
            if (left & h) {
#pragma unroll
                for (int j = 0; j < h; j++)
                    f[at + j] = (float)p[j];
                p += h;
            }
    }
}

// ------------------------------------------------------------ rows in registers
// The mean of a row is off by its sum's roundings, some 2^-19 of it.  Where the
// variance is no more than kNear of the mean's square (the elements differ by
// little, or not at all) the mean is corrected by the mean of the differences
// from it, and the variance taken again, less the square of what is left of
// these; so equal elements have that number as their mean and no variance.  The
// row is read again by elements, and summed one sum at a time: such rows take
// longer (16384 x 4096 bf16 of nothing else 134 us instead of 48), but all others
// keep the registers that they need (4000 x 16384 fp32: 105 us, with these sums
// taken from the packs 116).
constexpr float kNear = 0x1p-16f;

template <class T>
__device__ __forceinline__ void near_row(const T *x, int cols, int t, int tpr, float (*lds)[16],
                                         float &mean, float &var)
{
    const float n = (float)cols;
    float off = 0.f, d1 = 0.f, d2 = 0.f;
#pragma unroll 2
    for (int c = t; c < cols; c += tpr)
        off += (float)x[c] - mean;
    mean += group_reduce(off, tpr, lds[0], Add()) / n;
#pragma unroll 2
    for (int c = t; c < cols; c += tpr) {
        const float d = (float)x[c] - mean;
        d1 += d;
        d2 += d * d;
    }
    d1 = group_reduce(d1, tpr, lds[1], Add());
    d2 = group_reduce(d2, tpr, lds[2], Add());
    off = d1 / n;
    var = d2 / n;
    var -= off * off < var ? off * off : 0.f;
}

// A group of tpr threads (a power of two up to a wave, or a workgroup of some
// waves) holds a row: thread t the vectors t, t + tpr, ..., NV of them.
// The variance is taken about the mean, from the registers.  Groups take row
// after row; HOLD: with their weights and biases in registers.
// TAIL: all packs are whole, and beside them a thread holds one element of the
// row's last tpr places, some of which may be missing.
template <class T, class TW, int NV, bool TAIL, bool HOLD, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_fwd_rows(NormFwdArgs a, int tpr, bool stream)
{
    constexpr int N = Pack<T>::N;
    __shared__ float red[2][5][16];
    const TW *w = (const TW *)a.w, *b = (const TW *)a.b;
    const int cols = (int)a.cols;
    const int t = tpr > 64 ? threadIdx.x : threadIdx.x & (tpr - 1);
    const int groups = blockDim.x / tpr;
    const float n = (float)cols;
    const int last = NV * N * tpr + t;  // the column beside the packs
    float wv[HOLD ? NV : 1][N], bv[HOLD ? NV : 1][N], w1 = 1.f, b1 = 0.f;
    if constexpr (HOLD)
#pragma unroll
        for (int i = 0; i < NV; i++) {
            load_weights<N>(w, (t + i * tpr) * N, cols, 1.f, wv[i]);
            load_weights<N>(b, (t + i * tpr) * N, cols, 0.f, bv[i]);
        }
    if constexpr (TAIL) {
        load_weights<1>(w, last, cols, 1.f, &w1);
        load_weights<1>(b, last, cols, 0.f, &b1);
    }
    int turn = 0;
    for (long long row = (long long)blockIdx.x * groups + threadIdx.x / tpr; row < a.rows;
         row += (long long)gridDim.x * groups) {
        const T *xr = (const T *)a.x.p + row * a.x.ld;
        typename Pack<T>::V raw[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N;
            const int left = TAIL ? N : cols - c;
            raw[i] = typename Pack<T>::V{};
            if (left > 0) {
                if (stream)
                    raw[i] = load_places<T, true>(xr + c, left);
                else
                    raw[i] = load_places<T>(xr + c, left);
            }
        }
        const float x1 = TAIL && last < cols ? (float)xr[last] : 0.f;
        float s = x1;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++)
                s += (float)raw[i][j];
        float mean = group_reduce(s, tpr, red[turn][0], Add()) / n;
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int left = TAIL ? N : cols - (t + i * tpr) * N;
            if (left >= N) {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float d = (float)raw[i][j] - mean;
                    q += d * d;
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float d = (float)raw[i][j] - mean;
                    q += left > 0 && place<N>(j, left) >= 0 ? d * d : 0.f;
                }
            }
        }
        if (TAIL)
            q += last < cols ? (x1 - mean) * (x1 - mean) : 0.f;
        float var = group_reduce(q, tpr, red[turn][1], Add()) / n;
        if (__builtin_expect(var <= mean * mean * kNear && mean != 0.f && __builtin_isfinite(mean),
                             0))
            near_row(xr, cols, t, tpr, red[turn] + 2, mean, var);
        turn ^= 1;
        const float rstd = 1.f / sqrtf(var + a.eps);
        if (t == 0) {
            if (a.mean)
                a.mean[row] = mean;
            if (a.rstd)
                a.rstd[row] = rstd;
        }
        T *yr = (T *)a.y.p + row * a.y.ld;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N, h = HOLD ? i : 0;
            const int left = TAIL ? N : cols - c;
            if (left <= 0)
                continue;
            if constexpr (!HOLD) {
                load_weights<N>(w, c, cols, 1.f, wv[0]);
                load_weights<N>(b, c, cols, 0.f, bv[0]);
            }
            typename Pack<T>::V v;
#pragma unroll
            for (int j = 0; j < N; j++)
                v[j] = (T)(((float)raw[i][j] - mean) * rstd * wv[h][j] + bv[h][j]);
            store_places<T>(yr + c, left, v);
        }
        if (TAIL && last < cols)
            yr[last] = (T)((x1 - mean) * rstd * w1 + b1);
    }
}

// ------------------------------------------------------------------ long rows
// Count, mean and sum of squares about the mean of two sets of elements
// (Chan, Golub and LeVeque).
struct Moments {
    float n, mean, m2;
};

__device__ __forceinline__ Moments merge(Moments a, Moments b)
{
    const float n = a.n + b.n;
    if (b.n == 0.f)
        return a;
    if (a.n == 0.f)
        return b;
    const float d = b.mean - a.mean, f = b.n / n;
    const float mean = __builtin_isfinite(a.mean) ? a.mean + d * f : a.mean + b.mean;
    return Moments{n, mean, a.m2 + b.m2 + d * d * a.n * f};
}

__device__ __forceinline__ Moments wave_merge(Moments m)
{
    for (int o = 1; o < 64; o <<= 1) {
        Moments u{__shfl_xor(m.n, o), __shfl_xor(m.mean, o), __shfl_xor(m.m2, o)};
        // Both lanes merge in the same order: the lower lane's set first.
        m = (threadIdx.x & o) ? merge(u, m) : merge(m, u);
    }
    return m;
}

constexpr int kPieces = 64;
// Packs in flight a thread of norm_fwd_pieces (1000 x 100000 bf16: 130 us, with 4
// 136; 1 x 100000 11.5 and 13.9, with 1 10.5; 300 x 40000 fp32 31.3, 30.6 and 32.3).
constexpr int kFwdPacks = 2;

// Rows cut into `splits` (at most kPieces) pieces of `piece` elements (a multiple
// of a pack): the moments of each piece to ws[row][split].
template <class T>
__global__ __launch_bounds__(256) void norm_fwd_pieces(NormFwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N, F = kFwdPacks;
    __shared__ Moments part[4];
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const long long first = split * piece;
    const long long end = min(first + piece, a.cols);
    const T *x = (const T *)a.x.p + row * a.x.ld + first;
    const int len = (int)(end - first);
    Moments m{0.f, 0.f, 0.f};
    for (int c = threadIdx.x * N; c < len; c += F * 256 * N) {
        typename Pack<T>::V raw[F];
#pragma unroll
        for (int i = 0; i < F; i++) {
            const int at = c + i * 256 * N;
            raw[i] = typename Pack<T>::V{};
            if (at < len)
                raw[i] = load_places<T>(x + at, len - at);
        }
        // Equal elements have that number as their mean: sums of halves are exact
        // for them, and where places are missing the mean is corrected as above.
        float half[F * N], q = 0.f;
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int j = 0; j < N; j++)
                half[i * N + j] = (float)raw[i][j];
#pragma unroll
        for (int h = F * N / 2; h; h /= 2)
#pragma unroll
            for (int j = 0; j < h; j++)
                half[j] += half[j + h];
        const float s = half[0];
        if (c + ((F - 1) * 256 + 1) * N <= len) {
            const float mean = s * (1.f / (F * N));
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float d = (float)raw[i][j] - mean;
                    q += d * d;
                }
            m = merge(m, Moments{(float)(F * N), mean, q});
        } else {  // the last packs, of which some are short or missing
            int n = 0;
#pragma unroll
            for (int i = 0; i < F; i++)
                n += max(0, min(N, len - c - i * 256 * N));
            float mean = s / (float)n, off = 0.f;
            const auto in_row = [&](int i, int j) {
                const int left = len - c - i * 256 * N;
                return left > 0 && place<N>(j, left) >= 0;
            };
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int j = 0; j < N; j++)
                    off += in_row(i, j) ? (float)raw[i][j] - mean : 0.f;
            if (__builtin_isfinite(off))
                mean += off / (float)n;
#pragma unroll
            for (int i = 0; i < F; i++)
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float d = (float)raw[i][j] - mean;
                    q += in_row(i, j) ? d * d : 0.f;
                }
            m = merge(m, Moments{(float)n, mean, q});
        }
    }
    m = wave_merge(m);
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 4; i++)
            m = merge(m, part[i]);
        Moments *out = (Moments *)a.ws + row * splits + split;
        *out = m;
    }
}

// The pieces' results: every wave merges its row's moments (at most kPieces) and
// normalises its part of one piece.
template <class T, class TW>
__global__ __launch_bounds__(256) void norm_fwd_apply(NormFwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N, F = 2;
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const Moments *parts = (const Moments *)a.ws + row * splits;
    const int lane = threadIdx.x & 63;
    Moments m{0.f, 0.f, 0.f};
    if (lane < splits)
        m = parts[lane];
    m = wave_merge(m);
    const float mean = m.mean, rstd = 1.f / sqrtf(m.m2 / (float)a.cols + a.eps);
    if (split == 0 && threadIdx.x == 0) {
        if (a.mean)
            a.mean[row] = mean;
        if (a.rstd)
            a.rstd[row] = rstd;
    }
    const long long first = split * piece;
    const long long end = min(first + piece, a.cols);
    const int len = (int)(end - first);
    const T *x = (const T *)a.x.p + row * a.x.ld + first;
    T *y = (T *)a.y.p + row * a.y.ld + first;
    const TW *w = (const TW *)a.w, *b = (const TW *)a.b;
    for (int c0 = threadIdx.x * N; c0 < len; c0 += F * 256 * N) {
        typename Pack<T>::V raw[F];
        float wv[F][N], bv[F][N];
#pragma unroll
        for (int i = 0; i < F; i++) {
            const int c = c0 + i * 256 * N;
            raw[i] = typename Pack<T>::V{};
            if (c < len)
                raw[i] = load_places<T>(x + c, len - c);
            load_weights<N>(w, first + c, end, 1.f, wv[i]);
            load_weights<N>(b, first + c, end, 0.f, bv[i]);
        }
#pragma unroll
        for (int i = 0; i < F; i++) {
            const int c = c0 + i * 256 * N;
            if (c >= len)
                continue;
            typename Pack<T>::V v;
#pragma unroll
            for (int j = 0; j < N; j++)
                v[j] = (T)(((float)raw[i][j] - mean) * rstd * wv[i][j] + bv[i][j]);
            store_places<T>(y + c, len - c, v);
        }
    }
}

// -------------------------------------------------------------------- backward
// Rows in registers as forward, the next one's loads in flight while a row is
// worked on; a thread's columns are the same for all its rows, so it sums its
// columns' share of dw and db in registers over the rows of its group.  The
// groups of a workgroup meet in LDS, the workgroups in
// parts[workgroup][2][cols], or, if there is one only, it writes dw and db.
// Elements past the row's end are zeros in dy (and g u is summed as g (x - mean),
// whose zero times the finite -mean is 0).
template <class T, class TW, int NV, bool TAIL, int BLOCK>
__global__ __launch_bounds__(BLOCK) void norm_bwd_rows(NormBwdArgs a, int tpr, bool stream)
{
    constexpr int N = Pack<T>::N, K = NV * N + TAIL;  // elements a thread
    extern __shared__ float lds[];
    __shared__ float red[2][2][16];
    const int cols = (int)a.cols;
    const int t = tpr > 64 ? threadIdx.x : threadIdx.x & (tpr - 1);
    const int groups = blockDim.x / tpr, group = tpr > 64 ? 0 : threadIdx.x / tpr;
    const int last = NV * N * tpr + t;  // the column beside the packs
    const float inv_n = 1.f / (float)cols;
    float wv[K], sw[K], sb[K];
#pragma unroll
    for (int i = 0; i < NV; i++)
        load_weights<N>((const TW *)a.w, (t + i * tpr) * N, cols, 1.f, wv + i * N);
    if (TAIL)
        load_weights<1>((const TW *)a.w, last, cols, 1.f, wv + NV * N);
#pragma unroll
    for (int i = 0; i < K; i++)
        sw[i] = sb[i] = 0.f;
    typename Pack<T>::V rx[NV], rd[NV], nx[NV], nd[NV];
    T rx1 = (T)0.f, rd1 = (T)0.f, nx1 = (T)0.f, nd1 = (T)0.f;
    float mean = 0.f, rstd = 0.f, nmean = 0.f, nrstd = 0.f;
    const long long step = (long long)gridDim.x * groups;
    long long row = (long long)blockIdx.x * groups + group;
    // Where the row to load begins, and the row of dx to store.
    const T *xr = (const T *)a.x.p + row * a.x.ld, *dyr = (const T *)a.dy.p + row * a.dy.ld;
    T *dxr = (T *)a.dx.p + row * a.dx.ld;
    const float *meanr = a.mean + row, *rstdr = a.rstd + row;
    const long long x_step = step * a.x.ld, dy_step = step * a.dy.ld, dx_step = step * a.dx.ld;
    const auto load = [&](long long row) {
        if (row >= a.rows)
            return;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N;
            const int left = TAIL ? N : cols - c;
            nx[i] = nd[i] = typename Pack<T>::V{};
            if (left > 0) {
                if (stream) {
                    nx[i] = load_places<T, true>(xr + c, left);
                    nd[i] = load_places<T, true>(dyr + c, left);
                } else {
                    nx[i] = load_places<T>(xr + c, left);
                    nd[i] = load_places<T>(dyr + c, left);
                }
            }
        }
        if (TAIL && last < cols) {
            nx1 = xr[last];
            nd1 = dyr[last];
        }
        nmean = *meanr;
        nrstd = *rstdr;
        xr += x_step;
        dyr += dy_step;
        meanr += step;
        rstdr += step;
    };
    load(row);
    int turn = 0;
    for (; row < a.rows; row += step) {  // one row for the workgroup where it meets at the barrier
#pragma unroll
        for (int i = 0; i < NV; i++) {
            rx[i] = nx[i];
            rd[i] = nd[i];
        }
        rx1 = nx1;
        rd1 = nd1;
        mean = nmean;
        rstd = nrstd;
        load(row + step);
        float s1 = 0.f, s2 = 0.f;
        const auto sum = [&](int k, float d, float off) {
            const float g = d * wv[k];
            sw[k] += d * (off * rstd);
            sb[k] += d;
            s1 += g;
            s2 += g * off;
        };
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++)
                sum(i * N + j, (float)rd[i][j], (float)rx[i][j] - mean);
        if (TAIL)
            sum(NV * N, (float)rd1, (float)rx1 - mean);
        if (!a.dx.p)
            continue;
        s1 = wave_reduce(s1, tpr, Add());
        s2 = wave_reduce(s2, tpr, Add());
        if (tpr > 64) {
            if ((threadIdx.x & 63) == 0) {
                red[turn][0][threadIdx.x >> 6] = s1;
                red[turn][1][threadIdx.x >> 6] = s2;
            }
            __syncthreads();
            s1 = red[turn][0][0];
            s2 = red[turn][1][0];
            for (int v = 1; v < tpr >> 6; v++) {
                s1 += red[turn][0][v];
                s2 += red[turn][1][v];
            }
            turn ^= 1;
        }
        const float c1 = s1 * inv_n, c2 = s2 * rstd * inv_n;
        const auto result = [&](int k, T d, T x) {
            return (T)(rstd * ((float)d * wv[k] - c1 - ((float)x - mean) * rstd * c2));
        };
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N;
            const int left = TAIL ? N : cols - c;
            if (left <= 0)
                continue;
            typename Pack<T>::V v;
#pragma unroll
            for (int j = 0; j < N; j++)
                v[j] = result(i * N + j, rd[i][j], rx[i][j]);
            store_places<T>(dxr + c, left, v);
        }
        if (TAIL && last < cols)
            dxr[last] = result(NV * N, rd1, rx1);
        dxr += dx_step;
    }
    if (!a.dw && !a.db)
        return;
    float *part = a.ws + (size_t)blockIdx.x * 2 * cols;
    const auto put = [&](int k, int c, float v) {
        TW *out = (TW *)(k ? a.db : a.dw);
        if (gridDim.x > 1)
            part[(size_t)k * cols + c] = v;
        else if (out)
            out[c] = (TW)v;
    };
#pragma unroll
    for (int k = 0; k < 2; k++) {
        if (groups > 1)
            __syncthreads();
#pragma unroll
        for (int i = 0; i < K; i++) {
            int c = last;
            if (i < NV * N) {
                const int first = (t + i / N * tpr) * N;
                const int at = TAIL ? i % N : place<N>(i % N, max(1, cols - first));
                if (at < 0)
                    continue;
                c = first + at;
            }
            const float v = k ? sb[i] : sw[i];
            if (groups > 1)
                lds[group * tpr * K + c] = v;
            else if (c < cols)
                put(k, c, v);
        }
        if (groups == 1)
            continue;
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            float v = lds[c];
            for (int g = 1; g < groups; g++)
                v += lds[g * tpr * K + c];
            put(k, c, v);
        }
    }
}

// parts[n][2][cols] summed into dw and db: 32 columns a workgroup, its
// half-waves every 32nd part, eight loads in flight.
template <class TW>
__global__ __launch_bounds__(1024) void norm_bwd_sum(const float *parts, int n, long long cols,
                                                     TW *dw, TW *db)
{
    __shared__ float lds[32][33];
    const int k = blockIdx.y;
    TW *out = k ? db : dw;
    if (!out)
        return;
    const int lane = threadIdx.x & 31, half = threadIdx.x >> 5;
    const long long c = blockIdx.x * 32LL + lane;
    const float *in = parts + (size_t)k * cols + c;
    float s = 0.f;
    if (c < cols)
        for (int p = half; p < n; p += 256) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++)
                v[i] = p + 32 * i < n ? in[(size_t)(p + 32 * i) * 2 * cols] : 0.f;
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
    lds[half][lane] = s;
    __syncthreads();
    // Half-wave h of the transposed block: the 32 sums of column h.
    s = wave_reduce(lds[lane][half], 32, Add());
    const long long col = blockIdx.x * 32LL + half;
    if (lane == 0 && col < cols)
        out[col] = (TW)s;
}

// The same for few parts of many columns: a thread a column (187 x 35904 bf16, 7
// parts: 21.7 us in all, with half-waves 24.6).
constexpr int kFewParts = 32;

template <class TW>
__global__ __launch_bounds__(256) void norm_bwd_sum_few(const float *parts, int n, long long cols,
                                                        TW *dw, TW *db)
{
    const int k = blockIdx.y;
    TW *out = k ? db : dw;
    const long long c = blockIdx.x * 256LL + threadIdx.x;
    if (!out || c >= cols)
        return;
    const float *in = parts + (size_t)k * cols + c;
    float s = 0.f;
#pragma unroll 8
    for (int p = 0; p < n; p++)
        s += in[(size_t)p * 2 * cols];
    out[c] = (TW)s;
}

// Long rows: sums of g and g u of each piece to sums[row][split][2], four packs
// of x and dy in flight a thread.
template <class T, class TW>
__global__ __launch_bounds__(256) void norm_bwd_pieces(NormBwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N, F = 4;
    __shared__ float red[2][4];
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const long long first = split * piece;
    const long long end = min(first + piece, a.cols);
    const T *xr = (const T *)a.x.p + row * a.x.ld;
    const T *dyr = (const T *)a.dy.p + row * a.dy.ld;
    const TW *w = (const TW *)a.w;
    const float mean = a.mean[row], rstd = a.rstd[row];
    float s1 = 0.f, s2 = 0.f;
    const int len = (int)(end - first);
    for (int c0 = threadIdx.x * N; c0 < len; c0 += F * 256 * N) {
        typename Pack<T>::V rx[F], rd[F];  // zeros in dy past the end
        float wv[F][N];
#pragma unroll
        for (int i = 0; i < F; i++) {
            const int c = c0 + i * 256 * N;
            rx[i] = rd[i] = typename Pack<T>::V{};
            if (c < len) {
                rx[i] = load_places<T>(xr + first + c, len - c);
                rd[i] = load_places<T>(dyr + first + c, len - c);
            }
            load_weights<N>(w, first + c, end, 1.f, wv[i]);
        }
#pragma unroll
        for (int i = 0; i < F; i++)
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float g = (float)rd[i][j] * wv[i][j];
                s1 += g;
                s2 += g * ((float)rx[i][j] - mean);
            }
    }
    s1 = group_reduce(s1, 256, red[0], Add());
    s2 = group_reduce(s2, 256, red[1], Add()) * rstd;
    if (threadIdx.x == 0) {
        float *out = a.ws + ((size_t)row * splits + split) * 2;
        out[0] = s1;
        out[1] = s2;
    }
}

// Long rows: a workgroup owns 64 packs of columns and the chunk of rows
// blockIdx.y, of which its eight waves take every eighth: dx, and the columns'
// shares of dw and db, to parts[chunk][2][cols], or to dw and db if there is
// one chunk only.  The rows' sums are joined in LDS, kJoin rows at a time.
constexpr int kJoin = 64;

template <class T, class TW>
__global__ __launch_bounds__(512) void norm_bwd_cols(NormBwdArgs a, int splits, long long chunk,
                                                     float *parts)
{
    constexpr int N = Pack<T>::N, F = 2;
    __shared__ float lds[8][2][64 * N];
    __shared__ float join[kJoin][2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = ((long long)blockIdx.x * 64 + lane) * N;
    const long long end = min((long long)(blockIdx.y + 1) * chunk, a.rows);
    const int left = (int)max(0LL, min((long long)N, a.cols - c));
    const float inv_n = 1.f / (float)a.cols;
    float wv[N], sw[N], sb[N];
    load_weights<N>((const TW *)a.w, c, a.cols, 1.f, wv);
#pragma unroll
    for (int j = 0; j < N; j++)
        sw[j] = sb[j] = 0.f;
    for (long long base = blockIdx.y * chunk; base < end; base += kJoin) {
        const int here = (int)min((long long)kJoin, end - base);
        if (a.dx.p) {
            // Eight threads a row.
            const int r = threadIdx.x >> 3, part = threadIdx.x & 7;
            float s1 = 0.f, s2 = 0.f;
            if (r < here) {
                const float2 *sums = (const float2 *)a.ws + (size_t)(base + r) * splits;
                for (int i = part; i < splits; i += 8) {
                    const float2 v = sums[i];
                    s1 += v.x;
                    s2 += v.y;
                }
            }
            s1 = wave_reduce(s1, 8, Add());
            s2 = wave_reduce(s2, 8, Add());
            __syncthreads();
            if (part == 0) {
                join[r][0] = s1 * inv_n;
                join[r][1] = s2 * inv_n;
            }
            __syncthreads();
        }
        if (!left)
            continue;
        for (int r0 = wave; r0 < here; r0 += 8 * F) {
            typename Pack<T>::V rx[F], rd[F];
            float mean[F], rstd[F];
#pragma unroll
            for (int i = 0; i < F; i++) {
                const int r = r0 + 8 * i;
                rx[i] = rd[i] = typename Pack<T>::V{};
                mean[i] = rstd[i] = 0.f;
                if (r < here) {
                    const long long row = base + r;
                    mean[i] = a.mean[row];
                    rstd[i] = a.rstd[row];
                    rx[i] = load_places<T>((const T *)a.x.p + row * a.x.ld + c, left);
                    rd[i] = load_places<T>((const T *)a.dy.p + row * a.dy.ld + c, left);
                }
            }
#pragma unroll
            for (int i = 0; i < F; i++) {
                const int r = r0 + 8 * i;
                if (r >= here)
                    continue;
                const float s1 = a.dx.p ? join[r][0] : 0.f, s2 = a.dx.p ? join[r][1] : 0.f;
                typename Pack<T>::V v;
#pragma unroll
                for (int j = 0; j < N; j++) {
                    const float d = (float)rd[i][j];
                    const float u = ((float)rx[i][j] - mean[i]) * rstd[i];
                    sw[j] += d * u;
                    sb[j] += d;
                    v[j] = (T)(rstd[i] * (d * wv[j] - s1 - u * s2));
                }
                if (a.dx.p)
                    store_places<T>((T *)a.dx.p + (base + r) * a.dx.ld + c, left, v);
            }
        }
    }
    if (!a.dw && !a.db)
        return;
#pragma unroll
    for (int j = 0; j < N; j++) {
        const int at = place<N>(j, max(1, left));
        if (at < 0)
            continue;
        lds[wave][0][lane * N + at] = sw[j];
        lds[wave][1][lane * N + at] = sb[j];
    }
    __syncthreads();
    float *part = parts + (size_t)blockIdx.y * 2 * a.cols;
    for (int i = threadIdx.x; i < 2 * 64 * N; i += 512) {
        const int k = i / (64 * N), j = i - k * 64 * N;
        const long long col = (long long)blockIdx.x * 64 * N + j;
        if (col >= a.cols)
            continue;
        float s = lds[0][k][j];
#pragma unroll
        for (int v = 1; v < 8; v++)
            s += lds[v][k][j];
        TW *out = (TW *)(k ? a.db : a.dw);
        if (gridDim.y > 1)
            part[(size_t)k * a.cols + col] = s;
        else if (out)
            out[col] = (TW)s;
    }
}

// ----------------------------------------------------------------- launch rules
int pack_of(int xtype) { return xtype == 0 ? 4 : 8; }

size_t up16(size_t v) { return (v + 15) / 16 * 16; }

// A thread's elements of a row, at most: kValues with weights (and, backward,
// their gradients) in registers beside them; forward rows too long for that
// twice as many without.
constexpr int kValues = 16;

// Threads a row, packs a thread, threads a workgroup and the form of the last
// places of the register kernels; nv = 0: the row is too long for them.
struct RowPlan {
    int tpr, nv, block;
    bool tail;
};

RowPlan row_plan(int xtype, long long rows, long long cols, bool forward)
{
    const int n = pack_of(xtype);
    const long long packs = (cols + n - 1) / n;
    // Few rows above 16384 elements: by pieces over more CUs, which is faster in
    // the longest fp32 rows and about level else (16 x 32768 fp32 9.8 us, by
    // registers 11.8; bf16 9.8 and 9.6, 64 rows 10.5 and 9.8, 256 rows 17.9 and 12.0).
    if (forward && cols > 16384 && rows <= 64)
        return RowPlan{0, 0, 0, false};
    // Backward by pieces above 8192 elements (1024 threads have too few registers:
    // 4096 x 16384 fp32 285 us, by pieces 231; bf16 113 and 121), and where the
    // rows' partial sums of dw and db would be about as many as their elements:
    // up to 2048 rows from 4096 16-bit elements on (1040 x 4096 23.8 and 17.0, 4 x
    // 8192 14.8 and 8.5; 3100 x 8192 45.7 and 49.8), of 256 rows at least from 2048
    // on (520 x 2048 14.5 and 12.5; 60 x 2048 9.0 and 11.5), up to 512 rows from
    // 4096 fp32 elements on (260 x 8192 19.7 and 15.3; 1040 x 8192 30.5 and 36.0).
    const bool sums = n == 4 ? cols >= 4096 && rows <= 512
                             : rows <= 2048 && cols >= (rows < 256 ? 4096 : 2048);
    if (!forward && (cols > 8192 || sums))
        return RowPlan{0, 0, 0, false};
    if (packs <= 64) {
        int tpr = 1;
        while (packs > tpr)
            tpr *= 2;
        // Half the threads with an element more each where that holds the row
        // (30000 x 270 f16: forward 11.5 us instead of 17.7, backward 18.6 instead
        // of 22.9).
        const bool tail = tpr > 1 && cols <= tpr / 2 * (n + 1);
        return RowPlan{tail ? tpr / 2 : tpr, 1, 256, tail};
    }
    // As few idle places as can be; then more packs a thread before more
    // threads, as a row inside a wave needs no barrier.  Forward, few rows are
    // spread over more threads (4 x 2048 bf16: 5.4 us on 256 threads a row, 5.6 on
    // 128; 128 x 1000 fp32 5.4 and 5.6; 256 x 4096 fp32 6.5 and 6.2).
    const auto waves = [&](int nv) { return (packs + 64 * nv - 1) / (64 * nv); };
    const auto idle = [&](int nv) {
        const long long w = waves(nv);
        return w * nv + (!forward && (w == 2 || w == 3));  // small workgroups: many sums to join
    };
    const int most = forward ? 16 : 8;  // waves of a workgroup
    int best = 0;
    for (int nv = 1; nv * n <= kValues; nv++) {
        if (waves(nv) > most)
            continue;
        if (!best || (idle(nv) <= idle(best) && (!forward || rows * waves(nv) > 8LL * num_cus())))
            best = nv;
    }
    if (!best) {
        best = 2 * kValues / n;
        if (!forward || waves(best) > most)
            return RowPlan{0, 0, 0, false};
    }
    const int tpr = 64 * (int)waves(best);
    RowPlan p{tpr, best, tpr > 64 ? tpr : 256, false};
    if (forward && rows * waves(best) <= 8LL * num_cus())
        return p;
    // A row a little longer than whole packs of all its threads: one element a
    // thread beside them instead of a pack, where a thread then holds fewer places
    // and the row takes no more threads (forward 12544 x 1025 bf16 12.3 us, by packs
    // 19.2; 9000 x 3080 fp32 50.7 and 85.2; 4000 x 2049 fp32 14.9 and 14.8. Backward
    // 12544 x 513 fp32 21.1 and 22.8; 9000 x 3073 f16 55.2 and 58.3).  Not backward
    // over several waves in fp32 (9000 x 2049 55.6 and 50.1).
    int cost = tpr / 64 * best * n;
    for (int nv = 1; nv * n <= kValues; nv++)
        for (int w = 1; w <= (!forward && n == 4 ? 1 : tpr / 64); w++)
            if (64LL * w * nv * n <= cols && cols <= 64LL * w * (nv * n + 1) &&
                w * (nv * n + 1) < cost) {
                cost = w * (nv * n + 1);
                p = RowPlan{64 * w, nv, w > 1 ? 64 * w : 256, true};
            }
    return p;
}

// Workgroups of the register kernels.  Forward: 1536 threads a CU (16384 rows
// of 4096 bf16: 49.7 us; with 1024, 2048 and 4096 threads 52.9, 55.1 and 50.4).
int fwd_blocks(const RowPlan &p, long long rows)
{
    const long long groups = std::max(1, p.block / p.tpr);
    return (int)std::min((rows + groups - 1) / groups, 1536LL / p.block * num_cus());
}

// Backward: each workgroup adds 2 x cols partial sums to write and to read
// again, so 512 threads a CU (16384 x 4096 bf16: 83.4 us; with 768 and 1024
// 90.1 and 103.2); 1024 where a thread holds one pack, too little in flight,
// and takes at least five rows (31000 x 1500 bf16: 68.2 us instead of 94.1;
// 3000 x 1500, three rows: 24.6 instead of 18.6; with an element beside the pack
// 30000 x 300 fp32 26.8 instead of 24.7).  A single workgroup, which needs no sum
// after it, takes up to two rows a group (7 x 1024 bf16: 8.9 us instead of 9.9).
int bwd_blocks(const RowPlan &p, long long rows)
{
    const long long groups = std::max(1, p.block / p.tpr);
    if (rows <= 2 * groups)
        return 1;
    const auto blocks = [&](int threads) {
        return (long long)std::max(1, threads / p.block) * num_cus();
    };
    const bool more = p.nv == 1 && !p.tail && rows >= 5 * groups * blocks(1024);
    return (int)std::min((rows + groups - 1) / groups, blocks(more ? 1024 : 512));
}

// Loads that leave nothing in the caches, for inputs larger than the last-level
// one holds beside the rest (from 100 MB on: 16384 x 4096 bf16 49.3 us instead
// of 51.4 forward, 83.5 instead of 86.9 backward; 9000 x 4096 26.8, with them 29.6),
// of whole cache lines (16009 x 4369 bf16, lines shared by rows: 99.3 with them,
// 83.2 without).
bool streams(long long rows, long long cols, size_t elem, std::initializer_list<Rows> in)
{
    bool lines = rows * cols * (long long)elem > 100LL << 20;
    for (const Rows &r : in)
        lines = lines && (uintptr_t)r.p % 128 == 0 && r.ld * elem % 128 == 0;
    return lines;
}

// Pieces of long rows: forward as many as give every CU eight workgroups, of
// whole rounds of kFwdPacks packs, backward four, of at least 4096 elements (32 x
// 100352 fp32 16.9 us, with eight of 2048 17.7); at most kPieces a row.
struct PiecePlan {
    long long piece;
    int splits;
};

PiecePlan piece_plan(int xtype, long long rows, long long cols, bool forward)
{
    const long long per_cu = forward ? 8 : 4;
    const long long least = forward ? 256 * kFwdPacks * pack_of(xtype) : 4096;
    const long long unit = forward ? least : 2048;
    const long long want = std::max(1LL, per_cu * num_cus() / std::max(1LL, rows));
    const long long most = std::min((long long)kPieces, std::max(1LL, cols / least));
    const long long splits = std::min(want, most);
    const long long piece = ((cols + splits - 1) / splits + unit - 1) / unit * unit;
    return PiecePlan{piece, (int)((cols + piece - 1) / piece)};
}

// Chunks of rows of norm_bwd_cols: one up to 64 rows, which then needs no sum
// over the chunks; else as many as give every CU two workgroups, of 16 rows at
// least (169 x 25083 f16: 18.5 us, of 64 22.0).
int row_chunks(int xtype, long long rows, long long cols)
{
    const int n = pack_of(xtype);
    const long long tiles = (cols + 64 * n - 1) / (64 * n);
    const long long want = std::max(1LL, 2LL * num_cus() / tiles);
    return rows <= 64 ? 1 : (int)std::max(1LL, std::min(want, rows / 16));
}

template <class T, class TW, int NV, bool TAIL, bool HOLD>
void fwd_rows(const NormFwdArgs &a, const RowPlan &p, hipStream_t stream)
{
    const int n = fwd_blocks(p, a.rows);
    const bool through = streams(a.rows, a.cols, sizeof(T), {a.x});
    if (p.block <= 256)
        norm_fwd_rows<T, TW, NV, TAIL, HOLD, 256><<<n, p.block, 0, stream>>>(a, p.tpr, through);
    else
        norm_fwd_rows<T, TW, NV, TAIL, HOLD, 1024><<<n, p.block, 0, stream>>>(a, p.tpr, through);
}

template <class T, class TW, int NV>
void fwd_rows(const NormFwdArgs &a, const RowPlan &p, hipStream_t stream)
{
    if (p.tail)
        fwd_rows<T, TW, NV, true, true>(a, p, stream);
    else
        fwd_rows<T, TW, NV, false, true>(a, p, stream);
}

template <class T, class TW>
hipError_t fwd(int xtype, const NormFwdArgs &a, hipStream_t stream)
{
    constexpr int N = Pack<T>::N;
    if (!a.rows)
        return hipSuccess;
    const RowPlan p = row_plan(xtype, a.rows, a.cols, true);
    if (p.nv == 1)
        fwd_rows<T, TW, 1>(a, p, stream);
    else if (p.nv == 2)
        fwd_rows<T, TW, 2>(a, p, stream);
    else if (p.nv == 3 && N == 4)
        fwd_rows<T, TW, N == 4 ? 3 : 1>(a, p, stream);
    else if (p.nv == 4 && N == 4)
        fwd_rows<T, TW, kValues / N>(a, p, stream);
    else if (p.nv)
        fwd_rows<T, TW, 2 * kValues / N, false, false>(a, p, stream);
    if (p.nv)
        return hipGetLastError();
    // rows * cols is below 2^37 and a row above 2^15: below 2^23 workgroups.
    const PiecePlan s = piece_plan(xtype, a.rows, a.cols, true);
    const dim3 grid((unsigned)(a.rows * s.splits));
    norm_fwd_pieces<T><<<grid, 256, 0, stream>>>(a, s.piece, s.splits);
    norm_fwd_apply<T, TW><<<grid, 256, 0, stream>>>(a, s.piece, s.splits);
    return hipGetLastError();
}

template <class T, class TW, int NV, bool TAIL>
void bwd_rows(const NormBwdArgs &a, const RowPlan &p, int n, hipStream_t stream)
{
    const size_t lds =
        p.block > p.tpr ? (size_t)p.block * (NV * Pack<T>::N + TAIL) * sizeof(float) : 0;
    const bool through = streams(a.rows, a.cols, sizeof(T), {a.x, a.dy});
    if (p.block <= 256)
        norm_bwd_rows<T, TW, NV, TAIL, 256><<<n, p.block, lds, stream>>>(a, p.tpr, through);
    else
        norm_bwd_rows<T, TW, NV, TAIL, 512><<<n, p.block, lds, stream>>>(a, p.tpr, through);
}

template <class T, class TW, int NV>
void bwd_rows(const NormBwdArgs &a, const RowPlan &p, int n, hipStream_t stream)
{
    if (p.tail)
        bwd_rows<T, TW, NV, true>(a, p, n, stream);
    else
        bwd_rows<T, TW, NV, false>(a, p, n, stream);
}

template <class T, class TW>
hipError_t bwd(int xtype, const NormBwdArgs &a, hipStream_t stream)
{
    constexpr int N = Pack<T>::N;
    const RowPlan p = row_plan(xtype, a.rows, a.cols, false);
    const float *parts = a.ws;
    int n = 0;
    if (a.rows && p.nv) {
        n = bwd_blocks(p, a.rows);
        if (p.nv == 1)
            bwd_rows<T, TW, 1>(a, p, n, stream);
        else if (p.nv == 2)
            bwd_rows<T, TW, 2>(a, p, n, stream);
        else if (p.nv == 3)
            bwd_rows<T, TW, N == 4 ? 3 : 1>(a, p, n, stream);
        else
            bwd_rows<T, TW, kValues / N>(a, p, n, stream);
    } else if (a.rows) {
        const PiecePlan s = piece_plan(xtype, a.rows, a.cols, false);
        n = row_chunks(xtype, a.rows, a.cols);
        float *out = (float *)((char *)a.ws +
                               up16((size_t)a.rows * s.splits * 2 * sizeof(float)));
        parts = out;
        if (a.dx.p)
            norm_bwd_pieces<T, TW><<<(unsigned)(a.rows * s.splits), 256, 0, stream>>>(
                a, s.piece, s.splits);
        const dim3 grid((unsigned)((a.cols + 64 * N - 1) / (64 * N)), n);
        norm_bwd_cols<T, TW><<<grid, 512, 0, stream>>>(a, s.splits, (a.rows + n - 1) / n, out);
    }
    // One workgroup (or chunk) has written them itself; without rows they are 0.
    if (n != 1 && (a.dw || a.db)) {
        TW *dw = (TW *)a.dw, *db = (TW *)a.db;
        if (n <= kFewParts && a.cols >= 4096) {
            const dim3 grid((unsigned)((a.cols + 255) / 256), 2);
            norm_bwd_sum_few<TW><<<grid, 256, 0, stream>>>(parts, n, a.cols, dw, db);
        } else {
            const dim3 grid((unsigned)((a.cols + 31) / 32), 2);
            norm_bwd_sum<TW><<<grid, 1024, 0, stream>>>(parts, n, a.cols, dw, db);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t norm_fwd_ws(int xtype, long long rows, long long cols)
{
    if (row_plan(xtype, rows, cols, true).nv)
        return 0;
    return (size_t)rows * piece_plan(xtype, rows, cols, true).splits * sizeof(Moments);
}

size_t norm_bwd_ws(int xtype, long long rows, long long cols)
{
    const RowPlan p = row_plan(xtype, rows, cols, false);
    const size_t part = 2 * (size_t)cols * sizeof(float);
    if (!rows)
        return 0;
    if (p.nv)
        return bwd_blocks(p, rows) * part;
    const int n = row_chunks(xtype, rows, cols);  // one writes dw and db itself
    return up16((size_t)rows * piece_plan(xtype, rows, cols, false).splits * 2 * sizeof(float)) +
           (n > 1 ? n * part : 0);
}

hipError_t launch_norm_fwd(int xtype, bool w32, const NormFwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return fwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? fwd<__bf16, float>(xtype, a, stream) : fwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? fwd<_Float16, float>(xtype, a, stream)
               : fwd<_Float16, _Float16>(xtype, a, stream);
}

hipError_t launch_norm_bwd(int xtype, bool w32, const NormBwdArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return bwd<float, float>(xtype, a, stream);
    if (xtype == 1)
        return w32 ? bwd<__bf16, float>(xtype, a, stream) : bwd<__bf16, __bf16>(xtype, a, stream);
    return w32 ? bwd<_Float16, float>(xtype, a, stream)
               : bwd<_Float16, _Float16>(xtype, a, stream);
}

}  // namespace miconv
