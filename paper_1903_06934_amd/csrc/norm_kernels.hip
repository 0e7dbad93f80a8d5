// Layer norm of rows, forward and backward (include/mitrain.h).  Memory-bound:
// a row is read once and held in registers between its statistics and its
// result.
#include <algorithm>

#include "internal.h"
#include "rows.h"
#include "train.h"

namespace miconv {

namespace {

// ------------------------------------------------------------ rows in registers
// A group of tpr threads (a power of two: up to a wave, or the whole
// workgroup) holds a row: thread t the vectors t, t + tpr, ..., NV of them.
// The variance is taken about the mean, from the registers.
template <class T, class TW, int NV>
__global__ __launch_bounds__(1024) void norm_fwd_rows(NormFwdArgs a, int tpr)
{
    constexpr int N = Pack<T>::N;
    __shared__ float red[2][16];
    const T *x = (const T *)a.x.p;
    T *y = (T *)a.y.p;
    const TW *w = (const TW *)a.w, *b = (const TW *)a.b;
    const int cols = (int)a.cols;
    const int t = threadIdx.x & (tpr - 1);
    const long long row = (long long)blockIdx.x * (blockDim.x / tpr) + threadIdx.x / tpr;
    if (row >= a.rows)  // whole groups; a workgroup of one group has one row
        return;
    const T *xr = x + row * a.x.ld;
    typename Pack<T>::V raw[NV];
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = (t + i * tpr) * N;
        raw[i] = typename Pack<T>::V{};
        if (c < cols)
            raw[i] = load_pack<T>(xr + c, cols - c, (T)0.f);
    }
    const float n = (float)cols;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < N; j++)
            s += (float)raw[i][j];
    const float mean = group_reduce(s, tpr, red[0], Add()) / n;
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int left = cols - (t + i * tpr) * N;
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float d = (float)raw[i][j] - mean;
            q += j < left ? d * d : 0.f;
        }
    }
    const float var = group_reduce(q, tpr, red[1], Add()) / n;
    const float rstd = 1.f / sqrtf(var + a.eps);
    if (t == 0) {
        if (a.mean)
            a.mean[row] = mean;
        if (a.rstd)
            a.rstd[row] = rstd;
    }
    T *yr = y + row * a.y.ld;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = (t + i * tpr) * N;
        if (c >= cols)
            continue;
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++) {
            float f = ((float)raw[i][j] - mean) * rstd;
            if (c + j < cols) {
                if (w)
                    f *= (float)w[c + j];
                if (b)
                    f += (float)b[c + j];
            }
            v[j] = (T)f;
        }
        store_pack<T>(yr + c, cols - c, v);
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
    return Moments{n, a.mean + d * f, a.m2 + b.m2 + d * d * a.n * f};
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

// Rows cut into `splits` pieces of `piece` elements (a multiple of a pack):
// the moments of each piece to ws[row][split].
template <class T>
__global__ __launch_bounds__(256) void norm_fwd_pieces(NormFwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N;
    __shared__ Moments part[4];
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const long long first = split * piece;
    const long long end = min(first + piece, a.cols);
    const T *xr = (const T *)a.x.p + row * a.x.ld;
    Moments m{0.f, 0.f, 0.f};
    for (long long c = first + threadIdx.x * N; c < end; c += 256 * N) {
        const int left = (int)min((long long)N, end - c);
        const auto raw = load_pack<T>(xr + c, left, (T)0.f);
        float s = 0.f, q = 0.f;
#pragma unroll
        for (int j = 0; j < N; j++)
            s += (float)raw[j];
        const float mean = s / left;
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float d = (float)raw[j] - mean;
            q += j < left ? d * d : 0.f;
        }
        m = merge(m, Moments{(float)left, mean, q});
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

// The pieces' results: every workgroup merges its row's moments (in the order
// of the pieces) and normalises one piece.
template <class T, class TW>
__global__ __launch_bounds__(256) void norm_fwd_apply(NormFwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N;
    const long long row = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - row * splits);
    const Moments *parts = (const Moments *)a.ws + row * splits;
    Moments m = parts[0];
    for (int i = 1; i < splits; i++)
        m = merge(m, parts[i]);
    const float mean = m.mean, rstd = 1.f / sqrtf(m.m2 / (float)a.cols + a.eps);
    if (split == 0 && threadIdx.x == 0) {
        if (a.mean)
            a.mean[row] = mean;
        if (a.rstd)
            a.rstd[row] = rstd;
    }
    const long long first = split * piece;
    const long long end = min(first + piece, a.cols);
    const T *xr = (const T *)a.x.p + row * a.x.ld;
    T *yr = (T *)a.y.p + row * a.y.ld;
    const TW *w = (const TW *)a.w, *b = (const TW *)a.b;
    for (long long c = first + threadIdx.x * N; c < end; c += 256 * N) {
        const int left = (int)min((long long)N, end - c);
        const auto raw = load_pack<T>(xr + c, left, (T)0.f);
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++) {
            float f = ((float)raw[j] - mean) * rstd;
            if (j < left) {
                if (w)
                    f *= (float)w[c + j];
                if (b)
                    f += (float)b[c + j];
            }
            v[j] = (T)f;
        }
        store_pack<T>(yr + c, left, v);
    }
}

// -------------------------------------------------------------------- backward
// Rows in registers as forward; a thread's columns are the same for all its
// rows, so it sums its columns' share of dw and db in registers over the
// rows g, g + groups, ... of its group g.  The groups of a workgroup meet in
// LDS, the workgroups in parts[workgroup][2][cols].
template <class T, class TW, int NV>
__global__ __launch_bounds__(1024) void norm_bwd_rows(NormBwdArgs a, int tpr)
{
    constexpr int N = Pack<T>::N;
    extern __shared__ float lds[];
    __shared__ float red[2][2][16];
    const int cols = (int)a.cols;
    const int t = threadIdx.x & (tpr - 1), group = threadIdx.x / tpr;
    const int groups = blockDim.x / tpr;
    const TW *w = (const TW *)a.w;
    const float inv_n = 1.f / (float)cols;
    float wv[NV][N], sw[NV][N], sb[NV][N];
#pragma unroll
    for (int i = 0; i < NV; i++)
#pragma unroll
        for (int j = 0; j < N; j++) {
            const int c = (t + i * tpr) * N + j;
            wv[i][j] = c < cols ? (w ? (float)w[c] : 1.f) : 0.f;
            sw[i][j] = sb[i][j] = 0.f;
        }
    int turn = 0;
    for (long long row = (long long)blockIdx.x * groups + group; row < a.rows;
         row += (long long)gridDim.x * groups) {
        const T *xr = (const T *)a.x.p + row * a.x.ld;
        const T *dyr = (const T *)a.dy.p + row * a.dy.ld;
        typename Pack<T>::V rx[NV], rd[NV];
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N;
            rx[i] = rd[i] = typename Pack<T>::V{};
            if (c < cols) {
                rx[i] = load_pack<T>(xr + c, cols - c, (T)0.f);
                rd[i] = load_pack<T>(dyr + c, cols - c, (T)0.f);
            }
        }
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float d = (float)rd[i][j], u = ((float)rx[i][j] - mean) * rstd;
                sw[i][j] += d * u;
                sb[i][j] += d;
                s1 += d * wv[i][j];
                s2 += d * wv[i][j] * u;
            }
        if (!a.dx.p)
            continue;
        s1 = group_reduce(s1, tpr, red[turn][0], Add()) * inv_n;
        s2 = group_reduce(s2, tpr, red[turn][1], Add()) * inv_n;
        turn ^= 1;
        T *dxr = (T *)a.dx.p + row * a.dx.ld;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (t + i * tpr) * N;
            if (c >= cols)
                continue;
            typename Pack<T>::V v;
#pragma unroll
            for (int j = 0; j < N; j++) {
                const float d = (float)rd[i][j], u = ((float)rx[i][j] - mean) * rstd;
                v[j] = (T)(rstd * (d * wv[i][j] - s1 - u * s2));
            }
            store_pack<T>(dxr + c, cols - c, v);
        }
    }
    if (!a.dw && !a.db)
        return;
    float *part = a.ws + (size_t)blockIdx.x * 2 * cols;
#pragma unroll
    for (int k = 0; k < 2; k++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
            for (int j = 0; j < N; j++)
                lds[(group * tpr * NV + t + i * tpr) * N + j] = k ? sb[i][j] : sw[i][j];
        __syncthreads();
        for (int c = threadIdx.x; c < cols; c += blockDim.x) {
            float s = lds[c];
            for (int g = 1; g < groups; g++)
                s += lds[g * tpr * NV * N + c];
            part[(size_t)k * cols + c] = s;
        }
    }
}

// parts[n][2][cols] summed into dw and db: 64 columns a workgroup, each wave
// every fourth part.
template <class TW>
__global__ __launch_bounds__(256) void norm_bwd_sum(const float *parts, int n, long long cols,
                                                    TW *dw, TW *db)
{
    __shared__ float lds[4][64];
    const int k = blockIdx.y;
    TW *out = k ? db : dw;
    if (!out)
        return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = (long long)blockIdx.x * 64 + lane;
    float s = 0.f;
    if (c < cols)
        for (int p = wave; p < n; p += 4)
            s += parts[((size_t)p * 2 + k) * cols + c];
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < cols)
        out[c] = (TW)(lds[0][lane] + lds[1][lane] + (lds[2][lane] + lds[3][lane]));
}

// Long rows: sums of g and g u of each piece to sums[row][split][2].
template <class T, class TW>
__global__ __launch_bounds__(256) void norm_bwd_pieces(NormBwdArgs a, long long piece, int splits)
{
    constexpr int N = Pack<T>::N;
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
    for (long long c = first + threadIdx.x * N; c < end; c += 256 * N) {
        const int left = (int)min((long long)N, end - c);
        const auto rx = load_pack<T>(xr + c, left, (T)0.f);
        const auto rd = load_pack<T>(dyr + c, left, (T)0.f);
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float g = j < left ? (w ? (float)rd[j] * (float)w[c + j] : (float)rd[j]) : 0.f;
            s1 += g;
            s2 += j < left ? g * (((float)rx[j] - mean) * rstd) : 0.f;
        }
    }
    s1 = group_reduce(s1, 256, red[0], Add());
    s2 = group_reduce(s2, 256, red[1], Add());
    if (threadIdx.x == 0) {
        float *out = a.ws + ((size_t)row * splits + split) * 2;
        out[0] = s1;
        out[1] = s2;
    }
}

// Long rows: a workgroup owns 64 packs of columns, its waves rows of the
// chunk of rows blockIdx.y: dx, and the columns' shares of dw and db, to
// parts[chunk][2][cols].
template <class T, class TW>
__global__ __launch_bounds__(256) void norm_bwd_cols(NormBwdArgs a, int splits, long long chunk,
                                                     float *parts)
{
    constexpr int N = Pack<T>::N;
    __shared__ float lds[4][2][64 * N];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long c = ((long long)blockIdx.x * 64 + lane) * N;
    const long long end = min((long long)(blockIdx.y + 1) * chunk, a.rows);
    const int left = (int)max(0LL, min((long long)N, a.cols - c));
    const TW *w = (const TW *)a.w;
    const float inv_n = 1.f / (float)a.cols;
    float wv[N], sw[N], sb[N];
#pragma unroll
    for (int j = 0; j < N; j++) {
        wv[j] = j < left ? (w ? (float)w[c + j] : 1.f) : 0.f;
        sw[j] = sb[j] = 0.f;
    }
    for (long long row = blockIdx.y * chunk + wave; row < end; row += 4) {
        const float mean = a.mean[row], rstd = a.rstd[row];
        float s1 = 0.f, s2 = 0.f;
        if (a.dx.p) {
            const float *sums = a.ws + (size_t)row * splits * 2;
            for (int i = 0; i < splits; i++) {
                s1 += sums[2 * i];
                s2 += sums[2 * i + 1];
            }
            s1 *= inv_n;
            s2 *= inv_n;
        }
        if (!left)
            continue;
        const auto rx = load_pack<T>((const T *)a.x.p + row * a.x.ld + c, left, (T)0.f);
        const auto rd = load_pack<T>((const T *)a.dy.p + row * a.dy.ld + c, left, (T)0.f);
        typename Pack<T>::V v;
#pragma unroll
        for (int j = 0; j < N; j++) {
            const float d = (float)rd[j], u = ((float)rx[j] - mean) * rstd;
            sw[j] += d * u;
            sb[j] += d;
            v[j] = (T)(rstd * (d * wv[j] - s1 - u * s2));
        }
        if (a.dx.p)
            store_pack<T>((T *)a.dx.p + row * a.dx.ld + c, left, v);
    }
    if (!a.dw && !a.db)
        return;
#pragma unroll
    for (int j = 0; j < N; j++) {
        lds[wave][0][lane * N + j] = sw[j];
        lds[wave][1][lane * N + j] = sb[j];
    }
    __syncthreads();
    float *part = parts + (size_t)blockIdx.y * 2 * a.cols;
    for (int i = threadIdx.x; i < 2 * 64 * N; i += 256) {
        const int k = i / (64 * N), j = i - k * 64 * N;
        const long long col = (long long)blockIdx.x * 64 * N + j;
        if (col < a.cols)
            part[(size_t)k * a.cols + col] =
                lds[0][k][j] + lds[1][k][j] + (lds[2][k][j] + lds[3][k][j]);
    }
}

// ----------------------------------------------------------------- launch rules
int elem_size(int xtype) { return xtype == 0 ? 4 : 2; }

size_t up16(size_t v) { return (v + 15) / 16 * 16; }

// Threads a row and packs a thread of the register kernels; nv = 0: the row
// is too long for them.
struct RowPlan {
    int tpr, nv, block;
};

RowPlan row_plan(int xtype, long long cols, int max_values)
{
    const int n = 16 / elem_size(xtype);
    const long long packs = (cols + n - 1) / n;
    int tpr = 1;
    while (tpr < 1024 && packs > tpr)
        tpr *= 2;
    // Up to a wave, one pack a thread; then more packs a thread before more
    // threads, as a row inside a wave needs no barrier.
    int nv = 1;
    while (tpr > 64 && nv * 2 * n <= max_values) {
        tpr /= 2;
        nv *= 2;
    }
    if (tpr > 1024 || (long long)tpr * nv < packs) {
        tpr = 1024;
        nv = 1;
        while (nv * n < max_values && (long long)tpr * nv < packs)
            nv *= 2;
        if ((long long)tpr * nv < packs)
            return RowPlan{0, 0, 0};
    }
    return RowPlan{tpr, nv, tpr > 64 ? tpr : 256};
}

constexpr int kFwdValues = 32, kBwdValues = 16;  // a thread's elements of a row, at most

// Pieces of long rows: as many as give every CU four workgroups, of at least
// 4096 elements, at most 64 a row.
struct PiecePlan {
    long long piece;
    int splits;
};

PiecePlan piece_plan(long long rows, long long cols)
{
    const long long want = std::max(1LL, 4LL * num_cus() / std::max(1LL, rows));
    const long long most = std::min(64LL, std::max(1LL, cols / 4096));
    const long long splits = std::min(want, most);
    const long long piece = ((cols + splits - 1) / splits + 2047) / 2048 * 2048;
    return PiecePlan{piece, (int)((cols + piece - 1) / piece)};
}

int bwd_blocks(const RowPlan &p, long long rows)
{
    const long long groups = p.block / p.tpr;
    return (int)std::min((rows + groups - 1) / groups, 2LL * num_cus());
}

// Chunks of rows of norm_bwd_cols.
int row_chunks(int xtype, long long rows, long long cols)
{
    const int n = 16 / elem_size(xtype);
    const long long tiles = (cols + 64 * n - 1) / (64 * n);
    const long long want = std::max(1LL, 4LL * num_cus() / tiles);
    return (int)std::max(1LL, std::min(want, (rows + 15) / 16));
}

template <class T, class TW>
hipError_t fwd(int xtype, const NormFwdArgs &a, hipStream_t stream)
{
    const RowPlan p = row_plan(xtype, a.cols, kFwdValues);
    if (p.nv) {
        const long long groups = p.block / p.tpr, most = kMaxBlocks * groups;
        for (long long first = 0; first < a.rows; first += most) {
            NormFwdArgs c = a;  // the rows of this launch
            c.rows = std::min(most, a.rows - first);
            c.x.p = (const T *)a.x.p + first * a.x.ld;
            c.y.p = (const T *)a.y.p + first * a.y.ld;
            c.mean = a.mean ? a.mean + first : nullptr;
            c.rstd = a.rstd ? a.rstd + first : nullptr;
            const dim3 grid((unsigned)((c.rows + groups - 1) / groups));
            switch (p.nv) {
            case 1: norm_fwd_rows<T, TW, 1><<<grid, p.block, 0, stream>>>(c, p.tpr); break;
            case 2: norm_fwd_rows<T, TW, 2><<<grid, p.block, 0, stream>>>(c, p.tpr); break;
            case 4: norm_fwd_rows<T, TW, 4><<<grid, p.block, 0, stream>>>(c, p.tpr); break;
            default:
                norm_fwd_rows<T, TW, kFwdValues / Pack<T>::N>
                    <<<grid, p.block, 0, stream>>>(c, p.tpr);
                break;
            }
        }
        return hipGetLastError();
    }
    if (!a.rows)
        return hipSuccess;
    // rows * cols is below 2^37 and a row above 2^15: below 2^23 workgroups.
    const PiecePlan s = piece_plan(a.rows, a.cols);
    const dim3 grid((unsigned)(a.rows * s.splits));
    norm_fwd_pieces<T><<<grid, 256, 0, stream>>>(a, s.piece, s.splits);
    norm_fwd_apply<T, TW><<<grid, 256, 0, stream>>>(a, s.piece, s.splits);
    return hipGetLastError();
}

template <class T, class TW>
hipError_t bwd(int xtype, const NormBwdArgs &a, hipStream_t stream)
{
    const RowPlan p = row_plan(xtype, a.cols, kBwdValues);
    const bool params = a.dw || a.db;
    const float *parts;
    int n;
    if (p.nv) {
        constexpr int N = Pack<T>::N;
        n = bwd_blocks(p, a.rows);
        parts = a.ws;
        if (n) {
            const size_t lds = params ? (size_t)p.block * p.nv * N * sizeof(float) : 0;
            switch (p.nv) {
            case 1: norm_bwd_rows<T, TW, 1><<<n, p.block, lds, stream>>>(a, p.tpr); break;
            case 2: norm_bwd_rows<T, TW, 2><<<n, p.block, lds, stream>>>(a, p.tpr); break;
            default:
                norm_bwd_rows<T, TW, 16 / N><<<n, p.block, lds, stream>>>(a, p.tpr);
                break;
            }
        }
    } else {
        const PiecePlan s = piece_plan(a.rows, a.cols);
        n = a.rows ? row_chunks(xtype, a.rows, a.cols) : 0;
        const size_t sums = up16((size_t)a.rows * s.splits * 2 * sizeof(float));
        float *out = (float *)((char *)a.ws + sums);
        parts = out;
        if (a.rows && a.dx.p)
            norm_bwd_pieces<T, TW><<<(unsigned)(a.rows * s.splits), 256, 0, stream>>>(
                a, s.piece, s.splits);
        if (a.rows) {
            const long long cols_wg = 64 * Pack<T>::N;
            const dim3 grid((unsigned)((a.cols + cols_wg - 1) / cols_wg), n);
            const long long chunk = (a.rows + n - 1) / n;
            norm_bwd_cols<T, TW><<<grid, 256, 0, stream>>>(a, s.splits, chunk, out);
        }
    }
    if (params) {
        const dim3 grid((unsigned)((a.cols + 63) / 64), 2);
        norm_bwd_sum<TW><<<grid, 256, 0, stream>>>(parts, n, a.cols, (TW *)a.dw, (TW *)a.db);
    }
    return hipGetLastError();
}

}  // namespace

size_t norm_fwd_ws(int xtype, long long rows, long long cols)
{
    if (row_plan(xtype, cols, kFwdValues).nv)
        return 0;
    return (size_t)rows * piece_plan(rows, cols).splits * sizeof(Moments);
}

size_t norm_bwd_ws(int xtype, long long rows, long long cols)
{
    const RowPlan p = row_plan(xtype, cols, kBwdValues);
    if (p.nv)
        return (size_t)bwd_blocks(p, rows) * 2 * cols * sizeof(float);
    return up16((size_t)rows * piece_plan(rows, cols).splits * 2 * sizeof(float)) +
           (size_t)row_chunks(xtype, rows, cols) * 2 * cols * sizeof(float);
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
