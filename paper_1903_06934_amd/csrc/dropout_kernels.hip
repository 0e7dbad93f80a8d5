// Dropout, forward and backward (include/mistep.h).
//
// Element e's 16 random bits are computed where they are used, eight elements at
// a time (random.h), and nothing of the mask is stored; both directions are one
// kernel.  Bound by memory: 16384 x 4096 bf16 43 us (6.2 TB/s; a copy of as many bytes
// takes 50), onto a residual 64.7; 12544 x 513 fp32 inside wider rows 12.1 (a copy 11.5).
// The generator's twenty 32 x 32 bit products for eight elements are what else it does:
// with 32 bits an element there would be twice as many, more than the memory hides.
// The figures at the rules are of whole calls replayed from a graph on three inputs in
// turn, both sides of a rule in one run.
#include <algorithm>
#include <initializer_list>

#include "internal.h"
#include "random.h"
#include "rows.h"
#include "step.h"

namespace miconv {

namespace {

// Packs in flight a thread: of eight 16-bit elements (16384 x 4096 bf16 43.6 us, of two
// packs 46.4), or of four 32-bit ones (12544 x 513 fp32 12.1 us, of four packs 13.6; 128 x
// 4096 2.8 and 3.5).
template <class T>
constexpr int kPacksOf = Pack<T>::N == 8 ? 1 : 2;

template <class T>
__device__ __forceinline__ T dropped(const Dropper &drop, T x, T residual, uint32_t word, int odd)
{
    const float v = drop.kept(word, odd) ? (float)x * drop.scale : 0.f;
    return (T)(v + (float)residual);
}

// The words of a thread's packs q[0 .. U).  A group of eight 32-bit elements is two
// packs, of neighbouring threads: of two packs each the even thread computes the first
// one's group, the odd one the second one's, and they exchange halves (16384 x 2048 fp32:
// 43.9 us, with two packs side by side a thread 77.5).  All threads of a wave call it.
template <class T>
__device__ __forceinline__ void words_of(const Dropper &drop, const long long (&q)[kPacksOf<T>],
                                         uint32_t (&w)[kPacksOf<T>][Pack<T>::N / 2])
{
    constexpr int U = kPacksOf<T>;
    if constexpr (Pack<T>::N == 8) {
#pragma unroll
        for (int u = 0; u < U; u++)
            drop.group((unsigned long long)q[u], w[u]);
    } else {
        const bool odd = threadIdx.x & 1;
#pragma unroll
        for (int u = 0; u < U; u += 2) {
            // Values, not places in arrays, to choose from: places go through memory.
            const long long first = q[u], second = q[u + 1];
            uint32_t g[4];
            drop.group((unsigned long long)(odd ? second : first) >> 1, g);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const uint32_t low = g[i], high = g[2 + i];
                const uint32_t got = __builtin_amdgcn_mov_dpp((int)(odd ? low : high), 0xb1, 0xf,
                                                              0xf, true);
                w[u][i] = odd ? got : low;
                w[u + 1][i] = odd ? high : got;
            }
        }
    }
}

// FLAT: the rows lie behind each other in all tensors, as one row of all elements.
// Otherwise a pack's elements may lie in several rows.
template <class T, bool FLAT, bool STREAM>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, long long packs)
{
    constexpr int N = Pack<T>::N, U = kPacksOf<T>;
    typedef typename Pack<T>::V V;
    typedef typename Pack<T>::At At;
    const Dropper drop(a.drop);
    const T *x = (const T *)a.x.p, *res = (const T *)a.residual.p;
    T *y = (T *)a.y.p;
    const long long n = a.rows * a.cols;
    const double inv = 1.0 / (double)a.cols;
    for (long long first = (long long)blockIdx.x * 256 * U; first < packs;
         first += (long long)gridDim.x * 256 * U) {
        V vx[U], vr[U];
        long long q[U], row[U], col[U];
        bool whole[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            q[u] = first + u * 256 + threadIdx.x;
            const long long e = q[u] * N;
            row[u] = 0;
            col[u] = e;
            if (!FLAT && q[u] < packs) {
                row[u] = (long long)((double)e * inv);  // off by one at most
                col[u] = e - row[u] * a.cols;
                if (col[u] < 0) {
                    row[u]--;
                    col[u] += a.cols;
                } else if (col[u] >= a.cols) {
                    row[u]++;
                    col[u] -= a.cols;
                }
            }
            whole[u] = q[u] < packs && (FLAT ? e + N <= n : col[u] + N <= a.cols);
            vx[u] = vr[u] = V{};
            if (whole[u]) {
                const At *px = (const At *)(x + row[u] * a.x.ld + col[u]);
                vx[u] = STREAM ? __builtin_nontemporal_load(px) : *px;
                if (res) {
                    const At *pr = (const At *)(res + row[u] * a.residual.ld + col[u]);
                    vr[u] = STREAM ? __builtin_nontemporal_load(pr) : *pr;
                }
            }
        }
        uint32_t w[U][N / 2] = {};
        if (drop.below)
            words_of<T>(drop, q, w);
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (whole[u]) {
                V v;
#pragma unroll
                for (int j = 0; j < N; j++)
                    v[j] = dropped<T>(drop, vx[u][j], vr[u][j], w[u][j / 2], j & 1);
                __builtin_nontemporal_store(v, (At *)(y + row[u] * a.y.ld + col[u]));
                continue;
            }
            // A pack that the row's end cuts, or the last: element by element, all loads
            // before the stores.
            const int left = (int)max(0LL, min((long long)N, n - q[u] * N));
            long long at_x[N], at_r[N], at_y[N], c = col[u];
            long long px = row[u] * a.x.ld + c, pr = row[u] * a.residual.ld + c,
                      py = row[u] * a.y.ld + c;
            T tx[N], tr[N];
#pragma unroll
            for (int j = 0; j < N; j++) {
                at_x[j] = px++;
                at_r[j] = pr++;
                at_y[j] = py++;
                if (!FLAT && ++c == a.cols) {
                    c = 0;
                    px += a.x.ld - a.cols;
                    pr += a.residual.ld - a.cols;
                    py += a.y.ld - a.cols;
                }
                tx[j] = tr[j] = (T)0.f;
                if (j < left)
                    tx[j] = x[at_x[j]];
            }
            if (res)
#pragma unroll
                for (int j = 0; j < N; j++)
                    if (j < left)
                        tr[j] = res[at_r[j]];
#pragma unroll
            for (int j = 0; j < N; j++)
                if (j < left)
                    y[at_y[j]] = dropped<T>(drop, tx[j], tr[j], w[u][j / 2], j & 1);
        }
    }
}

// Loads that leave nothing in the caches, for inputs larger than the last-level one
// holds beside the rest, of whole cache lines (16384 x 4096 bf16 onto a residual 64.7 us,
// without 68.8; 16384 x 2048 32.2 and 35.5, without a residual 23.2 and 22.9; 30001 x 2049,
// lines shared by rows, 85.7 and 78.3).
bool streams(const DropoutArgs &a, size_t elem)
{
    bool lines = a.rows * a.cols * (long long)elem * (a.residual.p ? 2 : 1) > 100LL << 20;
    for (const Rows &r : {a.x, a.residual})
        lines = lines && (uintptr_t)r.p % 128 == 0 && (!r.p || r.ld * elem % 128 == 0);
    return lines;
}

template <class T, bool FLAT>
void launch(const DropoutArgs &a, long long packs, bool stream_through, hipStream_t stream)
{
    const long long each = 256 * kPacksOf<T>;
    const int n = (int)std::min((packs + each - 1) / each, kMaxBlocks);
    if (stream_through)
        dropout_kernel<T, FLAT, true><<<n, 256, 0, stream>>>(a, packs);
    else
        dropout_kernel<T, FLAT, false><<<n, 256, 0, stream>>>(a, packs);
}

template <class T>
hipError_t launch(const DropoutArgs &a, hipStream_t stream)
{
    const long long packs = (a.rows * a.cols + Pack<T>::N - 1) / Pack<T>::N;
    if (!packs)
        return hipSuccess;
    const bool flat = a.rows <= 1 || (a.x.ld == a.cols && a.y.ld == a.cols &&
                                      (!a.residual.p || a.residual.ld == a.cols));
    const bool through = streams(a, sizeof(T));
    if (flat)
        launch<T, true>(a, packs, through, stream);
    else
        launch<T, false>(a, packs, through, stream);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int xtype, const DropoutArgs &a, hipStream_t stream)
{
    if (xtype == 0)
        return launch<float>(a, stream);
    return xtype == 1 ? launch<__bf16>(a, stream) : launch<_Float16>(a, stream);
}

}  // namespace miconv
