// Dropout, forward and backward (include/mistep.h).
//
// Element e's 16 random bits are computed where they are used, eight elements at
// a time (random.h), and nothing of the mask is stored; both directions are one
// kernel.
#include <algorithm>

#include "internal.h"
#include "random.h"
#include "rows.h"
#include "step.h"

namespace miconv {

namespace {

constexpr int kGroups = 2;  // of eight elements, in flight a thread

template <class T>
__device__ __forceinline__ T dropped(const Dropper &drop, T x, T residual, uint32_t word, int odd)
{
    const float v = drop.kept(word, odd) ? (float)x * drop.scale : 0.f;
    return (T)(v + (float)residual);
}

// FLAT: the rows lie behind each other in all tensors, as one row of all elements.
// Otherwise a group's eight elements may lie in several rows.
template <class T, bool FLAT>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, long long groups)
{
    constexpr int N = Pack<T>::N, K = 8 / N;  // packs a group
    typedef typename Pack<T>::V V;
    const Dropper drop(a.drop);
    const T *x = (const T *)a.x.p, *res = (const T *)a.residual.p;
    T *y = (T *)a.y.p;
    const long long n = a.rows * a.cols;
    const double inv = 1.0 / (double)a.cols;
    for (long long first = (long long)blockIdx.x * 256 * kGroups; first < groups;
         first += (long long)gridDim.x * 256 * kGroups) {
        V vx[kGroups][K], vr[kGroups][K];
        long long row[kGroups], col[kGroups];
        bool whole[kGroups];
#pragma unroll
        for (int u = 0; u < kGroups; u++) {
            const long long g = first + u * 256 + threadIdx.x, e = g * 8;
            row[u] = 0;
            col[u] = e;
            if (!FLAT && g < groups) {
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
            whole[u] = g < groups && (FLAT ? e + 8 <= n : col[u] + 8 <= a.cols);
#pragma unroll
            for (int k = 0; k < K; k++) {
                vx[u][k] = vr[u][k] = V{};
                if (whole[u]) {
                    vx[u][k] = *(const typename Pack<T>::At *)(x + row[u] * a.x.ld + col[u] + k * N);
                    if (res)
                        vr[u][k] = *(const typename Pack<T>::At *)(res + row[u] * a.residual.ld +
                                                                   col[u] + k * N);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kGroups; u++) {
            const long long g = first + u * 256 + threadIdx.x;
            if (g >= groups)
                continue;
            uint32_t w[4] = {0, 0, 0, 0};
            if (drop.below)
                drop.group((unsigned long long)g, w);
            if (whole[u]) {
#pragma unroll
                for (int k = 0; k < K; k++) {
                    V v;
#pragma unroll
                    for (int j = 0; j < N; j++)
                        v[j] = dropped<T>(drop, vx[u][k][j], vr[u][k][j], w[(k * N + j) / 2], j & 1);
                    __builtin_nontemporal_store(
                        v, (typename Pack<T>::At *)(y + row[u] * a.y.ld + col[u] + k * N));
                }
                continue;
            }
            long long r = row[u], c = col[u];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                if (g * 8 + j >= n)
                    break;
                if (!FLAT && c == a.cols) {
                    c = 0;
                    r++;
                }
                const T xj = x[r * a.x.ld + c];
                const T rj = res ? res[r * a.residual.ld + c] : (T)0.f;
                y[r * a.y.ld + c] = dropped<T>(drop, xj, rj, w[j / 2], j & 1);
                c++;
            }
        }
    }
}

template <class T>
hipError_t launch(const DropoutArgs &a, hipStream_t stream)
{
    const long long groups = (a.rows * a.cols + 7) / 8;
    if (!groups)
        return hipSuccess;
    const long long each = 256 * kGroups;
    const int n = (int)std::min((groups + each - 1) / each, kMaxBlocks);
    const bool flat = a.rows <= 1 || (a.x.ld == a.cols && a.y.ld == a.cols &&
                                      (!a.residual.p || a.residual.ld == a.cols));
    if (flat)
        dropout_kernel<T, true><<<n, 256, 0, stream>>>(a, groups);
    else
        dropout_kernel<T, false><<<n, 256, 0, stream>>>(a, groups);
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
