// Argument checks of the C ABI of include/mitrain.h and include/mistep.h.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "mitrain.h"
#include "internal.h"

namespace miconv {

inline constexpr long long kMaxRowElems = (1LL << 29) - 1;
inline constexpr long long kMaxRows = (1LL << 31) - 1;
inline constexpr long long kMaxSpan = 1LL << 48, kMaxAll = 1LL << 37;

inline bool known_type(int t) { return t == MITRAIN_F32 || t == MITRAIN_BF16 || t == MITRAIN_F16; }
inline size_t type_size(int t) { return t == MITRAIN_F32 ? 4 : 2; }

inline bool good_shape(long long rows, long long cols)
{
    return rows >= 0 && rows <= kMaxRows && cols >= 1 && cols <= kMaxRowElems &&
           rows * cols <= kMaxAll;
}

// A buffer of `rows` pieces of `bytes` bytes, `pitch` bytes apart.
struct Buffer {
    const void *p;
    long long rows, bytes, pitch;
    size_t align;
    bool written, required;
};

inline Buffer flat(const void *p, long long bytes, size_t align, bool written, bool required)
{
    return Buffer{p, 1, bytes, bytes, align, written, required};
}

inline bool overlap(const Buffer &a, const Buffer &b)
{
    if (!a.p || !b.p || !a.rows || !b.rows || !a.bytes || !b.bytes)
        return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    const uintptr_t a1 = a0 + (a.rows - 1) * a.pitch + a.bytes;
    const uintptr_t b1 = b0 + (b.rows - 1) * b.pitch + b.bytes;
    if (a1 <= b0 || b1 <= a0)
        return false;
    if (a.rows > 1 && b.rows > 1 && a.pitch == b.pitch) {
        // Columns of one wider matrix: apart if they are so modulo the pitch.
        const long long d = (long long)((b0 > a0 ? b0 - a0 : a0 - b0) % (uintptr_t)a.pitch);
        const long long ahead = b0 > a0 ? d : (a.pitch - d) % a.pitch;  // b after a
        return ahead < a.bytes || ahead + b.bytes > a.pitch;
    }
    return true;
}

// Null, alignment, workspace and aliasing checks, in that order.
inline int check(const Buffer *b, int n, const void *ws, size_t ws_bytes, size_t ws_need)
{
    for (int i = 0; i < n; i++)
        if (b[i].required && b[i].rows && !b[i].p)
            return MICONV_ERR_NULL;
    for (int i = 0; i < n; i++)
        if (b[i].p && (uintptr_t)b[i].p % b[i].align)
            return MICONV_ERR_ALIGN;
    if (ws_need) {
        if (!ws || ws_bytes < ws_need)
            return MICONV_ERR_WORKSPACE;
        if ((uintptr_t)ws % 16)
            return MICONV_ERR_ALIGN;
    }
    const Buffer w = flat(ws, (long long)ws_need, 16, true, false);
    for (int i = 0; i < n; i++) {
        if (overlap(b[i], w))
            return MICONV_ERR_ALIAS;
        for (int j = i + 1; j < n; j++)
            if ((b[i].written || b[j].written) && overlap(b[i], b[j]))
                return MICONV_ERR_ALIAS;
    }
    return MICONV_OK;
}

inline bool good_stride(long long rows, long long cols, long long ld)
{
    return ld >= cols && ld <= kMaxSpan && (rows <= 1 || ld <= kMaxSpan / rows);
}

inline Buffer rows_of(const void *p, long long rows, long long cols, long long ld, int type, bool written,
               bool required)
{
    const size_t s = type_size(type);
    return Buffer{p, rows, cols * (long long)s, ld * (long long)s, s, written, required};
}

inline int ready()
{
    const int st = check_device();
    if (st == MICONV_OK)
        (void)hipGetLastError();
    return st;
}

}  // namespace miconv
