// C ABI of the training step's operators (declared in include/mitrain.h):
// argument validation and launches on the caller's stream.
#include <algorithm>
#include <math.h>
#include <new>
#include <stddef.h>
#include <stdint.h>
#include <vector>

#include "mitrain.h"
#include "internal.h"
#include "train.h"

namespace miconv {

namespace {

constexpr long long kMaxRowElems = (1LL << 29) - 1;
constexpr long long kMaxRows = (1LL << 31) - 1;
constexpr long long kMaxSpan = 1LL << 48, kMaxAll = 1LL << 37;

bool known_type(int t) { return t == MITRAIN_F32 || t == MITRAIN_BF16 || t == MITRAIN_F16; }
size_t type_size(int t) { return t == MITRAIN_F32 ? 4 : 2; }

bool good_shape(long long rows, long long cols)
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

Buffer flat(const void *p, long long bytes, size_t align, bool written, bool required)
{
    return Buffer{p, 1, bytes, bytes, align, written, required};
}

bool overlap(const Buffer &a, const Buffer &b)
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
int check(const Buffer *b, int n, const void *ws, size_t ws_bytes, size_t ws_need)
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

bool good_stride(long long rows, long long cols, long long ld)
{
    return ld >= cols && ld <= kMaxSpan && (rows <= 1 || ld <= kMaxSpan / rows);
}

Buffer rows_of(const void *p, long long rows, long long cols, long long ld, int type, bool written,
               bool required)
{
    const size_t s = type_size(type);
    return Buffer{p, rows, cols * (long long)s, ld * (long long)s, s, written, required};
}

int ready()
{
    const int st = check_device();
    if (st == MICONV_OK)
        (void)hipGetLastError();
    return st;
}

// Types, counts and pointers of a list of gradients.
int check_list(int n, const void *const *grads, const long long *count, const int *types)
{
    if (n < 0)
        return MICONV_ERR_SHAPE;
    if (n && (!grads || !count || !types))
        return MICONV_ERR_NULL;
    long long left = kMaxAll;
    for (int i = 0; i < n; i++) {
        if (!known_type(types[i]))
            return MICONV_ERR_TYPE;
        if (count[i] < 0 || count[i] > left)
            return MICONV_ERR_SHAPE;
        left -= count[i];
    }
    for (int i = 0; i < n; i++) {
        if (count[i] && !grads[i])
            return MICONV_ERR_NULL;
        if ((uintptr_t)grads[i] % type_size(types[i]))
            return MICONV_ERR_ALIGN;
    }
    return MICONV_OK;
}

struct Span {
    uintptr_t first, end;
};

// Sorted by beginning (lists of tensors often are already).
void sort_spans(std::vector<Span> &s)
{
    const auto before = [](const Span &a, const Span &b) { return a.first < b.first; };
    if (!std::is_sorted(s.begin(), s.end(), before))
        std::sort(s.begin(), s.end(), before);
}

// Whether any two written spans overlap, or a written one and a read one.
bool any_overlap(std::vector<Span> &written, std::vector<Span> &read)
{
    sort_spans(written);
    sort_spans(read);
    uintptr_t written_end = 0, read_end = 0;  // the farthest ends of the spans so far
    size_t r = 0;
    for (const Span &w : written) {
        for (; r < read.size() && read[r].first < w.first; r++) {
            if (read[r].first < written_end)
                return true;
            read_end = std::max(read_end, read[r].end);
        }
        if (w.first < written_end || w.first < read_end)
            return true;
        written_end = w.end;
    }
    return r < read.size() && read[r].first < written_end;
}

int some_tensors(int n, const long long *count)
{
    int some = 0;
    for (int i = 0; i < n; i++)
        some += count[i] > 0;
    return some;
}

// The tensors with elements; false: more chunks than their numbers hold.
bool entries(int n, const void *const *grads, const long long *count, const int *types,
             void *const *out, std::vector<GradEntry> &e, unsigned *chunks)
{
    unsigned long long c = 0;
    e.reserve(n);
    for (int i = 0; i < n; i++) {
        if (!count[i])
            continue;
        e.push_back(GradEntry{grads[i], out ? out[i] : nullptr, count[i], (unsigned)c, types[i]});
        const long long most = kGradChunk / (long long)type_size(types[i]);
        c += (unsigned long long)((count[i] + most - 1) / most);
        if (c >> 31)
            return false;
    }
    *chunks = (unsigned)c;
    return true;
}

}  // namespace
}  // namespace miconv

using namespace miconv;

extern "C" {

size_t layernorm_fwd_workspace_size(int xtype, long long rows, long long cols)
{
    return known_type(xtype) && good_shape(rows, cols) ? norm_fwd_ws(xtype, rows, cols) : 0;
}

size_t layernorm_bwd_workspace_size(int xtype, long long rows, long long cols)
{
    return known_type(xtype) && good_shape(rows, cols) ? norm_bwd_ws(xtype, rows, cols) : 0;
}

int layernorm_fwd(int xtype, int wtype, long long rows, long long cols, const void *x,
                  long long ldx, const void *w, const void *b, float eps, void *y, long long ldy,
                  float *mean, float *rstd, void *ws, size_t ws_bytes, hipStream_t stream)
{
    if (!known_type(xtype) || (wtype != xtype && wtype != MITRAIN_F32))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, cols) || !good_stride(rows, cols, ldx) || !good_stride(rows, cols, ldy))
        return MICONV_ERR_SHAPE;
    if (!(eps >= 0) || !isfinite(eps))
        return MICONV_ERR_VALUE;
    const size_t wsize = type_size(wtype);
    const Buffer bufs[] = {
        rows_of(x, rows, cols, ldx, xtype, false, true),
        flat(w, cols * (long long)wsize, wsize, false, false),
        flat(b, cols * (long long)wsize, wsize, false, false),
        rows_of(y, rows, cols, ldy, xtype, true, true),
        flat(mean, rows * 4, 4, true, false),
        flat(rstd, rows * 4, 4, true, false),
    };
    int st = check(bufs, 6, ws, ws_bytes, norm_fwd_ws(xtype, rows, cols));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const NormFwdArgs a{rows, cols, {x, ldx}, w, b, eps, {y, ldy}, mean, rstd, (float *)ws};
    return launch_status(launch_norm_fwd(xtype, wtype == MITRAIN_F32, a, stream));
}

int layernorm_bwd(int xtype, int wtype, long long rows, long long cols, const void *dy,
                  long long lddy, const void *x, long long ldx, const float *mean,
                  const float *rstd, const void *w, void *dx, long long lddx, void *dw, void *db,
                  void *ws, size_t ws_bytes, hipStream_t stream)
{
    if (!known_type(xtype) || (wtype != xtype && wtype != MITRAIN_F32))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, cols) || !good_stride(rows, cols, ldx) ||
        !good_stride(rows, cols, lddy) || (dx && !good_stride(rows, cols, lddx)))
        return MICONV_ERR_SHAPE;
    if (!dx && !dw && !db)
        return MICONV_ERR_NULL;
    const size_t wsize = type_size(wtype);
    Buffer bufs[] = {
        rows_of(dy, rows, cols, lddy, xtype, false, true),
        rows_of(x, rows, cols, ldx, xtype, false, true),
        flat(mean, rows * 4, 4, false, rows > 0),
        flat(rstd, rows * 4, 4, false, rows > 0),
        flat(w, cols * (long long)wsize, wsize, false, false),
        rows_of(dx, rows, cols, lddx, xtype, true, false),
        flat(dw, cols * (long long)wsize, wsize, true, false),
        flat(db, cols * (long long)wsize, wsize, true, false),
    };
    int st = check(bufs, 8, ws, ws_bytes, norm_bwd_ws(xtype, rows, cols));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const NormBwdArgs a{rows, cols, {dy, lddy}, {x, ldx}, mean, rstd, w, {dx, lddx}, dw, db,
                        (float *)ws};
    return launch_status(launch_norm_bwd(xtype, wtype == MITRAIN_F32, a, stream));
}

size_t logprob_fwd_workspace_size(int xtype, long long rows, long long vocab, int top)
{
    if (!known_type(xtype) || !good_shape(rows, vocab) || top < 0 || top > MITRAIN_TOP_MAX ||
        top > vocab)
        return 0;
    return logprob_ws(xtype, rows, vocab, top);
}

int logprob_fwd(int xtype, long long rows, long long vocab, const void *logits, long long ldl,
                const long long *targets, float scale, int top, float *logp, float *lse,
                float *entropy, float *stats, float *top_logp, long long *top_index, void *ws, size_t ws_bytes,
                hipStream_t stream)
{
    if (!known_type(xtype))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, vocab) || !good_stride(rows, vocab, ldl) || top < 0 ||
        top > MITRAIN_TOP_MAX || top > vocab)
        return MICONV_ERR_SHAPE;
    if (!(scale >= 1e-6f && scale <= 1e6f))
        return MICONV_ERR_VALUE;
    const bool some = rows > 0;
    const Buffer bufs[] = {
        rows_of(logits, rows, vocab, ldl, xtype, false, true),
        flat(targets, rows * 8, 8, false, some && logp),
        flat(logp, rows * 4, 4, true, false),
        flat(lse, rows * 4, 4, true, false),
        flat(entropy, rows * 4, 4, true, false),
        flat(stats, rows * 8, 4, true, false),
        flat(top ? top_logp : nullptr, rows * top * 4, 4, true, some && top),
        flat(top ? top_index : nullptr, rows * top * 8, 8, true, some && top),
    };
    int st = check(bufs, 8, ws, ws_bytes, logprob_ws(xtype, rows, vocab, top));
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const LogprobArgs a{rows, vocab, {logits, ldl}, targets, scale, top, logp, lse, entropy,
                        stats, top_logp, top_index, ws};
    return launch_status(launch_logprob_fwd(xtype, a, stream));
}

int logprob_bwd(int xtype, long long rows, long long vocab, const void *logits, long long ldl,
                const long long *targets, float scale, const float *stats, const float *dlogp,
                const float *entropy, const float *dentropy, void *dlogits, long long ldd,
                hipStream_t stream)
{
    if (!known_type(xtype))
        return MICONV_ERR_TYPE;
    if (!good_shape(rows, vocab) || !good_stride(rows, vocab, ldl) ||
        !good_stride(rows, vocab, ldd))
        return MICONV_ERR_SHAPE;
    if (!(scale >= 1e-6f && scale <= 1e6f))
        return MICONV_ERR_VALUE;
    const bool some = rows > 0, in_place = dlogits == logits && ldd == ldl;
    const Buffer bufs[] = {
        rows_of(in_place ? nullptr : logits, rows, vocab, ldl, xtype, false, !in_place || !logits),
        flat(targets, rows * 8, 8, false, some && dlogp),
        flat(stats, rows * 8, 4, false, some),
        flat(dlogp, rows * 4, 4, false, some && !dentropy),
        flat(entropy, rows * 4, 4, false, some && dentropy),
        flat(dentropy, rows * 4, 4, false, false),
        rows_of(dlogits, rows, vocab, ldd, xtype, true, true),
    };
    int st = check(bufs, 7, nullptr, 0, 0);
    if (st != MICONV_OK || (st = ready()) != MICONV_OK)
        return st;
    const LogprobBwdArgs a{rows, vocab, {logits, ldl}, targets, scale, stats, dlogp, entropy,
                           dentropy, {dlogits, ldd}};
    return launch_status(launch_logprob_bwd(xtype, a, stream));
}

size_t grad_workspace_size(int n, const long long *count, const int *types)
{
    if (n <= 0 || !count || !types)
        return 0;
    const int some = some_tensors(n, count);
    return some ? clip_ws(some) : 0;
}

int grad_norm(int n, const void *const *grads, const long long *count, const int *types,
              float *norm, void *ws, size_t ws_bytes, hipStream_t stream)
{
    int st = check_list(n, grads, count, types);
    if (st != MICONV_OK)
        return st;
    const size_t need = grad_workspace_size(n, count, types);
    const Buffer out = flat(norm, 4, 4, true, true);
    if ((st = check(&out, 1, ws, ws_bytes, need)) != MICONV_OK)
        return st;
    const Buffer w = flat(ws, (long long)need, 16, true, false);
    for (int i = 0; i < n; i++) {
        const Buffer g = flat(grads[i], count[i] * (long long)type_size(types[i]), 1, false, false);
        if (overlap(g, out) || overlap(g, w))
            return MICONV_ERR_ALIAS;
    }
    try {
        std::vector<GradEntry> e;
        unsigned chunks = 0;
        if (!entries(n, grads, count, types, nullptr, e, &chunks))
            return MICONV_ERR_SHAPE;
        if ((st = ready()) != MICONV_OK)
            return st;
        return launch_status(
            launch_clip(e.data(), (int)e.size(), chunks, 0.f, false, norm, ws, stream));
    } catch (const std::bad_alloc &) {
        return MICONV_ERR_LAUNCH;
    }
}

int grad_clip(int n, const void *const *grads, const long long *count, const int *types,
              float max_norm, void *const *out, float *norm, void *ws, size_t ws_bytes,
              hipStream_t stream)
{
    int st = check_list(n, grads, count, types);
    if (st != MICONV_OK)
        return st;
    if (!(max_norm >= 0))
        return MICONV_ERR_VALUE;
    if (n && !out)
        return MICONV_ERR_NULL;
    for (int i = 0; i < n; i++) {
        if (count[i] && !out[i])
            return MICONV_ERR_NULL;
        if ((uintptr_t)out[i] % type_size(types[i]))
            return MICONV_ERR_ALIGN;
    }
    const size_t need = grad_workspace_size(n, count, types);
    const Buffer nb = flat(norm, 4, 4, true, false);
    if ((st = check(&nb, 1, ws, ws_bytes, need)) != MICONV_OK)
        return st;
    try {
        std::vector<GradEntry> e;
        unsigned chunks = 0;
        if (!entries(n, grads, count, types, out, e, &chunks))
            return MICONV_ERR_SHAPE;
        std::vector<Span> written, read;
        written.reserve(e.size() + 2);
        read.reserve(e.size());
        for (const GradEntry &g : e) {
            const uintptr_t bytes = (uintptr_t)g.count * type_size(g.type);
            written.push_back(Span{(uintptr_t)g.out, (uintptr_t)g.out + bytes});
            if (g.out != g.in)
                read.push_back(Span{(uintptr_t)g.in, (uintptr_t)g.in + bytes});
        }
        if (norm)
            written.push_back(Span{(uintptr_t)norm, (uintptr_t)norm + 4});
        if (need)
            written.push_back(Span{(uintptr_t)ws, (uintptr_t)ws + need});
        if (any_overlap(written, read))
            return MICONV_ERR_ALIAS;
        if ((st = ready()) != MICONV_OK)
            return st;
        return launch_status(
            launch_clip(e.data(), (int)e.size(), chunks, max_norm, true, norm, ws, stream));
    } catch (const std::bad_alloc &) {
        return MICONV_ERR_LAUNCH;
    }
}

}  // extern "C"
