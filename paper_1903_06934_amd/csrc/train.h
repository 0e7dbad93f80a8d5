// Launches of the operators of include/mitrain.h (norm_kernels.hip,
// logprob_kernels.hip, clip_kernels.hip), called by train_api.hip with checked
// arguments.
#pragma once

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime.h>

namespace miconv {

// A tensor of rows: row r begins at element r * ld of p.
struct Rows {
    const void *p;
    long long ld;
};

// ---------------------------------------------------------------- layer norm
struct NormFwdArgs {
    long long rows, cols;
    Rows x;
    const void *w, *b;  // may be null
    float eps;
    Rows y;             // written
    float *mean, *rstd; // may be null
    float *ws;
};
struct NormBwdArgs {
    long long rows, cols;
    Rows dy, x;
    const float *mean, *rstd;
    const void *w;      // may be null
    Rows dx;            // written; p may be null
    void *dw, *db;      // may be null
    float *ws;
};
size_t norm_fwd_ws(int xtype, long long rows, long long cols);
size_t norm_bwd_ws(int xtype, long long rows, long long cols);
hipError_t launch_norm_fwd(int xtype, bool w32, const NormFwdArgs &a, hipStream_t stream);
hipError_t launch_norm_bwd(int xtype, bool w32, const NormBwdArgs &a, hipStream_t stream);

// --------------------------------------------------------- log probabilities
struct LogprobArgs {
    long long rows, vocab;
    Rows logits;
    const long long *targets;
    float scale;
    int top;
    float *logp, *lse, *entropy, *stats, *top_logp;
    long long *top_index;
    void *ws;
};
struct LogprobBwdArgs {
    long long rows, vocab;
    Rows logits;
    const long long *targets;
    float scale;
    const float *stats, *dlogp, *entropy, *dentropy;
    Rows dlogits;       // written
};
size_t logprob_ws(int xtype, long long rows, long long vocab, int top);
hipError_t launch_logprob_fwd(int xtype, const LogprobArgs &a, hipStream_t stream);
hipError_t launch_logprob_bwd(int xtype, const LogprobBwdArgs &a, hipStream_t stream);

// ------------------------------------------------------------------ clipping
constexpr int kGradChunk = 16384;  // bytes of a tensor that a workgroup takes at once
// A tensor with elements; first: the chunks of the tensors before it.
struct GradEntry {
    const void *in;
    void *out;
    long long count;
    unsigned first;
    int type;
};
size_t clip_ws(int n);
// The norm of n tensors, and if scale is set their clipping.
hipError_t launch_clip(const GradEntry *e, int n, unsigned chunks, float max_norm, bool scale,
                       float *norm, void *ws, hipStream_t stream);

}  // namespace miconv
