// Launches of the operators of include/mistep.h (dropout_kernels.hip,
// residual_kernels.hip, loss_kernels.hip), called by step_api.hip with checked
// arguments.
#pragma once

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime.h>

#include "train.h"

namespace miconv {

// Which elements are dropped: those whose 16 bits are below `below`.
struct Drop {
    uint32_t below, key0, key1, step, layer;
    float scale;               // of what is kept
    const long long *step_at;  // may be null
};

struct DropoutArgs {
    long long rows, cols;
    Rows x, residual;  // residual.p may be null
    Rows y;            // written
    Drop drop;
};
hipError_t launch_dropout(int xtype, const DropoutArgs &a, hipStream_t stream);

// ------------------------------------------------------------ residual branches
// x of the base is the branch.
struct ResidualFwdArgs : NormFwdArgs {
    Rows residual;
    Rows total;   // written
    Drop drop;
};
// x of the base is total, dx the branch's gradient.
struct ResidualBwdArgs : NormBwdArgs {
    Rows dtotal;     // p may be null
    Rows dresidual;  // written; p may be null
    Drop drop;
};
hipError_t launch_residual_fwd(int xtype, bool w32, const ResidualFwdArgs &a, hipStream_t stream);
hipError_t launch_residual_bwd(int xtype, bool w32, const ResidualBwdArgs &a, hipStream_t stream);

// ---------------------------------------------------------------------- losses
struct PolicyArgs {
    int tokens, seqs;
    const float *logp, *old_logp, *ref_logp, *entropy, *advantages;
    int by_sequence;
    const unsigned char *mask;
    const long long *starts;
    double log_low, log_high, log_dual;  // where the log ratio is clipped
    float low, high, dual;               // the ratio there
    int kl;
    float kl_weight, entropy_weight;
    int mean;
    double count, scale;
    float *stats, *dlogp, *dentropy;
    void *ws;
};
size_t policy_ws(long long tokens, long long seqs);
hipError_t launch_policy(const PolicyArgs &a, hipStream_t stream);

struct PreferenceArgs {
    int tokens, pairs;
    const float *logp, *ref_logp;
    const unsigned char *mask;
    const long long *starts;
    double beta;
    int form;
    double smoothing, margin;
    int length_mean;
    double scale;
    float *stats, *rewards, *dlogp;
    void *ws;
};
size_t preference_ws(long long tokens, long long pairs);
hipError_t launch_preference(const PreferenceArgs &a, hipStream_t stream);

}  // namespace miconv
