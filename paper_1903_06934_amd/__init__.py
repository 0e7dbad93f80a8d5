"""MI355X-native fp32 convolution training passes (forward, backward-data,
backward-weight) behind a C ABI (include/miconv.h), and the operators that
begin and end a training step around them (include/mitrain.h), with thin
bindings.  The library is loaded on first use; see ``miconv.lib``."""
from .miconv import (MiconvError, conv_bwd_data, conv_bwd_weight, conv_fwd, conv_tune, lib,
                     output_size, plan_clear, plan_count, plan_get, plan_name, plan_set,
                     plan_workspace_size, pool_bwd, pool_fwd, pool_output_size, workspace_size,
                     PASS_FWD, PASS_BWD_DATA, PASS_BWD_WEIGHT)
from .mitrain import (LogProbs, grad_clip, grad_norm, grad_workspace, layernorm_bwd,
                      layernorm_fwd, layernorm_workspace, logprob_bwd, logprob_fwd,
                      logprob_workspace)

__all__ = ["MiconvError", "conv_fwd", "conv_bwd_data", "conv_bwd_weight", "conv_tune", "lib",
           "output_size", "plan_clear", "plan_count", "plan_get", "plan_name", "plan_set",
           "plan_workspace_size", "pool_bwd", "pool_fwd", "pool_output_size", "workspace_size",
           "PASS_FWD", "PASS_BWD_DATA", "PASS_BWD_WEIGHT", "LogProbs", "grad_clip", "grad_norm",
           "grad_workspace", "layernorm_bwd", "layernorm_fwd", "layernorm_workspace",
           "logprob_bwd", "logprob_fwd", "logprob_workspace"]
