// Argument block of the log-probability kernels (bs_log_probs.hip), shared with the host code that fills it (bs_log_probs.cpp).
#pragma once

#include <cstdint>

#include "brainslug.h"

namespace bs {

struct LogProbsK {
    const void *logits;
    const void *targets;  // int64 or int32; nullptr: no given classes
    float *logp, *entropy, *lse, *top_logp;
    int32_t *top_index;
    const float *grad_logp, *grad_entropy;  // backward only; nullptr: zero
    void *grad_logits;
    uint64_t rows, stride, grad_stride;  // strides: elements from a row to the next
    int64_t ignore_index;
    uint32_t classes, top, wide_targets;
};

bs_status launch_log_probs(const LogProbsK &k, int32_t dtype, void *stream);
bs_status launch_log_probs_backward(const LogProbsK &k, int32_t dtype, void *stream);

}  // namespace bs
