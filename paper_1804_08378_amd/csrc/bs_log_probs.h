// Argument block of the log-probability kernels (bs_log_probs.hip), shared with the host code that fills it (bs_log_probs.cpp).
#pragma once

#include <cstdint>

#include "brainslug.h"

namespace bs {

struct LogProbsK {
    const void *logits;
    const void *targets;  // int64 or int32; nullptr: no given classes
    float *logp, *entropy, *top_logp;
    void *lse;  // float or double (wide_lse)
    int32_t *top_index;
    const float *grad_logp, *grad_entropy;  // backward only; nullptr: zero
    void *grad_logits;
    uint64_t rows, stride, grad_stride;  // strides: elements from a row to the next
    int64_t ignore_index;
    uint32_t classes, top, wide_targets, wide_lse;
    uint32_t parts, part;  // work-groups of a row, classes of one (a multiple of 8)
    uint64_t *part_keys;   // workspace, rows x parts x top: the parts' best classes as numbers (rank_key)
    float *part_sums;      // workspace, rows x parts x 4: reference, sum, weighted sum, unused
};

constexpr uint32_t K_LOG_PROBS_MOST_PARTS = 256;

// threads: of a work-group, 64 or 256.  join: behind the parts' launch, one work-group a row.
bs_status launch_log_probs(const LogProbsK &k, int32_t dtype, int threads, void *stream);
bs_status launch_log_probs_backward(const LogProbsK &k, int32_t dtype, bool vectors, void *stream);

}  // namespace bs
