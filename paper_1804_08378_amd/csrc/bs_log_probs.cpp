// Log probabilities: argument checks and launches.  Nothing here synchronises or allocates.
#include "bs_log_probs.h"

#include <algorithm>

#include "bs_internal.h"

using namespace bs;

namespace {

bs_status check_desc(const bs_log_probs_desc *d)
{
    if (!d) return BS_ERR_NULL;
    if (d->dtype != BS_F32 && d->dtype != BS_BF16 && d->dtype != BS_F16) return BS_ERR_UNSUPPORTED;
    if (d->rows < 0 || d->classes < 1) return BS_ERR_SHAPE;
    if (d->classes > (1ll << 30) || d->rows > (1ll << 23)) return BS_ERR_UNSUPPORTED;
    if (d->top < 0 || d->top > BS_MAX_TOP || d->top > d->classes) return BS_ERR_PARAM;
    if (d->target_bytes != 4 && d->target_bytes != 8) return BS_ERR_PARAM;
    if (d->lse_bytes != 0 && d->lse_bytes != 4 && d->lse_bytes != 8) return BS_ERR_PARAM;
    for (const int64_t s : {d->row_stride, d->grad_row_stride})
        if (s != 0 && (s < d->classes || s > (1ll << 40))) return BS_ERR_SHAPE;
    return BS_OK;
}

void fill(const bs_log_probs_desc &d, LogProbsK &k)
{
    k.rows = (uint64_t)d.rows;
    k.classes = (uint32_t)d.classes;
    k.top = (uint32_t)d.top;
    k.stride = (uint64_t)(d.row_stride ? d.row_stride : d.classes);
    k.grad_stride = (uint64_t)(d.grad_row_stride ? d.grad_row_stride : d.classes);
    k.ignore_index = d.ignore_index;
    k.wide_targets = d.target_bytes == 8;
    k.wide_lse = d.lse_bytes == 8;
}

uint64_t lse_bytes(const LogProbsK &k) { return k.wide_lse ? 8 : 4; }

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// Parts of a row, a work-group each: at least `least` classes, `wanted` work-groups in all.
void split(LogProbsK &k, uint64_t least, uint64_t wanted)
{
    const uint64_t parts = std::max<uint64_t>(1, std::min({ceil_div(wanted, k.rows), ceil_div(k.classes, least), (uint64_t)K_LOG_PROBS_MOST_PARTS}));
    k.part = (uint32_t)(ceil_div(ceil_div(k.classes, parts), 8) * 8);
    k.parts = (uint32_t)ceil_div(k.classes, k.part);
}

struct Space {
    uint64_t keys = 0, sums = 0, bytes = 0;  // offsets, size
};
Space space(const LogProbsK &k)
{
    Space s;
    if (k.parts == 1) return s;
    s.sums = ceil_div(k.rows * k.parts * k.top * 8, 256) * 256;
    s.bytes = s.sums + k.rows * k.parts * 16;
    return s;
}

// Few long rows are cut into parts of at least 8 KiB and joined by a second launch, which costs 7 us: from 96 KiB a row on, up to 128 rows
// (bfloat16, 20 alternatives, whole rows and parts: 1x32768 11.1 and 13.0 us, 1x65536 14.6 and 13.0, 1x131072 22.0 and 13.2, 128x131072 23.8 and
// 21.1, 256x131072 26.2 and 26.5).
void fill_forward(const bs_log_probs_desc &d, LogProbsK &k)
{
    fill(d, k);
    const uint64_t es = dtype_size(d.dtype);
    const bool cut = k.rows <= 128 && k.classes * es >= (96 << 10);
    split(k, cut ? 8192 / es : k.classes, 256);
}

bool aligned(const void *p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

TensorBytes rows_of(const void *p, const LogProbsK &k, uint64_t stride, uint64_t es) { return TensorBytes{p, k.rows, k.classes * es, stride * es}; }
TensorBytes bytes_of(const void *p, uint64_t n) { return TensorBytes{p, 1, n, n}; }

template <size_t NI, size_t NO>
bs_status check_overlap(const TensorBytes (&in)[NI], const TensorBytes (&out)[NO])
{
    for (size_t i = 0; i < NO; ++i) {
        if (!out[i].p || !out[i].image_bytes) continue;
        for (const TensorBytes &t : in)
            if (t.p && tensors_overlap(out[i], t)) return BS_ERR_ALIAS;
        for (size_t j = 0; j < i; ++j)
            if (out[j].p && out[j].image_bytes && tensors_overlap(out[i], out[j])) return BS_ERR_ALIAS;
    }
    return BS_OK;
}

}  // namespace

extern "C" {

uint64_t bs_log_probs_workspace_bytes(const bs_log_probs_desc *desc)
{
    if (check_desc(desc) != BS_OK || desc->rows == 0) return 0;
    LogProbsK k{};
    fill_forward(*desc, k);
    return space(k).bytes;
}

bs_status bs_log_probs(const bs_log_probs_desc *desc, const void *logits, const void *targets, float *logp, float *entropy, void *lse,
                       float *top_logp, int32_t *top_index, void *workspace, uint64_t workspace_bytes, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!logits || (logp && !targets) || (desc->top && (!top_logp || !top_index))) return BS_ERR_NULL;
    LogProbsK k{};
    fill_forward(*desc, k);
    const Space room = space(k);
    const uint64_t es = dtype_size(desc->dtype);
    if (room.bytes && (!workspace || workspace_bytes < room.bytes)) return BS_ERR_WORKSPACE;
    if (!aligned(logits, es) || !aligned(targets, (uint64_t)desc->target_bytes) || !aligned(lse, lse_bytes(k)) || !aligned(workspace, 16)) return BS_ERR_ALIGN;
    for (const void *p : {(const void *)logp, (const void *)entropy, (const void *)top_logp, (const void *)top_index})
        if (!aligned(p, 4)) return BS_ERR_ALIGN;
    if (!desc->top) top_logp = nullptr, top_index = nullptr;
    const uint64_t n = k.rows * 4;
    const bs_status alias = check_overlap({rows_of(logits, k, k.stride, es), bytes_of(targets, k.rows * (uint64_t)desc->target_bytes)},
                                          {bytes_of(logp, n), bytes_of(entropy, n), bytes_of(lse, k.rows * lse_bytes(k)), bytes_of(top_logp, n * k.top), bytes_of(top_index, n * k.top),
                                           bytes_of(workspace, room.bytes)});
    if (alias != BS_OK) return alias;
    k.logits = logits;
    k.targets = targets;
    k.logp = logp;
    k.entropy = entropy;
    k.lse = lse;
    k.top_logp = top_logp;
    k.top_index = top_index;
    k.part_keys = reinterpret_cast<uint64_t *>(workspace);
    k.part_sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + room.sums);
    // a row that a wave reads in four vectors a lane needs no more of them
    return launch_log_probs(k, desc->dtype, k.classes * es <= 64 * 16 * 4 ? 64 : 256, stream);
}

bs_status bs_log_probs_backward(const bs_log_probs_desc *desc, const void *logits, const void *targets, const void *lse, const float *entropy,
                                const float *grad_logp, const float *grad_entropy, void *grad_logits, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!logits || !lse || !grad_logits || (grad_logp && !targets) || (grad_entropy && !entropy)) return BS_ERR_NULL;
    LogProbsK k{};
    fill(*desc, k);
    const uint64_t es = dtype_size(desc->dtype);
    if (!aligned(logits, es) || !aligned(grad_logits, es) || !aligned(targets, (uint64_t)desc->target_bytes) || !aligned(lse, lse_bytes(k))) return BS_ERR_ALIGN;
    for (const float *p : {entropy, grad_logp, grad_entropy})
        if (!aligned(p, 4)) return BS_ERR_ALIGN;
    const uint64_t n = k.rows * 4;
    // the gradient may take the logits' place: every element is read before it is written, by the same lane
    const bool in_place = grad_logits == logits && k.stride == k.grad_stride;
    const bs_status alias = check_overlap({in_place ? bytes_of(nullptr, 0) : rows_of(logits, k, k.stride, es), bytes_of(targets, k.rows * (uint64_t)desc->target_bytes),
                                           bytes_of(lse, k.rows * lse_bytes(k)), bytes_of(entropy, n), bytes_of(grad_logp, n), bytes_of(grad_entropy, n)},
                                          {rows_of(grad_logits, k, k.grad_stride, es)});
    if (alias != BS_OK) return alias;
    k.logits = logits;
    k.targets = grad_logp ? targets : nullptr;
    k.lse = const_cast<void *>(lse);
    k.entropy = const_cast<float *>(entropy);
    k.grad_logp = grad_logp;
    k.grad_entropy = grad_entropy;
    k.grad_logits = grad_logits;
    split(k, 8192, 2048);
    // 128-bit accesses on both sides need rows that stand alike in them
    const bool vectors = (reinterpret_cast<uintptr_t>(logits) - reinterpret_cast<uintptr_t>(grad_logits)) % 16 == 0 &&
                         (k.rows == 1 || (k.stride - k.grad_stride) * es % 16 == 0);
    return launch_log_probs_backward(k, desc->dtype, vectors, stream);
}

}  // extern "C"
