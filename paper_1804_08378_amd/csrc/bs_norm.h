// Argument blocks of the group-normalisation kernels (bs_norm.hip), shared with the host code that fills them (bs_norm.cpp).
#pragma once

#include <cstdint>

#include "brainslug.h"

namespace bs {

constexpr int K_NORM_THREADS = 256;        // work-group size of every kernel here
constexpr int K_NORM_BLOCK_CHANNELS = 256; // channels of a work-group at most: a lane keeps one vector of them

// One tensor: N images of P pixels, `stride` elements from a pixel to the next (C where dense).
struct NormTensor {
    const void *p;
    uint64_t stride;
};

struct NormK {
    NormTensor x, r, y;     // r.p == nullptr: no residual operand
    NormTensor dy, dx, dr;  // backward only; dx.p, dr.p may be nullptr
    const void *weight, *bias;  // nullptr: ones, zeros
    void *dweight, *dbias;
    float *stats;           // N x G pairs: mean, 1 / sqrt(variance + eps)
    float *part;            // workspace: partial results of pixel chunks
    float *sums;            // workspace: backward, N x G pairs of a group's sums
    uint32_t N, P, C, G, per;  // per: channels of a group
    uint32_t chunks, chunk;    // pixel chunks of an image, pixels of one
    uint32_t blocks;           // channel blocks
    uint32_t spans;            // partial results of a group in a chunk: channel blocks that it may meet
    uint32_t activation, f32_params;
    float eps;
};

enum NormPass { NORM_STATS, NORM_JOIN, NORM_APPLY, NORM_GRAD_SUMS, NORM_GRAD_JOIN, NORM_GRAD_PARAMS, NORM_GRAD_APPLY };
// Enqueue one pass; vec: elements of a lane's vector (a power of two that divides C and every stride, addresses aligned to it).
bs_status launch_norm(NormPass pass, const NormK &k, int32_t dtype, int vec, void *stream);

}  // namespace bs
