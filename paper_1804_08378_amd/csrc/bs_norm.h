// Argument block and launches of the group-normalisation kernels (bs_norm.hip, bs_norm_resident.hip, bs_norm_resident_grad.hip), shared with the
// host code that fills and calls them (bs_norm.cpp).
#pragma once

#include <cstdint>

#include "brainslug.h"
#include "bs_kargs.h"

namespace bs {

constexpr int K_NORM_THREADS = 256;        // work-group size of the kernels that read x twice
constexpr int K_NORM_BLOCK_CHANNELS = 256; // channels of a work-group at most: a lane keeps one vector of them

constexpr int K_NORM_RESIDENT_THREADS = 512;  // work-group size of the kernels that keep their pixels in registers
constexpr uint64_t K_NORM_SLOTS = 512;     // of them at a time: two of each of the 256 compute units
constexpr int K_NORM_WORDS = 2048;         // words (groups of a block x chunks) that such a work-group can join
constexpr uint32_t K_NORM_POLLS = 1024;    // polls of a word before a work-group computes its neighbours' sums itself: about a millisecond

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
    // resident kernels: channels and groups of a block, pixel lanes of a work-group, polls, words of all groups' chunks; pixels of the last
    // chunk, pixels that every lane has of any other and of the last chunk; rows joined at a time, of a column a vector and a column a channel
    uint32_t block, groups, lanes, polls;
    uint32_t last, chunk_each, last_each, slices, slices_wide;
    uint64_t *words;
    uint32_t *departed;  // work-groups of a block that have collected their words; nullptr: the words were cleared by a launch and stay as they are
    FastDiv by_chunks, by_blocks, by_cvb, by_cols_wide, by_per, by_vectors;  // by_vectors: channel vectors of a group
};

enum NormPass { NORM_STATS, NORM_JOIN, NORM_APPLY, NORM_GRAD_SUMS, NORM_GRAD_JOIN, NORM_GRAD_PARAMS, NORM_GRAD_APPLY };
// Enqueue one pass; vec: elements of a lane's vector, 128 (forward only) or 64 bits or one element (it divides C and every stride, addresses are
// aligned to it).
bs_status launch_norm(NormPass pass, const NormK &k, int32_t dtype, int vec, void *stream);

// Pixels that a lane keeps in registers, as many as 128 of them hold without spilling (two work-groups of a compute unit).  bytes: of a lane's
// vector; few: the instances for small images; mixed: vectors that reach over groups, which need the statistics of every channel beside them.
// Parameters, sums and temporaries take registers for every channel of a vector, so that vectors of 64 bits leave more of them for pixels: backward
// there are no longer ones, forward none that reach over groups.
constexpr int norm_resident_pixels(int bytes, bool residual, bool few)
{
    if (few) return 4;
    return (bytes == 8 ? 32 : 16) / (residual ? 2 : 1);
}
constexpr int norm_resident_grad_pixels(int bytes, bool residual, bool few, bool mixed)
{
    if (few) return 2;
    if (bytes != 8) return 8;
    return residual ? (mixed ? 8 : 10) : mixed ? 12 : 16;
}
bs_status launch_norm_absent(const NormK &k, void *stream);
bs_status launch_norm_resident(const NormK &k, int32_t dtype, int vec, bool few, void *stream);
bs_status launch_norm_resident_grad(const NormK &k, int32_t dtype, int vec, bool few, void *stream);

}  // namespace bs
