// Argument block and launches of the layer-normalisation kernels (bs_layer_norm*.hip), shared with the host code that fills them (bs_layer_norm.cpp).
#pragma once

#include "bs_rows_args.h"

namespace bs {

constexpr uint32_t K_LAYER_NORM_ROW_GROUPS = 512;  // work-groups that walk over long rows, at most: two of each compute unit

constexpr int K_LAYER_NORM_GRAD_THREADS = 1024;  // of a work-group of the backward pass with the rows in registers
constexpr uint64_t K_LAYER_NORM_GROUPS = 256;     // of work-groups of that size at most: one of each compute unit

struct LayerNormK {
    RowTensor x, addend, y, total;  // backward: x is t; addend, total: p may be nullptr
    RowTensor dy, dt, dx;           // backward only; dt.p, dx.p may be nullptr
    HeldRows held;                  // forward: written; backward: read in x's place.  codes nullptr: not held
    const void *weight, *bias;      // nullptr: ones, zeros
    void *dweight, *dbias;
    float *stats;  // a pair a row: mean, 1 / sqrt(variance + eps)
    float *part;   // workspace: pairs of (grad bias, grad weight), parts x C
    uint64_t rows;
    uint32_t C;
    uint32_t parts;    // row parts of the gradients of weight and bias
    uint64_t per_part; // rows of one
    uint32_t f32_params;
    float eps;
};

enum LayerNormPass { LAYER_NORM, LAYER_NORM_GRAD, LAYER_NORM_GRAD_PARTS, LAYER_NORM_GRAD_JOIN };
bs_status launch_layer_norm(LayerNormPass pass, const LayerNormK &k, int32_t dtype, void *stream);

// Rows in the registers of teams of lanes: lanes of a team, vectors of a lane, work-groups; does the backward pass sum the gradients of weight and
// bias on its way?  team == 0: rows too long (or short) for that.
struct LayerNormTeam {
    int team, vectors;
    uint32_t groups;
    bool sums;
};
bs_status launch_layer_norm_team(const LayerNormK &k, const LayerNormTeam &t, int32_t dtype, void *stream);
bs_status launch_layer_norm_team_grad(const LayerNormK &k, const LayerNormTeam &t, int32_t dtype, void *stream);

}  // namespace bs
