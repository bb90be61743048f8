// Layer normalisation: argument checks, the split of the work, the launches.  Nothing here synchronises or allocates.
#include "bs_layer_norm.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

using namespace bs;

namespace {

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

bs_status check_desc(const bs_layer_norm_desc *d)
{
    if (!d) return BS_ERR_NULL;
    const bs_status st = check_rows(d->rows, d->features, d->dtype,
                                    {d->x_stride, d->addend_stride, d->total_stride, d->y_stride, d->grad_y_stride, d->grad_total_stride, d->grad_x_stride});
    if (st != BS_OK) return st;
    if (d->param_dtype != BS_F32 && d->param_dtype != d->dtype) return BS_ERR_UNSUPPORTED;
    return !std::isfinite(d->eps) || d->eps < 0 ? BS_ERR_PARAM : BS_OK;
}

void fill(const bs_layer_norm_desc &d, LayerNormK &k)
{
    k.rows = (uint64_t)d.rows;
    k.C = (uint32_t)d.features;
    k.f32_params = d.param_dtype == BS_F32;
    k.eps = (float)d.eps;
}

// Lanes that a row takes and their vectors; a row of 64 KiB is the longest that registers hold, one of 16384 elements the longest whose columns' sums
// the backward pass holds too.
LayerNormTeam team_of(const LayerNormK &k, int32_t dtype, bool backward)
{
    const uint64_t vec = dtype == BS_F32 ? 4 : 8, vectors = ceil_div(k.C, vec);
    LayerNormTeam t{8, 1, 0, k.C <= 16384};
    if (k.C < vec || vectors > 4096) return LayerNormTeam{0, 0, 0, false};  // (every lane reads a whole vector of the row)
    while (t.team < 1024 && (uint64_t)t.team < vectors) t.team *= 2;
    while ((uint64_t)t.team * t.vectors < vectors) t.vectors *= 2;
    const uint64_t threads = backward ? (uint64_t)K_LAYER_NORM_GRAD_THREADS : (uint64_t)(t.team <= 64 ? 256 : t.team), teams = threads / (uint64_t)t.team;
    // 1024 lanes a compute unit that walk over the rows in both directions.  Forward (8192 x 4096 bfloat16 behind an addition; both directions of 200704 x 256,
    // of 16384 x 2048 through 8 bits): 512 lanes 45, 99, 98 us; 768 48, 91, 101; 1024 43, 88, 100; 1280 50, 90, 102; 2048 48, 94, 101; a work-group for
    // every row 57, 93, 109.
    t.groups = (uint32_t)std::min<uint64_t>(ceil_div(k.rows, teams), K_LAYER_NORM_GROUPS * (K_LAYER_NORM_GRAD_THREADS / threads));
    return t;
}

// Parts of the rows, whose sums a second launch joins: what the backward pass's work-groups leave, or tiles of columns, 1024 of them in all.
void parts(LayerNormK &k, const LayerNormTeam &t, int32_t dtype)
{
    if (!k.rows) return;
    if (t.sums) {
        k.parts = t.groups;
        return;
    }
    const uint64_t tiles = ceil_div(k.C, 64 * (dtype == BS_F32 ? 4 : 8));
    k.per_part = ceil_div(k.rows, std::max<uint64_t>(1, std::min(ceil_div(1024, tiles), ceil_div(k.rows, 16))));
    k.parts = (uint32_t)ceil_div(k.rows, k.per_part);
}

uint64_t space(const LayerNormK &k) { return std::max<uint64_t>(16, (uint64_t)k.parts * k.C * 8); }

}  // namespace

extern "C" {

bs_status bs_layer_norm(const bs_layer_norm_desc *desc, const void *x, const void *addend, const void *weight, const void *bias, void *y, void *total,
                        float *stats, int8_t *codes, uint8_t *exponents, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!x || !y || !codes != !exponents) return BS_ERR_NULL;
    LayerNormK k{};
    fill(*desc, k);
    k.x = row_tensor(x, desc->x_stride, k.C);
    k.addend = row_tensor(addend, desc->addend_stride, k.C);
    k.y = row_tensor(y, desc->y_stride, k.C);
    k.total = row_tensor(total, desc->total_stride, k.C);
    k.held = HeldRows{codes, exponents};
    k.weight = weight;
    k.bias = bias;
    k.stats = stats;
    const uint64_t es = dtype_size(desc->dtype), ps = dtype_size(desc->param_dtype), C = k.C, cells = k.rows * C;
    for (const void *p : {x, addend, (const void *)y, (const void *)total})
        if (!aligned_to(p, es)) return BS_ERR_ALIGN;
    if (!aligned_to(weight, ps) || !aligned_to(bias, ps) || !aligned_to(stats, 8)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({bytes_of(k.x, k.rows, C, es), bytes_of(k.addend, k.rows, C, es), bytes_of(weight, C * ps), bytes_of(bias, C * ps)},
                                          {bytes_of(k.y, k.rows, C, es), bytes_of(k.total, k.rows, C, es), bytes_of(stats, k.rows * 8),
                                           bytes_of(codes, cells), bytes_of(exponents, k.rows * blocks_of(C))});
    if (alias != BS_OK) return alias;
    const LayerNormTeam team = team_of(k, desc->dtype, false);
    return team.team ? launch_layer_norm_team(k, team, desc->dtype, stream) : launch_layer_norm(LAYER_NORM, k, desc->dtype, stream);
}

uint64_t bs_layer_norm_workspace_bytes(const bs_layer_norm_desc *desc)
{
    if (check_desc(desc) != BS_OK) return 0;
    LayerNormK k{};
    fill(*desc, k);
    parts(k, team_of(k, desc->dtype, true), desc->dtype);
    return space(k);
}

bs_status bs_layer_norm_backward(const bs_layer_norm_desc *desc, const void *t, const int8_t *codes, const uint8_t *exponents, const float *stats,
                                 const void *weight, const void *grad_y, const void *grad_total, void *grad_x, void *grad_weight, void *grad_bias,
                                 void *workspace, uint64_t workspace_bytes, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    const bool params = grad_weight || grad_bias;
    if (desc->rows == 0 && !params) return BS_OK;
    if (desc->rows != 0 && (!t == !codes || !codes != !exponents || !stats || !grad_y)) return BS_ERR_NULL;
    LayerNormK k{};
    fill(*desc, k);
    k.x = row_tensor(t, desc->x_stride, k.C);
    k.dy = row_tensor(grad_y, desc->grad_y_stride, k.C);
    k.dt = row_tensor(grad_total, desc->grad_total_stride, k.C);
    k.dx = row_tensor(grad_x, desc->grad_x_stride, k.C);
    k.held = HeldRows{const_cast<int8_t *>(codes), const_cast<uint8_t *>(exponents)};
    k.weight = weight;
    k.dweight = grad_weight;
    k.dbias = grad_bias;
    k.stats = const_cast<float *>(stats);
    k.part = params ? static_cast<float *>(workspace) : nullptr;
    const LayerNormTeam team = team_of(k, desc->dtype, true);
    parts(k, team, desc->dtype);
    const uint64_t es = dtype_size(desc->dtype), ps = dtype_size(desc->param_dtype), C = k.C, cells = k.rows * C;
    if (params && (!workspace || workspace_bytes < space(k))) return BS_ERR_WORKSPACE;
    for (const void *p : {t, grad_y, grad_total, (const void *)grad_x})
        if (!aligned_to(p, es)) return BS_ERR_ALIGN;
    for (const void *p : {weight, (const void *)grad_weight, (const void *)grad_bias})
        if (!aligned_to(p, ps)) return BS_ERR_ALIGN;
    if (!aligned_to(stats, 8) || (params && !aligned_to(workspace, 16))) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({bytes_of(k.x, k.rows, C, es), bytes_of(k.dy, k.rows, C, es), bytes_of(k.dt, k.rows, C, es), bytes_of(weight, C * ps),
                                           bytes_of(stats, k.rows * 8), bytes_of(codes, cells), bytes_of(exponents, k.rows * blocks_of(C))},
                                          {bytes_of(k.dx, k.rows, C, es), bytes_of(grad_weight, C * ps), bytes_of(grad_bias, C * ps),
                                           bytes_of(params ? workspace : nullptr, space(k))});
    if (alias != BS_OK) return alias;
    if (!team.sums) k.part = nullptr;
    bs_status st = BS_OK;
    if (k.rows && team.team && (grad_x || (params && team.sums))) st = launch_layer_norm_team_grad(k, team, desc->dtype, stream);
    else if (k.rows && grad_x) st = launch_layer_norm(LAYER_NORM_GRAD, k, desc->dtype, stream);
    if (st != BS_OK || !params || (team.sums && k.parts == 1)) return st;  // (one work-group writes the parameters' gradients itself)
    k.part = static_cast<float *>(workspace);
    if (k.rows && !team.sums) st = launch_layer_norm(LAYER_NORM_GRAD_PARTS, k, desc->dtype, stream);
    return st == BS_OK ? launch_layer_norm(LAYER_NORM_GRAD_JOIN, k, desc->dtype, stream) : st;
}

}  // extern "C"
