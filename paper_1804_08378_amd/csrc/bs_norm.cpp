// Group normalisation: argument checks, the split of the work, the launches.  Nothing here synchronises or allocates.
#include "bs_norm.h"

#include <algorithm>
#include <cmath>
#include <numeric>

#include "bs_internal.h"

using namespace bs;

namespace {

uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }
uint64_t aligned(uint64_t bytes) { return ceil_div(bytes, 256) * 256; }

bs_status check_desc(const bs_group_norm_desc *d)
{
    if (!d) return BS_ERR_NULL;
    for (int i = 0; i < 4; ++i)
        if (d->shape[i] < 1) return BS_ERR_SHAPE;
    if (d->dtype != BS_F32 && d->dtype != BS_BF16 && d->dtype != BS_F16) return BS_ERR_UNSUPPORTED;
    if (d->param_dtype != BS_F32 && d->param_dtype != d->dtype) return BS_ERR_UNSUPPORTED;
    if (d->activation < BS_ACT_IDENTITY || d->activation > BS_ACT_GELU) return BS_ERR_UNSUPPORTED;
    if (!std::isfinite(d->eps) || d->eps < 0) return BS_ERR_PARAM;
    const int64_t C = d->shape[1], limit = (1ll << 31) - 1;
    if (d->groups < 1 || C % d->groups != 0) return BS_ERR_PARAM;
    if (d->shape[2] > limit || d->shape[3] > limit || d->shape[0] > limit || C > limit) return BS_ERR_UNSUPPORTED;
    if ((double)d->shape[1] * (double)d->shape[2] * (double)d->shape[3] > (double)limit) return BS_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(d->exchange) % 8 != 0) return BS_ERR_ALIGN;
    // grids are counted in 32 bits: images, groups
    if (d->shape[0] > (1ll << 22) || d->shape[0] * (int64_t)d->groups > (1ll << 24) || d->shape[0] * C > limit) return BS_ERR_UNSUPPORTED;
    for (const int64_t s : {d->x_stride, d->residual_stride, d->y_stride, d->grad_y_stride, d->grad_x_stride, d->grad_residual_stride})
        if (s != 0 && (s < C || s > limit)) return BS_ERR_SHAPE;
    return BS_OK;
}

// Pixel chunks and channel blocks of the kernels that read x twice.  Work-groups of at least 16 KiB of one tensor, 2048 of them where the
// tensor has so much.
void split(const bs_group_norm_desc &d, NormK &k)
{
    k.blocks = (uint32_t)ceil_div(k.C, K_NORM_BLOCK_CHANNELS);
    k.spans = (k.per + K_NORM_BLOCK_CHANNELS - 2) / K_NORM_BLOCK_CHANNELS + 1;
    const uint64_t row = std::min<uint64_t>(k.C, K_NORM_BLOCK_CHANNELS) * dtype_size(d.dtype);
    const uint64_t wanted = ceil_div(2048, (uint64_t)k.N * k.blocks), most = std::min<uint64_t>(256, ceil_div(k.P * row, 16384));
    const uint64_t chunks = std::max<uint64_t>(1, std::min(wanted, most));
    k.chunk = (uint32_t)ceil_div(k.P, chunks);
    k.chunks = (uint32_t)ceil_div(k.P, k.chunk);
}

// The same for the kernels that keep their pixels in registers; false where they do not apply: a group too wide, or an image of more chunks
// than a work-group joins.
bool split_resident(const bs_group_norm_desc &d, int vec, bool backward, bool residual, NormK &k, bool &few)
{
    const uint64_t es = dtype_size(d.dtype);
    const bool mixed = k.per % (uint32_t)vec != 0, in_gradient = residual && d.activation != BS_ACT_IDENTITY;
    auto pixels = [&](bool small) {
        const int bytes = vec * (int)es;
        return (uint64_t)(backward ? norm_resident_grad_pixels(bytes, in_gradient, small, mixed) : norm_resident_pixels(bytes, residual, small));
    };
    // backward, the chunks' sums of a channel stay small beside its pixels: 8 bytes for at least 256 of them, or few chunks
    const uint64_t small_sums = backward ? std::max<uint64_t>(16, k.P * es / 256) : 128;
    // A block: whole groups and whole vectors, a divisor of the channels, at least a cache line of every pixel.  Blocks that begin inside cache
    // lines share them with their neighbours, and read them twice (a block that begins at any 16 bytes touches 128 - 16 = 112 bytes more than
    // its own on average): in tensors of 16 MiB on the smallest block for which that is a sixth of it at most (9x288x83x83 binary16 forward
    // 47.7 -> 25.7 us, 7x336x143x143 both directions 183 -> 157), in smaller ones the smallest of all (8x640x32x32 binary16 forward 12.7 us,
    // 18.3 in such blocks, whose chunks are few pixels).
    const uint64_t unit = std::lcm((uint64_t)k.per, (uint64_t)vec), units = k.C / unit;
    uint64_t most = 0, lanes = 0, groups = 0;
    bool found = false;
    const bool large = (uint64_t)k.N * k.P * k.C * es >= (16 << 20);
    for (const bool whole_lines : {true, false}) {
        if (whole_lines && !large) continue;
        for (uint64_t m = 1; m <= units && !found; ++m) {
            const uint64_t bytes = unit * m * es;
            if (units % m != 0 || (m < units && bytes < 128)) continue;
            const bool apart = m == units || (bytes % 128 == 0 && k.C * es % 128 == 0);
            if (whole_lines && !apart && bytes < 6 * 112) continue;
            lanes = K_NORM_RESIDENT_THREADS / std::max<uint64_t>(1, unit * m / (uint64_t)vec);
            groups = unit * m / k.per;
            if (lanes < (whole_lines ? 4 : 1) || groups > (uint64_t)K_NORM_RESIDENT_THREADS) break;
            most = std::min({(uint64_t)128, small_sums, (uint64_t)K_NORM_WORDS / groups});
            const uint64_t chunks = ceil_div(k.P, lanes * pixels(false));
            found = chunks <= most && (uint64_t)k.N * (units / m) * chunks < (1ull << 23);  // (the launch's lanes are counted in 32 bits)
            if (found) k.block = (uint32_t)(unit * m);
        }
    }
    if (!found) return false;
    k.blocks = k.C / k.block;
    // One chunk needs no exchange and no second launch: few pixels a lane where they are enough for that, many where they are half empty (one
    // work-group that fills its registers is slower than four that exchange: 8x512x28x28 binary16 13.4 us against 9.6).  Images of several
    // chunks: many pixels a lane, or few where that leaves compute units without work.
    const uint64_t chunks[2] = {ceil_div(k.P, lanes * pixels(false)), ceil_div(k.P, lanes * pixels(true))};
    const bool half_empty = k.P <= lanes * pixels(false) / 2;
    few = chunks[1] == 1 || (!half_empty && chunks[1] <= most && (uint64_t)k.N * k.blocks * chunks[0] < K_NORM_SLOTS);
    k.chunk = (uint32_t)ceil_div(k.P, chunks[few]);
    k.chunks = (uint32_t)ceil_div(k.P, k.chunk);
    k.groups = (uint32_t)groups;
    k.lanes = (uint32_t)lanes;
    k.last = k.P - (k.chunks - 1) * k.chunk;
    k.chunk_each = k.chunk / k.lanes;
    k.last_each = k.last / k.lanes;
    const uint32_t cvb = k.block / (uint32_t)vec, root = (uint32_t)std::ceil(std::sqrt((double)lanes));
    k.slices = std::max<uint32_t>(1, std::min(root, K_NORM_RESIDENT_THREADS / cvb));
    k.slices_wide = std::max<uint32_t>(1, std::min(root, K_NORM_RESIDENT_THREADS / k.block));
    k.by_chunks = make_fastdiv(k.chunks);
    k.by_blocks = make_fastdiv(k.blocks);
    k.by_cvb = make_fastdiv(cvb);
    k.by_cols_wide = make_fastdiv(k.block);
    k.by_per = make_fastdiv(k.per);
    k.by_vectors = make_fastdiv(std::max<uint32_t>(1, k.per / (uint32_t)vec));
    return true;
}

struct Space {
    uint64_t pairs = 0, words = 0, part = 0, bytes = 0;  // offsets, size
};

// Bytes of the exchange memory that a call needs: words, and a count for every channel block of an image.
uint64_t exchange_bytes(const NormK &k) { return ((uint64_t)k.N * k.G * 8 * k.chunks) + (uint64_t)k.N * k.blocks * 4; }

Space space(const NormK &k, bool backward, bool resident, bool exchange)
{
    Space s;
    const uint64_t pairs = (uint64_t)k.N * k.G * 8;  // forward: the statistics, where the caller does not want them; backward: the groups' sums
    s.words = aligned(pairs);
    s.part = s.words + (resident && k.chunks > 1 && !exchange ? aligned(pairs * k.chunks) : 0);
    s.bytes = s.part + (backward ? aligned((uint64_t)k.N * k.chunks * k.C * 8) : resident ? 0 : aligned(pairs * k.chunks * k.spans));
    return s;
}

void sizes(const bs_group_norm_desc &d, NormK &k)
{
    k.N = (uint32_t)d.shape[0];
    k.C = (uint32_t)d.shape[1];
    k.P = (uint32_t)(d.shape[2] * d.shape[3]);
    k.G = (uint32_t)d.groups;
    k.per = k.C / k.G;
}

// Chooses the kernels and lays out the workspace.  `vec`: the vectors that channels, strides and addresses allow; made smaller where there is no
// instance of them (norm_resident_pixels says why).
bool plan(const bs_group_norm_desc &d, int &vec, bool backward, bool residual, NormK &k, Space &s, bool &few)
{
    const int full = (int)(16 / dtype_size(d.dtype));
    if (vec != full && vec != full / 2) vec = 1;
    if (vec == full && (backward || k.per % (uint32_t)full != 0)) vec = full / 2;
    const bool resident = split_resident(d, vec, backward, residual, k, few);
    if (!resident) split(d, k);
    // The exchange memory saves a launch and costs every work-group a count: worth it for two rounds of them (both directions of 5x60x37x29
    // binary16 25.6 us by launches, 21.5 through the memory; of 64x256x56x56 bfloat16, 13 rounds, 200 and 206).
    const bool exchange = d.exchange && exchange_bytes(k) <= d.exchange_bytes && (uint64_t)k.N * k.blocks * k.chunks <= 2 * K_NORM_SLOTS;
    s = space(k, backward, resident, exchange);
    if (resident && exchange) {
        k.words = static_cast<uint64_t *>(d.exchange);
        k.departed = reinterpret_cast<uint32_t *>(k.words + (uint64_t)k.N * k.G * k.chunks);
    }
    return resident;
}

NormTensor tensor(const void *p, int64_t stride, const NormK &k) { return NormTensor{p, (uint64_t)(stride ? stride : k.C)}; }

// Elements of a lane's vector: 128 bits, or less where the channels, a stride or an address are no multiple of that.
int vector_of(const NormK &k, int32_t dtype, std::initializer_list<const NormTensor *> tensors)
{
    const uint64_t es = dtype_size(dtype);
    uint64_t vec = 16 / es;
    for (; vec > 1; vec /= 2) {
        bool fits = k.C % vec == 0;
        for (const NormTensor *t : tensors)
            fits = fits && (!t->p || (t->stride % vec == 0 && reinterpret_cast<uintptr_t>(t->p) % (vec * es) == 0));
        if (fits) break;
    }
    return (int)vec;
}

uint32_t polls_of(const bs_group_norm_desc &d) { return d.wait_polls < 0 ? 0 : d.wait_polls ? (uint32_t)d.wait_polls : K_NORM_POLLS; }

TensorBytes bytes_of(const NormK &k, const NormTensor &t, uint64_t es) { return TensorBytes{t.p, (uint64_t)k.N * k.P, k.C * es, t.stride * es}; }
TensorBytes bytes_of(const void *p, uint64_t n) { return TensorBytes{p, 1, n, n}; }

bool element_aligned(const void *p, uint64_t es) { return reinterpret_cast<uintptr_t>(p) % es == 0; }

// No output shares a byte with an input, another output or the workspace.
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

uint64_t bs_group_norm_workspace_bytes(const bs_group_norm_desc *desc, int32_t backward)
{
    if (check_desc(desc) != BS_OK) return 0;
    // addresses and strides decide on the vectors later: room for every choice
    uint64_t bytes = 0;
    for (int vec = (int)(16 / dtype_size(desc->dtype)); vec; vec /= 2) {
        for (const bool residual : {false, true}) {
            NormK k{};
            sizes(*desc, k);
            if (k.C % (uint32_t)vec != 0) continue;
            Space s;
            bool few;
            int used = vec;
            plan(*desc, used, backward != 0, residual, k, s, few);
            bytes = std::max(bytes, s.bytes);
        }
    }
    return bytes;
}

bs_status bs_group_norm(const bs_group_norm_desc *desc, const void *x, const void *residual, const void *weight, const void *bias, void *y,
                        float *stats, void *workspace, uint64_t workspace_bytes, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (!x || !y) return BS_ERR_NULL;
    NormK k{};
    sizes(*desc, k);
    k.x = tensor(x, desc->x_stride, k);
    k.r = tensor(residual, desc->residual_stride, k);
    k.y = tensor(y, desc->y_stride, k);
    const uint64_t es = dtype_size(desc->dtype), ps = dtype_size(desc->param_dtype), pairs = (uint64_t)k.N * k.G * 8;
    int vec = vector_of(k, desc->dtype, {&k.x, &k.r, &k.y});
    Space s;
    bool few = false;
    const bool resident = plan(*desc, vec, false, residual != nullptr, k, s, few);
    if (!workspace || workspace_bytes < s.bytes) return BS_ERR_WORKSPACE;
    for (const void *p : {x, residual, (const void *)y})
        if (!element_aligned(p, es)) return BS_ERR_ALIGN;
    if (!element_aligned(weight, ps) || !element_aligned(bias, ps) || !element_aligned(stats, 8) || !element_aligned(workspace, 16)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({bytes_of(k, k.x, es), bytes_of(k, k.r, es), bytes_of(weight, k.C * ps), bytes_of(bias, k.C * ps)},
                                          {bytes_of(k, k.y, es), bytes_of(stats, pairs), bytes_of(workspace, s.bytes), bytes_of(desc->exchange, desc->exchange ? desc->exchange_bytes : 0)});
    if (alias != BS_OK) return alias;
    k.weight = weight;
    k.bias = bias;
    k.activation = (uint32_t)desc->activation;
    k.f32_params = desc->param_dtype == BS_F32;
    k.eps = (float)desc->eps;
    char *const ws = static_cast<char *>(workspace);
    if (!k.departed) k.words = reinterpret_cast<uint64_t *>(ws + s.words);
    k.polls = polls_of(*desc);
    if (resident) {
        k.stats = stats;
        const bs_status st = k.chunks > 1 && !k.departed ? launch_norm_absent(k, stream) : BS_OK;
        return st != BS_OK ? st : launch_norm_resident(k, desc->dtype, vec, few, stream);
    }
    k.stats = stats ? stats : reinterpret_cast<float *>(ws + s.pairs);
    k.part = reinterpret_cast<float *>(ws + s.part);
    for (const NormPass pass : {NORM_STATS, NORM_JOIN, NORM_APPLY}) {
        const bs_status st = launch_norm(pass, k, desc->dtype, vec, stream);
        if (st != BS_OK) return st;
    }
    return BS_OK;
}

bs_status bs_group_norm_backward(const bs_group_norm_desc *desc, const void *x, const void *residual, const void *weight, const void *bias,
                                 const float *stats, const void *grad_y, void *grad_x, void *grad_residual, void *grad_weight, void *grad_bias,
                                 void *workspace, uint64_t workspace_bytes, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (!x || !stats || !grad_y) return BS_ERR_NULL;
    NormK k{};
    sizes(*desc, k);
    k.x = tensor(x, desc->x_stride, k);
    k.r = tensor(residual, desc->residual_stride, k);
    k.dy = tensor(grad_y, desc->grad_y_stride, k);
    k.dx = tensor(grad_x, desc->grad_x_stride, k);
    k.dr = tensor(grad_residual, desc->grad_residual_stride, k);
    const uint64_t es = dtype_size(desc->dtype), ps = dtype_size(desc->param_dtype), pairs = (uint64_t)k.N * k.G * 8;
    int vec = vector_of(k, desc->dtype, {&k.x, &k.r, &k.dy, &k.dx, &k.dr});
    Space s;
    bool few = false;
    const bool resident = plan(*desc, vec, true, residual != nullptr, k, s, few);
    if (!workspace || workspace_bytes < s.bytes) return BS_ERR_WORKSPACE;
    for (const void *p : {x, residual, grad_y, (const void *)grad_x, (const void *)grad_residual})
        if (!element_aligned(p, es)) return BS_ERR_ALIGN;
    for (const void *p : {weight, bias, (const void *)grad_weight, (const void *)grad_bias})
        if (!element_aligned(p, ps)) return BS_ERR_ALIGN;
    if (!element_aligned(stats, 8) || !element_aligned(workspace, 16)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({bytes_of(k, k.x, es), bytes_of(k, k.r, es), bytes_of(weight, k.C * ps), bytes_of(bias, k.C * ps),
                                           bytes_of(stats, pairs), bytes_of(k, k.dy, es)},
                                          {bytes_of(k, k.dx, es), bytes_of(k, k.dr, es), bytes_of(grad_weight, k.C * ps), bytes_of(grad_bias, k.C * ps),
                                           bytes_of(workspace, s.bytes), bytes_of(desc->exchange, desc->exchange ? desc->exchange_bytes : 0)});
    if (alias != BS_OK) return alias;
    k.weight = weight;
    k.bias = bias;
    k.dweight = grad_weight;
    k.dbias = grad_bias;
    k.activation = (uint32_t)desc->activation;
    k.f32_params = desc->param_dtype == BS_F32;
    k.eps = (float)desc->eps;
    char *const ws = static_cast<char *>(workspace);
    k.stats = const_cast<float *>(stats);
    k.sums = reinterpret_cast<float *>(ws + s.pairs);
    k.part = reinterpret_cast<float *>(ws + s.part);
    if (!k.departed) k.words = reinterpret_cast<uint64_t *>(ws + s.words);
    k.polls = polls_of(*desc);
    const bool tensors = grad_x || grad_residual, params = grad_weight || grad_bias;
    if (resident) {
        if (!params) k.part = nullptr;
        bs_status st = k.chunks > 1 && tensors && !k.departed ? launch_norm_absent(k, stream) : BS_OK;
        if (st == BS_OK && (tensors || params)) st = launch_norm_resident_grad(k, desc->dtype, vec, few, stream);
        if (st == BS_OK && params) st = launch_norm(NORM_GRAD_PARAMS, k, desc->dtype, vec, stream);
        return st;
    }
    for (const NormPass pass : {NORM_GRAD_SUMS, NORM_GRAD_JOIN, NORM_GRAD_PARAMS, NORM_GRAD_APPLY}) {
        if (pass == NORM_GRAD_PARAMS ? !params : pass == NORM_GRAD_SUMS ? !params && !grad_x : pass == NORM_GRAD_JOIN ? !grad_x : !tensors) continue;
        const bs_status st = launch_norm(pass, k, desc->dtype, vec, stream);
        if (st != BS_OK) return st;
    }
    return BS_OK;
}

}  // extern "C"
