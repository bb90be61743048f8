// Activations and 8-bit checkpoints: argument checks and launches.  Nothing here synchronises or allocates.
#include "bs_activate.h"

using namespace bs;

namespace {

void fill(ActivateK &k, int64_t rows, int64_t columns, int32_t dtype)
{
    const uint32_t lanes = dtype == BS_F32 ? 8 : 4;  // of a block
    k.columns = (uint32_t)columns;
    k.per_row = (uint32_t)(blocks_of((uint64_t)columns) * lanes);
    k.vectors = (uint64_t)rows * k.per_row;
    k.by_row = make_fastdiv(k.per_row);
}

bs_status check_desc(const bs_activate_desc *d)
{
    if (!d) return BS_ERR_NULL;
    const bs_status st = check_rows(d->rows, d->columns, d->dtype, {d->x_stride, d->gate_stride, d->y_stride, d->grad_y_stride, d->grad_x_stride, d->grad_gate_stride});
    if (st != BS_OK) return st;
    return d->activation < BS_ACT_IDENTITY || d->activation > BS_ACT_GELU ? BS_ERR_UNSUPPORTED : BS_OK;
}

bs_status check_desc(const bs_pack8_desc *d) { return d ? check_rows(d->rows, d->columns, d->dtype, {d->x_stride}) : BS_ERR_NULL; }

struct Bytes {
    uint64_t rows, columns, es;
    TensorBytes operator()(const RowTensor &t) const { return bytes_of(t, rows, columns, es); }
    TensorBytes codes(const void *p) const { return bytes_of(p, rows * columns); }
    TensorBytes exponents(const void *p) const { return bytes_of(p, rows * blocks_of(columns)); }
};

}  // namespace

extern "C" {

bs_status bs_pack8(const bs_pack8_desc *desc, const void *x, int8_t *codes, uint8_t *exponents, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!x || !codes || !exponents) return BS_ERR_NULL;
    ActivateK k{};
    k.x = row_tensor(x, desc->x_stride, desc->columns);
    k.hx = HeldRows{codes, exponents};
    const Bytes b{(uint64_t)desc->rows, (uint64_t)desc->columns, dtype_size(desc->dtype)};
    if (!aligned_to(x, b.es)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({b(k.x)}, {b.codes(codes), b.exponents(exponents)});
    if (alias != BS_OK) return alias;
    fill(k, desc->rows, desc->columns, desc->dtype);
    return launch_rows(ROWS_PACK8, k, desc->dtype, BS_ACT_IDENTITY, stream);
}

bs_status bs_unpack8(const bs_pack8_desc *desc, const int8_t *codes, const uint8_t *exponents, void *x, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!x || !codes || !exponents) return BS_ERR_NULL;
    ActivateK k{};
    k.y = row_tensor(x, desc->x_stride, desc->columns);
    k.hx = HeldRows{const_cast<int8_t *>(codes), const_cast<uint8_t *>(exponents)};
    const Bytes b{(uint64_t)desc->rows, (uint64_t)desc->columns, dtype_size(desc->dtype)};
    if (!aligned_to(x, b.es)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({b.codes(codes), b.exponents(exponents)}, {b(k.y)});
    if (alias != BS_OK) return alias;
    fill(k, desc->rows, desc->columns, desc->dtype);
    return launch_rows(ROWS_UNPACK8, k, desc->dtype, BS_ACT_IDENTITY, stream);
}

bs_status bs_activate(const bs_activate_desc *desc, const void *x, const void *gate, void *y, int8_t *x_codes, uint8_t *x_exponents,
                      int8_t *gate_codes, uint8_t *gate_exponents, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    if (!x || !y || !x_codes != !x_exponents || !gate_codes != !gate_exponents || (gate_codes && !gate) || (gate && !x_codes != !gate_codes)) return BS_ERR_NULL;
    ActivateK k{};
    k.x = row_tensor(x, desc->x_stride, desc->columns);
    k.gate = row_tensor(gate, desc->gate_stride, desc->columns);
    k.y = row_tensor(y, desc->y_stride, desc->columns);
    k.hx = HeldRows{x_codes, x_exponents};
    k.hg = HeldRows{gate_codes, gate_exponents};
    const Bytes b{(uint64_t)desc->rows, (uint64_t)desc->columns, dtype_size(desc->dtype)};
    for (const void *p : {x, gate, (const void *)y})
        if (!aligned_to(p, b.es)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({b(k.x), b(k.gate)}, {b(k.y), b.codes(x_codes), b.exponents(x_exponents), b.codes(gate_codes), b.exponents(gate_exponents)});
    if (alias != BS_OK) return alias;
    fill(k, desc->rows, desc->columns, desc->dtype);
    return launch_rows(ROWS_ACTIVATE, k, desc->dtype, desc->activation, stream);
}

bs_status bs_activate_backward(const bs_activate_desc *desc, const void *x, const int8_t *x_codes, const uint8_t *x_exponents, const void *gate,
                               const int8_t *gate_codes, const uint8_t *gate_exponents, const void *grad_y, void *grad_x, void *grad_gate, void *stream)
{
    const bs_status checked = check_desc(desc);
    if (checked != BS_OK) return checked;
    if (desc->rows == 0) return BS_OK;
    const bool held = x_codes != nullptr, gated = gate || gate_codes;
    if (!grad_y || !x == !held || !x_codes != !x_exponents || !gate_codes != !gate_exponents || (gated && !gate == !held) || (gate && gate_codes) ||
        (grad_gate && !gated))
        return BS_ERR_NULL;
    if (!grad_x && !grad_gate) return BS_OK;
    ActivateK k{};
    k.x = row_tensor(x, desc->x_stride, desc->columns);
    k.gate = row_tensor(gate, desc->gate_stride, desc->columns);
    k.dy = row_tensor(grad_y, desc->grad_y_stride, desc->columns);
    k.dx = row_tensor(grad_x, desc->grad_x_stride, desc->columns);
    k.dg = row_tensor(grad_gate, desc->grad_gate_stride, desc->columns);
    k.hx = HeldRows{const_cast<int8_t *>(x_codes), const_cast<uint8_t *>(x_exponents)};
    k.hg = HeldRows{const_cast<int8_t *>(gate_codes), const_cast<uint8_t *>(gate_exponents)};
    const Bytes b{(uint64_t)desc->rows, (uint64_t)desc->columns, dtype_size(desc->dtype)};
    for (const void *p : {x, gate, grad_y, (const void *)grad_x, (const void *)grad_gate})
        if (!aligned_to(p, b.es)) return BS_ERR_ALIGN;
    const bs_status alias = check_overlap({b(k.x), b(k.gate), b(k.dy), b.codes(x_codes), b.exponents(x_exponents), b.codes(gate_codes), b.exponents(gate_exponents)},
                                          {b(k.dx), b(k.dg)});
    if (alias != BS_OK) return alias;
    fill(k, desc->rows, desc->columns, desc->dtype);
    return launch_rows(ROWS_ACTIVATE_GRAD, k, desc->dtype, desc->activation, stream);
}

}  // extern "C"
