// Rows of elements as arguments: what the layer-normalisation, activation and 8-bit kernels and their host code share.
#pragma once

#include <cstdint>

#include "brainslug.h"
#include "bs_internal.h"
#include "bs_kargs.h"

namespace bs {

// One tensor of rows: `stride` elements from a row to the next.
struct RowTensor {
    const void *p;
    uint64_t stride;
};
// Rows in 8 bits, dense: a byte an element, a byte for every 32 of a row.
struct HeldRows {
    int8_t *codes;
    uint8_t *exponents;
};

// Sizes that every one of these calls takes.
inline bs_status check_rows(int64_t rows, int64_t columns, int32_t dtype, std::initializer_list<int64_t> strides)
{
    if (dtype != BS_F32 && dtype != BS_BF16 && dtype != BS_F16) return BS_ERR_UNSUPPORTED;
    if (rows < 0 || columns < 1) return BS_ERR_SHAPE;
    // launches count lanes in 32 bits: four or eight of them a block
    if (columns > (1ll << 30) || rows > (1ll << 28) || (double)rows * (double)((columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK) > (double)(1ll << 28)) return BS_ERR_UNSUPPORTED;
    for (const int64_t s : strides) {
        if (s != 0 && s < columns) return BS_ERR_SHAPE;
        if (s > (1ll << 40) || (double)rows * (double)s > (double)(1ll << 50)) return BS_ERR_UNSUPPORTED;
    }
    return BS_OK;
}
inline RowTensor row_tensor(const void *p, int64_t stride, int64_t columns) { return RowTensor{p, (uint64_t)(stride ? stride : columns)}; }

inline bool aligned_to(const void *p, uint64_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

inline TensorBytes bytes_of(const RowTensor &t, uint64_t rows, uint64_t columns, uint64_t es) { return TensorBytes{t.p, rows, columns * es, t.stride * es}; }
inline TensorBytes bytes_of(const void *p, uint64_t n) { return TensorBytes{p, 1, n, n}; }

// No output shares a byte with an input or another output.
inline bs_status check_overlap(std::initializer_list<TensorBytes> in, std::initializer_list<TensorBytes> out)
{
    for (const TensorBytes *o = out.begin(); o != out.end(); ++o) {
        if (!o->p || !o->image_bytes) continue;
        for (const TensorBytes &t : in)
            if (t.p && t.image_bytes && tensors_overlap(*o, t)) return BS_ERR_ALIAS;
        for (const TensorBytes *q = out.begin(); q != o; ++q)
            if (q->p && q->image_bytes && tensors_overlap(*o, *q)) return BS_ERR_ALIAS;
    }
    return BS_OK;
}

inline uint64_t blocks_of(uint64_t columns) { return (columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK; }

}  // namespace bs
