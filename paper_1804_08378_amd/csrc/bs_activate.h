// Argument block of the activation and 8-bit kernels (bs_activate.hip), shared with the host code that fills it (bs_activate.cpp).
#pragma once

#include "bs_rows_args.h"

namespace bs {

constexpr int K_ACTIVATE_THREADS = 256;

struct ActivateK {
    RowTensor x, gate, y;     // y: what is written (pack8: nothing, unpack8: x)
    RowTensor dy, dx, dg;     // backward; dx.p, dg.p may be nullptr
    HeldRows hx, hg;          // forward: written; backward: read.  codes nullptr: not held
    uint64_t vectors;         // lanes' vectors of all rows
    uint32_t columns, per_row;  // vectors of a row: whole blocks
    FastDiv by_row;
};

enum RowPass { ROWS_ACTIVATE, ROWS_ACTIVATE_GRAD, ROWS_PACK8, ROWS_UNPACK8 };
bs_status launch_rows(RowPass pass, const ActivateK &k, int32_t dtype, int32_t activation, void *stream);

}  // namespace bs
