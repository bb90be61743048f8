// The exponential of the operators whose results are float32.
#pragma once

#include "bs_device.h"

namespace bs {

// The product with log2(e) in two parts, so that large arguments keep their last bits.  The second part corrects a finite power only: of an
// infinite one it would make NaN.
BS_DEV float exp_exact(float v)
{
    const float hi = v * 1.44269504088896341f;
    const float lo = __builtin_fmaf(v, 1.44269504088896341f, -hi) + v * 1.92596299112661746e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fabsf(hi) < 128.0f ? __builtin_fmaf(e, lo * 0.693147180559945309f, e) : e;  // (beyond: under 2^-128, 0, infinity or NaN)
}

}  // namespace bs
