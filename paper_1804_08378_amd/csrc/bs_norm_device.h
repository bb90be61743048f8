// Device code shared by the group-normalisation kernels: activations and their slopes, access to pixels, parameters.
#pragma once

#include "bs_device.h"
#include "bs_norm.h"

namespace bs {

// ------------------------------------------------------------------------------------------------ activations
// exp for float32 results: the product with log2(e) in two parts, so that large arguments keep their last bits.
BS_DEV float exp_exact(float v)
{
    const float hi = v * 1.44269504088896341f;
    const float lo = __builtin_fmaf(v, 1.44269504088896341f, -hi) + v * 1.92596299112661746e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fabsf(hi) < 160.0f ? __builtin_fmaf(e, lo * 0.693147180559945309f, e) : e;  // (beyond: 0, infinity or NaN)
}

// 16-bit results hide the last bits of the exponential and of the reciprocal; float32 ones do not.
template <int DT>
BS_DEV float sigmoid(float z)
{
    if constexpr (DT == DT_F32) return 1.0f / (1.0f + exp_exact(-z));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
}

template <int DT, int ACT>
BS_DEV float act(float z)
{
    if constexpr (ACT == BS_ACT_RELU) return z > 0.0f ? z : 0.0f;
    if constexpr (ACT == BS_ACT_SILU) return z * sigmoid<DT>(z);
    if constexpr (ACT == BS_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.707106781186547524f));
    return z;
}

template <int DT, int ACT>
BS_DEV float act_slope(float z)
{
    if constexpr (ACT == BS_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BS_ACT_SILU) {
        const float s = sigmoid<DT>(z);
        return s * (1.0f + z * (1.0f - s));
    }
    if constexpr (ACT == BS_ACT_GELU) {
        const float phi = 0.398942280401432678f * exp_exact(-0.5f * z * z);
        return 0.5f * (1.0f + erff(z * 0.707106781186547524f)) + z * phi;
    }
    return 1.0f;
}

template <int DT>
BS_DEV const char *at_pixel(const NormTensor &t, uint32_t P, uint32_t n, uint32_t p, uint32_t c)
{
    return static_cast<const char *>(t.p) + (((uint64_t)n * P + p) * t.stride + c) * (DT != DT_F32 ? 2 : 4);
}

template <int DT, int VEC>
BS_DEV void load_vec(const char *p, float (&v)[VEC])
{
    unpack<DT, VEC>(load_raw<DT, VEC>(p, 0), v);
}

// Parameters of VEC channels from c on, `none` where there are none.  128-bit loads need no more than the element's alignment here.
template <int DT, int VEC>
BS_DEV void load_params(const void *p, bool f32, uint32_t c, float none, float (&v)[VEC])
{
    struct __attribute__((packed, aligned(4))) Floats { float f[VEC]; };
    struct __attribute__((packed, aligned(2))) Halves { uint16_t h[VEC]; };
    if (!p) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = none;
    } else if (DT == DT_F32 || f32) {
        const Floats t = *reinterpret_cast<const Floats *>(static_cast<const float *>(p) + c);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = t.f[i];
    } else {
        const Halves t = *reinterpret_cast<const Halves *>(static_cast<const uint16_t *>(p) + c);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = half_up<DT>(t.h[i]);
    }
}

}  // namespace bs
