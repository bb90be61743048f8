// Device code shared by the group-normalisation kernels: activations and their slopes, access to pixels, parameters.
#pragma once

#include "bs_device.h"
#include "bs_exp_device.h"
#include "bs_norm.h"

namespace bs {

// ------------------------------------------------------------------------------------------------ activations
// 16-bit results hide the last bits of the exponential and of the reciprocal; float32 ones do not.
template <int DT>
BS_DEV float sigmoid(float z)
{
    if constexpr (DT == DT_F32) return 1.0f / (1.0f + exp_exact(-z));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f));
}

// The normal distribution function and its derivative times z.  16-bit results: the complementary error function by the rational approximation
// of Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26 (absolute error 1.5e-7, the exponential shared with the density; of GELU
// a tenth of a unit in binary16's last place above -3, up to one unit between -5 and -3, under a unit of bfloat16's above -6):
// both directions of 32x64x68x68 bfloat16 in 8 groups 72.6 us with erff.
template <int DT>
BS_DEV float normal(float z, float &density_z)
{
    if constexpr (DT == DT_F32) {
        density_z = z * (0.398942280401432678f * exp_exact(-0.5f * z * z));
        return 0.5f * (1.0f + erff(z * 0.707106781186547524f));
    } else {
        const float x = __builtin_fabsf(z) * 0.707106781186547524f;
        const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(x, 0.3275911f, 1.0f)), e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
        float p = __builtin_fmaf(t, 1.061405429f, -1.453152027f);
        p = __builtin_fmaf(t, p, 1.421413741f);
        p = __builtin_fmaf(t, p, -0.284496736f);
        p = __builtin_fmaf(t, p, 0.254829592f);
        const float tail = 0.5f * e * t * p;
        density_z = z * (0.398942280401432678f * e);
        return z < 0.0f ? tail : 1.0f - tail;
    }
}

template <int DT, int ACT>
BS_DEV float act(float z)
{
    if constexpr (ACT == BS_ACT_RELU) return z > 0.0f ? z : 0.0f;
    if constexpr (ACT == BS_ACT_SILU) return z * sigmoid<DT>(z);
    if constexpr (ACT == BS_ACT_GELU) {
        float unused;
        return z * normal<DT>(z, unused);
    }
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
        float density_z;
        const float below = normal<DT>(z, density_z);
        return below + density_z;
    }
    return 1.0f;
}

// ------------------------------------------------------------------------------------------------ access
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
