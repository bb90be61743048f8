// Layer normalisation with a row in the registers of a team of lanes: device code that both directions share.
//
// A team of TEAM lanes (a part of a wave, a wave, or several waves) holds a row, a vector of 128 bits a lane up to 1024 lanes, NV of them in longer rows, so
// that every tensor crosses memory once, and has the next row's vectors under way while it works on this one.  Weight and bias of a lane's columns stay
// in its registers from row to row.  Memory bounds it: 8192 x 4096 bfloat16 behind an addition 43 us (6.3 TB/s; a copy 6.6), 200704 x 256
// forward 37 and backward 52 us (5.5, 6.0), 16384 x 2048 through 8 bits 51 and 48 (5.9, 4.9), 8192 x 1024 float32 12 and 17.4 (5.6, 5.8).  What made it so,
// same cases: no load behind a condition (backward 57 -> 46, 20 -> 17.5); a row's last vector as one whole load that ends with the row (20000 x 771
// binary16 forward 50 -> 31); numbers made of their words anew for every use (64 registers forward, 8 waves a SIMD).  More vectors a lane for
// fewer lanes (64 x 4, 256 x 2) took 160 to 256 registers, and neighbouring rows for a work-group instead of strided ones cost 200704 x 256 forward 7 us.
#pragma once

#include "bs_layer_norm.h"
#include "bs_rows8_device.h"

namespace bs {

// A lane's team in a work-group of T lanes: in a scalar register, as its rows' addresses then, where a wave has one team only.
template <int TEAM, int T>
BS_DEV uint32_t team_of()
{
    if constexpr (TEAM == T) return 0;
    if constexpr (TEAM >= 64) return (uint32_t)__builtin_amdgcn_readfirstlane((int)(threadIdx.x / TEAM));
    return threadIdx.x / TEAM;
}

// Gradients of one column's bias and weight.
template <int DT>
BS_DEV void put_params(const LayerNormK &k, uint32_t c, float b, float w)
{
    auto put = [&](void *p, float v) {
        if (!p) return;
        if (DT == DT_F32 || k.f32_params) static_cast<float *>(p)[c] = v;
        else static_cast<uint16_t *>(p)[c] = half_bits<DT>(v);
    };
    put(k.dbias, b);
    put(k.dweight, w);
}

// Between two uses of words: the numbers are made of them anew, which is cheaper than the registers that would keep them.
BS_DEV void forget(uint4 &q) { asm("" : "+v"(q.x), "+v"(q.y), "+v"(q.z), "+v"(q.w)); }

// A number that the compiler takes for another one at every use: what is read at it is not kept in registers from row to row.
BS_DEV uint32_t afresh(uint32_t c)
{
    asm volatile("" : "+v"(c));
    return c;
}

// Sums over rows of lanes by exchanges inside the wave.
BS_DEV float half_wave_sum(float v)  // of rows of 16 lanes that hold one value each: over a half wave
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    const u2 r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}
BS_DEV float both_halves_sum(float v)
{
    typedef uint32_t u2 __attribute__((ext_vector_type(2)));
    const u2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}
// Over N neighbouring lanes, the same in each of them.
template <int N>
BS_DEV float lanes_sum(float v)
{
    if constexpr (N >= 2) v += __uint_as_float(swapped<K_SWAP1>(__float_as_uint(v)));
    if constexpr (N >= 4) v += __uint_as_float(swapped<K_SWAP2>(__float_as_uint(v)));
    if constexpr (N >= 8) v += __uint_as_float(swapped<K_MIRROR8>(__float_as_uint(v)));
    if constexpr (N >= 16) v += __uint_as_float(swapped<K_MIRROR16>(__float_as_uint(v)));
    if constexpr (N >= 32) v = half_wave_sum(v);
    if constexpr (N >= 64) v = both_halves_sum(v);
    return v;
}
// The other direction: over lanes of the same place in teams of N lanes, the same in each of them.
template <int N>
BS_DEV float teams_sum(float v)
{
    static_assert(N >= 8, "rows of 16 lanes hold two teams at most");
    if constexpr (N == 8) v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x128, 0xf, 0xf, false));  // row_ror:8
    if constexpr (N <= 16) v = half_wave_sum(v);
    if constexpr (N <= 32) v = both_halves_sum(v);
    return v;
}

}  // namespace bs
