// Device code shared by the kernels over rows: access at any alignment, blocks of 32 elements in 8 bits, sums over lanes.
#pragma once

#include "bs_device.h"
#include "bs_rows_args.h"

namespace bs {

// Elements of a lane's vector: 128 bits of a tensor, and how many lanes share a block.
template <int DT>
constexpr int K_VEC = DT == DT_F32 ? 4 : 8;
template <int DT>
constexpr int K_BLOCK_LANES = BS_PACK8_BLOCK / K_VEC<DT>;
template <int DT>
constexpr int K_ES = DT == DT_F32 ? 4 : 2;

// ------------------------------------------------------------------------------------------------ access
// VEC elements of a row from column c on; columns from `columns` on are 0 and are not read.  Rows may begin at any element: 128-bit accesses need no
// more than the element's alignment.
template <int DT>
BS_DEV void load_cols(const char *row, uint32_t c, uint32_t columns, float (&v)[K_VEC<DT>])
{
    typedef uint32_t u4 __attribute__((ext_vector_type(4)));
    const char *p = row + (uint64_t)c * K_ES<DT>;
    Raw<DT, K_VEC<DT>> r;
    r.q = make_uint4(0, 0, 0, 0);
    if (c + K_VEC<DT> <= columns) {
        const u4 t = *reinterpret_cast<const typename AtMultiplesOf<u4, K_ES<DT>>::type *>(p);
        r.q = make_uint4(t.x, t.y, t.z, t.w);
        unpack<DT, K_VEC<DT>>(r, v);
    } else {
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i) {
            v[i] = 0.0f;
            if (c + i < columns) {
                if constexpr (DT == DT_F32) v[i] = reinterpret_cast<const float *>(p)[i];
                else v[i] = half_up<DT>(reinterpret_cast<const uint16_t *>(p)[i]);
            }
        }
    }
}

template <int DT>
BS_DEV void store_cols(char *row, uint32_t c, uint32_t columns, const float (&v)[K_VEC<DT>])
{
    char *p = row + (uint64_t)c * K_ES<DT>;
    if (c + K_VEC<DT> <= columns) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == DT_F32) w[i] = __float_as_uint(v[i]);
            else w[i] = pack2<DT>(v[2 * i], v[2 * i + 1]);
        }
        store_words<4, K_ES<DT>, true>(p, w);
    } else {
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i)
            if (c + i < columns) {
                if constexpr (DT == DT_F32) reinterpret_cast<float *>(p)[i] = v[i];
                else reinterpret_cast<uint16_t *>(p)[i] = half_bits<DT>(v[i]);
            }
    }
}

// Parameters of a lane's columns, `none` where there are none and 0 behind the last column.
template <int DT>
BS_DEV void load_row_params(const void *p, bool f32, uint32_t c, uint32_t columns, float none, float (&v)[K_VEC<DT>])
{
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        v[i] = 0.0f;
        if (c + i < columns) {
            if (!p) v[i] = none;
            else if (DT == DT_F32 || f32) v[i] = static_cast<const float *>(p)[c + i];
            else v[i] = half_up<DT>(static_cast<const uint16_t *>(p)[c + i]);
        }
    }
}

// ------------------------------------------------------------------------------------------------ 8 bits
template <int CTRL>
BS_DEV uint32_t swapped(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
}
constexpr int K_SWAP1 = 0xb1, K_SWAP2 = 0x4e, K_MIRROR8 = 0x141, K_MIRROR16 = 0x140;  // quad_perm, row_half_mirror, row_mirror

constexpr uint32_t K_INF = 0x7f800000u;

// A lane's part of a block as codes, and the block's exponent.  All lanes of the block call it, columns behind the row's last hold 0.
template <int DT>
BS_DEV uint32_t to_8_bits(const float (&v)[K_VEC<DT>], uint32_t (&codes)[K_VEC<DT> / 4])
{
    uint32_t top = 0, all = 0;
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        top = max(top, b < K_INF ? b : 0u);
        all = max(all, b);
    }
    top = max(top, swapped<K_SWAP1>(top));
    top = max(top, swapped<K_SWAP2>(top));
    if constexpr (K_BLOCK_LANES<DT> == 8) top = max(top, swapped<K_MIRROR8>(top));
    const uint32_t e = min((top + 0x30000u) >> 23, DT == DT_F16 ? 142u : 254u);
    const int shift = 133 - (int)e;
#pragma unroll
    for (int w = 0; w < K_VEC<DT> / 4; ++w) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float q = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[4 * w + i], shift), -126.0f, 126.0f);
            b[i] = __float_as_uint(q + 12582912.0f) & 0xffu;  // 1.5 * 2^23 in front: the sum's last bits are the number rounded, ties to even
        }
        codes[w] = b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24;
    }
    if (all >= K_INF) {
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i) {
            const uint32_t b = __float_as_uint(v[i]), m = b & 0x7fffffffu, at = 8 * (i % 4);
            const uint32_t code = m > K_INF ? 0x80u : b == m ? 0x7fu : 0x81u;
            if (m >= K_INF) codes[i / 4] = (codes[i / 4] & ~(0xffu << at)) | code << at;
        }
    }
    return e;
}

template <int DT>
BS_DEV void from_8_bits(const uint32_t (&codes)[K_VEC<DT> / 4], uint32_t e, float (&v)[K_VEC<DT>])
{
    const float step = __builtin_amdgcn_ldexpf(1.0f, (int)e - 133);
    float n[K_VEC<DT>], most = 0.0f;
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        n[i] = (float)(int)(int8_t)(codes[i / 4] >> (8 * (i % 4)));
        most = __builtin_fmaxf(most, __builtin_fabsf(n[i]));
        v[i] = n[i] * step;
    }
    if (most >= 127.0f) {
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i)
            if (__builtin_fabsf(n[i]) >= 127.0f) v[i] = __uint_as_float(n[i] == 127.0f ? K_INF : n[i] == -127.0f ? K_INF | 0x80000000u : 0x7fc00000u);
    }
}

template <int DT>
BS_DEV void store_codes(int8_t *row, uint32_t c, uint32_t columns, const uint32_t (&codes)[K_VEC<DT> / 4])
{
    char *p = reinterpret_cast<char *>(row) + c;
    if (c + K_VEC<DT> <= columns) {
        store_words<K_VEC<DT> / 4, 1, true>(p, codes);
    } else {
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i)
            if (c + i < columns) p[i] = (char)(codes[i / 4] >> (8 * (i % 4)));
    }
}

template <int DT>
BS_DEV void load_codes(const int8_t *row, uint32_t c, uint32_t columns, uint32_t (&codes)[K_VEC<DT> / 4])
{
    constexpr int N = K_VEC<DT> / 4;
    const char *p = reinterpret_cast<const char *>(row) + c;
    if (c + K_VEC<DT> <= columns) {
        using V = typename WordsOf<N>::type;
        const V t = *reinterpret_cast<const typename AtMultiplesOf<V, 1>::type *>(p);
        if constexpr (N == 1) {
            codes[0] = t;
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) codes[i] = t[i];
        }
    } else {
#pragma unroll
        for (int w = 0; w < N; ++w) codes[w] = 0;
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i)
            if (c + i < columns) codes[i / 4] |= (uint32_t)(uint8_t)p[i] << (8 * (i % 4));
    }
}

// A lane's vector of a row held in 8 bits, as numbers (0 behind the last column).
template <int DT>
BS_DEV void load_held(const HeldRows &h, uint64_t row, uint32_t c, uint32_t columns, float (&v)[K_VEC<DT>])
{
    uint32_t codes[K_VEC<DT> / 4];
    load_codes<DT>(h.codes + row * columns, c, columns, codes);
    const uint32_t blocks = (columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK;
    const uint32_t e = c < columns ? h.exponents[row * blocks + c / BS_PACK8_BLOCK] : 0u;
    from_8_bits<DT>(codes, e, v);
}

// The other way: all lanes of a block call it together.
template <int DT>
BS_DEV void store_held(const HeldRows &h, uint64_t row, uint32_t c, uint32_t columns, const float (&v)[K_VEC<DT>])
{
    uint32_t codes[K_VEC<DT> / 4];
    const uint32_t e = to_8_bits<DT>(v, codes);
    store_codes<DT>(h.codes + row * columns, c, columns, codes);
    const uint32_t blocks = (columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK;
    if (c < columns && c % BS_PACK8_BLOCK == 0) h.exponents[row * blocks + c / BS_PACK8_BLOCK] = (uint8_t)e;
}

// ------------------------------------------------------------------------------------------------ sums
BS_DEV float lane_swapped_sum(float v)  // over rows of 16 lanes, the same in each of them
{
    v += __uint_as_float(swapped<K_SWAP1>(__float_as_uint(v)));
    v += __uint_as_float(swapped<K_SWAP2>(__float_as_uint(v)));
    v += __uint_as_float(swapped<K_MIRROR8>(__float_as_uint(v)));
    return v + __uint_as_float(swapped<K_MIRROR16>(__float_as_uint(v)));
}
BS_DEV float wave_sum(float v)  // over the 64 lanes of a wave, the same in each
{
    const int n = __float_as_int(lane_swapped_sum(v));
    return (__int_as_float(__builtin_amdgcn_readlane(n, 0)) + __int_as_float(__builtin_amdgcn_readlane(n, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(n, 32)) + __int_as_float(__builtin_amdgcn_readlane(n, 48)));
}
// Over a work-group of T lanes.  lds: T / 64 floats of this sum alone; all lanes call it.
template <int T>
BS_DEV float group_sum(float v, float *lds)
{
    v = wave_sum(v);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < T / 64; ++i) s += lds[i];
    return s;
}

}  // namespace bs
