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
template <int DT>
BS_DEV const char *row_of(const RowTensor &t, uint64_t row) { return static_cast<const char *>(t.p) + row * t.stride * K_ES<DT>; }

// Rows may begin at any element: accesses of up to 128 bits need no more than the element's alignment.
template <int N, int A>
BS_DEV void load_words(const char *p, uint32_t (&w)[N])
{
    using V = typename WordsOf<N>::type;
    const V t = *reinterpret_cast<const typename AtMultiplesOf<V, A>::type *>(p);
    if constexpr (N == 1) {
        w[0] = t;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = t[i];
    }
}

// The first `n` of the elements of E bytes that N words hold (not all of them), the others 0: a load for every bit of n, largest first.  (Words are
// chosen by masks: of conditions between elements of an array the compiler makes indexes, and puts the array into memory for them.)
BS_DEV uint32_t mask_if(bool b) { return 0u - (uint32_t)b; }
template <int N, int E>
BS_DEV void load_first(const char *p, uint32_t n, uint32_t (&w)[N])
{
    const uint32_t bytes = n * E;
    uint32_t at = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = 0;
    if constexpr (N > 4)
        if (bytes & 16) {
            uint32_t t[4];
            load_words<4, E>(p, t);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = t[i];
            at = 16;
        }
    if constexpr (N > 2)
        if (bytes & 8) {
            uint32_t t[2];
            load_words<2, E>(p + at, t);
#pragma unroll
            for (int i = 0; i < N; i += 4)
#pragma unroll
                for (int m = 0; m < 2; ++m) w[i + m] |= t[m] & mask_if(at == 4 * (uint32_t)i);
            at += 8;
        }
    if constexpr (N > 1)
        if (bytes & 4) {
            uint32_t t[1];
            load_words<1, E>(p + at, t);
#pragma unroll
            for (int i = 0; i < N; i += 2) w[i] |= t[0] & mask_if(at == 4 * (uint32_t)i);
            at += 4;
        }
    if constexpr (E <= 2)
        if (bytes & 2) {
            uint32_t t;
            if constexpr (E == 2) t = *reinterpret_cast<const uint16_t *>(p + at);
            else t = (uint32_t)(uint8_t)p[at] | (uint32_t)(uint8_t)p[at + 1] << 8;
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] |= t & mask_if(at == 4 * (uint32_t)i);
            at += 2;
        }
    if constexpr (E == 1)
        if (bytes & 1) {
            const uint32_t t = (uint32_t)(uint8_t)p[at] << (8 * (at & 2));
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] |= t & mask_if(at / 4 == (uint32_t)i);
        }
}

template <int N>
BS_DEV uint32_t word_at(const uint32_t (&w)[N], uint32_t at)
{
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) t |= w[i] & mask_if(at / 4 == (uint32_t)i);
    return t;
}
// The other way: nothing behind the n-th element is written.
template <int N, int E>
BS_DEV void store_first(char *p, uint32_t n, const uint32_t (&w)[N])
{
    const uint32_t bytes = n * E;
    uint32_t at = 0;
    if constexpr (N > 2)
        if (bytes & 8) {
            const uint32_t t[2] = {w[0], w[1]};
            store_words<2, E, false>(p, t);
            at = 8;
        }
    if constexpr (N > 1)
        if (bytes & 4) {
            const uint32_t t[1] = {word_at(w, at)};
            store_words<1, E, false>(p + at, t);
            at += 4;
        }
    if constexpr (E <= 2)
        if (bytes & 2) {
            const uint32_t t = word_at(w, at);
            if constexpr (E == 2) {
                *reinterpret_cast<uint16_t *>(p + at) = (uint16_t)t;
            } else {
                p[at] = (char)t;
                p[at + 1] = (char)(t >> 8);
            }
            at += 2;
        }
    if constexpr (E == 1)
        if (bytes & 1) p[at] = (char)(word_at(w, at) >> (8 * (at & 2)));
}

// A lane's vector of a row as it stands in memory.  The row's last vector, where it is not whole, is the whole one that ends with the row, so that it is
// one load whose result nothing waits for here; `settled` moves its columns to their places, with 0 behind the last.  (Rows shorter than a vector
// are read in pieces; lanes behind the last column read nothing and hold 0.)
template <int DT>
BS_DEV Raw<DT, K_VEC<DT>> load_vector(const char *row, uint32_t c, uint32_t columns)
{
    uint32_t w[4] = {};
    if (columns >= K_VEC<DT>) {
        if (c < columns) load_words<4, K_ES<DT>>(row + (uint64_t)min(c, columns - K_VEC<DT>) * K_ES<DT>, w);
    } else if (c < columns) {
        load_first<4, K_ES<DT>>(row + (uint64_t)c * K_ES<DT>, columns - c, w);
    }
    Raw<DT, K_VEC<DT>> r;
    r.q = make_uint4(w[0], w[1], w[2], w[3]);
    return r;
}
// Elements by which a lane's vector began early, `VEC` of a lane behind the last column: none of its elements is of the row.
template <int VEC>
BS_DEV uint32_t early_by(uint32_t c, uint32_t columns)
{
    return columns >= VEC && c + VEC > columns ? min(c + VEC - columns, (uint32_t)VEC) : 0;
}
template <int DT>
BS_DEV Raw<DT, K_VEC<DT>> moved(const Raw<DT, K_VEC<DT>> &r, uint32_t early)
{
    const uint32_t by = early * K_ES<DT> * 8;  // bits
    uint64_t lo = (uint64_t)r.q.y << 32 | r.q.x, hi = (uint64_t)r.q.w << 32 | r.q.z;
    lo = by & 64 ? hi : lo;
    hi = by & (64 | 128) ? 0 : hi;
    lo = by & 128 ? 0 : lo;
    lo = lo >> (by & 63) | (hi << 1) << (63 - (by & 63));
    hi >>= by & 63;
    Raw<DT, K_VEC<DT>> s;
    s.q = make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
    return s;
}
// The same of rows of a vector at least, where every lane reads one, so that no load stands behind a condition: the compiler counts the loads in flight,
// and waits for all of them where it cannot.  `moved` by `early_by` puts the columns to their places.
template <int DT>
BS_DEV uint32_t read_column(uint32_t c, uint32_t columns) { return min(c, columns - K_VEC<DT>); }
template <int DT>
BS_DEV Raw<DT, K_VEC<DT>> read_vector(const RowTensor &t, uint64_t row, uint32_t at)
{
    uint32_t w[4];
    load_words<4, K_ES<DT>>(row_of<DT>(t, row) + (uint64_t)at * K_ES<DT>, w);
    Raw<DT, K_VEC<DT>> r;
    r.q = make_uint4(w[0], w[1], w[2], w[3]);
    return r;
}
template <int DT>
BS_DEV Raw<DT, K_VEC<DT>> settled(const Raw<DT, K_VEC<DT>> &r, uint32_t c, uint32_t columns)
{
    return columns % K_VEC<DT> == 0 ? r : moved<DT>(r, early_by<K_VEC<DT>>(c, columns));  // (the same for all lanes)
}
template <int DT, bool NT = true>
BS_DEV void store_vector(char *row, uint32_t c, uint32_t columns, const Raw<DT, K_VEC<DT>> &r)
{
    char *p = row + (uint64_t)c * K_ES<DT>;
    const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
    if (c + K_VEC<DT> <= columns) store_words<4, K_ES<DT>, NT>(p, w);
    else if (c < columns) store_first<4, K_ES<DT>>(p, columns - c, w);
}

// Numbers rounded to their type.
template <int DT>
BS_DEV Raw<DT, K_VEC<DT>> to_words(const float (&v)[K_VEC<DT>])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (DT == DT_F32) w[i] = __float_as_uint(v[i]);
        else w[i] = pack2<DT>(v[2 * i], v[2 * i + 1]);
    }
    Raw<DT, K_VEC<DT>> r;
    r.q = make_uint4(w[0], w[1], w[2], w[3]);
    return r;
}

template <int DT>
BS_DEV void load_cols(const char *row, uint32_t c, uint32_t columns, float (&v)[K_VEC<DT>])
{
    unpack<DT, K_VEC<DT>>(settled<DT>(load_vector<DT>(row, c, columns), c, columns), v);
}
template <int DT, bool NT = true>
BS_DEV void store_cols(char *row, uint32_t c, uint32_t columns, const float (&v)[K_VEC<DT>])
{
    store_vector<DT, NT>(row, c, columns, to_words<DT>(v));
}

// Parameters of a lane's columns, `none` where there are none; behind the last column: any number.
template <int DT>
BS_DEV void load_row_params(const void *p, bool f32, uint32_t c, uint32_t columns, float none, float (&v)[K_VEC<DT>])
{
    constexpr int VEC = K_VEC<DT>;
    if (!p) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = none;
    } else if (DT == DT_F32 || f32) {
        struct __attribute__((packed, aligned(4))) Floats { float f[VEC]; };
        const float *q = static_cast<const float *>(p) + c;
        if (c + VEC <= columns) {
            const Floats t = *reinterpret_cast<const Floats *>(q);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = t.f[i];
        } else {
            uint32_t w[VEC] = {};
            if (c < columns) load_first<VEC, 4>(reinterpret_cast<const char *>(q), columns - c, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = __uint_as_float(w[i]);
        }
    } else {
        load_cols<DT>(static_cast<const char *>(p), c, columns, v);
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

// Over the lanes of a block.
template <int DT>
BS_DEV uint32_t block_max(uint32_t v)
{
    v = max(v, swapped<K_SWAP1>(v));
    v = max(v, swapped<K_SWAP2>(v));
    return K_BLOCK_LANES<DT> == 8 ? max(v, swapped<K_MIRROR8>(v)) : v;
}

// The largest magnitude of a lane's numbers as float32's bits, infinities and NaN above all others.
template <int DT>
BS_DEV uint32_t largest(const Raw<DT, K_VEC<DT>> &r)
{
    const uint32_t w[4] = {r.q.x, r.q.y, r.q.z, r.q.w};
    if constexpr (DT == DT_F32) {
        return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
    } else {  // two at a time
        typedef uint16_t h2 __attribute__((ext_vector_type(2)));
        h2 m = __builtin_bit_cast(h2, w[0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(h2, w[i] & 0x7fff7fffu));
        const uint32_t h = m.x > m.y ? m.x : m.y;
        return DT == DT_BF16 ? h << 16 : __float_as_uint(half_up<DT>(h));
    }
}

// Are there numbers in the wave that the short way does not serve?  (A branch that the compiler must not turn into choices of every lane.)
BS_DEV bool any_lane(bool b) { return __builtin_expect(__builtin_amdgcn_ballot_w64(b) != 0, 0); }

// A lane's part of a block as codes, and the block's exponent: one multiply-add an element, whose sum holds the rounded number of steps in its last byte.
// Blocks with infinities or NaN, or at the ends of float32's range, go the long way, with their wave (as a choice of every lane it took 10
// instructions an element instead of 3).  `r` and `v`: the same numbers.  All lanes of the block call it, columns behind the row's
// last hold 0.
template <int DT>
BS_DEV uint32_t to_8_bits(const Raw<DT, K_VEC<DT>> &r, const float (&v)[K_VEC<DT>], uint32_t (&codes)[K_VEC<DT> / 4])
{
    constexpr int VEC = K_VEC<DT>;
    constexpr uint32_t L = DT == DT_F16 ? 142u : 254u;
    uint32_t top = block_max<DT>(largest<DT>(r)), e = (top + 0x30000u) >> 23;
    float n[VEC];  // 1.5 * 2^23 and a number of steps: the sum's last bits are that number rounded, ties to even
    if (any_lane(e > L || (e < 6 && top != 0))) {
        asm volatile("");
        top = 0;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu;
            top = max(top, m < K_INF ? m : 0u);
        }
        top = block_max<DT>(top);
        e = min((top + 0x30000u) >> 23, L);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const uint32_t m = __float_as_uint(v[i]) & 0x7fffffffu;
            const float q = __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(v[i], 133 - (int)e), -126.0f, 126.0f);
            n[i] = 12582912.0f + (m > K_INF ? -128.0f : m < K_INF ? q : __uint_as_float(0x42fe0000u | (__float_as_uint(v[i]) & 0x80000000u)));  // (127)
        }
    } else {
        const float steps = __uint_as_float((260u - e) << 23);  // 2^(133 - e); of a block of zeros any number
#pragma unroll
        for (int i = 0; i < VEC; ++i) n[i] = __builtin_fmaf(v[i], steps, 12582912.0f);
    }
#pragma unroll
    for (int w = 0; w < VEC / 4; ++w) {
        // the lowest bytes of four numbers
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(n[4 * w + 1]), __float_as_uint(n[4 * w]), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(n[4 * w + 3]), __float_as_uint(n[4 * w + 2]), 0x04000c0cu);
        codes[w] = lo | hi;
    }
    return e;
}

template <int DT>
BS_DEV void from_8_bits(const uint32_t (&codes)[K_VEC<DT> / 4], uint32_t e, float (&v)[K_VEC<DT>])
{
    const float step = __builtin_amdgcn_ldexpf(1.0f, (int)e - 133);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        const float n = (float)(int)(int8_t)(codes[i / 4] >> (8 * (i % 4)));
        most = __builtin_fmaxf(most, __builtin_fabsf(n));
        v[i] = n * step;
    }
    if (any_lane(most >= 127.0f)) {
        asm volatile("");
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i) {
            const int n = (int)(int8_t)(codes[i / 4] >> (8 * (i % 4)));
            if (n >= 127 || n <= -127) v[i] = __uint_as_float(n == 127 ? K_INF : n == -127 ? K_INF | 0x80000000u : 0x7fc00000u);
        }
    }
}

template <int DT>
BS_DEV void store_codes(int8_t *row, uint32_t c, uint32_t columns, const uint32_t (&codes)[K_VEC<DT> / 4])
{
    char *p = reinterpret_cast<char *>(row) + c;
    if (c + K_VEC<DT> <= columns) store_words<K_VEC<DT> / 4, 1, false>(p, codes);
    else if (c < columns) store_first<K_VEC<DT> / 4, 1>(p, columns - c, codes);
}

// As load_vector and settled.
template <int DT>
BS_DEV void load_codes(const int8_t *row, uint32_t c, uint32_t columns, uint32_t (&codes)[K_VEC<DT> / 4])
{
    const char *p = reinterpret_cast<const char *>(row);
#pragma unroll
    for (int i = 0; i < K_VEC<DT> / 4; ++i) codes[i] = 0;
    if (columns >= K_VEC<DT>) {
        if (c < columns) load_words<K_VEC<DT> / 4, 1>(p + min(c, columns - K_VEC<DT>), codes);
    } else if (c < columns) {
        load_first<K_VEC<DT> / 4, 1>(p + c, columns - c, codes);
    }
}
template <int DT>
BS_DEV void move_codes(uint32_t (&codes)[K_VEC<DT> / 4], uint32_t early)
{
    uint64_t t = codes[0];
    if constexpr (K_VEC<DT> == 8) t |= (uint64_t)codes[1] << 32;
    t = early == K_VEC<DT> ? 0 : t >> (early * 8);
    codes[0] = (uint32_t)t;
    if constexpr (K_VEC<DT> == 8) codes[1] = (uint32_t)(t >> 32);
}
template <int DT>
BS_DEV void settle_codes(uint32_t (&codes)[K_VEC<DT> / 4], uint32_t c, uint32_t columns)
{
    if (columns % K_VEC<DT> != 0) move_codes<DT>(codes, early_by<K_VEC<DT>>(c, columns));
}

// A lane's vector of a row held in 8 bits: `load` and `settle` as load_vector and settled, `read` and `move` as read_vector and moved.
template <int DT>
struct HeldVector {
    uint32_t codes[K_VEC<DT> / 4], exponent;
    BS_DEV static uint64_t block_of(uint64_t row, uint32_t c, uint32_t columns)
    {
        return row * ((columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK) + min(c, columns - 1) / BS_PACK8_BLOCK;
    }
    BS_DEV void load(const HeldRows &h, uint64_t row, uint32_t c, uint32_t columns)
    {
        load_codes<DT>(h.codes + row * columns, c, columns, codes);
        exponent = h.exponents[block_of(row, c, columns)];
    }
    BS_DEV void settle(uint32_t c, uint32_t columns) { settle_codes<DT>(codes, c, columns); }
    BS_DEV void read(const HeldRows &h, uint64_t row, uint32_t c, uint32_t columns)
    {
        load_words<K_VEC<DT> / 4, 1>(reinterpret_cast<const char *>(h.codes) + row * columns + read_column<DT>(c, columns), codes);
        exponent = h.exponents[block_of(row, c, columns)];
    }
    BS_DEV void move(uint32_t early) { move_codes<DT>(codes, early); }
    BS_DEV void numbers(float (&v)[K_VEC<DT>]) const { from_8_bits<DT>(codes, exponent, v); }
};

// The other way: all lanes of a block call it together.
template <int DT>
BS_DEV void store_held(const HeldRows &h, uint64_t row, uint32_t c, uint32_t columns, const Raw<DT, K_VEC<DT>> &r, const float (&v)[K_VEC<DT>])
{
    uint32_t codes[K_VEC<DT> / 4];
    const uint32_t e = to_8_bits<DT>(r, v, codes);
    store_codes<DT>(h.codes + row * columns, c, columns, codes);
    const uint32_t blocks = (columns + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK;
    if (c < columns && c % BS_PACK8_BLOCK == 0) h.exponents[row * blocks + c / BS_PACK8_BLOCK] = (uint8_t)e;
}

// ------------------------------------------------------------------------------------------------ sums
// 1 / sqrt(v) by the instruction (a unit in the last place), which takes subnormal numbers for 0: small ones are scaled.
BS_DEV float reciprocal_root(float v)
{
    const bool small = v < 0x1p-64f;
    return __builtin_amdgcn_rsqf(small ? v * 0x1p80f : v) * (small ? 0x1p40f : 1.0f);
}
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
