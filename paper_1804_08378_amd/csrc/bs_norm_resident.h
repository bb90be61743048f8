// Group normalisation with the tensor resident in registers: what the forward and the backward kernel share.
//
// A work-group owns a pixel chunk of one channel block (whole groups) of one image and loads it once, a vector of channels a lane and pixel, all
// loads in flight together.  It reduces its part of each group's sums, publishes them as one 64-bit word a group, and waits for the words of
// the image's other chunks.  Then it finishes its pixels from registers: every tensor crosses memory once (statistics first and the tensor once
// more moves 4 tensors instead of 3 forward with a residual operand, 8 instead of 5 backward: 64x256x56x56 bfloat16, 88 and 147 us against 76 and
// 115, clearing launch included).
//
// What bounds it: two work-groups of 512 lanes share a compute unit, and of a work-group's 17 us 9 go by until its bursts have come (two thirds of
// the chip's rate), 4 with the sums, 2 with the exchange, 2 with the results.  The same loads and stores without any sums take 60 us forward
// at that size, of 71.  Work-groups of 256 lanes, delayed starts, non-temporal loads, a full last round and wider channel blocks change nothing.
//
// The wait ends by itself: after a number of polls a work-group that still misses a word computes that chunk's sums itself, from memory, by
// the same code and so to the same bits.  Nothing therefore depends on how many work-groups run at the same time or in which order they start.
#pragma once

#include <type_traits>

#include "bs_norm_device.h"

namespace bs {

constexpr int RT = K_NORM_RESIDENT_THREADS;
constexpr uint64_t ABSENT = 0;  // what a word holds before it is published: words are stored with all bits turned

BS_DEV uint64_t word_of(float a, float b)
{
    const uint64_t w = ~((uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a));
    return w == ABSENT ? ~0x7fc000007fc00000ull : w;  // (two NaN, whatever their bits)
}
BS_DEV float word_low(uint64_t w) { return __uint_as_float(~(uint32_t)w); }
BS_DEV float word_high(uint64_t w) { return __uint_as_float(~(uint32_t)(w >> 32)); }

// Where a work-group and a lane stand.
struct Spot {
    uint32_t n, chunk, b0;      // image, pixel chunk, first channel
    uint32_t g0;                // first group
    uint32_t cvi, pl, lanes;    // channel vector in the block, pixel lane, pixel lanes of the work-group
    bool on;

    template <int VEC>
    static BS_DEV Spot of(const NormK &k)
    {
        Spot s;
        const uint32_t rest = fdiv(blockIdx.x, k.by_chunks);
        s.chunk = blockIdx.x - rest * k.chunks;
        s.n = fdiv(rest, k.by_blocks);
        const uint32_t block = rest - s.n * k.blocks;
        s.b0 = block * k.block;
        s.g0 = block * k.groups;
        s.lanes = k.lanes;
        s.pl = fdiv(threadIdx.x, k.by_cvb);
        s.cvi = threadIdx.x - s.pl * k.by_cvb.d;
        s.on = s.pl < s.lanes;
        return s;
    }
};

// A pixel chunk: its first pixel and size; lane pl has pixels p0 + pl + u * lanes, `each` of them and one more for the first `more` lanes.
struct Chunk {
    uint32_t p0, pixels, each, more;
    BS_DEV Chunk(const NormK &k, uint32_t q)
    {
        p0 = q * k.chunk;
        const bool last = q + 1 == k.chunks;
        pixels = last ? k.last : k.chunk;
        each = last ? k.last_each : k.chunk_each;
        more = pixels - each * k.lanes;
    }
    BS_DEV uint32_t of_lane(uint32_t pl) const { return each + (pl < more); }
};

// The lane's pixels of a chunk.
template <int DT, int VEC, int E>
struct Pixels {
    Raw<DT, VEC> raw[E];

    BS_DEV void load(const NormTensor &t, const NormK &k, const Spot &s, const Chunk &q, uint32_t mine)
    {
        const char *src = at_pixel<DT>(t, k.P, s.n, q.p0 + s.pl, s.b0 + s.cvi * VEC);
        const uint64_t step = (uint64_t)s.lanes * t.stride * (DT != DT_F32 ? 2 : 4);
#pragma unroll
        for (int u = 0; u < E; ++u)
            if (u < (int)mine) raw[u] = load_raw<DT, VEC>(src + u * step, 0);
    }
    // What comes behind unpacks the pixels again: the compiler would keep them unpacked, twice the registers, and spill.
    BS_DEV void forget()
    {
#pragma unroll
        for (int u = 0; u < E; ++u) {
            if constexpr (sizeof(raw[u].q) == 16) asm volatile("" : "+v"(raw[u].q.x), "+v"(raw[u].q.y), "+v"(raw[u].q.z), "+v"(raw[u].q.w));
            else if constexpr (sizeof(raw[u].q) == 8) asm volatile("" : "+v"(raw[u].q.x), "+v"(raw[u].q.y));
            else asm volatile("" : "+v"(raw[u].q));
        }
    }
};

// Sums over 16 neighbouring lanes, in each of them; the lanes of a row meet in a different order but in the same pairs.
BS_DEV float sum16(float v)
{
    auto moved = [](float x, auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xf, 0xf, false));
    };
    v += moved(v, std::integral_constant<int, 0xb1>());   // quad_perm 1 0 3 2
    v += moved(v, std::integral_constant<int, 0x4e>());   // quad_perm 2 3 0 1
    v += moved(v, std::integral_constant<int, 0x141>());  // row_half_mirror
    v += moved(v, std::integral_constant<int, 0x140>());  // row_mirror
    return v;
}

// Columns in LDS: every pixel lane has NV values for its channel vector, cols = cvb * NV columns of `lanes` rows.  The rows are joined in
// two steps, about the square root of them each: a thread takes every slices-th row of one column, then the slices are joined.
template <int NV>
BS_DEV void put_columns(const NormK &k, const Spot &s, const float (&v)[NV], float *columns)
{
    if (!s.on) return;
    float *mine = columns + s.pl * (k.by_cvb.d * NV) + s.cvi * NV;
    if constexpr (NV % 4 == 0) {
#pragma unroll
        for (int i = 0; i < NV; i += 4) *reinterpret_cast<float4 *>(mine + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i) mine[i] = v[i];
    }
}

// The first step: body(column, slice) for every pair.  Behind a barrier.
template <int NV, typename BODY>
BS_DEV void each_slice(const NormK &k, BODY body)
{
    const uint32_t cols = k.by_cvb.d * NV, slices = NV > 1 ? k.slices_wide : k.slices, slice = fdiv(threadIdx.x, NV > 1 ? k.by_cols_wide : k.by_cvb);
    if (slice < slices)
        for (uint32_t c = threadIdx.x - slice * cols; c < cols; c += RT) body(c, slice, cols, slices);
}

// Publishes the word of group g (of the block).
BS_DEV void publish(const NormK &k, const Spot &s, uint32_t g, uint64_t w, uint64_t *words)
{
    words[g * k.chunks + s.chunk] = w;
    if (k.chunks > 1) __hip_atomic_store(k.words + ((uint64_t)s.n * k.G + s.g0 + g) * k.chunks + s.chunk, w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Collects the words of all chunks: words[g * chunks + chunk], valid behind the call.  `missing` is 0 before it (and a barrier between).
// False in every lane where some are missing after k.polls polls.
BS_DEV bool collect(const NormK &k, const Spot &s, uint64_t *words, uint32_t *missing)
{
    if (k.chunks > 1) {
        const uint64_t *all = k.words + ((uint64_t)s.n * k.G + s.g0) * k.chunks;
        const uint32_t n = k.groups * k.chunks;
        constexpr int U = 4;  // words of a thread that it looks for together
        for (uint32_t i = threadIdx.x; i < n; i += U * RT) {
            uint64_t w[U];
            bool all_there = k.polls == 0;
#pragma unroll
            for (int u = 0; u < U; ++u) w[u] = ABSENT;
            for (uint32_t polls = 0; polls < k.polls && !all_there; ++polls) {
                if (polls) __builtin_amdgcn_s_sleep(2);
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (w[u] == ABSENT && i + u * RT < n) w[u] = __hip_atomic_load(all + i + u * RT, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                all_there = true;
#pragma unroll
                for (int u = 0; u < U; ++u) all_there = all_there && (w[u] != ABSENT || i + u * RT >= n);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i + u * RT >= n) break;
                if (w[u] != ABSENT) words[i + u * RT] = w[u];
                else *missing = 1;  // (its own word is there already)
            }
        }
        // A barrier does not wait for the waves' stores: every wave's words have to be in memory before any wave counts the work-group out.  (The
        // words are stored through the L2 caches, so that they are when the wave's count of stores is 0; a release would write back all of the L2
        // cache for them: 8x512x28x28 binary16 22.1 us.)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    __syncthreads();
    return *missing == 0;
}

// Behind collect: counts the work-group out.  The last one of a block's finds that nobody looks for its words any more, and clears them (at
// the end, off the other lanes' way).  Every wave has waited for its words' stores, and a look at a word has brought its value, before the
// barrier that collect ends with and so before the count: no word and no look comes late, whether or not the work-group went on waiting.
BS_DEV uint32_t depart(const NormK &k, const Spot &s)
{
    if (!k.departed || k.chunks == 1 || threadIdx.x != 0) return 0;
    return __hip_atomic_fetch_add(k.departed + s.n * k.blocks + s.g0 / k.groups, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
BS_DEV void clear_words(const NormK &k, const Spot &s, uint32_t before)
{
    if (!k.departed || k.chunks == 1 || threadIdx.x >= 64) return;
    if ((uint32_t)__builtin_amdgcn_readfirstlane((int)before) != k.chunks - 1) return;
    uint64_t *all = k.words + ((uint64_t)s.n * k.G + s.g0) * k.chunks;
    for (uint32_t i = threadIdx.x; i < k.groups * k.chunks; i += 64) __hip_atomic_store(all + i, ABSENT, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (threadIdx.x == 0) __hip_atomic_store(k.departed + s.n * k.blocks + s.g0 / k.groups, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

}  // namespace bs
