// Group normalisation, backward, with the tensors resident in registers (bs_norm_resident.h): x, the upstream gradient and the residual
// operand are read once, the gradients written once.  Sums per channel go to the workspace for the gradients of weight and bias.
#include <hip/hip_runtime.h>

#include "bs_internal.h"
#include "bs_norm_resident.h"

namespace bs {
namespace {

// Registers of a lane: its pixels of the operands, and its channels' statistics and parameters.
template <int DT, int VEC, int E, int ACT, bool RES, int NG>
struct Operands {
    Pixels<DT, VEC, E> x, dy, r;
    float mean[NG], rstd[NG], w[VEC], b[VEC];

    BS_DEV void load(const NormK &k, const Spot &s, const Chunk &q, uint32_t mine)
    {
        x.load(k.x, k, s, q, mine);
        dy.load(k.dy, k, s, q, mine);
        if constexpr (RES) r.load(k.r, k, s, q, mine);
    }
    BS_DEV void slopes(int u, float (&dz)[VEC], float (&xh)[VEC]) const
    {
        unpack<DT, VEC>(x.raw[u], xh);
        unpack<DT, VEC>(dy.raw[u], dz);
        float z[VEC] = {};
        if constexpr (RES) unpack<DT, VEC>(r.raw[u], z);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            xh[i] = (xh[i] - mean[NG > 1 ? i : 0]) * rstd[NG > 1 ? i : 0];
            dz[i] *= act_slope<DT, ACT>(__builtin_fmaf(xh[i], w[i], b[i]) + z[i]);
        }
    }
    // The lane's sums of dz and dz * xh per channel.
    BS_DEV void sums(uint32_t mine, float (&s0)[VEC], float (&s1)[VEC]) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) s0[i] = s1[i] = 0.0f;
#pragma unroll
        for (int u = 0; u < E; ++u)
            if (u < (int)mine) {
                float dz[VEC], xh[VEC];
                slopes(u, dz, xh);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    s0[i] += dz[i];
                    s1[i] = __builtin_fmaf(dz[i], xh[i], s1[i]);
                }
                __builtin_amdgcn_sched_barrier(0);  // one pixel at a time: more at once would not fit the registers
            }
    }
};

// Sums of the rows of columns a and b, in their first `slices` rows.  Behind a barrier.
template <int NV>
BS_DEV void sum_slices(const NormK &k, float *a, float *b)
{
    each_slice<NV>(k, [&](uint32_t c, uint32_t slice, uint32_t cols, uint32_t slices) {
        float t0 = 0.0f, t1 = 0.0f;
#pragma unroll 4
        for (uint32_t r = slice; r < k.lanes; r += slices) {
            t0 += a[r * cols + c];
            t1 += b[r * cols + c];
        }
        a[slice * cols + c] = t0;  // (no other thread reads this row of the column)
        b[slice * cols + c] = t1;
    });
}

// The words of a chunk's groups, sums of dz * weight and dz * weight * xh, from the lanes' sums: put(group of the block, word).
template <int VEC, int NG, typename PUT>
BS_DEV void group_words(const NormK &k, const Spot &s, const float (&w)[VEC], const float (&s0)[VEC], const float (&s1)[VEC], float *a, float *b, PUT put)
{
    float t0[NG] = {}, t1[NG] = {};
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        t0[NG > 1 ? i : 0] = __builtin_fmaf(s0[i], w[i], t0[NG > 1 ? i : 0]);
        t1[NG > 1 ? i : 0] = __builtin_fmaf(s1[i], w[i], t1[NG > 1 ? i : 0]);
    }
    put_columns<NG>(k, s, t0, a);
    put_columns<NG>(k, s, t1, b);
    __syncthreads();
    sum_slices<NG>(k, a, b);
    __syncthreads();
    const uint32_t cols = k.by_cvb.d * NG, slices = NG > 1 ? k.slices_wide : k.slices, per = NG > 1 ? k.per : k.per / VEC, entries = per * slices;
    for (uint32_t g = threadIdx.x / 16; g < k.groups; g += RT / 16) {
        float u0 = 0.0f, u1 = 0.0f;
        for (uint32_t e = threadIdx.x % 16; e < entries; e += 16) {
            const uint32_t slice = fdiv(e, NG > 1 ? k.by_per : k.by_vectors), at = slice * cols + g * per + (e - slice * per);
            u0 += a[at];
            u1 += b[at];
        }
        u0 = sum16(u0);
        u1 = sum16(u1);
        if (threadIdx.x % 16 == 0) put(g, word_of(u0, u1));
    }
}

template <int DT, int VEC, int E, int ACT, bool RES, int NG>
__global__ __launch_bounds__(RT, 4) void norm_resident_grad_kernel(NormK k)
{
    __shared__ __align__(16) float col0[RT * VEC], col1[RT * VEC];
    __shared__ float group0[RT], group1[RT];
    __shared__ uint64_t words[K_NORM_WORDS];
    __shared__ uint32_t missing;
    const Spot s = Spot::of<VEC>(k);
    const Chunk own(k, s.chunk);
    const uint32_t mine = s.on ? own.of_lane(s.pl) : 0, c0 = s.b0 + (s.on ? s.cvi * VEC : 0);
    Operands<DT, VEC, E, ACT, RES, NG> o;
    o.load(k, s, own, mine);
    load_params<DT, VEC>(k.weight, k.f32_params, c0, 1.0f, o.w);
    load_params<DT, VEC>(k.bias, k.f32_params, c0, 0.0f, o.b);
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const float *in = k.stats + 2 * ((uint64_t)s.n * k.G + fdiv(c0 + i, k.by_per));
        o.mean[i] = in[0];
        o.rstd[i] = in[1];
    }
    if (threadIdx.x == 0) missing = 0;
    const bool tensors = k.dx.p || k.dr.p;
    {
        float s0[VEC], s1[VEC];
        o.sums(mine, s0, s1);
        if (tensors) group_words<VEC, NG>(k, s, o.w, s0, s1, col0, col1, [&](uint32_t g, uint64_t w) { publish(k, s, g, w, words); });
        if (k.part) {  // while the words are under way
            __syncthreads();
            put_columns<VEC>(k, s, s0, col0);
            put_columns<VEC>(k, s, s1, col1);
            __syncthreads();
            sum_slices<VEC>(k, col0, col1);
            __syncthreads();
            const uint32_t slices = VEC > 1 ? k.slices_wide : k.slices;
            float *out = k.part + 2 * (((uint64_t)s.n * k.chunks + s.chunk) * k.C + s.b0);
            for (uint32_t c = threadIdx.x; c < k.block; c += RT) {
                float t0 = 0.0f, t1 = 0.0f;
#pragma unroll 4
                for (uint32_t q = 0; q < slices; ++q) {
                    t0 += col0[q * k.block + c];
                    t1 += col1[q * k.block + c];
                }
                *reinterpret_cast<float2 *>(out + 2 * c) = make_float2(t0, t1);
            }
        }
    }
    if (!tensors) return;
    if (!collect(k, s, words, &missing)) {
        for (uint32_t q = 0; q < k.chunks; ++q) {
            if (q == s.chunk) continue;
            const Chunk other(k, q);
            const uint32_t its = s.on ? other.of_lane(s.pl) : 0;
            o.load(k, s, other, its);
            float s0[VEC], s1[VEC];
            o.sums(its, s0, s1);
            group_words<VEC, NG>(k, s, o.w, s0, s1, col0, col1, [&](uint32_t g, uint64_t w) { words[g * k.chunks + q] = w; });
            __syncthreads();
        }
        o.load(k, s, own, mine);
    }
    const uint32_t before = depart(k, s);
    for (uint32_t g = threadIdx.x / 16; g < k.groups; g += RT / 16) {
        const float cells = (float)k.P * (float)k.per;
        float a = 0.0f, b = 0.0f;
        for (uint32_t q = threadIdx.x % 16; q < k.chunks; q += 16) {
            a += word_low(words[g * k.chunks + q]);
            b += word_high(words[g * k.chunks + q]);
        }
        a = sum16(a);
        b = sum16(b);
        if (threadIdx.x % 16 == 0) {
            group0[g] = a / cells;
            group1[g] = b / cells;
        }
    }
    __syncthreads();
    o.x.forget();
    o.dy.forget();
    if constexpr (RES) o.r.forget();
    float m1[NG], m2[NG];
#pragma unroll
    for (int i = 0; i < NG; ++i) {
        const uint32_t g = fdiv(s.cvi * VEC + i, k.by_per);
        m1[i] = group0[g];
        m2[i] = group1[g];
    }
    constexpr uint64_t ES = DT != DT_F32 ? 2 : 4;
    char *const dr = const_cast<char *>(at_pixel<DT>(k.dr, k.P, s.n, own.p0 + s.pl, c0)), *const dx = const_cast<char *>(at_pixel<DT>(k.dx, k.P, s.n, own.p0 + s.pl, c0));
#pragma unroll
    for (int u = 0; u < E; ++u) {
        if (u >= (int)mine) continue;
        float dz[VEC], xh[VEC];
        o.slopes(u, dz, xh);
        if (k.dr.p) store_elems<DT, VEC>(dr + u * (s.lanes * k.dr.stride * ES), 0, dz);
        if (k.dx.p) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int g = NG > 1 ? i : 0;
                dz[i] = o.rstd[g] * (__builtin_fmaf(dz[i], o.w[i], -m1[g]) - xh[i] * m2[g]);
            }
            store_elems<DT, VEC>(dx + u * (s.lanes * k.dx.stride * ES), 0, dz);
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    clear_words(k, s, before);
}

template <int DT, int VEC, int ACT, bool RES>
void launch(const NormK &k, bool few, hipStream_t st)
{
    const dim3 grid(k.N * k.blocks * k.chunks), block(RT);
    constexpr int BYTES = VEC * (DT == DT_F32 ? 4 : 2), MANY = norm_resident_grad_pixels(BYTES, RES, false, false), FEW = norm_resident_grad_pixels(BYTES, RES, true, false);
    if (VEC == 1 || k.per % VEC == 0) {
        if (few) norm_resident_grad_kernel<DT, VEC, FEW, ACT, RES, 1><<<grid, block, 0, st>>>(k);
        else norm_resident_grad_kernel<DT, VEC, MANY, ACT, RES, 1><<<grid, block, 0, st>>>(k);
    } else if constexpr (VEC > 1) {
        constexpr int MIXED = norm_resident_grad_pixels(BYTES, RES, false, true);
        if (few) norm_resident_grad_kernel<DT, VEC, FEW, ACT, RES, VEC><<<grid, block, 0, st>>>(k);
        else norm_resident_grad_kernel<DT, VEC, MIXED, ACT, RES, VEC><<<grid, block, 0, st>>>(k);
    }
}

template <int DT, int VEC>
void launch_act(const NormK &k, bool few, hipStream_t st)
{
    const bool res = k.r.p;  // (without an activation the residual operand has no part in any gradient)
    switch (k.activation) {
    case BS_ACT_IDENTITY: launch<DT, VEC, BS_ACT_IDENTITY, false>(k, few, st); break;
    case BS_ACT_RELU: res ? launch<DT, VEC, BS_ACT_RELU, true>(k, few, st) : launch<DT, VEC, BS_ACT_RELU, false>(k, few, st); break;
    case BS_ACT_SILU: res ? launch<DT, VEC, BS_ACT_SILU, true>(k, few, st) : launch<DT, VEC, BS_ACT_SILU, false>(k, few, st); break;
    case BS_ACT_GELU: res ? launch<DT, VEC, BS_ACT_GELU, true>(k, few, st) : launch<DT, VEC, BS_ACT_GELU, false>(k, few, st); break;
    }
}

template <int DT>
void launch_vec(const NormK &k, int vec, bool few, hipStream_t st)
{
    constexpr int HALF = DT == DT_F32 ? 2 : 4;
    if (vec == HALF) launch_act<DT, HALF>(k, few, st);
    else launch_act<DT, 1>(k, few, st);
}

}  // namespace

bs_status launch_norm_resident_grad(const NormK &k, int32_t dtype, int vec, bool few, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) launch_vec<DT_F32>(k, vec, few, st);
    else if (dtype == BS_BF16) launch_vec<DT_BF16>(k, vec, few, st);
    else launch_vec<DT_F16>(k, vec, few, st);
    const hipError_t err = hipGetLastError();
    if (err == hipSuccess) return BS_OK;
    set_hip_error((int32_t)err);
    return BS_ERR_HIP;
}

}  // namespace bs
