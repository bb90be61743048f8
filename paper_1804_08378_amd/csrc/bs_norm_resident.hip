// Group normalisation, forward, with the tensor resident in registers (bs_norm_resident.h): x is read once, y written once.
#include <hip/hip_runtime.h>

#include "bs_internal.h"
#include "bs_norm_resident.h"

namespace bs {
namespace {

// What a lane, a slice, a chunk knows of a group: values seen, their mean, squared deviations from it.  Two parts join by sums of weighted
// means and of deviations from the joint mean: nothing cancels, however far the mean is from zero.
template <int DT, int VEC, int E, int NG>
struct Part {
    float *means, *devs;  // LDS: RT * NG each
    float *counts;        // LDS: pixels of a slice

    // The chunk's words: put(group of the block, word).
    template <typename PUT>
    BS_DEV void compute(const NormK &k, const Spot &s, Pixels<DT, VEC, E> &x, const Chunk &q, PUT put) const
    {
        const uint32_t mine = s.on ? q.of_lane(s.pl) : 0;
        float sum[VEC] = {}, m[NG], d2[NG];
#pragma unroll
        for (int u = 0; u < E; ++u)
            if (u < (int)mine) {
                float a[VEC];
                unpack<DT, VEC>(x.raw[u], a);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i] += a[i];
            }
        const float share = mine ? 1.0f / (float)(mine * (NG > 1 ? 1 : VEC)) : 0.0f;
        if constexpr (NG == 1) {
#pragma unroll
            for (int n = VEC / 2; n; n /= 2)
#pragma unroll
                for (int i = 0; i < n; ++i) sum[i] += sum[i + n];
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) m[i] = sum[i] * share;
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum[i] = 0.0f;
        x.forget();
#pragma unroll
        for (int u = 0; u < E; ++u)
            if (u < (int)mine) {
                float a[VEC];
                unpack<DT, VEC>(x.raw[u], a);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float d = a[i] - m[NG > 1 ? i : 0];
                    sum[i] = __builtin_fmaf(d, d, sum[i]);
                }
            }
        if constexpr (NG == 1) {
#pragma unroll
            for (int n = VEC / 2; n; n /= 2)
#pragma unroll
                for (int i = 0; i < n; ++i) sum[i] += sum[i + n];
        }
#pragma unroll
        for (int i = 0; i < NG; ++i) d2[i] = sum[i];
        put_columns<NG>(k, s, m, means);
        put_columns<NG>(k, s, d2, devs);
        __syncthreads();
        constexpr float WIDE = NG > 1 ? 1 : VEC;  // values of a pixel in a column
        each_slice<NG>(k, [&](uint32_t c, uint32_t slice, uint32_t cols, uint32_t slices) {
            float n = 0.0f, t = 0.0f, d = 0.0f;
#pragma unroll 4
            for (uint32_t r = slice; r < k.lanes; r += slices) {
                const float nr = (float)q.of_lane(r);
                n += nr;
                t = __builtin_fmaf(nr, means[r * cols + c], t);
            }
            const float mean = n > 0.0f ? t / n : 0.0f;
#pragma unroll 4
            for (uint32_t r = slice; r < k.lanes; r += slices) {
                const float e = means[r * cols + c] - mean;
                d += __builtin_fmaf(e * e, (float)q.of_lane(r) * WIDE, devs[r * cols + c]);
            }
            means[slice * cols + c] = mean;  // (no other thread reads this row of the column)
            devs[slice * cols + c] = d;
            if (c == 0) counts[slice] = n;
        });
        __syncthreads();
        // a group's columns and slices, 16 lanes a group
        const uint32_t cols = k.by_cvb.d * NG, slices = NG > 1 ? k.slices_wide : k.slices, per = NG > 1 ? k.per : k.per / VEC, entries = per * slices;
        for (uint32_t g = threadIdx.x / 16; g < k.groups; g += RT / 16) {
            float t = 0.0f, d = 0.0f;
            for (uint32_t e = threadIdx.x % 16; e < entries; e += 16) {
                const uint32_t slice = fdiv(e, NG > 1 ? k.by_per : k.by_vectors), c = g * per + (e - slice * per);
                t = __builtin_fmaf(counts[slice], means[slice * cols + c], t);
            }
            const float mean = sum16(t) / ((float)q.pixels * (float)per);
            for (uint32_t e = threadIdx.x % 16; e < entries; e += 16) {
                const uint32_t slice = fdiv(e, NG > 1 ? k.by_per : k.by_vectors), c = g * per + (e - slice * per);
                const float off = means[slice * cols + c] - mean;
                d += __builtin_fmaf(off * off, counts[slice] * WIDE, devs[slice * cols + c]);
            }
            d = sum16(d);
            if (threadIdx.x % 16 == 0) put(g, word_of(mean, d));
        }
    }
};

// NG: values of a channel vector that the lanes keep apart: 1 where every vector lies inside a group, else one a channel.
template <int DT, int VEC, int E, int ACT, bool RES, int NG>
__global__ __launch_bounds__(RT, 4) void norm_resident_kernel(NormK k)
{
    __shared__ __align__(16) float means[RT * NG], devs[RT * NG];
    __shared__ float counts[RT], group_mean[RT], group_rstd[RT];
    __shared__ uint64_t words[K_NORM_WORDS];
    __shared__ uint32_t missing;
    const Spot s = Spot::of<VEC>(k);
    const Chunk own(k, s.chunk);
    const uint32_t mine = s.on ? own.of_lane(s.pl) : 0, c0 = s.b0 + (s.on ? s.cvi * VEC : 0);
    Pixels<DT, VEC, E> x, r;
    x.load(k.x, k, s, own, mine);
    if constexpr (RES) r.load(k.r, k, s, own, mine);
    if (threadIdx.x == 0) missing = 0;
    const Part<DT, VEC, E, NG> part{means, devs, counts};
    part.compute(k, s, x, own, [&](uint32_t g, uint64_t w) { publish(k, s, g, w, words); });
    float a[VEC], b[VEC];
    load_params<DT, VEC>(k.weight, k.f32_params, c0, 1.0f, a);
    load_params<DT, VEC>(k.bias, k.f32_params, c0, 0.0f, b);
    if (!collect(k, s, words, &missing)) {
        for (uint32_t q = 0; q < k.chunks; ++q) {
            if (q == s.chunk) continue;
            const Chunk other(k, q);
            x.load(k.x, k, s, other, s.on ? other.of_lane(s.pl) : 0);
            part.compute(k, s, x, other, [&](uint32_t g, uint64_t w) { words[g * k.chunks + q] = w; });
            __syncthreads();
        }
        x.load(k.x, k, s, own, mine);
    }
    const uint32_t before = depart(k, s);
    // join the chunks of a group
    for (uint32_t g = threadIdx.x / 16; g < k.groups; g += RT / 16) {
        const uint64_t *w = words + g * k.chunks;
        float t = 0.0f, d = 0.0f;
        for (uint32_t q = threadIdx.x % 16; q < k.chunks; q += 16) t = __builtin_fmaf(word_low(w[q]), (float)(q + 1 == k.chunks ? k.last : k.chunk), t);
        const float mean = sum16(t) / (float)k.P, cells = (float)k.P * (float)k.per;
        for (uint32_t q = threadIdx.x % 16; q < k.chunks; q += 16) {
            const float off = word_low(w[q]) - mean;
            d += __builtin_fmaf(off * off, (float)(q + 1 == k.chunks ? k.last : k.chunk) * (float)k.per, word_high(w[q]));
        }
        const float rstd = 1.0f / sqrtf(sum16(d) / cells + k.eps);
        if (threadIdx.x % 16 == 0) {
            group_mean[g] = mean;
            group_rstd[g] = rstd;
            if (k.stats && s.chunk == 0) {
                float *out = k.stats + 2 * ((uint64_t)s.n * k.G + s.g0 + g);
                out[0] = mean;
                out[1] = rstd;
            }
        }
    }
    __syncthreads();
    x.forget();
    if constexpr (RES) r.forget();
    float m[NG];
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const uint32_t g = fdiv(s.cvi * VEC + (NG > 1 ? i : 0), k.by_per);
        if (i < NG) m[i] = group_mean[g];
        a[i] *= group_rstd[g];
    }
    char *dst = const_cast<char *>(at_pixel<DT>(k.y, k.P, s.n, own.p0 + s.pl, c0));
    const uint64_t step = (uint64_t)s.lanes * k.y.stride * (DT != DT_F32 ? 2 : 4);
#pragma unroll
    for (int u = 0; u < E; ++u) {
        if (u >= (int)mine) continue;
        float v[VEC], add[VEC] = {};
        unpack<DT, VEC>(x.raw[u], v);
        if constexpr (RES) unpack<DT, VEC>(r.raw[u], add);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = act<DT, ACT>(__builtin_fmaf(v[i] - m[NG > 1 ? i : 0], a[i], b[i]) + add[i]);
        store_elems<DT, VEC>(dst + u * step, 0, v);
    }
    clear_words(k, s, before);
}

__global__ __launch_bounds__(256) void norm_absent_kernel(uint64_t *words, uint32_t n)
{
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) __hip_atomic_store(words + i, ABSENT, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <int DT, int VEC, int E, bool RES, int NG>
void launch(const NormK &k, hipStream_t st)
{
    const dim3 grid(k.N * k.blocks * k.chunks), block(RT);
    switch (k.activation) {
    case BS_ACT_IDENTITY: norm_resident_kernel<DT, VEC, E, BS_ACT_IDENTITY, RES, NG><<<grid, block, 0, st>>>(k); break;
    case BS_ACT_RELU: norm_resident_kernel<DT, VEC, E, BS_ACT_RELU, RES, NG><<<grid, block, 0, st>>>(k); break;
    case BS_ACT_SILU: norm_resident_kernel<DT, VEC, E, BS_ACT_SILU, RES, NG><<<grid, block, 0, st>>>(k); break;
    case BS_ACT_GELU: norm_resident_kernel<DT, VEC, E, BS_ACT_GELU, RES, NG><<<grid, block, 0, st>>>(k); break;
    }
}

template <int DT, int VEC, bool RES>
void launch_res(const NormK &k, bool few, hipStream_t st)
{
    constexpr int BYTES = VEC * (DT == DT_F32 ? 4 : 2), MANY = norm_resident_pixels(BYTES, RES, false), FEW = norm_resident_pixels(BYTES, RES, true);
    if (VEC == 1 || BYTES == 16 || k.per % VEC == 0) few ? launch<DT, VEC, FEW, RES, 1>(k, st) : launch<DT, VEC, MANY, RES, 1>(k, st);
    else if constexpr (BYTES == 8) few ? launch<DT, VEC, FEW, RES, VEC>(k, st) : launch<DT, VEC, MANY, RES, VEC>(k, st);
}

template <int DT, int VEC>
void launch_e(const NormK &k, bool few, hipStream_t st)
{
    k.r.p ? launch_res<DT, VEC, true>(k, few, st) : launch_res<DT, VEC, false>(k, few, st);
}

template <int DT>
void launch_vec(const NormK &k, int vec, bool few, hipStream_t st)
{
    constexpr int FULL = DT == DT_F32 ? 4 : 8;
    if (vec == FULL) launch_e<DT, FULL>(k, few, st);
    else if (vec == FULL / 2) launch_e<DT, FULL / 2>(k, few, st);
    else launch_e<DT, 1>(k, few, st);
}

bs_status checked()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

}  // namespace

bs_status launch_norm_absent(const NormK &k, void *stream)
{
    const uint32_t n = k.N * k.G * k.chunks;
    norm_absent_kernel<<<dim3((n + 255) / 256), dim3(256), 0, static_cast<hipStream_t>(stream)>>>(k.words, n);
    return checked();
}

bs_status launch_norm_resident(const NormK &k, int32_t dtype, int vec, bool few, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) launch_vec<DT_F32>(k, vec, few, st);
    else if (dtype == BS_BF16) launch_vec<DT_BF16>(k, vec, few, st);
    else launch_vec<DT_F16>(k, vec, few, st);
    return checked();
}

}  // namespace bs
