// Group normalisation with a residual operand and an activation, channels last.
//
//   mean, var over a group's P pixels x per channels;  xh = (x - mean) / sqrt(var + eps);  z = xh * weight + bias (+ r);  y = act(z)
//   dz = dy * act'(z);  dr = dz;  dbias = sum dz;  dweight = sum dz * xh  (over images and pixels)
//   dx = (dz * weight - (S1 + xh * S2) / (P * per)) / sqrt(var + eps),  S1 = sum dz * weight, S2 = sum dz * weight * xh over the group
//
// A lane keeps one vector of neighbouring channels and walks over pixels, so that everything per channel stays in its registers and a
// wave reads whole rows of channels.  Statistics are float32: a lane takes batches of pixels, mean and squared deviations of each batch
// from the batch's own mean, and merges them (Chan's update), so that a mean far from zero cancels nothing.
#include <hip/hip_runtime.h>

#include "bs_internal.h"
#include "bs_norm_device.h"

namespace bs {
namespace {

constexpr int T = K_NORM_THREADS;

// ------------------------------------------------------------------------------------------------ lanes and channels
// Where a lane stands: its channel vector (c0 .. c0 + VEC - 1 of the tensor) and its first pixel; lanes beyond the block do nothing.
struct Lane {
    uint32_t n, chunk, block;  // image, pixel chunk, channel block of the work-group
    uint32_t b0, bc;           // first channel and channels of the block
    uint32_t cvi, pl, lanes;   // channel vector in the block, pixel lane, pixel lanes of the work-group
    uint32_t p0, p1;           // the chunk's pixels
    bool on;
};

template <int VEC>
BS_DEV Lane lane_of(const NormK &k, uint32_t bid)
{
    Lane l;
    l.block = bid % k.blocks;
    const uint32_t rest = bid / k.blocks;
    l.chunk = rest % k.chunks;
    l.n = rest / k.chunks;
    l.b0 = l.block * K_NORM_BLOCK_CHANNELS;
    l.bc = min(k.C - l.b0, (uint32_t)K_NORM_BLOCK_CHANNELS);
    const uint32_t cvb = l.bc / VEC;
    l.lanes = T / cvb;
    l.pl = threadIdx.x / cvb;
    l.cvi = threadIdx.x - l.pl * cvb;
    l.on = l.pl < l.lanes;
    l.p0 = l.chunk * k.chunk;
    l.p1 = min(l.p0 + k.chunk, k.P);
    return l;
}

// Sums of M values per channel over the work-group's pixel lanes: lds[m][channel of the block], valid after the call's barrier.
template <int VEC, int M>
BS_DEV void sum_lanes(const Lane &l, const float (&v)[M][VEC], float *lds /* M * T * VEC */)
{
    if (l.on)
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < VEC; ++i) lds[m * T * VEC + l.pl * l.bc + l.cvi * VEC + i] = v[m][i];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < l.bc; c += T) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            float s = 0.0f;
            for (uint32_t q = 0; q < l.lanes; ++q) s += lds[m * T * VEC + q * l.bc + c];
            lds[m * T * VEC + c] = s;  // (its own column only)
        }
    }
    __syncthreads();
}

// ------------------------------------------------------------------------------------------------ forward, in two passes over x
// Mean and squared deviations of every group's part in this chunk and channel block.
template <int DT, int VEC>
__global__ __launch_bounds__(T) void norm_stats_kernel(NormK k)
{
    __shared__ float lds[T * VEC];
    __shared__ float group_mean[K_NORM_BLOCK_CHANNELS];
    const Lane l = lane_of<VEC>(k, blockIdx.x);
    const uint32_t c0 = l.b0 + l.cvi * VEC;
    float mean[VEC] = {}, m2[VEC] = {}, count = 0.0f;
    if (l.on) {
        constexpr int U = 8;
        const uint64_t step = (uint64_t)l.lanes * k.x.stride * (DT != DT_F32 ? 2 : 4);
        const char *src = at_pixel<DT>(k.x, k.P, l.n, l.p0 + l.pl, c0);
        uint32_t p = l.p0 + l.pl;
        for (; p + (U - 1) * l.lanes < l.p1; p += U * l.lanes) {
            float v[U][VEC];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                load_vec<DT, VEC>(src, v[u]);
                src += step;
            }
            const float total = count + U, share = U / total, cross = count * share;
            count = total;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float s = 0.0f, q = 0.0f;
#pragma unroll
                for (int u = 0; u < U; ++u) s += v[u][i];
                const float mb = s * (1.0f / U);
#pragma unroll
                for (int u = 0; u < U; ++u) q = __builtin_fmaf(v[u][i] - mb, v[u][i] - mb, q);
                const float d = mb - mean[i];
                mean[i] = __builtin_fmaf(d, share, mean[i]);
                m2[i] += __builtin_fmaf(d * d, cross, q);
            }
        }
        for (; p < l.p1; p += l.lanes) {
            float v[VEC];
            load_vec<DT, VEC>(src, v);
            src += step;
            count += 1.0f;
            const float share = 1.0f / count;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = v[i] - mean[i];
                mean[i] = __builtin_fmaf(d, share, mean[i]);
                m2[i] = __builtin_fmaf(d, v[i] - mean[i], m2[i]);
            }
        }
    }
    // the part's mean, then the squared deviations from it
    float sum[1][VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum[0][i] = mean[i] * count;
    sum_lanes<VEC, 1>(l, sum, lds);
    const uint32_t g0 = l.b0 / k.per, groups = (l.b0 + l.bc - 1) / k.per - g0 + 1;
    const uint32_t pixels = l.p1 - l.p0;
    for (uint32_t g = threadIdx.x; g < groups; g += T) {
        const uint32_t from = max((g0 + g) * k.per, l.b0) - l.b0, to = min((g0 + g + 1) * k.per, l.b0 + l.bc) - l.b0;
        float s = 0.0f;
        for (uint32_t c = from; c < to; ++c) s += lds[c];
        group_mean[g] = s / ((float)pixels * (float)(to - from));
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const float d = l.on ? mean[i] - group_mean[(c0 + i) / k.per - g0] : 0.0f;
        sum[0][i] = __builtin_fmaf(d * d, count, m2[i]);
    }
    sum_lanes<VEC, 1>(l, sum, lds);
    for (uint32_t g = threadIdx.x; g < groups; g += T) {
        const uint32_t from = max((g0 + g) * k.per, l.b0) - l.b0, to = min((g0 + g + 1) * k.per, l.b0 + l.bc) - l.b0;
        float s = 0.0f;
        for (uint32_t c = from; c < to; ++c) s += lds[c];
        const uint32_t first = (g0 + g) * k.per / K_NORM_BLOCK_CHANNELS;
        float *out = k.part + 2 * ((((uint64_t)l.n * k.G + g0 + g) * k.chunks + l.chunk) * k.spans + (l.block - first));
        out[0] = group_mean[g];
        out[1] = s;
    }
}

// Joins the parts of one group of one image: a thread each.
__global__ __launch_bounds__(T) void norm_join_kernel(NormK k)
{
    const uint32_t i = blockIdx.x * T + threadIdx.x;
    if (i >= k.N * k.G) return;
    const uint32_t g = i % k.G, c0 = g * k.per, c1 = c0 + k.per, first = c0 / K_NORM_BLOCK_CHANNELS, last = (c1 - 1) / K_NORM_BLOCK_CHANNELS;
    float mean = 0.0f, m2 = 0.0f, count = 0.0f;
    for (uint32_t q = 0; q < k.chunks; ++q) {
        const float pixels = (float)(min((q + 1) * k.chunk, k.P) - q * k.chunk);
        for (uint32_t b = first; b <= last; ++b) {
            const uint32_t from = max(c0, b * K_NORM_BLOCK_CHANNELS), to = min(c1, (b + 1) * K_NORM_BLOCK_CHANNELS);
            const float *in = k.part + 2 * (((uint64_t)i * k.chunks + q) * k.spans + (b - first));
            const float nb = pixels * (float)(to - from), total = count + nb, d = in[0] - mean, share = nb / total;
            mean = __builtin_fmaf(d, share, mean);
            m2 += __builtin_fmaf(d * d, count * share, in[1]);
            count = total;
        }
    }
    k.stats[2 * i] = mean;
    k.stats[2 * i + 1] = 1.0f / sqrtf(m2 / count + k.eps);
}

// What a lane keeps of its channels: group mean, 1 / deviation, weight, bias.
template <int DT, int VEC>
struct Affine {
    float mean[VEC], rstd[VEC], w[VEC], b[VEC];
    BS_DEV void load(const NormK &k, uint32_t n, uint32_t c0)
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const uint64_t g = (uint64_t)n * k.G + (c0 + i) / k.per;
            mean[i] = k.stats[2 * g];
            rstd[i] = k.stats[2 * g + 1];
        }
        load_params<DT, VEC>(k.weight, k.f32_params, c0, 1.0f, w);
        load_params<DT, VEC>(k.bias, k.f32_params, c0, 0.0f, b);
    }
};

template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(T) void norm_apply_kernel(NormK k)
{
    const Lane l = lane_of<VEC>(k, blockIdx.x);
    if (!l.on) return;
    const uint32_t c0 = l.b0 + l.cvi * VEC;
    Affine<DT, VEC> a;
    a.load(k, l.n, c0);
    for (uint32_t p = l.p0 + l.pl; p < l.p1; p += l.lanes) {
        float v[VEC], r[VEC] = {};
        load_vec<DT, VEC>(at_pixel<DT>(k.x, k.P, l.n, p, c0), v);
        if (k.r.p) load_vec<DT, VEC>(at_pixel<DT>(k.r, k.P, l.n, p, c0), r);
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[i] = act<DT, ACT>(__builtin_fmaf((v[i] - a.mean[i]) * a.rstd[i], a.w[i], a.b[i]) + r[i]);
        store_elems<DT, VEC>(const_cast<char *>(at_pixel<DT>(k.y, k.P, l.n, p, c0)), 0, v);
    }
}

// ------------------------------------------------------------------------------------------------ backward
// dz and xh of one vector.
template <int DT, int VEC, int ACT>
BS_DEV void slopes(const NormK &k, const Affine<DT, VEC> &a, uint32_t n, uint32_t p, uint32_t c0, float (&dz)[VEC], float (&xh)[VEC])
{
    float r[VEC] = {};
    load_vec<DT, VEC>(at_pixel<DT>(k.x, k.P, n, p, c0), xh);
    load_vec<DT, VEC>(at_pixel<DT>(k.dy, k.P, n, p, c0), dz);
    if (ACT != BS_ACT_IDENTITY && k.r.p) load_vec<DT, VEC>(at_pixel<DT>(k.r, k.P, n, p, c0), r);
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        xh[i] = (xh[i] - a.mean[i]) * a.rstd[i];
        dz[i] *= act_slope<DT, ACT>(__builtin_fmaf(xh[i], a.w[i], a.b[i]) + r[i]);
    }
}

// Sums of dz and dz * xh per channel of a chunk.
template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(T) void norm_grad_sums_kernel(NormK k)
{
    __shared__ float lds[2 * T * VEC];
    const Lane l = lane_of<VEC>(k, blockIdx.x);
    const uint32_t c0 = l.b0 + l.cvi * VEC;
    float s[2][VEC] = {};
    if (l.on) {
        Affine<DT, VEC> a;
        a.load(k, l.n, c0);
        for (uint32_t p = l.p0 + l.pl; p < l.p1; p += l.lanes) {
            float dz[VEC], xh[VEC];
            slopes<DT, VEC, ACT>(k, a, l.n, p, c0, dz, xh);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s[0][i] += dz[i];
                s[1][i] = __builtin_fmaf(dz[i], xh[i], s[1][i]);
            }
        }
    }
    sum_lanes<VEC, 2>(l, s, lds);
    float *out = k.part + 2 * (((uint64_t)l.n * k.chunks + l.chunk) * k.C + l.b0);
    for (uint32_t c = threadIdx.x; c < l.bc; c += T) {
        out[2 * c] = lds[c];
        out[2 * c + 1] = lds[T * VEC + c];
    }
}

// A group's sums: one wave per group and image.
template <int DT>
__global__ __launch_bounds__(64) void norm_grad_join_kernel(NormK k)
{
    const uint32_t n = blockIdx.x / k.G, g = blockIdx.x - n * k.G;
    float s1 = 0.0f, s2 = 0.0f;
    for (uint32_t e = threadIdx.x; e < k.chunks * k.per; e += 64) {
        const uint32_t q = e / k.per, c = g * k.per + (e - q * k.per);
        float w[1];
        load_params<DT, 1>(k.weight, k.f32_params, c, 1.0f, w);
        const float *in = k.part + 2 * (((uint64_t)n * k.chunks + q) * k.C + c);
        s1 = __builtin_fmaf(in[0], w[0], s1);
        s2 = __builtin_fmaf(in[1], w[0], s2);
    }
#pragma unroll
    for (int m = 32; m; m >>= 1) {
        s1 += __shfl_xor(s1, m);
        s2 += __shfl_xor(s2, m);
    }
    if (threadIdx.x == 0) {
        k.sums[2 * (uint64_t)blockIdx.x] = s1;
        k.sums[2 * (uint64_t)blockIdx.x + 1] = s2;
    }
}

// Gradients of weight and bias: four channels of all images' chunks by a work-group, a thread every 256th chunk of one channel.
constexpr int PT = 1024;
template <int DT>
__global__ __launch_bounds__(PT) void norm_grad_params_kernel(NormK k)
{
    __shared__ float db[PT], dw[PT];
    const uint32_t c = blockIdx.x * 4 + threadIdx.x % 4, row = threadIdx.x / 4, rows = k.N * k.chunks;
    float s0 = 0.0f, s1 = 0.0f;
    if (c < k.C) {
#pragma unroll 8
        for (uint32_t q = row; q < rows; q += PT / 4) {
            const float2 in = *reinterpret_cast<const float2 *>(k.part + 2 * ((uint64_t)q * k.C + c));
            s0 += in.x;
            s1 += in.y;
        }
    }
    db[threadIdx.x] = s0;
    dw[threadIdx.x] = s1;
    for (uint32_t half = PT / 2; half >= 4; half /= 2) {
        __syncthreads();
        if (threadIdx.x < half) {
            db[threadIdx.x] += db[threadIdx.x + half];
            dw[threadIdx.x] += dw[threadIdx.x + half];
        }
    }
    if (threadIdx.x >= 4 || c >= k.C) return;
    auto put = [&](void *p, float v) {
        if (!p) return;
        if (DT == DT_F32 || k.f32_params) static_cast<float *>(p)[c] = v;
        else static_cast<uint16_t *>(p)[c] = half_bits<DT>(v);
    };
    put(k.dbias, db[threadIdx.x]);
    put(k.dweight, dw[threadIdx.x]);
}

template <int DT, int VEC, int ACT>
__global__ __launch_bounds__(T) void norm_grad_apply_kernel(NormK k)
{
    const Lane l = lane_of<VEC>(k, blockIdx.x);
    if (!l.on) return;
    const uint32_t c0 = l.b0 + l.cvi * VEC;
    Affine<DT, VEC> a;
    a.load(k, l.n, c0);
    float s1[VEC], s2[VEC];
    const float cells = (float)k.P * (float)k.per;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
        const uint64_t g = (uint64_t)l.n * k.G + (c0 + i) / k.per;
        s1[i] = k.sums[2 * g] / cells;
        s2[i] = k.sums[2 * g + 1] / cells;
    }
    for (uint32_t p = l.p0 + l.pl; p < l.p1; p += l.lanes) {
        float dz[VEC], xh[VEC], dx[VEC];
        slopes<DT, VEC, ACT>(k, a, l.n, p, c0, dz, xh);
        if (k.dr.p) store_elems<DT, VEC>(const_cast<char *>(at_pixel<DT>(k.dr, k.P, l.n, p, c0)), 0, dz);
        if (k.dx.p) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) dx[i] = a.rstd[i] * (__builtin_fmaf(dz[i], a.w[i], -s1[i]) - xh[i] * s2[i]);
            store_elems<DT, VEC>(const_cast<char *>(at_pixel<DT>(k.dx, k.P, l.n, p, c0)), 0, dx);
        }
    }
}

// ------------------------------------------------------------------------------------------------ launches
bs_status checked()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

template <int DT, int VEC, int ACT>
void launch(NormPass pass, const NormK &k, hipStream_t st)
{
    constexpr bool FULL = VEC * (DT == DT_F32 ? 4 : 2) == 16;  // (not backward)
    const dim3 grid(k.N * k.chunks * k.blocks), block(T);
    switch (pass) {
    case NORM_STATS:
        if constexpr (ACT == 0) norm_stats_kernel<DT, VEC><<<grid, block, 0, st>>>(k);
        break;
    case NORM_APPLY: norm_apply_kernel<DT, VEC, ACT><<<grid, block, 0, st>>>(k); break;
    case NORM_GRAD_SUMS:
        if constexpr (!FULL) norm_grad_sums_kernel<DT, VEC, ACT><<<grid, block, 0, st>>>(k);
        break;
    case NORM_GRAD_APPLY:
        if constexpr (!FULL) norm_grad_apply_kernel<DT, VEC, ACT><<<grid, block, 0, st>>>(k);
        break;
    default: break;
    }
}

template <int DT, int VEC>
void launch_act(NormPass pass, const NormK &k, hipStream_t st)
{
    switch (pass == NORM_STATS ? BS_ACT_IDENTITY : (int)k.activation) {
    case BS_ACT_IDENTITY: launch<DT, VEC, BS_ACT_IDENTITY>(pass, k, st); break;
    case BS_ACT_RELU: launch<DT, VEC, BS_ACT_RELU>(pass, k, st); break;
    case BS_ACT_SILU: launch<DT, VEC, BS_ACT_SILU>(pass, k, st); break;
    case BS_ACT_GELU: launch<DT, VEC, BS_ACT_GELU>(pass, k, st); break;
    }
}

template <int DT>
void launch_type(NormPass pass, const NormK &k, int vec, hipStream_t st)
{
    constexpr int FULL = DT == DT_F32 ? 4 : 8;
    if (pass == NORM_GRAD_JOIN) norm_grad_join_kernel<DT><<<dim3(k.N * k.G), dim3(64), 0, st>>>(k);
    else if (pass == NORM_GRAD_PARAMS) norm_grad_params_kernel<DT><<<dim3((k.C + 3) / 4), dim3(PT), 0, st>>>(k);
    else if (vec == FULL) launch_act<DT, FULL>(pass, k, st);
    else if (vec == FULL / 2) launch_act<DT, FULL / 2>(pass, k, st);
    else launch_act<DT, 1>(pass, k, st);
}

}  // namespace

bs_status launch_norm(NormPass pass, const NormK &k, int32_t dtype, int vec, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (pass == NORM_JOIN) norm_join_kernel<<<dim3((k.N * k.G + T - 1) / T), dim3(T), 0, st>>>(k);
    else if (dtype == BS_F32) launch_type<DT_F32>(pass, k, vec, st);
    else if (dtype == BS_BF16) launch_type<DT_BF16>(pass, k, vec, st);
    else launch_type<DT_F16>(pass, k, vec, st);
    return checked();
}

}  // namespace bs
