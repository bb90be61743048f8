// Layer normalisation of rows with an addition in front of it.
//
//   t = round(x + addend);  mean, var over the row;  xh = (t - mean) * rstd,  rstd = 1 / sqrt(var + eps);  y = xh * weight + bias
//   u = dy * weight;  dx = rstd * (u - S1 / C - xh * S2 / C) + dt,  S1 = sum u, S2 = sum u * xh over the row
//   dweight = sum dy * xh,  dbias = sum dy  over the rows
//
// Here: rows too long for registers (bs_layer_norm_team.h has the others), and the join of the parameters' gradients.  A work-group walks over its row
// in 128-bit vectors, as often as the formulas need it.  Statistics are float32: a lane takes mean and squared deviations of each vector from the
// vector's own mean and merges them (Chan's update), so that a mean far from zero cancels nothing.
#include <hip/hip_runtime.h>

#include "bs_layer_norm_team.h"

namespace bs {
namespace {

constexpr int T = 1024;  // lanes of a work-group that walks over a row
constexpr int PT = 256;  // of one that sums over rows

// t of a lane's columns.
template <int DT>
BS_DEV void load_total(const LayerNormK &k, uint64_t row, uint32_t c, float (&v)[K_VEC<DT>])
{
    load_cols<DT>(row_of<DT>(k.x, row), c, k.C, v);
    if (!k.addend.p) return;
    float a[K_VEC<DT>];
    load_cols<DT>(row_of<DT>(k.addend, row), c, k.C, a);
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) v[i] += a[i];
    round_store_all<DT, K_VEC<DT>>(v);
}

template <int DT>
__global__ __launch_bounds__(T) void layer_norm_kernel(LayerNormK k)
{
    constexpr int VEC = K_VEC<DT>;
    __shared__ float lds[2][T / 64];
    const uint32_t end = (k.C + BS_PACK8_BLOCK - 1) / BS_PACK8_BLOCK * BS_PACK8_BLOCK;  // whole blocks of lanes
    for (uint64_t row = blockIdx.x; row < k.rows; row += gridDim.x) {
        float mean = 0.0f, m2 = 0.0f, count = 0.0f;
        for (uint32_t c = threadIdx.x * VEC; c < end; c += T * VEC) {
            float v[VEC], s = 0.0f, q = 0.0f;
            load_total<DT>(k, row, c, v);
            if (k.total.p) store_cols<DT>(const_cast<char *>(row_of<DT>(k.total, row)), c, k.C, v);
            if (k.held.codes) store_held<DT>(k.held, row, c, k.C, to_words<DT>(v), v);
            if (c >= k.C) break;  // (the lane's last vector)
            const float n = (float)min(k.C - c, (uint32_t)VEC);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[i];
            const float mb = s / n;
#pragma unroll
            for (int i = 0; i < VEC; ++i) q += c + i < k.C ? (v[i] - mb) * (v[i] - mb) : 0.0f;
            const float total = count + n, share = n / total, d = mb - mean;
            mean = __builtin_fmaf(d, share, mean);
            m2 += __builtin_fmaf(d * d, count * share, q);
            count = total;
        }
        __syncthreads();  // (the row before has read its sums)
        const float all = group_sum<T>(mean * count, lds[0]) / (float)k.C;
        const float d = mean - all;
        const float var = group_sum<T>(__builtin_fmaf(d * d, count, m2), lds[1]) / (float)k.C;
        const float rstd = reciprocal_root(var + k.eps);
        if (k.stats && threadIdx.x == 0) {
            k.stats[2 * row] = all;
            k.stats[2 * row + 1] = rstd;
        }
        for (uint32_t c = threadIdx.x * VEC; c < k.C; c += T * VEC) {
            float v[VEC], w[VEC], b[VEC];
            load_total<DT>(k, row, c, v);
            load_row_params<DT>(k.weight, k.f32_params, c, k.C, 1.0f, w);
            load_row_params<DT>(k.bias, k.f32_params, c, k.C, 0.0f, b);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = __builtin_fmaf((v[i] - all) * rstd, w[i], b[i]);
            store_cols<DT>(const_cast<char *>(row_of<DT>(k.y, row)), c, k.C, v);
        }
    }
}

// xh and dy of a lane's columns, 0 behind the last.
template <int DT>
BS_DEV void load_grad(const LayerNormK &k, uint64_t row, uint32_t c, float mean, float rstd, float (&xh)[K_VEC<DT>], float (&dy)[K_VEC<DT>])
{
    if (k.held.codes) {
        HeldVector<DT> h;
        h.load(k.held, row, c, k.C);
        h.settle(c, k.C);
        h.numbers(xh);
    } else {
        load_cols<DT>(row_of<DT>(k.x, row), c, k.C, xh);
    }
    load_cols<DT>(row_of<DT>(k.dy, row), c, k.C, dy);
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) xh[i] = (xh[i] - mean) * rstd;
}

template <int DT>
__global__ __launch_bounds__(T) void layer_norm_grad_kernel(LayerNormK k)
{
    constexpr int VEC = K_VEC<DT>;
    __shared__ float lds[2][T / 64];
    for (uint64_t row = blockIdx.x; row < k.rows; row += gridDim.x) {
        const float mean = k.stats[2 * row], rstd = k.stats[2 * row + 1];
        float s1 = 0.0f, s2 = 0.0f;
        for (uint32_t c = threadIdx.x * VEC; c < k.C; c += T * VEC) {
            float xh[VEC], dy[VEC], w[VEC];
            load_grad<DT>(k, row, c, mean, rstd, xh, dy);
            load_row_params<DT>(k.weight, k.f32_params, c, k.C, 1.0f, w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float u = dy[i] * w[i];
                s1 += u;
                s2 += c + i < k.C ? u * xh[i] : 0.0f;
            }
        }
        __syncthreads();
        s1 = group_sum<T>(s1, lds[0]) / (float)k.C;
        s2 = group_sum<T>(s2, lds[1]) / (float)k.C;
        for (uint32_t c = threadIdx.x * VEC; c < k.C; c += T * VEC) {
            float xh[VEC], dy[VEC], w[VEC], dt[VEC] = {};
            load_grad<DT>(k, row, c, mean, rstd, xh, dy);
            load_row_params<DT>(k.weight, k.f32_params, c, k.C, 1.0f, w);
            if (k.dt.p) load_cols<DT>(row_of<DT>(k.dt, row), c, k.C, dt);
#pragma unroll
            for (int i = 0; i < VEC; ++i) xh[i] = __builtin_fmaf(rstd, (dy[i] * w[i] - s1) - xh[i] * s2, dt[i]);
            store_cols<DT>(const_cast<char *>(row_of<DT>(k.dx, row)), c, k.C, xh);
        }
    }
}

// Sums of dy and dy * xh over a part of the rows: a wave's worth of columns by a work-group, a wave every fourth row.
template <int DT>
__global__ __launch_bounds__(PT) void layer_norm_grad_parts_kernel(LayerNormK k)
{
    constexpr int VEC = K_VEC<DT>, W = PT / 64;
    __shared__ float lds[W][64 * VEC];
    const uint32_t lane = threadIdx.x % 64, wave = threadIdx.x / 64, tiles = (k.C + 64 * VEC - 1) / (64 * VEC);
    const uint32_t part = blockIdx.x / tiles, c0 = (blockIdx.x - part * tiles) * 64 * VEC, c = c0 + lane * VEC;
    const uint64_t end = min(k.rows, (part + 1) * k.per_part);
    float s[2][VEC] = {};
    if (c < k.C)
        for (uint64_t row = part * k.per_part + wave; row < end; row += W) {
            float xh[VEC], dy[VEC];
            load_grad<DT>(k, row, c, k.stats[2 * row], k.stats[2 * row + 1], xh, dy);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                s[0][i] += dy[i];
                s[1][i] = __builtin_fmaf(dy[i], xh[i], s[1][i]);
            }
        }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VEC; ++i) lds[wave][lane * VEC + i] = s[m][i];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < 64 * VEC && c0 + j < k.C; j += PT) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) sum += lds[w][j];
            k.part[2 * ((uint64_t)part * k.C + c0 + j) + m] = sum;
        }
    }
}

// Joins the parts: JC columns by a work-group, JT / JC lanes for each of them, in a fixed order.  Eight columns where there are few (256 columns, 256
// parts: 4.8 us), 32, whose pairs are two cache lines of a part, where that is work for every compute unit (2048 rows of 16384 columns 13.3 -> 6.8 us).
constexpr int JT = 1024;
template <int DT, int JC>
__global__ __launch_bounds__(JT) void layer_norm_grad_join_kernel(LayerNormK k)
{
    __shared__ float sums[2][JT / 64][JC];
    const uint32_t c = blockIdx.x * JC + threadIdx.x % JC;
    float s0 = 0.0f, s1 = 0.0f;
    if (c < k.C) {
#pragma unroll 8
        for (uint32_t p = threadIdx.x / JC; p < k.parts; p += JT / JC) {
            const float2 in = *reinterpret_cast<const float2 *>(k.part + 2 * ((uint64_t)p * k.C + c));
            s0 += in.x;
            s1 += in.y;
        }
    }
    s0 = teams_sum<JC>(s0);
    s1 = teams_sum<JC>(s1);
    if (threadIdx.x % 64 < JC) {
        sums[0][threadIdx.x / 64][threadIdx.x % JC] = s0;
        sums[1][threadIdx.x / 64][threadIdx.x % JC] = s1;
    }
    __syncthreads();
    if (threadIdx.x >= JC || c >= k.C) return;
    float b = 0.0f, w = 0.0f;
#pragma unroll
    for (int i = 0; i < JT / 64; ++i) {
        b += sums[0][i][threadIdx.x];
        w += sums[1][i][threadIdx.x];
    }
    put_params<DT>(k, c, b, w);
}

// ------------------------------------------------------------------------------------------------ launches
bs_status checked()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

template <int DT>
void launch(LayerNormPass pass, const LayerNormK &k, hipStream_t st)
{
    const dim3 rows((uint32_t)(k.rows < K_LAYER_NORM_ROW_GROUPS ? k.rows : K_LAYER_NORM_ROW_GROUPS)), block(T);
    const uint32_t tiles = (k.C + 64 * K_VEC<DT> - 1) / (64 * K_VEC<DT>);
    switch (pass) {
    case LAYER_NORM: layer_norm_kernel<DT><<<rows, block, 0, st>>>(k); break;
    case LAYER_NORM_GRAD: layer_norm_grad_kernel<DT><<<rows, block, 0, st>>>(k); break;
    case LAYER_NORM_GRAD_PARTS: layer_norm_grad_parts_kernel<DT><<<dim3(tiles * k.parts), dim3(PT), 0, st>>>(k); break;
    case LAYER_NORM_GRAD_JOIN:
        if (k.C >= 32 * 256) layer_norm_grad_join_kernel<DT, 32><<<dim3((k.C + 31) / 32), dim3(JT), 0, st>>>(k);
        else layer_norm_grad_join_kernel<DT, 8><<<dim3((k.C + 7) / 8), dim3(JT), 0, st>>>(k);
        break;
    }
}

}  // namespace

bs_status launch_layer_norm(LayerNormPass pass, const LayerNormK &k, int32_t dtype, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) launch<DT_F32>(pass, k, st);
    else if (dtype == BS_BF16) launch<DT_BF16>(pass, k, st);
    else launch<DT_F16>(pass, k, st);
    return checked();
}

}  // namespace bs
