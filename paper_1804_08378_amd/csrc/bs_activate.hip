// Activations with a gate, and tensors in 8 bits: kernels over the elements of rows.
//
//   y = act(x) * gate;  dx = dy * gate * act'(x),  dg = dy * act(x);  x and gate as they are, or as code * step of their block of 32
//
// A lane keeps 128 bits of every tensor; four (float32: eight) neighbouring lanes hold a block and find its largest magnitude by exchanges inside
// the wave.  A work-group takes neighbouring vectors across row ends, so that short rows leave no lanes without work but those behind a row's end.
#include <hip/hip_runtime.h>

#include "bs_activate.h"
#include "bs_norm_device.h"
#include "bs_rows8_device.h"

namespace bs {
namespace {

constexpr int T = K_ACTIVATE_THREADS, U = K_ACTIVATE_UNROLL;

struct At {
    uint64_t row;
    uint32_t c;
};

// The row and column of vector blockIdx.x * T * U + l.
struct Place {
    uint64_t row0;
    uint32_t rest;
    BS_DEV explicit Place(const ActivateK &k)
    {
        const uint64_t base = (uint64_t)blockIdx.x * (T * U);
        row0 = k.vectors < (1u << 31) ? fdiv((uint32_t)base, k.by_row) : base / k.per_row;
        rest = (uint32_t)(base - row0 * k.per_row);
    }
    template <int DT>
    BS_DEV At at(const ActivateK &k, uint32_t l) const
    {
        const uint32_t t = rest + l, r = fdiv(t, k.by_row);
        return At{row0 + r, (t - r * k.per_row) * K_VEC<DT>};
    }
};

template <int DT>
BS_DEV const char *row_of(const RowTensor &t, uint64_t row) { return static_cast<const char *>(t.p) + row * t.stride * K_ES<DT>; }

template <int DT, int ACT>
BS_DEV void act_and_slope(float z, float &value, float &slope)
{
    if constexpr (ACT == BS_ACT_SILU) {
        const float s = sigmoid<DT>(z);
        value = z * s;
        slope = s * (1.0f + z * (1.0f - s));
    } else if constexpr (ACT == BS_ACT_GELU) {
        float density_z;
        const float below = normal<DT>(z, density_z);
        value = z * below;
        slope = below + density_z;
    } else {
        value = act<DT, ACT>(z);
        slope = act_slope<DT, ACT>(z);
    }
}

template <int DT, int ACT, bool GATE, bool HELD>
__global__ __launch_bounds__(T) void activate_kernel(ActivateK k)
{
    const Place place(k);
    const uint64_t left = k.vectors - (uint64_t)blockIdx.x * (T * U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t l = u * T + threadIdx.x;
        if (l >= left) return;  // (whole blocks of lanes at a time)
        const At a = place.at<DT>(k, l);
        float x[K_VEC<DT>], g[K_VEC<DT>], y[K_VEC<DT>];
        Raw<DT, K_VEC<DT>> xw, gw;
        xw = load_vector<DT>(row_of<DT>(k.x, a.row), a.c, k.columns);
        if constexpr (GATE) gw = load_vector<DT>(row_of<DT>(k.gate, a.row), a.c, k.columns);
        xw = settled<DT>(xw, a.c, k.columns);
        if constexpr (GATE) gw = settled<DT>(gw, a.c, k.columns);
        unpack<DT, K_VEC<DT>>(xw, x);
        if constexpr (GATE) unpack<DT, K_VEC<DT>>(gw, g);
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i) {
            y[i] = act<DT, ACT>(x[i]);
            if constexpr (GATE) y[i] *= g[i];
        }
        store_cols<DT>(const_cast<char *>(row_of<DT>(k.y, a.row)), a.c, k.columns, y);
        if constexpr (HELD) {
            store_held<DT>(k.hx, a.row, a.c, k.columns, xw, x);
            if constexpr (GATE) store_held<DT>(k.hg, a.row, a.c, k.columns, gw, g);
        }
    }
}

template <int DT, int ACT, bool GATE, bool HELD>
__global__ __launch_bounds__(T) void activate_grad_kernel(ActivateK k)
{
    const Place place(k);
    const uint64_t left = k.vectors - (uint64_t)blockIdx.x * (T * U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t l = u * T + threadIdx.x;
        if (l >= left) return;
        const At a = place.at<DT>(k, l);
        float x[K_VEC<DT>], g[K_VEC<DT>], dy[K_VEC<DT>], dg[K_VEC<DT>];
        HeldVector<DT> hx, hg;
        Raw<DT, K_VEC<DT>> xw, gw, dw;
        if constexpr (HELD) hx.load(k.hx, a.row, a.c, k.columns);
        else xw = load_vector<DT>(row_of<DT>(k.x, a.row), a.c, k.columns);
        if constexpr (GATE && HELD) hg.load(k.hg, a.row, a.c, k.columns);
        if constexpr (GATE && !HELD) gw = load_vector<DT>(row_of<DT>(k.gate, a.row), a.c, k.columns);
        dw = load_vector<DT>(row_of<DT>(k.dy, a.row), a.c, k.columns);
        if constexpr (HELD) hx.numbers(a.c, k.columns, x);
        else unpack<DT, K_VEC<DT>>(settled<DT>(xw, a.c, k.columns), x);
        if constexpr (GATE && HELD) hg.numbers(a.c, k.columns, g);
        if constexpr (GATE && !HELD) unpack<DT, K_VEC<DT>>(settled<DT>(gw, a.c, k.columns), g);
        unpack<DT, K_VEC<DT>>(settled<DT>(dw, a.c, k.columns), dy);
#pragma unroll
        for (int i = 0; i < K_VEC<DT>; ++i) {
            float value, slope;
            act_and_slope<DT, ACT>(x[i], value, slope);
            dg[i] = dy[i] * value;
            x[i] = dy[i] * slope;
            if constexpr (GATE) x[i] *= g[i];
        }
        if (k.dx.p) store_cols<DT>(const_cast<char *>(row_of<DT>(k.dx, a.row)), a.c, k.columns, x);
        if (GATE && k.dg.p) store_cols<DT>(const_cast<char *>(row_of<DT>(k.dg, a.row)), a.c, k.columns, dg);
    }
}

template <int DT, bool BACK>
__global__ __launch_bounds__(T) void pack8_kernel(ActivateK k)
{
    const Place place(k);
    const uint64_t left = k.vectors - (uint64_t)blockIdx.x * (T * U);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t l = u * T + threadIdx.x;
        if (l >= left) return;
        const At a = place.at<DT>(k, l);
        float x[K_VEC<DT>];
        if constexpr (BACK) {
            HeldVector<DT> h;
            h.load(k.hx, a.row, a.c, k.columns);
            h.numbers(a.c, k.columns, x);
            store_cols<DT>(const_cast<char *>(row_of<DT>(k.y, a.row)), a.c, k.columns, x);
        } else {
            const Raw<DT, K_VEC<DT>> w = settled<DT>(load_vector<DT>(row_of<DT>(k.x, a.row), a.c, k.columns), a.c, k.columns);
            unpack<DT, K_VEC<DT>>(w, x);
            store_held<DT>(k.hx, a.row, a.c, k.columns, w, x);
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

template <int DT, int ACT, bool GATE, bool HELD>
void launch(RowPass pass, const ActivateK &k, dim3 grid, hipStream_t st)
{
    if (pass == ROWS_ACTIVATE) activate_kernel<DT, ACT, GATE, HELD><<<grid, dim3(T), 0, st>>>(k);
    else activate_grad_kernel<DT, ACT, GATE, HELD><<<grid, dim3(T), 0, st>>>(k);
}

template <int DT, int ACT>
void launch_act(RowPass pass, const ActivateK &k, dim3 grid, hipStream_t st)
{
    const bool gate = k.gate.p || k.hg.codes, held = k.hx.codes;
    if (gate && held) launch<DT, ACT, true, true>(pass, k, grid, st);
    else if (gate) launch<DT, ACT, true, false>(pass, k, grid, st);
    else if (held) launch<DT, ACT, false, true>(pass, k, grid, st);
    else launch<DT, ACT, false, false>(pass, k, grid, st);
}

template <int DT>
void launch_type(RowPass pass, const ActivateK &k, int32_t activation, dim3 grid, hipStream_t st)
{
    if (pass == ROWS_PACK8) pack8_kernel<DT, false><<<grid, dim3(T), 0, st>>>(k);
    else if (pass == ROWS_UNPACK8) pack8_kernel<DT, true><<<grid, dim3(T), 0, st>>>(k);
    else if (activation == BS_ACT_IDENTITY) launch_act<DT, BS_ACT_IDENTITY>(pass, k, grid, st);
    else if (activation == BS_ACT_RELU) launch_act<DT, BS_ACT_RELU>(pass, k, grid, st);
    else if (activation == BS_ACT_SILU) launch_act<DT, BS_ACT_SILU>(pass, k, grid, st);
    else launch_act<DT, BS_ACT_GELU>(pass, k, grid, st);
}

}  // namespace

bs_status launch_rows(RowPass pass, const ActivateK &k, int32_t dtype, int32_t activation, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((uint32_t)((k.vectors + T * U - 1) / (T * U)));
    if (dtype == BS_F32) launch_type<DT_F32>(pass, k, activation, grid, st);
    else if (dtype == BS_BF16) launch_type<DT_BF16>(pass, k, activation, grid, st);
    else launch_type<DT_F16>(pass, k, activation, grid, st);
    return checked();
}

}  // namespace bs
