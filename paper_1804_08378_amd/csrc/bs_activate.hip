// Activations with a gate, and tensors in 8 bits: kernels over the elements of rows.
//
//   y = act(x) * gate;  dx = dy * gate * act'(x),  dg = dy * act(x);  x and gate as they are, or as code * step of their block of 32
//
// A lane keeps 128 bits of every tensor; four (float32: eight) neighbouring lanes hold a block and find its largest magnitude by exchanges inside
// the wave.  A work-group takes neighbouring vectors across row ends, so that short rows leave no lanes without work but those behind a row's end.
// Memory bounds it: 8192 x 8192 bfloat16 with a gate, both operands to 8 bits, 82 us forward (6.6 TB/s) and 100 backward (5.4); 200704 x 256 to 8 bits 29 us
// and back 25 (5.4, 6.3).  Both directions of the former, before the loads of a lane stood side by side: two vectors a lane 195 us, four 205, one 184; with
// the codes' stores through the caches, where their next reader finds some of them, 182, with the tensors' too 192.
#include <hip/hip_runtime.h>

#include "bs_activate.h"
#include "bs_norm_device.h"
#include "bs_rows8_device.h"

#include <type_traits>

namespace bs {
namespace {

constexpr int T = K_ACTIVATE_THREADS;

struct At {
    uint64_t row;
    uint32_t c;
};

BS_DEV bool on(const ActivateK &k) { return (uint64_t)blockIdx.x * T + threadIdx.x < k.vectors; }  // (whole blocks of lanes at a time)

// The row and first column of the lane's vector.
template <int DT>
BS_DEV At place_of(const ActivateK &k)
{
    const uint64_t base = (uint64_t)blockIdx.x * T, row0 = k.vectors < (1u << 31) ? fdiv((uint32_t)base, k.by_row) : base / k.per_row;
    const uint32_t t = (uint32_t)(base - row0 * k.per_row) + threadIdx.x, r = fdiv(t, k.by_row);
    return At{row0 + r, (t - r * k.per_row) * K_VEC<DT>};
}

// A lane's vector of a tensor or of a tensor in 8 bits, behind `get` in flight, behind `place` as numbers' words.  SHORT: rows shorter than a vector, read
// in pieces.
template <int DT, bool SHORT>
struct Words {
    Raw<DT, K_VEC<DT>> r;
    BS_DEV void get(const RowTensor &t, const At &a, uint32_t columns)
    {
        if constexpr (SHORT) r = load_vector<DT>(row_of<DT>(t, a.row), a.c, columns);
        else r = read_vector<DT>(t, a.row, read_column<DT>(a.c, columns));
    }
    BS_DEV void place(const At &a, uint32_t columns)
    {
        if (!SHORT && columns % BS_PACK8_BLOCK != 0) r = moved<DT>(r, early_by<K_VEC<DT>>(a.c, columns));
    }
    BS_DEV void numbers(float (&v)[K_VEC<DT>]) const { unpack<DT, K_VEC<DT>>(r, v); }
};
template <int DT, bool SHORT>
struct Codes {
    HeldVector<DT> h;
    BS_DEV void get(const HeldRows &t, const At &a, uint32_t columns)
    {
        if constexpr (SHORT) h.load(t, a.row, a.c, columns);
        else h.read(t, a.row, a.c, columns);
    }
    BS_DEV void place(const At &a, uint32_t columns)
    {
        if (!SHORT && columns % BS_PACK8_BLOCK != 0) h.move(early_by<K_VEC<DT>>(a.c, columns));
    }
    BS_DEV void numbers(float (&v)[K_VEC<DT>]) const { h.numbers(v); }
};

template <int DT>
BS_DEV void store(const RowTensor &t, const At &a, uint32_t columns, const float (&v)[K_VEC<DT>])
{
    store_cols<DT>(const_cast<char *>(row_of<DT>(t, a.row)), a.c, columns, v);
}

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

template <int DT, int ACT, bool GATE, bool HELD, bool SHORT>
BS_DEV void activate(const ActivateK &k, const At &a)
{
    Words<DT, SHORT> xw, gw;
    xw.get(k.x, a, k.columns);
    if constexpr (GATE) gw.get(k.gate, a, k.columns);
    xw.place(a, k.columns);
    if constexpr (GATE) gw.place(a, k.columns);
    float x[K_VEC<DT>], g[K_VEC<DT>], y[K_VEC<DT>];
    xw.numbers(x);
    if constexpr (GATE) gw.numbers(g);
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        y[i] = act<DT, ACT>(x[i]);
        if constexpr (GATE) y[i] *= g[i];
    }
    store<DT>(k.y, a, k.columns, y);
    if constexpr (HELD) {
        store_held<DT>(k.hx, a.row, a.c, k.columns, xw.r, x);
        if constexpr (GATE) store_held<DT>(k.hg, a.row, a.c, k.columns, gw.r, g);
    }
}

template <int DT, int ACT, bool GATE, bool HELD, bool SHORT>
BS_DEV void activate_grad(const ActivateK &k, const At &a)
{
    using Kept = typename std::conditional<HELD, Codes<DT, SHORT>, Words<DT, SHORT>>::type;
    Kept xw, gw;
    Words<DT, SHORT> dw;
    if constexpr (HELD) {
        xw.get(k.hx, a, k.columns);
        if constexpr (GATE) gw.get(k.hg, a, k.columns);
    } else {
        xw.get(k.x, a, k.columns);
        if constexpr (GATE) gw.get(k.gate, a, k.columns);
    }
    dw.get(k.dy, a, k.columns);
    float x[K_VEC<DT>], g[K_VEC<DT>], dy[K_VEC<DT>], dg[K_VEC<DT>];
    xw.place(a, k.columns);
    if constexpr (GATE) gw.place(a, k.columns);
    dw.place(a, k.columns);
    xw.numbers(x);
    if constexpr (GATE) gw.numbers(g);
    dw.numbers(dy);
#pragma unroll
    for (int i = 0; i < K_VEC<DT>; ++i) {
        float value, slope;
        act_and_slope<DT, ACT>(x[i], value, slope);
        dg[i] = dy[i] * value;
        x[i] = dy[i] * slope;
        if constexpr (GATE) x[i] *= g[i];
    }
    if (k.dx.p) store<DT>(k.dx, a, k.columns, x);
    if (GATE && k.dg.p) store<DT>(k.dg, a, k.columns, dg);
}

template <int DT, bool BACK, bool SHORT>
BS_DEV void pack8(const ActivateK &k, const At &a)
{
    float x[K_VEC<DT>];
    if constexpr (BACK) {
        Codes<DT, SHORT> h;
        h.get(k.hx, a, k.columns);
        h.place(a, k.columns);
        h.numbers(x);
        store<DT>(k.y, a, k.columns, x);
    } else {
        Words<DT, SHORT> w;
        w.get(k.x, a, k.columns);
        w.place(a, k.columns);
        w.numbers(x);
        store_held<DT>(k.hx, a.row, a.c, k.columns, w.r, x);
    }
}

template <int DT, int ACT, bool GATE, bool HELD>
__global__ __launch_bounds__(T) void activate_kernel(ActivateK k)
{
    if (!on(k)) return;
    const At a = place_of<DT>(k);
    if (k.columns < K_VEC<DT>) activate<DT, ACT, GATE, HELD, true>(k, a);
    else activate<DT, ACT, GATE, HELD, false>(k, a);
}

template <int DT, int ACT, bool GATE, bool HELD>
__global__ __launch_bounds__(T) void activate_grad_kernel(ActivateK k)
{
    if (!on(k)) return;
    const At a = place_of<DT>(k);
    if (k.columns < K_VEC<DT>) activate_grad<DT, ACT, GATE, HELD, true>(k, a);
    else activate_grad<DT, ACT, GATE, HELD, false>(k, a);
}

template <int DT, bool BACK>
__global__ __launch_bounds__(T) void pack8_kernel(ActivateK k)
{
    if (!on(k)) return;
    const At a = place_of<DT>(k);
    if (k.columns < K_VEC<DT>) pack8<DT, BACK, true>(k, a);
    else pack8<DT, BACK, false>(k, a);
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
    const dim3 grid((uint32_t)((k.vectors + T - 1) / T));
    if (dtype == BS_F32) launch_type<DT_F32>(pass, k, activation, grid, st);
    else if (dtype == BS_BF16) launch_type<DT_BF16>(pass, k, activation, grid, st);
    else launch_type<DT_F16>(pass, k, activation, grid, st);
    return checked();
}

}  // namespace bs
