// Layer normalisation, forward, with the rows in registers (bs_layer_norm_team.h); formulas: bs_layer_norm.hip.
#include <hip/hip_runtime.h>

#include "bs_layer_norm_team.h"

namespace bs {
namespace {

// Lanes of a work-group: a team of several waves, or as many teams as four waves hold.
template <int TEAM>
constexpr int K_THREADS = TEAM <= 64 ? 256 : TEAM;

template <int DT, int TEAM, int NV, bool ADD>
__global__ __launch_bounds__(K_THREADS<TEAM>) void layer_norm_team_kernel(LayerNormK k)
{
    constexpr int VEC = K_VEC<DT>, T = K_THREADS<TEAM>, W = TEAM / 64;  // W: waves of a team, 0: several teams in a wave
    constexpr bool HOLD = NV * VEC <= 16, AHEAD = TEAM * NV < 4096;  // weight and bias stay in registers; the next row is loaded ahead
    constexpr uint32_t TEAMS = T / TEAM;
    __shared__ float lds[2][W > 1 ? W : 1][2];
    const uint32_t lane = threadIdx.x % TEAM, team = team_of<TEAM, T>();
    const bool whole = k.C % VEC == 0;
    float w[HOLD ? NV : 1][VEC], b[HOLD ? NV : 1][VEC];
    if constexpr (HOLD)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = (j * TEAM + lane) * VEC;
            load_row_params<DT>(k.weight, k.f32_params, c, k.C, 1.0f, w[j]);
            load_row_params<DT>(k.bias, k.f32_params, c, k.C, 0.0f, b[j]);
        }
    // columns of a wave of the team
    auto columns_of = [&](uint32_t wave) {
        uint32_t n = 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = (j * TEAM + wave * 64) * VEC;
            n += c < k.C ? min(k.C - c, (uint32_t)(64 * VEC)) : 0;
        }
        return (float)n;
    };
    const float share = 1.0f / (float)k.C, own = W > 1 ? columns_of(threadIdx.x / 64) : 0.0f;
    const float wave_share = W > 1 ? (own > 0.0f ? 1.0f / own : 0.0f) : share;
    const float other = W > 1 ? columns_of(threadIdx.x % (W > 1 ? W : 1)) : 0.0f;  // columns of the wave whose sums the lane joins
    const bool full = k.C == (uint32_t)(TEAM * NV * VEC);
    Raw<DT, VEC> x[NV], a[NV];
    auto load = [&](uint64_t row) {
        row = min(row, k.rows - 1);  // (rows behind the last are not written)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t at = read_column<DT>((j * TEAM + lane) * VEC, k.C);
            x[j] = read_vector<DT>(k.x, row, at);
            if constexpr (ADD) a[j] = read_vector<DT>(k.addend, row, at);
        }
    };
    uint64_t first = (uint64_t)blockIdx.x * TEAMS;  // the same for all lanes of a work-group
    if constexpr (AHEAD) load(first + team);
    for (uint32_t turn = 0; first < k.rows; first += (uint64_t)gridDim.x * TEAMS, turn ^= 1) {
        const uint64_t row = first + team;
        if constexpr (!AHEAD) load(row);
        Raw<DT, VEC> t[NV];
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            t[j] = x[j];
            float v[VEC];
            if constexpr (ADD) {
                float add[VEC];
                unpack<DT, VEC>(t[j], v);
                unpack<DT, VEC>(a[j], add);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] += add[i];
                t[j] = to_words<DT>(v);
            }
            if (!full) t[j] = moved<DT>(t[j], early_by<VEC>((j * TEAM + lane) * VEC, k.C));
            unpack<DT, VEC>(t[j], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) s += v[i];
        }
        if constexpr (AHEAD) load(first + (uint64_t)gridDim.x * TEAMS + team);
        s = lanes_sum<TEAM < 64 ? TEAM : 64>(s);
        float mean = s * wave_share, m2 = 0.0f;  // of a wave's columns
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = (j * TEAM + lane) * VEC;
            forget(t[j].q);
            if (c < k.C) {
                float v[VEC];
                unpack<DT, VEC>(t[j], v);
                if (whole) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) m2 = __builtin_fmaf(v[i] - mean, v[i] - mean, m2);
                } else {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        const float d = c + i < k.C ? v[i] - mean : 0.0f;
                        m2 = __builtin_fmaf(d, d, m2);
                    }
                }
            }
        }
        m2 = lanes_sum<TEAM < 64 ? TEAM : 64>(m2);
        if constexpr (W > 1) {
            if (threadIdx.x % 64 == 0) {
                lds[turn][threadIdx.x / 64][0] = mean;
                lds[turn][threadIdx.x / 64][1] = m2;
            }
            __syncthreads();  // (the other turn's values are read before the next barrier)
            const float mw = lds[turn][threadIdx.x % W][0], qw = lds[turn][threadIdx.x % W][1];
            mean = lanes_sum<W>(other * mw) * share;
            m2 = lanes_sum<W>(__builtin_fmaf(other * (mw - mean), mw - mean, qw));
        }
        const float rstd = reciprocal_root(__builtin_fmaf(m2, share, k.eps));
        if (row >= k.rows) continue;  // (teams of one wave)
        if (k.stats && lane == 0) *reinterpret_cast<float2 *>(k.stats + 2 * row) = make_float2(mean, rstd);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = (j * TEAM + lane) * VEC;
            forget(t[j].q);
            if (k.total.p) store_vector<DT>(const_cast<char *>(row_of<DT>(k.total, row)), c, k.C, t[j]);
            float v[VEC], wj[VEC], bj[VEC];
            unpack<DT, VEC>(t[j], v);
            if (k.held.codes) store_held<DT>(k.held, row, c, k.C, t[j], v);
            if constexpr (!HOLD) {
                load_row_params<DT>(k.weight, k.f32_params, afresh(c), k.C, 1.0f, wj);
                load_row_params<DT>(k.bias, k.f32_params, afresh(c), k.C, 0.0f, bj);
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = __builtin_fmaf((v[i] - mean) * rstd, HOLD ? w[HOLD ? j : 0][i] : wj[i], HOLD ? b[HOLD ? j : 0][i] : bj[i]);
            // y through the caches behind an addition, past them without one (the total always past them).  8192 x 4096 bfloat16 behind an addition: y
            // past the caches too 53 us, through them 49.  Without one, both directions of 200704 x 256 and 8192 x 1024 float32: past them 98 and 33 us, through 102
            // and 35.
            store_cols<DT, !ADD>(const_cast<char *>(row_of<DT>(k.y, row)), c, k.C, v);
            if constexpr (!HOLD) __builtin_amdgcn_sched_barrier(0);  // (one vector's numbers at a time in registers)
        }
    }
}

template <int DT, int TEAM, int NV>
void launch(const LayerNormK &k, uint32_t groups, hipStream_t st)
{
    const dim3 grid(groups), block(K_THREADS<TEAM>);
    if (k.addend.p) layer_norm_team_kernel<DT, TEAM, NV, true><<<grid, block, 0, st>>>(k);
    else layer_norm_team_kernel<DT, TEAM, NV, false><<<grid, block, 0, st>>>(k);
}

template <int DT>
void launch_type(const LayerNormK &k, const LayerNormTeam &t, hipStream_t st)
{
    switch (t.team * 16 + t.vectors) {
    case 8 * 16 + 1: launch<DT, 8, 1>(k, t.groups, st); break;
    case 16 * 16 + 1: launch<DT, 16, 1>(k, t.groups, st); break;
    case 32 * 16 + 1: launch<DT, 32, 1>(k, t.groups, st); break;
    case 64 * 16 + 1: launch<DT, 64, 1>(k, t.groups, st); break;
    case 128 * 16 + 1: launch<DT, 128, 1>(k, t.groups, st); break;
    case 256 * 16 + 1: launch<DT, 256, 1>(k, t.groups, st); break;
    case 512 * 16 + 1: launch<DT, 512, 1>(k, t.groups, st); break;
    case 1024 * 16 + 1: launch<DT, 1024, 1>(k, t.groups, st); break;
    case 1024 * 16 + 2: launch<DT, 1024, 2>(k, t.groups, st); break;
    case 1024 * 16 + 4: launch<DT, 1024, 4>(k, t.groups, st); break;
    }
}

}  // namespace

bs_status launch_layer_norm_team(const LayerNormK &k, const LayerNormTeam &t, int32_t dtype, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) launch_type<DT_F32>(k, t, st);
    else if (dtype == BS_BF16) launch_type<DT_BF16>(k, t, st);
    else launch_type<DT_F16>(k, t, st);
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

}  // namespace bs
