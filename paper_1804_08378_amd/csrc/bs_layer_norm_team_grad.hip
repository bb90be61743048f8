// Layer normalisation, backward, with the rows in registers (bs_layer_norm_team.h); formulas: bs_layer_norm.hip.
//
// A lane keeps the sums of dy and dy * xh of its columns over all rows of its team, in registers or, of long rows, in LDS (of rows over 16384 columns nowhere: bs_layer_norm.hip sums them); a work-group's teams are
// added through LDS at the end, and the work-groups' sums are joined by a second launch, in orders that depend on sizes only: equal calls give equal
// bits.  A work-group is as large as a compute unit takes, and there is one for each: the fewer there are, the fewer sums cross memory (256 parts of 4096
// columns are 8.4 MB beside the 201 MB of 8192 rows).  The join is a launch of 2.5 to 7 us.
#include <hip/hip_runtime.h>

#include "bs_layer_norm_team.h"

namespace bs {
namespace {

// A lane's vector of the normalised rows: as they are, or codes and the block's exponent.
template <int DT, bool HELD>
struct Kept {
    Raw<DT, K_VEC<DT>> words;
    BS_DEV void read(const LayerNormK &k, uint64_t row, uint32_t c, uint32_t at) { words = read_vector<DT>(k.x, row, at); }
    BS_DEV void move(uint32_t early) { words = moved<DT>(words, early); }
    BS_DEV void numbers(float (&v)[K_VEC<DT>]) const { unpack<DT, K_VEC<DT>>(words, v); }
    BS_DEV void forget() { bs::forget(words.q); }
};
template <int DT>
struct Kept<DT, true> {
    HeldVector<DT> h;
    BS_DEV void read(const LayerNormK &k, uint64_t row, uint32_t c, uint32_t at) { h.read(k.held, row, c, k.C); }
    BS_DEV void move(uint32_t early) { h.move(early); }
    BS_DEV void numbers(float (&v)[K_VEC<DT>]) const { h.numbers(v); }
    BS_DEV void forget()
    {
#pragma unroll
        for (int i = 0; i < K_VEC<DT> / 4; ++i) asm("" : "+v"(h.codes[i]));
    }
};

constexpr int T = K_LAYER_NORM_GRAD_THREADS;

enum Sums { SUMS_NONE, SUMS_REGISTERS, SUMS_LDS };  // of a lane's columns: where they are kept

template <int DT, int TEAM, int NV, bool HELD, bool TOTAL, Sums SUMS>
__global__ __launch_bounds__(T) void layer_norm_team_grad_kernel(LayerNormK k)
{
    constexpr int VEC = K_VEC<DT>, W = TEAM / 64;
    constexpr bool HOLD = NV * VEC <= 8, AHEAD = NV <= 2;  // weights stay in registers; the next row is loaded ahead
    constexpr bool AGAIN = HELD && SUMS == SUMS_NONE;  // codes are read once more from the cache instead of kept in registers
    constexpr uint32_t TEAMS = T / TEAM;
    constexpr int COLUMNS = TEAM * NV * VEC;
    constexpr uint32_t SUMMED = TEAM < 64 ? T / 64 : TEAMS;  // parts of a column's sum in a work-group
    static_assert(SUMMED == 1 || (SUMS == SUMS_REGISTERS && NV == 1), "long rows: a team a work-group");
    __shared__ float lds[2][T / 64][2];
    __shared__ float sums[2][SUMS == SUMS_LDS ? COLUMNS : SUMMED > 1 ? SUMMED / 2 * COLUMNS : 1];  // [j][i][lane]: neighbouring lanes in neighbouring banks
    const uint32_t lane = threadIdx.x % TEAM, team = team_of<TEAM, T>();
    constexpr int NS = SUMS == SUMS_REGISTERS ? NV : 1;
    float w[HOLD ? NV : 1][VEC], db[NS][VEC] = {}, dw[NS][VEC] = {};
    if constexpr (HOLD)
#pragma unroll
        for (int j = 0; j < NV; ++j) load_row_params<DT>(k.weight, k.f32_params, (j * TEAM + lane) * VEC, k.C, 1.0f, w[j]);
    if constexpr (SUMS == SUMS_LDS)  // (a lane adds to its own columns only)
        for (int i = 0; i < NV * VEC; ++i) sums[0][i * TEAM + lane] = sums[1][i * TEAM + lane] = 0.0f;
    const float share = 1.0f / (float)k.C;
    // a lane's first column of its j-th vector; of several ones worked out at every use, where the compiler would keep all that follows from it
    auto column = [&](int j) { return HOLD ? (j * TEAM + lane) * VEC : afresh((j * TEAM + lane) * VEC); };
    Kept<DT, HELD> x[NV], nx[NV];
    Raw<DT, VEC> dy[NV], dt[NV], ndy[NV], ndt[NV];
    float2 stats;
    const bool full = k.C == (uint32_t)COLUMNS;
    auto load = [&](uint64_t row) {
        row = min(row, k.rows - 1);  // (rows behind the last are emptied at their first use)
        stats = *reinterpret_cast<const float2 *>(k.stats + 2 * row);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const uint32_t c = column(j), at = read_column<DT>(c, k.C);
            nx[j].read(k, row, c, at);
            ndy[j] = read_vector<DT>(k.dy, row, at);
            if constexpr (AHEAD && TOTAL) ndt[j] = read_vector<DT>(k.dt, row, at);
        }
    };
    // xh and u of a vector, made of its words
    auto numbers = [&](int j, float mean, float rstd, float (&xh)[VEC], float (&g)[VEC], float (&u)[VEC]) {
        float wj[VEC];
        x[j].numbers(xh);
        unpack<DT, VEC>(dy[j], g);
        if constexpr (!HOLD) load_row_params<DT>(k.weight, k.f32_params, column(j), k.C, 1.0f, wj);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            xh[i] = (xh[i] - mean) * rstd;
            u[i] = g[i] * (HOLD ? w[HOLD ? j : 0][i] : wj[i]);
        }
    };
    uint64_t first = (uint64_t)blockIdx.x * TEAMS;  // the same for all lanes of a work-group
    if constexpr (AHEAD) load(first + team);
    for (uint32_t turn = 0; first < k.rows; first += (uint64_t)gridDim.x * TEAMS, turn ^= 1) {
        const uint64_t row = first + team;
        if constexpr (!AHEAD) load(row);
        const bool on = row < k.rows;
        const float mean = on ? stats.x : 0.0f, rstd = on ? stats.y : 0.0f;
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            x[j] = nx[j];
            dy[j] = ndy[j];
            if constexpr (AHEAD && TOTAL) dt[j] = ndt[j];
        }
        if constexpr (AHEAD) load(first + (uint64_t)gridDim.x * TEAMS + team);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float xh[VEC], g[VEC], u[VEC];
            if (!full || !on) {
                const uint32_t early = on ? early_by<VEC>(column(j), k.C) : VEC;
                x[j].move(early);
                dy[j] = moved<DT>(dy[j], early);
            }
            numbers(j, mean, rstd, xh, g, u);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                if constexpr (SUMS == SUMS_REGISTERS) {
                    db[j][i] += g[i];
                    dw[j][i] = __builtin_fmaf(g[i], xh[i], dw[j][i]);
                }
                if constexpr (SUMS == SUMS_LDS) {
                    const uint32_t at = (j * VEC + i) * TEAM + lane;
                    sums[0][at] += g[i];
                    sums[1][at] = __builtin_fmaf(g[i], xh[i], sums[1][at]);
                }
                s1 += u[i];
                s2 = __builtin_fmaf(u[i], xh[i], s2);
            }
            if constexpr (!HOLD) __builtin_amdgcn_sched_barrier(0);
        }
        s1 = lanes_sum<TEAM < 64 ? TEAM : 64>(s1);
        s2 = lanes_sum<TEAM < 64 ? TEAM : 64>(s2);
        if constexpr (W > 1) {
            if (threadIdx.x % 64 == 0) {
                lds[turn][threadIdx.x / 64][0] = s1;
                lds[turn][threadIdx.x / 64][1] = s2;
            }
            __syncthreads();  // (the other turn's values are read before the next barrier)
            s1 = lanes_sum<W>(lds[turn][team * W + threadIdx.x % W][0]);
            s2 = lanes_sum<W>(lds[turn][team * W + threadIdx.x % W][1]);
        }
        s1 *= share;
        s2 *= share;
        if (k.dx.p && on)
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                float xh[VEC], g[VEC], u[VEC], add[VEC] = {};
                if constexpr (AGAIN) {
                    const uint32_t c = column(j);
                    x[j].read(k, row, c, read_column<DT>(c, k.C));
                    if (!full) x[j].move(early_by<VEC>(c, k.C));
                } else {
                    x[j].forget();
                }
                forget(dy[j].q);
                numbers(j, mean, rstd, xh, g, u);
                if constexpr (TOTAL) {
                    if constexpr (!AHEAD) dt[j] = read_vector<DT>(k.dt, row, read_column<DT>(column(j), k.C));
                    unpack<DT, VEC>(full ? dt[j] : moved<DT>(dt[j], early_by<VEC>(column(j), k.C)), add);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) u[i] = __builtin_fmaf(rstd, (u[i] - s1) - xh[i] * s2, add[i]);
                store_cols<DT>(const_cast<char *>(row_of<DT>(k.dx, row)), column(j), k.C, u);
                if constexpr (!HOLD) __builtin_amdgcn_sched_barrier(0);  // (one vector's numbers at a time in registers)
            }
    }
    if (SUMS == SUMS_NONE || !k.part) return;
    auto put = [&](int j, int i, float b, float g) {
        const uint32_t c = (j * TEAM + lane) * VEC + i;
        if (c >= k.C) return;
        if (gridDim.x == 1) put_params<DT>(k, c, b, g);
        else *reinterpret_cast<float2 *>(k.part + 2 * ((uint64_t)blockIdx.x * k.C + c)) = make_float2(b, g);
    };
    if constexpr (SUMS == SUMS_LDS) {
        for (int j = 0; j < NV; ++j)
            for (int i = 0; i < VEC; ++i) put(j, i, sums[0][(j * VEC + i) * TEAM + lane], sums[1][(j * VEC + i) * TEAM + lane]);
    } else if constexpr (SUMS == SUMS_REGISTERS) {
        if constexpr (TEAM < 64)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                db[0][i] = teams_sum<TEAM>(db[0][i]);
                dw[0][i] = teams_sum<TEAM>(dw[0][i]);
            }
        if constexpr (SUMMED > 1) {
            const uint32_t mine = threadIdx.x / (T / SUMMED);  // the upper half of the parts is added to the lower one, until one is left
            const bool part = threadIdx.x % (T / SUMMED) < TEAM;
            for (uint32_t half = SUMMED / 2; half; half /= 2) {
                __syncthreads();
                if (part && mine >= half && mine < 2 * half)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        sums[0][((mine - half) * VEC + i) * TEAM + lane] = db[0][i];
                        sums[1][((mine - half) * VEC + i) * TEAM + lane] = dw[0][i];
                    }
                __syncthreads();
                if (part && mine < half)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        db[0][i] += sums[0][(mine * VEC + i) * TEAM + lane];
                        dw[0][i] += sums[1][(mine * VEC + i) * TEAM + lane];
                    }
            }
            if (mine || !part) return;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) put(j, i, db[j][i], dw[j][i]);
    }
}

template <int DT, int TEAM, int NV, Sums SUMS>
void launch(const LayerNormK &k, uint32_t groups, hipStream_t st)
{
    const dim3 grid(groups), block(T);
    if (k.held.codes && k.dt.p) layer_norm_team_grad_kernel<DT, TEAM, NV, true, true, SUMS><<<grid, block, 0, st>>>(k);
    else if (k.held.codes) layer_norm_team_grad_kernel<DT, TEAM, NV, true, false, SUMS><<<grid, block, 0, st>>>(k);
    else if (k.dt.p) layer_norm_team_grad_kernel<DT, TEAM, NV, false, true, SUMS><<<grid, block, 0, st>>>(k);
    else layer_norm_team_grad_kernel<DT, TEAM, NV, false, false, SUMS><<<grid, block, 0, st>>>(k);
}

template <int DT>
void launch_type(const LayerNormK &k, const LayerNormTeam &t, hipStream_t st)
{
    switch (t.team * 16 + t.vectors) {
    case 8 * 16 + 1: launch<DT, 8, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 16 * 16 + 1: launch<DT, 16, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 32 * 16 + 1: launch<DT, 32, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 64 * 16 + 1: launch<DT, 64, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 128 * 16 + 1: launch<DT, 128, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 256 * 16 + 1: launch<DT, 256, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 512 * 16 + 1: launch<DT, 512, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 1024 * 16 + 1: launch<DT, 1024, 1, SUMS_REGISTERS>(k, t.groups, st); break;
    case 1024 * 16 + 2: launch<DT, 1024, 2, SUMS_LDS>(k, t.groups, st); break;
    case 1024 * 16 + 4:
        // two floats a column: 128 KiB of LDS hold those of 16384 columns
        if constexpr (DT == DT_F32) launch<DT, 1024, 4, SUMS_LDS>(k, t.groups, st);
        else launch<DT, 1024, 4, SUMS_NONE>(k, t.groups, st);
        break;
    }
}

}  // namespace

bs_status launch_layer_norm_team_grad(const LayerNormK &k, const LayerNormTeam &t, int32_t dtype, void *stream)
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
