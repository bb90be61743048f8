// Log probabilities of given classes, the entropy of every row's distribution and its top alternatives; and their gradient.
//
//   m = max x,  s = sum exp(x - m),  t = sum exp(x - m) (x - m);   lse = m + log s,  logp = x[target] - lse,  entropy = log s - t / s
//   dx_j = g (delta_j,target - p_j) - h p_j (log p_j + entropy),   p = exp(x - lse), g and h the gradients of logp and of entropy
//
// A lane keeps s and t running in float32 against a reference that need not be the maximum: one of the values seen, at most 1 below their
// maximum, so that it moves a few times in a row however long.  A class at -infinity has probability 0 and adds nothing.
//
// The top classes cost one comparison a vector: a lane remembers its best value and the vector that has it.  The k-th best of these bests
// bounds the k-th best class from below, and only the few lanes whose best passes the bound read their vectors again.
#include <hip/hip_runtime.h>

#include "bs_device.h"
#include "bs_exp_device.h"
#include "bs_internal.h"
#include "bs_log_probs.h"

namespace bs {
namespace {

constexpr float LOG2E = 1.44269504088896341f;
constexpr float FAR = -300.0f;      // 2 to this power is 0: stands for larger distances where they are multiplied by it
constexpr uint32_t LIST = 512;      // candidates for the top classes that a work-group keeps

template <int DT>
BS_DEV float element(const char *p, uint64_t i)
{
    if constexpr (DT == DT_F32) return reinterpret_cast<const float *>(p)[i];
    else return half_up<DT>(reinterpret_cast<const uint16_t *>(p)[i]);
}

// A class as one number: larger values first, then lower indices; NaN above all, -0 equal to 0.  Never 0 for a class.
BS_DEV uint64_t rank_key(float x, uint32_t j)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t o = x != x ? 0xffffffffu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (uint64_t)o << 32 | (0xffffffffu - j);
}
BS_DEV uint32_t key_index(uint64_t key) { return 0xffffffffu - (uint32_t)key; }
BS_DEV float key_value(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

BS_DEV int64_t target_of(const LogProbsK &k, uint64_t row)
{
    return k.wide_targets ? static_cast<const int64_t *>(k.targets)[row] : static_cast<const int32_t *>(k.targets)[row];
}

// ------------------------------------------------------------------------------------------------ sums
// Exponents in units of log2(e) x: one multiply-add an element.  The product is not rounded before the reference's is taken off, and the
// factor's own rounding stretches all logits alike, by 1.3e-8; t is taken back by the factor's reciprocal.
//
// The reference's product is rounded, and settle() takes that rounding out again: by a factor near 1 where references are below NEAR, but the
// factor leaves the range of float32 where they are 2^31.  So a lane takes no reference of a value beyond FINITE: below -FINITE (masks) classes
// count 0, which is exact next to any other, 64 from them at least; above it everything counts 0 until far_sums() has the largest.  That takes
// over too where the work-group's reference is beyond NEAR.
constexpr float UNIT = (float)(1.0 / (double)LOG2E);
constexpr float NEAR = 1048576.0f, FINITE = 1073741824.0f;
constexpr float UNSET = -FINITE;  // no reference yet

struct Sums {
    float ref = 0.0f, base = 0.0f;  // reference: a value seen, and its product with log2(e)
    float above = UNSET;            // the reference moves for values above this
    float s = 0.0f, t = 0.0f;       // sum of 2^d, of 2^d d,  d = log2(e) x - base

    template <int N>
    BS_DEV void add(const float (&v)[N], float most)
    {
        if (most > above) {
            const bool first = above == UNSET;
            const float to = most > FINITE ? INFINITY : most * LOG2E;
            const float d = first ? 0.0f : __builtin_fmaxf(base - to, FAR), f = first ? 0.0f : __builtin_amdgcn_exp2f(d);
            t = f * __builtin_fmaf(s, d, t);
            s *= f;
            ref = most;
            base = to;
            above = most + 1.0f;
        }
        float e[N], w = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = __builtin_fmaf(v[i], LOG2E, -base);
            e[i] = __builtin_amdgcn_exp2f(d);
            w = __builtin_fmaf(e[i], max2(d, FAR), w);
        }
#pragma unroll
        for (int n = N / 2; n; n /= 2)
#pragma unroll
            for (int i = 0; i < n; ++i) e[i] += e[i + n];
        s += e[0];
        t += w;
    }
    BS_DEV bool any() const { return above != UNSET; }
    // Sums that are complete, against this reference (-infinity: there is none).
    BS_DEV void against(float reference)
    {
        ref = reference;
        above = reference == -INFINITY ? UNSET : INFINITY;
    }
    // From the rounded product of the reference to the reference itself.
    BS_DEV void settle()
    {
        const float off = __builtin_fmaf(ref, LOG2E, -base);
        if (__builtin_fabsf(base) == INFINITY) return;  // (the sums are 0 or NaN)
        const float f = __builtin_amdgcn_exp2f(-off);
        t = f * __builtin_fmaf(-off, s, t);
        s *= f;
    }
    // Settled sums against another, larger reference (there is one, or the sums are 0 or NaN and stay so).
    BS_DEV void shift(float to)
    {
        const float d = any() ? __builtin_fmaxf((ref - to) * LOG2E, FAR) : FAR, f = __builtin_amdgcn_exp2f(d);
        t = f * __builtin_fmaf(s, d, t);
        s *= f;
        ref = to;
    }
    BS_DEV float log_s() const { return logf(s); }
    BS_DEV float entropy() const { return logf(s) - t / s * UNIT; }
    BS_DEV bool none() const { return s == 0.0f; }  // every class masked
    BS_DEV bool far() const { return none() || (__builtin_fabsf(ref) > NEAR && s == s); }  // joined: far_sums() has to take over
};

// One lane's value from another by a fixed pattern inside rows of 16 lanes.
template <int CTRL>
BS_DEV float in_row(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false));
}
constexpr int SWAP1 = 0xb1, SWAP2 = 0x4e, MIRROR8 = 0x141, MIRROR16 = 0x140;  // quad_perm, row_half_mirror, row_mirror

BS_DEV float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// Over the 64 lanes of a wave, the same in each: inside rows by patterns, the four rows by scalar reads (a shuffle through LDS costs five times a step).
BS_DEV float wave_sum(float v)
{
    v += in_row<SWAP1>(v);
    v += in_row<SWAP2>(v);
    v += in_row<MIRROR8>(v);
    v += in_row<MIRROR16>(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
BS_DEV float wave_max(float v)  // (NaN is left out)
{
    v = max2(v, in_row<SWAP1>(v));
    v = max2(v, in_row<SWAP2>(v));
    v = max2(v, in_row<MIRROR8>(v));
    v = max2(v, in_row<MIRROR16>(v));
    return max2(max2(lane_value(v, 0), lane_value(v, 16)), max2(lane_value(v, 32), lane_value(v, 48)));
}

// The work-group's sums from its lanes' settled ones, in every lane.  lds: 3 * T / 64 floats.
template <int T>
BS_DEV Sums join_lanes(const Sums &mine, float *lds)
{
    float ref = wave_max(mine.any() ? mine.ref : -INFINITY);
    Sums r = mine;
    r.shift(ref);
    r.s = wave_sum(r.s);
    r.t = wave_sum(r.t);
    if constexpr (T > 64) {
        constexpr int W = T / 64;
        const uint32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
        if (lane == 0) {
            lds[wave] = ref;
            lds[W + wave] = r.s;
            lds[2 * W + wave] = r.t;
        }
        __syncthreads();
        // every wave joins the waves' results, one a lane
        Sums part;
        part.against(lane < W ? lds[lane] : -INFINITY);
        part.s = lane < W ? lds[W + lane] : 0.0f;
        part.t = lane < W ? lds[2 * W + lane] : 0.0f;
        ref = wave_max(part.ref);
        part.shift(ref);
        r.s = wave_sum(part.s);
        r.t = wave_sum(part.t);
        __syncthreads();
    }
    r.against(ref);
    return r;
}

// ------------------------------------------------------------------------------------------------ top classes
template <int T>
struct Selection {
    uint64_t lane[T];
    uint64_t list[LIST];
    uint64_t bound;
    uint32_t count, lanes;
    uint16_t chosen[T];
};

// A lower bound of the k-th best class's number: the k-th best of 64 numbers that have a class each, the best of 64 sets of lanes (0: fewer than
// k sets have any).  `key`: the lane's best, 0 for none.  Valid in every lane.
template <int T>
BS_DEV uint64_t bound_of(uint64_t key, uint32_t k, Selection<T> &sel)
{
    sel.lane[threadIdx.x] = key;
    if (threadIdx.x == 0) {
        sel.bound = 0;
        sel.count = sel.lanes = 0;
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        uint64_t best = key;
#pragma unroll
        for (int w = 1; w < T / 64; ++w) {
            const uint64_t other = sel.lane[threadIdx.x + 64 * w];
            best = other > best ? other : best;
        }
        if constexpr (T > 64) sel.list[threadIdx.x] = best;  // (the wave's own: no other wave touches the list before the barrier)
        const uint64_t *from = T > 64 ? sel.list : sel.lane;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        uint32_t rank = 0;
#pragma unroll 16
        for (int i = 0; i < 64; ++i) rank += from[i] > best;
        if (rank == k - 1) sel.bound = best;
    }
    __syncthreads();
    return sel.bound;
}

template <int T>
BS_DEV void offer(uint64_t key, uint64_t bound, Selection<T> &sel)
{
    if (key >= bound && key != 0) {
        const uint32_t at = atomicAdd(&sel.count, 1u);
        if (at < LIST) sel.list[at] = key;
    }
}

// The k best of the offered numbers, best first: put(place, key); places beyond the number offered get 0.  The caller has synchronised.
template <int T, typename PUT>
BS_DEV void put_ranked(uint32_t k, const Selection<T> &sel, PUT put)
{
    const uint32_t n = sel.count;
    for (uint32_t i = threadIdx.x; i < n; i += T) {
        const uint64_t key = sel.list[i];
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t j = 0; j < n; ++j) rank += sel.list[j] > key;
        if (rank < k) put(rank, key);
    }
    for (uint32_t i = n + threadIdx.x; i < k; i += T) put(i, 0);
}

// As long as more than the list holds were offered, the k-th best of those in the list is the bound of the next scan: every scan leaves out
// LIST - k of them or more, and of candidates in any mixed order 15 of 16.  Periodic rows, whose best classes belong to few lanes, come
// here, and masked or equal classes where they are most of a row (400 x 128256 bfloat16, 32 best: 69 us, and 35 of
// other rows).  scan(bound) offers every class again; the caller has synchronised.
template <int T, typename SCAN>
BS_DEV void tighten(uint32_t k, Selection<T> &sel, SCAN scan)
{
    while (sel.count > LIST) {  // (the same in every lane)
        for (uint32_t i = threadIdx.x; i < LIST; i += T) {
            const uint64_t key = sel.list[i];
            uint32_t rank = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < LIST; ++j) rank += sel.list[j] > key;
            if (rank == k - 1) sel.bound = key;
        }
        __syncthreads();
        if (threadIdx.x == 0) sel.count = 0;
        const uint64_t bound = sel.bound;
        __syncthreads();
        scan(bound);
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------ a row's results
// lse = ref + log s for the backward pass, which needs the difference of a logit from it: as one float it would lose of log s what lies below
// the last place of ref, and with it the size of every probability.  A double keeps it: times a power of two from 2^30 on, which leaves it
// below half a unit of the float's last place (log s is at most 21), so that the float in the double is ref.
BS_DEV int raised(float ref) { return max(0, __builtin_amdgcn_frexp_expf(ref) - 31); }
BS_DEV double join_lse(float ref, float log_s) { return (double)ref + ldexp((double)log_s, raised(ref)); }
BS_DEV void split_lse(double lse, float &hi, float &lo)
{
    hi = (float)lse;
    lo = (float)ldexp(lse - (double)hi, -raised(hi));
}

// The row's given class: requested before anything else of the row, used behind everything.
struct Given {
    int64_t c = 0;
    float x = 0.0f;
    template <int DT>
    BS_DEV void request(const LogProbsK &k, uint64_t row, const char *logits)
    {
        if (!k.logp) return;
        c = target_of(k, row);
        if (c >= 0 && c < (int64_t)k.classes) x = element<DT>(logits, (uint64_t)c);
    }
};

BS_DEV void put_row(const LogProbsK &k, uint64_t row, const Given &given, const Sums &r)
{
    const bool none = r.none();
    const float log_s = r.log_s();
    if (k.entropy) k.entropy[row] = none ? 0.0f : r.entropy();
    if (k.lse && k.wide_lse) static_cast<double *>(k.lse)[row] = none ? -INFINITY : join_lse(r.ref, log_s);
    else if (k.lse) static_cast<float *>(k.lse)[row] = none ? -INFINITY : r.ref + log_s;
    if (k.logp) {
        float v;
        if (given.c == k.ignore_index) v = 0.0f;
        else if (given.c < 0 || given.c >= (int64_t)k.classes) v = __builtin_nanf("");
        else v = none ? -INFINITY : (given.x - r.ref) - log_s;
        k.logp[row] = v;
    }
}

struct PutTop {
    const LogProbsK &k;
    uint64_t row;
    float ref, log_s;
    bool none;
    BS_DEV PutTop(const LogProbsK &k_, uint64_t row_, const Sums &r) : k(k_), row(row_), ref(r.ref), log_s(r.log_s()), none(r.none()) {}
    BS_DEV void operator()(uint32_t place, uint64_t key) const
    {
        k.top_index[row * k.top + place] = (int32_t)key_index(key);
        k.top_logp[row * k.top + place] = none ? -INFINITY : (key_value(key) - ref) - log_s;
    }
};

// Sums of elements whose largest is not in the range that Sums::add works on: all of them masked, or all far below zero (rows that hold nothing
// but the value that masks), or some far above it.  The largest first, then differences from it: two passes more (8192 x 32000 bfloat16: 218 us where every
// row is at the lowest value, 147 at -infinity, 95 otherwise; a load at a time 423 and 242).
template <int DT, int T>
BS_DEV Sums far_sums(const char *x, uint32_t n, float *lds)
{
    constexpr uint32_t U = 8;  // loads under way
    Sums mine;
    float most = -INFINITY;
    uint32_t j = threadIdx.x;
    for (; j + (U - 1) * T < n; j += U * T) {
        float v[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) v[u] = element<DT>(x, j + u * T);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) most = max2(most, v[u]);
    }
    for (; j < n; j += T) most = max2(most, element<DT>(x, j));
    most = wave_max(most);
    if constexpr (T > 64) {
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = most;
        __syncthreads();
        for (int w = 0; w < T / 64; ++w) most = max2(most, lds[w]);
        __syncthreads();
    }
    if (most == -INFINITY) return mine;
    auto add = [&](float v) {
        const float d = (v - most) * LOG2E, e = __builtin_amdgcn_exp2f(d);
        mine.s += e;
        mine.t = __builtin_fmaf(e, max2(d, FAR), mine.t);
    };
    for (j = threadIdx.x; j + (U - 1) * T < n; j += U * T) {
        float v[U];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) v[u] = element<DT>(x, j + u * T);
#pragma unroll
        for (uint32_t u = 0; u < U; ++u) add(v[u]);
    }
    for (; j < n; j += T) add(element<DT>(x, j));
    mine.against(most);
    return join_lanes<T>(mine, lds);
}

// One part of one row (or, with PARTS false, the whole row) by a work-group of T threads.  A part begins at any element: the elements in
// front of its first and behind its last whole 128-bit vector are a lane's each.
template <int DT, int T, bool TOP, bool PARTS>
__global__ __launch_bounds__(T) void log_probs_kernel(LogProbsK k)
{
    constexpr int VEC = DT == DT_F32 ? 4 : 8, U = 4;
    constexpr uint64_t ES = DT == DT_F32 ? 4 : 2;
    __shared__ float lds[3 * T / 64];
    quiet_maxima();
    const uint64_t row = PARTS ? blockIdx.x / k.parts : blockIdx.x;
    const uint32_t part = PARTS ? blockIdx.x - (uint32_t)row * k.parts : 0, first = part * k.part;
    const uint32_t n = PARTS ? min(k.classes - first, k.part) : k.classes;
    const char *whole = static_cast<const char *>(k.logits) + row * k.stride * ES;
    const char *x = whole + first * ES;
    const uint32_t head = min(n, (uint32_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (uint32_t)ES);
    const uint32_t vectors = (n - head) / VEC, edges = n - vectors * VEC, tid = threadIdx.x;
    const uint32_t edge = tid < head ? tid : n - (edges - tid);  // the lane's odd element, for tid < edges
    Given given;
    if constexpr (!PARTS) given.request<DT>(k, row, whole);

    Sums sums;
    float best = -INFINITY;
    uint32_t at = tid < head ? tid : tid < vectors ? head + tid * VEC : edge;  // where the lane's first class stands
    const bool any = tid < vectors || tid < edges;
    auto take = [&](const auto &v, float most, uint32_t where) {
        sums.add(v, most);
        if constexpr (TOP) {
            const bool better = most > best;
            best = better ? most : best;
            at = better ? where : at;
        }
    };
    float odd[1] = {0.0f};
    if (tid < edges) odd[0] = element<DT>(x, edge);
    if (tid < head) take(odd, odd[0], tid);
    const char *src = x + head * ES + tid * 16ull;
    uint32_t i = tid;
    auto whole_vector = [&](const Raw<DT, VEC> &raw, uint32_t where) {
        float v[VEC];
        unpack<DT, VEC>(raw, v);
        float most;
        if constexpr (VEC == 4) most = max2(max3(v[0], v[1], v[2]), v[3]);
        else most = max3(max3(v[0], v[1], v[2]), max3(v[3], v[4], v[5]), max2(v[6], v[7]));
        take(v, most, where);
    };
    // batches of U vectors; the next one is under way while one is worked on
    Raw<DT, VEC> raw[U];
    uint32_t batches = vectors / (U * T);
    if (batches) {
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_raw<DT, VEC>(src + u * T * 16, 0);
    }
    for (; batches > 1; --batches, i += U * T) {
        Raw<DT, VEC> next[U];
        src += U * T * 16;
#pragma unroll
        for (int u = 0; u < U; ++u) next[u] = load_raw<DT, VEC>(src + u * T * 16, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) whole_vector(raw[u], head + (i + u * T) * VEC);
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = next[u];
    }
    // the last full batch, and up to U - 1 vectors of a lane behind it
    Raw<DT, VEC> rest[U];
    const uint32_t behind = i + (batches ? U * T : 0);
    src += batches ? U * T * 16 : 0;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (behind + u * T < vectors) rest[u] = load_raw<DT, VEC>(src + u * T * 16, 0);
    if (batches) {
#pragma unroll
        for (int u = 0; u < U; ++u) whole_vector(raw[u], head + (i + u * T) * VEC);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (behind + u * T < vectors) whole_vector(rest[u], head + (behind + u * T) * VEC);
    if (tid >= head && tid < edges) take(odd, odd[0], edge);

    sums.settle();
    Sums r = join_lanes<T>(sums, lds);
    if (r.far()) r = far_sums<DT, T>(x, n, lds);
    if constexpr (PARTS) {
        if (tid == 0) {
            float *out = k.part_sums + 4 * (uint64_t)blockIdx.x;
            out[0] = r.any() ? r.ref : -INFINITY;
            out[1] = r.s;
            out[2] = r.t;
        }
    } else if (tid == 0) {
        put_row(k, row, given, r);
    }
    if constexpr (TOP) {
        __shared__ Selection<T> sel;
        const PutTop top(k, row, r);
        auto put = [&](uint32_t place, uint64_t key) {
            if constexpr (PARTS) k.part_keys[(uint64_t)blockIdx.x * k.top + place] = key;
            else top(place, key);
        };
        uint64_t key = any ? rank_key(best, first + at) : 0;
        if (r.s != r.s) {  // (the same in every lane) NaN, which is above all here and which the comparisons have passed by
            key = tid < edges ? rank_key(odd[0], first + edge) : 0;
            for (uint32_t j = tid; j < vectors; j += T) {
                float v[VEC];
                unpack<DT, VEC>(load_raw<DT, VEC>(x + head * ES + j * 16ull, 0), v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const uint64_t other = rank_key(v[i], first + head + j * VEC + i);
                    key = other > key ? other : key;
                }
            }
        }
        uint64_t bound = bound_of<T>(key, k.top, sel);
        if (bound) bound -= VEC - 1;  // the class is any of its vector
        if (key >= bound && tid < vectors) sel.chosen[atomicAdd(&sel.lanes, 1u)] = (uint16_t)tid;
        __syncthreads();
        // the chosen lanes' vectors once more, one a thread
        const uint32_t each = (vectors + T - 1) / T, again = sel.lanes * each;
        auto scan = [&](uint64_t from) {
            if (tid < edges) offer(rank_key(odd[0], first + edge), from, sel);
            for (uint32_t e = tid; e < again; e += T) {
                const uint32_t c = e / each, j = sel.chosen[c] + (e - c * each) * T;
                if (j >= vectors) continue;
                float v[VEC];
                unpack<DT, VEC>(load_raw<DT, VEC>(x + head * ES + j * 16ull, 0), v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) offer(rank_key(v[i], first + head + j * VEC + i), from, sel);
            }
        };
        scan(bound);
        __syncthreads();
        tighten<T>(k.top, sel, scan);
        put_ranked<T>(k.top, sel, put);
    }
}

// Joins the parts of a row.
template <int DT, bool TOP>
__global__ __launch_bounds__(256) void log_probs_join_kernel(LogProbsK k)
{
    constexpr int T = 256;
    __shared__ float lds[3 * T / 64];
    const uint64_t row = blockIdx.x;
    Given given;
    given.request<DT>(k, row, static_cast<const char *>(k.logits) + row * k.stride * (DT != DT_F32 ? 2 : 4));
    // the best classes of the parts, up to U of a lane at once
    constexpr int U = 4;
    const uint64_t *keys = k.part_keys + row * k.parts * k.top;
    const uint32_t n = k.parts * k.top;
    uint64_t first[U], best = 0;
    if constexpr (TOP) {
#pragma unroll
        for (int u = 0; u < U; ++u) first[u] = threadIdx.x + u * T < n ? keys[threadIdx.x + u * T] : 0;
    }
    Sums mine;
    if (threadIdx.x < k.parts) {  // at most 256
        const float *in = k.part_sums + 4 * (row * k.parts + threadIdx.x);
        mine.against(in[0]);
        mine.s = in[1];
        mine.t = in[2];
    }
    const Sums r = join_lanes<T>(mine, lds);
    if (threadIdx.x == 0) put_row(k, row, given, r);
    if constexpr (TOP) {
        __shared__ Selection<T> sel;
        const PutTop put(k, row, r);
#pragma unroll
        for (int u = 0; u < U; ++u) best = first[u] > best ? first[u] : best;
        for (uint32_t j = threadIdx.x + U * T; j < n; j += T) best = keys[j] > best ? keys[j] : best;
        const uint64_t bound = bound_of<T>(best, k.top, sel);
        auto scan = [&](uint64_t from) {
            if (best < from) return;
#pragma unroll
            for (int u = 0; u < U; ++u) offer(first[u], from, sel);
            for (uint32_t j = threadIdx.x + U * T; j < n; j += T) offer(keys[j], from, sel);
        };
        scan(bound);
        __syncthreads();
        tighten<T>(k.top, sel, scan);
        put_ranked<T>(k.top, sel, put);
    }
}

// ------------------------------------------------------------------------------------------------ gradient
// STREAM: the logits go past the caches.
template <int DT, bool VECTORS, bool STREAM>
__global__ __launch_bounds__(256) void log_probs_backward_kernel(LogProbsK k)
{
    constexpr int T = 256, VEC = DT == DT_F32 ? 4 : 8, U = 4;
    constexpr uint64_t ES = DT == DT_F32 ? 4 : 2;
    quiet_maxima();
    // the last rows first: the forward pass has read them last, and the caches hold them still
    const uint32_t bid = gridDim.x - 1 - blockIdx.x;
    const uint64_t row = bid / k.parts;
    const uint32_t first = (bid - (uint32_t)row * k.parts) * k.part, n = min(k.classes - first, k.part);
    const char *x = static_cast<const char *>(k.logits) + (row * k.stride + first) * ES;
    char *dx = static_cast<char *>(k.grad_logits) + (row * k.grad_stride + first) * ES;
    float lse, low = 0.0f;  // and what a float loses of it
    if (k.wide_lse) split_lse(static_cast<const double *>(k.lse)[row], lse, low);
    else lse = static_cast<const float *>(k.lse)[row];
    const float H = k.entropy ? k.entropy[row] : 0.0f, h = k.grad_entropy ? k.grad_entropy[row] : 0.0f;
    const int64_t c = k.targets ? target_of(k, row) : k.ignore_index;
    float g = k.grad_logp && c != k.ignore_index ? k.grad_logp[row] : 0.0f;
    const bool bad = c != k.ignore_index && (c < 0 || c >= (int64_t)k.classes);
    if (bad) g = __builtin_nanf("");
    const bool none = lse == -INFINITY;
    const uint32_t target = c >= first && c < (int64_t)(first + n) ? (uint32_t)(c - first) : 0xffffffffu;
    // none: -p (0 - 0) of p = 2^-infinity, without a test in the loop; a target that is no class makes NaN there too
    const float gh = none ? (bad ? g : 0.0f) : __builtin_fmaf(h, H, g), hd = none ? 0.0f : h, off = none ? INFINITY : lse;
    low = none ? 0.0f : low;
    // 16-bit results hide the last bits of the exponential; low takes part in its multiply-add
    const float low2 = -low * LOG2E, gh_low = DT == DT_F32 ? gh : __builtin_fmaf(-hd, low, gh);
    auto grad = [&](float v) {
        const float d = DT == DT_F32 ? (v - off) - low : v - off;
        const float p = DT == DT_F32 ? exp_exact(d) : __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E, low2));
        return -p * __builtin_fmaf(hd, max2(d, FAR), gh_low);
    };
    auto one = [&](uint32_t j) {
        float v[1] = {grad(element<DT>(x, j))};
        if (j == target && !none) v[0] += g;
        store_elems<DT, 1>(dx, j, v);
    };
    if constexpr (!VECTORS) {
        for (uint32_t j = threadIdx.x; j < n; j += T) one(j);
        return;
    }
    const uint32_t head = min(n, (uint32_t)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (uint32_t)ES);
    const uint32_t vectors = (n - head) / VEC, edges = n - vectors * VEC, tid = threadIdx.x;
    if (tid < edges) one(tid < head ? tid : n - (edges - tid));
    x += head * ES;
    dx += head * ES;
    auto whole_vector = [&](const Raw<DT, VEC> &raw, uint32_t i) {
        float v[VEC];
        unpack<DT, VEC>(raw, v);
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[e] = grad(v[e]);
        const uint32_t in = target - head - i * VEC;
        if (in < VEC && !none) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) v[e] += e == (int)in ? g : 0.0f;
        }
        store_elems<DT, VEC>(dx + i * 16ull, 0, v);
    };
    uint32_t i = tid;
    for (; i + (U - 1) * T < vectors; i += U * T) {
        Raw<DT, VEC> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load_raw<DT, VEC, STREAM>(x + (i + u * T) * 16ull, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) whole_vector(raw[u], i + u * T);
    }
    for (; i < vectors; i += T) whole_vector(load_raw<DT, VEC>(x + i * 16ull, 0), i);
}

bs_status checked()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

template <int DT, bool TOP>
void launch(const LogProbsK &k, int threads, hipStream_t st)
{
    const dim3 grid((uint32_t)(k.rows * k.parts));
    if (k.parts > 1) {
        log_probs_kernel<DT, 256, TOP, true><<<grid, dim3(256), 0, st>>>(k);
        log_probs_join_kernel<DT, TOP><<<dim3((uint32_t)k.rows), dim3(256), 0, st>>>(k);
    } else if (threads == 64) {
        log_probs_kernel<DT, 64, TOP, false><<<grid, dim3(64), 0, st>>>(k);
    } else {
        log_probs_kernel<DT, 256, TOP, false><<<grid, dim3(256), 0, st>>>(k);
    }
}

template <int DT>
void launch_backward(const LogProbsK &k, bool vectors, hipStream_t st)
{
    const dim3 grid((uint32_t)(k.rows * k.parts)), block(256);
    // logits that the last cache (256 MiB) holds from the forward pass are read through it: 8192x32000 bfloat16 181 us cached, 174 streamed;
    // 1001x10007 float32 15.0 and 17.4
    const bool stream = k.rows * k.classes * (DT == DT_F32 ? 4 : 2) > (256ull << 20);
    if (!vectors) log_probs_backward_kernel<DT, false, false><<<grid, block, 0, st>>>(k);
    else if (stream) log_probs_backward_kernel<DT, true, true><<<grid, block, 0, st>>>(k);
    else log_probs_backward_kernel<DT, true, false><<<grid, block, 0, st>>>(k);
}

}  // namespace

bs_status launch_log_probs(const LogProbsK &k, int32_t dtype, int threads, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) k.top ? launch<DT_F32, true>(k, threads, st) : launch<DT_F32, false>(k, threads, st);
    else if (dtype == BS_BF16) k.top ? launch<DT_BF16, true>(k, threads, st) : launch<DT_BF16, false>(k, threads, st);
    else k.top ? launch<DT_F16, true>(k, threads, st) : launch<DT_F16, false>(k, threads, st);
    return checked();
}

bs_status launch_log_probs_backward(const LogProbsK &k, int32_t dtype, bool vectors, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == BS_F32) launch_backward<DT_F32>(k, vectors, st);
    else if (dtype == BS_BF16) launch_backward<DT_BF16>(k, vectors, st);
    else launch_backward<DT_F16>(k, vectors, st);
    return checked();
}

}  // namespace bs
