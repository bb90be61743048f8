// Log probabilities of given classes, the entropy of every row's distribution and its top alternatives; and their gradient.
//
//   m = max x,  s = sum exp(x - m),  t = sum exp(x - m) (x - m);   lse = m + log s,  logp = x[target] - lse,  entropy = log s - t / s
//   dx_j = g (delta_j,target - p_j) - h p_j (log p_j + entropy),   p = exp(x - lse), g and h the gradients of logp and of entropy
//
// Maximum and sums are kept running in float32 over one pass; a class at -infinity has probability 0 and adds nothing.
#include <hip/hip_runtime.h>

#include "bs_device.h"
#include "bs_internal.h"
#include "bs_log_probs.h"

namespace bs {
namespace {

constexpr int T = 256;

// exp for float32 results: the product with log2(e) in two parts, so that large arguments keep their last bits.
BS_DEV float exp_exact(float v)
{
    const float hi = v * 1.44269504088896341f;
    const float lo = __builtin_fmaf(v, 1.44269504088896341f, -hi) + v * 1.92596299112661746e-8f;
    const float e = __builtin_amdgcn_exp2f(hi);
    return __builtin_fabsf(hi) < 160.0f ? __builtin_fmaf(e, lo * 0.693147180559945309f, e) : e;  // (beyond: 0, infinity or NaN)
}

// Running maximum, sum of exp(x - m) and sum of exp(x - m) (x - m).
struct Running {
    float m = -INFINITY, s = 0.0f, t = 0.0f;

    BS_DEV void join(float mo, float so, float to)
    {
        const float mn = __builtin_fmaxf(m, mo);
        const float base = mn == -INFINITY ? 0.0f : mn;
        const float da = m - base, db = mo - base;  // (-infinity where that side is empty: its sums are 0, or NaN)
        const float fa = exp_exact(da), fb = exp_exact(db);
        t = fa * __builtin_fmaf(s, __builtin_fmaxf(da, -1e30f), t) + fb * __builtin_fmaf(so, __builtin_fmaxf(db, -1e30f), to);
        s = __builtin_fmaf(s, fa, so * fb);
        m = mn;
    }
    BS_DEV void add(float x)
    {
        const float one = x == -INFINITY ? 0.0f : 1.0f;
        join(x, x != x ? x : one, 0.0f);
    }
};

template <int DT>
BS_DEV float element(const void *p, uint64_t i)
{
    if constexpr (DT == DT_F32) return static_cast<const float *>(p)[i];
    else return half_up<DT>(static_cast<const uint16_t *>(p)[i]);
}

// A class as one number: larger values first, then lower indices; NaN above all, -0 equal to 0.  Never 0 for a class.
BS_DEV uint64_t rank_key(float x, uint32_t j)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    const uint32_t o = x != x ? 0xffffffffu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return (uint64_t)o << 32 | (0xffffffffu - j);
}

BS_DEV int64_t target_of(const LogProbsK &k, uint64_t row)
{
    return k.wide_targets ? static_cast<const int64_t *>(k.targets)[row] : static_cast<const int32_t *>(k.targets)[row];
}

template <int DT>
__global__ __launch_bounds__(T) void log_probs_kernel(LogProbsK k)
{
    __shared__ float part[3][T / 64];
    __shared__ uint64_t best[T / 64];
    const uint64_t row = blockIdx.x;
    const char *x = static_cast<const char *>(k.logits) + row * k.stride * (DT != DT_F32 ? 2 : 4);
    Running r;
    for (uint32_t j = threadIdx.x; j < k.classes; j += T) r.add(element<DT>(x, j));
#pragma unroll
    for (int o = 32; o; o >>= 1) r.join(__shfl_xor(r.m, o), __shfl_xor(r.s, o), __shfl_xor(r.t, o));
    const uint32_t wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) {
        part[0][wave] = r.m;
        part[1][wave] = r.s;
        part[2][wave] = r.t;
    }
    __syncthreads();
    r = Running();
    for (uint32_t w = 0; w < T / 64; ++w) r.join(part[0][w], part[1][w], part[2][w]);
    const bool none = r.s == 0.0f;  // every class masked
    const float lse = none ? -INFINITY : r.m + logf(r.s);
    if (threadIdx.x == 0) {
        if (k.entropy) k.entropy[row] = none ? 0.0f : logf(r.s) - r.t / r.s;
        if (k.lse) k.lse[row] = lse;
        if (k.targets && k.logp) {
            const int64_t c = target_of(k, row);
            float v;
            if (c == k.ignore_index) v = 0.0f;
            else if (c < 0 || c >= (int64_t)k.classes) v = __builtin_nanf("");
            else v = none ? -INFINITY : (element<DT>(x, (uint64_t)c) - r.m) - logf(r.s);
            k.logp[row] = v;
        }
    }
    uint64_t last = ~0ull;
    for (uint32_t i = 0; i < k.top; ++i) {
        uint64_t mine = 0;
        for (uint32_t j = threadIdx.x; j < k.classes; j += T) {
            const uint64_t key = rank_key(element<DT>(x, j), j);
            if (key < last && key > mine) mine = key;
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const uint64_t other = __shfl_xor(mine, o);
            mine = other > mine ? other : mine;
        }
        __syncthreads();
        if (threadIdx.x % 64 == 0) best[wave] = mine;
        __syncthreads();
        last = best[0];
        for (uint32_t w = 1; w < T / 64; ++w) last = best[w] > last ? best[w] : last;
        if (threadIdx.x == 0) {
            const uint32_t j = 0xffffffffu - (uint32_t)last;
            k.top_index[row * k.top + i] = (int32_t)j;
            k.top_logp[row * k.top + i] = none ? -INFINITY : (element<DT>(x, j) - r.m) - logf(r.s);
        }
    }
}

template <int DT>
__global__ __launch_bounds__(T) void log_probs_backward_kernel(LogProbsK k)
{
    const uint64_t row = blockIdx.x;
    const char *x = static_cast<const char *>(k.logits) + row * k.stride * (DT != DT_F32 ? 2 : 4);
    char *dx = static_cast<char *>(k.grad_logits) + row * k.grad_stride * (DT != DT_F32 ? 2 : 4);
    const float lse = k.lse[row], H = k.entropy ? k.entropy[row] : 0.0f, h = k.grad_entropy ? k.grad_entropy[row] : 0.0f;
    const int64_t c = k.targets ? target_of(k, row) : k.ignore_index;
    float g = k.grad_logp && c != k.ignore_index ? k.grad_logp[row] : 0.0f;
    if (c != k.ignore_index && (c < 0 || c >= (int64_t)k.classes)) g = __builtin_nanf("");
    const bool none = lse == -INFINITY;
    for (uint32_t j = threadIdx.x; j < k.classes; j += T) {
        const float d = element<DT>(x, j) - lse, p = exp_exact(d);
        float v = -g * p - (p != 0.0f ? h * p * (d + H) : 0.0f);
        if ((int64_t)j == c) v += g;
        if (none) v = 0.0f;
        if constexpr (DT == DT_F32) reinterpret_cast<float *>(dx)[j] = v;
        else reinterpret_cast<uint16_t *>(dx)[j] = half_bits<DT>(v);
    }
}

bs_status checked()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BS_OK;
    set_hip_error((int32_t)e);
    return BS_ERR_HIP;
}

}  // namespace

bs_status launch_log_probs(const LogProbsK &k, int32_t dtype, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((uint32_t)k.rows), block(T);
    if (dtype == BS_F32) log_probs_kernel<DT_F32><<<grid, block, 0, st>>>(k);
    else if (dtype == BS_BF16) log_probs_kernel<DT_BF16><<<grid, block, 0, st>>>(k);
    else log_probs_kernel<DT_F16><<<grid, block, 0, st>>>(k);
    return checked();
}

bs_status launch_log_probs_backward(const LogProbsK &k, int32_t dtype, void *stream)
{
    hipStream_t st = static_cast<hipStream_t>(stream);
    const dim3 grid((uint32_t)k.rows), block(T);
    if (dtype == BS_F32) log_probs_backward_kernel<DT_F32><<<grid, block, 0, st>>>(k);
    else if (dtype == BS_BF16) log_probs_backward_kernel<DT_BF16><<<grid, block, 0, st>>>(k);
    else log_probs_backward_kernel<DT_F16><<<grid, block, 0, st>>>(k);
    return checked();
}

}  // namespace bs
