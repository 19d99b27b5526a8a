// Loss of a student's logits against a teacher's best words, and its gradient.  Per token, with z = logits / tau,
// q = softmax(z) over the vocabulary and p = softmax(top / tau) over the teacher's words that are in use:
//   loss    = tau^2 w sum_j p_j (log p_j - log q[id_j])
//   grad[i] = scale tau w (q[i] - sum_{j: id_j = i} p_j)
// All of it is in fp32; the sum over the vocabulary is taken relative to the row's largest logit.
#include <cmath>

#include "pdelta_device.h"
#include "pdelta_host.h"

namespace pdelta {

constexpr int kDistillThreads = 1024, kDistillWaves = kDistillThreads / kWave, kDistillMaxWords = 1024;

template <int DT>
__device__ __forceinline__ float load_logit(const void* p, int64_t at)
{
    if constexpr (DT == kF32) return ((const float*)p)[at];
    else return bits_to_f32<DT>(((const uint16_t*)p)[at]);
}
__device__ __forceinline__ float load_logit(int dtype, const void* p, int64_t at)
{
    return dtype == kF32 ? load_logit<kF32>(p, at) : dtype == kBF16 ? load_logit<kBF16>(p, at) : load_logit<kF16>(p, at);
}

// exp(x / tau) for x <= 0: 2^(x hi + x lo) with log2(e) / tau = hi + lo, so that the rounding of that factor, the same for
// the whole vocabulary, does not add up.  hi is below the quotient and lo above 0: with x = -inf both products are -inf.
struct Temperature { float hi, lo, tau; };
__device__ __forceinline__ float exp_tau(float x, Temperature t) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, t.hi, x * t.lo)); }

__device__ __forceinline__ float block_sum(float x, float* red)
{
    x = wave_sum(x);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < kDistillWaves; ++w) sum += red[w];
    return sum;
}
__device__ __forceinline__ float block_max(float x, float* red)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, kWave));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
    float most = red[0];
#pragma unroll
    for (int w = 1; w < kDistillWaves; ++w) most = fmaxf(most, red[w]);
    return most;
}

// One workgroup per token.
template <int DT>
__global__ void __launch_bounds__(kDistillThreads)
distill_kernel(const void* logits, const int* __restrict__ ids, const void* __restrict__ top, int top_dtype,
               const float* __restrict__ weight, float* __restrict__ loss, void* grad, int64_t V, int k, Temperature tau, float grad_scale)
{
    __shared__ float red[kDistillWaves];
    __shared__ int word[kDistillMaxWords];
    __shared__ float share[kDistillMaxWords];
    const int64_t row = blockIdx.x, at = row * V;
    const int tid = threadIdx.x;
    const float w = weight != nullptr ? weight[row] : 1.f;
    if (w == 0.f) {                                   // whole workgroup; the row's logits do not matter
        if (tid == 0) loss[row] = 0.f;
        if (grad != nullptr)
            for (int64_t i = tid; i < V; i += kDistillThreads) store_y<DT>(grad, at + i, 0.f);
        return;
    }
    float most = -INFINITY;
    for (int64_t i = tid; i < V; i += kDistillThreads) most = fmaxf(most, load_logit<DT>(logits, at + i));
    most = block_max(most, red);
    if (most == -INFINITY) most = 0.f;                // nothing may be answered: every term below is 0
    float total = 0.f;
    for (int64_t i = tid; i < V; i += kDistillThreads) total += exp_tau(load_logit<DT>(logits, at + i) - most, tau);
    total = block_sum(total, red);

    // the teacher's words, one thread each
    int id = -1;
    float t = -INFINITY, z = 0.f;
    if (tid < k) {
        id = ids[row * k + tid];
        if (id < 0 || id >= V) id = -1;
        if (id >= 0) {
            t = load_logit(top_dtype, top, row * k + tid);
            z = load_logit<DT>(logits, at + id);
        }
    }
    float best = block_max(t, red);
    const bool some = best != -INFINITY;
    if (!some) best = 0.f;
    const float e = exp_tau(t - best, tau);
    const float mass = block_sum(e, red);
    const float p = some ? e / mass : 0.f;
    const float log_p = (t - best) / tau.tau - logf(mass), log_q = total > 0.f ? (z - most) / tau.tau - logf(total) : -INFINITY;
    const float kl = block_sum(p > 0.f ? p * (log_p - log_q) : 0.f, red);
    if (tid == 0) loss[row] = some ? tau.tau * tau.tau * w * kl : 0.f;
    if (grad == nullptr) return;

    const float factor = grad_scale * tau.tau * w, q_factor = some && total > 0.f ? factor / total : 0.f;
    if (tid < k) {
        word[tid] = p > 0.f ? id : -1;
        share[tid] = p;
    }
    for (int64_t i = tid; i < V; i += kDistillThreads)
        store_y<DT>(grad, at + i, q_factor * exp_tau(load_logit<DT>(logits, at + i) - most, tau));
    __syncthreads();                                  // the words' own entries are written again
    if (p > 0.f) {
        float sum = 0.f;                              // a word that is named more than once gets all its shares, from each of its threads
        for (int j = 0; j < k; ++j) sum += word[j] == id ? share[j] : 0.f;
        store_y<DT>(grad, at + id, q_factor * exp_tau(z - most, tau) - factor * sum);
    }
}

size_t distill_workspace_bytes(int64_t T, int64_t V, int64_t k, int dtype)
{
    (void)T, (void)V, (void)k, (void)dtype;
    return 0;
}

template <int DT>
static int launch_rows(const DistillCall& c, hipStream_t stream)
{
    const double factor = 1.4426950408889634 / (double)c.temperature;
    Temperature tau;
    tau.hi = (float)factor;
    if ((double)tau.hi >= factor) tau.hi = std::nextafterf(tau.hi, 0.f);
    tau.lo = (float)(factor - (double)tau.hi);
    tau.tau = c.temperature;
    hipLaunchKernelGGL(distill_kernel<DT>, dim3((unsigned)c.T), dim3(kDistillThreads), 0, stream, c.logits, c.ids, c.top, c.top_dtype,
                       c.weight, c.loss, c.grad, c.V, (int)c.k, tau, c.grad_scale);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_distill(const DistillCall& c, hipStream_t stream)
{
    if (c.dtype == kF32) return launch_rows<kF32>(c, stream);
    if (c.dtype == kBF16) return launch_rows<kBF16>(c, stream);
    return launch_rows<kF16>(c, stream);
}

}  // namespace pdelta
