// Loss of a student's logits against a teacher's best words, and its gradient.  Per token, with z = logits / tau,
// q = softmax(z) over the vocabulary and p = softmax(top / tau) over the teacher's words that are in use:
//   loss    = tau^2 w sum_j p_j (log p_j - log q[id_j])
//   grad[i] = scale tau w (q[i] - sum_{j: id_j = i} p_j)
// All of it is in fp32; sums over the vocabulary are taken relative to the largest logit.
//
// Bound by memory: logits once in, gradient once out (2048 x 128256 bf16, three tenths of the tokens without weight, 195 to 210 us: 0.38 GB
// read and 0.53 written, 4.3 to 4.7 TB/s; an elementwise copy of 1 GiB reaches 6.2.  The loss alone of 640 x 32000 fp16 in 13 us: the launch, and
// 2.5 rows for each CU).  A workgroup keeps its part of the row in registers, as the 16-byte vectors it was loaded as, between the sum over the
// vocabulary and the gradient; what does not fit is read again.  Every wave sums relative to the largest logit of its own, and the
// waves meet once; the first wave deals with the teacher's words meanwhile.  The gradient is written as if the teacher had named no
// word, and the words' own entries again after a barrier.
//
// Of few tokens, a long row is split among workgroups: one launch leaves the largest logit and the sum of every part (and the
// words' logits, since the gradient may replace the logits) in the workspace, a second one joins them in their order.
#include <algorithm>
#include <cmath>

#include "pdelta_device.h"
#include "pdelta_host.h"

namespace pdelta {

constexpr int kDistillMaxWords = 1024;
constexpr float kNothing = -INFINITY;
constexpr float kNear = 8.f;                          // RowPart::wave_sum_of

// exp(x / tau) is 2^(x hi + x lo) with log2(e) / tau = hi + lo; hi is below the quotient and lo above 0, so that with x = -inf
// both products are -inf.  16-bit logits are taken with `near`, the quotient itself in fp32: the rounding of that factor, 2^-25
// of an exponent, is the same for the whole vocabulary, but far below what the logits' own type leaves.
struct Temperature { float hi, lo, near, tau; };
__device__ __forceinline__ float exp_tau(float x, Temperature t) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, t.hi, x * t.lo)); }
// exp((z - most) / tau), exactly 1 for the largest logit itself.
template <int DT>
__device__ __forceinline__ float exp_logit(float z, float most, Temperature t)
{
    if constexpr (DT == kF32) return exp_tau(z - most, t);
    else return __builtin_amdgcn_exp2f((z - most) * t.near);
}

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

// Element e of the 16 bytes of a vector.
template <int DT>
__device__ __forceinline__ float element(uint4v a, int e)
{
    if constexpr (DT == kF32) {
        const uint32_t u = a[e];
        return __builtin_bit_cast(float, u);
    } else {
        const uint32_t u = a[e >> 1];
        if constexpr (DT == kBF16) return __builtin_bit_cast(float, e & 1 ? u & 0xFFFF0000u : u << 16);
        else return (float)as_half2(u)[e & 1];
    }
}
template <int DT>
__device__ __forceinline__ uint32_t pack_pair(float a, float b)
{
    if constexpr (DT == kBF16) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        typedef float float2v __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((float2v){a, b}, bf16x2));     // one instruction, to nearest even
    } else {
        return f32_to_f16_bits(a) | f32_to_f16_bits(b) << 16;
    }
}
// One entry, with the conversion of the vectors: a NaN of any pattern stays one.
template <int DT>
__device__ __forceinline__ void store_entry(void* p, int64_t at, float x)
{
    if constexpr (DT == kF32) ((float*)p)[at] = x;
    else ((uint16_t*)p)[at] = (uint16_t)pack_pair<DT>(x, 0.f);
}
// The largest of three; none of them is a NaN that signals.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, kWave));
    return x;
}

// The largest logit and the sum of exponentials relative to it; (-inf, 0) is nothing.  A logit that is NaN or +inf makes the sum NaN, which
// no joining takes out again, and with it the loss and the row of the gradient.
struct Sum { float most, total; };
__device__ __forceinline__ Sum join(Sum a, Sum b, Temperature t)
{
    const float most = fmaxf(a.most, b.most);
    if (most == kNothing) return {kNothing, a.total + b.total};       // 0, or not a number
    return {most, a.total * exp_tau(a.most - most, t) + b.total * exp_tau(b.most - most, t)};
}

// The words [begin, end) of one row: those before the first 16-byte boundary and behind the last one, at most 2 (PER - 1), are one
// per thread; the vectors between them go round the threads, the first NV rounds stay in registers.
template <int DT, int THREADS, int NV>
struct RowPart {
    static constexpr int PER = DT == kF32 ? 4 : 8;
    const char* src;                                  // the row
    char* dst;
    int64_t first, vectors, edge;                     // first vector's word; number of vectors; this thread's edge word or -1
    uint4v held[NV > 0 ? NV : 1];
    float edge_z;

    __device__ __forceinline__ void load(const void* logits, void* grad, int64_t row, int64_t V, int64_t begin, int64_t end)
    {
        constexpr int SIZE = DT == kF32 ? 4 : 2;
        src = (const char*)logits + row * V * SIZE;
        dst = (char*)grad + row * V * SIZE;
        const int64_t head = min((int64_t)((16 - ((uintptr_t)(src + begin * SIZE) & 15)) & 15) / SIZE, end - begin);
        first = begin + head;
        vectors = (end - first) / PER;
        const int64_t behind = first + vectors * PER;
        const int tid = threadIdx.x;
        edge = tid < head ? begin + tid : tid >= 8 && behind + tid - 8 < end ? behind + tid - 8 : -1;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            constexpr uint32_t nothing = DT == kF32 ? 0xFF800000u : DT == kBF16 ? 0xFF80FF80u : 0xFC00FC00u;       // -inf
            held[i] = (uint4v){nothing, nothing, nothing, nothing};
            if ((int64_t)i * THREADS + tid < vectors) held[i] = vector(i);
        }
        edge_z = edge >= 0 ? load_logit<DT>(src, edge) : kNothing;
    }
    // A vector that stays a vector until it is used: otherwise the row is kept in registers a second time, as single words.
    __device__ __forceinline__ uint4v kept(int i) const
    {
        uint4v a = held[i];
        asm volatile("" : "+v"(a));
        return a;
    }
    __device__ __forceinline__ int64_t place(int64_t i) const { return (first + (i * THREADS + threadIdx.x) * PER) * (DT == kF32 ? 4 : 2); }
    __device__ __forceinline__ uint4v vector(int64_t i) const { return *(const uint4v*)(src + place(i)); }

    // The wave's largest logit, and the sum relative to it (every lane has both).  The sum is taken while the vectors arrive, relative to the
    // largest of the first ones; the same pass finds the largest of all, and one factor brings the sum to it.  Where that is more than
    // kNear powers of two above (a word that stands out), or the first ones are all masked, the sum is taken again relative to it:
    // a logit far above makes the arguments of the exponentials large, and their rounding is most of what is left of 1 - q and log q.
    // us with the largest first, in a pass of its own, and so: 1024 x 128256 fp32 272, 242, x 152064 bf16 151, 144; 2048 x 10000 fp16 23.5, 22.1.
    __device__ __forceinline__ Sum wave_sum_of(Temperature t) const
    {
        auto larger = [&](float most, uint4v a) {
#pragma unroll
            for (int e = 0; e < PER; e += 2) most = max3(most, element<DT>(a, e), element<DT>(a, e + 1));
            return most;
        };
        auto sum = [&](float base, auto each) {
            float a0 = 0.f, a1 = 0.f;
            auto add = [&](uint4v a) {
#pragma unroll
                for (int e = 0; e < PER; e += 2) {
                    const float x = element<DT>(a, e), y = element<DT>(a, e + 1);
                    each(x, y);
                    a0 += exp_logit<DT>(x, base, t);
                    a1 += exp_logit<DT>(y, base, t);
                    __builtin_amdgcn_sched_barrier(0);             // (else 6 registers more, and fewer waves on a CU: 2048 x 70001 bf16 145 us, 124)
                }
            };
#pragma unroll
            for (int i = 0; i < NV; ++i) add(kept(i));
            for (int64_t i = NV; i * THREADS + threadIdx.x < vectors; ++i) add(vector(i));
            a0 += exp_logit<DT>(edge_z, base, t);
            return wave_sum(a0 + a1);
        };
        const float near_most = wave_max(larger(kNothing, kept(0)));
        float most = edge_z;
        if (near_most != kNothing) {
            const float total = sum(near_most, [&](float x, float y) { most = max3(most, x, y); });
            most = wave_max(most);
            if ((most - near_most) * t.near <= kNear) return {most, total * exp_logit<DT>(near_most, most, t)};       // all lanes alike
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i) most = larger(most, kept(i));
            for (int64_t i = NV; i * THREADS + threadIdx.x < vectors; ++i) most = larger(most, vector(i));
            most = wave_max(most);
        }
        return {most, sum(most == kNothing ? 0.f : most, [](float, float) {})};
    }

    // grad = factor exp((z - most) / tau), or zeros
    template <bool ZERO>
    __device__ __forceinline__ void store(float factor, float most, Temperature t) const
    {
        auto value = [&](float z) { return ZERO ? 0.f : factor * exp_logit<DT>(z, most, t); };
        auto put = [&](int64_t i, uint4v a) {
            uint4v r;
            if constexpr (DT == kF32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = __builtin_bit_cast(uint32_t, value(element<DT>(a, e)));
            } else {
#pragma unroll
                for (int p = 0; p < 4; ++p) r[p] = pack_pair<DT>(value(element<DT>(a, 2 * p)), value(element<DT>(a, 2 * p + 1)));
            }
            // (not to be kept in the caches: us otherwise and so, 2048 x 128256 bf16 235, 227, x 70001 141, 125, 1024 x 128256 fp32 269, 248)
            __builtin_nontemporal_store(r, (uint4v*)(dst + place(i)));
        };
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((int64_t)i * THREADS + threadIdx.x < vectors) put(i, kept(i));
        for (int64_t i = NV; i * THREADS + threadIdx.x < vectors; ++i) put(i, ZERO ? (uint4v){0, 0, 0, 0} : vector(i));
        if (edge >= 0) store_entry<DT>(dst, edge, value(edge_z));
    }
};

struct DistillArgs {
    const void* logits;
    const int* ids;
    const void* top;
    const float* weight;
    float* loss;
    void* grad;
    int64_t V;
    int k, top_dtype;
    Temperature tau;
    float grad_scale;
    Sum* sums;                                        // split rows: [T][parts]
    float* words_z;                                   // and [T][k] logits of the teacher's words
    int parts;
};

// The teacher's words of a row, by its first wave; all in LDS.
struct Words {
    int id[kDistillMaxWords];                         // -1: no share
    float share[kDistillMaxWords], gap[kDistillMaxWords];         // p, and log p - z / tau
    float wave_most[16], wave_total[16], z[kDistillMaxWords];
    int some;                                         // a slot is in use
};

// p_j of the row's words in LDS; z_of(j, id): the student's logit of word j.  A NaN or +inf among the teacher's logits makes all of its
// shares NaN, and with them the loss and the gradient's entries of the words.
template <typename Z>
__device__ __forceinline__ void teacher(const DistillArgs& g, int64_t row, Words& words, Z z_of)
{
    const int lane = threadIdx.x & 63;
    float best = kNothing;
    bool mine = false;
    for (int j = lane; j < g.k; j += kWave) {
        int id = g.ids[row * g.k + j];
        float t = kNothing, z = 0.f;
        if (id >= 0 && id < g.V) {
            t = load_logit(g.top_dtype, g.top, row * g.k + j);
            z = z_of(j, id);
        }
        words.id[j] = t == kNothing ? -1 : id;
        words.share[j] = t;
        words.z[j] = z;
        best = fmaxf(best, t);
        mine = mine || t != kNothing;
    }
    best = wave_max(best);
    const bool some = __ballot(mine) != 0;
    float mass = 0.f;
    for (int j = lane; j < g.k; j += kWave) mass += words.id[j] >= 0 ? exp_tau(words.share[j] - best, g.tau) : 0.f;
    mass = wave_sum(mass);
    const float log_mass = logf(mass);
    for (int j = lane; j < g.k; j += kWave) {
        const float t = words.share[j], p = words.id[j] >= 0 ? exp_tau(t - best, g.tau) / mass : 0.f;
        words.share[j] = p;
        if (p == 0.f) words.id[j] = -1;               // (a share that is not a number keeps its word)
        words.gap[j] = (t - best) / g.tau.tau - log_mass;
    }
    if (lane == 0) words.some = some;
}

// The first wave: loss of the row from its words and the student's sum.
__device__ __forceinline__ void write_loss(const DistillArgs& g, int64_t row, const Words& words, Sum all, float w)
{
    const int lane = threadIdx.x & 63;
    const float log_total = all.total == 0.f ? 0.f : logf(all.total);
    float kl = 0.f;
    for (int j = lane; j < g.k; j += kWave)
        if (words.id[j] >= 0) {
            const float log_q = all.total == 0.f ? kNothing : (words.z[j] - all.most) / g.tau.tau - log_total;
            kl += words.share[j] * (words.gap[j] - log_q);
        }
    kl = wave_sum(kl);
    if (lane == 0) g.loss[row] = words.some ? g.tau.tau * g.tau.tau * w * kl : 0.f;
}

// The entries of the words in [begin, end): a word that is named more than once gets all its shares, from each of its threads.
template <int DT>
__device__ __forceinline__ void store_words(const DistillArgs& g, int64_t row, const Words& words, float q_factor, float factor, float most,
                                            int64_t begin, int64_t end)
{
    for (int j = threadIdx.x; j < g.k; j += blockDim.x) {
        const int id = words.id[j];
        if (id < begin || id >= end) continue;
        float sum = 0.f;
        for (int i = 0; i < g.k; ++i) sum += words.id[i] == id ? words.share[i] : 0.f;
        const float q = q_factor * exp_logit<DT>(words.z[j], most, g.tau);
        store_entry<DT>(g.grad, row * g.V + id, q - factor * sum);
    }
}

// One workgroup per token.
template <int DT, int THREADS, int NV>
__global__ void __launch_bounds__(THREADS)
distill_kernel(DistillArgs g)
{
    __shared__ Words words;
    const int64_t row = blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const float w = g.weight != nullptr ? g.weight[row] : 1.f;
    RowPart<DT, THREADS, NV> part;
    if (w == 0.f) {                                   // whole workgroup; the row's logits do not matter
        if (threadIdx.x == 0) g.loss[row] = 0.f;
        if (g.grad != nullptr) {
            RowPart<DT, THREADS, 0> none;
            none.load(g.logits, g.grad, row, g.V, 0, g.V);
            none.template store<true>(0.f, 0.f, g.tau);
        }
        return;
    }
    part.load(g.logits, g.grad, row, g.V, 0, g.V);
    if (wave == 0) teacher(g, row, words, [&](int, int id) { return load_logit<DT>(part.src, id); });
    const Sum mine = part.wave_sum_of(g.tau);
    if ((threadIdx.x & 63) == 0) {
        words.wave_most[wave] = mine.most;
        words.wave_total[wave] = mine.total;
    }
    __syncthreads();
    Sum all{kNothing, 0.f};
#pragma unroll
    for (int k = 0; k < THREADS / kWave; ++k) all = join(all, {words.wave_most[k], words.wave_total[k]}, g.tau);
    if (all.most == kNothing) all.most = 0.f;         // nothing may be answered: every q is 0
    if (wave == 0) write_loss(g, row, words, all, w);
    if (g.grad == nullptr) return;
    if (!words.some) {                                // whole workgroup; the row's logits do not matter here either
        part.template store<true>(0.f, 0.f, g.tau);
        return;
    }
    const float factor = g.grad_scale * g.tau.tau * w, q_factor = all.total != 0.f ? factor / all.total : 0.f;
    part.template store<false>(q_factor, all.most, g.tau);
    __syncthreads();
    store_words<DT>(g, row, words, q_factor, factor, all.most, 0, g.V);
}

constexpr int kPartVectors = 8;                       // of a thread: 32 KB for a workgroup

// Words of part `part` of a row that is split into g.parts: multiples of 64 words.
__device__ __forceinline__ void part_of(const DistillArgs& g, int part, int64_t& begin, int64_t& end)
{
    const int64_t units = (g.V + 63) / 64;
    begin = units * part / g.parts * 64;
    end = min(units * (part + 1) / g.parts * 64, g.V);
}

// Split rows: largest logit and sum of one part, and the logits of the teacher's words in it.
template <int DT>
__global__ void __launch_bounds__(256)
distill_part_kernel(DistillArgs g)
{
    __shared__ float most[4], total[4];
    const int64_t row = blockIdx.x / g.parts;
    const int part = blockIdx.x % g.parts, wave = threadIdx.x >> 6;
    int64_t begin, end;
    part_of(g, part, begin, end);
    if (g.weight != nullptr && g.weight[row] == 0.f) return;      // whole workgroup
    RowPart<DT, 256, kPartVectors> p;
    p.load(g.logits, nullptr, row, g.V, begin, end);
    for (int j = threadIdx.x; j < g.k; j += 256) {
        const int id = g.ids[row * g.k + j];
        if (id >= begin && id < end) g.words_z[row * g.k + j] = load_logit<DT>(p.src, id);
    }
    const Sum mine = p.wave_sum_of(g.tau);
    if ((threadIdx.x & 63) == 0) {
        most[wave] = mine.most;
        total[wave] = mine.total;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        Sum all{kNothing, 0.f};
        for (int k = 0; k < 4; ++k) all = join(all, {most[k], total[k]}, g.tau);
        g.sums[row * g.parts + part] = all;
    }
}

// Split rows: the parts' sums together; the loss (from the first part's workgroup) and the part's gradient.
template <int DT>
__global__ void __launch_bounds__(256)
distill_join_kernel(DistillArgs g, int groups)
{
    __shared__ Words words;
    const int64_t row = blockIdx.x / groups;
    const int part = blockIdx.x % groups, wave = threadIdx.x >> 6;
    int64_t begin, end;
    part_of(g, part, begin, end);
    const float w = g.weight != nullptr ? g.weight[row] : 1.f;
    if (w == 0.f) {                                   // whole workgroup
        if (part == 0 && threadIdx.x == 0) g.loss[row] = 0.f;
        if (g.grad != nullptr) {
            RowPart<DT, 256, 0> none;
            none.load(g.logits, g.grad, row, g.V, begin, end);
            none.template store<true>(0.f, 0.f, g.tau);
        }
        return;
    }
    RowPart<DT, 256, kPartVectors> p;
    if (g.grad != nullptr) p.load(g.logits, g.grad, row, g.V, begin, end);
    Sum all{kNothing, 0.f};
    for (int k = 0; k < g.parts; ++k) all = join(all, g.sums[row * g.parts + k], g.tau);
    if (all.most == kNothing) all.most = 0.f;
    if (wave == 0) {
        teacher(g, row, words, [&](int j, int) { return g.words_z[row * g.k + j]; });
        if (part == 0) write_loss(g, row, words, all, w);
    }
    if (g.grad == nullptr) return;
    __syncthreads();
    if (!words.some) {                                // whole workgroup
        p.template store<true>(0.f, 0.f, g.tau);
        return;
    }
    const float factor = g.grad_scale * g.tau.tau * w, q_factor = all.total != 0.f ? factor / all.total : 0.f;
    p.template store<false>(q_factor, all.most, g.tau);
    __syncthreads();
    store_words<DT>(g, row, words, q_factor, factor, all.most, begin, end);
}

// Parts of a row: of few tokens, rows of more than 128 KB are split into parts of 32 KB.  us of a call in one part, 4, 8 and 16: 1 x 128256
// bf16 21.7, 18.1, 15.2 and 15.1, 64 tokens 22.4, 21.7, 17.9 and 21.0, 150 tokens 24.8, 30.6, 28.1 and 35.9; 16 x 128256 fp32 26.5, 27.8, 18.8
// and 15.8; but 3 x 32001 fp32 (125 KB) 9.2, 13.9, 14.3 and 14.1.
static int row_parts(int64_t T, int64_t V, int dtype)
{
    const int64_t bytes = V * (dtype == kF32 ? 4 : 2);
    return T > 128 || bytes <= 128 * 1024 ? 1 : (int)std::min<int64_t>(32, bytes / (32 * 1024));
}

size_t distill_workspace_bytes(int64_t T, int64_t V, int64_t k, int dtype)
{
    if (T == 0) return 0;
    const int parts = row_parts(T, V, dtype);
    return parts == 1 ? 0 : (size_t)T * ((size_t)parts * sizeof(Sum) + (size_t)k * 4);
}

template <int DT>
static int launch_rows(const DistillCall& c, hipStream_t stream)
{
    constexpr int PER = DT == kF32 ? 4 : 8;
    const double factor = 1.4426950408889634 / (double)c.temperature;
    Temperature tau;
    tau.near = (float)factor;
    tau.hi = (double)tau.near >= factor ? std::nextafterf(tau.near, 0.f) : tau.near;
    tau.lo = (float)(factor - (double)tau.hi);
    tau.tau = c.temperature;
    DistillArgs g{c.logits, c.ids, c.top, c.weight, c.loss, c.grad, c.V, (int)c.k, c.top_dtype, tau, c.grad_scale, nullptr, nullptr, 1};
    g.parts = row_parts(c.T, c.V, c.dtype);
    if (g.parts > 1) {
        g.sums = (Sum*)c.workspace;
        g.words_z = (float*)(g.sums + c.T * g.parts);
        const int groups = c.grad != nullptr ? g.parts : 1;
        hipLaunchKernelGGL(distill_part_kernel<DT>, dim3((unsigned)(c.T * g.parts)), dim3(256), 0, stream, g);
        hipLaunchKernelGGL(distill_join_kernel<DT>, dim3((unsigned)(c.T * groups)), dim3(256), 0, stream, g, groups);
    } else {
        // Threads and the 16-byte vectors that each keeps in registers.  Eight let twice as many waves run on a CU as sixteen, for which the
        // rest of a row that is too long is read again.  us with sixteen and eight, 16-bit: 8192 x 10000 94, 69, the loss
        // alone 65, 43; 2048 x 82000 173, 149, x 100000 207, 187, x 120000 223, 215, x 128256 227, 230; the loss alone of 70000 100, 56.  fp32:
        // 2048 x 46000 161, 163, x 57000 206, 216, the loss alone 94, 80 and 107, 98.  8192 x 32000 in 512 threads of eight 205, in 256 of sixteen
        // 208.  The loss alone takes what the gradient would: its bits are the same.
        const int64_t vectors = c.V / PER;
#define PDELTA_GO(THREADS, NV) hipLaunchKernelGGL((distill_kernel<DT, THREADS, NV>), dim3((unsigned)c.T), dim3(THREADS), 0, stream, g)
        if (vectors <= 256) PDELTA_GO(256, 1);
        else if (vectors <= 4 * 256) PDELTA_GO(256, 4);
        else if (vectors <= 8 * 256) PDELTA_GO(256, 8);
        else if (vectors <= 16 * 256) PDELTA_GO(256, 16);
        else if (vectors <= (DT == kF32 ? 12 : 15) * 1024) PDELTA_GO(1024, 8);
        else PDELTA_GO(1024, 16);
#undef PDELTA_GO
    }
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_distill(const DistillCall& c, hipStream_t stream)
{
    if (c.dtype == kF32) return launch_rows<kF32>(c, stream);
    if (c.dtype == kBF16) return launch_rows<kBF16>(c, stream);
    return launch_rows<kF16>(c, stream);
}

}  // namespace pdelta
