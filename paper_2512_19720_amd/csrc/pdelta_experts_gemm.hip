// Products of tokens sorted by expert with every expert's W_hat = W_b + v (.) B, never written to memory:
//   forward   Y[m, o]  = sum_i X[m, i]  W_hat_e[o, i]
//   backward  dX[m, i] = sum_o dY[m, o] W_hat_e[o, i]
// for the tokens m of every expert e.  The arithmetic is that of the prefill kernels: the tile of W_hat is formed as
// fp16(W_b +- v) with one rounding, fp32 sums.  (That rounding weighs as much as the one of fp16 outputs: 2.9e-4 from the exact products
// in norm, 2.1e-4 without it; of bf16 outputs 1.67e-3 and 1.66e-3.  W_b and v (.) B as two operands would do without it, for twice the
// matrix instructions.)  This file prepares the operands; the tiles are in pdelta_experts_gemm_dma.hip, and
// those of experts with few tokens in pdelta_experts_skinny.hip.
//
// The token operand is always multiplied as fp16.  A bf16 one is converted first, by experts_prepare_kernel, every row
// times the power of two that brings its largest element to [2^14, 2^15): gradients are often far below fp16's range,
// and differ in size from token to token.  The conversion is exact for elements within 2^28 of their row's largest and
// off by at most 2^-39 of the largest for the others; the outputs are multiplied by the inverse power in fp32, exactly.
// The same kernel copies fp16 rows that are no multiple of 128 values into rows that are, zeros behind them.
#include "pdelta_experts.h"
#include "pdelta_host.h"

namespace pdelta {

// One workgroup per row.  Reads the row twice (the second time out of the cache), writes it once.
template <int DT>
__global__ void __launch_bounds__(256)
experts_prepare_kernel(const uint16_t* __restrict__ A, uint16_t* __restrict__ out, float* __restrict__ inverse, int K, int lda)
{
    __shared__ uint32_t most[4];
    const int64_t row = blockIdx.x;
    const uint16_t* src = A + row * K;
    uint16_t* dst = out + row * lda;
    const bool wide = (K & 7) == 0;                   // every row starts at a multiple of 16 bytes
    float scale = 1.f;
    if constexpr (DT == kBF16) {
        uint32_t big = 0;                             // largest magnitude, as bits
        if (wide) {
            for (int c = threadIdx.x; c < K / 8; c += 256) {
                const uint4v a = *(const uint4v*)(src + c * 8);
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const uint32_t d = a[p];
                    big = max(big, max(d & 0x7FFFu, (d >> 16) & 0x7FFFu));
                }
            }
        } else {
            for (int c = threadIdx.x; c < K; c += 256) big = max(big, src[c] & 0x7FFFu);
        }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) big = max(big, (uint32_t)__shfl_xor((int)big, d, kWave));
        if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = big;
        __syncthreads();
        big = max(max(most[0], most[1]), max(most[2], most[3]));
        // 2^(14 - exponent) for the exponent of the largest element; a row of zeros or subnormals gets the largest power
        const int power = min(14 - ((int)(big >> 7) - 127), 126);
        scale = __builtin_bit_cast(float, (uint32_t)(power + 127) << 23);
        if (threadIdx.x == 0) inverse[row] = __builtin_bit_cast(float, (uint32_t)(127 - power) << 23);
    }
    auto one = [&](uint32_t bits) {
        if constexpr (DT == kBF16) return (uint16_t)f32_to_f16_bits(bf16_bits_to_f32(bits) * scale);
        else return (uint16_t)bits;
    };
    if (wide) {
        for (int c = threadIdx.x; c < lda / 8; c += 256) {
            uint4v a = {0, 0, 0, 0};
            if (c * 8 < K) a = *(const uint4v*)(src + c * 8);
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                const uint32_t d = a[p];
                a[p] = one(d & 0xFFFFu) | (uint32_t)one(d >> 16) << 16;
            }
            *(uint4v*)(dst + c * 8) = a;
        }
    } else {
        for (int c = threadIdx.x; c < lda; c += 256) dst[c] = c < K ? one(src[c]) : 0;
    }
}

// Signs of rows of `words` words copied into rows of `wide` (a multiple of four), for the experts that have tokens.
__global__ void __launch_bounds__(256)
experts_signs_kernel(const uint32_t* __restrict__ B, uint32_t* __restrict__ out, const int* __restrict__ offsets, int M, int64_t each, int words, int wide)
{
    const int e = blockIdx.y;
    int first, end;
    expert_rows(offsets, e, M, first, end);
    if (first == end) return;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;       // word of the expert's copy
    if (at >= each) return;
    const int64_t row = at / wide;
    const int col = (int)(at - row * wide);
    out[e * each + at] = col < words ? B[(e * (each / wide) + row) * words + col] : 0;
}

void launch_experts_copy_rows(const void* rows, void* out, int64_t M, int64_t K, hipStream_t stream)
{
    hipLaunchKernelGGL(experts_prepare_kernel<kF16>, dim3((unsigned)M), dim3(256), 0, stream, (const uint16_t*)rows, (uint16_t*)out, nullptr,
                       (int)K, (int)experts_padded(K));
}

// The workspace of a product, from its start: prepared tokens (fp16 rows of experts_padded(K) values) and their factors; forward, signs
// in rows of 16 bytes; sums of the parts.
struct ProductLayout {
    bool prepare, wide_signs;
    int parts;
    size_t factors, signs, partial, all;

    ProductLayout(bool grad, int64_t M, int64_t E, int64_t d_out, int64_t d_in, int dtype)
    {
        const int64_t K = grad ? d_out : d_in, N = grad ? d_in : d_out;
        prepare = dtype == kBF16 || K % 128 != 0;
        wide_signs = !grad && d_in % 128 != 0;
        parts = experts_parts(M, E, N, K);
        factors = prepare ? (size_t)(M * experts_padded(K)) * 2 : 0;
        signs = factors + (prepare ? (size_t)(M + 3) / 4 * 16 : 0);
        partial = signs + (wide_signs ? (size_t)(E * d_out * experts_padded(d_in) / 8) : 0);
        all = partial + (parts > 1 ? (size_t)(parts * M * experts_pitch(N)) * 4 : 0);
    }
};

static int launch_product(const ExpertsCall& call, bool grad, hipStream_t stream)
{
    ExpertsCall c = call;
    const ProductLayout at(grad, c.M, c.E, c.d_out, c.d_in, c.dtype);
    const int64_t K = grad ? c.d_out : c.d_in;
    char* workspace = (char*)c.workspace;
    const uint16_t* A = (const uint16_t*)c.tokens;
    const float* inverse = nullptr;
    const int lda = (int)experts_padded(K);
    int sign_ld = (int)(c.d_in / 8);
    if (at.prepare && c.dtype == kBF16) {
        inverse = (const float*)(workspace + at.factors);
        hipLaunchKernelGGL(experts_prepare_kernel<kBF16>, dim3((unsigned)c.M), dim3(256), 0, stream, A, (uint16_t*)workspace,
                           (float*)(workspace + at.factors), (int)K, lda);
    } else if (at.prepare) {
        launch_experts_copy_rows(A, workspace, c.M, K, stream);
    }
    if (at.prepare) A = (const uint16_t*)workspace;
    if (at.wide_signs) {
        sign_ld = (int)(experts_padded(c.d_in) / 8);
        const int64_t each = c.d_out * sign_ld / 4, blocks = (each + 255) / 256;
        if (blocks > 0x7FFFFFFF) return -2;
        hipLaunchKernelGGL(experts_signs_kernel, dim3((unsigned)blocks, (unsigned)c.E), dim3(256), 0, stream, c.B_packed,
                           (uint32_t*)(workspace + at.signs), c.offsets, (int)c.M, each, (int)(c.d_in / 32), sign_ld / 4);
        c.B_packed = (const uint32_t*)(workspace + at.signs);
    }
    return launch_experts_big(c, grad, A, lda, inverse, (float*)(workspace + at.partial), at.parts, sign_ld, stream);
}

size_t experts_linear_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int dtype)
{
    if (M == 0 || experts_decode_tokens(M, E, d_out, d_in) > 0) return 0;
    return ProductLayout(false, M, E, d_out, d_in, dtype).all;
}
size_t experts_grad_x_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int dtype)
{
    return M == 0 ? 0 : ProductLayout(true, M, E, d_out, d_in, dtype).all;
}
int launch_experts_linear(const ExpertsCall& c, hipStream_t stream)
{
    const int mt = experts_decode_tokens(c.M, c.E, c.d_out, c.d_in);
    return mt > 0 ? launch_experts_skinny(c, mt, stream) : launch_product(c, false, stream);
}
int launch_experts_grad_x(const ExpertsCall& c, hipStream_t stream) { return launch_product(c, true, stream); }

}  // namespace pdelta
