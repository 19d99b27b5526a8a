// Products of tokens sorted by expert with every expert's W_hat = W_b + v (.) B, never written to memory:
//   forward   Y[m, o]  = sum_i X[m, i]  W_hat_e[o, i]
//   backward  dX[m, i] = sum_o dY[m, o] W_hat_e[o, i]
// for the tokens m of every expert e.  The arithmetic is that of the prefill kernels: the tile of W_hat is formed as
// fp16(W_b +- v) with one rounding, fp32 sums.
//
// The token operand is always multiplied as fp16.  A bf16 one is converted first, by experts_prepare_kernel, every row
// times the power of two that brings its largest element to [2^14, 2^15): gradients are often far below fp16's range,
// and differ in size from token to token.  The conversion is exact for elements within 2^28 of their row's largest and
// off by at most 2^-39 of the largest for the others; the outputs are multiplied by the inverse power in fp32, exactly.
// The same kernel copies fp16 rows that are no multiple of 16 bytes into rows that are.
#include <algorithm>
#include <type_traits>

#include "pdelta_experts.h"
#include "pdelta_gemm_tile.h"
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

// The general tile: 64 tokens x 64 outputs x 64 of the contraction, 4 waves of 32 x 32 outputs, for any sizes.
// GRAD: the contraction runs over d_out and the tile of W_hat is transposed on its way into LDS.
constexpr int kSimpleTile = 64, kSimpleBK = 64, kSimpleLD = kSimpleBK + 8;

template <int WDT, int AXIS, bool GRAD>
__global__ void __launch_bounds__(256)
experts_tile_kernel(const uint16_t* __restrict__ A, int lda, const float* __restrict__ inverse, const int* __restrict__ offsets,
                    const uint16_t* __restrict__ W_b, int64_t w_stride, const uint32_t* __restrict__ B_packed,
                    const uint16_t* __restrict__ v, void* __restrict__ Y, int M, int E, int d_out, int d_in, int y_dtype, int n_tiles)
{
    __shared__ __attribute__((aligned(16))) uint16_t As[kSimpleTile * kSimpleLD], Ws[kSimpleTile * kSimpleLD];
    const int tile_n = blockIdx.x % n_tiles;
    ExpertTile t;
    if (!find_expert_tile<kSimpleTile>(offsets, E, M, blockIdx.x / n_tiles, t)) return;     // whole workgroup
    const int N = GRAD ? d_in : d_out, K = GRAD ? d_out : d_in;
    const int n0 = tile_n * kSimpleTile;
    const uint16_t* W = W_b + t.expert * w_stride;
    const unsigned char* signs = (const unsigned char*)(B_packed + (int64_t)t.expert * d_out * (d_in / 32));
    const uint16_t* scales = v + (int64_t)t.expert * (AXIS == 0 ? d_out : d_in);

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int c8 = (tid & 7) * 8, r0 = tid >> 3;      // staging: rows r0 and r0 + 32 of the tile, 8 values at c8
    float16v acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;

    for (int kb = 0; kb < K; kb += kSimpleBK) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int r = r0 + q * 32;
            const uint4v zero = {0, 0, 0, 0};
            // (a row of A holds lda values; what is behind K in it is zero)
            const int row = min(t.row0 + r, t.end - 1);
            *(uint4v*)(As + r * kSimpleLD + c8) = kb + c8 < lda ? *(const uint4v*)(A + (int64_t)row * lda + kb + c8) : zero;
            // eight weights of one output row: [o, i .. i + 7]
            const int o = GRAD ? kb + r : min(n0 + r, d_out - 1);
            const int i = GRAD ? n0 + c8 : kb + c8;
            uint4v what = zero;
            if (o < d_out && i < d_in) {
                const int64_t at = (int64_t)o * d_in + i;
                const uint4v w16 = to_f16x8<WDT>(*(const uint4v*)(W + at));
                uint4v vv;
                if constexpr (AXIS == 0) {
                    const uint32_t h = scales[o];
                    vv = (uint4v){h * 0x10001u, h * 0x10001u, h * 0x10001u, h * 0x10001u};
                } else {
                    vv = *(const uint4v*)(scales + i);
                }
                const uint32_t minus = ~(uint32_t)signs[at >> 3];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const uint32_t flip = ((minus >> (2 * p)) & 1u) << 15 | ((minus >> (2 * p + 1)) & 1u) << 31;
                    const uint32_t wp = w16[p], vp = vv[p];
                    what[p] = as_u32(as_half2(wp) + as_half2(vp ^ flip));
                }
            }
            if constexpr (GRAD) {
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    const uint32_t d = what[p];
                    Ws[(c8 + 2 * p) * kSimpleLD + r] = (uint16_t)d;
                    Ws[(c8 + 2 * p + 1) * kSimpleLD + r] = (uint16_t)(d >> 16);
                }
            } else {
                *(uint4v*)(Ws + r * kSimpleLD + c8) = what;
            }
        }
        __syncthreads();
        const int at = (lane & 31) * kSimpleLD + (lane >> 5) * 8;
#pragma unroll
        for (int ks = 0; ks < kSimpleBK; ks += 16) {
            const half8 a = *(const half8*)(As + (wave >> 1) * 32 * kSimpleLD + at + ks);
            const half8 b = *(const half8*)(Ws + (wave & 1) * 32 * kSimpleLD + at + ks);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, acc, 0, 0, 0);
        }
        __syncthreads();
    }
    // 32x32 accumulator: element r of lane l is row (r/4)*8 + (l/32)*4 + r%4, column l%32
    const int n = n0 + (wave & 1) * 32 + (lane & 31);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int m = t.row0 + (wave >> 1) * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
        if (m < t.end && n < N) {
            const int64_t yi = (int64_t)m * N + n;
            const float val = inverse != nullptr ? acc[r] * inverse[m] : acc[r];
            if (y_dtype == kF32) store_y<kF32>(Y, yi, val);
            else if (y_dtype == kBF16) store_y<kBF16>(Y, yi, val);
            else store_y<kF16>(Y, yi, val);
        }
    }
}

void launch_experts_copy_rows(const void* rows, void* out, int64_t M, int64_t K, hipStream_t stream)
{
    hipLaunchKernelGGL(experts_prepare_kernel<kF16>, dim3((unsigned)M), dim3(256), 0, stream, (const uint16_t*)rows, (uint16_t*)out, nullptr,
                       (int)K, (int)experts_padded(K));
}

// The prepared token operand: fp16 rows of `lda` values, behind them an fp32 factor for each row.
static bool needs_prepare(int64_t K, int dtype) { return dtype == kBF16 || (K & 127) != 0; }

static size_t prepared_bytes(int64_t M, int64_t K, int dtype)
{
    if (!needs_prepare(K, dtype)) return 0;
    return (size_t)M * (size_t)experts_padded(K) * 2 + ((size_t)M * 4 + 15) / 16 * 16;
}
// Whether the tiles with direct loads take a product whose contraction is K long.
static bool takes_big(bool grad, int64_t K) { return grad || (K & 127) == 0; }
static size_t product_bytes(bool grad, int64_t M, int64_t E, int64_t N, int64_t K, int dtype)
{
    const int64_t parts = takes_big(grad, K) ? experts_parts(M, E, N, K) : 1;
    return prepared_bytes(M, K, dtype) + (parts > 1 ? (size_t)(parts * M * N) * 4 : 0);
}

template <int WDT, int AXIS, bool GRAD>
static int launch_tiles(const ExpertsCall& c, const uint16_t* A, int lda, const float* inverse, hipStream_t stream)
{
    const int64_t N = GRAD ? c.d_in : c.d_out;
    const int n_tiles = (int)((N + kSimpleTile - 1) / kSimpleTile);
    const int64_t blocks = most_expert_tiles(c.M, c.E, kSimpleTile) * n_tiles;
    if (blocks > 0x7FFFFFFF) return -2;
    hipLaunchKernelGGL((experts_tile_kernel<WDT, AXIS, GRAD>), dim3((unsigned)blocks), dim3(256), 0, stream, A, lda, inverse, c.offsets,
                       (const uint16_t*)c.W_b, c.w_stride, c.B_packed, c.v, c.out, (int)c.M, (int)c.E, (int)c.d_out, (int)c.d_in,
                       c.out_dtype, n_tiles);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

static int launch_product(const ExpertsCall& c, bool grad, hipStream_t stream)
{
    const int64_t K = grad ? c.d_out : c.d_in;
    const uint16_t* A = (const uint16_t*)c.tokens;
    const float* inverse = nullptr;
    int lda = (int)K;
    if (needs_prepare(K, c.dtype)) {
        lda = (int)experts_padded(K);
        uint16_t* rows = (uint16_t*)c.workspace;
        float* factors = (float*)(rows + c.M * lda);
        if (c.dtype == kBF16) {
            hipLaunchKernelGGL(experts_prepare_kernel<kBF16>, dim3((unsigned)c.M), dim3(256), 0, stream, A, rows, factors, (int)K, lda);
            inverse = factors;
        } else {
            launch_experts_copy_rows(A, rows, c.M, K, stream);
        }
        A = rows;
    }
    if (takes_big(grad, K)) {
        const int64_t N = grad ? c.d_in : c.d_out;
        return launch_experts_big(c, grad, A, lda, inverse, (float*)((char*)c.workspace + prepared_bytes(c.M, K, c.dtype)),
                                  experts_parts(c.M, c.E, N, K), stream);
    }
#define PDELTA_GO(WDT, AXIS) \
    return grad ? launch_tiles<WDT, AXIS, true>(c, A, lda, inverse, stream) : launch_tiles<WDT, AXIS, false>(c, A, lda, inverse, stream)
    if (c.dtype == kBF16) {
        if (c.axis == 0) PDELTA_GO(kBF16, 0);
        PDELTA_GO(kBF16, 1);
    }
    if (c.axis == 0) PDELTA_GO(kF16, 0);
    PDELTA_GO(kF16, 1);
#undef PDELTA_GO
}

size_t experts_linear_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int dtype)
{
    return experts_decode_tokens(M, E, d_out, d_in, dtype) > 0 ? 0 : product_bytes(false, M, E, d_out, d_in, dtype);
}
size_t experts_grad_x_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int dtype)
{
    return product_bytes(true, M, E, d_in, d_out, dtype);
}
int launch_experts_linear(const ExpertsCall& c, hipStream_t stream)
{
    const int mt = experts_decode_tokens(c.M, c.E, c.d_out, c.d_in, c.dtype);
    return mt > 0 ? launch_experts_skinny(c, mt, stream) : launch_product(c, false, stream);
}
int launch_experts_grad_x(const ExpertsCall& c, hipStream_t stream) { return launch_product(c, true, stream); }

}  // namespace pdelta
