// Gradient with respect to the scale vectors of tokens sorted by expert.  Both modes are sums of
//   D_e = dY_e^T X_e   [d_out, d_in]   (the products of the tokens of expert e)
// with the signs:  row  grad[e, o] = sum_i B_e[o, i] D_e[o, i],   col  grad[e, i] = sum_o B_e[o, i] D_e[o, i].
// D is formed tile by tile on the matrix cores in the operands' own format (exact products, fp32 sums) and never written:
// the signs meet it in the accumulators, so they are read once for every expert that has tokens, and its few tokens are
// all that the contraction runs over.  The dimension that is summed over is the accumulator's row dimension, the other one
// its columns: a lane adds its own elements, and two lanes meet once.
#include <algorithm>

#include "pdelta_experts.h"
#include "pdelta_host.h"
#include "pdelta_skinny_tile.h"

namespace pdelta {

template <int DT>
__device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c)
{
    if constexpr (DT == kBF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// The general tile: 64 of the summed dimension x 64 of the kept one, steps of 64 tokens, 4 waves of 32 x 32.
constexpr int kGradTile = 64, kGradTokens = 64, kGradLD = kGradTokens + 8;

template <int DT, int AXIS>
__global__ void __launch_bounds__(256)
experts_grad_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ dY, const int* __restrict__ offsets,
                    const uint32_t* __restrict__ B_packed, float* __restrict__ partial, int M, int d_out, int d_in, int kept_tiles,
                    int sum_tiles)
{
    __shared__ __attribute__((aligned(16))) uint16_t Ps[kGradTile * kGradLD], Qs[kGradTile * kGradLD];
    __shared__ float red[2][kGradTile];
    const int kt = blockIdx.x % kept_tiles, st = blockIdx.x / kept_tiles % sum_tiles, e = blockIdx.x / kept_tiles / sum_tiles;
    int first, end;
    expert_rows(offsets, e, M, first, end);
    if (first == end) return;                         // whole workgroup
    const uint16_t* P = AXIS == 0 ? X : dY;           // summed dimension
    const uint16_t* Q = AXIS == 0 ? dY : X;           // kept dimension
    const int dP = AXIS == 0 ? d_in : d_out, dQ = AXIS == 0 ? d_out : d_in;
    const int p0 = st * kGradTile, q0 = kt * kGradTile;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;

    // [token][column] -> LDS [column][token]; what is behind the expert's tokens or the matrix is zero
    auto stage = [&](const uint16_t* src, int width, int c0, int m0, uint16_t* lds) {
        for (int c = tid; c < kGradTile * kGradTokens; c += 256) {
            const int col = c % kGradTile, tok = c / kGradTile;
            lds[col * kGradLD + tok] = m0 + tok < end && c0 + col < width ? src[(int64_t)(m0 + tok) * width + c0 + col] : 0;
        }
    };
    float16v acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    for (int m0 = first; m0 < end; m0 += kGradTokens) {
        stage(P, dP, p0, m0, Ps);
        stage(Q, dQ, q0, m0, Qs);
        __syncthreads();
        const int at = (lane & 31) * kGradLD + (lane >> 5) * 8;
#pragma unroll
        for (int ks = 0; ks < kGradTokens; ks += 16) {
            const uint4v a = *(const uint4v*)(Ps + (wave >> 1) * 32 * kGradLD + at + ks);
            const uint4v b = *(const uint4v*)(Qs + (wave & 1) * 32 * kGradLD + at + ks);
            acc = mfma32<DT>(a, b, acc);
        }
        __syncthreads();
    }
    // 32x32 accumulator: element r of lane l is row (r/4)*8 + (l/32)*4 + r%4, column l%32
    const uint32_t* words = B_packed + (int64_t)e * d_out * (d_in / 32);
    const int pw = p0 + (wave >> 1) * 32, q = q0 + (wave & 1) * 32 + (lane & 31);
    const int qc = min(q, dQ - 1);
    float sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int row = (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
        const int o = AXIS == 0 ? qc : min(pw + row, d_out - 1), i = AXIS == 0 ? min(pw, d_in - 32) + row : qc;
        const uint32_t plus = (words[(int64_t)o * (d_in / 32) + i / 32] >> (i & 31)) & 1u;
        sum += plus ? acc[r] : -acc[r];               // (rows behind the matrix are zero)
    }
    sum += __shfl_xor(sum, 32, kWave);
    if (lane < 32) red[wave >> 1][(wave & 1) * 32 + lane] = sum;
    __syncthreads();
    if (tid < kGradTile && q0 + tid < dQ)
        partial[((int64_t)e * sum_tiles + st) * dQ + q0 + tid] = red[0][tid] + red[1][tid];
}

// The sums of the tiles of one expert, in their order.
__global__ void __launch_bounds__(256)
experts_grad_sum_kernel(const float* __restrict__ partial, const int* __restrict__ offsets, float* __restrict__ grad, int M, int dQ,
                        int sum_tiles, int blocks)
{
    const int e = blockIdx.x / blocks, q = (blockIdx.x % blocks) * 256 + threadIdx.x;
    int first, end;
    expert_rows(offsets, e, M, first, end);
    if (q >= dQ) return;
    float sum = 0.f;
    if (first < end)
        for (int s = 0; s < sum_tiles; ++s) sum += partial[((int64_t)e * sum_tiles + s) * dQ + q];
    grad[(int64_t)e * dQ + q] = sum;
}

size_t experts_grad_v_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int axis)
{
    (void)M;
    const int64_t kept = axis == 0 ? d_out : d_in, summed = axis == 0 ? d_in : d_out;
    return (size_t)E * (size_t)((summed + kGradTile - 1) / kGradTile) * (size_t)kept * 4;
}

template <int DT, int AXIS>
static int launch_grad(const void* X, const void* dY, const int* offsets, const uint32_t* B_packed, float* grad, int64_t M, int64_t E,
                       int64_t d_out, int64_t d_in, void* workspace, hipStream_t stream)
{
    const int64_t kept = AXIS == 0 ? d_out : d_in, summed = AXIS == 0 ? d_in : d_out;
    const int64_t kept_tiles = (kept + kGradTile - 1) / kGradTile, sum_tiles = (summed + kGradTile - 1) / kGradTile;
    const int64_t sum_blocks = (kept + 255) / 256;
    if (E * kept_tiles * sum_tiles > 0x7FFFFFFF || E * sum_blocks > 0x7FFFFFFF) return -2;
    if (M > 0)
        hipLaunchKernelGGL((experts_grad_kernel<DT, AXIS>), dim3((unsigned)(E * kept_tiles * sum_tiles)), dim3(256), 0, stream,
                           (const uint16_t*)X, (const uint16_t*)dY, offsets, B_packed, (float*)workspace, (int)M, (int)d_out, (int)d_in,
                           (int)kept_tiles, (int)sum_tiles);
    hipLaunchKernelGGL(experts_grad_sum_kernel, dim3((unsigned)(E * sum_blocks)), dim3(256), 0, stream, (const float*)workspace, offsets,
                       grad, (int)M, (int)kept, (int)sum_tiles, (int)sum_blocks);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_experts_grad_v(int dtype, int axis, const void* X, const void* dY, const int* offsets, const uint32_t* B_packed, float* grad,
                          int64_t M, int64_t E, int64_t d_out, int64_t d_in, void* workspace, hipStream_t stream)
{
#define PDELTA_GO(DT, AXIS) return launch_grad<DT, AXIS>(X, dY, offsets, B_packed, grad, M, E, d_out, d_in, workspace, stream)
    if (dtype == kBF16) {
        if (axis == 0) PDELTA_GO(kBF16, 0);
        PDELTA_GO(kBF16, 1);
    }
    if (axis == 0) PDELTA_GO(kF16, 0);
    PDELTA_GO(kF16, 1);
#undef PDELTA_GO
}

}  // namespace pdelta
