// Decode-shaped delta linear layer (1 to 64 tokens), d_in a multiple of 128: the arithmetic of pdelta_linear_skinny.hip (two
// accumulators, base and sign part, in the operands' own dtype) with all operands coming by direct loads into LDS.
//
// What bounds the register-staged kernel for batches: it reads X (61 tokens on 4096 inputs: 0.5 MB) once per 16 output
// rows and gets every 16 bytes into the MFMA's layout with four lane permutations, 80 per wave and 128 inputs at 64 tokens.
// A direct load puts them where one 16-byte LDS read finds them, and a workgroup takes 16, 32 or 48 rows, so X crosses the
// L2 a third as often.
//
// Work split: 8 waves, wave w with the units w, w + 8, ... of 128 inputs (the sums of the other decode kernels, bit for bit),
// LDS of its own and no barrier before the last sum.  A step is 64 inputs, whole 128-byte lines of every row (with 64-byte pieces 16 rows more cost a workgroup 4.5 us instead of 2.1: what
// a CU gets from memory is limited in requests, about 480 a us).  Several row tiles leave room for one stage per wave: a
// step goes to registers as a whole and the next is asked for before the products.  That beats more stages for four waves,
// whatever their number: alone on its SIMD a wave issues too slowly (61 tokens, 11008 x 4096, 48 rows: 29.4 us, and 22.9
// of them without any load in the loop).  Measured and dropped as well: waves that share X behind a barrier per step
// (28.7), the same with W_b asked for eight steps ahead (29.8).
//
// What is left is waiting.  Counters of 61 tokens, 11008 x 4096 bf16 (100.5 MB fetched, 1.04 of what has to be): matrix cores
// busy 24 % of the CU's cycles, vector ALUs 17 %, LDS 14 %; waves issue during 18 % of their life and spend 49 % on
// instructions that are under way.
//
// Calls in a row in a graph, weights changing, us, the kernels that took these calls before -> this one:
// bf16 row, 11008 x 4096, 61 tokens 46.9 -> 27.2, 24 tokens 33.4 -> 22.4, 16 tokens 23.3 -> 22.1; 4096 x 11008, 64 tokens
// 44.8 -> 36.9; 4096 x 4096, 64 tokens 18.8 -> 15.6, 24 tokens 13.6 -> 10.8.
#include <algorithm>
#include <type_traits>

#include "pdelta.h"
#include "pdelta_host.h"
#include "pdelta_skinny_dma_tile.h"

namespace pdelta {

// MT tiles of 16 tokens, NT tiles of 16 output rows.
template <int XDT, int AXIS, int MT, int NT>
__global__ void __launch_bounds__(kDmaWaves * 64, 2)
linear_skinny_dma_kernel(const uint16_t* __restrict__ X, const uint16_t* __restrict__ W_b, const uint32_t* __restrict__ B_packed,
                         const uint16_t* __restrict__ v, void* __restrict__ Y, int M, int d_out, int d_in, int y_dtype,
                         int v_stride, int g_shift)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char dma_lds[];
    linear_skinny_dma_tile<XDT, AXIS, MT, NT, dma_depth(AXIS, MT, NT)>(X, W_b, B_packed, v, Y, M, d_out, d_in, y_dtype, v_stride, g_shift,
                                                                       blockIdx.x * (NT * 16), dma_lds);
}

template <int XDT, int AXIS, int MT, int NT>
static int launch_dma(const void* X, const void* W_b, const uint32_t* B_packed, const uint16_t* v, void* Y, int64_t M,
                      int64_t d_out, int64_t d_in, int y_dtype, int v_stride, int g_shift, hipStream_t stream)
{
    constexpr int wave_lds = dma_wave_bytes(AXIS, MT, NT, dma_depth(AXIS, MT, NT)), lds = kDmaWaves * wave_lds;
    static_assert(wave_lds >= MT * NT * 1024 && lds <= 160 * 1024, "LDS of a workgroup");
    auto kernel = linear_skinny_dma_kernel<XDT, AXIS, MT, NT>;
    static unsigned lds_opted_in = 0;                 // per template instance: one kernel
    if (opt_in_dynamic_lds((const void*)kernel, lds, &lds_opted_in) != 0) return -1;
    hipLaunchKernelGGL(kernel, dim3((unsigned)((d_out + NT * 16 - 1) / (NT * 16))), dim3(kDmaWaves * 64), lds, stream, (const uint16_t*)X,
                       (const uint16_t*)W_b, B_packed, v, Y, (int)M, (int)d_out, (int)d_in, y_dtype, v_stride, g_shift);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

template <int XDT, int AXIS>
static int launch_dma_tokens(const void* X, const void* W_b, const uint32_t* B_packed, const uint16_t* v, void* Y, int64_t M,
                             int64_t d_out, int64_t d_in, int y_dtype, int v_stride, int g_shift, int nt, hipStream_t stream)
{
    const int mt = (int)((M + 15) / 16);
#define PDELTA_GO(MT, NT) \
    return launch_dma<XDT, AXIS, MT, NT>(X, W_b, B_packed, v, Y, M, d_out, d_in, y_dtype, v_stride, g_shift, stream)
#define PDELTA_ROWS(MT)           \
    {                             \
        if (nt == 1) PDELTA_GO(MT, 1); \
        if (nt == 2) PDELTA_GO(MT, 2); \
        PDELTA_GO(MT, 3);         \
    }
    if (mt == 1) PDELTA_ROWS(1)
    if (mt == 2) PDELTA_ROWS(2)
    if (mt == 3) PDELTA_ROWS(3)
    PDELTA_ROWS(4)
#undef PDELTA_ROWS
#undef PDELTA_GO
}

int launch_linear_skinny_dma(int x_dtype, int y_dtype, int axis, const void* X, const void* W_b, const uint32_t* B_packed,
                             const uint16_t* v, void* Y, int64_t M, int64_t d_out, int64_t d_in, int v_stride, int g_shift,
                             int rows, hipStream_t stream)
{
#define PDELTA_GO(XDT, AXIS) return launch_dma_tokens<XDT, AXIS>(X, W_b, B_packed, v, Y, M, d_out, d_in, y_dtype, v_stride, g_shift, rows, stream)
    if (x_dtype == kBF16) {
        if (axis == 0) PDELTA_GO(kBF16, 0);
        if (axis == 1) PDELTA_GO(kBF16, 1);
        PDELTA_GO(kBF16, 2);
    }
    if (axis == 0) PDELTA_GO(kF16, 0);
    if (axis == 1) PDELTA_GO(kF16, 1);
    PDELTA_GO(kF16, 2);
#undef PDELTA_GO
}

}  // namespace pdelta
