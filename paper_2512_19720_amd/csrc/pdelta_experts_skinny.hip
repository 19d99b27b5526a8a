// Forward product of tokens sorted by expert where an expert has few of them (decode of a mixture of experts): the decode tile of
// the dense layer, 16 MT tokens of one expert x 16 NT output rows, for every expert that has tokens.  Memory-bound: the weights
// of every expert that is met are read once for each 16 MT tokens of its, and those of the others not at all (32 tokens x 2 of 64 experts,
// 2048 x 4096 bf16: 0.50 GB in 81 us, 6.2 TB/s).
//
// A workgroup first looks its expert up, a load and a prefix sum away from its first weight, and ends with a sum over its waves;
// two stages of a wave (or two row tiles and one) leave room for two workgroups on a CU, which cover each other's ends.
#include <algorithm>

#include "pdelta_experts.h"
#include "pdelta_host.h"
#include "pdelta_skinny_dma_tile.h"

namespace pdelta {

constexpr int expert_depth(int nt) { return nt == 1 ? 2 : 1; }

template <int XDT, int AXIS, int MT, int NT>
__global__ void __launch_bounds__(kDmaWaves * 64, 4)
experts_skinny_kernel(const uint16_t* __restrict__ X, const int* __restrict__ offsets, const uint16_t* __restrict__ W_b, int64_t w_stride,
                      const uint32_t* __restrict__ B_packed, const uint16_t* __restrict__ v, void* __restrict__ Y, int M, int E, int d_out,
                      int d_in, int y_dtype, int row_tiles)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char dma_lds[];
    ExpertTile t;
    if (!find_expert_tile<MT * 16>(offsets, E, M, blockIdx.x / row_tiles, t)) return;       // whole workgroup
    const int rows = min(t.end - t.row0, MT * 16);
    char* out = (char*)Y + (int64_t)t.row0 * d_out * (y_dtype == kF32 ? 4 : 2);
    linear_skinny_dma_tile<XDT, AXIS, MT, NT, expert_depth(NT)>(
        X + (int64_t)t.row0 * d_in, W_b + t.expert * w_stride, B_packed + (int64_t)t.expert * d_out * (d_in / 32),
        v + (int64_t)t.expert * (AXIS == 0 ? d_out : d_in), out, rows, d_out, d_in, y_dtype, 0, 0, blockIdx.x % row_tiles * (NT * 16), dma_lds);
}

template <int XDT, int AXIS, int MT, int NT>
static int launch_skinny(const ExpertsCall& c, hipStream_t stream)
{
    constexpr int wave_lds = dma_wave_bytes(AXIS, MT, NT, expert_depth(NT)), lds = kDmaWaves * wave_lds;
    static_assert(wave_lds >= MT * NT * 1024 && lds <= 160 * 1024, "LDS of a workgroup");
    const int64_t row_tiles = (c.d_out + NT * 16 - 1) / (NT * 16), blocks = most_expert_tiles(c.M, c.E, MT * 16) * row_tiles;
    if (blocks > 0x7FFFFFFF) return -2;
    auto kernel = experts_skinny_kernel<XDT, AXIS, MT, NT>;
    static unsigned lds_opted_in = 0;                 // per template instance: one kernel
    if (opt_in_dynamic_lds((const void*)kernel, lds, &lds_opted_in) != 0) return -1;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kDmaWaves * 64), lds, stream, (const uint16_t*)c.tokens, c.offsets,
                       (const uint16_t*)c.W_b, c.w_stride, c.B_packed, c.v, c.out, (int)c.M, (int)c.E, (int)c.d_out, (int)c.d_in, c.out_dtype,
                       (int)row_tiles);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

// Up to 16 tokens for each expert that can be met, always; up to 32 where those experts have at most 128 tiles of 256 outputs, half a
// tile for each CU: with more of them the large tiles fill the CUs, and with fewer they are cut into parts and summed by another launch.
// Uneven experts read their weights once for each 16 (32) of their tokens.  us here and on the large tiles, experts x outputs x inputs, bf16 row:
// 32 x 2048 x 4096, 10 tokens each 99 and 131; 4 x 11008 x 4096 10 67 and 81.  Of 17 to 32 tokens each, over nine layers of 256 x 512 to
// 14336 x 4096, 1 to 64 experts, even and uneven, both types and kinds of scales: time over the better of the two 1.026 on average with this
// limit (geometric mean; own bases 1.022, one base 1.031), 1.067 always here, 1.38 always there.  fp16 row, 20 tokens each: 4 x 4096 x 4096
// (64 tiles) 34.7 and 36.7, with one base 18.0 and 36.4; 8 x 4096 x 4096 (128) 65.8 and 61.1, with one base 31.7 and 57.4.  What the limit
// gets wrong most: two uneven experts of 14336 x 4096 (112), fp16 column, 1.6 times the large tiles' time; 32 of 1408 x 2048 with one base (192), bf16 row,
// 1.7 times the time here.
int experts_decode_tokens(int64_t M, int64_t E, int64_t d_out, int64_t d_in)
{
    if (M == 0 || d_in % kDmaUnitK != 0) return 0;
    const int64_t met = std::min(E, M), each = (M + met - 1) / met;
    return each <= 16 ? 1 : each <= 32 && met * ((d_out + 255) / 256) <= 128 ? 2 : 0;
}

int launch_experts_skinny(const ExpertsCall& c, int mt, hipStream_t stream)
{
    // Two row tiles for a workgroup, which share the loads of the tokens.  One where the rows of W_b are a multiple of 8 KB apart, so that the
    // same inputs of 32 rows lie in few of the memory's channels, and come from there: not out of the caches, where one base of up to 64 MB
    // stays.  us with one and two, 10 tokens each, bf16 row, experts x outputs x inputs: 16 x 2048 x 4096 51.8, 65.1, x 3584 39.0, 37.3, x 5120 67.9,
    // 63.6; 32 x 1408 x 2048 40.9, 38.4; one base: 16 x 4096 x 4096 58.9, 46.7, 4 x 14336 x 4096 76.5, 91.7, 8 x 4096 x 8192 87.1, 60.3.  Over 25 layers of
    // 256 x 512 to 28672 x 1024, 1 to 64 experts of 1 to 16 tokens: time over the better one's 1.007 on average (geometric mean), 1.15 with one, 1.04
    // with two.
    const bool one = c.d_in % 4096 == 0 && (c.w_stride != 0 || c.d_out * c.d_in > 1 << 25);
#define PDELTA_GO(XDT, AXIS)                                              \
    {                                                                     \
        if (mt == 2) return launch_skinny<XDT, AXIS, 2, 2>(c, stream);    \
        if (one) return launch_skinny<XDT, AXIS, 1, 1>(c, stream);        \
        return launch_skinny<XDT, AXIS, 1, 2>(c, stream);                 \
    }
    if (c.dtype == kBF16) {
        if (c.axis == 0) PDELTA_GO(kBF16, 0)
        PDELTA_GO(kBF16, 1)
    }
    if (c.axis == 0) PDELTA_GO(kF16, 0)
    PDELTA_GO(kF16, 1)
#undef PDELTA_GO
}

}  // namespace pdelta
