// Pieces shared by the kernels that work on tokens sorted by expert: expert e owns the rows
// offsets[e] .. offsets[e + 1] - 1 of the token matrices.
#pragma once

#include "pdelta_device.h"

namespace pdelta {

// Rows of one tile of up to BM tokens of one expert; `end` is the first row behind the expert's own.
struct ExpertTile { int expert, row0, end; };

// The tokens of expert e, in bounds whatever the offsets hold; without offsets all of them (one expert).
__device__ __forceinline__ void expert_rows(const int* __restrict__ offsets, int e, int M, int& first, int& end)
{
    if (offsets == nullptr) {
        first = 0;
        end = M;
        return;
    }
    first = min(max(offsets[e], 0), M);
    end = max(first, min(offsets[e + 1], M));
}

// Tiles are numbered expert by expert.  Every wave looks its tile up by itself: a lane per expert, a prefix sum of their
// tiles.  Returns false (all lanes) behind the last tile.  `tile` is uniform across the wave.
template <int BM>
__device__ __forceinline__ bool find_expert_tile(const int* __restrict__ offsets, int E, int M, int tile, ExpertTile& out)
{
    const int lane = threadIdx.x & 63;
    for (int e0 = 0; e0 < E; e0 += kWave) {
        int first, end;
        expert_rows(offsets, min(e0 + lane, E - 1), M, first, end);
        const int tiles = e0 + lane < E ? (end - first + BM - 1) / BM : 0;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int below = __shfl_up(upto, d, kWave);
            if (lane >= d) upto += below;
        }
        const int all = __builtin_amdgcn_readlane(upto, kWave - 1);
        if (tile < all) {
            const int at = __builtin_ctzll(__ballot(upto > tile));
            out.expert = e0 + at;
            out.row0 = __builtin_amdgcn_readlane(first, at) + (tile - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(tiles, at))) * BM;
            out.end = __builtin_amdgcn_readlane(end, at);
            return true;
        }
        tile -= all;
    }
    return false;
}

// The most tiles of BM tokens that M tokens of E experts can make: every expert that has tokens may end in a short one.
inline int64_t most_expert_tiles(int64_t M, int64_t E, int BM)
{
    const int64_t met = E < M ? E : M;
    return (M - met) / BM + met;
}

}  // namespace pdelta
