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

// The tile of output tile and token tile that a workgroup takes: XCD `xcd` takes a contiguous range of all tiles (numbered expert
// by expert, then by output tile, then by token tile), the workgroup its `local`-th.  False (all lanes) behind the last.
template <int BM>
__device__ __forceinline__ bool find_expert_block(const int* __restrict__ offsets, int E, int M, int n_tiles, int xcd, int local,
                                                  ExpertTile& out, int& tile_n)
{
    const int lane = threadIdx.x & 63;
    int64_t tile = -1, all = 0, before = 0;           // first round: how many there are; second: where this one is
    for (int round = 0; round < 2; ++round) {
        before = 0;
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
            const int here = __builtin_amdgcn_readlane(upto, kWave - 1);
            if (round == 0 && E <= kWave) {           // one round is enough
                all = (int64_t)here * n_tiles;
                const int64_t per = (all + 7) / 8;
                tile = xcd * per + local;
                if (local >= per || tile >= all) return false;
            }
            if (tile >= 0 && tile < before + (int64_t)here * n_tiles) {
                const int64_t rest = tile - before;
                const int at = __builtin_ctzll(__ballot((int64_t)upto * n_tiles > rest));
                const int mine = __builtin_amdgcn_readlane(tiles, at);
                const int place = (int)(rest - (int64_t)(__builtin_amdgcn_readlane(upto, at) - mine) * n_tiles);
                tile_n = place / mine;
                out.expert = e0 + at;
                out.row0 = __builtin_amdgcn_readlane(first, at) + place % mine * BM;
                out.end = __builtin_amdgcn_readlane(end, at);
                return true;
            }
            before += (int64_t)here * n_tiles;
        }
        if (round == 0) {
            all = before;
            const int64_t per = (all + 7) / 8;
            tile = xcd * per + local;
            if (local >= per || tile >= all) return false;
        }
    }
    return false;
}

typedef short short4v __attribute__((ext_vector_type(4)));
// Four values of one column from 16 lanes' rows of four: lane 4 r + c of 16 points at columns 4 c .. 4 c + 3 of row r, lane i gets
// rows 0 .. 3 of column i.
__device__ __forceinline__ uint2v read_transposed(const unsigned char* p)
{
    return __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4v*)p));
}

// The most tiles of BM tokens that M tokens of E experts can make: every expert that has tokens may end in a short one.
inline int64_t most_expert_tiles(int64_t M, int64_t E, int BM)
{
    const int64_t met = E < M ? E : M;
    return (M - met) / BM + met;
}

}  // namespace pdelta
