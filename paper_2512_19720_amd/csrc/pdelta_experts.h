// Pieces shared by the kernels that work on tokens sorted by expert: expert e owns the rows
// offsets[e] .. offsets[e + 1] - 1 of the token matrices.
#pragma once

#include <algorithm>

#include "pdelta_device.h"

namespace pdelta {

// Rows of one tile of up to BM tokens of one expert; `end` is the first row behind the expert's own.  It is the `index`-th of
// the expert's `tiles`.
struct ExpertTile { int expert, row0, end, index, tiles; };

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
            out.tiles = __builtin_amdgcn_readlane(tiles, at);
            out.index = tile - (__builtin_amdgcn_readlane(upto, at) - out.tiles);
            out.row0 = __builtin_amdgcn_readlane(first, at) + out.index * BM;
            out.end = __builtin_amdgcn_readlane(end, at);
            return true;
        }
        tile -= all;
    }
    return false;
}

// The tiles of a product, up to `height` tokens x one output tile each, numbered expert by expert, then by output tile, then by token
// tile (an expert's last token tile may be a short one), dealt to the 8 XCDs in contiguous ranges of about the same cost: the CUs
// of an XCD then share panels of weights in its L2.  A tile of 64 f tokens costs f + 2, as measured next to a full one.
struct ExpertTiles {
    const int* offsets;
    int E, M, n_tiles;
    int height;                                       // 256, 192 or 128
    int at, e0;                                       // this range's next tile; first expert of the chunk that the lanes hold
    int first, end, tiles, cost;                      // of expert e0 + lane
    int tiles_upto, cost_upto;                        // sums up to and with it
    int tiles_before, cost_before;                    // sums of the chunks before

    __host__ __device__ static int full_cost(int rows) { return (rows + 63) / 64 + 2; }
    __device__ __forceinline__ int full() const { return full_cost(height); }
    __device__ __forceinline__ int lane() const { return threadIdx.x & 63; }
    __device__ __forceinline__ static int prefix(int x)
    {
#pragma unroll
        for (int d = 1; d < kWave; d <<= 1) {
            const int below = __shfl_up(x, d, kWave);
            if ((int)(threadIdx.x & 63) >= d) x += below;
        }
        return x;
    }
    __device__ __forceinline__ void rows_of(int from)
    {
        e0 = from;
        expert_rows(offsets, min(e0 + lane(), E - 1), M, first, end);
        if (e0 + lane() >= E) end = first;
    }
    __device__ __forceinline__ void count()
    {
        const int whole = (int)((uint32_t)(end - first) / (uint32_t)height), rest = end - first - whole * height;
        tiles = whole + (rest > 0);
        cost = whole * full_cost(height) + (rest > 0 ? full_cost(rest) : 0);
        tiles_upto = prefix(tiles);
        cost_upto = prefix(cost);
    }
    __device__ __forceinline__ void chunk(int from, int tiles_sum, int cost_sum)
    {
        tiles_before = tiles_sum;
        cost_before = cost_sum;
        rows_of(from);
        count();
    }
    __device__ __forceinline__ int chunk_tiles() const { return __builtin_amdgcn_readlane(tiles_upto, kWave - 1); }
    __device__ __forceinline__ int chunk_cost() const { return __builtin_amdgcn_readlane(cost_upto, kWave - 1); }
    // Holds the chunk of the expert for which `found` (of the sums up to and with an expert) is true first; its lane, or -1.
    template <typename F>
    __device__ __forceinline__ int seek(F found)
    {
        if (E > kWave) chunk(0, 0, 0);                // (else the lanes hold all experts)
        for (;;) {
            const uint64_t hit = __ballot(found(tiles_before + tiles_upto, cost_before + cost_upto));
            if (hit != 0) return __builtin_ctzll(hit);
            if (e0 + kWave >= E) return -1;
            chunk(e0 + kWave, tiles_before + chunk_tiles(), cost_before + chunk_cost());
        }
    }
    // Number of the first tile with at least `bound` of cost before it.
    __device__ __forceinline__ int first_at(int bound, int all)
    {
        const int n = n_tiles;
        const int l = seek([&](int, int upto) { return upto * n > bound; });
        if (l < 0) return all;
        const int mine = __builtin_amdgcn_readlane(tiles, l), each = __builtin_amdgcn_readlane(cost, l);
        const int rest = bound - (cost_before + __builtin_amdgcn_readlane(cost_upto, l) - each) * n;
        const int behind = (rest % each + full() - 1) / full();       // token tiles that start before the bound
        return (tiles_before + __builtin_amdgcn_readlane(tiles_upto, l) - mine) * n + rest / each * mine + min(behind, mine);
    }
    // Twice the time in which the 256 CUs work `tiles` off, the largest of cost `largest`, `cost` all together: whole rounds if they
    // are alike or there is one round, else a CU's mean and half a tile.
    __host__ __device__ static int64_t finish(int64_t tiles, int64_t cost, int largest, bool alike)
    {
        return alike || tiles <= 256 ? 2 * ((tiles + 255) / 256) * largest : cost / 128 + largest;
    }
    // A smaller height reads the weights more often: it is taken for a gain of an eighth.
    __host__ __device__ static bool gains(int64_t t, int64_t least) { return t * 8 <= least * 7; }
    // Heights by the tokens that the experts have, of one wave's lanes of experts.  See launch_big_tiles.
    __device__ __forceinline__ void choose_height()
    {
        rows_of(0);
        int most = 0;
#pragma unroll
        for (int f = 0; f < 4; ++f) most += __ballot(end - first > 64 * f) != 0;
        int best = height;
        int64_t least = 0;
        if (most > 2)
            for (int h = 256; h >= 128; h -= 64) {
                height = h;
                count();
                const int64_t t = finish((int64_t)chunk_tiles() * n_tiles, (int64_t)chunk_cost() * n_tiles, min(most, h / 64) + 2, false);
                if (h == 256 || gains(t, least)) { best = h; least = t; }
            }
        height = best;
    }
    static int height_of_one(int64_t M, int64_t n_tiles)
    {
        int best = 256;
        int64_t least = 0;
        for (int h = 256; h >= 128 && (M + 255) / 256 * n_tiles <= 768; h -= 64) {                // (three rounds)
            const int64_t t = finish((M + h - 1) / h * n_tiles, 0, full_cost((int)std::min<int64_t>(M, h)), true);
            if (h == 256 || gains(t, least)) { best = h; least = t; }
        }
        return best;
    }
    // Range [at, stop) of XCD `xcd`.
    __device__ __forceinline__ int range(int xcd)
    {
        int all_cost = 0, all = 0;
        for (e0 = 0; e0 < E; e0 += kWave) {
            chunk(e0, all, all_cost);
            all += chunk_tiles();
            all_cost += chunk_cost();
            if (E <= kWave) break;
        }
        all *= n_tiles;
        all_cost *= n_tiles;
        auto bound = [&](int x) { return all_cost / 8 * x + all_cost % 8 * x / 8; };
        const int stop = xcd == 7 ? all : first_at(bound(xcd + 1), all);
        at = first_at(bound(xcd), all);
        return stop;
    }
    // The most tiles that a range can have: M tokens cost full() for each `height` of them and, the last tile of each expert, at most 3 more;
    // the cheapest tile costs 3.
    static int64_t most_in_a_range(int64_t M, int64_t E, int64_t n_tiles, int height)
    {
        // one expert: runs of its token tiles, one for each output tile, in eight parts that may begin and end inside a run
        if (E == 1) return ((n_tiles + 7) / 8 + 1) * ((M + height - 1) / height);
        const int64_t cost = (M * full_cost(height) / height + 1 + 3 * std::min(E, M)) * n_tiles;
        return (cost / 8 + 2) / 3 + 1;
    }
    // Tile `number`; false (all lanes) if the offsets, which nobody has checked, do not add up to one.
    __device__ __forceinline__ bool tile(int number, ExpertTile& out, int& tile_n)
    {
        const int n = n_tiles;
        const int l = seek([&](int upto, int) { return upto * n > number; });
        if (l < 0) return false;
        const int mine = __builtin_amdgcn_readlane(tiles, l);
        const int place = number - (tiles_before + __builtin_amdgcn_readlane(tiles_upto, l) - mine) * n;
        if (mine <= 0 || place < 0 || place / n >= mine) return false;
        tile_n = place / mine;
        out.tiles = mine;
        out.index = place % mine;
        out.expert = e0 + l;
        out.row0 = __builtin_amdgcn_readlane(first, l) + out.index * height;
        out.end = __builtin_amdgcn_readlane(end, l);
        return true;
    }
};

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
