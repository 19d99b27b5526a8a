// Gradient with respect to the scale vectors of tokens sorted by expert.  Both modes are sums of
//   D_e = dY_e^T X_e   [d_out, d_in]   (the products of the tokens of expert e)
// with the signs:  row  grad[e, o] = sum_i B_e[o, i] D_e[o, i],   col  grad[e, i] = sum_o B_e[o, i] D_e[o, i].
// D is formed tile by tile on the matrix cores in the operands' own format (exact products, fp32 sums) and never written:
// the signs meet it in the accumulators, so they are read once for every expert that has tokens, and its few tokens are
// all that the contraction runs over.  Bound by the matrix cores: 2048 tokens x 2 of 8 experts, 14336 x 4096 bf16 column in 505 to 540 us, 890
// to 950 TFLOP/s or 60 % of a large library product, the cores 48 % busy at clocks that power limits; 1.3 GB from memory.  The dimension
// that is summed over is the accumulator's row dimension, the other one its columns: a lane adds its own elements, and two lanes meet once.
#include <algorithm>

#include "pdelta_experts.h"
#include "pdelta_host.h"
#include "pdelta_lds_load.h"

namespace pdelta {

template <int DT>
__device__ __forceinline__ float16v mfma32(uint4v a, uint4v b, float16v c)
{
    if constexpr (DT == kBF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// Tiles of 256 of the summed dimension (P) x 256 of the kept one (Q), 8 waves of 128 x 64, steps of 64 tokens, two stages in
// LDS filled by direct loads.  Both operands lie in memory with the tokens as rows, and the contraction runs over the tokens:
// the fragments are read from LDS by transposing reads, 4 tokens x 16 columns for 16 lanes.
constexpr int kGradTile = 256, kGradTokens = 64;
constexpr int kGradOperand = kGradTokens * kGradTile * 2, kGradStage = 2 * kGradOperand, kGradLds = 2 * kGradStage + 8192 + 2048;

// A workgroup takes `run` tiles of the summed dimension one after another, at one place of the kept one: its loads go on over the
// tiles' ends, where it would otherwise wait for the first ones of the next with nothing to multiply, and the kept sums stay in
// registers.
template <int DT, int AXIS>
__global__ void __launch_bounds__(512, 2)
experts_grad_kernel(const uint16_t* __restrict__ X, int x_ld, const uint16_t* __restrict__ dY, int y_ld, const int* __restrict__ offsets,
                    const uint32_t* __restrict__ B_packed, float* __restrict__ partial, int M, int d_out, int d_in, int kept_tiles,
                    int sum_tiles, int run, int runs)
{
    constexpr int FP = 4, FQ = 2;
    extern __shared__ __attribute__((aligned(16))) unsigned char grad_smem[];
    const int kt = blockIdx.x % kept_tiles, rt = blockIdx.x / kept_tiles % runs, e = blockIdx.x / kept_tiles / runs;
    int first, end;
    expert_rows(offsets, e, M, first, end);
    const int dP = AXIS == 0 ? d_in : d_out, dQ = AXIS == 0 ? d_out : d_in;
    if (first == end) {                               // whole workgroup
        const int q = kt * kGradTile + threadIdx.x;   // one run: these are the gradients
        if (runs == 1 && threadIdx.x < kGradTile && q < dQ) partial[(int64_t)e * dQ + q] = 0.f;
        return;
    }
    const int p_ld = AXIS == 0 ? x_ld : y_ld, q_ld = AXIS == 0 ? y_ld : x_ld;
    const int q0 = kt * kGradTile, words = d_in / 32, first_tile = rt * run, tiles = min(run, sum_tiles - first_tile);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wp = wave >> 2, wq = wave & 3;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)grad_smem;
    const uint32_t* signs = B_packed + (int64_t)e * d_out * words;

    // One load instruction brings 512 bytes of two tokens; a wave brings 8 tokens of each operand.  The 16-byte piece c of token t
    // goes to place c ^ 4 (t & 3), so that the four tokens of a transposing read are in different banks.
    const char* pbase = (const char*)((AXIS == 0 ? X : dY) + (int64_t)first * p_ld);
    const char* qbase = (const char*)((AXIS == 0 ? dY : X) + (int64_t)first * q_ld);
    int piece[2];
    uint32_t qcol[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        piece[q] = ((lane & 31) ^ ((q * 2 + (lane >> 5)) << 2)) * 8;
        qcol[q] = (uint32_t)min(q0 + piece[q], (dQ - 1) / 8 * 8) * 2u;
    }
    const int tok = wave * 8 + (lane >> 5), n = end - first, n_steps = (n + kGradTokens - 1) / kGradTokens;
    int asked_tile = 0, asked_step = 0;               // what is asked for next
    auto request = [&](uint32_t stage) {
        const int most = n - 1 - asked_step * kGradTokens;        // rows behind the expert's last repeat it
        const char* pb = pbase + (int64_t)asked_step * kGradTokens * p_ld * 2;
        const char* qb = qbase + (int64_t)asked_step * kGradTokens * q_ld * 2;
        const int p0 = (first_tile + asked_tile) * kGradTile;
        uint32_t pcol[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) pcol[q] = (uint32_t)min(p0 + piece[q], (dP - 1) / 8 * 8) * 2u;
        if (wave * 8 <= (most | 15)) {                // (a wave whose tokens are behind the last ones' 16 has nothing to bring)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t row = (uint32_t)min(tok + q * 2, most);
                load_lds_16(lds0 + stage + (wave * 4 + q) * 1024, row * (uint32_t)p_ld * 2u + pcol[q & 1], pb);
                load_lds_16(lds0 + stage + kGradOperand + (wave * 4 + q) * 1024, row * (uint32_t)q_ld * 2u + qcol[q & 1], qb);
            }
        }
        if (++asked_step == n_steps) {
            asked_step = 0;
            ++asked_tile;
        }
    };
    // Zeros for tokens behind the expert's last and for what is summed over behind its end.  (What the wave has loaded itself: nothing
    // but its own loads has to be waited for.)
    auto clear_behind = [&](int tile, int s, uint32_t stage) {
        const int p0 = (first_tile + tile) * kGradTile;
        if ((s + 1) * kGradTokens <= n && p0 + kGradTile <= dP) return;       // uniform
        if (wave * 8 > ((n - 1 - s * kGradTokens) | 15)) return;              // these tokens are not multiplied
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const bool none = s * kGradTokens + tok + q * 2 >= n;
            if (none || p0 + piece[q & 1] >= dP)
                *(uint4v*)(grad_smem + stage + (wave * 4 + q) * 1024 + lane * 16) = (uint4v){0, 0, 0, 0};
            if (none) *(uint4v*)(grad_smem + stage + kGradOperand + (wave * 4 + q) * 1024 + lane * 16) = (uint4v){0, 0, 0, 0};
        }
    };

    // The signs of a tile.  Row mode (P are inputs, Q outputs): the lane's output row h holds the wave's 128 inputs in four words.
    // Column mode: a thread brings half a row of the tile to LDS.
    uint32_t sw[AXIS == 0 ? FQ : 1][FP];
    auto load_signs = [&](int p0) {
        if constexpr (AXIS == 0) {
#pragma unroll
            for (int h = 0; h < FQ; ++h)
#pragma unroll
                for (int f = 0; f < FP; ++f)
                    sw[h][f] = signs[(int64_t)min(q0 + wq * 64 + h * 32 + (lane & 31), d_out - 1) * words + min(p0 / 32 + wp * 4 + f, words - 1)];
        } else {
#pragma unroll
            for (int f = 0; f < FP; ++f)
                sw[0][f] = signs[(int64_t)min(p0 + (int)threadIdx.x / 2, d_out - 1) * words + min(q0 / 32 + ((int)threadIdx.x & 1) * 4 + f, words - 1)];
        }
    };
    uint32_t* tile_signs = (uint32_t*)(grad_smem + 2 * kGradStage);   // column mode: [256][8]
    float* red = (float*)(grad_smem + 2 * kGradStage + 8192);         // [2][256]

    float16v acc[FP][FQ];
    float sum[FQ] = {0.f, 0.f}, tile_sum[FQ];         // of the run, and of one of its tiles: 64 additions, then one for each tile

    // this lane's part of a transposing read: token (lane / 32) * 8 + lane % 16 / 4, columns (lane / 16 % 2) * 16 + lane % 4 * 4; 32
    // columns further is 64 bytes, exclusive or with the place's own bits
    const int tr = (lane & 15) >> 2;
    const uint32_t row_at = (uint32_t)((lane >> 5) * 8 + tr) * 512u, col_at = (uint32_t)(((lane >> 4) & 1) * 32 + (lane & 3) * 8);
    uint32_t p_at[FP], q_at[FQ];
#pragma unroll
    for (int f = 0; f < FP; ++f) p_at[f] = row_at + ((uint32_t)(wp * 256 + f * 64 + col_at) ^ (uint32_t)(tr << 6));
#pragma unroll
    for (int h = 0; h < FQ; ++h) q_at[h] = kGradOperand + row_at + ((uint32_t)(wq * 128 + h * 64 + col_at) ^ (uint32_t)(tr << 6));
    uint4v a[2][FP], b[2][FQ];
    auto read_one = [&](uint32_t at) {
        const uint2v lo = read_transposed(grad_smem + at), hi = read_transposed(grad_smem + at + 4 * 512);
        return (uint4v){lo[0], lo[1], hi[0], hi[1]};
    };
    auto read_frags = [&](uint32_t stage, int ks) {
#pragma unroll
        for (int h = 0; h < FQ; ++h) b[ks & 1][h] = read_one(stage + ks * 16 * 512 + q_at[h]);
#pragma unroll
        for (int f = 0; f < FP; ++f) a[ks & 1][f] = read_one(stage + ks * 16 * 512 + p_at[f]);
    };
    auto multiply = [&](int ks) {
#pragma unroll
        for (int f = 0; f < FP; ++f)
#pragma unroll
            for (int h = 0; h < FQ; ++h) acc[f][h] = mfma32<DT>(a[ks & 1][f], b[ks & 1][h], acc[f][h]);
    };

    // 32x32 accumulator: element r of lane l is row (r/4)*8 + (l/32)*4 + r%4, column l%32
    auto add = [&](int h, float x, uint32_t word, int left) {     // +-x by the bit that `left` brings to the top
        const uint32_t one = ((word << left) & 0x80000000u) ^ 0xBF800000u;
        tile_sum[h] = __builtin_fmaf(x, __builtin_bit_cast(float, one), tile_sum[h]);
    };
    auto add_tile = [&]() {
#pragma unroll
        for (int h = 0; h < FQ; ++h) tile_sum[h] = 0.f;
        if constexpr (AXIS == 0) {
#pragma unroll
            for (int f = 0; f < FP; ++f)
#pragma unroll
                for (int h = 0; h < FQ; ++h) {
                    const uint32_t word = sw[h][f] >> ((lane >> 5) * 4);          // the lane's rows are bits 0-3, 8-11, 16-19, 24-27
#pragma unroll
                    for (int r = 0; r < 16; ++r) add(h, acc[f][h][r], word, 31 - ((r >> 2) * 8 + (r & 3)));
                }
        } else {
            lds_barrier();                            // all of the tile's signs are in LDS
            const uint32_t* mine = tile_signs + (wp * 128 + (lane >> 5) * 4) * 8 + wq * 2;
#pragma unroll
            for (int f = 0; f < FP; ++f) {
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const uint2v w = *(const uint2v*)(mine + (f * 32 + (r >> 2) * 8 + (r & 3)) * 8);
#pragma unroll
                    for (int h = 0; h < FQ; ++h) {
                        const uint32_t wh = w[h];
                        add(h, acc[f][h][r], wh, 31 - (lane & 31));
                    }
                }
                __builtin_amdgcn_sched_barrier(0);    // (else all of the words are read at once, into registers that are not there)
            }
        }
#pragma unroll
        for (int h = 0; h < FQ; ++h) sum[h] += tile_sum[h];
    };

    // Step `now` of all the tiles' steps, step s of its tile.  The barrier is three quarters into it: by then every wave has read its
    // last fragments of this step's stage, which the loads of step now + 2 may fill, and has the next step's loads.
    const int all = tiles * n_steps;
    int tile = 0, s = 0;
    auto step = [&](int now, uint32_t cur, uint32_t nxt) {
        if (s == 0) {
            load_signs((first_tile + tile) * kGradTile);
#pragma unroll
            for (int f = 0; f < FP; ++f)
#pragma unroll
                for (int h = 0; h < FQ; ++h)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[f][h][r] = 0.f;
        }
        const int left = n - s * kGradTokens;         // 16 tokens for each quarter of a step: the last one may have fewer quarters
        if (left > 16) read_frags(cur, 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(0);
        __builtin_amdgcn_sched_barrier(0);
        if (left > 16) {
            if (left > 32) read_frags(cur, 2);
            __builtin_amdgcn_sched_barrier(0);
            multiply(1);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (left > 32) {
            if (left > 48) read_frags(cur, 3);
            __builtin_amdgcn_sched_barrier(0);
            multiply(2);
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_loads<0>();
#pragma unroll
        for (int h = 0; h < (AXIS == 0 ? FQ : 1); ++h)            // (a use of the signs where all loads have been waited for anyway)
#pragma unroll
            for (int f = 0; f < FP; ++f) asm volatile("" : "+v"(sw[h][f]));
        const int after = s + 1 == n_steps ? 0 : s + 1;
        if (now + 1 < all) clear_behind(after == 0 ? tile + 1 : tile, after, nxt);
        lds_barrier();
        if (now + 1 < all) read_frags(nxt, 0);
        if (AXIS == 1 && s == 0) *(uint4v*)(tile_signs + threadIdx.x * 4) = (uint4v){sw[0][0], sw[0][1], sw[0][2], sw[0][3]};
        if (now + 2 < all) request(cur);
        __builtin_amdgcn_sched_barrier(0);
        if (left > 48) multiply(3);
        __builtin_amdgcn_sched_barrier(0);
        if (after == 0) {
            add_tile();
            ++tile;
        }
        s = after;
    };
    request(0);
    wait_loads<0>();
    clear_behind(0, 0, 0);
    lds_barrier();
    if (all > 1) request(kGradStage);
    read_frags(0, 0);
    for (int now = 0; now < all; now += 2) {
        step(now, 0, kGradStage);
        if (now + 1 < all) step(now + 1, kGradStage, 0);
    }

#pragma unroll
    for (int h = 0; h < FQ; ++h) {
        sum[h] += __shfl_xor(sum[h], 32, kWave);
        if (lane < 32) red[wp * kGradTile + wq * 64 + h * 32 + lane] = sum[h];
    }
    __syncthreads();
    const int q = threadIdx.x;
    if (q < kGradTile && q0 + q < dQ) partial[((int64_t)e * runs + rt) * dQ + q0 + q] = red[q] + red[kGradTile + q];
}

// The sums of the runs of one expert, in their order.
__global__ void __launch_bounds__(256)
experts_grad_sum_kernel(const float* __restrict__ partial, const int* __restrict__ offsets, float* __restrict__ grad, int M, int dQ,
                        int runs, int blocks)
{
    const int e = blockIdx.x / blocks, q = (blockIdx.x % blocks) * 256 + threadIdx.x;
    int first, end;
    expert_rows(offsets, e, M, first, end);
    if (q >= dQ) return;
    float sum = 0.f;
    if (first < end)
#pragma unroll 8
        for (int s = 0; s < runs; ++s) sum += partial[((int64_t)e * runs + s) * dQ + q];
    grad[(int64_t)e * dQ + q] = sum;
}

// Tiles that a workgroup takes: as many as leave eight rounds of 256 workgroups where the tiles are long (experts differ in their
// tokens, and the longest run is waited for in the end), one where they are a step.
static int tiles_in_a_run(int64_t M, int64_t E, int64_t kept, int64_t summed)
{
    const int64_t met = std::max<int64_t>(1, std::min(E, M)), steps = (M + met * kGradTokens - 1) / (met * kGradTokens);
    const int64_t tiles = met * ((kept + kGradTile - 1) / kGradTile) * ((summed + kGradTile - 1) / kGradTile);
    return (int)std::max<int64_t>(1, std::min<int64_t>(8, tiles / 256 / std::max<int64_t>(1, std::min<int64_t>(8, steps))));
}
static int64_t grad_runs(int64_t M, int64_t E, int64_t kept, int64_t summed)
{
    const int64_t tiles = (summed + kGradTile - 1) / kGradTile, run = tiles_in_a_run(M, E, kept, summed);
    return (tiles + run - 1) / run;
}

// dY with rows that are no multiple of 16 bytes is copied into rows that are, behind the runs' sums.
static int64_t sums_bytes(int64_t M, int64_t E, int64_t kept, int64_t summed)
{
    const int64_t runs = grad_runs(M, E, kept, summed);
    return runs == 1 ? 0 : (E * runs * kept * 4 + 15) / 16 * 16;
}

size_t experts_grad_v_workspace_bytes(int64_t M, int64_t E, int64_t d_out, int64_t d_in, int axis)
{
    const int64_t rows = (d_out & 7) != 0 ? M * experts_padded(d_out) * 2 : 0;
    return (size_t)(sums_bytes(M, E, axis == 0 ? d_out : d_in, axis == 0 ? d_in : d_out) + rows);
}

template <int DT, int AXIS>
static int launch_grad(const void* X, const void* dY, const int* offsets, const uint32_t* B_packed, float* grad, int64_t M, int64_t E,
                       int64_t d_out, int64_t d_in, void* workspace, hipStream_t stream)
{
    const int64_t kept = AXIS == 0 ? d_out : d_in, summed = AXIS == 0 ? d_in : d_out;
    const int64_t kept_tiles = (kept + kGradTile - 1) / kGradTile, sum_tiles = (summed + kGradTile - 1) / kGradTile;
    const int64_t sum_blocks = (kept + 255) / 256;
    const int64_t runs = grad_runs(M, E, kept, summed);
    if (E * kept_tiles * runs > 0x7FFFFFFF || E * sum_blocks > 0x7FFFFFFF) return -2;
    auto kernel = experts_grad_kernel<DT, AXIS>;
    static unsigned lds_opted_in = 0;                 // per template instance: one kernel
    if (opt_in_dynamic_lds((const void*)kernel, kGradLds, &lds_opted_in) != 0) return -1;
    int64_t y_ld = d_out;
    float* sums = runs == 1 ? grad : (float*)workspace;
    if (M > 0) {
        if ((d_out & 7) != 0) {
            void* rows = (char*)workspace + sums_bytes(M, E, kept, summed);
            y_ld = experts_padded(d_out);
            launch_experts_copy_rows(dY, rows, M, d_out, stream);
            dY = rows;
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)(E * kept_tiles * runs)), dim3(512), kGradLds, stream, (const uint16_t*)X, (int)d_in,
                           (const uint16_t*)dY, (int)y_ld, offsets, B_packed, sums, (int)M, (int)d_out, (int)d_in,
                           (int)kept_tiles, (int)sum_tiles, tiles_in_a_run(M, E, kept, summed), (int)runs);
    }
    if (M == 0 || runs > 1)
        hipLaunchKernelGGL(experts_grad_sum_kernel, dim3((unsigned)(E * sum_blocks)), dim3(256), 0, stream, (const float*)workspace, offsets,
                           grad, (int)M, (int)kept, (int)runs, (int)sum_blocks);
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
