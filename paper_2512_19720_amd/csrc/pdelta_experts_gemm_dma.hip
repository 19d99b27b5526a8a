// Products of tokens sorted by expert with W_hat (forward) or its transpose (GRAD) on tiles of up to 256 tokens x 256 outputs x 64
// of the contraction, 8 waves.  The arithmetic is that of pdelta_experts_gemm.hip.  Tokens, signs and scales come by direct loads into
// LDS; W_b comes through registers and goes to LDS as W_hat, between the matrix instructions of the step before; one barrier per step,
// three quarters into it, which publishes step s + 1 and frees the stages of step s.
//
// What bounds it: full tiles of one expert (2048 tokens, 8192 x 4096 fp16, one round of 256 tiles) take 140 to 147 us, 930 to 980 TFLOP/s, three
// quarters of what a library product of these sizes reaches (106 us), the matrix cores busy 56 % of the time at clocks that power
// limits (1.4 to 1.7 GHz).  Uneven experts lose more: 2048 tokens x 2 of 8 experts, 14336 x 4096 bf16, 680 TFLOP/s: 8 % of the tiles' rows are no tokens, the
// busiest CUs work half a tile longer than the others, and bf16 weights cost 10 % for their conversion (matrix cores 50 % busy).  HBM
// is not it: 1.8 GB in 700 us.
//
// The tokens come as fp16 rows of a multiple of 128 values (prepared ones, or X and dY themselves); forward, the signs as rows of a
// multiple of 16 bytes.
//
// Forward: a tile of W_hat is 256 output rows x 64 inputs; both operands' fragments are 16 consecutive bytes of a row.
// GRAD: it is 64 output rows x 256 inputs, as it lies in memory, and the contraction runs over the rows: fragments are read by
// transposing LDS reads, 4 rows x 16 columns for 16 lanes.  Nothing is transposed in memory, and the signs and scales are those of
// the forward layout.
//
// Workgroup -> tile: see ExpertTiles; XCD w % 8, and there tile w / 8 of its range.
#include <algorithm>
#include <type_traits>

#include "pdelta_experts.h"
#include "pdelta_gemm_tile.h"
#include "pdelta_host.h"
#include "pdelta_lds_load.h"

namespace pdelta {

constexpr int kTileM = 256, kTileN = 256, kTileK = 64;
constexpr int kWBytes = kTileN * kTileK * 2;          // W_b in a stage
// behind the stages: a wave's signs (2 KB: forward, its 32 rows for two groups of four steps; GRAD, its 8 rows of 256 inputs for
// four steps), and its scales (1 KB: forward column mode, v for two groups of four steps; GRAD row mode, its 8 rows' for four)
constexpr int kTileW = 2 * kTileM * kTileK * 2, kTileSigns = kTileW + 2 * kWBytes, kTileScales = kTileSigns + 8 * 2048, kTileLds = kTileScales + 8 * 1024;

// The wave tile's outputs one by one, columns in 128-byte pieces of a row: 16-bit outputs whose rows are no multiple of 16 bytes, fp32
// ones and the parts' sums (rows `pitch` apart).  A row's address is scalar, the lane's place in it one register; rows behind
// `end` and columns behind N are left out.
template <int YDT, int FM>
__device__ __forceinline__ void store_rows(const float16v (&acc)[FM][2], void* Y, int64_t pitch, int m0, int n0, int end, int N, int lane)
{
    constexpr int SIZE = YDT == kF32 ? 4 : 2;
    const int low = (lane >> 5) * 4;
    const uint32_t at = (uint32_t)((int64_t)low * pitch + (lane & 31)) * (uint32_t)SIZE;          // pitch <= 2^22 + 255
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = m0 + f * 32 + (r >> 2) * 8 + (r & 3);
            char* const base = (char*)Y + ((int64_t)row * pitch + n0) * SIZE;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (row + low < end && n0 + h * 32 + (lane & 31) < N) {
                    const float x = acc[f][h][r];
                    char* const p = base + h * 32 * SIZE + at;
                    if constexpr (YDT == kF32) *(float*)p = x;
                    else *(uint16_t*)p = (uint16_t)(YDT == kBF16 ? f32_to_bf16_bits(x) : f32_to_f16_bits(x));
                }
        }
}

struct TileArgs {
    const uint16_t* A;
    int lda;
    const float* inverse;
    const uint16_t* W_b;
    int64_t w_stride;
    const uint32_t* B_packed;
    const uint16_t* v;
    void* Y;
    float* partial;
    int M, d_out, d_in, y_dtype, parts, sign_ld, pitch;     // bytes from one output row's signs to the next; values of a row of the parts' sums
};

// One tile of 64 FM tokens, waves of 32 FM x 64 outputs.
template <int WDT, int AXIS, bool GRAD, int FM>
__device__ __forceinline__ void experts_tile(const TileArgs& g, const ExpertTile& t, int tile_n, int part, unsigned char* tile_smem)
{
    constexpr int BM = FM * 64, FN = 2, AQ = FM;      // tokens; MFMA tiles of a wave along outputs; load instructions of a wave for the tokens
    // Up to 128 tokens four steps of tokens are on their way in LDS and four of W_b in registers: a step is then shorter than the
    // memory's latency.  Larger tiles: two, and as many steps of W_b as there are registers free.
    constexpr bool DEEP = FM <= 2;
    constexpr int STEPS = DEEP ? 4 : 2, AHEAD = DEEP ? 4 : FM == 3 && (GRAD || AXIS == 0) ? 2 : 1;
    constexpr int AB = BM * kTileK * 2;
    auto a_stage = [](int s) { return (uint32_t)(s % STEPS * AB); };
    auto w_stage = [](int s) { return (uint32_t)(kTileW + s % 2 * kWBytes); };
    const uint16_t *A = g.A, *v = g.v;
    // (a part leaves its sums as they are; experts_sum_kernel does the rest)
    const float* inverse = g.parts > 1 ? nullptr : g.inverse;
    const int lda = g.lda, d_out = g.d_out, d_in = g.d_in, y_dtype = g.parts > 1 ? kF32 : g.y_dtype;
    void* Y = g.parts > 1 ? (void*)(g.partial + (int64_t)part * g.M * g.pitch) : g.Y;
    const int N = GRAD ? d_in : d_out;
    const int n0 = tile_n * kTileN;
    // the steps of this part of the contraction: an even number of them, at least 2
    const int first_step = (int)((int64_t)(lda / kTileK / 2) * part / g.parts) * 2;
    const int n_steps = (int)((int64_t)(lda / kTileK / 2) * (part + 1) / g.parts) * 2 - first_step;
    const uint16_t* W = g.W_b + t.expert * g.w_stride;
    const char* B = (const char*)g.B_packed + (int64_t)t.expert * d_out * g.sign_ld;
    const uint16_t* scales = v + (int64_t)t.expert * (AXIS == 0 ? d_out : d_in);

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave >> 2, wn = wave & 3;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char*)tile_smem;

    // Tokens: a load instruction covers 8 rows of 128 bytes; the 16-byte piece p of row r holds values 8 (p ^ ((r >> 1) & 7)) .. +7.
    // Rows behind the expert's last one repeat it (they feed outputs that are never stored).
    const char* abase = (const char*)(A + (int64_t)t.row0 * lda);
    uint32_t aoff[AQ], piece[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) piece[q] = (uint32_t)((lane & 7) ^ (q * 4 + (lane >> 4)));
#pragma unroll
    for (int q = 0; q < AQ; ++q)
        aoff[q] = (uint32_t)(min(t.row0 + wave * (BM / 8) + q * 8 + (lane >> 3), t.end - 1) - t.row0) * (uint32_t)lda * 2u +
                  (uint32_t)((lane & 7) ^ (((wave * FM + q) & 1) * 4 + (lane >> 4))) * 16u;

    // W_b.  Forward: the same for the tile's 256 output rows.  GRAD: a load instruction covers 512 bytes of two rows; the piece c of
    // row r is at place c ^ 4 (r & 3), which puts the four rows of a transposing read into different banks.
    const char* wbase;
    const char* sbase;
    uint32_t woff[4], soff, chunk[2];
    uint32_t vrow[4];                                 // forward row mode: the scale of the wave's rows
    uint4v vcol[2];                                   // GRAD column mode: the scales of the lane's inputs
    if constexpr (GRAD) {
        wbase = (const char*)W;
        sbase = B;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            chunk[q] = (uint32_t)((lane & 31) ^ ((q * 2 + (lane >> 5)) << 2));
            const int col = min(n0 + (int)chunk[q] * 8, d_in - 8);
            woff[q] = (uint32_t)col * 2u;
            if constexpr (AXIS == 1) vcol[q] = *(const uint4v*)(scales + col);
        }
        soff = (uint32_t)min(n0 / 32 + (lane & 7), d_in / 32 - 1) * 4u;
    } else {
        wbase = (const char*)(W + (int64_t)n0 * d_in);
        sbase = B + (int64_t)n0 * g.sign_ld;
#pragma unroll
        for (int q = 0; q < 2; ++q) chunk[q] = piece[q];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int row = min(n0 + wave * 32 + q * 8 + (lane >> 3), d_out - 1) - n0;
            woff[q] = (uint32_t)row * (uint32_t)d_in * 2u;
            if constexpr (AXIS == 0) vrow[q] = (uint32_t)scales[n0 + row] * 0x10001u;
        }
        // lanes 0-31: sign words of the wave's rows for two steps, lanes 32-63 for the next two
        soff = (uint32_t)(min(n0 + wave * 32 + (lane & 31), d_out - 1) - n0) * (uint32_t)g.sign_ld;
    }

    // Where step s is in the contraction.  Forward, with one token tile: the output tiles start at different places of d_in, since rows
    // of W_b are often a power of two apart and the same inputs of all rows then in few of the memory's channels (16 experts of 64
    // tokens, 4096 x 4096 fp16: 138 -> 117 us).  With more of them, or one base for all experts, the weights or tokens that workgroups
    // share are better read by all at once (2048 tokens of one expert, 8192 x 4096: 131 and 135; 1501 of 12 fine-tunes: 118 and 122).
    const int start = GRAD || t.tiles > 1 || g.w_stride == 0 ? 0 : (tile_n + t.expert * 5) * 6 % n_steps / 2 * 2;
    auto place = [&](int s) {
        if constexpr (GRAD) return first_step + s;
        s += start;
        return first_step + (s >= n_steps ? s - n_steps : s);
    };
    // Signs and scales.  Forward: for the four steps from s on (a row's last 16 bytes again behind its end).
    const uint32_t my_signs = lds0 + kTileSigns + wave * 2048, my_scales = lds0 + kTileScales + wave * 1024;
    auto request_signs = [&](int s) {
        if constexpr (GRAD) {
            const int kb = place(s) * kTileK, k0 = min(kb, d_out - 1);        // rows behind the last one repeat it: the tokens are zero there
            auto row = [&](int r) { return (uint32_t)(min(kb + r, d_out - 1) - k0); };
            load_lds_4(my_signs + (s & 3) * 256, row(wave * 8 + (lane >> 3)) * (uint32_t)g.sign_ld + soff, sbase + (int64_t)k0 * g.sign_ld);
            if constexpr (AXIS == 0)
                if (lane < 8) load_lds_2(my_scales + (s & 3) * 32, row(wave * 8 + lane) * 2u, scales + k0);
        } else {
            const int group = (s >> 2) & 1;
            load_lds_16(my_signs + group * 1024, soff + (uint32_t)place(min(s + (lane >> 5) * 2, n_steps - 2)) * 8u, sbase);
            if constexpr (AXIS == 1)
                if (lane < 32) load_lds_16(my_scales + group * 512, (uint32_t)min(place(min(s + (lane >> 3), n_steps - 1)) * 64 + (lane & 7) * 8, d_in - 8) * 2u, scales);
        }
    };
    auto request_a = [&](int s, uint32_t stage) {
#pragma unroll
        for (int q = 0; q < AQ; ++q) load_lds_16(lds0 + stage + (wave * AQ + q) * 1024, aoff[q], abase + (int64_t)place(s) * (kTileK * 2));
    };
    // W_b goes through registers, AHEAD steps of it: it comes out of HBM, and with loads into the two LDS stages, which are free for
    // half a step only, a step took twice the memory's latency (16 experts of 64 tokens, 4096 x 4096 fp16, input gradient: 123 -> 96 us).
    uint4v raw[AHEAD][4];
    auto request_w = [&](int s, auto which) {
        uint4v(&into)[4] = raw[decltype(which)::value % AHEAD];
        if constexpr (GRAD) {
            const int kb = place(s) * kTileK, k0 = min(kb, d_out - 1);
            const char* base = wbase + (int64_t)k0 * d_in * 2;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                into[q] = *(const uint4v*)(base + ((uint32_t)(min(kb + wave * 8 + q * 2 + (lane >> 5), d_out - 1) - k0) * (uint32_t)d_in * 2u + woff[q & 1]));
        } else {
            const int kb = place(s) * kTileK;             // inputs behind the last ones repeat them: the tokens are zero there
            uint32_t col[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) col[q] = (uint32_t)min(kb + (int)chunk[q] * 8, d_in - 8) * 2u;
#pragma unroll
            for (int q = 0; q < 4; ++q) into[q] = *(const uint4v*)(wbase + (woff[q] + col[q & 1]));
        }
    };

    // The lane's pieces of W_b -> W_hat in LDS.
    uint4v wvec[2];
    uint32_t sbyte[4], wscale[4];
    auto fetch_signs = [&](int s) {
        const unsigned char* sg = tile_smem + kTileSigns + wave * 2048 + (GRAD ? (s & 3) * 256 : ((s >> 2) & 1) * 1024);
        const unsigned char* sc = tile_smem + kTileScales + wave * 1024 + (GRAD ? (s & 3) * 32 : ((s >> 2) & 1) * 512);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (GRAD) {
                sbyte[q] = sg[(q * 2 + (lane >> 5)) * 32 + chunk[q & 1]];
                if constexpr (AXIS == 0) wscale[q] = *(const uint16_t*)(sc + (q * 2 + (lane >> 5)) * 4);
            } else {
                sbyte[q] = sg[((s >> 1) & 1) * 512 + (s & 1) * 8 + (q * 8 + (lane >> 3)) * 16 + chunk[q & 1]];
            }
        }
        if constexpr (!GRAD && AXIS == 1) {
#pragma unroll
            for (int q = 0; q < 2; ++q) wvec[q] = *(const uint4v*)(sc + (s & 3) * 128 + chunk[q] * 16);
        }
    };
    auto convert_w = [&](uint32_t stage, auto which) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t minus = ~sbyte[q] & 0xFFu;
            uint32_t y = minus | (minus << 15);       // bit 2p + 1 at 2p + 16
            asm("" : "+v"(y));                        // (else y and its shifts become full multiplications)
            uint32_t vv = 0;
            if constexpr (AXIS == 0) vv = GRAD ? wscale[q] | (wscale[q] << 16) : vrow[q];
            const uint4v w16 = to_f16x8<WDT>(raw[decltype(which)::value % AHEAD][q]);
            uint4v r;
#pragma unroll
            for (int p = 0; p < 4; ++p) {
                uint32_t vp = vv;
                if constexpr (AXIS == 1) vp = GRAD ? vcol[q & 1][p] : wvec[q & 1][p];
                const uint32_t wp = w16[p], sv = ((y << (15 - 2 * p)) & 0x80008000u) ^ vp;      // -v where the bit is set
                r[p] = as_u32(as_half2(wp) + as_half2(sv));
            }
            *(uint4v*)(tile_smem + stage + (wave * 4 + q) * 1024 + lane * 16) = r;
        }
    };

    float16v acc[FM][FN];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int h = 0; h < FN; ++h)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[f][h][r] = 0.f;

    // this lane's piece of 16 values ks of a row is at byte frag ^ (32 ks)
    const uint32_t frag = (uint32_t)((lane & 31) * 128 + (((lane >> 5) ^ ((lane >> 1) & 7)) * 16));
    // GRAD: row (lane / 32) * 8 + lane % 16 / 4, columns (lane / 16 % 2) * 16 + lane % 4 * 4; 32 columns further: exclusive or 64
    const int tr = (lane & 15) >> 2;
    const uint32_t tfrag = (uint32_t)((lane >> 5) * 8 + tr) * 512u +
                           ((uint32_t)(wn * 128 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8) ^ (uint32_t)(tr << 6));
    half8 a[2][FM], b[2][FN];
    auto read_frags = [&](uint32_t as, uint32_t ws, auto step16) {
        constexpr int ks = decltype(step16)::value;
        uint32_t at = frag ^ (uint32_t)(ks * 32);
        // (where registers are short: computed here, not kept)
        if constexpr (FM == 4 && AXIS == 1 && !GRAD) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(at) : "n"(ks * 32), "v"(frag));
        const unsigned char* xa = tile_smem + as + wm * (BM / 2) * 128 + at;
#pragma unroll
        for (int h = 0; h < FN; ++h) {
            if constexpr (GRAD) {
                const unsigned char* p = tile_smem + ws + ks * 16 * 512 + (tfrag ^ (uint32_t)(h * 64));
                const uint2v lo = read_transposed(p), hi = read_transposed(p + 4 * 512);
                b[ks & 1][h] = __builtin_bit_cast(half8, (uint4v){lo[0], lo[1], hi[0], hi[1]});
            } else {
                b[ks & 1][h] = *(const half8*)(tile_smem + ws + wn * 64 * 128 + at + h * 32 * 128);
            }
        }
#pragma unroll
        for (int f = 0; f < FM; ++f) a[ks & 1][f] = *(const half8*)(xa + f * 32 * 128);
    };
    auto multiply = [&](int ks) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int h = 0; h < FN; ++h)
                acc[f][h] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[ks & 1][f], b[ks & 1][h], acc[f][h], 0, 0, 0);
    };

    using I0 = std::integral_constant<int, 0>;
    using I1 = std::integral_constant<int, 1>;
    using I2 = std::integral_constant<int, 2>;
    using I3 = std::integral_constant<int, 3>;
    const int last = n_steps - 1;

    // The fences keep the LDS reads above the MFMAs, the conversion between them, and the loads in their order: a wait counts the
    // loads asked for since.
    if constexpr (DEEP) {
        // The first loads of all four steps.  Behind the last step the last one's are asked for again, into places that nobody reads.
        request_signs(0);
        if constexpr (GRAD) {
#pragma unroll
            for (int k = 1; k < 4; ++k) request_signs(k);
        }
        auto first = [&](auto k) {
            request_a(min((int)decltype(k)::value, last), a_stage(decltype(k)::value));
            __builtin_amdgcn_sched_barrier(0);
            request_w(min((int)decltype(k)::value, last), k);
            __builtin_amdgcn_sched_barrier(0);
        };
        first(I0{});
        first(I1{});
        first(I2{});
        first(I3{});
        wait_loads<0>();
        fetch_signs(0);
        convert_w(w_stage(0), I0{});
        lds_barrier();
        request_w(min(4, last), I0{});
        read_frags(a_stage(0), w_stage(0), I0{});

        // Step s, s % 4 = P.  In its last quarter the signs and the tokens of step s + 4 and W_b of step s + 5 are asked for; what the
        // next step needs is then behind at least three steps' W_b, 12 loads.
        auto step = [&](int s, auto phase) {
            constexpr int P = decltype(phase)::value;
            using Next = std::integral_constant<int, (P + 1) % 4>;
            read_frags(a_stage(P), w_stage(P), I1{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            wait_loads<12>();
            fetch_signs(s + 1);
            read_frags(a_stage(P), w_stage(P), I2{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(1);
            convert_w(w_stage(P + 1), Next{});
            __builtin_amdgcn_sched_barrier(0);
            read_frags(a_stage(P), w_stage(P), I3{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(2);
            __builtin_amdgcn_sched_barrier(0);
            lds_barrier();
            read_frags(a_stage(P + 1), w_stage(P + 1), I0{});
            if constexpr (GRAD) request_signs(s + 4);
            else if constexpr (P == 0) request_signs(s + 4);
            request_a(min(s + 4, last), a_stage(P));
            __builtin_amdgcn_sched_barrier(0);
            request_w(min(s + 5, last), Next{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(3);
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int s = 0; s < n_steps; s += 4) {
            step(s, I0{});
            step(s + 1, I1{});
            if (s + 2 < n_steps) {                    // uniform
                step(s + 2, I2{});
                step(s + 3, I3{});
            }
        }
        wait_loads<0>();
        lds_barrier();                                // nothing is on its way into LDS any more
    } else {
        request_signs(0);
        if constexpr (GRAD) request_signs(1);
        request_a(0, a_stage(0));
        __builtin_amdgcn_sched_barrier(0);
        request_w(0, I0{});
        if constexpr (AHEAD == 2) request_w(1, I1{});
        wait_loads<0>();
        fetch_signs(0);
        convert_w(w_stage(0), I0{});
        lds_barrier();
        request_a(1, a_stage(1));
        __builtin_amdgcn_sched_barrier(0);
        request_w(min(AHEAD, last), I0{});
        read_frags(a_stage(0), w_stage(0), I0{});

        // Step s, s % 2 = P.  What is asked for in its last quarter: the signs, then the tokens of step s + 2, then W_b of step s + 1 +
        // AHEAD (one step ahead: as soon as it is converted); in the next step's second quarter all but those last four loads have to
        // be there.  REQ: there is a step s + 2, MORE: a step s + 1.
        auto step = [&](int s, auto phase, auto req, auto more) {
            constexpr int P = decltype(phase)::value;
            constexpr bool REQ = decltype(req)::value, MORE = decltype(more)::value;
            using Next = std::integral_constant<int, 1 - P>;
            read_frags(a_stage(P), w_stage(P), I1{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(0);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (MORE) {
                wait_loads<AHEAD == 2 ? 4 : 0>();
                fetch_signs(s + 1);
            }
            read_frags(a_stage(P), w_stage(P), I2{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(1);
            if constexpr (MORE) convert_w(w_stage(P + 1), Next{});        // (the compiler's own order among the MFMAs: 1-2 % better than a fixed one)
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (REQ && AHEAD == 1) request_w(s + 2, I0{});
            read_frags(a_stage(P), w_stage(P), I3{});
            __builtin_amdgcn_sched_barrier(0);
            multiply(2);
            __builtin_amdgcn_sched_barrier(0);
            lds_barrier();
            if constexpr (MORE) read_frags(a_stage(P + 1), w_stage(P + 1), I0{});
            if constexpr (REQ) {
                if constexpr (GRAD) request_signs(s + 2);
                else if ((s & 3) == 0) request_signs(s + 4);
                request_a(s + 2, a_stage(P));
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (AHEAD == 2) request_w(min(s + 3, last), Next{});
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(3);
            __builtin_amdgcn_sched_barrier(0);
        };
        int s = 0;
        for (; s + 2 < n_steps; s += 2) {
            step(s, I0{}, std::true_type{}, std::true_type{});
            step(s + 1, I1{}, std::true_type{}, std::true_type{});
        }
        step(s, I0{}, std::false_type{}, std::true_type{});
        step(s + 1, I1{}, std::false_type{}, std::false_type{});
    }

    // (the last barrier came after the last fragment read: the stages are free)
    const int m0 = t.row0 + wm * (BM / 2);
    if (inverse != nullptr) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float x = inverse[min(m0 + f * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3), t.end - 1)];
#pragma unroll
                for (int h = 0; h < FN; ++h) acc[f][h][r] *= x;
            }
    }
    const int o0 = n0 + wn * 64;
    if (store_tile_16bit<FM>(acc, (uint16_t*)tile_smem + wave * 32 * kGemmLDK, Y, y_dtype, m0, o0, t.end, N, lane)) return;
    if (y_dtype == kF32) store_rows<kF32, FM>(acc, Y, g.parts > 1 ? g.pitch : N, m0, o0, t.end, N, lane);
    else if (y_dtype == kBF16) store_rows<kBF16, FM>(acc, Y, N, m0, o0, t.end, N, lane);
    else store_rows<kF16, FM>(acc, Y, N, m0, o0, t.end, N, lane);
}

// A tile of fewer tokens takes as many MFMA tiles as they need: the ends of ragged experts cost what they are.
template <int WDT, int AXIS, bool GRAD>
__global__ void __launch_bounds__(512, 2)
experts_big_kernel(const uint16_t* __restrict__ A, int lda, const float* __restrict__ inverse, const int* __restrict__ offsets,
                   const uint16_t* __restrict__ W_b, int64_t w_stride, const uint32_t* __restrict__ B_packed,
                   const uint16_t* __restrict__ v, void* __restrict__ Y, float* __restrict__ partial, int M, int E, int d_out, int d_in, int y_dtype,
                   int n_tiles, int parts, int sign_ld, int height)
{
    extern __shared__ __attribute__((aligned(16))) unsigned char tile_smem[];
    const TileArgs g{A, lda, inverse, W_b, w_stride, B_packed, v, Y, partial, M, d_out, d_in, y_dtype, parts, sign_ld, n_tiles * kTileN};
    ExpertTile t;
    int tile_n, rows;
    {
        ExpertTiles list{offsets, E, M, n_tiles * parts, height > 0 ? height : kTileM};     // a part is a tile of its own here
        if (height == 0) list.choose_height();
        const int stop = list.range((int)blockIdx.x % kXcds), number = list.at + (int)blockIdx.x / kXcds;
        if (number >= stop || !list.tile(number, t, tile_n)) return;          // whole workgroup
        rows = min(t.end - t.row0, list.height);
    }
    const int part = tile_n % parts;
    tile_n /= parts;
    if (rows > 192) experts_tile<WDT, AXIS, GRAD, 4>(g, t, tile_n, part, tile_smem);
    else if (rows > 128) experts_tile<WDT, AXIS, GRAD, 3>(g, t, tile_n, part, tile_smem);
    else if (rows > 64) experts_tile<WDT, AXIS, GRAD, 2>(g, t, tile_n, part, tile_smem);
    else experts_tile<WDT, AXIS, GRAD, 1>(g, t, tile_n, part, tile_smem);
}

// The parts' sums of a split contraction, in their order, for rows that belong to an expert.
template <int YDT>
__global__ void __launch_bounds__(256)
experts_sum_kernel(const float* __restrict__ partial, const float* __restrict__ inverse, const int* __restrict__ offsets, void* __restrict__ Y,
                   int M, int E, int N, int pitch, int parts, int blocks)
{
    const int m = blockIdx.x / blocks, n = (blockIdx.x % blocks * 256 + threadIdx.x) * 4;
    if (n >= N || (offsets != nullptr && (m < offsets[0] || m >= offsets[E]))) return;
    const float x = inverse != nullptr ? inverse[m] : 1.f;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
        const float4v a = *(const float4v*)(partial + ((int64_t)p * M + m) * pitch + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] += a[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < N) store_y<YDT>(Y, (int64_t)m * N + n + e, sum[e] * x);
}

int64_t experts_pitch(int64_t N) { return (N + kTileN - 1) / kTileN * kTileN; }

// Parts of the contraction: tiles that leave most of the 256 CUs idle are cut into as many parts as fill three quarters of them, or
// all where experts have few tokens and their sums are short, of six (four) steps at least.  us in 1, 2, 3, 4, 6, 8 and 12 parts: 2 experts,
// 456 tokens, 1667 x 3328 fp16, 14 tiles: 79, 48, 38, 34, 30, 30, 38; 64 tokens, input gradient of 11008 x 4096, 16 tiles: 142, 79, 57,
// 46, 37, 32, 32; 1000 tokens, 4096 x 4096, 64 tiles: 93, 64, 58, 61, 76, 86, 104; 17 experts, 2741 tokens, input gradient of 982 x 1280, 85
// tiles: 43, 42, 51, 55.  The sums take at most 64 MiB of workspace.
int experts_parts(int64_t M, int64_t E, int64_t N, int64_t K)
{
    if (M == 0) return 1;
    const int64_t met = std::min(E, M), tiles = (N + kTileN - 1) / kTileN * met * ((M + met * kTileM - 1) / (met * kTileM));
    const int64_t steps = experts_padded(K) / kTileK;
    const bool few = M <= 128 * met;
    return (int)std::max<int64_t>(1, std::min<int64_t>({12, (few ? 256 : 192) / tiles, steps / (few ? 4 : 6)}));
}

// Tokens of a full tile: 256, or as many of 192 and 128 as let the CUs finish an eighth sooner by the tiles' costs.  For one expert the
// host takes its M tokens for it; for up to 64, of which about one round of tiles is expected, the kernel (0) looks at the offsets.
// us with 256 and with the rule: input gradient of 4096 x 11008, 777 tokens 118, 105 (192); 2048 tokens 238, 225 (192); 4 experts, 1500
// tokens, 4096 x 4096 bf16 110, 94 (128); 12 experts, 1501 tokens 114, 106 (192).  More rounds of uneven experts gain nothing and
// pay for the look: 16 experts, 3000 tokens 116, 123; 8 experts, 1024 tokens, 14336 x 4096 288, 295.
template <int WDT, int AXIS, bool GRAD>
static int launch_big_tiles(const ExpertsCall& c, const uint16_t* A, int lda, const float* inverse, float* partial, int parts, int sign_ld,
                            hipStream_t stream)
{
    constexpr int lds = kTileLds;
    const int64_t n_tiles = ((GRAD ? c.d_in : c.d_out) + kTileN - 1) / kTileN;
    const bool few = (c.M / kTileM + std::min(c.E, c.M) / 2) * n_tiles <= 256;
    const int height = parts > 1 || c.M <= 128 ? kTileM : c.E == 1 ? ExpertTiles::height_of_one(c.M, n_tiles) : c.E <= kWave && few ? 0 : kTileM;
    const int64_t most = ExpertTiles::most_in_a_range(c.M, c.E, n_tiles * parts, height > 0 ? height : 128), blocks = most * kXcds;
    if (most > (1 << 24)) return -2;                  // (costs are summed in 32 bits)
    auto kernel = experts_big_kernel<WDT, AXIS, GRAD>;
    static unsigned lds_opted_in = 0;                 // per template instance: one kernel
    if (opt_in_dynamic_lds((const void*)kernel, lds, &lds_opted_in) != 0) return -1;
    hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(512), lds, stream, A, lda, inverse, c.offsets, (const uint16_t*)c.W_b, c.w_stride,
                       c.B_packed, c.v, c.out, partial, (int)c.M, (int)c.E, (int)c.d_out, (int)c.d_in, c.out_dtype, (int)n_tiles, parts, sign_ld, height);
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

int launch_experts_big(const ExpertsCall& c, bool grad, const uint16_t* A, int lda, const float* inverse, float* partial, int parts,
                       int sign_ld, hipStream_t stream)
{
    auto tiles = [&]() {
#define PDELTA_GO(WDT, AXIS, GRAD) return launch_big_tiles<WDT, AXIS, GRAD>(c, A, lda, inverse, partial, parts, sign_ld, stream)
        if (c.dtype == kBF16) {
            if (c.axis == 0 && grad) PDELTA_GO(kBF16, 0, true);
            if (c.axis == 0) PDELTA_GO(kBF16, 0, false);
            if (grad) PDELTA_GO(kBF16, 1, true);
            PDELTA_GO(kBF16, 1, false);
        }
        if (c.axis == 0 && grad) PDELTA_GO(kF16, 0, true);
        if (c.axis == 0) PDELTA_GO(kF16, 0, false);
        if (grad) PDELTA_GO(kF16, 1, true);
        PDELTA_GO(kF16, 1, false);
#undef PDELTA_GO
    };
    if (const int rc = tiles(); rc != 0 || parts == 1) return rc;
    const int64_t N = grad ? c.d_in : c.d_out, blocks = (N + 1023) / 1024;
#define PDELTA_GO(YDT)                                                                                                              \
    hipLaunchKernelGGL(experts_sum_kernel<YDT>, dim3((unsigned)(c.M * blocks)), dim3(256), 0, stream, partial, inverse, c.offsets, c.out, \
                       (int)c.M, (int)c.E, (int)N, (int)experts_pitch(N), parts, (int)blocks)
    if (c.out_dtype == kF32) PDELTA_GO(kF32);
    else if (c.out_dtype == kBF16) PDELTA_GO(kBF16);
    else PDELTA_GO(kF16);
#undef PDELTA_GO
    return hipGetLastError() == hipSuccess ? 0 : -1;
}

}  // namespace pdelta
