// MFMA matmuls of the Gated MLP's backward pass for gfx950.
//
// With H = act(G) U and Y = H Wd the chain rule gives five matmuls,
//     dH = dY Wd^T,   dX = dG Wg^T + dU Wu^T,
//     dWd = H^T dY,   dWg = X^T dG,   dWu = X^T dU,
// with dU = dH act(G) and dG = dH U act'(G) between the first and the others.
// One template computes all of them as
//     C[n, m] = sum_k B(n, k) A(m, k)
// from tensors as they lie in memory: an operand is "k-contiguous" (rows of k:
// Wd, Wg, Wu, dY, dG and dU in the first two) or "line-contiguous" (rows of m or
// n, one row per k: all six operands of the weight gradients, which contract the
// tokens).  Nothing is transposed in memory: a k-contiguous tile is read from LDS
// with ds_read_b128, a line-contiguous one with the transposing ds_read_b64_tr_b16.
//
// Three launches:
//   * dH, whose epilogue reads G and U once and writes dG, dU and H = act(G) U
//     as bf16; dH itself stays in the fp32 accumulators.
//   * dX, one contraction over 2 F: the k-tiles of dG Wg^T, then of dU Wu^T.
//   * the three weight gradients as one grid of tiles, so that only one partial
//     last round of blocks is left.
// dG, dU and H are rounded to bf16 because they are MFMA operands next.
//
// The pipeline is that of the forward tiles (gemm_mfma.hpp): a ring of LDS stages
// filled by DMA, XOR-swizzled 16-byte chunks, v_mfma_f32_16x16x32_bf16 fed by
// fragments read one k32 step ahead.
// Where there are many tokens the kernels are bound by the rate at which operand
// tiles reach LDS and leave it again, 128 FLOP per staged byte for the 256 x 256
// tiles; where there are few, by the weights read (dH, dX) and the gradients written.
// Measured (us): T = 4096, D = 4096, F = 14336 dH 500 to 510 (0.96 PFLOP/s: its outputs have
// no MFMAs beside them), dX 675 to 690 (1.41), dW 1110 to 1160 (1.27); the vendor library's
// 8192^3 products of these operand orders reach 1.61 and 1.19.  T = 30 dW 74 (outputs of
// 352 MB: 4.8 TB/s).  Tried without gain for the large tiles: k-tiles of 32 in four stages
// (dX +11%); a persistent grid that loads the next tile's operands during the outputs (its
// control flow cost 0.2 us a k-tile, more than the loads it hid).
#pragma once

#include <utility>

#include "gemm_mfma.hpp"
#include "grad_plan.hpp"

namespace gmlp {

enum GradEpilogue {
    GRAD_STORE = 0, // out = bf16(C)
    GRAD_GATE = 1,  // C = dH: dG, dU and H from it
};

struct GradParams {
    // Problems (weight gradients) or segments of k (dX: problem 0's second pair).
    const uint16_t *a[3], *b[3];
    uint16_t *out[3];
    int M[3], N[3];    // output columns and rows
    int K;             // contracted elements of a segment
    int kt_seg;        // k-tiles of a segment
    int nk;            // k-tiles of a tile
    int problem_tiles; // tiles of one problem
    int whole;         // tiles of one block each
    int rest;          // tiles after these, each split over k into
    int splits;        // this many blocks
    int kt_split;      // of so many k-tiles
    float *partial;
    uint32_t *counters;
    // GRAD_GATE
    const uint16_t *g, *u;
    uint16_t *dg, *du, *h;
    int activation;
    float beta;
};

// The chunk swizzle of w_swizzle for line-contiguous rows of 16 or 32 chunks, from
// a table in a register: rows k of bits 0, 1 and 4.
__device__ __forceinline__ int grad_swizzle(int k)
{
    return 0xe842ca60u >> (4 * ((k & 3) | (k >> 2 & 4))) & 15;
}

// The staging addresses of one operand's tiles of LINES lines x BK k.
//
// k-contiguous (KC): LDS rows of 128 bytes, 8 chunks, hold one line of 64 k or, of
// 32 k, line r in chunks 0..3 and line r + LINES / 2 in chunks 4..7; chunk c of row
// r is at position c ^ x_swizzle(r).  Line-contiguous: one LDS row per k.
template <bool KC, int LINES, int NWAVES, int BK>
struct GradLoader {
    static constexpr int LOADS = LINES * BK * 2 / (NWAVES * 1024);
    static constexpr int ROWS = LINES * BK / 64; // KC: LDS rows
    static constexpr int CPR = LINES / 8;        // chunks of a line-contiguous LDS row
    static constexpr int LPR = 64 / CPR;         // such rows per wave load
    static constexpr int RPI = NWAVES * LPR;     // such rows per load step
    static_assert(LOADS * NWAVES * 1024 == LINES * BK * 2, "whole 16-byte loads");
    static_assert(KC || ((CPR == 16 || CPR == 32) && RPI >= 8 && RPI <= 32), "row bits 0, 1 and 4 of the swizzle");
    // Distinct per-lane addresses; load i takes number `which(i)` of them, i times
    // soff_step further.
    static constexpr int ADDRS = KC ? (NWAVES % 8 ? 2 : 1) : (RPI < 32 ? 2 : 1);
    __device__ static constexpr int which(int i) { return KC ? i % ADDRS : (i * RPI >> 4) % ADDRS; }
    static constexpr int ROW_STEP = 8 * NWAVES; // KC: LDS rows from one load to the next

    uint32_t voff[ADDRS];
    uint32_t soff_step;
    int lines;              // KC: lines of the tile that exist
    size_t start, k_stride; // elements to line l0 of k = 0, and from one k to the next

    // KC: the line and the first k of the chunk that load i (i < ADDRS) brings.
    __device__ __forceinline__ static int chunk(int i, int wave, int lane)
    {
        return (lane & 7) ^ x_swizzle((i * NWAVES + wave) * 8 + (lane >> 3));
    }
    __device__ __forceinline__ static int line(int i, int wave, int lane)
    {
        return wave * 8 + (lane >> 3) + (BK == 32 ? (chunk(i, wave, lane) >> 2) * ROWS : 0);
    }
    __device__ __forceinline__ static int first_k(int i, int wave, int lane)
    {
        return (chunk(i, wave, lane) & (BK / 8 - 1)) * 8;
    }

    // The tile at line l0 of L lines, row stride ld elements.
    __device__ __forceinline__ void init(int l0, int L, int ld, int wave, int lane)
    {
        lines = L - l0;
        start = KC ? (size_t)l0 * ld : (size_t)l0;
        k_stride = KC ? 1 : (size_t)ld;
        soff_step = (uint32_t)(KC ? ROW_STEP : RPI) * (uint32_t)ld * 2u;
#pragma unroll
        for (int b = 0; b < ADDRS; ++b) {
            if constexpr (KC) {
                voff[b] = ((uint32_t)line(b, wave, lane) * (uint32_t)ld + (uint32_t)first_k(b, wave, lane)) * 2u;
            } else {
                const int k = wave * LPR + lane / CPR, c = (lane % CPR) ^ grad_swizzle(k ^ (16 * b));
                voff[b] = c * 8 < lines ? ((uint32_t)k * (uint32_t)ld + (uint32_t)c * 8u) * 2u : kOutOfRange;
            }
        }
    }

    // The DMA of the k-tile from k0 on: k past krem and lines past L read as zeros.
    // STREAM: elements that no other block reads.
    template <bool STREAM = false>
    __device__ __forceinline__ void issue(const uint16_t *p, int k0, int krem, uint8_t *buf, int wave, int lane) const
    {
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(p + start + (size_t)k0 * k_stride);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int b = which(i);
            const bool in_k = (KC ? first_k(b, wave, lane) : i * RPI + wave * LPR + lane / CPR) < krem;
            const bool in = in_k && (!KC || i * ROW_STEP + line(b, wave, lane) < lines);
            const uint32_t at = in ? voff[b] : kOutOfRange;
            if constexpr (STREAM)
                load16_to_lds_stream(rs, buf + (i * NWAVES + wave) * 1024, at, (uint32_t)i * soff_step);
            else
                load16_to_lds(rs, buf + (i * NWAVES + wave) * 1024, at, (uint32_t)i * soff_step);
        }
    }
};

// The MFMA fragments of one operand's staged tile, 16 lines each from line `first`
// (a multiple of 32) on: the same lane layout and k order for both operands.
//
// One address register serves all fragments: the swizzles differ between them by
// an XOR with a constant.  k-contiguous, fragment q is 16 q rows on, where the row's
// swizzle (r ^ r / 8) % 8 is that of the first with 2 q % 8 in it; line-contiguous,
// its chunk is 2 q further, in bits that the first chunk has clear.
template <bool KC, int LINES, int BK>
struct GradFragments {
    static constexpr int ROW_BYTES = LINES * 2, ROWS = LINES * BK / 64;
    int at;
    __device__ __forceinline__ void init(int first, int lane)
    {
        const int kg = ((lane >> 4) & 1) << 1 | (lane >> 5);
        if constexpr (KC) {
            const int r = first % ROWS + (lane & 15), c = kg + 4 * (first / ROWS);
            at = r * 128 + ((c ^ x_swizzle(r)) << 4);
        } else {
            const int k = 8 * kg + ((lane & 15) >> 2), c = first / 8 + ((lane & 3) >> 1);
            at = k * ROW_BYTES + ((c ^ grad_swizzle(k)) << 4) + (lane & 1) * 8;
        }
    }
    // Fragment q of k32 step kk.
    __device__ __forceinline__ bf16x8 read(const uint8_t *buf, int kk, int q) const
    {
        if constexpr (KC) {
            return *(const bf16x8 *)(buf + (at ^ ((2 * q & 6) << 4 ^ 64 * kk)) + q * 16 * 128);
        } else {
            const uint8_t *p = buf + (at ^ (2 * q << 4)) + kk * 32 * ROW_BYTES;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)GMLP_LDS(p));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) i16x4 *)GMLP_LDS(p + 4 * ROW_BYTES));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// dG, dU and H of eight neighbouring elements.  sigmoid' = s (1 - s); above zero, where s
// nears 1 and the difference would lose its digits (at g = 16 all of them), 1 - s is
// e^-bg s.  beta g may be infinite where g is not, and s (1 - s) is 0 then: beta comes
// after it.
__device__ __forceinline__ void gate_gradients(const float (&dh)[8], const u32x4 &g4, const u32x4 &u4, int act, float beta,
                                               u32x4 &dg4, u32x4 &du4, u32x4 &h4)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float dg[2], du[2], h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float g = e ? bf16_hi(g4[q]) : bf16_lo(g4[q]), u = e ? bf16_hi(u4[q]) : bf16_lo(u4[q]);
            const float x = beta * g, t = __expf(-x), s = __builtin_amdgcn_rcpf(1.0f + t);
            const float c = s * (x > 0.0f ? t * s : 1.0f - s); // sigmoid'
            const bool glu = act == ACT_SIGMOID;
            const float a = glu ? s : g * s;
            const float da = glu ? c : s + beta * c * g;
            h[e] = a * u;
            du[e] = dh[2 * q + e] * a;
            dg[e] = dh[2 * q + e] * u * da;
        }
        dg4[q] = pack_bf16x2(dg[0], dg[1]);
        du4[q] = pack_bf16x2(du[0], du[1]);
        h4[q] = pack_bf16x2(h[0], h[1]);
    }
}

// Two neighbouring runs of 32 columns of 16 rows, 16 bytes per lane each, lane l row
// l % 16, become the first and the last eight rows with all 64 columns: 128-byte lines
// are written whole by one store.  Rows r < 8 give their second run for the first run
// of rows r + 8.
__device__ __forceinline__ void store_lines(u32x4 &first, u32x4 &second, int lane)
{
    const bool high = lane & 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = first[i], b = second[i];
        const uint32_t got = __builtin_amdgcn_update_dpp(0, high ? a : b, 0x128, 0xf, 0xf, false); // row_ror:8
        first[i] = high ? got : a;
        second[i] = high ? b : got;
    }
}

// One block: one output tile, or one split of its k-tiles.  KC: both operands
// k-contiguous; SEGS = 2: dX's two pairs; otherwise a problem per range of
// problem_tiles tiles.  STREAM_OUT: outputs past the L2.
template <class S, bool KC, int EPI, int SEGS, bool STREAM_OUT>
__global__ __launch_bounds__(S::NTHREADS, S::BLOCKS) void gemm_grad_kernel(GradParams p)
{
    constexpr int TM = S::TM, TN = S::TN, STAGES = S::STAGES, BK = S::BK;
    constexpr int OUT_POLICY = STREAM_OUT ? kNonTemporal : 0;
    __shared__ __attribute__((aligned(1024))) uint8_t lds0[S::STAGE_BYTES];
    __shared__ __attribute__((aligned(1024))) uint8_t lds1[S::STAGE_BYTES];
    __shared__ __attribute__((aligned(1024))) uint8_t lds2[STAGES > 2 ? S::STAGE_BYTES : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t lds3[STAGES > 3 ? S::STAGE_BYTES : 16];
    __shared__ int s_last;
    auto stage_ptr = [&](auto s) __attribute__((always_inline)) -> uint8_t * {
        if constexpr (decltype(s)::value == 0) return lds0;
        else if constexpr (decltype(s)::value == 1) return lds1;
        else if constexpr (decltype(s)::value == 2) return lds2;
        else return lds3;
    };

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave % S::WM, wn = wave / S::WM;
    const int bid = blockIdx.x, K = p.K;

    // Block -> tile: the whole tiles first, then the pieces of the rest.  Each XCD
    // takes a contiguous range of either; neighbouring tiles share operand strips,
    // in sweeps of 8 column tiles (gemm_mfma.hpp).
    const bool whole = bid < p.whole;
    const int id = whole ? xcd_contiguous_id(bid, p.whole) : xcd_contiguous_id(bid - p.whole, p.rest * p.splits);
    const int split = whole ? 0 : id / p.rest, piece_tile = whole ? 0 : id - split * p.rest;
    const int tile = whole ? id : p.whole + piece_tile;
    const int kt_begin = split * p.kt_split, kt_end = whole ? p.nk : min(p.nk, kt_begin + p.kt_split);
    const int nk = kt_end - kt_begin;
    const int prob = SEGS == 1 ? tile / p.problem_tiles : 0;
    const int local = tile - prob * p.problem_tiles;
    const int M = p.M[prob], N = p.N[prob];
    const int tiles_m = (M + S::BM - 1) / S::BM, tiles_n = (N + S::BN - 1) / S::BN;
    if (local >= tiles_m * tiles_n) // the transposed shape may have fewer tiles
        return;
    const int per_group = 8 * tiles_n;
    const int group = local / per_group, in_group = local - group * per_group;
    const int group_w = min(tiles_m - group * 8, 8);
    const int m0 = (group * 8 + in_group % group_w) * S::BM, n0 = (in_group / group_w) * S::BN;

    GradLoader<KC, S::BM, S::NWAVES, BK> la;
    GradLoader<KC, S::BN, S::NWAVES, BK> lb;
    la.init(m0, M, KC ? K : M, wave, lane);
    lb.init(n0, N, KC ? K : N, wave, lane);
    // Past the end zeros are read, so that every step has the same number of loads
    // in flight.
    int load_kt = kt_begin;
    auto issue = [&](uint8_t *buf) __attribute__((always_inline)) {
        const int seg = SEGS == 2 && load_kt >= p.kt_seg ? 1 : 0;
        const int k0 = load_kt < kt_end ? (load_kt - seg * p.kt_seg) * BK : 0;
        const int krem = load_kt < kt_end ? K - k0 : 0;
        const int q = SEGS == 2 ? seg : prob;
        la.issue(p.a[q], k0, krem, buf, wave, lane);
        lb.issue(p.b[q], k0, krem, buf + S::A_BYTES, wave, lane);
        ++load_kt;
    };

    GradFragments<KC, S::BM, BK> qa;
    GradFragments<KC, S::BN, BK> qb;
    qa.init(wm * TM * 32, lane);
    qb.init(wn * TN * 32, lane);

    using Acc = AccBlock<true>;
    Acc acc[TM][TN];
#pragma unroll
    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
        for (int ni = 0; ni < TN; ++ni)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[mi][ni].set_piece(j, f32x4{});

    // The MFMAs of one k32 step, one group per 16-row B fragment, with the next
    // step's fragment reads among them (as gemm_block's mma_roll).
    struct FragA {
        bf16x8 a[TM * 2];
    };
    FragA fa0, fa1;
    bf16x8 fb[TN * 2];
    auto mma_roll = [&](const FragA &fa, FragA &fa_next, const uint8_t *nbuf, int nkk) __attribute__((always_inline)) {
        constexpr int GROUPS = TN * 2, AFRAGS = TM * 2, APG = (AFRAGS + GROUPS - 1) / GROUPS;
        [&]<int... G>(std::integer_sequence<int, G...>) __attribute__((always_inline)) {
            (
                [&] {
#pragma unroll
                    for (int a = 0; a < AFRAGS; ++a)
                        acc[a / 2][G / 2].v[a % 2 + 2 * (G % 2)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            fa.a[a], fb[G], acc[a / 2][G / 2].v[a % 2 + 2 * (G % 2)], 0, 0, 0);
#pragma unroll
                    for (int q = G * APG; q < (G + 1) * APG && q < AFRAGS; ++q)
                        fa_next.a[q] = qa.read(nbuf, nkk, q);
                    fb[G] = qb.read(nbuf + S::A_BYTES, nkk, G);
                    __builtin_amdgcn_sched_barrier(0);
                }(),
                ...);
        }(std::make_integer_sequence<int, GROUPS>{});
    };
    auto wait_tile = [&]() __attribute__((always_inline)) {
        wait_vmcnt<(STAGES - 2) * S::LOADS_PER_STAGE>();
        wait_lgkm0();
        barrier_only();
    };

    [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
        (issue(stage_ptr(std::integral_constant<int, I>{})), ...);
    }(std::make_integer_sequence<int, STAGES - 1>{});
    wait_tile();
    issue(stage_ptr(std::integral_constant<int, STAGES - 1>{}));
#pragma unroll
    for (int q = 0; q < TM * 2; ++q)
        fa0.a[q] = qa.read(lds0, 0, q);
#pragma unroll
    for (int q = 0; q < TN * 2; ++q)
        fb[q] = qb.read(lds0 + S::A_BYTES, 0, q);
    // The k-tile in stage I % STAGES.  At its last k32 step, whose fragments have
    // been read, a barrier frees the stage for the DMA of the k-tile STAGES ahead
    // and the next k-tile's first fragments are read.
    auto step = [&](auto index) __attribute__((always_inline)) {
        constexpr int I = decltype(index)::value;
        uint8_t *buf = stage_ptr(std::integral_constant<int, I % STAGES>{});
        uint8_t *next = stage_ptr(std::integral_constant<int, (I + 1) % STAGES>{});
        if constexpr (BK == 64)
            mma_roll(fa0, fa1, buf, 1);
        wait_tile();
        issue(buf);
        if constexpr (BK == 64 || I % 2 == 1)
            mma_roll(fa1, fa0, next, 0);
        else
            mma_roll(fa0, fa1, next, 0);
    };
    // A round of steps brings stages and fragment buffers back to the first.
    constexpr int ROUND = BK == 64 || STAGES % 2 == 0 ? STAGES : 2 * STAGES;
    int i = 0;
    for (; i + ROUND <= nk; i += ROUND) {
        [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
            (step(std::integral_constant<int, I>{}), ...);
        }(std::make_integer_sequence<int, ROUND>{});
    }
    [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
        ((i + I < nk ? step(std::integral_constant<int, I>{}) : void()), ...);
    }(std::make_integer_sequence<int, ROUND - 1>{});
    wait_vmcnt<0>(); // loads past the end, before LDS is given to another block

    // ---- outputs ---------------------------------------------------------------
    // A batch is the wave's 16 output rows of one B fragment: TM runs of 32 columns,
    // eight of them per lane.  Batch b is half b % 2 of acc[.][b / 2].
    constexpr int BATCHES = TN * 2;
    const auto corner = [&](const uint16_t *t, bool used) __attribute__((always_inline)) {
        return make_rsrc(used ? t + (size_t)n0 * M + m0 : nullptr);
    };
    const __amdgpu_buffer_rsrc_t ro = corner(p.out[prob], EPI == GRAD_STORE);
    const __amdgpu_buffer_rsrc_t rg = corner(p.g, EPI == GRAD_GATE), ru = corner(p.u, EPI == GRAD_GATE);
    const __amdgpu_buffer_rsrc_t rdg = corner(p.dg, EPI == GRAD_GATE), rdu = corner(p.du, EPI == GRAD_GATE);
    const __amdgpu_buffer_rsrc_t rh = corner(p.h, EPI == GRAD_GATE);
    auto offset = [&](int b, int mi) __attribute__((always_inline)) {
        const int ml = wm * TM * 32 + mi * 32 + wide_column(lane), nl = wn * TN * 32 + b * 16 + (lane & 15);
        const int in = (int)(n0 + nl < N) & (int)(m0 + ml < M); // without a branch
        return in ? ((uint32_t)nl * (uint32_t)M + (uint32_t)ml) * 2u : kOutOfRange;
    };
    // Of a pair of runs: store `half` takes eight rows of 128 bytes (store_lines).
    auto line_offset = [&](int b, int mi, int half) __attribute__((always_inline)) {
        const int ml = wm * TM * 32 + mi * 32 + wide_column(lane) + 4 * (lane & 8);
        const int nl = wn * TN * 32 + b * 16 + 8 * half + (lane & 7);
        const int in = (int)(n0 + nl < N) & (int)(m0 + ml < M);
        return in ? ((uint32_t)nl * (uint32_t)M + (uint32_t)ml) * 2u : kOutOfRange;
    };
    struct Gates {
        u32x4 g[TM], u[TM];
    };
    // G and U of the batches ahead are on their way while one is computed.
    constexpr int AHEAD = EPI == GRAD_GATE ? (BATCHES < 4 ? BATCHES : 4) : 1;
    Gates gates[AHEAD];
    auto load_gates = [&](Gates &v, int b) __attribute__((always_inline)) {
#pragma unroll
        for (int mi = 0; mi < TM; ++mi) {
            v.g[mi] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rg, offset(b, mi), 0, 0));
            v.u[mi] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ru, offset(b, mi), 0, 0));
        }
    };
    // lo, hi: the two MFMA results of each run.
    auto emit = [&](int b, const f32x4 (&lo)[TM], const f32x4 (&hi)[TM]) __attribute__((always_inline)) {
        u32x4 c[TM];
#pragma unroll
        for (int mi = 0; mi < TM; ++mi) {
            float v[8];
            wide_columns(lo[mi], hi[mi], v);
            if constexpr (EPI == GRAD_GATE) {
                const uint32_t off = offset(b, mi);
                const Gates &gu = gates[b % AHEAD];
                u32x4 dg, du, h;
                gate_gradients(v, gu.g[mi], gu.u[mi], p.activation, p.beta, dg, du, h);
                __builtin_amdgcn_raw_buffer_store_b128(dg, rdg, off, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(du, rdu, off, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b128(h, rh, off, 0, 0);
            } else {
                c[mi] = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
            }
        }
        if constexpr (EPI == GRAD_STORE && TM % 2 == 0) {
#pragma unroll
            for (int mi = 0; mi < TM; mi += 2) {
                store_lines(c[mi], c[mi + 1], lane);
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    __builtin_amdgcn_raw_buffer_store_b128(c[mi + half], ro, line_offset(b, mi, half), 0, OUT_POLICY);
            }
        } else if constexpr (EPI == GRAD_STORE) {
#pragma unroll
            for (int mi = 0; mi < TM; ++mi)
                __builtin_amdgcn_raw_buffer_store_b128(c[mi], ro, offset(b, mi), 0, OUT_POLICY);
        }
        if constexpr (EPI == GRAD_GATE)
            if (b + AHEAD < BATCHES)
                load_gates(gates[b % AHEAD], b + AHEAD);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto piece = [&](int b, int mi, int sa) __attribute__((always_inline)) { return acc[mi][b / 2].v[sa + 2 * (b % 2)]; };
    auto first_gates = [&]() __attribute__((always_inline)) {
        if constexpr (EPI == GRAD_GATE)
#pragma unroll
            for (int b = 0; b < AHEAD; ++b)
                load_gates(gates[b], b);
    };

    if (!whole && p.splits > 1) {
        // Partial sums out with device-coherent stores, [split][tile][wave]
        // [batch][piece][lane]; the last block of a tile reads them all back and
        // adds them in the order of the splits, whichever block it is.
        const __amdgpu_buffer_rsrc_t prs = make_rsrc(p.partial);
        const uint32_t lane_off = lane * 16;
        auto wave_base = [&](int sp) __attribute__((always_inline)) {
            return (uint32_t)(((sp * p.rest + piece_tile) * S::NWAVES + wave) * S::PIECES) * 1024u;
        };
        const uint32_t own = wave_base(split);
#pragma unroll
        for (int b = 0; b < BATCHES; ++b)
#pragma unroll
            for (int mi = 0; mi < TM; ++mi)
#pragma unroll
                for (int sa = 0; sa < 2; ++sa)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, piece(b, mi, sa)), prs, lane_off,
                                                           own + ((b * TM + mi) * 2 + sa) * 1024u, kCoherent);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) {
            const uint32_t before =
                __hip_atomic_fetch_add(p.counters + piece_tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)(p.splits - 1);
        }
        __syncthreads();
        if (!s_last)
            return;
        if (tid == 0)
            __hip_atomic_store(p.counters + piece_tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        first_gates();
        // GROUP batches' sums at once: the loads of one split, of up to 20 pieces, are in
        // flight together, and each split costs their latency (about 2 us) for every group.
        constexpr int GROUP = [] {
            int g = BATCHES;
            while (g * 2 * TM > 20 || BATCHES % g)
                --g;
            return g;
        }();
#pragma unroll
        for (int b0 = 0; b0 < BATCHES; b0 += GROUP) {
            f32x4 sum[GROUP][2][TM];
            for (int sp = 0; sp < p.splits; ++sp) {
                const uint32_t base = wave_base(sp) + b0 * TM * 2 * 1024u;
                f32x4 x[GROUP][2][TM];
#pragma unroll
                for (int g = 0; g < GROUP; ++g)
#pragma unroll
                    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
                        for (int sa = 0; sa < 2; ++sa)
                            x[g][sa][mi] = __builtin_bit_cast(
                                f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                           prs, lane_off, base + ((g * TM + mi) * 2 + sa) * 1024u, kCoherent));
#pragma unroll
                for (int g = 0; g < GROUP; ++g)
#pragma unroll
                    for (int sa = 0; sa < 2; ++sa)
#pragma unroll
                        for (int mi = 0; mi < TM; ++mi)
                            sum[g][sa][mi] = sp == 0 ? x[g][sa][mi] : sum[g][sa][mi] + x[g][sa][mi];
            }
#pragma unroll
            for (int g = 0; g < GROUP; ++g)
                emit(b0 + g, sum[g][0], sum[g][1]);
        }
        return;
    }
    first_gates();
#pragma unroll
    for (int b = 0; b < BATCHES; ++b) {
        f32x4 lo[TM], hi[TM];
#pragma unroll
        for (int mi = 0; mi < TM; ++mi) {
            lo[mi] = piece(b, mi, 0);
            hi[mi] = piece(b, mi, 1);
        }
        emit(b, lo, hi);
    }
}

} // namespace gmlp
