// MFMA matmuls of the experts' Gated MLPs for gfx950: the products of gemm_mfma.hpp and
// gemm_grad.hpp for E experts in one launch, over rows sorted by expert.
//
//     products with a weight   C[n, m] = sum_k B(n, k) A_e(m, k)   for the rows n of expert e
//     weight gradients         C_e[n, m] = sum over expert e's rows r of B(r, n) A(r, m)
//
// Operands are taken as they lie in memory, through the loaders and fragments of
// gemm_grad.hpp: the rows of X, H, dY, dG and dU are k-contiguous where they meet a
// weight and line-contiguous where they are contracted; a weight is line-contiguous in
// the forward pass and k-contiguous in the backward pass.
//
// Which rows are whose is known on the device only.  A block's waves read the offsets
// (256 experts at once, four per lane), add up the tiles of rows that the experts before
// have, and find the expert and the rows of the block's tile; blocks past the last tile
// end.  All blocks come to the same counts, and so does the split of k where the tiles
// do not fill the chip: the last, partial round of tiles is given to as many blocks as
// there are CUs, and the last block of a tile adds the sums in the order of the splits.
// A tile's rows end with its expert's, in loads (zeros, no fetch) and in stores: no
// value of one expert's rows reaches another's.
//
// Few rows are bound by the weights: 2 of 8 experts of 4096 x 14336 with a row each 80 us
// gate/up and 40 down, 5.9 TB/s.  Many by the matrix cores, as the kernels for one MLP: 8192
// rows of one expert 1608 us gate/up, 700 down, 963 dH, 1406 dX, 2322 the weight gradients,
// 1.19, 1.37, 1.00, 1.37 and 1.24 PFLOP/s; of 8 experts with 558 to 1879 rows 1821, 838, 1092,
// 1715 and 2718, for the tiles of few rows at the experts' ends (half a whole one's time)
// and a last round that is not full.
#pragma once

#include <utility>

#include "experts_plan.hpp"
#include "gemm_grad.hpp"

namespace gmlp {

struct GroupedParams {
    const uint16_t *a[3], *b[3]; // weights (or rows) and rows, by weight or segment or problem
    uint16_t *out[3];
    const int32_t *offsets;
    int32_t *offsets_fall; // whether they do: GROUPED_DH finds out for GROUPED_DW
    int experts, rows;
    int M, K; // products with a weight: output columns, contracted elements of a segment
    int kt_seg, nk;
    int columns, most_row_tiles, slots, most_splits;
    int pM[3], pN[3]; // weight gradients: columns and rows of each
    int problems, problem_tiles;
    int first_block; // of this launch
    float *partial;
    uint32_t *counters;
    const uint16_t *g, *u; // GROUPED_DH
    uint16_t *dg, *du, *h;
    int activation;
    float beta;
};

// The rows of 256 experts from e0 on, four per lane (none past the last expert): one
// latency for all.  FELL: offsets that no sort gives, since some are below ones before
// them; their running maximum takes their place.  Else they are only looked at for that,
// which costs 0.1 to 0.3 us a call, and with 1024 experts 1 to 2% (45.7 us become 46.7).
template <bool FELL>
struct Experts {
    int first[4], count[4];
    int reached; // FELL: the largest offset up to the last of them
    bool falls;  // whether an offset of this lane's is below the one before it
    __device__ __forceinline__ void load(const GroupedParams &p, int e0, int lane)
    {
        int lo[4], hi[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int e = min(e0 + 64 * g + lane, p.experts - 1);
            lo[g] = p.offsets[e];
            hi[g] = p.offsets[e + 1];
        }
        if constexpr (FELL) {
            if (e0 == 0)
                reached = 0;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                lo[g] = max(lo[g], reached);
                for (int d = 1; d < 64; d <<= 1)
                    lo[g] = max(lo[g], __shfl_up(lo[g], d)); // below lane d its own
                reached = __builtin_amdgcn_readlane(lo[g], 63);
            }
        }
        falls = false;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            falls |= hi[g] < lo[g];
            const GroupedRows r = grouped_rows(lo[g], hi[g], p.rows);
            first[g] = r.first;
            count[g] = e0 + 64 * g + lane < p.experts ? r.count : 0;
        }
    }
};

// Tiles of ROWS rows of all experts; `head`: the first 256.  falls: whether an offset does.
template <int ROWS, bool FELL>
__device__ __forceinline__ int count_row_tiles(const GroupedParams &p, const Experts<FELL> &head, int lane, bool &falls)
{
    int tiles = 0;
    Experts<FELL> x = head;
    falls = false;
    for (int e0 = 0; e0 < p.experts; e0 += 256) {
        if (e0 > 0)
            x.load(p, e0, lane);
        falls |= x.falls;
#pragma unroll
        for (int g = 0; g < 4; ++g)
            tiles += (x.count[g] + ROWS - 1) / ROWS;
    }
    falls = __any(falls);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
        tiles += __shfl_xor(tiles, d);
    return min(__builtin_amdgcn_readfirstlane(tiles), p.most_row_tiles);
}

struct RowTile {
    int expert, first, count; // and its rows
    int before;               // row tiles of the experts before
};

// The expert that has row tile r of all (r < count_row_tiles).
template <int ROWS, bool FELL>
__device__ __forceinline__ RowTile find_row_tile(const GroupedParams &p, const Experts<FELL> &head, int r, int lane)
{
    RowTile t{0, 0, 0, 0};
    Experts<FELL> x = head;
    for (int e0 = 0; e0 < p.experts; e0 += 256) {
        if (e0 > 0)
            x.load(p, e0, lane);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int tiles = (x.count[g] + ROWS - 1) / ROWS;
            int sum = tiles;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int up = __shfl_up(sum, d);
                sum += lane >= d ? up : 0;
            }
            const uint64_t reached = __ballot(t.before + sum > r);
            if (reached) {
                const int l = __builtin_ctzll(reached);
                t.expert = e0 + 64 * g + l;
                t.first = __builtin_amdgcn_readlane(x.first[g], l);
                t.count = __builtin_amdgcn_readlane(x.count[g], l);
                t.before += __builtin_amdgcn_readlane(sum - tiles, l);
                return t;
            }
            t.before += __builtin_amdgcn_readlane(sum, 63);
        }
    }
    return t;
}

// The rows of expert e where offsets fall.
__device__ __forceinline__ GroupedRows risen_rows(const GroupedParams &p, int e, int lane)
{
    Experts<true> x;
    for (int e0 = 0; e0 <= e; e0 += 256)
        x.load(p, e0, lane);
    GroupedRows r{0, 0};
#pragma unroll
    for (int g = 0; g < 4; ++g)
        if ((e >> 6 & 3) == g)
            r = GroupedRows{__builtin_amdgcn_readlane(x.first[g], e & 63), __builtin_amdgcn_readlane(x.count[g], e & 63)};
    return r;
}

// One block: one output tile, or one split of its k-tiles.
template <class S, GroupedOp OP, bool STREAM_OUT>
__global__ __launch_bounds__(S::NTHREADS, S::BLOCKS) void gemm_grouped_kernel(GroupedParams p)
{
    constexpr bool GATE_UP = OP == GROUPED_GATE_UP || OP == GROUPED_SAVE;
    constexpr bool WEIGHTS = OP == GROUPED_DW;                // weight gradients
    constexpr bool KCA = OP == GROUPED_DH || OP == GROUPED_DX; // A k-contiguous
    constexpr bool KCB = !WEIGHTS;
    constexpr int NW = GATE_UP ? 2 : 1; // weights side by side in a tile
    constexpr int SEGS = OP == GROUPED_DX ? 2 : 1;
    constexpr int TM = S::TM, TN = S::TN, STAGES = S::STAGES, BK = S::BK;
    constexpr int TMW = TM / NW, BMW = S::BM / NW; // of one weight
    constexpr bool SIMPLE = S::BLOCKS > 2; // the weight gradients of few rows
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
    const int bid = p.first_block + (int)blockIdx.x;

    // ---- block -> tile ---------------------------------------------------------
    // As in gemm_grad.hpp: each XCD takes a contiguous range of the tiles, an expert's
    // in sweeps of 8 column tiles.
    int expert, first, count; // and the expert's rows
    int M, N, K;              // of the tile's problem
    int prob = 0, local, tiles_m, tiles_n;
    int kt_begin = 0, kt_end, splits = 1, split = 0, piece_tile = 0, rest = 0;
    bool whole = true;
    if constexpr (WEIGHTS) {
        // Every XCD takes an eighth of each expert's tiles, since experts have more or
        // less to contract: with whole experts by XCD the one with the most rows kept
        // the others waiting (8 experts of 558 to 1879 rows, 4096 x 14336: 4350 us).
        const int per = p.problems * p.problem_tiles, padded = (per + 7) / 8 * 8;
        expert = bid / padded;
        if (bid - expert * padded >= per)
            return;
        const int tile = xcd_contiguous_id(bid - expert * padded, per);
        prob = tile / p.problem_tiles;
        local = tile - prob * p.problem_tiles;
        first = count = 0;
        if (p.rows > 0) { // else there may be no offsets
            GroupedRows r = grouped_rows(p.offsets[expert], p.offsets[expert + 1], p.rows);
            if (__builtin_expect(*p.offsets_fall != 0, 0))
                r = risen_rows(p, expert, lane);
            first = r.first;
            count = r.count;
        }
        M = p.pM[prob];
        N = p.pN[prob];
        K = count;
        tiles_m = (M + BMW - 1) / BMW;
        tiles_n = (N + S::BN - 1) / S::BN;
        if (local >= tiles_m * tiles_n) // the transposed shape may have fewer tiles
            return;
        kt_end = (K + BK - 1) / BK;
    } else {
        Experts<false> head;
        bool fell;
        head.load(p, 0, lane);
        int row_tiles = count_row_tiles<S::BN>(p, head, lane, fell);
        Experts<true> risen;
        if (__builtin_expect(fell, 0)) {
            bool falls;
            risen.load(p, 0, lane);
            row_tiles = count_row_tiles<S::BN>(p, risen, lane, falls);
        }
        if constexpr (OP == GROUPED_DH)
            if (bid == 0 && tid == 0)
                *p.offsets_fall = fell;
        const int tiles = row_tiles * p.columns;
        const GroupedSplit lay = grouped_split(tiles, p.slots, p.most_splits, p.nk);
        const int in_rounds = lay.in_rounds;
        rest = lay.rest;
        splits = lay.splits;
        if (bid >= in_rounds + rest * splits)
            return;
        whole = bid < in_rounds;
        const int id = whole ? xcd_contiguous_id(bid, in_rounds) : xcd_contiguous_id(bid - in_rounds, rest * splits);
        split = whole ? 0 : id / rest;
        piece_tile = whole ? 0 : id - split * rest;
        const int tile = whole ? id : in_rounds + piece_tile;
        const int r = tile / p.columns;
        const RowTile t = __builtin_expect(fell, 0) ? find_row_tile<S::BN>(p, risen, r, lane) : find_row_tile<S::BN>(p, head, r, lane);
        expert = t.expert;
        first = t.first;
        count = t.count;
        local = tile - t.before * p.columns;
        M = p.M;
        N = count;
        K = p.K;
        tiles_m = p.columns;
        tiles_n = (N + S::BN - 1) / S::BN;
        kt_begin = split * lay.kt_split;
        kt_end = whole ? p.nk : min(p.nk, kt_begin + lay.kt_split);
    }
    const int nk = kt_end - kt_begin;
    const GroupedTileAt at = grouped_tile_at(local, tiles_m, tiles_n);
    const int m0 = at.column * BMW, n0 = at.row * S::BN;

    // The tile with TX of its TN row blocks per wave; STREAM_A: a weight past the L2.
    const int own_lane = lane;
    auto run = [&]<int TX, bool STREAM_A>() __attribute__((always_inline)) {
        // Opaque, so that no address of one TX is computed ahead of the choice between
        // them and kept in registers.
        int lane = own_lane;
        asm volatile("" : "+v"(lane));
        constexpr int BX = S::WN * TX * 32, PIECES = TM * TX * 4;
        constexpr int LOADS = (S::A_BYTES + BX * BK * 2) / (S::NTHREADS * 16);
        // Operands and outputs of this expert: the weights by expert, the rows from its first.
        const size_t a_at = WEIGHTS ? (size_t)first * M : (size_t)expert * M * K;
        const size_t b_at = WEIGHTS ? (size_t)first * N : (size_t)first * K;
        const size_t out_at = WEIGHTS ? (size_t)expert * M * N : (size_t)first * M;
        GradLoader<KCA, BMW, S::NWAVES, BK> la;
        GradLoader<KCB, BX, S::NWAVES, BK> lb;
        la.init(m0, M, KCA ? K : M, wave, lane);
        lb.init(n0, N, KCB ? K : N, wave, lane);
        // Past the end zeros are read, so that every step has the same number of loads
        // in flight.
        int load_kt = kt_begin;
        auto issue = [&](uint8_t *buf) __attribute__((always_inline)) {
            const int seg = SEGS == 2 && load_kt >= p.kt_seg ? 1 : 0;
            const int k0 = load_kt < kt_end ? (load_kt - seg * p.kt_seg) * BK : 0;
            const int krem = load_kt < kt_end ? K - k0 : 0;
            const int q = SEGS == 2 ? seg : prob;
            la.template issue<STREAM_A>(p.a[q] + a_at, k0, krem, buf, wave, lane);
            if constexpr (NW == 2)
                la.template issue<STREAM_A>(p.a[1] + a_at, k0, krem, buf + S::A_BYTES / 2, wave, lane);
            lb.issue(p.b[q] + b_at, k0, krem, buf + S::A_BYTES, wave, lane);
            ++load_kt;
        };

        GradFragments<KCA, BMW, BK> qa;
        GradFragments<KCB, BX, BK> qb;
        qa.init(wm * TMW * 32, lane);
        qb.init(wn * TX * 32, lane);
        // Fragment q of the wave's A rows: those of the second weight behind the first's.
        auto read_a = [&](const uint8_t *buf, int kk, int q) __attribute__((always_inline)) {
            return qa.read(buf + (q / (2 * TMW)) * (S::A_BYTES / 2), kk, q % (2 * TMW));
        };

        using Acc = AccBlock<true>;
        Acc acc[TM][TX];
#pragma unroll
        for (int mi = 0; mi < TM; ++mi)
#pragma unroll
            for (int ni = 0; ni < TX; ++ni)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[mi][ni].set_piece(j, f32x4{});

        if constexpr (SIMPLE) {
            // One stage is computed while the other is on its way, fragments as they are
            // needed: few registers, so that four blocks are on a CU.
            static_assert(!SIMPLE || (BK == 32 && STAGES == 2), "two stages of one k32 step");
            auto step = [&](auto s) __attribute__((always_inline)) {
                wait_vmcnt<LOADS>();
                barrier_only();
                const uint8_t *buf = stage_ptr(s);
                bf16x8 fa[TM * 2];
#pragma unroll
                for (int q = 0; q < TM * 2; ++q)
                    fa[q] = read_a(buf, 0, q);
#pragma unroll
                for (int g = 0; g < TX * 2; ++g) {
                    const bf16x8 fb = qb.read(buf + S::A_BYTES, 0, g);
#pragma unroll
                    for (int a = 0; a < TM * 2; ++a)
                        acc[a / 2][g / 2].v[a % 2 + 2 * (g % 2)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            fa[a], fb, acc[a / 2][g / 2].v[a % 2 + 2 * (g % 2)], 0, 0, 0);
                }
                wait_lgkm0();
                barrier_only();
                issue(stage_ptr(s));
            };
            issue(lds0);
            issue(lds1);
            for (int i = 0; i < nk; i += 2) {
                step(std::integral_constant<int, 0>{});
                if (i + 1 < nk)
                    step(std::integral_constant<int, 1>{});
            }
        } else {
            // The MFMAs of one k32 step, one group per 16-row B fragment, with the next
            // step's fragment reads among them (as gemm_grad.hpp).
            struct FragA {
                bf16x8 a[TM * 2];
            };
            FragA fa0, fa1;
            bf16x8 fb[TX * 2];
            auto mma_roll = [&](const FragA &fa, FragA &fa_next, const uint8_t *nbuf, int nkk) __attribute__((always_inline)) {
                constexpr int GROUPS = TX * 2, AFRAGS = TM * 2, APG = (AFRAGS + GROUPS - 1) / GROUPS;
                [&]<int... G>(std::integer_sequence<int, G...>) __attribute__((always_inline)) {
                    (
                        [&] {
#pragma unroll
                            for (int a = 0; a < AFRAGS; ++a)
                                acc[a / 2][G / 2].v[a % 2 + 2 * (G % 2)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                    fa.a[a], fb[G], acc[a / 2][G / 2].v[a % 2 + 2 * (G % 2)], 0, 0, 0);
#pragma unroll
                            for (int q = G * APG; q < (G + 1) * APG && q < AFRAGS; ++q)
                                fa_next.a[q] = read_a(nbuf, nkk, q);
                            fb[G] = qb.read(nbuf + S::A_BYTES, nkk, G);
                            __builtin_amdgcn_sched_barrier(0);
                        }(),
                        ...);
                }(std::make_integer_sequence<int, GROUPS>{});
            };
            auto wait_tile = [&]() __attribute__((always_inline)) {
                wait_vmcnt<(STAGES - 2) * LOADS>();
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
                fa0.a[q] = read_a(lds0, 0, q);
#pragma unroll
            for (int q = 0; q < TX * 2; ++q)
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
        }
        wait_vmcnt<0>(); // loads past the end, before LDS is given to another block
        asm volatile("" : "+v"(lane)); // the outputs' addresses are made here, not before the loop

        // ---- outputs ---------------------------------------------------------------
        // A batch is the wave's 16 output rows of one B fragment: TM runs of 32 columns,
        // eight of them per lane.  Batch b is half b % 2 of acc[.][b / 2].
        constexpr int BATCHES = TX * 2;
        const auto corner = [&](const uint16_t *t, bool used) __attribute__((always_inline)) {
            return make_rsrc(used ? t + out_at + (size_t)n0 * M + m0 : nullptr);
        };
        constexpr bool DH = OP == GROUPED_DH, SAVE = OP == GROUPED_SAVE;
        const __amdgpu_buffer_rsrc_t ro = corner(p.out[prob], !DH);
        const __amdgpu_buffer_rsrc_t rg = corner(DH ? p.g : p.out[1], DH || SAVE), ru = corner(DH ? p.u : p.out[2], DH || SAVE);
        const __amdgpu_buffer_rsrc_t rdg = corner(p.dg, DH), rdu = corner(p.du, DH), rh = corner(p.h, DH);
        auto offset = [&](int b, int mi) __attribute__((always_inline)) {
            const int ml = wm * TMW * 32 + mi * 32 + wide_column(lane), nl = wn * TX * 32 + b * 16 + (lane & 15);
            const int in = (int)(n0 + nl < N) & (int)(m0 + ml < M); // without a branch
            return in ? ((uint32_t)nl * (uint32_t)M + (uint32_t)ml) * 2u : kOutOfRange;
        };
        // Of a pair of runs: store `half` takes eight rows of 128 bytes (store_lines).
        auto line_offset = [&](int b, int mi, int half) __attribute__((always_inline)) {
            const int ml = wm * TM * 32 + mi * 32 + wide_column(lane) + 4 * (lane & 8);
            const int nl = wn * TX * 32 + b * 16 + 8 * half + (lane & 7);
            const int in = (int)(n0 + nl < N) & (int)(m0 + ml < M);
            return in ? ((uint32_t)nl * (uint32_t)M + (uint32_t)ml) * 2u : kOutOfRange;
        };
        struct Gates {
            u32x4 g[TM], u[TM];
        };
        // G and U of the batches ahead are on their way while one is computed.
        constexpr int AHEAD = DH ? (BATCHES < 4 ? BATCHES : 4) : 1;
        Gates gates[AHEAD];
        auto load_gates = [&](Gates &v, int b) __attribute__((always_inline)) {
#pragma unroll
            for (int mi = 0; mi < TM; ++mi) {
                v.g[mi] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rg, offset(b, mi), 0, 0));
                v.u[mi] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ru, offset(b, mi), 0, 0));
            }
        };
        auto pack8 = [](const float (&v)[8]) __attribute__((always_inline)) {
            return u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        };
        // lo, hi: the two MFMA results of each run.
        auto emit = [&](int b, const f32x4 (&lo)[TM], const f32x4 (&hi)[TM]) __attribute__((always_inline)) {
            if constexpr (GATE_UP) {
#pragma unroll
                for (int mi = 0; mi < TMW; ++mi) {
                    float g[8], u[8], h[8];
                    wide_columns(lo[mi], hi[mi], g);
                    wide_columns(lo[TMW + mi], hi[TMW + mi], u);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        h[e] = gate_act(g[e], p.activation, p.beta) * u[e];
                    const uint32_t off = offset(b, mi);
                    if constexpr (SAVE) {
                        __builtin_amdgcn_raw_buffer_store_b128(pack8(g), rg, off, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(pack8(u), ru, off, 0, 0);
                    }
                    __builtin_amdgcn_raw_buffer_store_b128(pack8(h), ro, off, 0, 0);
                }
            } else {
                u32x4 c[TM];
#pragma unroll
                for (int mi = 0; mi < TM; ++mi) {
                    float v[8];
                    wide_columns(lo[mi], hi[mi], v);
                    if constexpr (DH) {
                        const uint32_t off = offset(b, mi);
                        const Gates &gu = gates[b % AHEAD];
                        u32x4 dg, du, h;
                        gate_gradients(v, gu.g[mi], gu.u[mi], p.activation, p.beta, dg, du, h);
                        __builtin_amdgcn_raw_buffer_store_b128(dg, rdg, off, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(du, rdu, off, 0, 0);
                        __builtin_amdgcn_raw_buffer_store_b128(h, rh, off, 0, 0);
                    } else {
                        c[mi] = pack8(v);
                    }
                }
                if constexpr (!DH && TM % 2 == 0) {
#pragma unroll
                    for (int mi = 0; mi < TM; mi += 2) {
                        store_lines(c[mi], c[mi + 1], lane);
#pragma unroll
                        for (int half = 0; half < 2; ++half)
                            __builtin_amdgcn_raw_buffer_store_b128(c[mi + half], ro, line_offset(b, mi, half), 0, OUT_POLICY);
                    }
                } else if constexpr (!DH) {
#pragma unroll
                    for (int mi = 0; mi < TM; ++mi)
                        __builtin_amdgcn_raw_buffer_store_b128(c[mi], ro, offset(b, mi), 0, OUT_POLICY);
                }
            }
            if constexpr (DH)
                if (b + AHEAD < BATCHES)
                    load_gates(gates[b % AHEAD], b + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto piece = [&](int b, int mi, int sa) __attribute__((always_inline)) { return acc[mi][b / 2].v[sa + 2 * (b % 2)]; };
        auto first_gates = [&]() __attribute__((always_inline)) {
            if constexpr (DH)
#pragma unroll
                for (int b = 0; b < AHEAD; ++b)
                    load_gates(gates[b], b);
        };

        if constexpr (!WEIGHTS) {
            if (splits > 1 && !whole) {
                // Partial sums out with device-coherent stores, [split][tile][wave]
                // [batch][piece][lane]; the last block of a tile reads them all back and
                // adds them in the order of the splits, whichever block it is.
                const __amdgpu_buffer_rsrc_t prs = make_rsrc(p.partial);
                const uint32_t lane_off = lane * 16;
                auto wave_base = [&](int sp) __attribute__((always_inline)) {
                    return (uint32_t)(((sp * rest + piece_tile) * S::NWAVES + wave) * S::PIECES) * 1024u; // tiles of any TX side by side
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
                    s_last = before == (uint32_t)(splits - 1);
                }
                __syncthreads();
                if (!s_last)
                    return;
                if (tid == 0)
                    __hip_atomic_store(p.counters + piece_tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                first_gates();
                // GROUP batches' sums at once: the loads of one split, of up to 20 pieces, are
                // in flight together, and each split costs their latency for every group.
                // Fewer beside the accumulators of a 256-row tile, which more would spill.
                constexpr int GROUP = [] {
                    int g = BATCHES, most = PIECES < 32 ? 20 : DH ? 4 : 8;
                    while (g * 2 * TM > most || BATCHES % g)
                        --g;
                    return g;
                }();
#pragma unroll
                for (int b0 = 0; b0 < BATCHES; b0 += GROUP) {
                    f32x4 sum[GROUP][2][TM];
                    for (int sp = 0; sp < splits; ++sp) {
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
    };
    // A tile whose rows end early leaves out the blocks behind them.  A weight that only one
    // tile of rows reads is streamed, and then the memory is read faster (us: 2 of 8
    // experts of 4096 x 14336 with a row each 122, through the L2 135; 8 with 4 rows each
    // 445 and 497).  Where several tiles read it the L2 is for it (streamed all the same: 8
    // experts of 1024 x 512, 60 rows each on tiles of 32, 19 us become 23).
    auto by_rows = [&]<bool STREAM_A>() __attribute__((always_inline)) {
        if constexpr (!WEIGHTS && TN > 1)
            if (N - n0 <= S::WN * 32)
                return run.template operator()<1, STREAM_A>();
        if constexpr (!WEIGHTS && TN > 2)
            if (N - n0 <= S::WN * 64)
                return run.template operator()<2, STREAM_A>();
        run.template operator()<TN, STREAM_A>();
    };
    if constexpr (!WEIGHTS)
        if (tiles_n == 1)
            return by_rows.template operator()<true>();
    by_rows.template operator()<false>();
}

} // namespace gmlp
