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
// The pipeline is that of the forward tiles (gemm_mfma.hpp): a ring of LDS
// stages filled by DMA, XOR-swizzled 16-byte chunks, v_mfma_f32_16x16x32_bf16
// fed by fragments read one k32 step ahead.  Bound by the rate at which operand
// tiles reach LDS (128 FLOP per staged byte for the 256 x 256 tiles) where there
// are many tokens, and by the weights' bytes where there are few.
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
    int M[3], N[3];   // output columns and rows
    int K;            // contracted elements of a segment
    int kt_seg;       // k-tiles of a segment
    int nk, kt_split, splits;
    int problem_tiles, tiles; // of one problem, of the launch
    float *partial;
    uint32_t *counters;
    // GRAD_GATE
    const uint16_t *g, *u;
    uint16_t *dg, *du, *h;
    int activation;
    float beta;
};

// Staging and fragment addresses of one operand's tiles of LINES lines x 64 k.
template <bool KC, int LINES, int NWAVES, int T>
struct GradOperand {
    static constexpr int LOADS = LINES * 128 / (NWAVES * 1024);
    static constexpr int CPR = LINES / 8;       // chunks of a line-contiguous LDS row
    static constexpr int ROW_BYTES = LINES * 2;
    static constexpr int LPR = 64 / CPR;        // such rows per wave load
    static constexpr int RPI = NWAVES * LPR;    // such rows per load step
    static_assert(KC || (RPI % 4 == 0 && (RPI >= 16 || 16 % RPI == 0)), "row bits 0, 1 and 4 of the swizzle");

    uint32_t voff[KC ? LOADS : 2];
    int kpos[KC ? LOADS : 1]; // KC: first k of the chunk; else: the row of load 0
    uint32_t soff_step;
    int frag[T][2];

    // Tile at line l0 of L lines, row stride ld elements; fragments from line
    // `first` of the tile on.
    __device__ __forceinline__ void init(int l0, int L, int ld, int first, int wave, int lane)
    {
        if constexpr (KC) {
            // LDS row r = line l0 + r, chunk position lane % 8 holding chunk
            // (lane % 8) ^ swizzle; lines past L are clamped to the last one
            // and feed only outputs that are not stored.
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = (i * NWAVES + wave) * 8 + (lane >> 3);
                const int c = (lane & 7) ^ x_swizzle(r);
                kpos[i] = c * 8;
                voff[i] = ((uint32_t)(min(l0 + r, L - 1) - l0) * (uint32_t)ld + (uint32_t)c * 8u) * 2u;
            }
            soff_step = 0;
        } else {
            const int k = wave * LPR + lane / CPR;
            kpos[0] = k;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int c = (lane % CPR) ^ w_swizzle<CPR, true>(k ^ (16 * b));
                voff[b] = l0 + c * 8 < L ? ((uint32_t)k * (uint32_t)ld + (uint32_t)c * 8u) * 2u : kOutOfRange;
            }
            soff_step = (uint32_t)RPI * (uint32_t)ld * 2u;
        }
        const int kg = ((lane >> 4) & 1) << 1 | (lane >> 5);
        const int r_lane = 8 * kg + ((lane & 15) >> 2);
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if constexpr (KC) {
                    const int r = first + 32 * i + 16 * s + (lane & 15);
                    frag[i][s] = r * 128 + ((kg ^ x_swizzle(r)) << 4);
                } else {
                    const int c = first / 8 + 4 * i + 2 * s + ((lane & 3) >> 1);
                    frag[i][s] = r_lane * ROW_BYTES + ((c ^ w_swizzle<CPR, true>(r_lane)) << 4) + (lane & 1) * 8;
                }
            }
    }

    // Where a tile starts in memory.
    __device__ __forceinline__ static const uint16_t *tile(const uint16_t *p, int l0, int k0, int ld)
    {
        return KC ? p + (size_t)l0 * ld + k0 : p + (size_t)k0 * ld + l0;
    }

    // The DMA of one k-tile: k past krem reads as zeros.
    __device__ __forceinline__ void issue(const uint16_t *at, uint8_t *buf, int krem, int wave) const
    {
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(at);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            uint32_t v;
            if constexpr (KC)
                v = kpos[i] >= krem ? kOutOfRange : voff[i];
            else
                v = i * RPI + kpos[0] >= krem ? kOutOfRange : voff[((i * RPI) >> 4) & 1];
            load16_to_lds(rs, buf + (i * NWAVES + wave) * 1024, v, (uint32_t)i * soff_step);
        }
    }

    __device__ __forceinline__ bf16x8 read(const uint8_t *buf, int kk, int i, int s) const
    {
        if constexpr (KC) {
            return *(const bf16x8 *)(buf + (frag[i][s] ^ (64 * kk)));
        } else {
            const uint8_t *p = buf + kk * 32 * ROW_BYTES + frag[i][s];
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)GMLP_LDS(p));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) i16x4 *)GMLP_LDS(p + 4 * ROW_BYTES));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

// dG, dU and H of four neighbouring elements.
__device__ __forceinline__ void gate_gradients(const f32x4 &dh, const u32x2 &g2, const u32x2 &u2, int act, float beta,
                                               u32x2 &dg2, u32x2 &du2, u32x2 &h2)
{
    float dg[4], du[4], h[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = e & 1 ? bf16_hi(g2[e >> 1]) : bf16_lo(g2[e >> 1]);
        const float u = e & 1 ? bf16_hi(u2[e >> 1]) : bf16_lo(u2[e >> 1]);
        const float s = __builtin_amdgcn_rcpf(1.0f + __expf(-(beta * g)));
        const float c = s * (1.0f - s); // sigmoid'
        const bool glu = act == ACT_SIGMOID;
        const float a = glu ? s : g * s;
        const float da = glu ? c : s + beta * g * c;
        h[e] = a * u;
        du[e] = dh[e] * a;
        dg[e] = dh[e] * u * da;
    }
    dg2 = u32x2{pack_bf16x2(dg[0], dg[1]), pack_bf16x2(dg[2], dg[3])};
    du2 = u32x2{pack_bf16x2(du[0], du[1]), pack_bf16x2(du[2], du[3])};
    h2 = u32x2{pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3])};
}

// One block: one output tile, or one split of its k-tiles.  KC: both operands
// k-contiguous; SEGS = 2: dX's two pairs; otherwise a problem per range of
// problem_tiles tiles.
template <class S, bool KC, int EPI, int SEGS>
__global__ __launch_bounds__(S::NTHREADS, 1) void gemm_grad_kernel(GradParams p)
{
    constexpr int TM = S::TM, TN = S::TN, STAGES = S::STAGES;
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

    // Block -> split, problem and tile; neighbouring tiles, which share operand
    // strips, on one XCD (gemm_mfma.hpp), in sweeps of 8 column tiles.
    const int id = xcd_contiguous_id(blockIdx.x, p.tiles * p.splits);
    const int split = id / p.tiles, tile = id - split * p.tiles;
    const int prob = SEGS == 1 ? tile / p.problem_tiles : 0;
    const int local = tile - prob * p.problem_tiles;
    const int M = p.M[prob], N = p.N[prob], K = p.K;
    const int tiles_m = (M + S::BM - 1) / S::BM, tiles_n = (N + S::BN - 1) / S::BN;
    const int per_group = 8 * tiles_n;
    const int group = local / per_group, in_group = local - group * per_group;
    const int group_w = min(tiles_m - group * 8, 8);
    const int m0 = (group * 8 + in_group % group_w) * S::BM, n0 = (in_group / group_w) * S::BN;
    const int kt_begin = split * p.kt_split, kt_end = min(p.nk, kt_begin + p.kt_split);
    const int nk = kt_end - kt_begin;
    const int lda = KC ? K : M, ldb = KC ? K : N;

    GradOperand<KC, S::BM, S::NWAVES, TM> opa;
    GradOperand<KC, S::BN, S::NWAVES, TN> opb;
    opa.init(m0, M, lda, wm * TM * 32, wave, lane);
    opb.init(n0, N, ldb, wn * TN * 32, wave, lane);

    // A k-tile past the end reads zeros only, so that every step has the same
    // number of loads in flight.
    auto issue = [&](uint8_t *buf, int i) __attribute__((always_inline)) {
        const int kt = kt_begin + i;
        const int seg = SEGS == 2 && kt >= p.kt_seg ? 1 : 0;
        const int k0 = i < nk ? (kt - seg * p.kt_seg) * S::BK : 0;
        const int krem = i < nk ? K - k0 : 0;
        const int q = SEGS == 2 ? seg : prob;
        opa.issue(opa.tile(p.a[q], m0, k0, lda), buf, krem, wave);
        opb.issue(opb.tile(p.b[q], n0, k0, ldb), buf + S::A_BYTES, krem, wave);
    };

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
        bf16x8 a[TM][2];
    };
    struct FragB {
        bf16x8 b[TN][2];
    };
    auto mma_roll = [&](const FragA &fa, FragA &fa_next, FragB &fb, const uint8_t *nbuf, int nkk)
                        __attribute__((always_inline)) {
        constexpr int GROUPS = TN * 2, AFRAGS = TM * 2, APG = (AFRAGS + GROUPS - 1) / GROUPS;
        [&]<int... G>(std::integer_sequence<int, G...>) __attribute__((always_inline)) {
            (
                [&] {
                    constexpr int ni = G / 2, sb = G % 2;
#pragma unroll
                    for (int mi = 0; mi < TM; ++mi)
#pragma unroll
                        for (int sa = 0; sa < 2; ++sa)
                            acc[mi][ni].v[sa + 2 * sb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                                fa.a[mi][sa], fb.b[ni][sb], acc[mi][ni].v[sa + 2 * sb], 0, 0, 0);
#pragma unroll
                    for (int q = G * APG; q < (G + 1) * APG && q < AFRAGS; ++q)
                        fa_next.a[q / 2][q % 2] = opa.read(nbuf, nkk, q / 2, q % 2);
                    fb.b[ni][sb] = opb.read(nbuf + S::A_BYTES, nkk, ni, sb);
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

    FragA fa0, fa1;
    FragB fb;
    [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
        (issue(stage_ptr(std::integral_constant<int, I>{}), I), ...);
    }(std::make_integer_sequence<int, STAGES - 1>{});
    wait_tile();
    issue(stage_ptr(std::integral_constant<int, STAGES - 1>{}), STAGES - 1);
    {
        const uint8_t *buf = lds0;
#pragma unroll
        for (int q = 0; q < TM * 2; ++q)
            fa0.a[q / 2][q % 2] = opa.read(buf, 0, q / 2, q % 2);
#pragma unroll
        for (int q = 0; q < TN * 2; ++q)
            fb.b[q / 2][q % 2] = opb.read(buf + S::A_BYTES, 0, q / 2, q % 2);
    }
    // A k-tile in stage I: its second k32 step's fragments are read among the
    // first's MFMAs; then a barrier frees the stage for the DMA of tile
    // i + STAGES, and the next tile's first fragments are read.
    auto step = [&](auto stage, int i) __attribute__((always_inline)) {
        constexpr int I = decltype(stage)::value;
        uint8_t *buf = stage_ptr(stage);
        uint8_t *next = stage_ptr(std::integral_constant<int, (I + 1) % STAGES>{});
        mma_roll(fa0, fa1, fb, buf, 1);
        wait_tile();
        issue(buf, i + STAGES);
        mma_roll(fa1, fa0, fb, next, 0);
    };
    int i = 0;
    for (; i + STAGES <= nk; i += STAGES) {
        [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
            (step(std::integral_constant<int, I>{}, i + I), ...);
        }(std::make_integer_sequence<int, STAGES>{});
    }
    [&]<int... I>(std::integer_sequence<int, I...>) __attribute__((always_inline)) {
        ((i + I < nk ? step(std::integral_constant<int, I>{}, i + I) : void()), ...);
    }(std::make_integer_sequence<int, STAGES - 1>{});
    wait_vmcnt<0>(); // loads past the end, before LDS is given to another block

    // ---- outputs ---------------------------------------------------------------
    // Piece g = (mi * TN + ni) * 4 + j: 4 consecutive columns of one row.
    const __amdgpu_buffer_rsrc_t ro = make_rsrc(EPI == GRAD_STORE ? p.out[prob] + (size_t)n0 * M + m0 : nullptr);
    const __amdgpu_buffer_rsrc_t rg = make_rsrc(EPI == GRAD_GATE ? p.g + (size_t)n0 * M + m0 : nullptr);
    const __amdgpu_buffer_rsrc_t ru = make_rsrc(EPI == GRAD_GATE ? p.u + (size_t)n0 * M + m0 : nullptr);
    const __amdgpu_buffer_rsrc_t rdg = make_rsrc(EPI == GRAD_GATE ? p.dg + (size_t)n0 * M + m0 : nullptr);
    const __amdgpu_buffer_rsrc_t rdu = make_rsrc(EPI == GRAD_GATE ? p.du + (size_t)n0 * M + m0 : nullptr);
    const __amdgpu_buffer_rsrc_t rh = make_rsrc(EPI == GRAD_GATE ? p.h + (size_t)n0 * M + m0 : nullptr);
    auto offset = [&](int g) __attribute__((always_inline)) {
        const int mi = g / (4 * TN), ni = g / 4 % TN, j = g % 4;
        const int ml = wm * TM * 32 + mi * 32 + Acc::col(j, lane), nl = wn * TN * 32 + ni * 32 + Acc::tok(j, lane);
        return n0 + nl < N && m0 + ml < M ? ((uint32_t)nl * (uint32_t)M + (uint32_t)ml) * 2u : kOutOfRange;
    };
    // CH pieces at once, so that their loads and stores overlap.
    constexpr int CH = 8;
    static_assert(S::PIECES % CH == 0, "whole passes");
    auto emit = [&](int c0, const f32x4 (&v)[CH]) __attribute__((always_inline)) {
        if constexpr (EPI == GRAD_GATE) {
            u32x2 g[CH], u[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                g[c] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rg, offset(c0 + c), 0, 0));
                u[c] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(ru, offset(c0 + c), 0, 0));
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                u32x2 dg, du, h;
                gate_gradients(v[c], g[c], u[c], p.activation, p.beta, dg, du, h);
                const uint32_t off = offset(c0 + c);
                __builtin_amdgcn_raw_buffer_store_b64(dg, rdg, off, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b64(du, rdu, off, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b64(h, rh, off, 0, 0);
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c)
                __builtin_amdgcn_raw_buffer_store_b64(u32x2{pack_bf16x2(v[c][0], v[c][1]), pack_bf16x2(v[c][2], v[c][3])},
                                                      ro, offset(c0 + c), 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto piece = [&](int g) __attribute__((always_inline)) { return acc[g / (4 * TN)][g / 4 % TN].piece(g % 4); };

    if (p.splits > 1) {
        // Partial sums out with device-coherent stores, [split][tile][wave]
        // [piece][lane]; the last block of a tile reads them all back and adds
        // them in the order of the splits, whichever block it is.
        const __amdgpu_buffer_rsrc_t prs = make_rsrc(p.partial);
        const uint32_t lane_off = lane * 16;
        auto wave_base = [&](int sp) __attribute__((always_inline)) {
            return (uint32_t)(((sp * p.tiles + tile) * S::NWAVES + wave) * S::PIECES) * 1024u;
        };
        const uint32_t own = wave_base(split);
#pragma unroll
        for (int g = 0; g < S::PIECES; ++g)
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, piece(g)), prs, lane_off, own + g * 1024u,
                                                   kCoherent);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) {
            const uint32_t before = __hip_atomic_fetch_add(p.counters + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)(p.splits - 1);
        }
        __syncthreads();
        if (!s_last)
            return;
        if (tid == 0)
            __hip_atomic_store(p.counters + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int c0 = 0; c0 < S::PIECES; c0 += CH) {
            f32x4 sum[CH];
            for (int sp = 0; sp < p.splits; ++sp) {
                const uint32_t base = wave_base(sp);
                f32x4 x[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    x[c] = __builtin_bit_cast(
                        f32x4, __builtin_amdgcn_raw_buffer_load_b128(prs, lane_off, base + (c0 + c) * 1024u, kCoherent));
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    sum[c] = sp == 0 ? x[c] : sum[c] + x[c];
            }
            emit(c0, sum);
        }
        return;
    }
#pragma unroll
    for (int c0 = 0; c0 < S::PIECES; c0 += CH) {
        f32x4 v[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c)
            v[c] = piece(c0 + c);
        emit(c0, v);
    }
}

} // namespace gmlp
