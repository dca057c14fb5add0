// Products with 4-bit weights (include/gmlp_w4.h) for gfx950.
//
// Y[t, n] = sum_k X[t, k] (q[k, n] - z) s for few tokens t, bound by the bytes of
// q.  The arithmetic follows from making the matrix cores do all of it:
//
//   * A 4-bit q in the low mantissa bits of a bf16 one is the bf16 number
//     1 + q / 128, exactly: one v_and_or_b32 makes two weights, 7 VALU
//     instructions 8 of them.
//   * sum x (q - z) / 128 = sum x (1 + q / 128) - sum x (1 + z / 128).  The second
//     sum is an MFMA with a constant operand; its result is the accumulator the
//     first starts from.  Without zero points (z = 8) it is shared by all columns.
//   * v_mfma_f32_16x16x32_bf16 with X as operand A (16 tokens) and the weights as
//     B: a lane then holds results of one column, so a group's scale is one
//     number per lane and one FMA per result.  Tokens sit at rows 0, 4, 8, 12, 1,
//     5, ...: up to 4 tokens use one result register of the four.
//
// Packed layout: tiles of 128 rows x 16 columns, 1 KB each, k-tiles of a column
// tile consecutive.  Lane l of a wave reads 16 bytes, column l % 16; its dword j
// holds rows 32 j + 8 (l / 16) .. + 7, the operand of MFMA j, row e in bits
// 4 (e / 2) + 16 (e % 2).  So a wave streams 1 KB per load, in order, straight
// into registers.  Scales [tile][column][group of the tile], zero points likewise.
//
// A block of 8 waves computes CT column tiles (of both weights for gate/up), each
// wave a contiguous range of the block's k-tiles with several of them in flight; the
// waves' sums are added in order through LDS, and where there are few column tiles
// those of several blocks over k through the workspace.  From 16 tokens on, where k is
// long, w4_shared_kernel.
// Measured, D = 4096, F = 14336, groups of 128: T = 1 gate/up 14.6 us (60.6 MB, 4.2 TB/s),
// down 7.6 us (30.3 MB, 4.0 TB/s); T = 8 15.7 and 10.0 us.  A launch and the sums take
// about 4 us of each; at T = 5 and above the unpacking and the MFMAs of a CU's blocks
// are as long as its loads.
#pragma once

#include "common.hpp"

namespace gmlp {

struct W4Params {
    const uint16_t *x;       // [T, K]
    const uint8_t *tiles[2]; // packed weights
    const uint8_t *scales[2], *zeros[2];
    uint16_t *out;           // [T, N]
    float *partial;          // [split][strip][slot][lane]
    uint32_t *counters;      // one per strip, zero on entry and exit
    int T, K, N;
    int ktiles;              // tiles of 128 rows
    int strips, splits;      // column strips of CT tiles; blocks over k of each
    int split_ktiles;        // k-tiles of a block
    int activation;
    float beta;
};

constexpr uint32_t kW4Nibbles = 0x000f000fu, kW4One = 0x3f803f80u;
constexpr uint32_t kW4MinusMid = 0xbf88bf88u; // -(1 + 8 / 128), twice

// The k-tile's scales (or zero points) of one column, G of them.
template <int G>
struct W4Group;
template <>
struct W4Group<1> {
    typedef uint16_t scales;
    typedef uint8_t zeros;
    __device__ static uint32_t scale(scales s, int) { return (uint32_t)s << 16; }
    __device__ static uint32_t zero(zeros z, int) { return z; }
};
template <>
struct W4Group<2> {
    typedef uint32_t scales;
    typedef uint16_t zeros;
    __device__ static uint32_t scale(scales s, int g) { return g ? s & 0xffff0000u : s << 16; }
    __device__ static uint32_t zero(zeros z, int g) { return z >> (8 * g) & 0xffu; }
};
template <>
struct W4Group<4> {
    typedef u32x2 scales;
    typedef uint32_t zeros;
    __device__ static uint32_t scale(const scales &s, int g) { return g & 1 ? s[g >> 1] & 0xffff0000u : s[g >> 1] << 16; }
    __device__ static uint32_t zero(zeros z, int g) { return z >> (8 * g) & 0xffu; }
};

// Eight weights 1 + q / 128 of one packed dword.
__device__ __forceinline__ bf16x8 w4_unpack(uint32_t d)
{
    return __builtin_bit_cast(bf16x8, u32x4{(d & kW4Nibbles) | kW4One, (d >> 4 & kW4Nibbles) | kW4One,
                                            (d >> 8 & kW4Nibbles) | kW4One, (d >> 12 & kW4Nibbles) | kW4One});
}

// TOK: tokens, rounded up to 4, 8 or a multiple of 16.  GPT: scale groups per k-tile
// (128 / group).  DEPTH: k-tiles of a wave in flight.
//
// Up to 8 tokens the rows of a k-tile, 1 or 2 KB, are loaded as they lie and reach
// the MFMA layout through LDS: loaded in that layout, with 16 lanes for every token
// that is not there, they would take four times the weights' loads.
template <int TOK, int NW, int CT, int GPT, bool ZEROS, int WAVES, int DEPTH>
__global__ __launch_bounds__(WAVES * 64, 8 / WAVES) void w4_kernel(W4Params p)
{
    constexpr int NB = (TOK + 15) / 16, NR = TOK >= 16 ? 4 : TOK / 4, MPG = 4 / GPT;
    constexpr int SLOTS = NW * CT * NB * NR; // results per lane
    constexpr bool VIA_LDS = TOK <= 8;
    constexpr int X_REGS = VIA_LDS ? TOK / 4 : NB * 4; // 16-byte registers of a k-tile of X
    using Group = W4Group<GPT>;
    __shared__ float part[WAVES * SLOTS * 64];
    __shared__ __attribute__((aligned(256))) uint8_t rows[VIA_LDS ? WAVES * TOK * 256 : 16];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int K = p.K, ntiles = (p.N + 15) >> 4;
    const int strip = blockIdx.x % p.strips, split = blockIdx.x / p.strips;
    const int first = strip * CT;
    const int split_begin = split * p.split_ktiles, split_end = min(p.ktiles, split_begin + p.split_ktiles);
    const int per = (split_end - split_begin + WAVES - 1) / WAVES;
    const int begin = split_begin + wave * per, end = min(split_end, begin + per);

    // Row r of operand A is token r / 4 + 4 (r % 4) of its 16.  Tokens past T repeat
    // the last one and feed results that are not stored.
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x);
    const int kq = lane >> 4, row = lane & 15;
    uint32_t x_off[VIA_LDS ? X_REGS : NB];
    int x_read = 0, x_write = 0;
    if constexpr (VIA_LDS) {
        // Register i: token 4 i + lane / 16, chunk lane % 16 (8 k).  In LDS a token's
        // chunks are XORed with the token so that the reads of different tokens
        // do not meet on a bank.
#pragma unroll
        for (int i = 0; i < X_REGS; ++i)
            x_off[i] = ((uint32_t)min(4 * i + kq, p.T - 1) * (uint32_t)K + 8u * row) * 2u;
        const int t = (row >> 2) + 4 * ((row & 3) % NR);
        x_write = wave * TOK * 256 + kq * 256 + ((row ^ kq << 2) << 4);
        x_read = wave * TOK * 256 + t * 256 + ((kq ^ (t & 3) << 2) << 4);
    } else {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            x_off[nb] = ((uint32_t)min(16 * nb + (row >> 2) + 4 * (row & 3), p.T - 1) * (uint32_t)K + 8u * kq) * 2u;
    }
    size_t tile[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
        tile[c] = (size_t)min(first + c, ntiles - 1) * p.ktiles;

    struct Batch {
        u32x4 w[NW][CT];
        typename Group::scales s[NW][CT];
        typename Group::zeros z[ZEROS ? NW : 1][ZEROS ? CT : 1];
        u32x4 x[X_REGS];
    };
    auto load = [&](Batch &b, int kt) __attribute__((always_inline)) {
        kt = min(kt, p.ktiles - 1); // past the end: loaded, not used
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const size_t at = tile[c] + kt;
                b.w[w][c] = __builtin_nontemporal_load((const u32x4 *)(p.tiles[w] + at * 1024 + lane * 16));
                b.s[w][c] = ((const typename Group::scales *)p.scales[w])[at * 16 + row];
                if constexpr (ZEROS)
                    b.z[w][c] = ((const typename Group::zeros *)p.zeros[w])[at * 16 + row];
            }
#pragma unroll
        for (int i = 0; i < X_REGS; ++i) {
            // Columns of X past K read as zeros: rows past K of the weight count
            // for nothing.
            const int k = kt * 128 + (VIA_LDS ? 0 : 32 * (i % 4));
            const uint32_t off = k + 8 * (VIA_LDS ? row : kq) < K ? x_off[VIA_LDS ? i : i / 4] + (uint32_t)k * 2u : kOutOfRange;
            b.x[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, off, 0, 0));
        }
    };
    float total[NW][CT][NB][NR] = {};
    const auto constant = [](uint32_t v) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, u32x4{v, v, v, v});
    };
    auto use = [&](const Batch &b) __attribute__((always_inline)) {
        bf16x8 x[NB][4];
        if constexpr (VIA_LDS) {
            // The wave's own rows: its LDS operations run in order, and the fences
            // tell the compiler that other lanes' rows are read (no instruction).
            wave_lds_fence();
#pragma unroll
            for (int i = 0; i < X_REGS; ++i)
                *(u32x4 *)(rows + x_write + i * 1024) = b.x[i];
            wave_lds_fence();
#pragma unroll
            for (int j = 0; j < 4; ++j)
                x[0][j] = *(const bf16x8 *)(rows + (x_read ^ j << 6));
        } else {
#pragma unroll
            for (int i = 0; i < X_REGS; ++i)
                x[i / 4][i % 4] = __builtin_bit_cast(bf16x8, b.x[i]);
        }
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            f32x4 mid[NB];
            if constexpr (!ZEROS)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb) {
                    mid[nb] = f32x4{};
#pragma unroll
                    for (int m = 0; m < MPG; ++m)
                        mid[nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[nb][g * MPG + m], constant(kW4MinusMid),
                                                                          mid[nb], 0, 0, 0);
                }
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    bf16x8 q[MPG];
#pragma unroll
                    for (int m = 0; m < MPG; ++m)
                        q[m] = w4_unpack(b.w[w][c][g * MPG + m]);
                    const float s = __builtin_bit_cast(float, Group::scale(b.s[w][c], g));
#pragma unroll
                    for (int nb = 0; nb < NB; ++nb) {
                        f32x4 acc;
                        if constexpr (ZEROS) {
                            const uint32_t z = 0xbf80u | Group::zero(b.z[w][c], g); // -(1 + z / 128)
                            acc = f32x4{};
#pragma unroll
                            for (int m = 0; m < MPG; ++m)
                                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[nb][g * MPG + m], constant(z | z << 16),
                                                                              acc, 0, 0, 0);
                        } else {
                            acc = mid[nb];
                        }
#pragma unroll
                        for (int m = 0; m < MPG; ++m)
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[nb][g * MPG + m], q[m], acc, 0, 0, 0);
#pragma unroll
                        for (int i = 0; i < NR; ++i)
                            total[w][c][nb][i] += s * acc[i];
                    }
                }
        }
    };

    Batch batch[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        load(batch[d], begin + d);
    int kt = begin;
    for (; kt + DEPTH < end; kt += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            use(batch[d]);
            load(batch[d], kt + d + DEPTH);
        }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d)
        if (kt + d < end)
            use(batch[d]);

    // ---- sums of the waves, in order ---------------------------------------------
#pragma unroll
    for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < NR; ++i)
                    part[(wave * SLOTS + ((w * CT + c) * NB + nb) * NR + i) * 64 + lane] = total[w][c][nb][i];
    __syncthreads();
    auto block_sum = [&](int slot) __attribute__((always_inline)) {
        float v = part[slot * 64 + lane];
#pragma unroll
        for (int o = 1; o < WAVES; ++o)
            v += part[(o * SLOTS + slot) * 64 + lane];
        return v;
    };
    // ---- and of the blocks over k -------------------------------------------------
    // Written through to memory (device-coherent), counted in, and added in order by
    // the last block of the strip.
    const __amdgpu_buffer_rsrc_t prs = make_rsrc(p.partial);
    auto partial_at = [&](int sp, int slot) __attribute__((always_inline)) {
        return (uint32_t)((sp * p.strips + strip) * SLOTS + slot) * 256u;
    };
    if (p.splits > 1) {
        for (int slot = wave; slot < SLOTS; slot += WAVES)
            __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, block_sum(slot)), prs, lane * 4,
                                                  partial_at(split, slot), kCoherent);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) {
            const uint32_t before =
                __hip_atomic_fetch_add(p.counters + strip, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)(p.splits - 1);
        }
        __syncthreads();
        if (!s_last)
            return;
        if (tid == 0)
            __hip_atomic_store(p.counters + strip, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    constexpr int OUT = CT * NB * NR; // result slots of one weight
    for (int slot = wave; slot < OUT; slot += WAVES) {
        float v[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const int at = w * OUT + slot;
            if (p.splits > 1) {
                v[w] = 0.0f;
                for (int sp = 0; sp < p.splits; ++sp)
                    v[w] += __builtin_bit_cast(float, (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(
                                                          prs, lane * 4, partial_at(sp, at), kCoherent));
            } else {
                v[w] = block_sum(at);
            }
            v[w] *= 128.0f; // the weights were (q - z) / 128
        }
        const int i = slot % NR, nb = slot / NR % NB, c = slot / (NR * NB);
        const int t = 16 * nb + kq + 4 * i, n = (first + c) * 16 + row;
        if (t < p.T && n < p.N) {
            const float y = NW == 2 ? gate_act(v[0], p.activation, p.beta) * v[NW - 1] : v[0];
            p.out[(size_t)t * p.N + n] = __builtin_bit_cast(uint16_t, (__bf16)y);
        }
    }
}

// ---- more tokens: X shared by the waves of a block ----------------------------------
// A block of 4 waves computes 64 columns (of both weights for gate/up), 16 per wave,
// over all the block's k-tiles: for 16 tokens and more, where k is long.  A k-tile of X, 16 NB tokens, is loaded once by the
// block and read by the four waves from LDS; it would otherwise be loaded in the MFMA
// layout by every wave, 4 NB KB for each KB of a weight tile.  LDS holds two k-tiles, X
// is XD of them ahead in registers and the weights DEPTH.  What bounds it is the MFMAs
// (a third of them for the zero point) and the LDS reads of a step one after the other:
// 2 blocks to a CU, or the two sums of a group in separate registers, gain nothing.
//
// LDS rows of one token, 16 chunks of 8 k, chunk c at position c ^ token % 16: the 16
// lanes that read one chunk of 16 tokens meet all banks.
constexpr int kW4SharedWaves = 4, kW4SharedColumns = 16 * kW4SharedWaves;
template <int NB, int NW, int GPT, bool ZEROS, int DEPTH>
__global__ __launch_bounds__(kW4SharedWaves * 64, 1) void w4_shared_kernel(W4Params p)
{
    constexpr int MPG = 4 / GPT, XD = 2;
    using Group = W4Group<GPT>;
    __shared__ __attribute__((aligned(256))) uint8_t rows[2][NB * 16 * 256];
    __shared__ int s_last;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int K = p.K, ntiles = (p.N + 15) >> 4;
    const int strip = blockIdx.x % p.strips, split = blockIdx.x / p.strips;
    const int begin = split * p.split_ktiles, end = min(p.ktiles, begin + p.split_ktiles);
    const int kq = lane >> 4, row = lane & 15;
    const int column_tile = strip * kW4SharedWaves + wave;
    const size_t tile = (size_t)min(column_tile, ntiles - 1) * p.ktiles;

    // X: thread t brings chunk t % 16 of tokens t / 16 + 16 nb; tokens past T and
    // columns past K read as zeros.
    const __amdgpu_buffer_rsrc_t rx = make_rsrc(p.x);
    const int x_token = tid >> 4, x_chunk = tid & 15;
    const int x_write = x_token * 256 + ((x_chunk ^ x_token) << 4);
    struct Rows {
        u32x4 v[NB];
    };
    auto load_rows = [&](Rows &r, int kt) __attribute__((always_inline)) {
        const int k = kt * 128 + x_chunk * 8;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            const int t = x_token + 16 * nb;
            const uint32_t off = k < K && t < p.T ? ((uint32_t)t * (uint32_t)K + (uint32_t)k) * 2u : kOutOfRange;
            r.v[nb] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rx, off, 0, 0));
        }
    };
    auto store_rows = [&](const Rows &r, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
            *(u32x4 *)(rows[stage] + x_write + nb * 16 * 256) = r.v[nb];
    };
    const int x_read = row * 256 + ((kq ^ row) << 4); // chunk 4 j + kq: XOR 64 j

    struct Batch {
        u32x4 w[NW];
        typename Group::scales s[NW];
        typename Group::zeros z[ZEROS ? NW : 1];
    };
    auto load = [&](Batch &b, int kt) __attribute__((always_inline)) {
        const size_t at = tile + min(kt, p.ktiles - 1); // past the end: loaded, not used
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            b.w[w] = __builtin_nontemporal_load((const u32x4 *)(p.tiles[w] + at * 1024 + lane * 16));
            b.s[w] = ((const typename Group::scales *)p.scales[w])[at * 16 + row];
            if constexpr (ZEROS)
                b.z[w] = ((const typename Group::zeros *)p.zeros[w])[at * 16 + row];
        }
    };
    f32x4 total[NW][NB] = {};
    const auto constant = [](uint32_t v) __attribute__((always_inline)) {
        return __builtin_bit_cast(bf16x8, u32x4{v, v, v, v});
    };
    auto use = [&](const Batch &b, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < GPT; ++g) {
            bf16x8 q[NW][MPG];
            float s[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                s[w] = __builtin_bit_cast(float, Group::scale(b.s[w], g));
#pragma unroll
                for (int m = 0; m < MPG; ++m)
                    q[w][m] = w4_unpack(b.w[w][g * MPG + m]);
            }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
                bf16x8 x[MPG];
#pragma unroll
                for (int m = 0; m < MPG; ++m)
                    x[m] = *(const bf16x8 *)(rows[stage] + nb * 16 * 256 + (x_read ^ (g * MPG + m) << 6));
                f32x4 mid{};
                if constexpr (!ZEROS)
#pragma unroll
                    for (int m = 0; m < MPG; ++m)
                        mid = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[m], constant(kW4MinusMid), mid, 0, 0, 0);
#pragma unroll
                for (int w = 0; w < NW; ++w) {
                    f32x4 acc = mid;
                    if constexpr (ZEROS) {
                        const uint32_t z = 0xbf80u | Group::zero(b.z[w], g); // -(1 + z / 128)
#pragma unroll
                        for (int m = 0; m < MPG; ++m)
                            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[m], constant(z | z << 16), acc, 0, 0, 0);
                    }
#pragma unroll
                    for (int m = 0; m < MPG; ++m)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[m], q[w][m], acc, 0, 0, 0);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        total[w][nb][i] += s[w] * acc[i];
                }
            }
        }
    };

    // Step kt: the rows of kt + 1 go to the other stage, those of kt + 1 + XD and the
    // weights of kt + DEPTH are asked for, kt is multiplied.  The barrier at its end
    // (after this wave's LDS reads and writes) hands both stages over.
    static_assert(DEPTH % XD == 0, "the rows' registers go round with the weights'");
    Batch batch[DEPTH];
    Rows ahead[XD];
    {
        Rows now;
        load_rows(now, begin);
#pragma unroll
        for (int d = 0; d < XD; ++d)
            load_rows(ahead[d], begin + 1 + d);
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            load(batch[d], begin + d);
        store_rows(now, 0);
    }
    wait_lgkm0();
    barrier_only();
    auto step = [&](int kt, int d) __attribute__((always_inline)) {
        const int stage = (kt - begin) & 1;
        store_rows(ahead[d % XD], stage ^ 1);
        load_rows(ahead[d % XD], kt + 1 + XD);
        use(batch[d], stage);
        load(batch[d], kt + DEPTH);
        wait_lgkm0();
        barrier_only();
    };
    int kt = begin;
    for (; kt + DEPTH <= end; kt += DEPTH)
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            step(kt + d, d);
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d)
        if (kt + d < end)
            step(kt + d, d);

    // ---- the blocks over k, in order (as w4_kernel) --------------------------------
    if (p.splits > 1) {
        const __amdgpu_buffer_rsrc_t prs = make_rsrc(p.partial);
        auto partial_at = [&](int sp, int w, int nb) __attribute__((always_inline)) {
            return (uint32_t)((((sp * p.strips + strip) * kW4SharedWaves + wave) * NW + w) * NB + nb) * 1024u;
        };
#pragma unroll
        for (int w = 0; w < NW; ++w)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, total[w][nb]), prs, lane * 16,
                                                       partial_at(split, w, nb), kCoherent);
        wait_vmcnt<0>();
        __syncthreads();
        if (tid == 0) {
            const uint32_t before =
                __hip_atomic_fetch_add(p.counters + strip, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            s_last = before == (uint32_t)(p.splits - 1);
        }
        __syncthreads();
        if (!s_last)
            return;
        if (tid == 0)
            __hip_atomic_store(p.counters + strip, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        for (int sp = 0; sp < p.splits; ++sp) {
            f32x4 x[NW][NB];
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    x[w][nb] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(prs, lane * 16,
                                                                                              partial_at(sp, w, nb), kCoherent));
#pragma unroll
            for (int w = 0; w < NW; ++w)
#pragma unroll
                for (int nb = 0; nb < NB; ++nb)
                    total[w][nb] = sp == 0 ? x[w][nb] : total[w][nb] + x[w][nb];
        }
    }
    const int n = column_tile * 16 + row;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 16 * nb + 4 * kq + i;
            const float a = total[0][nb][i] * 128.0f, b = total[NW - 1][nb][i] * 128.0f; // (q - z) / 128 so far
            if (t < p.T && n < p.N)
                p.out[(size_t)t * p.N + n] =
                    __builtin_bit_cast(uint16_t, (__bf16)(NW == 2 ? gate_act(a, p.activation, p.beta) * b : a));
        }
}

// ---- laying out, rounding and restoring weights -----------------------------------
// Once per weight; [4096, 14336], groups of 128: rounding 98 us, layout 46, restoring 26
// ([14336, 4096] 51: a wave writes 16 columns of a row, 32 bytes).

struct W4LayoutParams {
    uint8_t *tiles, *scales, *zeros; // packed
    uint8_t *q, *z;                  // [K, N], [groups, N]
    uint16_t *s, *w;                 // [groups, N], [K, N]
    int K, N, group, ktiles, ntiles;
};

// Thread i of the layout kernels: lane i % 64 of tile i / 64.
__global__ __launch_bounds__(256) void w4_pack_kernel(W4LayoutParams p)
{
    const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t tile = id >> 6;
    if (tile >= (size_t)p.ktiles * p.ntiles)
        return;
    const int lane = id & 63, kt = tile % p.ktiles, n = (int)(tile / p.ktiles) * 16 + (lane & 15);
    u32x4 out{};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t d = 0;
        for (int e = 0; e < 8; ++e) {
            const int k = kt * 128 + 32 * j + 8 * (lane >> 4) + e;
            if (k < p.K && n < p.N)
                d |= (uint32_t)(p.q[(size_t)k * p.N + n] & 15) << (4 * (e >> 1) + 16 * (e & 1));
        }
        out[j] = d;
    }
    *(u32x4 *)(p.tiles + id * 16) = out;
    if (lane < 16) {
        const int gpt = 128 / p.group, groups = (p.K + p.group - 1) / p.group;
        for (int g = 0; g < gpt; ++g) {
            const int at = kt * gpt + g;
            const bool in = at < groups && n < p.N;
            const size_t to = (tile * 16 + lane) * gpt + g;
            ((uint16_t *)p.scales)[to] = in ? p.s[(size_t)at * p.N + n] : 0;
            if (p.zeros)
                p.zeros[to] = in ? p.z[(size_t)at * p.N + n] & 15 : 0;
        }
    }
}

__global__ __launch_bounds__(256) void w4_dequantize_kernel(W4LayoutParams p)
{
    const size_t id = (size_t)blockIdx.x * 256 + threadIdx.x;
    const size_t tile = id >> 6;
    if (tile >= (size_t)p.ktiles * p.ntiles)
        return;
    const int lane = id & 63, kt = tile % p.ktiles, n = (int)(tile / p.ktiles) * 16 + (lane & 15);
    if (n >= p.N)
        return;
    const u32x4 in = *(const u32x4 *)(p.tiles + id * 16);
    const int gpt = 128 / p.group;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const size_t at = (tile * 16 + (lane & 15)) * gpt + 32 * j / p.group;
        const uint32_t sb = ((const uint16_t *)p.scales)[at];
        const float s = __builtin_bit_cast(float, sb << 16);
        const int z = p.zeros ? p.zeros[at] : 8;
        for (int e = 0; e < 8; ++e) {
            const int k = kt * 128 + 32 * j + 8 * (lane >> 4) + e;
            const int q = in[j] >> (4 * (e >> 1) + 16 * (e & 1)) & 15;
            if (k < p.K)
                p.w[(size_t)k * p.N + n] = __builtin_bit_cast(uint16_t, (__bf16)((float)(q - z) * s));
        }
    }
}

// One thread per column and group; the groups' blocks follow one another.
__global__ __launch_bounds__(256) void w4_quantize_kernel(W4LayoutParams p)
{
    const int columns = (p.N + 255) / 256, g = blockIdx.x / columns;
    const int n = (blockIdx.x % columns) * 256 + threadIdx.x;
    if (n >= p.N)
        return;
    const int first = g * p.group, last = min(p.K, first + p.group);
    float lo = 0.0f, hi = 0.0f;
    bool finite = true;
    for (int k = first; k < last; ++k) {
        const float w = __builtin_bit_cast(float, (uint32_t)p.w[(size_t)k * p.N + n] << 16);
        finite &= __builtin_isfinite(w);
        lo = fminf(lo, w);
        hi = fmaxf(hi, w);
    }
    float range = p.z ? (hi - lo) / 15.0f : fmaxf(-lo, hi) / 7.0f;
    if (p.z && !__builtin_isfinite(range)) // hi - lo passed the range of fp32
        range = hi / 15.0f - lo / 15.0f;
    const uint16_t bits = finite ? __builtin_bit_cast(uint16_t, (__bf16)range) : 0x7fc0; // NaN
    const float s = __builtin_bit_cast(float, (uint32_t)bits << 16);
    const float z = !p.z ? 8.0f : s > 0.0f ? fminf(rintf(-lo / s), 15.0f) : 0.0f;
    for (int k = first; k < last; ++k) {
        const float w = __builtin_bit_cast(float, (uint32_t)p.w[(size_t)k * p.N + n] << 16);
        const float q = s > 0.0f ? fminf(fmaxf(rintf(w / s) + z, 0.0f), 15.0f) : z;
        p.q[(size_t)k * p.N + n] = (uint8_t)q;
    }
    p.s[(size_t)g * p.N + n] = bits;
    if (p.z)
        p.z[(size_t)g * p.N + n] = (uint8_t)z;
}

} // namespace gmlp
