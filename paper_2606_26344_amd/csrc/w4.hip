// The C ABI of include/gmlp_w4.h: validation and launches of the products with
// 4-bit weights (w4.hpp).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "gmlp_w4.h"
#include "launch.hpp"
#include "w4.hpp"

using namespace gmlp;

namespace {

// Where the parts of a packed weight lie.
struct W4Packed {
    int64_t ktiles = 0, ntiles = 0;
    size_t scales = 0, zeros = 0, total = 0;
};

W4Packed w4_packed(int64_t K, int64_t N, int group, int zeros)
{
    W4Packed l;
    l.ktiles = cdiv(K, 128);
    l.ntiles = cdiv(N, 16);
    const size_t groups = (size_t)l.ktiles * l.ntiles * 16 * (128 / group);
    l.scales = (size_t)l.ktiles * l.ntiles * 1024;
    l.zeros = l.scales + align_up(groups * 2);
    l.total = l.zeros + (zeros ? align_up(groups) : 0);
    return l;
}

int check_w4_weight(int64_t K, int64_t N, int group)
{
    int rc;
    if ((rc = check_smm_shape(0, K, N)))
        return rc;
    if (group != 32 && group != 64 && group != 128)
        return fail(GMLP_ERR_UNSUPPORTED, "groups of 32, 64 or 128 rows (got %d)", group);
    return GMLP_OK;
}

int check_w4_tokens(int64_t T)
{
    if (T < 0)
        return fail(GMLP_ERR_INVALID_ARG, "invalid T=%lld", (long long)T);
    if (T > GMLP_W4_MAX_TOKENS)
        return fail(GMLP_ERR_UNSUPPORTED, "%lld tokens: at most %d (gmlp_w4_dequantize gives the weight for more)",
                    (long long)T, GMLP_W4_MAX_TOKENS);
    return GMLP_OK;
}

int check_w4_packed(const void *p, const char *name)
{
    int rc;
    if ((rc = check_ptr(p, name, true)))
        return rc;
    if (reinterpret_cast<uintptr_t>(p) % kAlign)
        return fail(GMLP_ERR_UNSUPPORTED, "%s (%p) is not %zu-byte aligned", name, p, kAlign);
    return GMLP_OK;
}

int check_w4_path(int path)
{
    return path == GMLP_PATH_AUTO || path == (GMLP_PATH_AUTO | GMLP_FRESH_WORKSPACE)
               ? GMLP_OK
               : fail(GMLP_ERR_INVALID_ARG, "4-bit products have the automatic path only (got %d)", path);
}

// The launch of one product: column strips, split over k where there are too few of
// them to fill the chip and each piece keeps work for its waves.
struct W4Step {
    int tokens = 4; // rounded up: the kernel's
    bool shared = false;
    int strips = 0, splits = 1, split_ktiles = 0;
    size_t partial_bytes = 0;
};

// The column tiles of a strip and the k-tiles a wave has asked for before it uses one.
// One tile and 4 ahead for T <= 4 (D = 4096, F = 14336, T = 1: gate/up 14.6 us, down 7.6);
// from there on two tiles, since X comes through LDS once for both, and 2 ahead, 1 where
// more would not fit the registers (T = 33, D = 2048, F = 8192, groups of 32: 10.2 us and 12.8).
constexpr int kW4Waves = 8;
constexpr int w4_ct(int tok) { return tok == 4 ? 1 : 2; }
constexpr int w4_depth(int tok) { return tok == 4 ? 4 : tok <= 32 ? 2 : 1; }

// The same for the kernel whose waves share X.
constexpr int w4_shared_depth(int tok, int weights) { return weights == 1 ? 6 : tok <= 48 ? 4 : 2; }

// The waves share X from 16 tokens on, if 16 k-tiles a block still fill three quarters
// of the chip.  us shared against not, gate/up and down of D = 4096, F = 14336, groups of
// 128: 15.0 against 17.6 and 13.4 against 13.7 at T = 16, 26.6 against 31.5 and 20.8
// against 24.9 at 40, 31.1 against 43.2 and 24.2 against 32.5 at 64.  With 128 blocks of 16
// k-tiles (D = 2048, F = 8192, T = 33) gate/up takes 19.7 against 10.6.  Groups of 32 gain
// nothing, their scales cost the wave more than X: 35.9 against 33.1 and 26.1 against 26.8
// at T = 40.
constexpr int kW4SharedTokens = 16, kW4SharedTiles = 16, kW4SharedGroup = 64;

W4Step w4_step(int64_t T, int64_t K, int64_t N, int weights, int group)
{
    W4Step s;
    s.tokens = T <= 4 ? 4 : T <= 8 ? 8 : (int)cdiv(T, 16) * 16;
    const int64_t ktiles = cdiv(K, 128);
    auto split = [&](int64_t strips, int64_t least) {
        s.strips = (int)strips;
        s.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kBlockTarget / strips, ktiles / least));
        s.split_ktiles = (int)cdiv(ktiles, s.splits);
        s.splits = (int)cdiv(ktiles, s.split_ktiles);
    };
    int columns = kW4SharedColumns;
    split(cdiv(N, columns), kW4SharedTiles);
    s.shared = s.tokens >= kW4SharedTokens && group >= kW4SharedGroup && s.split_ktiles >= kW4SharedTiles &&
               s.strips * s.splits >= kBlockTarget * 3 / 4;
    if (!s.shared) {
        columns = 16 * w4_ct(s.tokens);
        split(cdiv(N, columns), 2 * kW4Waves);
    }
    s.partial_bytes = s.splits > 1 ? (size_t)s.splits * s.strips * weights * s.tokens * columns * sizeof(float) : 0;
    return s;
}

// The counter block of every workspace, H [T, F], then the partial sums of any step.
struct W4Layout {
    size_t partial = 0, total = 0;
};

W4Layout w4_workspace(int64_t T, int64_t D, int64_t F)
{
    T = std::max<int64_t>(T, 1);
    W4Layout l;
    l.partial = kCounterBytes + align_up((size_t)T * std::max(D, F) * 2);
    size_t partial = 0;
    for (int group : {32, kW4SharedGroup})
        for (int weights : {1, 2})
            partial = std::max({partial, w4_step(T, D, F, weights, group).partial_bytes,
                                w4_step(T, F, D, weights, group).partial_bytes});
    l.total = l.partial + align_up(partial);
    return l;
}

int check_w4_workspace(void *ws, size_t bytes, size_t need)
{
    if (!ws)
        return fail(GMLP_ERR_INVALID_ARG, "workspace is NULL");
    if (reinterpret_cast<uintptr_t>(ws) % kAlign)
        return fail(GMLP_ERR_UNSUPPORTED, "workspace %p is not %zu-byte aligned", ws, kAlign);
    if (bytes < need)
        return fail(GMLP_ERR_NO_MEMORY, "workspace of %zu bytes, %zu needed", bytes, need);
    return GMLP_OK;
}

template <int TOK, int NW, int GPT, bool ZEROS>
int launch_w4(const W4Params &p, bool shared, hipStream_t st)
{
    const dim3 grid((unsigned)(p.strips * p.splits));
    if constexpr (TOK >= kW4SharedTokens && 128 / GPT >= kW4SharedGroup)
        if (shared) {
            hipLaunchKernelGGL((w4_shared_kernel<TOK / 16, NW, GPT, ZEROS, w4_shared_depth(TOK, NW)>), grid,
                               dim3(kW4SharedWaves * 64), 0, st, p);
            return hip_check(hipGetLastError(), "4-bit product launch");
        }
    hipLaunchKernelGGL((w4_kernel<TOK, NW, w4_ct(TOK), GPT, ZEROS, kW4Waves, w4_depth(TOK)>), grid,
                       dim3(kW4Waves * 64), 0, st, p);
    return hip_check(hipGetLastError(), "4-bit product launch");
}

template <int TOK, int NW>
int launch_w4_group(const W4Params &p, bool shared, int group, bool zeros, hipStream_t st)
{
    switch (group) {
    case 32: return zeros ? launch_w4<TOK, NW, 4, true>(p, shared, st) : launch_w4<TOK, NW, 4, false>(p, shared, st);
    case 64: return zeros ? launch_w4<TOK, NW, 2, true>(p, shared, st) : launch_w4<TOK, NW, 2, false>(p, shared, st);
    default: return zeros ? launch_w4<TOK, NW, 1, true>(p, shared, st) : launch_w4<TOK, NW, 1, false>(p, shared, st);
    }
}

template <int NW>
int run_w4(const void *X, const void *const (&packed)[2], void *out, int64_t T, int64_t K, int64_t N, int group, bool zeros,
           int activation, float beta, void *workspace, const W4Layout &ws, hipStream_t st)
{
    const W4Packed l = w4_packed(K, N, group, zeros);
    const W4Step s = w4_step(T, K, N, NW, group);
    W4Params p{};
    p.x = static_cast<const uint16_t *>(X);
    for (int w = 0; w < NW; ++w) {
        p.tiles[w] = static_cast<const uint8_t *>(packed[w]);
        p.scales[w] = p.tiles[w] + l.scales;
        p.zeros[w] = p.tiles[w] + l.zeros;
    }
    p.out = static_cast<uint16_t *>(out);
    p.partial = reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + ws.partial);
    p.counters = static_cast<uint32_t *>(workspace);
    p.T = (int)T;
    p.K = (int)K;
    p.N = (int)N;
    p.ktiles = (int)l.ktiles;
    p.strips = s.strips;
    p.splits = s.splits;
    p.split_ktiles = s.split_ktiles;
    p.activation = activation;
    p.beta = beta;
    switch (s.tokens) {
    case 4: return launch_w4_group<4, NW>(p, s.shared, group, zeros, st);
    case 8: return launch_w4_group<8, NW>(p, s.shared, group, zeros, st);
    case 16: return launch_w4_group<16, NW>(p, s.shared, group, zeros, st);
    case 32: return launch_w4_group<32, NW>(p, s.shared, group, zeros, st);
    case 48: return launch_w4_group<48, NW>(p, s.shared, group, zeros, st);
    default: return launch_w4_group<64, NW>(p, s.shared, group, zeros, st);
    }
}

// The counters that a call's products use, cleared for a workspace that has not
// been prepared.
int clear_w4_counters(int path, std::initializer_list<W4Step> steps, void *workspace, hipStream_t st)
{
    int words = 0;
    for (const W4Step &s : steps)
        words = std::max(words, s.splits > 1 ? s.strips : 0);
    return path & GMLP_FRESH_WORKSPACE ? clear_words(static_cast<uint32_t *>(workspace), words, st) : GMLP_OK;
}

W4LayoutParams w4_layout_params(void *packed, int64_t K, int64_t N, int group, int zeros)
{
    const W4Packed l = w4_packed(K, N, group, zeros);
    W4LayoutParams p{};
    p.tiles = static_cast<uint8_t *>(packed);
    p.scales = p.tiles + l.scales;
    p.zeros = zeros ? p.tiles + l.zeros : nullptr;
    p.K = (int)K;
    p.N = (int)N;
    p.group = group;
    p.ktiles = (int)l.ktiles;
    p.ntiles = (int)l.ntiles;
    return p;
}

unsigned w4_layout_blocks(const W4LayoutParams &p) { return (unsigned)cdiv((int64_t)p.ktiles * p.ntiles, 4); }

} // namespace

extern "C" {

size_t gmlp_w4_packed_size(int64_t K, int64_t N, int group, int zeros)
{
    if (check_w4_weight(K, N, group))
        return 0;
    return w4_packed(K, N, group, zeros).total;
}

int gmlp_w4_quantize(const void *W, void *Q, void *S, void *Z, int64_t K, int64_t N, int group, void *stream)
{
    int rc;
    if ((rc = check_w4_weight(K, N, group)) || (rc = check_ptr(W, "W", true)) || (rc = check_ptr(Q, "Q", true)) ||
        (rc = check_ptr(S, "S", true)) || (rc = check_ptr(Z, "Z", false)))
        return rc;
    const size_t n = (size_t)K * N, g = (size_t)cdiv(K, group) * N;
    if (overlaps(Q, n, W, 2 * n) || overlaps(S, 2 * g, W, 2 * n) || overlaps(S, 2 * g, Q, n) ||
        (Z && (overlaps(Z, g, W, 2 * n) || overlaps(Z, g, Q, n) || overlaps(Z, g, S, 2 * g))))
        return fail(GMLP_ERR_INVALID_ARG, "W, Q, S and Z must not overlap");
    W4LayoutParams p{};
    p.w = const_cast<uint16_t *>(static_cast<const uint16_t *>(W));
    p.q = static_cast<uint8_t *>(Q);
    p.s = static_cast<uint16_t *>(S);
    p.z = static_cast<uint8_t *>(Z);
    p.K = (int)K;
    p.N = (int)N;
    p.group = group;
    hipLaunchKernelGGL(w4_quantize_kernel, dim3((unsigned)(cdiv(N, 256) * cdiv(K, group))), dim3(256), 0,
                       static_cast<hipStream_t>(stream), p);
    rc = hip_check(hipGetLastError(), "quantise launch");
    return rc ? rc : ok();
}

int gmlp_w4_pack(const void *Q, const void *S, const void *Z, void *packed, int64_t K, int64_t N, int group, void *stream)
{
    int rc;
    if ((rc = check_w4_weight(K, N, group)) || (rc = check_ptr(Q, "Q", true)) || (rc = check_ptr(S, "S", true)) ||
        (rc = check_ptr(Z, "Z", false)) || (rc = check_w4_packed(packed, "packed")))
        return rc;
    const size_t n = (size_t)K * N, g = (size_t)cdiv(K, group) * N, b = w4_packed(K, N, group, Z != nullptr).total;
    if (overlaps(packed, b, Q, n) || overlaps(packed, b, S, 2 * g) || (Z && overlaps(packed, b, Z, g)))
        return fail(GMLP_ERR_INVALID_ARG, "packed overlaps an input");
    W4LayoutParams p = w4_layout_params(packed, K, N, group, Z != nullptr);
    p.q = const_cast<uint8_t *>(static_cast<const uint8_t *>(Q));
    p.s = const_cast<uint16_t *>(static_cast<const uint16_t *>(S));
    p.z = const_cast<uint8_t *>(static_cast<const uint8_t *>(Z));
    hipLaunchKernelGGL(w4_pack_kernel, dim3(w4_layout_blocks(p)), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    rc = hip_check(hipGetLastError(), "pack launch");
    return rc ? rc : ok();
}

int gmlp_w4_dequantize(const void *packed, void *W, int64_t K, int64_t N, int group, int zeros, void *stream)
{
    int rc;
    if ((rc = check_w4_weight(K, N, group)) || (rc = check_w4_packed(packed, "packed")) || (rc = check_ptr(W, "W", true)))
        return rc;
    if (overlaps(W, 2 * (size_t)K * N, packed, w4_packed(K, N, group, zeros).total))
        return fail(GMLP_ERR_INVALID_ARG, "W overlaps packed");
    W4LayoutParams p = w4_layout_params(const_cast<void *>(packed), K, N, group, zeros);
    p.w = static_cast<uint16_t *>(W);
    hipLaunchKernelGGL(w4_dequantize_kernel, dim3(w4_layout_blocks(p)), dim3(256), 0, static_cast<hipStream_t>(stream), p);
    rc = hip_check(hipGetLastError(), "dequantise launch");
    return rc ? rc : ok();
}

size_t gmlp_w4_workspace_size(int64_t T, int64_t D, int64_t F)
{
    if (check_w4_tokens(T) || check_smm_shape(0, D, F))
        return 0;
    return w4_workspace(T, D, F).total;
}

int gmlp_w4_matmul(const void *X, const void *packed, void *Y, int64_t T, int64_t K, int64_t N, int group, int zeros,
                   int path, void *workspace, size_t ws_bytes, void *stream)
{
    int rc;
    const bool rows = T > 0;
    if ((rc = check_w4_tokens(T)) || (rc = check_w4_weight(K, N, group)) || (rc = check_ptr(X, "X", rows)) ||
        (rc = check_w4_packed(packed, "packed")) || (rc = check_ptr(Y, "Y", rows)) || (rc = check_w4_path(path)))
        return rc;
    if (!rows)
        return ok();
    const W4Layout l = w4_workspace(T, K, N);
    const size_t need = l.total, yb = 2 * (size_t)T * N;
    if ((rc = check_w4_workspace(workspace, ws_bytes, need)))
        return rc;
    if (overlaps(Y, yb, X, 2 * (size_t)T * K) || overlaps(Y, yb, packed, w4_packed(K, N, group, zeros).total) ||
        overlaps(Y, yb, workspace, need))
        return fail(GMLP_ERR_INVALID_ARG, "Y overlaps an input or the workspace");
    const void *const w[2] = {packed, nullptr};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if ((rc = clear_w4_counters(path, {w4_step(T, K, N, 1, group)}, workspace, st)) ||
        (rc = run_w4<1>(X, w, Y, T, K, N, group, zeros, 0, 1.0f, workspace, l, st)))
        return rc;
    return ok();
}

int gmlp_w4_gate_up(const void *X, const void *packed_g, const void *packed_u, void *H, int64_t T, int64_t D, int64_t F,
                    int group, int zeros, int activation, float beta, int path, void *workspace, size_t ws_bytes,
                    void *stream)
{
    int rc;
    Variant v;
    const bool rows = T > 0;
    if ((rc = check_w4_tokens(T)) || (rc = check_w4_weight(D, F, group)) || (rc = check_ptr(X, "X", rows)) ||
        (rc = check_w4_packed(packed_g, "packed_g")) || (rc = check_w4_packed(packed_u, "packed_u")) ||
        (rc = check_ptr(H, "H", rows)) || (rc = check_w4_path(path)) || (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    if (!rows)
        return ok();
    const W4Layout l = w4_workspace(T, D, F);
    const size_t need = l.total, hb = 2 * (size_t)T * F, pb = w4_packed(D, F, group, zeros).total;
    if ((rc = check_w4_workspace(workspace, ws_bytes, need)))
        return rc;
    if (overlaps(H, hb, X, 2 * (size_t)T * D) || overlaps(H, hb, packed_g, pb) || overlaps(H, hb, packed_u, pb) ||
        overlaps(H, hb, workspace, need))
        return fail(GMLP_ERR_INVALID_ARG, "H overlaps an input or the workspace");
    const void *const w[2] = {packed_g, packed_u};
    hipStream_t st = static_cast<hipStream_t>(stream);
    if ((rc = clear_w4_counters(path, {w4_step(T, D, F, 2, group)}, workspace, st)) ||
        (rc = run_w4<2>(X, w, H, T, D, F, group, zeros, v.act, v.beta, workspace, l, st)))
        return rc;
    return ok();
}

int gmlp_w4_forward(const void *X, const void *packed_g, const void *packed_u, const void *packed_d, void *Y, int64_t T,
                    int64_t D, int64_t F, int group, int zeros, int activation, float beta, int path, void *workspace,
                    size_t ws_bytes, void *stream)
{
    int rc;
    Variant v;
    const bool rows = T > 0;
    if ((rc = check_w4_tokens(T)) || (rc = check_w4_weight(D, F, group)) || (rc = check_ptr(X, "X", rows)) ||
        (rc = check_w4_packed(packed_g, "packed_g")) || (rc = check_w4_packed(packed_u, "packed_u")) ||
        (rc = check_w4_packed(packed_d, "packed_d")) || (rc = check_ptr(Y, "Y", rows)) || (rc = check_w4_path(path)) ||
        (rc = check_variant(activation, beta, 0, 0.0f, &v)))
        return rc;
    if (!rows)
        return ok();
    const W4Layout l = w4_workspace(T, D, F);
    const size_t need = l.total, yb = 2 * (size_t)T * D;
    const size_t gb = w4_packed(D, F, group, zeros).total, db = w4_packed(F, D, group, zeros).total;
    if ((rc = check_w4_workspace(workspace, ws_bytes, need)))
        return rc;
    if (overlaps(Y, yb, X, 2 * (size_t)T * D) || overlaps(Y, yb, packed_g, gb) || overlaps(Y, yb, packed_u, gb) ||
        overlaps(Y, yb, packed_d, db) || overlaps(Y, yb, workspace, need))
        return fail(GMLP_ERR_INVALID_ARG, "Y overlaps an input or the workspace");
    hipStream_t st = static_cast<hipStream_t>(stream);
    void *H = static_cast<uint8_t *>(workspace) + kCounterBytes;
    const void *const gu[2] = {packed_g, packed_u}, *const dn[2] = {packed_d, nullptr};
    if ((rc = clear_w4_counters(path, {w4_step(T, D, F, 2, group), w4_step(T, F, D, 1, group)}, workspace, st)) ||
        (rc = run_w4<2>(X, gu, H, T, D, F, group, zeros, v.act, v.beta, workspace, l, st)) ||
        (rc = run_w4<1>(H, dn, Y, T, F, D, group, zeros, 0, 1.0f, workspace, l, st)))
        return rc;
    return ok();
}

} // extern "C"
