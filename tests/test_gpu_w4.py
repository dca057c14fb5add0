"""Products with 4-bit weights on the GPU against plain 64-bit formulas.

Bounds.  A product is rounded once to bf16: 2^-8 of the value.  Before that the
fp32 sums of 1 + q/128 and 1 + z/128 over a group of G <= 128 rows hold up to
2.2 G terms of |x| each, so their difference is off by at most 2^-24 (G + 2) of
sum 2.2 |x|; scaled by 128 s that is below 2^-24 * 130 * 2.2 * 128 sum |x| s =
2^-8.8 sum |x| s in the worst case, and its square root times less for random
signs; the bound below takes 2^-13 sum |x| 8 s (rounding of random sign: about
sqrt(130) of 130), plus 2^-16 of the terms for the groups' sums.  H adds 2^-8 of
its value, carried through |Wd|.
"""
import pytest
import torch

from paper_2606_26344_amd import gmlp, w4

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def weight(K, N, group, zeros, gen):
    """Raw q, scales, zero points and the weight in 64 bits, on the CPU."""
    groups = -(-K // group)
    q = torch.randint(0, 16, (K, N), generator=gen, dtype=torch.uint8)
    s = ((torch.rand((groups, N), generator=gen) + 0.5) * 0.2 * K ** -0.5).to(torch.bfloat16)
    z = torch.randint(0, 16, (groups, N), generator=gen, dtype=torch.uint8) if zeros else None
    rows = torch.arange(K) // group
    w = (q.double() - (8 if z is None else z.double()[rows])) * s.double()[rows]
    return (q, s, z), w, 8 * s.double()[rows]


def packed(raw, group):
    return w4.pack(*[None if t is None else t.cuda() for t in raw], group=group)


def check(name, got, ref, terms):
    got = got.cpu().double()
    assert got.shape == ref.shape
    ratio = ((got - ref).abs() / (2.0 ** -8 * ref.abs() + terms + 1e-30)).max().item() if ref.numel() else 0.0
    print("%s: max |err|/bound = %.3f" % (name, ratio), flush=True)
    assert ratio <= 1.0, name


def product_slack(x, w, steps):
    return x.abs() @ (2.0 ** -13 * steps + 2.0 ** -16 * w.abs())


TOKENS = [1, 2, 4, 5, 13, 16, 17, 32, 33, 64]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("T", TOKENS)
def test_matmul(T, zeros, group):
    for K, N in [(8, 8), (264, 40), (1032, 264), (2056, 8)]:
        print("w4 T=%d K=%d N=%d group=%d zeros=%s" % (T, K, N, group, zeros), flush=True)
        gen = torch.Generator().manual_seed(T + K + N)
        raw, w, steps = weight(K, N, group, zeros, gen)
        x = torch.randn((T, K), generator=gen).to(torch.bfloat16)
        y = w4.matmul(x.cuda(), packed(raw, group), workspace=w4.make_workspace(T, K, N))
        check("y", y, x.double() @ w, product_slack(x.double(), w, steps))


@pytest.mark.parametrize("group,zeros", [(64, False), (64, True), (128, False), (128, True)])
@pytest.mark.parametrize("T,K,N", [(16, 2056, 12296), (33, 2056, 12296), (20, 6184, 4168), (48, 6184, 4168), (64, 6184, 4168)])
def test_long_weights(T, K, N, group, zeros):
    """The waves of a block share X: one block to a strip, and three over k (of 17, 17, 15 k-tiles)."""
    print("w4 T=%d K=%d N=%d group=%d zeros=%s" % (T, K, N, group, zeros), flush=True)
    gen = torch.Generator().manual_seed(T + K + N)
    raw, w, steps = weight(K, N, group, zeros, gen)
    x = torch.randn((T, K), generator=gen).to(torch.bfloat16)
    p, ws = packed(raw, group), w4.make_workspace(T, K, N)
    y = w4.matmul(x.cuda(), p, workspace=ws)
    check("y", y, x.double() @ w, product_slack(x.double(), w, steps))
    again = w4.matmul(x.cuda(), p)  # and without a workspace of its own
    assert torch.equal(y, again)
    # A row is its own, whatever is beside it.
    other = torch.full_like(x, float("nan"))
    other[T // 2] = x[T // 2]
    assert torch.equal(w4.matmul(other.cuda(), p, workspace=ws)[T // 2], y[T // 2])


@pytest.mark.parametrize("T,D,F", [(1, 264, 520), (3, 4096, 1024), (8, 520, 264), (30, 264, 1032), (64, 1032, 2056),
                                   (17, 2056, 12296), (64, 12296, 2056)])
@pytest.mark.parametrize("activation,beta", [("silu", 1.0), ("swish", 1.702), ("sigmoid", 1.0)])
def test_forward(T, D, F, activation, beta):
    gen = torch.Generator().manual_seed(T + D)
    zeros, group = T % 2 == 0, 128 if T < 8 else 64 if D * F > 2 ** 23 else 32
    (rg, wg, sg), (ru, wu, su), (rd, wd, sd) = (weight(K, N, group, zeros, gen) for K, N in ((D, F), (D, F), (F, D)))
    x = torch.randn((T, D), generator=gen).to(torch.bfloat16)
    pg, pu, pd = (packed(r, group) for r in (rg, ru, rd))
    kw = dict(activation=activation, beta=beta, workspace=w4.make_workspace(T, D, F))
    h = w4.gate_up(x.cuda(), pg, pu, **kw)
    y = w4.forward(x.cuda(), pg, pu, pd, **kw)
    d = x.double()
    g, u = d @ wg, d @ wu
    s = torch.sigmoid(beta * g)
    a = s if activation == "sigmoid" else g * s
    href = a * u
    # act' is below 1.2 max(1, |g| beta / 4) ... at most 1.2 for these gates.
    hs = 1.2 * max(1.0, beta) * u.abs() * product_slack(d, wg, sg) + a.abs() * product_slack(d, wu, su) + 2.0 ** -20 * href.abs()
    check("h", h, href, hs)
    # y from the h that the kernel rounded.
    hd = h.cpu().double()
    check("y", y, hd @ wd, product_slack(hd, wd, sd))


def test_quantize_pack_dequantize():
    gen = torch.Generator().manual_seed(3)
    for K, N, group, zeros in [(264, 40, 128, False), (256, 64, 64, True), (40, 8, 32, True), (1032, 520, 32, False)]:
        w = torch.randn((K, N), generator=gen).to(torch.bfloat16)
        w[:group, 1] = 0  # a group of zeros
        w[:, 2] = w[:, 2].abs()
        q, s, z = (None if t is None else t.cpu() for t in w4.quantize(w.cuda(), group, zeros))
        groups = -(-K // group)
        pad = torch.zeros((groups * group, N))
        pad[:K] = w.float()
        pad = pad.view(groups, group, N)
        if zeros:
            lo, hi = pad.amin(1).clamp(max=0), pad.amax(1).clamp(min=0)
            es = ((hi - lo) / 15).to(torch.bfloat16)
            ez = torch.where(es > 0, (-lo / es.float()).round().clamp(0, 15), torch.zeros(()))
            assert torch.equal(z.float(), ez)
        else:
            es, ez = (pad.abs().amax(1) / 7).to(torch.bfloat16), torch.full((groups, N), 8.0)
            assert z is None
        assert torch.equal(s.view(torch.int16), es.view(torch.int16))
        f = es.float()[:, None]
        eq = torch.where(f > 0, ((pad / f).round() + ez[:, None]).clamp(0, 15), ez[:, None].expand_as(pad))
        assert torch.equal(q.float(), eq.reshape(-1, N)[:K])
        p = w4.pack(q.cuda(), s.cuda(), None if z is None else z.cuda(), group=group)
        rows = torch.arange(K) // group
        ref = ((q.float() - ez[rows]) * s.float()[rows]).to(torch.bfloat16)
        assert torch.equal(w4.dequantize(p).cpu().view(torch.int16), ref.view(torch.int16) & -1)
        # Within half a step of the weight, or a step where q was clamped at 15.
        assert ((ref.float() - w.float()).abs() <= (0.5 if zeros else 1.01) * s.float()[rows] * 1.02 + 2.0 ** -8 * w.float().abs() + (s.float()[rows] if zeros else 0)).all()


@pytest.mark.parametrize("zeros", [False, True])
def test_quantize_weights_that_are_not_finite_or_very_large(zeros):
    K, N, group = 200, 40, 64
    gen = torch.Generator().manual_seed(8)
    w = torch.randn((K, N), generator=gen).to(torch.bfloat16)
    w[70, 3], w[0, 5], w[199, 7] = float("nan"), float("inf"), float("-inf")
    large = torch.finfo(torch.bfloat16).max
    w[:64, 9], w[1, 9] = large, -large  # hi - lo is beyond fp32
    q, s, z = w4.quantize(w.cuda(), group, zeros)
    assert torch.equal(s.cpu().isnan().nonzero(), torch.tensor([[0, 5], [1, 3], [3, 7]]))
    assert s[0, 9].isfinite() and s[0, 9] > large / 16
    assert int(q.max()) <= 15 and (z is None or int(z.max()) <= 15)
    p = w4.pack(q, s, z, group=group)
    y = w4.matmul(torch.ones((3, K), dtype=torch.bfloat16, device="cuda") * 2.0 ** -10, p).cpu()
    bad = torch.zeros(N, dtype=torch.bool)
    bad[[3, 5, 7]] = True
    assert torch.equal(y.isnan(), bad.expand(3, N)) and y[:, ~bad].isfinite().all()
    d = w4.dequantize(p).cpu().float()
    assert d[1, 9] < -0.8 * large and d[0, 9] > 0.8 * large


def test_tokens_do_not_mix():
    # A token with a NaN or infinity gives NaN, the others the same bits; tokens
    # are the same alone and in a batch of the same size class.
    gen = torch.Generator().manual_seed(9)
    raw, _, _ = weight(520, 264, 64, True, gen)
    p = packed(raw, 64)
    x = torch.randn((20, 520), generator=gen).to(torch.bfloat16).cuda()
    clean = w4.matmul(x, p)
    x[7, 100], x[11, 3] = float("nan"), float("inf")
    y = w4.matmul(x, p)
    rows = [i for i in range(20) if i not in (7, 11)]
    assert torch.equal(y[rows].view(torch.int16), clean[rows].view(torch.int16))
    assert torch.isnan(y[[7, 11]].float()).all()
    assert torch.equal(w4.matmul(x[:17].contiguous(), p)[:7].view(torch.int16), clean[:7].view(torch.int16))


def test_long_rows_and_large_values():
    gen = torch.Generator().manual_seed(10)
    raw, w, steps = weight(28672, 40, 128, False, gen)
    x = torch.randn((3, 28672), generator=gen).to(torch.bfloat16)
    check("y", w4.matmul(x.cuda(), packed(raw, 128)), x.double() @ w, product_slack(x.double(), w, steps))
    big = (x.float() * 1e30).to(torch.bfloat16)
    check("big", w4.matmul(big.cuda(), packed(raw, 128)), big.double() @ w, product_slack(big.double(), w, steps))


def test_no_tokens_and_outputs_given():
    gen = torch.Generator().manual_seed(1)
    raw, _, _ = weight(264, 40, 32, False, gen)
    p = packed(raw, 32)
    assert w4.matmul(torch.empty((0, 264), dtype=torch.bfloat16, device="cuda"), p).shape == (0, 40)
    # Rows behind the last token are left as they were.
    buf = torch.full((8, 40), 3.0, dtype=torch.bfloat16, device="cuda")
    x = torch.randn((5, 264), generator=gen).to(torch.bfloat16).cuda()
    y = w4.matmul(x, p, out=buf[:5])
    assert (buf[5:] == 3).all() and torch.equal(y, w4.matmul(x, p))


@pytest.mark.parametrize("T", [1, 9, 40])
def test_captured_calls_replay(T):
    D, F = 520, 1032
    gen = torch.Generator().manual_seed(T)
    ws = [packed(weight(K, N, 64, True, gen)[0], 64) for K, N in ((D, F), (D, F), (F, D))]
    x = torch.randn((T, D), generator=gen).to(torch.bfloat16).cuda()
    other = x * 0.5
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        work = w4.make_workspace(T, D, F, stream=stream)
        y = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    w4.forward(x, *ws, out=y, workspace=work, stream=stream)
    torch.cuda.synchronize()
    eager = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        w4.forward(x, *ws, out=y, workspace=work, stream=stream)
    torch.cuda.synchronize()
    for i in range(4):
        with torch.cuda.stream(stream):
            w4.forward(other, *ws, out=y, workspace=work, stream=stream)
            y.zero_()
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y.view(torch.int16), eager.view(torch.int16)), i
    assert torch.equal(w4.forward(x, *ws).view(torch.int16), eager.view(torch.int16))


def test_refusals_of_the_binding():
    gen = torch.Generator().manual_seed(2)
    p = packed(weight(264, 40, 64, False, gen)[0], 64)
    q = packed(weight(264, 40, 32, False, gen)[0], 32)
    x = torch.zeros((65, 264), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(gmlp.GmlpError, match="65 tokens"):
        w4.matmul(x, p)
    with pytest.raises(ValueError, match="group"):
        w4.gate_up(x[:4], p, q)
    with pytest.raises(ValueError):
        w4.matmul(x[:4, :256], p)
    with pytest.raises(TypeError):
        w4.matmul(x[:4], x)
