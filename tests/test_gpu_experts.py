"""The experts' Gated MLPs on the GPU against plain 64-bit formulas, expert by expert.

Bounds, for every expert those of one Gated MLP's training step: each output is an fp32
sum of products of bf16 numbers, rounded once to bf16 (2^-8 of the value).  Before that

  * G and U carry fp32 sums of D <= 4104 products: at most D 2^-24 <= 2^-12 of the sum S
    of the terms' absolute values;
  * H, dG and dU are rounded to bf16: 2^-8 of the terms of the sums that they enter, and
    act and act' in fp32 (exp and rcp to 2 units in the last place) 2^-20;
  * dH in fp32 carries 2^-12 of its terms into dG and dU; dX sums 2 F <= 8208 products,
    formed 32 at a time: 257 roundings of 2^-24 S, and the weights' gradients fewer.

So results are within 2^-8 |ref| + 1.02 2^-8 S + 2^-12 S, and G and U within 2^-8 |ref| +
2^-12 S.  S is some sqrt(K) times the result where K products add up, and a block of k that
is left out would hide in it; so each expert's results are compared as a whole too.  A
rounding moves a tensor by at most 2^-8 of its L2 norm, and a product with a random
matrix has about the same gain for that as for the tensor: with the roundings of the
operands (H; dG and dU) and of the result 3 2^-8 of its norm.  64 of 4104 terms left out
would be 2^-3.
"""
import pytest
import torch

from paper_2606_26344_amd import experts, gmlp

pytestmark = pytest.mark.gpu

HALF_STEP = 2.0 ** -8
ROUNDED = 1.02 * 2.0 ** -8 + 2.0 ** -12
MARK = 7.0  # in rows that no expert has


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def act(g, activation, beta):
    b = beta if activation == "swish" else 1.0
    s = torch.sigmoid(b * g)
    if activation == "sigmoid":
        return s, s * torch.sigmoid(-g)
    return g * s, s + b * g * s * torch.sigmoid(-b * g)


def inputs(N, E, D, F, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *shape, s=1.0: (torch.randn(shape, generator=gen, device="cuda") * s).to(torch.bfloat16)  # noqa: E731
    return dict(xs=n(N, D), wg=n(E, D, F, s=D ** -0.5), wu=n(E, D, F, s=D ** -0.5), wd=n(E, F, D, s=F ** -0.5), dys=n(N, D))


def offsets_of(counts, first=0):
    return torch.tensor([first] + counts, dtype=torch.int32).cumsum(0).int().cuda()


def check(name, got, ref, terms, rounded=True):
    bound = HALF_STEP * ref.abs() + (ROUNDED if rounded else 2.0 ** -12) * terms + 1e-30
    ratio = ((got.double() - ref).abs() / bound).max().item() if ref.numel() else 0.0
    assert ratio <= 1.0, (name, ratio)
    off = (got.double() - ref).norm().item()
    assert off <= 3 * HALF_STEP * ref.norm().item(), (name, off)
    return ratio


def run(counts, D, F, behind=0, before=0, activation="silu", beta=1.0, seed=0, want=experts.GRADIENTS, workspace=None):
    """Forward and backward of experts with so many rows each, `behind` rows behind the
    last and `before` in front of the first."""
    E, N = len(counts), before + sum(counts) + behind
    print("experts N=%d E=%d D=%d F=%d counts=%s" % (N, E, D, F, counts if E < 12 else "..."), flush=True)
    t = inputs(N, E, D, F, seed)
    offsets = offsets_of(counts, before)
    dead = torch.ones(N, dtype=torch.bool, device="cuda")
    dead[before:before + sum(counts)] = False
    t["xs"][dead] = t["dys"][dead] = float("nan")  # of no expert, not read
    w = (t["wg"], t["wu"], t["wd"])
    kw = dict(activation=activation, beta=beta, workspace=workspace)
    buffer = lambda cols: torch.full((N, cols), MARK, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    y, g, u = experts.train_forward(t["xs"], offsets, *w, out=buffer(D), g=buffer(F), u=buffer(F), **kw)
    alone = experts.forward(t["xs"], offsets, *w, out=buffer(D), **kw)
    assert torch.equal(alone, y)
    ga, ua = g.clone(), u.clone()
    ga[dead] = ua[dead] = float("nan")
    dxs = buffer(D) if "dxs" in want else None
    grads = dict(zip(experts.GRADIENTS, experts.backward(t["dys"], t["xs"], offsets, *w, ga, ua, dxs=dxs, want=want, **kw)))
    for r in (y, g, u, grads["dxs"]):
        assert r is None or (r[dead] == MARK).all()
    worst = {}
    for e, n in enumerate(counts):
        lo = before + sum(counts[:e])
        x, dy, wg, wu, wd = (v.double() for v in (t["xs"][lo:lo + n], t["dys"][lo:lo + n], t["wg"][e], t["wu"][e], t["wd"][e]))
        refs = {}
        ge, ue = x @ wg, x @ wu
        gt = x.abs() @ torch.maximum(wg.abs(), wu.abs())
        refs["g"], refs["u"] = (g[lo:lo + n], ge, x.abs() @ wg.abs(), False), (u[lo:lo + n], ue, x.abs() @ wu.abs(), False)
        a, _ = act(ge, activation, beta)
        h = a * ue
        slack = (a.abs() + 1.2 * max(1.0, beta) * ue.abs()) * 2.0 ** -12 * gt
        refs["y"] = (y[lo:lo + n], h @ wd, (h.abs() + 2.0 ** 8 * slack) @ wd.abs(), True)
        gd, ud = g[lo:lo + n].double(), u[lo:lo + n].double()
        a, da = act(gd, activation, beta)
        dh, dh_terms = dy @ wd.T.contiguous(), dy.abs() @ wd.abs().T.contiguous()
        dg, du, h = dh * ud * da, dh * a, a * ud
        dgt, dut = dg.abs() + 2.0 ** -4 * (dh_terms * ud * da).abs(), du.abs() + 2.0 ** -4 * (dh_terms * a).abs()
        every = {"dxs": (dg @ wg.T + du @ wu.T, dgt @ wg.abs().T + dut @ wu.abs().T), "dwg": (x.T @ dg, x.abs().T @ dgt),
                 "dwu": (x.T @ du, x.abs().T @ dut), "dwd": (h.T @ dy, h.abs().T @ dy.abs())}
        for name, (ref, terms) in every.items():
            if name in want:
                got = grads[name]
                refs[name] = (got[lo:lo + n] if name == "dxs" else got[e], ref, terms, True)
            else:
                assert grads[name] is None
        for name, r in refs.items():
            assert r[0].shape == r[1].shape
            worst[name] = max(worst.get(name, 0.0), check((e, name), *r))
            if n == 0:
                assert (r[0] == 0).all()  # weight gradients of no rows
    print({k: round(v, 3) for k, v in worst.items()}, flush=True)
    return y, g, u, grads


SMALL = [([1], 8, 8, 0, 0), ([0], 8, 8, 3, 0), ([1, 0, 1], 264, 520, 0, 0), ([0, 0, 5, 0], 264, 520, 2, 1), ([31, 32, 33], 136, 264, 5, 0),
         ([64, 1, 65, 0, 63], 264, 136, 1, 0), ([3] * 70, 72, 40, 7, 0), ([0] * 130 + [9], 264, 264, 0, 2),
         ([1] * 65, 128, 64, 0, 0), ([i % 4 for i in range(1024)], 16, 24, 9, 0)]


@pytest.mark.parametrize("counts,D,F,behind,before", SMALL, ids=[str(i) for i in range(len(SMALL))])
def test_small(counts, D, F, behind, before):
    run(counts, D, F, behind, before, seed=len(counts) + D)


# Each tile of the plan (rows of an expert up to 24, 48, 160 and more), with ragged ones,
# with and without split sums.
TILES = [([20, 24, 1, 30, 7], 1032, 2056), ([2, 0, 0, 0, 0, 0, 0, 0], 2056, 4104), ([1, 1], 4104, 1032),
         ([40, 70, 10, 50], 1032, 2056), ([129, 150, 0, 260, 100], 520, 1032), ([100] * 3, 2056, 4104),
         ([300, 511, 1, 700], 520, 1032), ([257, 256, 255], 1032, 2056), ([2000, 3000], 264, 520), ([4096, 0, 1, 90], 520, 264),
         ([600], 2056, 4104)]


@pytest.mark.parametrize("counts,D,F", TILES, ids=[str(i) for i in range(len(TILES))])
def test_tiles(counts, D, F):
    run(counts, D, F, 3, seed=D + len(counts))


# The 256-row tiles, with last tiles of up to 64, 128 and 256 rows of experts with one tile and
# with several; the others with splits of long products; weight gradients in whole lines.
RAGGED = [300, 511, 1, 700, 260, 64, 129, 400, 0, 100, 356]
MORE_TILES = [(RAGGED, 4096, 4096), (RAGGED, 4104, 4104), ([30, 33, 20, 40, 1, 29], 2056, 4104), ([40, 30], 4104, 4104),
              ([90, 120, 70], 4104, 4104), ([110, 60, 100, 90], 1024, 4096), ([1700, 1600], 256, 512), ([9, 2, 0, 4], 4096, 1024),
              ([150, 200], 512, 4096)]


@pytest.mark.parametrize("counts,D,F", MORE_TILES, ids=[str(i) for i in range(len(MORE_TILES))])
def test_more_tiles(counts, D, F):
    run(counts, D, F, 3, seed=D + F + len(counts))


def test_every_tile_is_tested():
    names, split = set(), set()
    for counts, D, F in [(c[0], c[1], c[2]) for c in SMALL] + TILES + MORE_TILES:
        for backward in (False, True):
            for name, _, _, splits in experts.describe(sum(counts) + 3, len(counts), D, F, backward):
                names.add(name)
                if splits > 1:
                    split.add(name)
    # Gate/up, down, dH and dX on four tiles each, the weight gradients on three and both ways out.
    assert len(names) == 4 * 4 + 3 * 2
    assert len(split) == 4 * 4


@pytest.mark.parametrize("activation,beta", [("swish", 1.702), ("sigmoid", 1.0), ("swish", -0.5)])
@pytest.mark.parametrize("counts", [[2, 0, 3], [200, 90, 310]])
def test_activations(counts, activation, beta):
    run(counts, 264, 520, 1, activation=activation, beta=beta)


@pytest.mark.parametrize("want", [("dxs",), ("dwd",), ("dwg", "dwd"), ("dwu", "dxs")])
def test_wanted_gradients(want):
    run([5, 0, 40], 264, 520, want=want)


def test_a_workspace_serves_fewer_rows():
    D, F = 520, 1032
    ws = experts.make_workspace(2000, 8, D, F)
    assert ws.fits(2000, 8, D, F) and ws.fits(3, 8, D, F) and not ws.fits(1 << 20, 8, D, F)
    for counts in ([250] * 8, [1, 0, 2, 0, 0, 0, 0, 0], [0] * 7 + [400], [40] * 8, [250] * 8):
        first = run(counts, D, F, workspace=ws)
        again = run(counts, D, F)
        assert all(torch.equal(a, b) for a, b in zip(first[:3], again[:3]))
        assert all(torch.equal(first[3][k], again[3][k]) for k in experts.GRADIENTS)


def test_no_rows():
    E, D, F = 3, 264, 520
    t = inputs(0, E, D, F, 1)
    offsets = offsets_of([0] * E)
    y, g, u = experts.train_forward(t["xs"], offsets, t["wg"], t["wu"], t["wd"])
    assert y.shape == (0, D) and g.shape == u.shape == (0, F)
    grads = experts.backward(t["dys"], t["xs"], offsets, t["wg"], t["wu"], t["wd"], g, u)
    assert grads[0].shape == (0, D) and all((w == 0).all() for w in grads[1:])


def test_offsets_past_the_rows_are_cut():
    """Ends past N and an end before its begin: rows of no expert, no access past N."""
    N, E, D, F = 50, 4, 264, 520
    t = inputs(N, E, D, F, 2)
    w = (t["wg"], t["wu"], t["wd"])
    mark = lambda: torch.full((N, D), MARK, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    for bad, good in (([0, 10, 30, 99, 200], [0, 10, 30, 50, 50]), ([-7, 10, 10, 2 ** 31 - 1, 60], [0, 10, 10, 50, 50]),
                      ([0, 20, 10, 10, 50], None)):
        bad = torch.tensor(bad, dtype=torch.int32, device="cuda")
        got = experts.forward(t["xs"], bad, *w, out=mark())
        if good:
            good = torch.tensor(good, dtype=torch.int32, device="cuda")
            assert torch.equal(got, experts.forward(t["xs"], good, *w, out=mark()))
            f = experts.train_forward(t["xs"], good, *w)
            for a, b in zip(experts.backward(t["dys"], t["xs"], bad, *w, *f[1:]), experts.backward(t["dys"], t["xs"], good, *w, *f[1:])):
                assert torch.equal(a, b)


def test_other_experts_values_stay_out():
    """Infinities and NaN in one expert's rows and weights change no other's results."""
    counts, D, F = [30, 3, 40, 0, 17], 264, 520
    N, E = sum(counts), len(counts)
    t = inputs(N, E, D, F, 3)
    offsets = offsets_of(counts)

    def step():
        w = (t["wg"], t["wu"], t["wd"])
        y, g, u = experts.train_forward(t["xs"], offsets, *w)
        return (y, g, u) + experts.backward(t["dys"], t["xs"], offsets, *w, g, u)

    want = step()
    t["xs"][30:33] = float("nan")
    t["dys"][31] = float("inf")
    t["wg"][1] = float("-inf")
    t["wd"][3] = float("nan")
    got = step()
    rows = [i for i in range(N) if not 30 <= i < 33]
    for i, (a, b) in enumerate(zip(got, want)):
        keep = rows if i < 4 else [0, 2, 3, 4]
        assert torch.equal(a[keep], b[keep])
    assert got[0][30:33].isnan().all()


def test_rows_and_weights_past_32_bits():
    """An expert whose weights, and rows that, begin past 2^32 bytes."""
    E, D, F, N = 9, 8192, 32768, 70000
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = [torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((E, D, F), (E, D, F), (E, F, D))]
    last = [(torch.randn(v.shape[1:], generator=gen, device="cuda") * v.shape[1] ** -0.5).to(torch.bfloat16) for v in w]
    for v, l in zip(w, last):
        v[-1] = l
    xs = torch.zeros((N, D), dtype=torch.bfloat16, device="cuda")
    n = 40
    xs[-n:] = torch.randn((n, D), generator=gen, device="cuda").to(torch.bfloat16)
    offsets = torch.full((E + 1,), N - n, dtype=torch.int32, device="cuda")
    offsets[0], offsets[-1] = N - n - 5, N
    y, g, u = experts.train_forward(xs, offsets, *w)
    one = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ref = experts.train_forward(xs[-n:].contiguous(), one, *[l[None] for l in last])
    for a, b in zip((y, g, u), ref):
        # Other tiles may be split otherwise: sums of the same products in fp32.
        assert ((a[-n:].double() - b.double()).abs() <= 2.0 ** -6 * b.double().abs() + 2.0 ** -7).all()
        assert (a[-n:] != 0).any() and (a[-n - 5:-n] == 0).all()


@pytest.mark.parametrize("counts,D,F", [([3, 0, 40], 8, 1 << 20), ([300, 5], 8, 1 << 20), ([3, 40], 1 << 20, 8), ([270], 1 << 20, 8)])
def test_widest(counts, D, F):
    """The widest D and F.  The sums of 2^20 products are formed 32 at a time: 2^15 roundings
    of 2^-24 S, where 2^-12 S stands for those of the other tests."""
    N, E = sum(counts), len(counts)
    t = inputs(N, E, D, F, 4)
    offsets = offsets_of(counts)
    w = (t["wg"], t["wu"], t["wd"])
    y, g, u = experts.train_forward(t["xs"], offsets, *w)
    dxs, dwg, _, dwd = experts.backward(t["dys"], t["xs"], offsets, *w, g, u, want=("dxs", "dwg", "dwd"))
    sums = 2.0 ** -9

    def close(got, ref, terms, rounded=True):
        assert ((got.double() - ref).abs() <= HALF_STEP * ref.abs() + ((1.02 * 2.0 ** -8 if rounded else 0.0) + sums) * terms + 1e-30).all()

    for e, n in enumerate(counts):
        if n == 0:
            assert (dwg[e] == 0).all() and (dwd[e] == 0).all()
            continue
        lo = sum(counts[:e])
        rows = slice(lo + max(0, n - 4), lo + n)  # the last of the expert's; the weights' gradients sum all
        x, dy, wg, wu, wd = (v.double() for v in (t["xs"][rows], t["dys"][rows], t["wg"][e], t["wu"][e], t["wd"][e]))
        close(g[rows], x @ wg, x.abs() @ wg.abs(), rounded=False)
        gd, ud = g[rows].double(), u[rows].double()
        a, da = act(gd, "silu", 1.0)
        # g and u were rounded on their way to here, not to y: 2^-8 (1.1 |g| + |act(g)|) |u|
        # beside the 2^-8 |h| of the rounding of h.
        h = a * ud
        close(y[rows], h @ wd, 3.0 * (a.abs() + gd.abs()) * ud.abs() @ wd.abs())
        dh, dh_terms = dy @ wd.T.contiguous(), dy.abs() @ wd.abs().T.contiguous()
        dg, du = dh * ud * da, dh * a
        spread = 1.0 if F > D else 2.0  # of dh, a sum of D products
        close(dxs[rows], dg @ wg.T + du @ wu.T,
              (dg.abs() + spread * (dh_terms * ud * da).abs()) @ wg.abs().T + (du.abs() + spread * (dh_terms * a).abs()) @ wu.abs().T)
        some = slice(lo, lo + n)
        gd, ud = g[some].double(), u[some].double()
        h = act(gd, "silu", 1.0)[0] * ud
        close(dwd[e], h.T @ t["dys"][some].double(), h.abs().T @ t["dys"][some].double().abs())


def test_gradients_against_differences():
    """Central differences of <dys, ys> in fp64 around the gradients of the kernels: the
    directional derivatives agree to the roundings of the gradients."""
    counts, D, F = [7, 0, 12, 4], 72, 136
    N, E = sum(counts), len(counts)
    t = inputs(N, E, D, F, 5)
    offsets = offsets_of(counts)
    w = (t["wg"], t["wu"], t["wd"])
    _, g, u = experts.train_forward(t["xs"], offsets, *w)
    grads = experts.backward(t["dys"], t["xs"], offsets, *w, g, u)

    def loss(xs, wg, wu, wd):
        total = 0.0
        for e, n in enumerate(counts):
            x = xs[sum(counts[:e]):sum(counts[:e]) + n]
            total = total + ((torch.nn.functional.silu(x @ wg[e]) * (x @ wu[e])) @ wd[e] * t["dys"][sum(counts[:e]):sum(counts[:e]) + n].double()).sum()
        return total

    leaves = [t["xs"].double(), *[v.double() for v in w]]
    gen = torch.Generator(device="cuda").manual_seed(6)
    for i, grad in enumerate(grads):
        d = torch.randn(grad.shape, generator=gen, device="cuda", dtype=torch.float64)
        h = 1e-5
        up, down = ([v + s * h * d if j == i else v for j, v in enumerate(leaves)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * h)
        # g and u, dG, dU and H, and the gradient are rounded to bf16: five roundings of
        # 2^-8 of the terms, in directions of their own.
        assert abs(slope - (grad.double() * d).sum()) <= 5 * 2.0 ** -8 * (grad.double().norm() * d.norm() / d.numel() ** 0.5) * 6


def test_captured_with_other_offsets():
    """A captured step replayed with other routings and rows, between eager steps."""
    E, D, F, N = 6, 264, 520, 300
    t = inputs(N, E, D, F, 7)
    offsets = offsets_of([50] * 6)
    w = (t["wg"], t["wu"], t["wd"])
    ws, own = experts.make_workspace(N, E, D, F), experts.make_workspace(N, E, D, F)
    zeros = lambda cols: torch.zeros((N, cols), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    out = [zeros(D), zeros(F), zeros(F), zeros(D)]

    def step(workspace, out=None):
        y, g, u, dx = out or [zeros(D), zeros(F), zeros(F), zeros(D)]
        experts.train_forward(t["xs"], offsets, *w, out=y, g=g, u=u, workspace=workspace)
        return (y, g, u) + experts.backward(t["dys"], t["xs"], offsets, *w, g, u, dxs=dx, workspace=workspace)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(ws, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = step(ws, out)
    for i, counts in enumerate(([50] * 6, [300, 0, 0, 0, 0, 0], [1, 2, 3, 4, 5, 6], [0] * 6, [0, 150, 0, 149, 1, 0], [50] * 6)):
        offsets.copy_(offsets_of(counts))
        t["xs"].copy_(inputs(N, E, D, F, 20 + i)["xs"])
        for o in out:
            o.zero_()
        graph.replay()
        want = step(own)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(captured, want)), counts


def test_refusals():
    N, E, D, F = 8, 2, 264, 520
    t = inputs(N, E, D, F, 1)
    offsets = offsets_of([4, 4])
    w = (t["wg"], t["wu"], t["wd"])
    g = torch.zeros((N, F), dtype=torch.bfloat16, device="cuda")
    for bad in (lambda: experts.forward(t["xs"].float(), offsets, *w), lambda: experts.forward(t["xs"], offsets.long(), *w),
                lambda: experts.forward(t["xs"], offsets, *w, workspace=torch.zeros(1 << 20, device="cuda"))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: experts.forward(t["xs"], offsets[:-1], *w), lambda: experts.forward(t["xs"], offsets, w[0], w[1], w[0]),
                lambda: experts.forward(t["xs"][:, :256], offsets, *w), lambda: experts.forward(t["xs"], offsets.cpu(), *w),
                lambda: experts.forward(t["xs"], offsets, w[0][0], w[1], w[2]), lambda: experts.forward(t["xs"], offsets, *w, activation="relu"),
                lambda: experts.train_forward(t["xs"], offsets, *w, g=g[:-1]), lambda: experts.backward(t["dys"], t["xs"], offsets, *w, g, g, want=("dx",)),
                lambda: experts.backward(t["dys"], t["xs"], offsets, *w, g, g, dwg=torch.empty_like(w[0]), want=("dxs",)),
                lambda: experts.make_workspace(8, 2, 260, 520)):
        with pytest.raises(ValueError):
            bad()
    small = experts.make_workspace(1, 1, 8, 8)
    with pytest.raises(gmlp.GmlpError, match="NO_MEMORY"):
        experts.forward(t["xs"], offsets, *w, workspace=small)
    # A prepared workspace of another module that is large enough will do.
    y = experts.forward(t["xs"], offsets, *w)
    assert torch.equal(experts.forward(t["xs"], offsets, *w, workspace=gmlp.Workspace(8, D, F, nbytes=1 << 26)), y)
