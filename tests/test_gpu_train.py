"""The Gated MLP's training step on the GPU against plain 64-bit formulas.

Bounds.  Every output is an fp32 sum of products of bf16 numbers, rounded once
to bf16 (relative error at most 2^-8 of the value; half a step).  Before that:

  * G and U have no other rounding than fp32 sums of K products: an error of at
    most K 2^-24 sum |terms|, with K <= 4104, 2^-12 sum |terms| (worst case; the
    sums are random).  dX sums 2 F <= 16400 products, whose worst case, 2^-10, is
    below the 2^-8 for the rounding of its operands that S carries in full.
  * Y = H Wd with H rounded to bf16: sum |H| |Wd| 2^-8.
  * dX, dWg, dWu: dG and dU rounded to bf16, likewise; dWd: H.
  * act and act' in fp32: exp and rcp to 2 units in the last place, 2^-20 is ample.

So each output is within  2^-8 |ref| + (2^-8 + 2^-12 + 2^-20) S (1 + 2^-8),  S the
sum of the absolute values of its terms, with the last factor for the terms of
second order; 1.02 * 2^-8 * S + 2^-8 |ref| covers them at the sizes used, and 2^-12 S + 2^-8 |ref| where no operand was rounded.
"""
import numpy as np
import pytest
import torch

from paper_2606_26344_amd import gmlp, train

pytestmark = pytest.mark.gpu

HALF_STEP = 2.0 ** -8
ROUNDED = 1.02 * 2.0 ** -8 + 2.0 ** -12


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


def inputs(T, D, F, seed):
    gen = torch.Generator().manual_seed(seed)
    n = lambda r, c, s: (torch.randn((r, c), generator=gen) * s).to(torch.bfloat16)  # noqa: E731
    t = dict(x=n(T, D, 1.0), wg=n(D, F, D ** -0.5), wu=n(D, F, D ** -0.5), wd=n(F, D, F ** -0.5), dy=n(T, D, 1.0))
    return t


def check(name, got, ref, terms, rounded=True):
    got = got.double()
    assert got.shape == ref.shape, name
    bound = HALF_STEP * ref.abs() + (ROUNDED if rounded else 2.0 ** -12) * terms + 1e-30
    ratio = ((got - ref).abs() / bound).max().item() if ref.numel() else 0.0
    print("%s: max |err|/bound = %.3f" % (name, ratio), flush=True)
    assert ratio <= 1.0, name


def run(T, D, F, activation="silu", beta=1.0, seed=0, want=train.GRADIENTS, workspace=True, data=None):
    print("train T=%d D=%d F=%d %s want=%s" % (T, D, F, activation, want), flush=True)
    t = data or inputs(T, D, F, seed)
    dev = {k: v.cuda() for k, v in t.items()}
    kw = dict(activation=activation, beta=beta, workspace=train.make_workspace(T, D, F) if workspace else None)
    y, g, u = train.forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], **kw)
    grads = train.backward(dev["dy"], dev["x"], dev["wg"], dev["wu"], dev["wd"], g, u, want=want, **kw)
    torch.cuda.synchronize()
    d = {k: v.double() for k, v in dev.items()}  # plain 64-bit matrix products
    check("g", g, d["x"] @ d["wg"], d["x"].abs() @ d["wg"].abs(), rounded=False)
    check("u", u, d["x"] @ d["wu"], d["x"].abs() @ d["wu"].abs(), rounded=False)
    # Y from the unrounded G and U.
    ge, ue = d["x"] @ d["wg"], d["x"] @ d["wu"]
    h = act(ge, activation, beta)[0] * ue
    # G and U in fp32 carry up to 2^-12 of their terms into H.
    slack = (act(ge, activation, beta)[0].abs() + 1.2 * max(1.0, beta) * ue.abs()) * 2.0 ** -12 * \
        (d["x"].abs() @ torch.maximum(d["wg"].abs(), d["wu"].abs()))
    check("y", y, h @ d["wd"], (h.abs() + 2.0 ** 8 * slack) @ d["wd"].abs())
    # The backward pass from the G and U it was given.
    gd, ud = g.double(), u.double()
    a, da = act(gd, activation, beta)
    dh, dh_terms = d["dy"] @ d["wd"].T, d["dy"].abs() @ d["wd"].abs().T
    dg, du, h = dh * ud * da, dh * a, a * ud
    # dH in fp32: 2^-12 of its terms, beside the rounding of dG and dU (2^-8).
    dgt = dg.abs() + 2.0 ** -4 * (dh_terms * ud * da).abs()
    dut = du.abs() + 2.0 ** -4 * (dh_terms * a).abs()
    refs = {"dx": (dg @ d["wg"].T + du @ d["wu"].T, dgt @ d["wg"].abs().T + dut @ d["wu"].abs().T),
            "dwg": (d["x"].T @ dg, d["x"].abs().T @ dgt), "dwu": (d["x"].T @ du, d["x"].abs().T @ dut),
            "dwd": (h.T @ d["dy"], h.abs().T @ d["dy"].abs())}
    for name, got in zip(train.GRADIENTS, grads):
        if name in want:
            check(name, got, *refs[name])
        else:
            assert got is None
    return y, g, u, grads


SHAPES = [(1, 8, 8), (1, 264, 520), (3, 264, 520), (16, 256, 512), (33, 520, 264), (64, 136, 1032), (65, 264, 264),
          (127, 264, 1032), (130, 1032, 520), (300, 1032, 2056), (520, 264, 520)]


@pytest.mark.parametrize("T,D,F", SHAPES, ids=["T%dD%dF%d" % s for s in SHAPES])
def test_training_step(T, D, F):
    run(T, D, F, seed=T * 7 + D)


@pytest.mark.parametrize("activation,beta", [("swish", 1.702), ("sigmoid", 1.0), ("swish", -0.5)])
@pytest.mark.parametrize("T,D,F", [(5, 264, 520), (200, 264, 520)])
def test_activations(T, D, F, activation, beta):
    run(T, D, F, activation, beta, seed=T)


# (T, D, F, tile of dH, of dX, of dW): every tile of the plan, most of them with
# whole tiles, ragged ones and split sums.
LARGE, PAIR, SMALL, SHORT, T32, T64, T96, T160, T192, T320 = (
    "4, 2, 2, 4, 2, 64, 1", "2, 2, 2, 4, 3, 32, 2", "2, 2, 2, 2, 4, 64, 1", "2, 4, 2, 1, 4, 32, 2", "4, 1, 1, 1, 4, 64, 1",
    "4, 1, 1, 2, 4, 64, 1", "4, 1, 1, 3, 4, 64, 1", "4, 1, 1, 5, 4, 64, 1", "4, 1, 1, 6, 3, 64, 1", "4, 2, 1, 5, 2, 64, 1")
TILES = [(3, 264, 520, T32, T32, SHORT), (260, 264, 520, None, None, SHORT), (80, 1032, 4104, None, None, PAIR),
         (600, 264, 520, None, None, SMALL), (3000, 264, 520, None, None, SMALL), (5000, 1032, 2056, None, None, PAIR),
         (1030, 520, 1032, T64, None, None),
         (1030, 1032, 2056, T96, SMALL, None), (600, 520, 1032, None, T64, None), (330, 1288, 2312, None, T96, PAIR),
         (400, 2056, 4104, None, T160, None), (520, 2056, 4104, None, T192, None), (40, 2056, 8200, T64, None, None),
         (130, 4104, 8200, T160, T160, None), (180, 4104, 8200, T192, T192, None), (300, 4104, 8200, T320, T320, None),
         (100, 4104, 8200, SMALL, None, None), (600, 4104, 8200, LARGE, None, None), (400, 4104, 8200, None, LARGE, None),
         (2100, 2056, 8200, None, None, LARGE)]


@pytest.mark.parametrize("T,D,F,dh,dx,dw", TILES, ids=["T%dD%dF%d" % c[:3] for c in TILES])
def test_tiles(T, D, F, dh, dx, dw):
    names = [k[0].split("Shape<")[1].split(">")[0] for k in train.describe(T, D, F)]
    assert all(want in (None, have) for want, have in zip((dh, dx, dw), names)), names
    run(T, D, F, seed=3)


# (T, D, F, tile of the forward pass, streamed weights).
FORWARD_TILES = [(20, 264, 520, "2, 4, 1, 1, 1, 4, 64", True), (50, 264, 520, "2, 4, 1, 1, 2, 3, 64", True),
                 (90, 264, 520, "2, 4, 1, 1, 3, 3, 64", True),
                 (100, 264, 520, "2, 4, 2, 1, 2, 3, 64", True), (150, 264, 16648, "2, 4, 1, 1, 6, 4, 32", True),
                 (250, 264, 16648, "2, 4, 2, 1, 4, 2, 64", True), (300, 264, 12296, "2, 4, 1, 1, 6, 4, 32", False),
                 (500, 136, 16392, "2, 4, 2, 1, 4, 2, 64", False), (300, 264, 520, "2, 4, 2, 1, 2, 3, 64", False)]


@pytest.mark.parametrize("T,D,F,tile,stream", FORWARD_TILES, ids=["T%dD%dF%d" % c[:3] for c in FORWARD_TILES])
def test_forward_tiles(T, D, F, tile, stream):
    name = train.describe(T, D, F, backward=False)[0][0]
    assert tile is None or "<%s>, 3" % tile in name, name
    assert name.endswith("true>" if stream else "false>"), name
    run(T, D, F, seed=5, want=())


@pytest.mark.parametrize("T", [1, 256])
def test_widest_tensors(T):
    """F = 2^22: the last of 256 rows ends 2 GiB after the first begins.

    dX sums 2^23 products, in fp32 in 85 (T = 1: more) pieces of MFMA steps of 32: (2^23 /
    85 / 32 + 32 + 256) 2^-24 < 2^-12 of its terms, as above."""
    D, F = 8, 1 << 22
    print("train T=%d D=%d F=%d" % (T, D, F), flush=True)
    gen = torch.Generator(device="cuda").manual_seed(T)
    n = lambda r, c, s: (torch.randn((r, c), generator=gen, device="cuda") * s).to(torch.bfloat16)  # noqa: E731
    x, wg, wu, wd, dy = n(T, D, 1.0), n(D, F, D ** -0.5), n(D, F, D ** -0.5), n(F, D, F ** -0.5), n(T, D, 1.0)
    ws = train.make_workspace(T, D, F)
    y, g, u = train.forward(x, wg, wu, wd, workspace=ws)
    dx, dwg, dwu, dwd = train.backward(dy, x, wg, wu, wd, g, u, workspace=ws)
    xd, dyd = x.double(), dy.double()
    total = torch.zeros((3, T, D), dtype=torch.float64, device="cuda")
    step = 1 << 18
    for c in range(0, F, step):
        cols = slice(c, c + step)
        wgd, wud, wdd = wg[:, cols].double(), wu[:, cols].double(), wd[cols].double()
        gd, ud = g[:, cols].double(), u[:, cols].double()
        assert ((gd - xd @ wgd).abs() <= HALF_STEP * gd.abs() * 1.01 + 2.0 ** -12 * (xd.abs() @ wgd.abs())).all(), c
        assert ((ud - xd @ wud).abs() <= HALF_STEP * ud.abs() * 1.01 + 2.0 ** -12 * (xd.abs() @ wud.abs())).all(), c
        a, da = act(gd, "silu", 1.0)
        dh, dht = dyd @ wdd.T, dyd.abs() @ wdd.abs().T
        dg, du, h = dh * ud * da, dh * a, a * ud
        dgt, dut = dg.abs() + 2.0 ** -4 * (dht * ud * da).abs(), du.abs() + 2.0 ** -4 * (dht * a).abs()
        total[0] += dg @ wgd.T + du @ wud.T
        total[1] += dgt @ wgd.abs().T + dut @ wud.abs().T
        total[2] += h @ wdd
        for name, got, ref, terms in (("dwg", dwg[:, cols], xd.T @ dg, xd.abs().T @ dgt),
                                      ("dwu", dwu[:, cols], xd.T @ du, xd.abs().T @ dut),
                                      ("dwd", dwd[cols], h.T @ dyd, h.abs().T @ dyd.abs())):
            bound = HALF_STEP * ref.abs() + ROUNDED * terms + 1e-30
            assert ((got.double() - ref).abs() <= bound).all(), (name, c)
    check("dx", dx, total[0], total[1])


@pytest.mark.parametrize("T,D,F", [(20, 256, 512), (200, 1024, 4096), (130, 4096, 8192)])
def test_outputs_off_their_lines(T, D, F):
    """Weight gradients that start inside a 128-byte line, and those that start on one."""
    assert train.describe(T, D, F)[2][0].endswith("true>")
    t = {k: v.cuda() for k, v in inputs(T, D, F, 4).items()}
    _, g, u = train.forward(t["x"], t["wg"], t["wu"], t["wd"])
    args = (t["dy"], t["x"], t["wg"], t["wu"], t["wd"], g, u)
    want = run(T, D, F, seed=4)[3]
    for off in (8, 40):
        room = [torch.full((D * F + 128,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        outs = [b[off:off + D * F].view(shape) for b, shape in zip(room, ((D, F), (D, F), (F, D)))]
        got = train.backward(*args, dwg=outs[0], dwu=outs[1], dwd=outs[2])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert all((b[:off] == 7).all() and (b[off + D * F:] == 7).all() for b in room)


@pytest.mark.parametrize("want", [("dx",), ("dwd",), ("dwg", "dwu"), ("dx", "dwu"), ()])
def test_wanted_gradients_only(want):
    run(70, 264, 520, want=want, seed=9)


def test_without_workspace_is_bitwise_the_same():
    a = run(130, 264, 1032, seed=4)
    b = run(130, 264, 1032, seed=4, workspace=False)
    for p, q in zip((*a[:3], *a[3]), (*b[:3], *b[3])):
        assert torch.equal(p.view(torch.int16), q.view(torch.int16))


def test_no_tokens():
    t = {k: v.cuda() for k, v in inputs(0, 264, 520, 1).items()}
    y, g, u = train.forward(t["x"], t["wg"], t["wu"], t["wd"])
    assert y.shape == (0, 264) and g.shape == u.shape == (0, 520)
    outs = [torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((264, 520), (264, 520), (520, 264))]
    dx, *dw = train.backward(t["dy"], t["x"], t["wg"], t["wu"], t["wd"], g, u, dwg=outs[0], dwu=outs[1], dwd=outs[2])
    torch.cuda.synchronize()
    assert dx.shape == (0, 264)
    assert all(not w.any() for w in dw)


def test_saturated_gates_have_finite_gradients():
    # Gates of +-3e4: the sigmoid is 0 or 1, its derivative 0.
    t = inputs(9, 264, 520, 2)
    t["x"] = (t["x"].float() * 1e4).to(torch.bfloat16)
    dev = {k: v.cuda() for k, v in t.items()}
    for activation in ("silu", "sigmoid"):
        y, g, u = train.forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], activation=activation)
        grads = train.backward(dev["dy"], dev["x"], dev["wg"], dev["wu"], dev["wd"], g, u, activation=activation)
        assert all(torch.isfinite(v.float()).all() for v in (y, *grads))


def test_nan_stays_in_its_token():
    t = inputs(40, 264, 520, 6)
    dev = {k: v.cuda() for k, v in t.items()}
    ws = train.make_workspace(40, 264, 520)
    y, g, u = train.forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], workspace=ws)
    clean = train.backward(dev["dy"], dev["x"], dev["wg"], dev["wu"], dev["wd"], g, u, workspace=ws)[0].clone()
    g[17, 5] = float("nan")
    dx = train.backward(dev["dy"], dev["x"], dev["wg"], dev["wu"], dev["wd"], g, u, want=("dx",), workspace=ws)[0]
    rows = [i for i in range(40) if i != 17]
    assert torch.isnan(dx[17].float()).all()
    assert torch.equal(dx[rows].view(torch.int16), clean[rows].view(torch.int16))


def test_gradients_against_differences():
    # The loss sum(dy * y) in 64 bits, its directional derivatives by central
    # differences against the kernels' gradients.
    T, D, F = 24, 136, 264
    t = inputs(T, D, F, 11)
    _, g, u, grads = run(T, D, F, data=t)
    d = {k: v.double() for k, v in t.items()}

    def loss(p):
        gg = p["x"] @ p["wg"]
        return ((gg * torch.sigmoid(gg) * (p["x"] @ p["wu"])) @ p["wd"] * d["dy"]).sum()

    gen = torch.Generator().manual_seed(5)
    for name, got in zip(("x", "wg", "wu", "wd"), grads):
        v = torch.randn(d[name].shape, generator=gen, dtype=torch.float64) * d[name].abs().mean()
        eps = 1e-4
        up, down = dict(d), dict(d)
        up[name], down[name] = d[name] + eps * v, d[name] - eps * v
        numeric = (loss(up) - loss(down)).item() / (2 * eps)
        mine = (got.cpu().double() * v).sum().item()
        # The gradient's elements are off by independent roundings of 2^-8 of
        # their size at most, twice (dG or H, and the result), and G and U by
        # another each; five times the root of the sum of their squares.
        scale = (got.cpu().double() * v).norm().item()
        assert abs(mine - numeric) <= 5 * 4 * HALF_STEP * scale + 1e-6 * abs(numeric), name


@pytest.mark.parametrize("T,D,F", [(16, 256, 512), (200, 1032, 2056)])
def test_captured_steps_replay(T, D, F):
    t = {k: v.cuda() for k, v in inputs(T, D, F, 8).items()}
    stream = torch.cuda.Stream()
    outs = {}

    def call(x):
        y, g, u = train.forward(x, t["wg"], t["wu"], t["wd"], out=outs["y"], g=outs["g"], u=outs["u"],
                                workspace=outs["ws"], stream=stream)
        train.backward(t["dy"], x, t["wg"], t["wu"], t["wd"], g, u, dx=outs["dx"], dwg=outs["dwg"], dwu=outs["dwu"],
                       dwd=outs["dwd"], workspace=outs["ws"], stream=stream)

    names = {"y": (T, D), "g": (T, F), "u": (T, F), "dx": (T, D), "dwg": (D, F), "dwu": (D, F), "dwd": (F, D)}
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        outs["ws"] = train.make_workspace(T, D, F, stream=stream)
        outs.update({k: torch.empty(s, dtype=torch.bfloat16, device="cuda") for k, s in names.items()})
        call(t["x"])
    torch.cuda.synchronize()
    eager = {k: outs[k].clone() for k in names}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(t["x"])
    other = t["x"] * 0.5
    torch.cuda.synchronize()
    for i in range(4):
        with torch.cuda.stream(stream):
            call(other)
            for k in names:
                outs[k].zero_()
            graph.replay()
        torch.cuda.synchronize()
        for k in names:
            assert torch.equal(outs[k].view(torch.int16), eager[k].view(torch.int16)), (i, k)


def test_forward_is_the_forward_of_the_inference_path():
    # The same y as gmlp.forward up to the order of the fp32 sums.
    T, D, F = 300, 1032, 2056
    t = {k: v.cuda() for k, v in inputs(T, D, F, 21).items()}
    y = train.forward(t["x"], t["wg"], t["wu"], t["wd"])[0].float()
    z = gmlp.forward(t["x"], t["wg"], t["wu"], t["wd"]).float()
    assert (y - z).abs().max() <= 4 * HALF_STEP * z.abs().max()
    assert np.isfinite(y.cpu().numpy()).all()
