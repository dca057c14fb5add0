"""The norms between two blocks on the GPU against plain 64-bit formulas.

Bounds.  The kernels compute in fp32 and round once: 2^-8 of the value for a bf16
output, 2^-24 for an fp32 one, plus the fp32 work before it.  A sum over a row of
D <= 16384 values is a tree of at most 16 additions per thread, 6 levels and 16
waves, so its relative error is below 47 * 2^-24 of the sum of absolute values; the
squares' sums enter under a root.  Every output is a handful of products and
sums of such, so its error before rounding is below 2^-17 of the sum of the
absolute values of its terms ("terms" below).  Sums over T <= 1100 rows (the
gradients of gains) add 2^-24 per addition, at most 2^-13 of their terms.
"""
import pytest
import torch

from paper_2606_26344_amd import block_norm, gmlp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def inputs(T, D, res=torch.bfloat16, post=True, gate="channel", seed=0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda shape, s=1.0, m=0.0, t=torch.bfloat16: (torch.randn(shape, generator=gen) * s + m).to(t)  # noqa: E731
    return {"y": n((T, D)), "res": n((T, D), 2.0, t=res), "w_pre": n((D,), 0.3, 1.0),
            "w_post": n((D,), 0.3, 1.0) if post else None,
            "gate": n((D,), 0.3, 1.0) if gate == "channel" else n((T, D)) if gate == "token" else None,
            "dxn": n((T, D)), "dr": n((T, D), t=res)}


def check(name, got, ref, terms, slack=2.0 ** -17):
    half = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    got = got.cpu().double()
    assert got.shape == ref.shape, name
    bound = half * ref.abs() + slack * terms + 1e-35
    ratio = ((got - ref).abs() / bound).max().item() if ref.numel() else 0.0
    print("%s: max |err|/bound = %.3f" % (name, ratio), flush=True)
    assert ratio <= 1.0, name


def rms(v, eps):
    return (v.square().mean(1, keepdim=True) + eps).sqrt()


def run(T, D, res=torch.bfloat16, post=True, gate="channel", res_scale=1.0, eps=1e-6, seed=0, with_dr=True, data=None,
        workspace=True):
    print("norm T=%d D=%d %s post=%s gate=%s" % (T, D, res, post, gate), flush=True)
    t = data or inputs(T, D, res, post, gate, seed)
    dev = {k: None if v is None else v.cuda() for k, v in t.items()}
    kw = dict(w_pre=dev["w_pre"], w_post=dev["w_post"], gate=dev["gate"], post=post, res_scale=res_scale, eps=eps)
    r, xn = block_norm.forward(dev["y"], dev["res"], **kw)
    ws = block_norm.make_workspace(T, D) if workspace else None
    grads = block_norm.backward(dev["dxn"], dev["dr"] if with_dr else None, dev["y"], r, workspace=ws, **kw)
    torch.cuda.synchronize()
    d = {k: None if v is None else v.double() for k, v in t.items()}
    one = torch.ones(1, dtype=torch.float64)
    w_pre = one if d["w_pre"] is None else d["w_pre"]
    w_post = one if d["w_post"] is None else d["w_post"]
    g = one if d["gate"] is None else d["gate"]
    z = torch.zeros_like(d["res"]) if d["y"] is None else d["y"] / rms(d["y"], eps) * w_post if post else d["y"]
    re = res_scale * d["res"] + g * z
    terms = (res_scale * d["res"]).abs() + (g * z).abs()
    check("r", r, re, terms)
    check("xn", xn, re / rms(re, eps) * w_pre, terms / rms(re, eps) * w_pre.abs())
    dy, dres, dw_pre, dw_post, dgate = grads
    r64 = r.cpu().double()
    xhat, a = r64 / rms(r64, eps), d["dxn"] * w_pre
    dr = d["dr"] if with_dr else torch.zeros_like(r64)
    total = dr + (a - xhat * (a * xhat).mean(1, keepdim=True)) / rms(r64, eps)
    tt = dr.abs() + (a.abs() + xhat.abs() * (a * xhat).abs().mean(1, keepdim=True)) / rms(r64, eps)
    check("dres", dres, res_scale * total, abs(res_scale) * tt)
    if d["w_pre"] is None:
        assert dw_pre is None
    else:
        check("dw_pre", dw_pre, (d["dxn"] * xhat).sum(0), (d["dxn"] * xhat).abs().sum(0), 2.0 ** -13)
    if d["y"] is None:
        assert dy is None and dw_post is None and dgate is None
        return r, xn, grads
    dz, dzt = total * g, tt * g.abs()
    if post:
        yhat, b = d["y"] / rms(d["y"], eps), dz * w_post
        bt = dzt * w_post.abs()
        check("dy", dy, (b - yhat * (b * yhat).mean(1, keepdim=True)) / rms(d["y"], eps),
              (bt + yhat.abs() * (bt * yhat.abs()).mean(1, keepdim=True)) / rms(d["y"], eps))
    else:
        check("dy", dy, dz, dzt)
    if d["w_post"] is None:
        assert dw_post is None
    else:
        check("dw_post", dw_post, (dz * yhat).sum(0), (dzt * yhat.abs()).sum(0), 2.0 ** -13)
    if gate == "token":
        check("dgate", dgate, total * z, tt * z.abs())
    elif gate == "channel":
        check("dgate", dgate, (total * z).sum(0), (tt * z.abs()).sum(0), 2.0 ** -13)
    else:
        assert dgate is None
    return r, xn, grads


SHAPES = [(1, 8), (3, 8), (1, 4096), (5, 504), (33, 520), (7, 1032), (300, 1024), (64, 2056), (1100, 264), (9, 4104),
          (20, 8192), (3, 12296), (700, 8200), (5, 16384), (600, 4096)]


@pytest.mark.parametrize("T,D", SHAPES, ids=["T%dD%d" % s for s in SHAPES])
def test_widths(T, D):
    run(T, D, seed=T + D)


@pytest.mark.parametrize("res", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("post", [False, True])
def test_options(res, gate, post):
    run(37, 1288, res, post, gate, res_scale=0.5, eps=1e-5, seed=3)


@pytest.mark.parametrize("T", [1, 700])
def test_fp32_stream_many_rows(T):
    run(T, 2048, torch.float32, seed=T)


def test_first_block_and_last_block():
    t = inputs(11, 776, post=False, gate="none", seed=1)
    t["y"] = None
    run(11, 776, post=False, gate="none", res_scale=0.25, data=t)
    run(11, 776, with_dr=False, seed=2)


def test_no_gains():
    t = inputs(19, 264, post=True, gate="none", seed=5)
    t["w_pre"] = t["w_post"] = None
    run(19, 264, post=True, gate="none", data=t)


def test_zero_rows_and_padding():
    # A row of zeros has a norm of zero with eps > 0, and finite gradients; a
    # NaN stays in its row, the gains' gradients aside.
    t = inputs(12, 520, seed=7)
    t["y"][3] = 0
    t["res"][3] = 0
    run(12, 520, data=t, eps=1e-5)
    clean = inputs(12, 520, seed=7)
    dirty = {k: v.clone() for k, v in clean.items()}
    dirty["y"][5, 3] = float("nan")
    outs = []
    for data in (clean, dirty):
        dev = {k: v.cuda() for k, v in data.items()}
        kw = dict(w_pre=dev["w_pre"], w_post=dev["w_post"], gate=dev["gate"], post=True)
        r, xn = block_norm.forward(dev["y"], dev["res"], **kw)
        outs.append((r, xn) + block_norm.backward(dev["dxn"], dev["dr"], dev["y"], r, **kw)[:2])
    rows = [i for i in range(12) if i != 5]
    for a, b in zip(*outs):
        assert torch.equal(a[rows].view(torch.int16), b[rows].view(torch.int16))
        assert torch.isnan(b[5].float()).all()


def test_gains_that_are_not_finite_stay_in_their_channel():
    # A row shorter than the block's threads: the threads past it add nothing.
    t = inputs(4, 72, seed=8)
    t["w_pre"][0] = float("inf")
    dev = {k: v.cuda() for k, v in t.items()}
    r, xn = block_norm.forward(dev["y"], dev["res"], w_pre=dev["w_pre"], w_post=dev["w_post"], gate=dev["gate"], post=True)
    assert torch.isinf(xn[:, 0].float()).all() and torch.isfinite(xn[:, 1:].float()).all()


def test_no_rows():
    t = inputs(0, 264)
    dev = {k: v.cuda() for k, v in t.items()}
    kw = dict(w_pre=dev["w_pre"], w_post=dev["w_post"], gate=dev["gate"], post=True)
    r, xn = block_norm.forward(dev["y"], dev["res"], **kw)
    assert r.shape == xn.shape == (0, 264)
    dy, dres, *sums = block_norm.backward(dev["dxn"], dev["dr"], dev["y"], r, **kw)
    assert dy.shape == dres.shape == (0, 264) and all(not s.any() for s in sums)


def test_in_place():
    t = inputs(30, 1032, seed=4)
    dev = {k: v.cuda() for k, v in t.items()}
    kw = dict(w_pre=dev["w_pre"], w_post=dev["w_post"], gate=dev["gate"], post=True, res_scale=0.5)
    r, xn = block_norm.forward(dev["y"], dev["res"], **kw)
    dy, dres, *sums = block_norm.backward(dev["dxn"], dev["dr"], dev["y"], r, **kw)
    res, dxn, dr, y = (dev[k].clone() for k in ("res", "dxn", "dr", "y"))
    dy2, dres2, *sums2 = block_norm.backward(dxn, dr, y, r, dy=dxn, dres=dr, **kw)
    r2, xn2 = block_norm.forward(y, res, r=res, xn=y, **kw)
    assert r2 is res and xn2 is y and dy2 is dxn and dres2 is dr
    for a, b in zip((r, xn, dy, dres, *sums), (r2, xn2, dy2, dres2, *sums2)):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_gradients_against_differences():
    T, D, eps = 6, 136, 1e-3
    t = inputs(T, D, torch.float32, seed=12)
    _, _, grads = run(T, D, torch.float32, data=t, eps=eps, res_scale=0.75)
    d = {k: v.double() for k, v in t.items()}

    def loss(p):
        r = 0.75 * p["res"] + p["gate"] * p["y"] / rms(p["y"], eps) * p["w_post"]
        return (r * d["dr"]).sum() + (r / rms(r, eps) * p["w_pre"] * d["dxn"]).sum()

    gen = torch.Generator().manual_seed(6)
    for name, got in zip(("y", "res", "w_pre", "w_post", "gate"), grads):
        v = torch.randn(d[name].shape, generator=gen, dtype=torch.float64)
        up, down = dict(d), dict(d)
        up[name], down[name] = d[name] + 1e-5 * v, d[name] - 1e-5 * v
        numeric = (loss(up) - loss(down)).item() / 2e-5
        mine = (got.cpu().double() * v).sum().item()
        # Independent roundings of 2^-8 at most per element: five times the
        # root of the sum of squares; the differences' own error 1e-6.
        assert abs(mine - numeric) <= 5 * 2.0 ** -8 * (got.cpu().double() * v).norm().item() + 1e-6 * abs(numeric), name


def test_captured_calls_replay():
    T, D = 300, 1032
    t = {k: v.cuda() for k, v in inputs(T, D, seed=15).items()}
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ws = block_norm.make_workspace(T, D, stream=stream)
        r, xn, dy, dres = (torch.empty_like(t["y"]) for _ in range(4))
    outs = {}

    def call(y):
        kw = dict(w_pre=t["w_pre"], w_post=t["w_post"], gate=t["gate"], post=True, stream=stream)
        block_norm.forward(y, t["res"], r=r, xn=xn, **kw)
        outs["sums"] = block_norm.backward(t["dxn"], t["dr"], y, r, dy=dy, dres=dres, workspace=ws, **kw)[2:]

    call(t["y"])
    torch.cuda.synchronize()
    eager = [v.clone() for v in (r, xn, dy, dres, *outs["sums"])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call(t["y"])
    kept = outs["sums"]
    other = t["y"] * 0.5
    torch.cuda.synchronize()
    for i in range(4):
        with torch.cuda.stream(stream):
            call(other)
            for v in (r, xn, dy, dres, *kept):
                v.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((r, xn, dy, dres, *kept), eager):
            assert torch.equal(a.view(torch.int16), b.view(torch.int16)), i


def test_runs_are_reproducible_without_a_workspace():
    a = run(700, 520, seed=9)
    b = run(700, 520, seed=9, workspace=False)
    for p, q in zip((*a[:2], *a[2]), (*b[:2], *b[2])):
        assert torch.equal(p.view(torch.int16), q.view(torch.int16))
