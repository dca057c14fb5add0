"""The training step, the norms between blocks and the 4-bit products together, as a
model uses them: two blocks trained, and two blocks decoding with 4-bit weights.

Bounds.  A rounding to bf16 moves each element of a tensor by at most 2^-8 of its
value, hence the tensor by at most 2^-8 of its L2 norm.  On its way to a result such
a displacement goes through products and norms whose gain for a random direction is
about that of the tensor itself; where gate and up are multiplied, twice (both move).
A result of the two blocks' step depends on at most 2 (Xn, G, U, H, Y) = 10 roundings
of the forward pass, counted twice, and 2 (dY, dG, dU, dX) + 3 of the backward pass:
31 2^-8 = 0.12 of its norm if all of them pointed one way; a path, a gain or a factor
left out is an error of the order of 1.  Decoding: 2 (Xn, H, Y) + R and the last Xn,
8 twice = 16 2^-8.
"""
import pytest
import torch

from paper_2606_26344_amd import block_norm, gmlp, train, w4

pytestmark = pytest.mark.gpu

EPS, SCALE = 1e-6, 0.75


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def model(T, D, F, res, seed=0):
    """Two blocks' weights and gains, x and the gradient that reaches the last norm."""
    gen = torch.Generator().manual_seed(seed)
    n = lambda *shape, s=1.0, at=0.0: (torch.randn(shape, generator=gen) * s + at).to(torch.bfloat16).cuda()  # noqa: E731
    m = dict(res=n(T, D).to(res), dout=n(T, D), pre0=n(D, s=0.1, at=1.0))
    for i in (1, 2):
        m.update({"wg%d" % i: n(D, F, s=D ** -0.5), "wu%d" % i: n(D, F, s=D ** -0.5), "wd%d" % i: n(F, D, s=F ** -0.5),
                  "pre%d" % i: n(D, s=0.1, at=1.0), "post%d" % i: n(D, s=0.1, at=1.0), "gate%d" % i: n(D, s=0.3, at=0.5)})
    return m


def options(m, i):
    return dict(w_pre=m["pre%d" % i], w_post=m["post%d" % i], gate=m["gate%d" % i], post=True, res_scale=SCALE, eps=EPS)


def step(m, workspace=None, norm_workspace=None, stream=None):
    """Forward and backward through norm, block, norm, block, norm; every gradient by name."""
    kw = dict(workspace=workspace, stream=stream)
    r, xn = block_norm.forward(None, m["res"], w_pre=m["pre0"], eps=EPS, stream=stream)
    kept = []
    for i in (1, 2):
        w = [m["w%s%d" % (k, i)] for k in "gud"]
        y, g, u = train.forward(xn, *w, **kw)
        r_next, xn_next = block_norm.forward(y, r, stream=stream, **options(m, i))
        kept.append((r, xn, w, y, g, u, r_next))
        r, xn = r_next, xn_next
    out = {"out": xn, "r": r}
    dxn, dr = m["dout"], None
    for i in (2, 1):
        r0, x, w, y, g, u, r1 = kept[i - 1]
        dy, dr, out["pre%d" % i], out["post%d" % i], out["gate%d" % i] = block_norm.backward(
            dxn, dr, y, r1, workspace=norm_workspace, stream=stream, **options(m, i))
        dxn, out["wg%d" % i], out["wu%d" % i], out["wd%d" % i] = train.backward(dy, x, *w, g, u, **kw)
    _, out["res"], out["pre0"], _, _ = block_norm.backward(dxn, dr, None, kept[0][0], w_pre=m["pre0"], eps=EPS,
                                                           workspace=norm_workspace, stream=stream)
    return out


def norm64(v, w):
    return v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w


def step64(m):
    """The same in 64 bits, with gradients by automatic differentiation."""
    p = {k: v.double().requires_grad_(k != "dout") for k, v in m.items()}
    r, xn = p["res"], norm64(p["res"], p["pre0"])
    for i in (1, 2):
        g, u = xn @ p["wg%d" % i], xn @ p["wu%d" % i]
        y = (torch.nn.functional.silu(g) * u) @ p["wd%d" % i]
        r = SCALE * r + p["gate%d" % i] * norm64(y, p["post%d" % i])
        xn = norm64(r, p["pre%d" % i])
    xn.backward(p["dout"])
    out = {k: v.grad for k, v in p.items() if v.requires_grad}
    out.update(out=xn.detach(), r=r.detach())
    return out


def check(got, want, roundings):
    assert set(got) == set(want)
    for name in want:
        assert got[name].shape == want[name].shape
        off = ((got[name].double() - want[name]).norm() / want[name].norm()).item()
        print("%s: %.5f of its norm" % (name, off), flush=True)
        assert off <= roundings * 2.0 ** -8, name


@pytest.mark.parametrize("T,D,F,res", [(1, 256, 520, torch.float32), (7, 264, 520, torch.bfloat16),
                                       (200, 520, 1032, torch.float32), (300, 1032, 2056, torch.bfloat16)])
def test_training_two_blocks(T, D, F, res):
    m = model(T, D, F, res, seed=T)
    check(step(m, train.make_workspace(T, D, F), block_norm.make_workspace(T, D)), step64(m), 31)


def same(a, b):
    assert set(a) == set(b)
    return all(torch.equal(a[k], b[k]) for k in a)


def test_captured_step_replays():
    """A step captured once, replayed on new inputs between eager steps of the same leaves."""
    T, D, F = 130, 520, 1032
    m, other = model(T, D, F, torch.float32, seed=1), model(T, D, F, torch.float32, seed=2)
    ws, nws = train.make_workspace(T, D, F), block_norm.make_workspace(T, D)
    own = (train.make_workspace(T, D, F), block_norm.make_workspace(T, D))
    first, second = step(m, *own), step(other, *own)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    leaves = {k: v.clone() for k, v in m.items()}
    with torch.cuda.stream(stream):
        step(leaves, ws, nws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = step(leaves, ws, nws)
    for source, want in ((m, first), (other, second), (m, first), (other, second)):
        for k, v in leaves.items():
            v.copy_(source[k])
        graph.replay()
        assert same(step(m, *own), first)
        torch.cuda.synchronize()
        assert same(captured, want)


class Handle:
    """A stream object that is only its handle."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.parametrize("workspace", [False, True])
def test_two_steps_at_once(workspace):
    """On two streams that do not wait for each other, with memory churning on the current one."""
    T, D, F = 130, 520, 1032
    models = [model(T, D, F, torch.bfloat16, seed=s) for s in (3, 4)]
    want = [step(m) for m in models]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [(train.make_workspace(T, D, F), block_norm.make_workspace(T, D)) if workspace else () for _ in models]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for m, st, ws in zip(models, streams, spaces):
            got.append(step(m, *ws, stream=Handle(st)))
            junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]
            del junk
        torch.cuda.synchronize()
        assert all(same(g, w) for g, w in zip(got, want))


def test_one_prepared_workspace_serves_every_call():
    """Training step, inference and 4-bit products one after the other; each leaves it prepared."""
    T, D, F = 40, 1032, 2056
    m = model(T, D, F, torch.bfloat16, seed=5)
    ws = train.make_workspace(T, D, F)
    assert ws.nbytes >= max(gmlp.workspace_size(T, D, F), w4.workspace_size(T, D, F))
    weights = [m["wg1"], m["wu1"], m["wd1"]]
    packed = [w4.from_weight(w, 64) for w in weights]
    x = m["dout"]
    calls = [lambda **kw: gmlp.forward(x, *weights, **kw), lambda **kw: w4.forward(x, *packed, **kw),
             lambda **kw: train.forward(x, *weights, **kw)[0]]
    want = [call() for call in calls]
    grads = step(m)
    for _ in range(3):
        for call, y in zip(calls, want):
            assert torch.equal(call(workspace=ws), y)
        assert same(step(m, ws), grads)


@pytest.mark.parametrize("T", [1, 7, 40])
@pytest.mark.parametrize("group,zeros", [(32, True), (128, False)])
def test_decoding_two_blocks(T, group, zeros):
    D, F = 520, 1032
    m = model(T, D, F, torch.bfloat16, seed=T)
    packed = {i: [w4.from_weight(m["w%s%d" % (k, i)], group, zeros) for k in "gud"] for i in (1, 2)}
    for i in (1, 2):  # the reference has the rounded weights
        for k, w in zip("gud", packed[i]):
            m["w%s%d" % (k, i)] = w4.dequantize(w)
    ws = w4.make_workspace(64, D, F)  # for the largest batch

    def decode(m):
        r, xn = block_norm.forward(None, m["res"], w_pre=m["pre0"], eps=EPS)
        for i in (1, 2):
            r, xn = block_norm.forward(w4.forward(xn, *packed[i], workspace=ws), r, **options(m, i))
        return {"r": r, "out": xn}

    got, ref = decode(m), step64(m)
    check(got, {k: ref[k] for k in got}, 16)
    # A captured token step, replayed for other tokens.
    others = [model(T, D, F, torch.bfloat16, seed=s) for s in (11, 12)]
    leaves = {k: v.clone() for k, v in m.items()}
    want = []
    for o in others:
        leaves["res"].copy_(o["res"])
        want.append(decode(leaves))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        decode(leaves)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = decode(leaves)
    for _ in range(2):
        for o, w in zip(others, want):
            leaves["res"].copy_(o["res"])
            graph.replay()
            torch.cuda.synchronize()
            assert same(captured, w)
            assert same(decode(m), got)


def test_another_device_or_workspace_is_refused(monkeypatch):
    T, D, F = 4, 264, 520
    m = model(T, D, F, torch.bfloat16)
    w = [m["wg1"], m["wu1"], m["wd1"]]
    x, g = m["dout"], torch.zeros((T, F), dtype=torch.bfloat16, device="cuda")
    packed = [w4.from_weight(v) for v in w]
    tw, nw = train.make_workspace(T, D, F), block_norm.make_workspace(T, D)
    for call in (lambda: train.forward(x, *w, workspace=nw), lambda: train.backward(x, x, *w, g, g, workspace=nw),
                 lambda: w4.forward(x, *packed, workspace=nw), lambda: w4.matmul(x, packed[0], workspace=nw),
                 lambda: block_norm.backward(x, None, None, x, w_pre=m["pre0"], workspace=tw)):
        with pytest.raises(TypeError, match="workspace"):
            call()
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: train.forward(x, *w), lambda: train.backward(x, x, *w, g, g), lambda: w4.forward(x, *packed),
                 lambda: w4.matmul(x, packed[0]), lambda: w4.gate_up(x, *packed[:2]), lambda: w4.quantize(w[0]),
                 lambda: w4.dequantize(packed[0]), lambda: block_norm.forward(None, x),
                 lambda: block_norm.backward(x, None, None, x)):
        with pytest.raises(ValueError, match="current device"):
            call()
