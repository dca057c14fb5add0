"""A block whose MLP is sparse, as a model runs it: norm, sort by expert, dispatch, the
experts' Gated MLPs, combine, dropout into the residual stream, norm; forward and
backward, captured, on two streams, and as a decoding step.

Bounds.  A rounding to bf16 moves each element by at most 2^-8 of its value, hence a
tensor by at most 2^-8 of its L2 norm; on its way to a result such a displacement goes
through products and norms whose gain for a random direction is about that of the tensor
itself, twice that where gate and up are multiplied.  A result depends on at most xn, g,
u, h, ys, y, the dropped y and the last xn (8, counted twice) and dr's dy, dys, dg, du, dxs,
dx, dxn and its own (8): 24 2^-8 = 0.09 of its norm if all of them pointed one way.  A
path, weight or factor left out is an error of the order of 1.
"""
import pytest
import torch

from paper_2606_26344_amd import block_norm, dropout, experts, gmlp, route

pytestmark = pytest.mark.gpu

EPS, P, SEED = 1e-6, 0.25, 99


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def model(T, k, E, D, F, seed=0, padding=0):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *shape, s=1.0, at=0.0: (torch.randn(shape, generator=gen) * s + at).to(torch.bfloat16).cuda()  # noqa: E731
    m = dict(res=n(T, D).float(), dout=n(T, D), pre=n(D, s=0.1, at=1.0), last=n(D, s=0.1, at=1.0),
             wg=n(E, D, F, s=D ** -0.5), wu=n(E, D, F, s=D ** -0.5), wd=n(E, F, D, s=F ** -0.5))
    top = torch.randn((T, E), generator=gen).topk(k, dim=1)
    ids, w = top.indices.clone(), top.values.softmax(1)
    if padding:
        ids[-padding:] = -1
    m.update(ids=ids.cuda(), weights=w.cuda())
    return m


class Buffers:
    """What a program keeps: rows behind the last expert's stay as they are (zeros)."""

    def __init__(self, m):
        T, k = m["ids"].shape
        E, D, F = m["wg"].shape
        rows = lambda cols: torch.zeros((T * k, cols), dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.xs, self.ys, self.dys, self.dxs = rows(D), rows(D), rows(D), rows(D)
        self.g, self.u = rows(F), rows(F)
        self.workspace = experts.make_workspace(T * k, E, D, F)
        self.norms = block_norm.make_workspace(T, D)


def step(m, b=None, stream=None, position=None):
    """Every result by name."""
    E = m["wg"].shape[0]
    w = (m["wg"], m["wu"], m["wd"])
    kw = dict(stream=stream)
    ws = dict(workspace=b.workspace if b else None, **kw)
    nws = b.norms if b else None
    take = (lambda name: getattr(b, name)) if b else (lambda name: None)
    r0, xn = block_norm.forward(None, m["res"], w_pre=m["pre"], eps=EPS, **kw)
    offsets, slots = route.sort(m["ids"], E, **kw)
    xs = route.dispatch(xn, slots, out=take("xs"), **kw)
    ys, g, u = experts.train_forward(xs, offsets, *w, out=take("ys"), g=take("g"), u=take("u"), **ws)
    y = route.combine(ys, slots, m["weights"], **kw)
    r1 = dropout.forward(y, P, SEED, 7, res=r0, position=position, **kw)
    r, out = block_norm.forward(None, r1, w_pre=m["last"], eps=EPS, **kw)
    got = {"y": y, "r": r, "out": out}
    _, dr1, got["last"], _, _ = block_norm.backward(m["dout"], None, None, r, w_pre=m["last"], eps=EPS, workspace=nws, **kw)
    dy = dropout.backward(dr1, P, SEED, 7, position=position, **kw)
    dys, got["weights"] = route.combine_backward(dy, ys, slots, m["weights"], dys=take("dys"), **kw)
    dxs, got["wg"], got["wu"], got["wd"] = experts.backward(dys, xs, offsets, *w, g, u, dxs=take("dxs"), **ws)
    dxn = route.dispatch_backward(dxs, slots, **kw)
    _, got["res"], got["pre"], _, _ = block_norm.backward(dxn, dr1, None, r0, w_pre=m["pre"], eps=EPS, workspace=nws, **kw)
    return got


def mask_of(m, position=0):
    T, D = m["res"].shape
    ones = torch.ones((T, D), dtype=torch.bfloat16, device="cuda")
    return dropout.forward(ones, P, SEED, 7 + position) != 0


def step64(m):
    names = ("res", "pre", "last", "wg", "wu", "wd", "weights")
    p = {k: m[k].double().requires_grad_() for k in names}
    norm = lambda v, w: v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w  # noqa: E731
    xn = norm(p["res"], p["pre"])
    y = torch.zeros_like(xn)
    for e in range(m["wg"].shape[0]):
        token, j = torch.nonzero(m["ids"] == e, as_tuple=True)
        x = xn[token]
        ye = (torch.nn.functional.silu(x @ p["wg"][e]) * (x @ p["wu"][e])) @ p["wd"][e]
        y = y.index_add(0, token, p["weights"][token, j, None] * ye)
    r = p["res"] + torch.where(mask_of(m), y / (1 - P), 0.0)
    out = norm(r, p["last"])
    out.backward(m["dout"].double())
    got = {k: v.grad for k, v in p.items()}
    got.update(y=y.detach(), r=r.detach(), out=out.detach())
    return got


def check(got, want):
    assert set(got) == set(want)
    for name in want:
        off = ((got[name].double() - want[name]).norm() / want[name].norm().clamp(min=1e-30)).item()
        print("%s: %.5f of its norm" % (name, off), flush=True)
        assert got[name].shape == want[name].shape and off <= 24 * 2.0 ** -8, name


@pytest.mark.parametrize("T,k,E,D,F,padding", [(1, 1, 1, 72, 136, 0), (1, 2, 8, 264, 520, 0), (7, 8, 16, 264, 136, 3),
                                               (100, 2, 5, 520, 264, 25), (300, 4, 70, 264, 520, 0), (700, 2, 3, 264, 1032, 70)])
def test_training_step(T, k, E, D, F, padding):
    m = model(T, k, E, D, F, T, padding)
    got = step(m, Buffers(m))
    check(got, step64(m))
    assert (got["weights"][T - padding:] == 0).all() and (got["y"][T - padding:] == 0).all()
    # Without buffers and workspaces of its own the same bits.
    again = step(m)
    assert all(torch.equal(again[n], got[n]) for n in got)


def test_a_batch_of_padding_only():
    m = model(5, 2, 3, 264, 520, 1, padding=5)
    got = step(m, Buffers(m))
    assert (got["y"] == 0).all() and all((got[n] == 0).all() for n in ("wg", "wu", "wd", "weights"))
    assert torch.equal(got["r"], m["res"])


def same(a, b):
    assert set(a) == set(b)
    return all(torch.equal(a[k], b[k]) for k in a)


def test_captured_step_replays():
    """Replayed with other inputs, routings and masks between eager steps of the same leaves."""
    shape = (130, 2, 6, 264, 520)
    models = [model(*shape, seed=s, padding=p) for s, p in ((1, 0), (2, 30), (3, 129))]
    leaves = {k: v.clone() for k, v in models[0].items()}
    b, own = Buffers(leaves), Buffers(leaves)
    position = torch.zeros(1, dtype=torch.int64, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(leaves, b, position=position)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = step(leaves, b, position=position)
    for i, at in ((0, 0), (1, 1000), (2, 5), (0, 77), (1, 0)):
        for k, v in leaves.items():
            v.copy_(models[i][k])
        position.fill_(at)
        graph.replay()
        want = step(models[i], own, position=position)
        torch.cuda.synchronize()
        # Rows of dxs and the like behind the last expert's differ by what was there: not in these.
        assert same(captured, want), i


class Handle:
    """A stream object that is only its handle."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.parametrize("buffers", [False, True])
def test_two_steps_at_once(buffers):
    models = [model(130, 2, 6, 264, 520, seed=s) for s in (4, 5)]
    want = [step(m) for m in models]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    kept = [Buffers(m) if buffers else None for m in models]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for m, st, b in zip(models, streams, kept):
            got.append(step(m, b, stream=Handle(st)))
            junk = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(4)]
            del junk
        torch.cuda.synchronize()
        assert all(same(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("T", [1, 5, 64])
def test_decoding(T):
    """A token step captured once, with the workspace of the largest batch."""
    k, E, D, F = 2, 8, 520, 264
    ws = experts.make_workspace(64 * k, E, D, F)

    def decode(m):
        r, xn = block_norm.forward(None, m["res"], w_pre=m["pre"], eps=EPS)
        offsets, slots = route.sort(m["ids"], E)
        ys = experts.forward(route.dispatch(xn, slots), offsets, m["wg"], m["wu"], m["wd"], workspace=ws)
        return route.combine(ys, slots, m["weights"])

    models = [model(T, k, E, D, F, seed=s) for s in range(3)]
    for m in models[1:]:
        m.update({n: models[0][n] for n in ("wg", "wu", "wd", "pre")})
    want = [decode(m) for m in models]
    for m, y in zip(models, want):
        ref = step64(m)["y"]
        assert (y.double() - ref).norm() <= 24 * 2.0 ** -8 * ref.norm()
    leaves = {n: v.clone() for n, v in models[0].items()}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        decode(leaves)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        captured = decode(leaves)
    for _ in range(2):
        for m, y in zip(models, want):
            for n in ("res", "ids", "weights"):
                leaves[n].copy_(m[n])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(captured, y)


def test_another_device_is_refused(monkeypatch):
    m = model(4, 2, 3, 264, 520)
    offsets, slots = route.sort(m["ids"], 3)
    x = m["dout"]
    xs = route.dispatch(x, slots)
    w = (m["wg"], m["wu"], m["wd"])
    g = torch.zeros((8, 520), dtype=torch.bfloat16, device="cuda")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: route.sort(m["ids"], 3), lambda: route.dispatch(x, slots), lambda: route.combine(xs, slots),
                 lambda: route.combine_backward(x, xs, slots, m["weights"]), lambda: experts.forward(xs, offsets, *w),
                 lambda: experts.backward(xs, xs, offsets, *w, g, g), lambda: dropout.forward(x, 0.1, 1),
                 lambda: dropout.backward(x, 0.1, 1)):
        with pytest.raises(ValueError, match="current device"):
            call()
