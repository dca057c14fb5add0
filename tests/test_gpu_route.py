"""Tokens sorted by expert and back on the GPU, against plain 64-bit formulas.

The sort is exact.  Dispatch moves bits.  Combine adds k products in fp32: each of them
and each sum is off by at most 2^-24 of the sum S of the terms' absolute values, 2 k
roundings, and the result is rounded once to bf16 (2^-8 of its value).  The rows'
gradients are one fp32 product, rounded once: 2^-8 + 2^-23 of the value.  The weights'
are sums of D products in fp32, 2 D roundings of at most 2^-24 S (a fused one counts
once), and rounded once to their type.
"""
import pytest
import torch

from paper_2606_26344_amd import gmlp, route

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def reference_sort(ids, E):
    flat = ids.cpu().long().reshape(-1)
    key = torch.where((flat < 0) | (flat >= E), E, flat)
    order = key.sort(stable=True).indices
    slots = torch.empty_like(flat)
    slots[order] = torch.arange(flat.numel())
    slots[key == E] = -1
    offsets = torch.zeros(E + 1, dtype=torch.long)
    offsets[1:] = torch.bincount(key, minlength=E + 1)[:E].cumsum(0)
    return offsets.int(), slots.view(ids.shape).int()


def random_ids(T, k, E, seed, kind="some", dtype=torch.int32):
    gen = torch.Generator().manual_seed(seed)
    if kind == "one":  # all to one expert
        ids = torch.full((T, k), E - 1)
    elif kind == "none":
        ids = torch.full((T, k), -1)
    else:
        ids = torch.randint(0, E, (T, k), generator=gen)
        if kind == "some":  # a fifth without an expert, in every way there is
            out = torch.tensor([-1, E, E + 1, -2 ** 31, 2 ** 31 - 1])
            hole = torch.rand((T, k), generator=gen) < 0.2
            ids = torch.where(hole, out[torch.randint(0, 5, (T, k), generator=gen)], ids)
    return ids.to(dtype).cuda()


@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 2, 8), (1, 64, 1024), (33, 8, 64), (63, 1, 2), (64, 1, 3), (65, 1, 256),
                                   (500, 4, 60), (1024, 2, 8), (1025, 2, 9), (2049, 7, 1000), (4096, 8, 256),
                                   (30011, 3, 17), (32768, 1, 64), (32769, 1, 1024),
                                   (70001, 8, 128), (70001, 3, 1), (33333, 2, 1000), (1048579, 8, 5)])
@pytest.mark.parametrize("kind", ["all", "some", "one", "none"])
def test_sort(T, k, E, kind):
    print("sort", T, k, E, kind, flush=True)
    want = None
    for dtype in (torch.int32, torch.int64):
        ids = random_ids(T, k, E, T + k, kind, dtype)
        want = want or reference_sort(ids, E)
        got = route.sort(ids, E)
        assert all(torch.equal(g.cpu(), w) for g, w in zip(got, want))


def test_sort_takes_64_bit_ids_whole():
    ids = torch.tensor([[1 << 32, (1 << 32) + 1, 1, -(1 << 32)]], device="cuda")
    offsets, slots = route.sort(ids, 2)
    assert offsets.tolist() == [0, 0, 1] and slots.tolist() == [[-1, -1, 0, -1]]


def test_sort_of_nothing():
    offsets, slots = route.sort(torch.zeros((0, 2), dtype=torch.int64, device="cuda"), 5)
    assert offsets.tolist() == [0] * 6 and slots.shape == (0, 2)


def rows(n, D, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn((n, D), generator=gen) * scale).to(torch.bfloat16).cuda()


def weights_of(T, k, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.rand((T, k), generator=gen).to(dtype).cuda()


SHAPES = [(1, 1, 1, 8), (1, 2, 8, 4096), (3, 8, 64, 264), (33, 8, 64, 2056), (5, 3, 4, 8), (40, 13, 16, 520), (300, 4, 16, 5120),
          (7, 64, 100, 136), (1000, 2, 8, 1032), (2500, 6, 32, 776)]


@pytest.mark.parametrize("T,k,E,D", SHAPES)
@pytest.mark.parametrize("kind", ["all", "some", "none"])
def test_dispatch(T, k, E, D, kind):
    offsets, slots = route.sort(random_ids(T, k, E, T, kind), E)
    x = rows(T, D, 1)
    x.view(torch.int16)[0, 0] = -1  # a NaN's bits
    xs = torch.full((T * k, D), 7.0, dtype=torch.bfloat16, device="cuda")
    assert route.dispatch(x, slots, out=xs) is xs
    want = torch.full_like(xs, 7.0)
    flat = slots.reshape(-1).long()
    live = flat >= 0
    want[flat[live]] = x.repeat_interleave(k, 0)[live]
    assert int(offsets[-1]) == int(live.sum())
    assert torch.equal(xs.view(torch.int16), want.view(torch.int16))  # rows behind the last are left as they were


@pytest.mark.parametrize("T,k,E,D", SHAPES)
@pytest.mark.parametrize("weights", [None, torch.float32, torch.bfloat16])
def test_combine_and_gradients(T, k, E, D, weights):
    print("combine", T, k, E, D, weights, flush=True)
    offsets, slots = route.sort(random_ids(T, k, E, T + 1), E)
    n = int(offsets[-1])
    ys = rows(T * k, D, 2)
    ys[n:] = float("nan")  # not read
    live = slots >= 0
    at = slots.clamp(min=0).long()
    taken = torch.where(live[..., None], ys[at].double(), 0.0)
    w = None if weights is None else weights_of(T, k, weights, 3)
    if w is not None:
        w[~live] = float("nan")  # nothing of a weight without a row
    wd = torch.ones((T, k), dtype=torch.float64, device="cuda") if w is None else torch.where(live, w.double(), 0.0)
    y = route.combine(ys, slots, w).double()
    ref, terms = (wd[..., None] * taken).sum(1), (wd[..., None] * taken).abs().sum(1)
    assert ((y - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.02 * k * 2.0 ** -24 * terms).all()
    if w is None:
        assert torch.equal(route.dispatch_backward(ys, slots).double(), y)
        return
    dy = rows(T, D, 4)
    dead = ~live.any(1)
    dy[dead] = float("inf")  # nor of a token without one
    dys = torch.full((T * k, D), 3.0, dtype=torch.bfloat16, device="cuda")
    _, dw = route.combine_backward(dy, ys, slots, w, dys=dys)
    assert dw.dtype == weights and (dys[n:] == 3.0).all()
    dyd = torch.where(dead[:, None], 0.0, dy.double())
    want = (wd[..., None] * dyd[:, None])[live]
    assert ((dys[at[live]].double() - want).abs() <= (2.0 ** -8 + 2.0 ** -23) * want.abs()).all()
    ref, terms = (dyd[:, None] * taken).sum(2), (dyd[:, None] * taken).abs().sum(2)
    half = 2.0 ** -8 if weights is torch.bfloat16 else 2.0 ** -24
    assert ((dw.double() - ref).abs() <= half * ref.abs() + 2.02 * D * 2.0 ** -24 * terms).all()
    assert (dw[~live] == 0).all()
    # One of them at a time gives the same, and dys may be ys.
    only, none = route.combine_backward(dy, ys, slots, w, want=("dys",))
    assert none is None and torch.equal(only[:n], dys[:n])
    none, only = route.combine_backward(dy, ys, slots, w, want=("dweights",))
    assert none is None and torch.equal(only, dw)
    _, again = route.combine_backward(dy, ys, slots, w, dys=ys)
    assert torch.equal(again, dw) and torch.equal(ys[:n], dys[:n])


def test_gradients_against_differences():
    """<dy, combine(ys + h d, w + h e)> moves by h (<dys, d> + <dw, e>): combine is
    linear in each, so central differences are exact but for its roundings, at most
    2^-8 |y| each, of both sides."""
    T, k, E, D = 40, 4, 8, 264
    _, slots = route.sort(random_ids(T, k, E, 9), E)
    ys, dy, w = rows(T * k, D, 1), rows(T, D, 2), weights_of(T, k, torch.float32, 3)
    dys, dw = route.combine_backward(dy, ys, slots, w)
    n = int((slots >= 0).sum())
    e = weights_of(T, k, torch.float32, 4)
    d = rows(T * k, D, 5)
    up, down = route.combine(ys, slots, w + e), route.combine(ys, slots, w - e)
    off = ((up.double().abs() + down.double().abs()) * dy.double().abs()).sum() * 2.0 ** -8
    slope = ((up.double() - down.double()) * dy.double()).sum() / 2
    assert abs(slope - (dw.double() * e.double()).sum()) <= off
    # In a row's direction: combine of d alone.
    moved = (route.combine(d, slots, w).double() * dy.double())
    off = (moved.abs() * 2.0 ** -8).sum() + ((dys[:n].double() * d[:n].double()).abs() * 2.0 ** -8).sum()
    assert abs(moved.sum() - (dys[:n].double() * d[:n].double()).sum()) <= off


def test_slots_out_of_range_are_none():
    T, k, D = 6, 2, 264
    slots = torch.tensor([[0, 12], [1, -5], [2 ** 31 - 1, 2], [3, -2 ** 31], [11, 4], [5, 6]], dtype=torch.int32, device="cuda")
    x, ys, dy, w = rows(T, D, 1), rows(T * k, D, 2), rows(T, D, 3), weights_of(T, k, torch.float32, 4)
    fixed = torch.where((slots >= 0) & (slots < 12), slots, -1)
    a, b = (torch.zeros((T * k, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    assert torch.equal(route.dispatch(x, slots, out=a), route.dispatch(x, fixed, out=b))
    assert torch.equal(route.combine(ys, slots, w), route.combine(ys, fixed, w))
    c, d = torch.zeros_like(a), torch.zeros_like(a)
    got, want = route.combine_backward(dy, ys, slots, w, dys=c), route.combine_backward(dy, ys, fixed, w, dys=d)
    assert all(torch.equal(g, r) for g, r in zip(got, want))


def test_rows_past_32_bits():
    """Rows that begin more than 2^32 bytes into a tensor."""
    T, k, D = 600, 1, 1 << 22
    slots = (T - 1 - torch.arange(T, dtype=torch.int32, device="cuda")).view(T, 1)
    x = torch.empty((T, D), dtype=torch.bfloat16, device="cuda")
    x[:] = torch.arange(T, device="cuda")[:, None] % 251
    x[:, -1] = 300.0
    xs = route.dispatch(x, slots)
    assert torch.equal(xs, x.flip(0))
    assert torch.equal(route.combine(xs, slots), x)
    dy = torch.zeros_like(x)
    dy[:, -8:] = 1.0
    dys, dw = route.combine_backward(dy, xs, slots, torch.ones((T, 1), device="cuda"))
    assert torch.equal(dys, dy)  # every row the same
    assert torch.equal(dw[:, 0], 7.0 * (torch.arange(T, device="cuda") % 251) + 300.0)


def test_refusals():
    T, k, D = 4, 2, 264
    ids = random_ids(T, k, 8, 1)
    offsets, slots = route.sort(ids, 8)
    x, ys, w = rows(T, D, 1), rows(T * k, D, 2), weights_of(T, k, torch.float32, 1)
    for bad in (lambda: route.sort(ids.float(), 8), lambda: route.dispatch(x, slots.long()),
                lambda: route.combine(ys.float(), slots), lambda: route.combine(ys, slots, w.half()),
                lambda: route.combine_backward(x, ys, slots, w, dweights=torch.empty_like(w, dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: route.sort(ids.t(), 8), lambda: route.sort(ids.cpu(), 8), lambda: route.sort(ids, 8, offsets=offsets[:-1]),
                lambda: route.dispatch(x[:-1], slots), lambda: route.dispatch(x[:, ::2], slots),
                lambda: route.dispatch(x, slots, out=x), lambda: route.combine(ys[:-1], slots),
                lambda: route.combine(ys, slots, w.t().contiguous()), lambda: route.combine_backward(x, ys, slots, w, want=("dx",)),
                lambda: route.combine_backward(x, ys, slots, w, dys=ys.clone(), want=("dweights",))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: route.sort(ids, 0), lambda: route.sort(ids, 1025), lambda: route.dispatch(rows(T, 260, 1), slots)):
        with pytest.raises(gmlp.GmlpError):
            bad()
