"""Dropout on the GPU: its mask against the generator written out with Python's
integers, its values against 64-bit arithmetic.

Bounds.  x times the factor is one fp32 product, of a factor that was rounded to fp32
(2 roundings, 2^-24 of the product each), the sum with the residual one more, and the
result is rounded once: to fp32 with that sum, to bf16 by 2^-8 of its value.
"""
import pytest
import torch

from paper_2606_26344_amd import block_norm, dropout, gmlp

pytestmark = pytest.mark.gpu

M32 = 0xffffffff


def philox(counter, key):
    x, k = list(counter), list(key)
    for _ in range(10):
        a, b = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(b >> 32) ^ x[1] ^ k[0], b & M32, (a >> 32) ^ x[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return x


def kept(T, D, p, seed, offset):
    """The mask [T, D]."""
    m = round(65536 * p)
    bits = []
    for c in range(T * D // 8):
        n = (offset + c) % (1 << 64)
        for w in philox((n & M32, n >> 32, 0, 0), (seed & M32, seed >> 32)):
            bits += [w & 0xffff, w >> 16]
    return (torch.tensor(bits) >= m).view(T, D).cuda()


def data(T, D, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randn((T, D), generator=gen).to(dtype).cuda()


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def test_known_answers_of_the_reference():
    """The published test vectors of the generator."""
    assert philox((0,) * 4, (0,) * 2) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    assert philox((M32,) * 4, (M32,) * 2) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert philox((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0)) == [
        0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1]


@pytest.mark.parametrize("T,D", [(1, 8), (1, 264), (7, 520), (33, 1032)])
@pytest.mark.parametrize("p,seed,offset", [(0.1, 0, 0), (0.5, (1 << 64) - 1, (1 << 64) - 5), (0.3, 0x299f31d0a4093822, (1 << 32) - 3),
                                           (0.0, 3, 4), (1.0, 3, 4), (2.0 ** -18, 5, 6), (0.99999, 5, 6)])
def test_forward_and_backward(T, D, p, seed, offset):
    mask, m = kept(T, D, p, seed, offset), round(65536 * p)
    factor = 65536 / (65536 - m) if m < 65536 else 0.0
    x = data(T, D, torch.bfloat16, 1)
    for res in (None, torch.bfloat16, torch.float32):
        r = None if res is None else data(T, D, res, 2)
        out = dropout.forward(x, p, seed, offset, res=r)
        assert out.dtype == (res or torch.bfloat16)
        term = torch.where(mask, x.double() * factor, 0.0)
        ref = term + (0.0 if r is None else r.double())
        half = 2.0 ** -24 if res is torch.float32 else 2.0 ** -8 + 2.0 ** -24
        assert ((out.double() - ref).abs() <= 1.001 * (half * ref.abs() + 2 * 2.0 ** -24 * term.abs())).all()
    for kind in (torch.bfloat16, torch.float32):
        dout = data(T, D, kind, 3)
        dx = dropout.backward(dout, p, seed, offset)
        ref = torch.where(mask, dout.double() * factor, 0.0)
        assert dx.dtype is torch.bfloat16
        assert ((dx.double() - ref).abs() <= 1.001 * (2.0 ** -8 + 2 * 2.0 ** -24) * ref.abs()).all()


def test_dropped_values_do_not_count():
    T, D = 16, 264
    x, r = data(T, D, torch.bfloat16, 1), data(T, D, torch.float32, 2)
    mask = kept(T, D, 0.5, 7, 0)
    want = dropout.forward(x, 0.5, 7, res=r)
    x[~mask] = float("nan")
    assert torch.equal(dropout.forward(x, 0.5, 7, res=r), want)
    x[~mask] = float("-inf")
    assert torch.equal(dropout.forward(x, 0.5, 7, res=r), want) and torch.equal(want[~mask], r[~mask])
    assert (dropout.forward(torch.full_like(x, float("nan")), 1.0, 7, res=r) == r).all()
    x[mask] = float("nan")
    assert torch.equal(dropout.forward(x, 0.5, 7).isnan(), mask)


def test_in_place():
    T, D = 33, 520
    x, r, rb = data(T, D, torch.bfloat16, 1), data(T, D, torch.float32, 2), data(T, D, torch.bfloat16, 3)
    want = [dropout.forward(x, 0.2, 5, 9, res=v) for v in (r, rb, None)]
    assert torch.equal(dropout.forward(x, 0.2, 5, 9, res=rb, out=x.clone()), want[1])
    assert dropout.forward(x, 0.2, 5, 9, res=r, out=r) is r and torch.equal(r, want[0])
    assert dropout.forward(x, 0.2, 5, 9, res=rb, out=rb) is rb and torch.equal(rb, want[1])
    dx = dropout.backward(x, 0.2, 5, 9)
    assert torch.equal(dx, want[2])
    assert dropout.backward(x, 0.2, 5, 9, dx=x) is x and torch.equal(x, dx)
    y = data(T, D, torch.bfloat16, 1)
    assert dropout.forward(y, 0.2, 5, 9, res=data(T, D, torch.bfloat16, 3), out=y) is y and torch.equal(y, want[1])


def test_rate_over_many_elements():
    """Of n elements n p' are dropped, within six deviations; neighbours independently."""
    T, D, p = 2048, 4096, 0.1
    y = dropout.forward(torch.ones((T, D), dtype=torch.bfloat16, device="cuda"), p, 1234) == 0
    q, n = round(65536 * p) / 65536, T * D
    for t, mean in ((y, q), (y[:, 1:] & y[:, :-1], q * q), (y[1:] & y[:-1], q * q)):
        m = t.numel()
        # Pairs share elements: their sum's variance is at most three times that of independent ones.
        assert abs(t.sum().item() - m * mean) <= 6 * (3 * m * mean) ** 0.5
    assert not torch.equal(y, dropout.forward(torch.ones((T, D), dtype=torch.bfloat16, device="cuda"), p, 1235) == 0)


def test_calls_continue_each_other():
    """A tensor in parts, each with the offset behind the last, has the mask of the whole."""
    T, D = 96, 264
    x = data(T, D, torch.bfloat16, 1)
    whole = dropout.forward(x, 0.3, 11, 100)
    at = 100
    for lo, hi in ((0, 1), (1, 40), (40, 96)):
        assert torch.equal(dropout.forward(x[lo:hi], 0.3, 11, at), whole[lo:hi])
        at += dropout.counters(hi - lo, D)
    position = torch.tensor([60], device="cuda")
    assert torch.equal(dropout.forward(x, 0.3, 11, 40, position=position), whole)


def test_elements_past_32_bits():
    """The counters and addresses of a tensor of more than 2^32 elements."""
    T, D = (1 << 10) + 1, 1 << 22
    x = torch.ones((T, D), dtype=torch.bfloat16, device="cuda")
    y = dropout.forward(x, 0.5, 3, 8)
    assert torch.equal(y[-1:, -512:], dropout.forward(x[:1, :512].contiguous(), 0.5, 3, 8 + dropout.counters(T, D) - 64))
    assert torch.equal(y[-2:], dropout.forward(x[:2], 0.5, 3, 8 + dropout.counters(T - 2, D)))


def test_replays_move_on():
    """A captured call with a position in device memory, moved on by the graph itself."""
    T, D = 40, 520
    x, r = data(T, D, torch.bfloat16, 1), data(T, D, torch.float32, 2)
    position = torch.zeros(1, dtype=torch.int64, device="cuda")
    out, dx = torch.empty_like(r), torch.empty_like(x)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        dropout.forward(x, 0.4, 21, 3, res=r, position=position, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        dropout.forward(x, 0.4, 21, 3, res=r, position=position, out=out)
        dropout.backward(r, 0.4, 21, 3, position=position, dx=dx)
        position.add_(dropout.counters(T, D))
    for i in range(4):
        graph.replay()
        at = 3 + i * dropout.counters(T, D)
        want = dropout.forward(x, 0.4, 21, at, res=r), dropout.backward(r, 0.4, 21, at)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(dx, want[1])


def test_between_a_block_and_the_next_norm():
    """With the norms between blocks: the gradients of a step with dropout on y."""
    T, D = 24, 264
    y, res, dxn = data(T, D, torch.bfloat16, 1), data(T, D, torch.float32, 2), data(T, D, torch.bfloat16, 3)
    dropped = dropout.forward(y, 0.25, 17, 5)
    r, xn = block_norm.forward(dropped, res)
    dd, dres, _, _, _ = block_norm.backward(dxn, None, dropped, r)
    dy = dropout.backward(dd, 0.25, 17, 5)
    mask = kept(T, D, 0.25, 17, 5)
    yd, rd = y.double().requires_grad_(), res.double().requires_grad_()
    rr = rd + torch.where(mask, yd / 0.75, 0.0)
    (rr / (rr.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()).backward(dxn.double())
    # Roundings to bf16 on the way: dropped, and dd and dy.  Each moves a gradient by at
    # most 2^-8 of its norm, dropped through the norm's slope twice.
    for got, want in ((dy, yd.grad), (dres, rd.grad)):
        assert (got.double() - want).norm() <= 4 * 2.0 ** -8 * want.norm()
    assert torch.equal(dy == 0, ~mask | (dd == 0))


def test_refusals():
    x, r = data(4, 264, torch.bfloat16, 1), data(4, 264, torch.float32, 2)
    for bad in (lambda: dropout.forward(r, 0.1, 1), lambda: dropout.forward(x, 0.1, 1, res=r.half()), lambda: dropout.backward(x.half(), 0.1, 1)):
        with pytest.raises(TypeError):
            bad()
    for bad in (lambda: dropout.forward(x, 0.1, -1), lambda: dropout.forward(x, 0.1, 1, 1 << 64), lambda: dropout.forward(x[0], 0.1, 1),
                lambda: dropout.forward(x.t(), 0.1, 1), lambda: dropout.forward(x.cpu(), 0.1, 1), lambda: dropout.forward(x, 0.1, 1, res=r[:2]),
                lambda: dropout.forward(x, 0.1, 1, res=r, out=x), lambda: dropout.forward(x, 0.1, 1, position=torch.zeros(1, device="cuda")),
                lambda: dropout.forward(x, 0.1, 1, position=torch.zeros(1, dtype=torch.int64)),
                lambda: dropout.backward(r, 0.1, 1, dx=r)):
        with pytest.raises((ValueError, TypeError)):
            bad()
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(gmlp.GmlpError):
            dropout.forward(x, p, 1)
