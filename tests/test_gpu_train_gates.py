"""act and act' of single gates through the backward pass, against 64-bit formulas.

One token x = (1, 0, ..) with dY = (1, 0, ..), Wd[:, 0] = 1 and U = 1 makes dH = 1, and
the first rows of dWg and dWu and the first column of dWd are bf16(act'(g)), bf16(act(g))
and bf16(act(g)): sums with one term that is not zero.

Bounds.  One rounding to bf16, 2^-8 of the value.  The sigmoid s = 1 / (1 + e), e = exp(-b g)
as 2^x: the rounding of x = -b g log2(e) moves e by at most |b g| 2^-24 < 2^-17 of it for
|b g| <= 104, where e is neither 0 nor infinite, and 2^x, the reciprocal and the handful of
products and sums add 2^-20.  So s, s (1 - s) and b g s (1 - s) are within 2^-16 of their
sizes ("terms"), unless they fall below the smallest normal fp32 number, 2^-126, where
they may be zero: 2^-125 for each factor 1, g or b g in front.
"""
import pytest
import torch

from paper_2606_26344_amd import gmlp, train

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def slopes(gates, activation, beta):
    """(dwg[0], dwu[0], dwd[:, 0]) of the step above, and the same in 64 bits with their terms."""
    g = gates.to(torch.bfloat16)
    F, D = g.numel(), 8
    assert F % 8 == 0
    one = torch.zeros((1, D), dtype=torch.bfloat16)
    one[0, 0] = 1
    w = torch.zeros((D, F), dtype=torch.bfloat16).cuda()
    wd = torch.zeros((F, D), dtype=torch.bfloat16)
    wd[:, 0] = 1
    x, wd, g = one.cuda(), wd.cuda(), g.view(1, F).cuda()
    _, dwg, dwu, dwd = train.backward(x, x, w, w, wd, g, torch.ones_like(g), activation=activation, beta=beta)
    got = [t.cpu().double() for t in (dwg[0], dwu[0], dwd[:, 0])]
    v, b = g[0].cpu().double(), beta if activation == "swish" else 1.0
    s, c = torch.sigmoid(b * v), torch.sigmoid(b * v) * torch.sigmoid(-b * v)
    if activation == "sigmoid":
        return v, got, (c, s, s), (c, s, s), torch.ones_like(v)
    return v, got, (s + b * v * c, v * s, v * s), (s + (b * v * c).abs(), (v * s).abs(), (v * s).abs()), 1 + v.abs() + (b * v).abs()


def check(gates, activation, beta):
    v, got, refs, terms, factors = slopes(gates, activation, beta)
    for name, a, r, t in zip(("act'", "act (dU)", "act (H)"), got, refs, terms):
        bound = 2.0 ** -8 * r.abs() + 2.0 ** -16 * t + 2.0 ** -125 * factors
        ratio = (a - r).abs() / bound
        i = ratio.nan_to_num(nan=float("inf")).argmax()
        print("%s of %s, beta %g: max |err|/bound = %.3f at g = %g" % (name, activation, beta, ratio[i], v[i]), flush=True)
        assert (ratio <= 1).all(), (name, v[i].item(), a[i].item(), r[i].item())


VARIANTS = [("silu", 1.0), ("sigmoid", 1.0), ("swish", 1.702), ("swish", -0.5), ("swish", 0.0)]


@pytest.mark.parametrize("activation,beta", VARIANTS)
def test_gates_to_saturation(activation, beta):
    """Both sides alike: a gate that is nearly open has the slope of one that is nearly shut."""
    check(torch.arange(-100, 100, 0.03125), activation, beta)


def test_sigmoid_slope_is_even():
    v, got, *_ = slopes(torch.tensor([8.0, 12.0, 16.0, 20.0, -8.0, -12.0, -16.0, -20.0]), "sigmoid", 1.0)
    assert (got[0][:4] > 0).all()
    assert ((got[0][:4] - got[0][4:]).abs() <= 2.0 ** -7 * got[0][4:]).all()  # two roundings and what is before them


@pytest.mark.parametrize("activation,beta", VARIANTS + [("swish", 4.0), ("swish", -1e3), ("swish", 3e38)])
def test_largest_and_smallest_gates(activation, beta):
    """Every power of two of bf16: b g may pass the range of fp32, the slope stays 0 or 1."""
    p = 2.0 ** torch.arange(-124, 128, dtype=torch.float64)
    large = torch.finfo(torch.bfloat16).max
    check(torch.cat([p, -p, torch.tensor([large, -large, 0.0, -0.0, 1.0, -1.0, 3.0, -3.0], dtype=torch.float64)]), activation, beta)
