"""The backward pass of experts whose weights and rows begin 2^32 bytes and more into a
tensor, against the formulas.  The bounds are those of tests/test_gpu_experts.py: sums of
D = 8192 products, and for dX of 2 F = 65536, formed 32 at a time, carry at most 2049
roundings of 2^-24 of their terms, less than the 2^-12 that stand for them there.
"""
import pytest
import torch

from paper_2606_26344_amd import experts, gmlp

from test_gpu_experts import MARK, act, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


@pytest.mark.parametrize("n", [40, 300])
def test_gradients_past_32_bits(n):
    E, D, F, N = 9, 8192, 32768, 70000
    assert (E - 1) * D * F * 2 >= 1 << 32 and (N - n) * F * 2 > 1 << 32
    gen = torch.Generator(device="cuda").manual_seed(n)
    r = lambda *shape, s=1.0: (torch.randn(shape, generator=gen, device="cuda") * s).to(torch.bfloat16)  # noqa: E731
    # Expert 0 has five rows, the last one n, the others none: their weights are not read.
    w = [torch.full(s, float("nan"), dtype=torch.bfloat16, device="cuda") for s in ((E, D, F), (E, D, F), (E, F, D))]
    for v in w:
        for e in (0, E - 1):
            v[e] = r(*v.shape[1:], s=v.shape[1] ** -0.5)

    def rows(cols):
        t = torch.full((N, cols), float("nan"), dtype=torch.bfloat16, device="cuda")
        t[N - n - 5:] = r(n + 5, cols)
        return t

    xs, dys, g, u = rows(D), rows(D), rows(F), rows(F)
    offsets = torch.full((E + 1,), N - n, dtype=torch.int32, device="cuda")
    offsets[0], offsets[-1] = N - n - 5, N
    dxs = torch.full((N, D), MARK, dtype=torch.bfloat16, device="cuda")
    _, *dw = experts.backward(dys, xs, offsets, *w, g, u, dxs=dxs)
    assert (dxs[:N - n - 5] == MARK).all()
    for e, at in ((0, slice(N - n - 5, N - n)), (E - 1, slice(N - n, N))):
        x, dy, gd, ud = (v[at].double() for v in (xs, dys, g, u))
        wg, wu, wd = (v[e].double() for v in w)
        dh, terms = dy @ wd.T.contiguous(), dy.abs() @ wd.abs().T.contiguous()
        a, da = act(gd, "silu", 1.0)
        dg, du, h = dh * ud * da, dh * a, a * ud
        dgt, dut = dg.abs() + 2.0 ** -4 * (terms * ud * da).abs(), du.abs() + 2.0 ** -4 * (terms * a).abs()
        for name, got, ref, of in (("dxs", dxs[at], dg @ wg.T + du @ wu.T, dgt @ wg.abs().T + dut @ wu.abs().T),
                                   ("dwg", dw[0][e], x.T @ dg, x.abs().T @ dgt), ("dwu", dw[1][e], x.T @ du, x.abs().T @ dut),
                                   ("dwd", dw[2][e], h.T @ dy, h.abs().T @ dy.abs())):
            print(e, name, check((e, name), got, ref, of), flush=True)
    assert all((v[1:-1] == 0).all() for v in dw)
