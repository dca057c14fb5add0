"""Weight gradients whose tiles are more than one launch takes, against the formulas: 1024
experts of 8 x 2^20 (25 million blocks, 17 GB a tensor), some of them with rows.  The bounds
are those of tests/test_gpu_experts.py, with sums of at most 8 products before dG, dU and H
and of an expert's few rows after them.
"""
import pytest
import torch

from paper_2606_26344_amd import experts, gmlp

from test_gpu_experts import act, check, offsets_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


@pytest.mark.parametrize("D,F", [(8, 1 << 20), (1 << 20, 8)])
def test_more_tiles_than_a_launch_has_blocks(D, F):
    E = 1024
    rows = {0: 5, 1: 1, 340: 3, 682: 2, 683: 4, 1000: 7, 1023: 6}
    counts = [rows.get(e, 0) for e in range(E)]
    N = sum(counts)
    launches = [k for k in experts.describe(N, E, D, F, True) if "(GroupedOp)5" in k[0]]
    assert len(launches) == 2
    gen = torch.Generator(device="cuda").manual_seed(D)
    n = lambda *shape, s=1.0: (torch.randn(shape, generator=gen, device="cuda") * s).to(torch.bfloat16)  # noqa: E731
    wg, wu, wd = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((E, D, F), (E, D, F), (E, F, D)))
    for e in rows:
        wd[e] = n(F, D, s=F ** -0.5)
    xs, dys, g, u = n(N, D), n(N, D), n(N, F), n(N, F)
    grads = [torch.full_like(w, float("nan")) for w in (wg, wu, wd)]
    experts.backward(dys, xs, offsets_of(counts), wg, wu, wd, g, u, want=experts.GRADIENTS[1:], dwg=grads[0], dwu=grads[1], dwd=grads[2])
    del wg, wu
    lo = 0
    for e, k in rows.items():
        x, dy, gd, ud = (v[lo:lo + k].double() for v in (xs, dys, g, u))
        lo += k
        dh, terms = dy @ wd[e].double().T.contiguous(), dy.abs() @ wd[e].double().abs().T.contiguous()
        a, da = act(gd, "silu", 1.0)
        dg, du, h = dh * ud * da, dh * a, a * ud
        dgt, dut = dg.abs() + 2.0 ** -4 * (terms * ud * da).abs(), du.abs() + 2.0 ** -4 * (terms * a).abs()
        for name, got, ref, of in (("dwg", grads[0][e], x.T @ dg, x.abs().T @ dgt), ("dwu", grads[1][e], x.T @ du, x.abs().T @ dut),
                                   ("dwd", grads[2][e], h.T @ dy, h.abs().T @ dy.abs())):
            print(e, name, check((e, name), got, ref, of), flush=True)
    none = [e for e in range(E) if e not in rows]
    for e in range(0, len(none), 64):
        at = none[e:e + 64]
        assert all((w[at] == 0).all() for w in grads)
