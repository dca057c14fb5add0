"""Gradients of gains and gates over no rows: zeros, also where the gain or gate itself is
not finite (a sum without terms, times nothing)."""
import pytest
import torch

from paper_2606_26344_amd import block_norm, gmlp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


@pytest.mark.parametrize("res", [torch.bfloat16, torch.float32])
def test_no_rows_with_values_that_are_not_finite(res):
    D = 264
    empty = torch.empty((0, D), dtype=torch.bfloat16, device="cuda")
    gains = [torch.ones(D, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    for i, g in enumerate(gains):
        g[i], g[100 + i], g[200] = float("inf"), float("nan"), float("-inf")
    dy, dres, *sums = block_norm.backward(empty, empty.to(res), empty, empty.to(res), w_pre=gains[0], w_post=gains[1],
                                          gate=gains[2], post=True)
    assert dy.shape == dres.shape == (0, D)
    assert all(torch.equal(s, torch.zeros_like(s)) for s in sums)
