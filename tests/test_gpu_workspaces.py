"""Workspaces of the modules: what fits in them, and which calls take them."""
import pytest
import torch

from paper_2606_26344_amd import block_norm, gmlp, train, w4
from paper_2606_26344_amd import softmax_matmul as smm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def test_fits_is_the_makers():
    """fits() answers for the calls of the module that made the workspace."""
    D, F = 1024, 4096
    plain = gmlp.Workspace(300, D, F)
    assert plain.fits(300, D, F) and not plain.fits(4096, D, F)
    # What a training step of the same shape takes is more, and its workspace says so.
    ws = train.make_workspace(300, D, F)
    assert all(ws.fits(T, D, F) for T in (300, 256, 1)) and not ws.fits(4096, D, F)
    small = train.make_workspace(16, D, F)
    T = next(t for t in range(17, 4096) if train.workspace_size(t, D, F) > small.nbytes)
    assert gmlp.workspace_size(T, D, F) <= small.nbytes and not small.fits(T, D, F)
    # 4-bit products end at 64 tokens.
    ws = w4.make_workspace(64, D, F)
    assert ws.fits(64, D, F) and ws.fits(1, D, F) and ws.fits(40, F, D) and not ws.fits(65, D, F)
    ws = smm.make_workspace(40, 264, 520)
    assert ws.fits(40, 264, 520) and not ws.fits(4000, 264, 520)
    assert not any(ws.fits(4, 260, 520) for ws in (plain, ws))  # no valid shape


def test_the_norms_workspace_is_refused():
    """It has no prepared counters, without which split sums are never finished."""
    T, D, F = 40, 264, 520
    gen = torch.Generator().manual_seed(1)
    x, wg, wu, wd = (torch.randn(s, generator=gen).to(torch.bfloat16).cuda() for s in ((T, D), (D, F), (D, F), (F, D)))
    h = gmlp.gate_up(x, wg, wu)
    p, s = smm.exp_rows(h)
    ws = block_norm.make_workspace(4096, 4096)
    calls = [lambda ws: gmlp.forward(x, wg, wu, wd, workspace=ws), lambda ws: gmlp.gate_up(x, wg, wu, workspace=ws),
             lambda ws: gmlp.forward(x, wg, wu, wd, workspace=ws, activation="sigmoid"),
             lambda ws: gmlp.down(h, wd, workspace=ws), lambda ws: smm.softmax_matmul(h, wd, workspace=ws),
             lambda ws: smm.divide(p, s, wd, workspace=ws)]
    for call in calls:
        with pytest.raises(TypeError, match="workspace"):
            call(ws)
        assert torch.isfinite(call(train.make_workspace(T, D, F)).float()).all()
