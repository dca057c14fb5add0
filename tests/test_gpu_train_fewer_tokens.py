"""A training workspace made for one number of tokens serves the shorter sequences of the
same run, whose plans may split their sums more: the same bits as with their own."""
import pytest
import torch

from paper_2606_26344_amd import gmlp, train
from test_gpu_train import inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


def step(t, rows, ws):
    x, dy = t["x"][:rows], t["dy"][:rows]
    y, g, u = train.forward(x, t["wg"], t["wu"], t["wd"], workspace=ws)
    return (y, g, u) + train.backward(dy, x, t["wg"], t["wu"], t["wd"], g, u, workspace=ws)


@pytest.mark.parametrize("T,D,F", [(300, 2048, 8192), (1300, 1032, 2056)])
def test_fewer_tokens(T, D, F):
    t = {k: v.cuda() for k, v in inputs(T, D, F, 1).items()}
    ws = train.make_workspace(T, D, F)
    for rows in (T, 257, 256, 128, 33, 1, T):
        print("T=%d D=%d F=%d rows=%d" % (T, D, F, rows), flush=True)
        for a, b in zip(step(t, rows, ws), step(t, rows, train.make_workspace(rows, D, F))):
            assert torch.equal(a, b)
    with pytest.raises(gmlp.GmlpError, match="workspace"):
        step({k: v.repeat(40, 1) if k in ("x", "dy") else v for k, v in t.items()}, 40 * T, ws)
