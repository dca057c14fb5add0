"""Gradients asked for one by one, on tiles whose number depends on the orientation of
the gradient (128 x 256 outputs: dWd of D columns and F rows takes other tiles than dWg
of F columns and D rows).  Bounds as in test_gpu_train.py."""
import pytest
import torch

from paper_2606_26344_amd import gmlp, train
from test_gpu_train import act, check, inputs

pytestmark = pytest.mark.gpu

# ceil(F / 128) is odd, so that the orientations differ; whole tiles only, and the tokens
# of every tile or of the last round split over blocks.
SHAPES = [(30, 2048, 8200), (16, 1024, 2056), (2000, 2048, 8200), (4096, 1024, 2056)]
WANTS = [("dwd",), ("dx", "dwd"), ("dwg",), ("dwu",), ("dwg", "dwd"), ("dwg", "dwu"), ("dx",)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


@pytest.mark.parametrize("T,D,F", SHAPES, ids=["T%dD%dF%d" % s for s in SHAPES])
def test_each_gradient_alone_is_whole(T, D, F):
    dev = {k: v.cuda() for k, v in inputs(T, D, F, T + F).items()}
    ws = train.make_workspace(T, D, F)
    _, g, u = train.forward(dev["x"], dev["wg"], dev["wu"], dev["wd"], workspace=ws)
    d = {k: v.double() for k, v in dev.items()}
    gd, ud = g.double(), u.double()
    a, da = act(gd, "silu", 1.0)
    dh, dh_terms = d["dy"] @ d["wd"].T, d["dy"].abs() @ d["wd"].abs().T
    dg, du, h = dh * ud * da, dh * a, a * ud
    dgt = dg.abs() + 2.0 ** -4 * (dh_terms * ud * da).abs()
    dut = du.abs() + 2.0 ** -4 * (dh_terms * a).abs()
    refs = {"dx": (dg @ d["wg"].T + du @ d["wu"].T, dgt @ d["wg"].abs().T + dut @ d["wu"].abs().T),
            "dwg": (d["x"].T @ dg, d["x"].abs().T @ dgt), "dwu": (d["x"].T @ du, d["x"].abs().T @ dut),
            "dwd": (h.T @ d["dy"], h.abs().T @ d["dy"].abs())}
    shapes = {"dx": (T, D), "dwg": (D, F), "dwu": (D, F), "dwd": (F, D)}
    for want in WANTS:
        print("T=%d D=%d F=%d want=%s" % (T, D, F, want), flush=True)
        room = {k: torch.full((shapes[k][0] * shapes[k][1] + 128,), float("nan"), dtype=torch.bfloat16, device="cuda")
                for k in want}
        outs = {k: room[k][64:-64].view(shapes[k]) for k in want}
        grads = train.backward(dev["dy"], dev["x"], dev["wg"], dev["wu"], dev["wd"], g, u, want=want, workspace=ws, **outs)
        for name, got in zip(train.GRADIENTS, grads):
            if name in want:
                check(name, got, *refs[name])
                assert room[name][:64].isnan().all() and room[name][-64:].isnan().all()
            else:
                assert got is None
