"""Host-side checks of the training entry points (no GPU): arguments are
refused before any device is touched."""
import pytest

from paper_2606_26344_amd import gmlp, train

A = 0x10000000  # fake addresses: validation never dereferences
MB = 1 << 20
T, D, F = 16, 256, 512
NAMES = ("dY", "X", "Wg", "Wu", "Wd", "G", "U", "dX", "dWg", "dWu", "dWd")


def forward(shape=(T, D, F), act=0, beta=1.0, path=0, ws=A + 100 * MB, n=None, **p):
    at = {k: A + 4 * MB * i for i, k in enumerate(("X", "Wg", "Wu", "Wd", "Y", "G", "U"))}
    at.update(p)
    n = train.workspace_size(T, D, F) if n is None else n
    return gmlp.library().gmlp_train_forward(*at.values(), *shape, act, beta, path, ws, n, None)


def backward(shape=(T, D, F), act=0, beta=1.0, path=0, ws=A + 100 * MB, n=None, **p):
    at = {k: A + 4 * MB * i for i, k in enumerate(NAMES)}
    at.update(p)
    n = train.workspace_size(T, D, F) if n is None else n
    return gmlp.library().gmlp_train_backward(*at.values(), *shape, act, beta, path, ws, n, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_refusals(call):
    assert call(shape=(-1, D, F)) == 1 and call(shape=(T, 260, F)) == 2 and call(shape=(T, D, 0)) == 1
    assert call(act=7) == 1 and call(beta=float("inf")) == 1
    assert call(path=gmlp.PATH_MFMA) == 1 and call(path=gmlp.PATH_GEMV | gmlp.FRESH_WORKSPACE) == 1
    assert call(ws=None) == 1 and call(ws=A + 100 * MB + 16) == 2 and call(n=1 << 16) == 4
    for name in ("X", "Wg", "Wu", "Wd", "G", "U"):
        assert call(**{name: None}) == 1 and name in gmlp.last_error()
        assert call(**{name: A + 60 * MB + 8}) == 2 and name in gmlp.last_error()


def test_overlaps_are_refused():
    assert forward(Y=A) == 1 and "overlaps X" in gmlp.last_error() or "overlaps an input" in gmlp.last_error()
    assert forward(U=A + 5 * 4 * MB) == 1 and "U overlaps G" in gmlp.last_error()
    assert forward(G=A + 100 * MB) == 1 and "workspace" in gmlp.last_error()
    assert backward(dX=A) == 1 and "dX overlaps dY" in gmlp.last_error()
    assert backward(dWu=A + 8 * 4 * MB + 256) == 1 and "dWu overlaps dWg" in gmlp.last_error()
    assert backward(dWd=A + 100 * MB + (1 << 18)) == 1 and "workspace" in gmlp.last_error()
    assert backward(dX=A + 60 * MB + 8) == 2


def test_calls_that_launch_nothing():
    assert forward(shape=(0, D, F), X=None, Y=None, G=None, U=None) == 0
    assert backward(dX=None, dWg=None, dWu=None, dWd=None) == 0
    assert backward(shape=(0, D, F), dY=None, X=None, G=None, U=None, dX=None, dWg=None, dWu=None, dWd=None) == 0


def test_workspace_and_plans():
    assert train.workspace_size(-1, 256, 512) == 0 and train.workspace_size(4, 260, 512) == 0
    with pytest.raises(ValueError):
        train.make_workspace(4, 260, 512)
    for shape in [(0, 8, 8), (1, 8, 8), (16, 256, 512), (300, 1032, 2056), (4096, 4096, 14336), (1, 8, 1 << 22)]:
        n = train.workspace_size(*shape)
        assert n >= gmlp.workspace_size(*shape) and n >= 3 * shape[0] * shape[2] * 2, shape
        for name, grid, block, splits in train.describe(*shape) if shape[0] else []:
            assert grid * block < 1 << 32 and splits >= 1
    assert [k[0].split("<")[0] for k in train.describe(300, 1032, 2056, False)] == ["gemm_mfma_kernel"] * 2
    assert len(train.describe(300, 1032, 2056)) == 3 and len(train.describe(0, 8, 8)) == 1


def test_tiles_of_the_widest_tensors():
    """A tile's rows are addressed with 31 bits: fewer than 256 of a width of 2^22."""
    for D, F in ((8, 1 << 22), (1 << 22, 8), (256, 1 << 22)):
        for T in (1, 64, 257, 512, 4096):
            kernels = train.describe(T, D, F) + (train.describe(T, D, F, backward=False)[:1] if F > D else [])
            for name, *_ in kernels:
                wm, wn, tm, tn = (int(v) for v in name.split("Shape<")[1].split(",")[:4])
                if "Grad" in name:
                    assert max(wm * tm, wn * tn) * 32 < 256, (T, D, F, name)
    assert any("<4, 2, 2, 4" in k[0] for k in train.describe(4096, 4096, 1 << 21))
