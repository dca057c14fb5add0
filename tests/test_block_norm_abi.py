"""Host-side checks of the block norm entry points (no GPU)."""
import pytest

from paper_2606_26344_amd import block_norm, gmlp

A = 0x10000000  # fake addresses: validation never dereferences
MB = 1 << 20
FORWARD = ("Y", "res", "w_pre", "w_post", "gate", "R", "Xn")
BACKWARD = ("dXn", "dR", "Y", "R", "w_pre", "w_post", "gate", "dY", "dres", "dw_pre", "dw_post", "dgate")


def forward(T=16, D=256, flags=1, scale=1.0, eps=1e-6, **p):
    at = {k: A + MB * i for i, k in enumerate(FORWARD)}
    at.update(p)
    return gmlp.library().gmlp_block_norm(*at.values(), T, D, flags, scale, eps, None)


def backward(T=16, D=256, flags=1, scale=1.0, eps=1e-6, ws=A + 100 * MB, n=None, **p):
    at = {k: A + MB * i for i, k in enumerate(BACKWARD)}
    at.update(p)
    n = block_norm.workspace_size(T, D) if n is None else n
    return gmlp.library().gmlp_block_norm_backward(*at.values(), T, D, flags, scale, eps, ws, n, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_refusals(call):
    assert call(T=-1) == 1 and call(D=0) == 1 and call(D=260) == 2 and call(D=16392) == 2 and call(T=1 << 25) == 2
    assert call(flags=8) == 1 and call(scale=float("nan")) == 1 and call(eps=-1.0) == 1 and call(eps=float("inf")) == 1
    assert call(flags=0) == 1 and "w_post" in gmlp.last_error()
    assert call(flags=5, gate=None, **({"dgate": None} if call is backward else {})) == 1
    assert call(Y=None) == 1
    for name in ("res", "Xn") if call is forward else ("dXn", "R"):
        assert call(**{name: None}) == 1 and name in gmlp.last_error()
        assert call(**{name: A + 50 * MB + 8}) == 2 and name in gmlp.last_error()
    assert call(w_pre=A + 50 * MB + 4) == 2


def test_missing_partners():
    assert forward(R=None) == 1
    assert backward(w_pre=None) == 1 and "dw_pre" in gmlp.last_error()
    assert backward(w_post=None) == 1 and "dw_post" in gmlp.last_error()
    assert backward(gate=None) == 1 and "dgate" in gmlp.last_error()
    assert backward(flags=0, w_post=None, gate=None, dw_post=None, dgate=None, Y=None) == 1  # dY without Y
    assert backward(ws=None) == 1 and backward(ws=A + 100 * MB + 16) == 2 and backward(n=256) == 4


def test_overlaps():
    assert forward(R=A) == 1 and "R overlaps Y" in gmlp.last_error()
    assert forward(Xn=A + MB) == 1 and "Xn overlaps res" in gmlp.last_error()
    assert forward(R=A + MB + 512) == 1 and forward(Xn=A + 512) == 1  # res or Y, but not exactly
    assert backward(dY=A + 2 * MB) == 1 and backward(dres=A + 3 * MB) == 1 and backward(dY=A + 512) == 1
    assert backward(dw_post=A + 9 * MB + 256) == 1 and "dw_post overlaps dw_pre" in gmlp.last_error()
    assert backward(dgate=A + 100 * MB) == 1 and "workspace" in gmlp.last_error()


def test_no_rows_launches_nothing_where_nothing_is_wanted():
    assert forward(T=0, **{k: None for k in FORWARD}) == 0
    nothing = {k: None for k in BACKWARD if k not in ("w_pre", "w_post", "gate")}
    assert backward(T=0, ws=None, **nothing) == 0


def test_workspace_size():
    assert block_norm.workspace_size(0, 8) > 0 and block_norm.workspace_size(4096, 4096) >= 3 * 4096 * 4
    assert block_norm.workspace_size(4, 12) == 0 and block_norm.workspace_size(-1, 8) == 0
    for D in (8, 520, 2048, 4096, 16384):
        sizes = [block_norm.workspace_size(T, D) for T in range(0, 1200)]
        assert sizes == sorted(sizes)  # one made for many rows serves fewer
        for T in (1 << 14, 1 << 23):
            assert block_norm.workspace_size(T, D) == sizes[-1]
