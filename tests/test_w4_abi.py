"""Host-side checks of the 4-bit entry points (no GPU)."""
import pytest

from paper_2606_26344_amd import gmlp, w4

A = 0x10000000  # fake addresses: validation never dereferences
MB = 1 << 20


def at(i):
    return A + 4 * MB * i


def matmul(T=4, K=256, N=512, group=128, zeros=0, path=0, ws=at(20), n=None, X=at(0), P=at(1), Y=at(2)):
    n = w4.workspace_size(max(0, min(T, 64)), 256, 512) if n is None else n
    return gmlp.library().gmlp_w4_matmul(X, P, Y, T, K, N, group, zeros, path, ws, n, None)


def forward(T=4, D=256, F=512, group=64, zeros=1, act=0, beta=1.0, path=0, ws=at(20), n=None, X=at(0), G=at(1), U=at(2),
            P=at(3), Y=at(4)):
    n = w4.workspace_size(max(0, min(T, 64)), 256, 512) if n is None else n
    return gmlp.library().gmlp_w4_forward(X, G, U, P, Y, T, D, F, group, zeros, act, beta, path, ws, n, None)


@pytest.mark.parametrize("call", [matmul, forward])
def test_refusals(call):
    assert call(T=-1) == 1 and call(T=65) == 2 and "dequantize" in gmlp.last_error()
    assert call(group=16) == 2 and call(group=0) == 2 and call(path=gmlp.PATH_MFMA) == 1
    assert call(ws=None) == 1 and call(ws=at(20) + 16) == 2 and call(n=1024) == 4
    for name in ("X", "P", "Y"):
        assert call(**{name: None}) == 1 and call(**{name: at(9) + 8}) == 2
    assert call(P=at(9) + 16) == 2 and "256-byte" in gmlp.last_error()
    assert call(Y=at(0)) == 1 and call(Y=at(1)) == 1 and call(Y=at(20) + 4096) == 1
    assert matmul(K=260) == 2 and matmul(N=0) == 1 and forward(D=12) == 2
    assert forward(act=9) == 1 and forward(beta=float("nan")) == 1 and forward(U=None) == 1


def test_no_tokens():
    assert matmul(T=0, X=None, Y=None, ws=None) == 0 and forward(T=0, X=None, Y=None, ws=None) == 0


def test_sizes():
    lib = gmlp.library()
    assert lib.gmlp_w4_packed_size(128, 16, 128, 0) == 1024 + 256
    assert lib.gmlp_w4_packed_size(136, 24, 32, 1) == 4 * 1024 + 4 * 16 * 4 * 2 + 256
    assert lib.gmlp_w4_packed_size(12, 16, 128, 0) == 0 and lib.gmlp_w4_packed_size(128, 16, 100, 0) == 0
    assert w4.workspace_size(65, 256, 512) == 0 and w4.workspace_size(0, 256, 512) > 0


def test_layout_refusals():
    lib = gmlp.library()
    assert lib.gmlp_w4_pack(at(0), at(1), None, at(2), 256, 512, 96, None) == 2
    assert lib.gmlp_w4_pack(None, at(1), None, at(2), 256, 512, 64, None) == 1
    assert lib.gmlp_w4_pack(at(0), at(1), None, at(2) + 64, 256, 512, 64, None) == 2
    assert lib.gmlp_w4_pack(at(0), at(1), None, at(0), 256, 512, 64, None) == 1
    assert lib.gmlp_w4_quantize(at(0), at(0), at(1), None, 256, 512, 64, None) == 1
    assert lib.gmlp_w4_quantize(at(0), at(2), None, None, 256, 512, 64, None) == 1
    assert lib.gmlp_w4_dequantize(at(0), at(0) + 1024, 256, 512, 64, 0, None) == 1
    assert lib.gmlp_w4_dequantize(at(0), None, 256, 512, 64, 0, None) == 1


def test_a_workspace_serves_fewer_tokens():
    for D, F in ((8, 8), (1024, 4096), (4168, 6184), (8192, 2048), (2056, 12296), (12296, 2056)):
        sizes = [w4.workspace_size(T, D, F) for T in range(1, 65)]
        assert sizes == sorted(sizes)
