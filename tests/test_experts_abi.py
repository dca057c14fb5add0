"""Host-side checks of the experts' entry points (no GPU)."""
import pytest

from paper_2606_26344_amd import experts, gmlp

A = 0x10000000  # fake addresses: validation never dereferences
MB = 1 << 20
FORWARD = ("X", "offsets", "Wg", "Wu", "Wd", "Y", "G", "U")
BACKWARD = ("dY", "X", "offsets", "Wg", "Wu", "Wd", "G", "U", "dX", "dWg", "dWu", "dWd")


def forward(N=16, E=4, D=256, F=512, act=0, beta=1.0, path=0, ws=A + 500 * MB, n=None, **p):
    at = {k: A + 16 * MB * i for i, k in enumerate(FORWARD)}
    at.update(p)
    n = experts.workspace_size(N, E, D, F) if n is None else n
    return gmlp.library().gmlp_experts_forward(*at.values(), N, E, D, F, act, beta, path, ws, n, None)


def backward(N=16, E=4, D=256, F=512, act=0, beta=1.0, path=0, ws=A + 500 * MB, n=None, **p):
    at = {k: A + 16 * MB * i for i, k in enumerate(BACKWARD)}
    at.update(p)
    n = experts.workspace_size(N, E, D, F) if n is None else n
    return gmlp.library().gmlp_experts_backward(*at.values(), N, E, D, F, act, beta, path, ws, n, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_refusals(call):
    assert call(N=-1) == 1 and call(E=0) == 1 and call(D=0) == 1 and call(F=-8) == 1
    assert call(D=260) == 2 and call(F=12) == 2 and call(E=1025) == 2 and call(N=(1 << 24) + 1) == 2
    assert call(D=(1 << 20) + 8) == 2 and call(F=(1 << 20) + 8) == 2 and call(E=1024, D=1 << 20, F=1 << 20) == 2
    assert call(N=1 << 24, F=1 << 16) == 2
    assert call(act=3) == 1 and call(beta=float("nan")) == 1 and call(path=1) == 1 and call(path=257) == 1
    for name in FORWARD[:6] if call is forward else BACKWARD[:8]:
        assert call(**{name: None}) == 1 and name in gmlp.last_error()
        assert call(**{name: A + 400 * MB + (2 if name == "offsets" else 8)}) == 2 and name in gmlp.last_error()
    assert call(ws=None) == 1 and call(ws=A + 500 * MB + 16) == 2 and call(n=4096) == 4


def test_gates_are_kept_together():
    assert forward(G=None) == 1 and forward(U=None) == 1 and "U" in gmlp.last_error()


@pytest.mark.parametrize("call,outputs", [(forward, FORWARD[5:]), (backward, BACKWARD[8:])])
def test_overlaps(call, outputs):
    for name in outputs:
        assert call(**{name: A + 256}) == 1 and name in gmlp.last_error()
        assert call(**{name: A + 500 * MB + 512}) == 1 and "workspace" in gmlp.last_error()
    assert call(**{outputs[0]: A + 16 * MB * (5 if call is backward else 4)}) == 1
    assert call(**{outputs[1]: A + 16 * MB * (8 if call is backward else 5)}) == 1
    assert call(offsets=A + 16 * MB * (8 if call is backward else 5)) == 1 and "offsets" in gmlp.last_error()


def test_nothing_to_do():
    rows = {"X": None, "offsets": None, "Y": None, "G": None, "U": None}
    assert forward(N=0, ws=None, **rows) == 0
    grads = {k: None for k in BACKWARD[8:]}
    assert backward(**grads) == 0
    assert backward(N=0, dY=None, X=None, offsets=None, G=None, U=None, dX=None, dWg=None, dWu=None, dWd=None) == 0


def test_workspace_sizes():
    assert experts.workspace_size(0, 1, 8, 8) > 0
    assert experts.workspace_size(4, 4, 12, 8) == 0 and experts.workspace_size(-1, 4, 8, 8) == 0
    assert experts.workspace_size(4, 0, 8, 8) == 0 and experts.workspace_size(4, 1 << 11, 8, 8) == 0
    for E, D, F in ((1, 264, 520), (8, 4096, 14336), (64, 2048, 1024), (1000, 512, 256)):
        sizes = [experts.workspace_size(n, E, D, F) for n in list(range(0, 400)) + list(range(400, 40000, 97))]
        assert sizes == sorted(sizes)  # one made for many rows serves fewer


@pytest.mark.parametrize("N,E,D,F", [(1, 1, 8, 8), (2, 8, 4096, 14336), (300, 32, 2048, 1024), (8192, 8, 4096, 14336),
                                     (4096, 1024, 256, 512), (65536, 256, 2048, 768), (1 << 24, 8, 64, 64)])
def test_plans(N, E, D, F):
    names = [experts.describe(N, E, D, F, b) for b in (False, True)]
    assert [len(n) for n in names] == [2, 3]
    for name, grid, block, splits in sum(names, []):
        assert name.startswith("gemm_grouped_kernel") and 0 < grid * block < 1 << 32 and splits >= 1
    assert experts.describe(0, E, D, F) == [] and len(experts.describe(0, E, D, F, True)) == 1
