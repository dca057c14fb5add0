"""The experts' calls with offsets that no sort gives: they count as their running maximum
within 0 .. N, so no row is two experts', every gradient is of rows that were computed, and
nothing outside of the tensors is touched.  Results are compared bit for bit with those of
offsets that hold this maximum, which tests/test_gpu_experts.py compares with the formulas.
"""
import pytest
import torch

from paper_2606_26344_amd import experts, gmlp

from test_gpu_experts import MARK, inputs, run

pytestmark = pytest.mark.gpu

COUNTERS = (1 << 17) + 256  # bytes in front of a workspace that calls leave as they were


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    assert torch.cuda.is_available(), "GPU tests need a HIP device"
    gmlp.library()


class Guarded:
    """Rows to write with marks in front of and behind them."""

    def __init__(self, n, cols):
        self.n = n
        self.whole = torch.full((n + 600, cols), MARK, dtype=torch.bfloat16, device="cuda")
        self.rows = self.whole[300:300 + n]

    def untouched(self):
        return bool((self.whole[:300] == MARK).all() and (self.whole[300 + self.n:] == MARK).all())


def results(t, offsets, workspace):
    N, D = t["xs"].shape
    F = t["wg"].shape[2]
    w = (t["wg"], t["wu"], t["wd"])
    guards = [Guarded(N, cols) for cols in (D, D, F, F, D)]
    alone, y, g, u, dxs = (v.rows for v in guards)
    workspace.buffer[COUNTERS:].fill_(0xff)  # NaN in what earlier calls left
    experts.forward(t["xs"], offsets, *w, out=alone, workspace=workspace)
    experts.train_forward(t["xs"], offsets, *w, out=y, g=g, u=u, workspace=workspace)
    workspace.buffer[COUNTERS:].fill_(0xff)
    grads = experts.backward(t["dys"], t["xs"], offsets, *w, g, u, dxs=dxs, workspace=workspace)
    assert all(v.untouched() for v in guards)
    assert torch.equal(alone, y)
    return (y, g, u, *grads)


def sorted_offsets(offsets, N):
    return torch.tensor(offsets, dtype=torch.int64).clamp(0, N).cummax(0).values.int().cuda()


def random_offsets(E, N, seed):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randint(0, N + 40, (E + 1,), generator=gen) - 20).tolist()


def falls_at(E, N, at):
    """Sorted but for one offset in front of and one behind place `at`."""
    o = [N * e // E for e in range(E + 1)]
    o[at - 1], o[at] = o[min(E, at + 5)], max(0, o[at] - N // 3)
    return o


CASES = [(50, [0, 20, 10, 10, 50]), (50, [20, 10, 30, 0, 50]), (50, [0, 50, 0, 50, 0]), (40, [2 ** 31 - 1, -2 ** 31, 0, 40]),
         (700, [0, 400, 100, 650, 300, 700]), (90, random_offsets(3, 90, 1)), (600, random_offsets(70, 600, 2)),
         (2000, random_offsets(300, 2000, 3)), (900, random_offsets(1024, 900, 4)), (400, falls_at(130, 400, 64)),
         (900, falls_at(600, 900, 256)), (900, falls_at(600, 900, 512)), (900, falls_at(1024, 900, 1023))]


@pytest.mark.parametrize("N,offsets", CASES, ids=[str(i) for i in range(len(CASES))])
def test_offsets_that_fall(N, offsets):
    E, D, F = len(offsets) - 1, 72, 136
    print("offsets N=%d E=%d %s" % (N, E, offsets if E < 12 else "..."), flush=True)
    t = inputs(N, E, D, F, N + E)
    workspace = experts.make_workspace(N, E, D, F)
    bad = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    good = sorted_offsets(offsets, N)
    got, want = results(t, bad, workspace), results(t, good, workspace)
    for a, b in zip(got, want):
        assert torch.equal(a, b) and not b.isnan().any()
    # An expert without rows has zeros for weight gradients.
    none = (good[1:] == good[:-1]).nonzero()[:, 0]
    assert all((w[none] == 0).all() for w in got[4:])


def test_split_sums_of_offsets_that_fall():
    """Few tiles of a long product, whose k is split over blocks."""
    N, E, D, F = 60, 3, 264, 4104
    t = inputs(N, E, D, F, 1)
    assert any(s > 1 for b in (False, True) for _, _, _, s in experts.describe(N, E, D, F, b))
    workspace = experts.make_workspace(N, E, D, F)
    for offsets in ([0, 40, 20, 60], [30, 10, 60, 0], [60, 0, 0, 60]):
        bad = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        got, want = results(t, bad, workspace), results(t, sorted_offsets(offsets, N), workspace)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("E", [63, 64, 65, 255, 256, 257, 512, 1024])
def test_counts_of_experts(E):
    """Sorted offsets of as many experts as lanes and groups of them have, against the
    formulas."""
    run([(7 * e) % 5 for e in range(E)], 16, 24, 4, 3, seed=E)
