"""Calls whose tiles are more than one launch takes (no GPU): every shape within the limits
of include/gmlp_experts.h is taken, and its blocks are launched in parts."""
import os
import shutil

import pytest

from paper_2606_26344_amd import experts

from test_sanitizers import HERE, ROOT, SAN, _build_and_run

WIDE = 1 << 20


def test_one_launch_a_product_elsewhere():
    for N, E, D, F in ((1, 1, 8, 8), (8192, 8, 4096, 14336), (1 << 24, 8, 64, 64), (1, 512, 8, WIDE)):
        assert [len(experts.describe(N, E, D, F, b)) for b in (False, True)] == [2, 3]


@pytest.mark.parametrize("N,E,D,F,forward,backward", [
    (1, 1024, 8, WIDE, 2, 4), (1, 1024, WIDE, 8, 2, 4), (1, 963, 136, WIDE, 2, 5), (40000, 1024, 8, WIDE, 2, 4),
    (100000, 1024, 8, WIDE, 3, 4), (1 << 17, 1024, 8, WIDE, 3, 4), (0, 1024, 8, WIDE, 0, 2)])
def test_wide_and_narrow_weights(N, E, D, F, forward, backward):
    assert experts.workspace_size(N, E, D, F) > 0
    for kernels, n in ((experts.describe(N, E, D, F), forward), (experts.describe(N, E, D, F, True), backward)):
        assert len(kernels) == n
        for name, grid, block, splits in kernels:
            assert 0 < grid * block < 1 << 32
        for a, b in zip(kernels, kernels[1:]):
            assert a[0] != b[0] or a[1] % 8 == 0  # a part that another follows


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_parts_under_sanitizers(tmp_path):
    exe = str(tmp_path / "experts_launch_check")
    out = _build_and_run(["g++", "-std=c++20", *SAN, "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                          "-I", os.path.join(ROOT, "paper_2606_26344_amd", "csrc"), "-o", exe,
                          os.path.join(HERE, "sanitize", "experts_launch_check.cpp")], exe)
    assert " 0 failures" in out
