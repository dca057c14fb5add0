"""The planning of the training step on the host (csrc/grad_plan.hpp, plain C++), built
with AddressSanitizer and UndefinedBehaviorSanitizer: tests/sanitize/grad_plan_check.cpp."""
import os
import shutil

import pytest

from test_sanitizers import HERE, ROOT, SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_training_plans_under_sanitizers(tmp_path):
    exe = str(tmp_path / "grad_plan_check")
    out = _build_and_run(["g++", "-std=c++20", *SAN, "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                          "-I", os.path.join(ROOT, "paper_2606_26344_amd", "csrc"), "-o", exe,
                          os.path.join(HERE, "sanitize", "grad_plan_check.cpp")], exe)
    assert "0 failures" in out
