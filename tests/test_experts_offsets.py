"""Which rows the experts have, whatever the offsets hold (csrc/experts_plan.hpp, plain
C++), built with AddressSanitizer and UndefinedBehaviorSanitizer:
tests/sanitize/experts_offsets_check.cpp."""
import os
import shutil

import pytest

from test_sanitizers import HERE, ROOT, SAN, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_of_any_offsets_under_sanitizers(tmp_path):
    exe = str(tmp_path / "experts_offsets_check")
    out = _build_and_run(["g++", "-std=c++20", *SAN, "-Wno-unused-function", "-I", os.path.join(ROOT, "include"),
                          "-I", os.path.join(ROOT, "paper_2606_26344_amd", "csrc"), "-o", exe,
                          os.path.join(HERE, "sanitize", "experts_offsets_check.cpp")], exe)
    assert " 0 failures" in out
