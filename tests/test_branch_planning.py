"""Plans and entry points over rows under host sanitizers, the launchers stubbed (tests/sanitize/branch_fuzz.cpp).  No GPU is needed."""
import os
import shutil

import pytest

from test_sanitize import ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_planning_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "branch_fuzz.cpp"),
                                           os.path.join(ROOT, "paper_2002_00552_amd", "csrc", "branch.cpp")], ["-std=c++17", "-Wall"], ["20000"])
    assert "branch fuzz:" in out
