"""What plans of matrix products say against what their calls launch, under host sanitizers, the launchers stubbed (tests/sanitize/branch_launches.cpp).  No GPU is needed."""
import os
import shutil

import pytest

from test_sanitize import ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans_say_what_runs(tmp_path):
    out = _build_and_run(tmp_path, "g++", [os.path.join(ROOT, "tests", "sanitize", "branch_launches.cpp"),
                                           os.path.join(ROOT, "paper_2002_00552_amd", "csrc", "branch.cpp")], ["-std=c++17", "-Wall"], ["40000"])
    assert "branch launches:" in out
