"""The layer norms' plans, checks and index rules under the address and undefined-behaviour sanitizers, CPU only."""
import os
import shutil

import pytest

from test_sanitize import ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_norm_planning_under_sanitizers(tmp_path):
    out = _build_and_run(tmp_path, "g++",
                         [os.path.join(ROOT, "tests", "sanitize", "norm_fuzz.cpp"), os.path.join(ROOT, "paper_2002_00552_amd", "csrc", "norm.cpp")],
                         ["-std=c++17", "-Wall"], ["3000"])
    assert "norm fuzz:" in out
