"""Which kernels a layer norm's backward call launches, by what it is asked for: no GPU is needed, the launchers are stubs."""
import os
import shutil

import pytest

from test_sanitize import ROOT, _build_and_run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_backward_calls_launch_what_they_are_asked_for(tmp_path):
    out = _build_and_run(tmp_path, "g++",
                         [os.path.join(ROOT, "tests", "sanitize", "norm_launches.cpp"), os.path.join(ROOT, "paper_2002_00552_amd", "csrc", "norm.cpp")],
                         ["-std=c++17", "-Wall"], [])
    assert "norm launches:" in out
