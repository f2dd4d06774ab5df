"""The host's plan for windowed attention at the shapes that the GPU tests rely on (CPU only)."""
import os
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _have
from window_shapes import BY_ROWS, IN_ORDER, PLAN, in_order, line

pytestmark = pytest.mark.skipif(not _have("g++"), reason="g++ not found")


def test_plans(tmp_path):
    exe, csrc = tmp_path / "window_plan_print", os.path.join(ROOT, "paper_2607_25852_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(ROOT, "tests", "sanitize", "window_plan_print.cpp"), os.path.join(csrc, "sv_host.cpp"),
                    "-o", str(exe)], check=True)
    cases = BY_ROWS + [in_order(*c) for c in BY_ROWS] + IN_ORDER
    r = subprocess.run([str(exe)], input="".join(line(s) for s, _ in cases), capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr[-2000:]
    for (shape, want), got in zip(cases, r.stdout.splitlines()):
        assert dict(zip(PLAN, map(int, got.split()))) == dict(zip(PLAN, want)), shape
    assert len(r.stdout.splitlines()) == len(cases)
