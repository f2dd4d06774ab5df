"""Work of the paged cache's calls run on the host under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only).

The page-table work (csrc/pages_ops.h) is built with g++ against a stand-in for hip_runtime.h and driven by
tests/sanitize/pages_driver.cpp, on consistent tables against the definitions and on arbitrary words."""
import os
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _have, _run

pytestmark = pytest.mark.skipif(not _have("g++"), reason="g++ not found")


def test_page_work_on_the_host(tmp_path):
    exe, san = tmp_path / "pages_driver", os.path.join(ROOT, "tests", "sanitize")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", *SAN, "-pthread", "-include", "memory",
                    "-I", os.path.join(san, "host_hip"), "-I", os.path.join(ROOT, "paper_2607_25852_amd", "csrc"),
                    os.path.join(san, "pages_driver.cpp"), "-o", str(exe)], check=True)
    r = _run([str(exe)])
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-4000:]
    assert r.stdout.startswith("ok"), r.stdout


def test_key_lists_and_plans_on_the_host(tmp_path):
    """sv_window_attn's key lists against the keys its rows see, and the host's bound, splits and workspace."""
    exe, csrc = tmp_path / "window_list_driver", os.path.join(ROOT, "paper_2607_25852_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", *SAN, "-I", os.path.join(ROOT, "include"),
                    "-I", csrc, os.path.join(ROOT, "tests", "sanitize", "window_list_driver.cpp"),
                    os.path.join(csrc, "sv_host.cpp"), "-o", str(exe)], check=True)
    r = _run([str(exe)])
    assert r.returncode == 0, r.stdout[-1000:] + r.stderr[-4000:]
    assert r.stdout.startswith("ok"), r.stdout
