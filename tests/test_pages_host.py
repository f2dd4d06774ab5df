"""The page-table work of sv_fork_pages, sv_reserve_pages, sv_release_pages and sv_compact_pages run on the host
under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): csrc/pages_ops.h is built with g++
against a stand-in for hip_runtime.h and driven by tests/sanitize/pages_driver.cpp, on consistent
tables against the definitions and on arbitrary words."""
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
