"""sv_copy_pages numbers the steps of a copy in 32 bits: more are refused (CPU only, nothing is launched)."""
import ctypes
import os

import pytest

from paper_2607_25852_amd import binding as B

UNSUPPORTED, HIP = 2, 4


@pytest.mark.parametrize("layers,Hkv,page,d,status", [
    (1 << 16, 1024, 4096, 128, UNSUPPORTED),         # 2^16 pieces of 16 KB in 2^16 layers and two caches: 2^33 steps
    (1 << 14, 1024, 4096, 128, UNSUPPORTED),         # 2^31
    ((1 << 14) - 1, 1024, 4096, 128, HIP), (1 << 16, 8, 64, 128, HIP)])
def test_steps_of_a_copy(layers, Hkv, page, d, status, monkeypatch):
    if not os.path.exists(B.LIB_PATH):
        from paper_2607_25852_amd import build
        build.build()
    monkeypatch.setenv("SV_FAULT_INJECT", "launch")  # stands before the launch
    desc = B.copy_desc(1, layers, Hkv, d, page, 1, B.SV_BF16)
    p = [ctypes.c_void_p(4096 * (i + 1)) for i in range(6)]
    assert B.load().sv_copy_pages(ctypes.byref(desc), *p, None) == status, B.last_error()
    assert ("layers" if status == UNSUPPORTED else "injected") in B.last_error()
