"""Argument checks of the paged cache's calls, on the host before anything is enqueued (CPU only). Pointers
are fakes and SV_FAULT_INJECT=launch stands before every launch, so nothing here can reach a GPU."""
import ctypes
import os

import pytest

from paper_2607_25852_amd import binding as B

INVALID, UNSUPPORTED, WORKSPACE, HIP = 1, 2, 3, 4
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2607_25852_amd import build
        build.build()
    return B.load()


@pytest.fixture(autouse=True)
def no_launch(monkeypatch):
    monkeypatch.setenv("SV_FAULT_INJECT", "launch")


def fake(i=0):
    return ctypes.c_void_p(4096 + (i << 30))


def sweep_pointers(call, n, optional=(), wide=(), words=8, at16=()):
    """Every required pointer NULL, and every pointer misaligned, is refused; all of them sound reach the launch."""
    ptrs = [fake(i + 1) for i in range(n)]
    assert call(*ptrs) == HIP and "injected" in B.last_error(), B.last_error()
    for i in range(n):
        p = list(ptrs)
        p[i] = None
        assert call(*p) == (HIP if i in optional else INVALID), i
        p[i] = ctypes.c_void_p(ptrs[i].value + (8 if i in at16 else 4 if i in wide else 2))
        assert call(*p) == INVALID and "aligned" in B.last_error(), i


ROPE = dict(R=4, total_max=64, Hq=8, Hkv=2, d=128, sections=(24, 20, 20), page_size=16, max_pages_per_req=9,
            num_pages=40, dtype=B.SV_BF16)


def rope(lib, d, *p):
    return lib.sv_rope_append(ctypes.byref(d), *(p or [fake(i) for i in range(11)]), None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(R=0), INVALID, "num_reqs"), (dict(R=65536), INVALID, "num_reqs"), (dict(total_max=0), INVALID, "total_max"),
    (dict(total_max=(1 << 23) + 1), UNSUPPORTED, "launch"), (dict(Hq=0), INVALID, "num_q_heads"),
    (dict(Hkv=-1), INVALID, "num_kv_heads"), (dict(d=130), UNSUPPORTED, "head_dim"), (dict(d=2048), UNSUPPORTED, "head_dim"),
    (dict(d=64), INVALID, "rot_dim"), (dict(rot_dim=63), INVALID, "rot_dim"), (dict(rot_dim=126), INVALID, "sum"),
    (dict(sections=(64, 1)), INVALID, "rot_dim"), (dict(sections=(65, -1)), INVALID, "section[1]"),
    (dict(sections=(2 ** 31 - 1, 2 ** 31 - 1), rot_dim=128), INVALID, "sum"),
    (dict(sections=(2, 62), order=B.SV_ROPE_CYCLE), INVALID, "section[1]"), (dict(order=2), INVALID, "order"),
    (dict(pairing=-1), INVALID, "pairing"), (dict(page_size=48), INVALID, "page_size"),
    (dict(page_size=8192), INVALID, "page_size"), (dict(max_pages_per_req=0), INVALID, "max_pages_per_req"),
    (dict(num_pages=0), INVALID, "num_pages"), (dict(dtype=2), INVALID, "dtype"), (dict(scale=float("inf")), INVALID, "scale"),
    (dict(scale=float("nan")), INVALID, "scale"), (dict(q_stride=1023), INVALID, "q_stride"),
    (dict(q_stride=1028), INVALID, "q_stride"), (dict(k_stride=248), INVALID, "k_stride"),
    (dict(v_stride=-256), INVALID, "v_stride"), (dict(Hq=1 << 20), UNSUPPORTED, "elements"),
    (dict(Hq=1 << 14, total_max=1 << 20), UNSUPPORTED, "launch")])
def test_rope_descriptor(lib, kw, status, msg):
    assert rope(lib, B.rope_desc(**{**ROPE, **kw})) == status
    assert msg in B.last_error(), B.last_error()


def test_rope_arguments(lib):
    d = B.rope_desc(**ROPE)
    sweep_pointers(lambda *p: rope(lib, d, *p), 11, at16=(0, 1, 2, 8, 9, 10), wide=(4,))
    assert lib.sv_rope_append(None, *[fake()] * 11, None) == INVALID
    p = [fake(i) for i in range(11)]
    p[8] = p[0]
    assert rope(lib, d, *p) == HIP  # in place
    d = B.rope_desc(**ROPE, q_stride=2048)
    assert rope(lib, d, *p) == INVALID and "q_out is q" in B.last_error()
    with pytest.raises(ValueError):
        B.rope_desc(**{**ROPE, "sections": (10,) * 5})


WINDOW = dict(R=4, total_q_max=64, block=16, Hq=32, Hkv=8, d=128, page_size=64, max_pages_per_req=130, num_pages=1000,
              max_kv_len=8200, dtype=B.SV_BF16)


@pytest.mark.parametrize("kw,window,sinks,status,msg", [
    ({}, 0, 0, INVALID, "window"), ({}, -5, 0, INVALID, "window"), ({}, 1, -1, INVALID, "sinks"),
    (dict(Hq=30), 1, 0, INVALID, "multiple"), (dict(d=96), 1, 0, UNSUPPORTED, "head_dim"), (dict(block=17), 1, 0, INVALID, "block"),
    (dict(total_q_max=65), 1, 0, INVALID, "num_reqs*block"),
    (dict(R=65535, kv_split=64, max_kv_len=8192), 1 << 20, 0, UNSUPPORTED, "one launch"),
    (dict(R=65535, kv_split=64, max_kv_len=8192, dtype=B.SV_F32), 1 << 20, 0, UNSUPPORTED, "one launch"), (dict(kv_split=63), 1, 0, INVALID, "kv_split")])
def test_window_descriptor(lib, kw, window, sinks, status, msg):
    d = B.window_desc(B.attn_desc(**{**WINDOW, **kw}), window, sinks)
    assert lib.sv_window_attn(ctypes.byref(d), *[fake(i) for i in range(9)], BIG, None) == status
    assert msg in B.last_error(), B.last_error()
    assert lib.sv_window_attn_workspace_size(ctypes.byref(d)) == 0


@pytest.mark.parametrize("kw", [
    dict(R=65535, block=1, total_q_max=1, Hq=2 ** 31 - 1, Hkv=2 ** 31 - 1, d=4, max_pages_per_req=1 << 16, page_size=64,
         max_kv_len=1 << 22, kv_split=64, dtype=B.SV_F32),  # 2^32 lists for 2^31 blocks: just inside 64 bits
    dict(R=1, block=16, total_q_max=1, Hq=1 << 22, Hkv=1, d=256, kv_split=64, dtype=B.SV_F32)])
def test_window_calls_beyond_a_launch(lib, kw):
    d = B.window_desc(B.attn_desc(**{**WINDOW, **kw}), 2 ** 31 - 1, 0)
    assert lib.sv_window_attn(ctypes.byref(d), *[fake(i) for i in range(9)], BIG, None) == UNSUPPORTED
    assert "one launch" in B.last_error(), B.last_error()


def test_window_arguments(lib):
    d = B.window_desc(B.attn_desc(**{**WINDOW, "R": 2, "total_q_max": 2}), 6000, 4)
    need = B.window_attn_workspace_size(d)
    call = lambda *p: lib.sv_window_attn(ctypes.byref(d), *p, fake(20), need, None)
    sweep_pointers(call, 8, optional=(7,), at16=(0, 1, 2, 6))
    assert lib.sv_window_attn(None, *[fake()] * 9, BIG, None) == INVALID
    if need:
        args = [fake(i) for i in range(8)]
        assert lib.sv_window_attn(ctypes.byref(d), *args, fake(20), need - 1, None) == WORKSPACE
        assert lib.sv_window_attn(ctypes.byref(d), *args, None, need, None) == WORKSPACE
        assert lib.sv_window_attn(ctypes.byref(d), *args, ctypes.c_void_p(4104), need, None) == INVALID


PAGES = dict(R=8, max_pages_per_req=10, num_pages=100, page_size=16)


def page_calls(lib, d):
    """name -> call(pointers ...), number of pointers"""
    r = ctypes.byref(d)
    return {
        "fork": (lambda *p: lib.sv_fork_pages(r, 3, *p, None), 6),
        "reserve": (lambda *p: lib.sv_reserve_pages(r, *p, fake(30), BIG, None), 8),
        "release": (lambda *p: lib.sv_release_pages(r, 5, 1, *p, None), 3),
        "compact": (lambda *p: lib.sv_compact_pages(r, 0, *p, fake(30), BIG, None), 5),
    }


@pytest.mark.parametrize("kw,msg", [
    (dict(R=0), "num_reqs"), (dict(R=65536), "num_reqs"), (dict(max_pages_per_req=0), "max_pages_per_req"),
    (dict(max_pages_per_req=1 << 28), "2^30"), (dict(num_pages=0), "num_pages"), (dict(num_pages=(1 << 24) + 1), "num_pages"),
    (dict(page_size=0), "page_size"), (dict(page_size=24), "page_size"), (dict(page_size=8192), "page_size")])
def test_pages_descriptor(lib, kw, msg):
    d = B.pages_desc(**{**PAGES, **kw})
    for name, (call, n) in page_calls(lib, d).items():
        assert call(*[fake(i + 1) for i in range(n)]) == INVALID and msg in B.last_error(), name
        assert name in B.last_error()
    assert B.reserve_pages_workspace_size(d) == B.compact_pages_workspace_size(d) == 0


def test_pages_arguments(lib):
    d = B.pages_desc(**PAGES)
    for call, n in page_calls(lib, d).values():
        sweep_pointers(call, n)
    r = ctypes.byref(d)
    for size, call in ((B.reserve_pages_workspace_size(d), lambda ws, n: lib.sv_reserve_pages(
            r, *[fake(i) for i in range(8)], ws, n, None)),
            (B.compact_pages_workspace_size(d), lambda ws, n: lib.sv_compact_pages(r, 0, *[fake(i) for i in range(5)], ws,
                                                                                  n, None))):
        assert size > 0
        assert call(fake(20), size - 1) == WORKSPACE and call(None, size) == WORKSPACE
        assert call(ctypes.c_void_p(4100), size) == INVALID and call(fake(20), size) == HIP
    p = [fake(i) for i in range(6)]
    assert lib.sv_fork_pages(r, 0, *p, None) == INVALID and "rows_in" in B.last_error()
    assert lib.sv_fork_pages(r, 65536, *p, None) == INVALID
    for off in (0, 4 * 3 * 10 - 4, -(4 * 8 * 10 - 4)):  # table_out inside table_in, and the other way round
        p[3] = ctypes.c_void_p(p[0].value + off)
        assert lib.sv_fork_pages(r, 3, *p, None) == INVALID and "overlap" in B.last_error(), off
    for off in (4 * 3 * 10, -4 * 8 * 10):
        p[3] = ctypes.c_void_p(p[0].value + off)
        assert lib.sv_fork_pages(r, 3, *p, None) == HIP, off
    for off, status in ((0, INVALID), (4 * 2, INVALID), (-4 * 7, INVALID), (4 * 3, HIP), (-4 * 8, HIP)):  # the lengths
        p[4] = ctypes.c_void_p(p[1].value + off)
        assert lib.sv_fork_pages(r, 3, *p, None) == status, off
    p = [fake(i) for i in range(3)]
    assert lib.sv_release_pages(r, -1, 0, *p, None) == INVALID and lib.sv_release_pages(r, 1, -1, *p, None) == INVALID
    assert lib.sv_compact_pages(r, -1, *[fake(i) for i in range(5)], fake(9), BIG, None) == INVALID
    many = B.pages_desc(**{**PAGES, "R": 4097})
    assert B.reserve_pages_workspace_size(many) == 0
    assert lib.sv_reserve_pages(ctypes.byref(many), *[fake(i) for i in range(9)], BIG, None) == UNSUPPORTED
    assert "4096" in B.last_error()


COPY = dict(max_copies=5, layers=2, Hkv=8, d=128, page_size=16, num_pages=100, dtype=B.SV_BF16)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(max_copies=0), INVALID, "max_copies"), (dict(layers=0), INVALID, "num_layers"), (dict(Hkv=0), INVALID, "num_kv_heads"),
    (dict(num_pages=0), INVALID, "num_pages"), (dict(page_size=12), INVALID, "page_size"), (dict(dtype=9), INVALID, "dtype"),
    (dict(d=4), UNSUPPORTED, "head_dim"), (dict(d=0), UNSUPPORTED, "head_dim"), (dict(d=1 << 16), UNSUPPORTED, "head_dim"),
    (dict(Hkv=1 << 20, page_size=4096), UNSUPPORTED, "2^30"), (dict(layers=1 << 17), UNSUPPORTED, "2^16"),
    (dict(layer_stride=1), INVALID, "layer_stride"), (dict(layer_stride=100 * 8 * 16 * 128 + 4), INVALID, "layer_stride"),
    (dict(layer_stride=1 << 60), INVALID, "layer_stride")])
def test_copy_descriptor(lib, kw, status, msg):
    d = B.copy_desc(**{**COPY, **kw})
    assert lib.sv_copy_pages(ctypes.byref(d), *[fake(i) for i in range(6)], None) == status
    assert msg in B.last_error(), B.last_error()


def test_copy_arguments(lib):
    d = B.copy_desc(**COPY)
    sweep_pointers(lambda *p: lib.sv_copy_pages(ctypes.byref(d), *p, None), 6, optional=(2,), at16=(4, 5))


def test_null_descriptors(lib):
    p = [fake(i) for i in range(9)]
    assert lib.sv_fork_pages(None, 1, *p[:6], None) == INVALID
    assert lib.sv_reserve_pages(None, *p[:9], BIG, None) == INVALID
    assert lib.sv_release_pages(None, 0, 0, *p[:3], None) == INVALID
    assert lib.sv_compact_pages(None, 0, *p[:6], BIG, None) == INVALID
    assert lib.sv_copy_pages(None, *p[:6], None) == INVALID
    assert "NULL" in B.last_error()


def test_rows_of_other_strides_are_refused():
    """The binding passes rows of the descriptor's stride only."""
    import torch
    t = torch.zeros((4, 10 * 8))
    with pytest.raises(ValueError):
        B._rows_ptr(t[:, :16].view(4, 2, 8), 16, "q")
    with pytest.raises(ValueError):
        B._rows_ptr(torch.zeros((4, 8, 2)).transpose(1, 2), 0, "q")
    assert B._rows_ptr(t[:, :16].view(4, 2, 8), 80, "q") == t.data_ptr()
