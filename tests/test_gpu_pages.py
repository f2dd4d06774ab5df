"""sv_fork_pages, sv_reserve_pages, sv_release_pages, sv_compact_pages and sv_copy_pages on the GPU against their
definitions written out in order: every output equal bit for bit."""
import numpy as np
import pytest

import cache_reference as ref
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    import torch
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2607_25852_amd import binding
    binding.load()
    return torch


def cu(torch, x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def run_reserve(torch, table, refs, ctx, new, page, ws_fill=0x77):
    from paper_2607_25852_amd import binding as B
    R, cols = table.shape
    d = B.pages_desc(R, cols, len(refs), page)
    ws = torch.full((B.reserve_pages_workspace_size(d),), ws_fill, dtype=torch.uint8, device="cuda")
    t, r = cu(torch, table), cu(torch, refs)
    src, dst, tok = (torch.full((R,), -9, dtype=torch.int32, device="cuda") for _ in range(3))
    info = torch.full((4,), -9, dtype=torch.int32, device="cuda")
    B.reserve_pages(d, t, r, cu(torch, ctx), cu(torch, new), src, dst, tok, info, ws)
    torch.cuda.synchronize()
    return t, r, src, dst, tok, info


def check_reserve(torch, table, refs, ctx, new, page):
    got = run_reserve(torch, table, refs, ctx, new, page)
    t, r, copies, info = ref.reserve(table, refs, ctx, new, page)
    n = len(copies)
    assert got[5].tolist() == info
    np.testing.assert_array_equal(got[0].cpu().numpy(), t)
    np.testing.assert_array_equal(got[1].cpu().numpy(), r)
    for k in range(3):
        assert got[2 + k].tolist() == [c[k] for c in copies] + [-9] * (len(table) - n)
    return info


SHAPES = [(1, 1, 1, 1), (3, 4, 16, 20), (17, 9, 64, 150), (64, 12, 16, 700), (200, 5, 1, 2000), (1100, 3, 8, 4096),
          (4096, 2, 4, 4096), (9, 40, 4, 4097), (4096, 2, 64, 9000), (50, 6, 16, 70001)]


@pytest.mark.parametrize("R,cols,page,pages", SHAPES)
def test_reserve_release(dev, R, cols, page, pages):
    rng = np.random.default_rng(R + pages)
    for others in (0.1, 0.9):
        say("reserve", R, cols, page, pages, others)
        table, refs, lens = ref.random_tables(rng, R, cols, page, pages, others=others)
        new = np.minimum(lens + rng.integers(0, 2 * page + 2, R), cols * page).astype(np.int32)
        check_reserve(dev, table, refs, lens, new, page)
        from paper_2607_25852_amd import binding as B
        for window, sinks in ((0, 0), (1, 0), (page + 1, 3), (2 * page, page), (2 ** 31 - 1, 2 ** 31 - 1)):
            t, r = cu(dev, table), cu(dev, refs)
            kept = rng.integers(-1, cols * page + 3, R).astype(np.int32)
            B.release_pages(B.pages_desc(R, cols, pages, page), t, r, cu(dev, kept), window, sinks)
            et, er = ref.release(table, refs, kept, page, window, sinks)
            np.testing.assert_array_equal(t.cpu().numpy(), et)
            np.testing.assert_array_equal(r.cpu().numpy(), er)


def test_reserve_order_and_limits(dev):
    """Samples of one prompt: all but the last copy its partly filled page. A request that cannot be served ends
    the batch: no page left, more columns than the table, a negative context."""
    page, cols, pages = 16, 4, 12
    table = np.full((4, cols), -1, np.int32)
    table[:, 0], table[:, 1] = 7, 3
    refs = np.zeros(pages, np.int32)
    refs[7] = refs[3] = 4
    ctx = np.full(4, 20, np.int32)
    say("reserve four samples")
    assert check_reserve(dev, table, refs, ctx, ctx + 5, page) == [4, 3, 3, 7]
    assert check_reserve(dev, table, refs, ctx, ctx + 13, page) == [4, 7, 3, 3]  # and a page each
    refs[3] = 5  # another holder elsewhere: everybody copies
    assert check_reserve(dev, table, refs, ctx, ctx + 5, page) == [4, 4, 4, 6]
    refs[3], refs[:3], refs[4:7], refs[8] = 4, 1, 1, 1  # three pages left
    assert check_reserve(dev, table, refs, ctx, ctx + 13, page) == [1, 2, 1, 1]
    refs[9:] = 1
    assert check_reserve(dev, table, refs, ctx, ctx + 13, page) == [0, 0, 0, 0]
    refs[9:] = 0
    for bad in (page * cols + 1, 2 ** 31 - 1):
        new = ctx + 1
        new[1] = bad
        assert check_reserve(dev, table, refs, ctx, new, page)[0] == 1
    neg = ctx.copy()
    neg[2] = -1
    assert check_reserve(dev, table, refs, neg, ctx + 1, page)[0] == 2
    assert check_reserve(dev, table, refs, ctx, ctx, page) == [4, 0, 0, 3]  # nothing to write


@pytest.mark.parametrize("R,cols,page,pages", SHAPES)
def test_fork(dev, R, cols, page, pages):
    from paper_2607_25852_amd import binding as B
    rng = np.random.default_rng(R + pages + 1)
    table, refs, lens = ref.random_tables(rng, R, cols, page, pages)
    lens[rng.random(R) < 0.1] = -4
    for out_rows in (1, R, 2 * R + 3):
        say("fork", R, cols, page, pages, "to", out_rows)
        parent = rng.integers(-1, R + 1, out_rows).astype(np.int32)
        t, r = cu(dev, table), cu(dev, refs)
        out = dev.full((out_rows, cols), -9, dtype=dev.int32, device="cuda")
        lo = dev.full((out_rows,), -9, dtype=dev.int32, device="cuda")
        B.fork_pages(B.pages_desc(out_rows, cols, pages, page), R, t, cu(dev, lens), cu(dev, parent), out, lo, r)
        et, er, el = ref.fork(table, refs, lens, parent, page)
        np.testing.assert_array_equal(out.cpu().numpy(), et)
        np.testing.assert_array_equal(r.cpu().numpy(), er)
        np.testing.assert_array_equal(lo.cpu().numpy(), el)
        np.testing.assert_array_equal(t.cpu().numpy(), table)


@pytest.mark.parametrize("R,cols,page,pages", SHAPES)
def test_compact(dev, R, cols, page, pages):
    from paper_2607_25852_amd import binding as B
    rng = np.random.default_rng(R + pages + 2)
    for others, limit in ((0.0, 0), (0.4, 0), (0.4, 3), (1.0, 0), (0.2, pages)):
        say("compact", R, cols, page, pages, others, limit)
        table, refs, _ = ref.random_tables(rng, R, cols, page, pages, others=others)
        if others == 1.0:
            refs[:] = 1  # a full cache
        d = B.pages_desc(R, cols, pages, page)
        t, r = cu(dev, table), cu(dev, refs)
        n = min(limit or pages // 2, pages // 2)
        src, dst = (dev.full((max(n, 1),), -9, dtype=dev.int32, device="cuda") for _ in range(2))
        info = dev.full((2,), -9, dtype=dev.int32, device="cuda")
        ws = dev.full((B.compact_pages_workspace_size(d),), 0x55, dtype=dev.uint8, device="cuda")
        B.compact_pages(d, limit, t, r, src, dst, info, ws)
        et, er, moves, live = ref.compact(table, refs, limit)
        assert info.tolist() == [len(moves), live]
        np.testing.assert_array_equal(t.cpu().numpy(), et)
        np.testing.assert_array_equal(r.cpu().numpy(), er)
        pad = [-9] * (max(n, 1) - len(moves))
        assert src.tolist() == [m[0] for m in moves] + pad and dst.tolist() == [m[1] for m in moves] + pad
    refs[:] = 0  # an empty cache
    t, r = cu(dev, np.full_like(table, -1)), cu(dev, refs)
    B.compact_pages(d, 0, t, r, src, dst, info, ws)
    assert info.tolist() == [0, 0] and int(r.abs().sum()) == 0


@pytest.mark.parametrize("Hkv,d,page,dtype,layers", [(1, 8, 1, "bf16", 1), (3, 128, 16, "bf16", 2), (2, 100, 64, "f32", 3),
                                                     (8, 128, 64, "bf16", 2), (1, 64, 4096, "f32", 1), (5, 72, 2, "bf16", 4)])
def test_copy(dev, Hkv, d, page, dtype, layers):
    from paper_2607_25852_amd import binding as B
    say("copy", Hkv, d, page, dtype, layers)
    rng = np.random.default_rng(d + page)
    pages, n = 40, 13
    dt = dev.bfloat16 if dtype == "bf16" else dev.float32
    gap = 64  # elements between the layers
    per = pages * Hkv * page * d
    flat = [dev.randn((layers * (per + gap),), device="cuda").to(dt) for _ in range(2)]
    ids = rng.permutation(pages)
    src, dst = ids[:n].astype(np.int32), ids[n:2 * n].astype(np.int32)
    src[3], dst[5] = pages, -1  # skipped
    tokens = rng.integers(0, page + 1, n).astype(np.int32)
    tokens[0], tokens[1], tokens[2] = -3, page + 9, 0
    desc = B.copy_desc(n, layers, Hkv, d, page, pages, B.SV_BF16 if dtype == "bf16" else B.SV_F32, layer_stride=per + gap)
    for count in (0, 1, n - 2, n + 50):
        for tk in (None, tokens):
            kc, vc = (f.clone() for f in flat)
            B.copy_pages(desc, cu(dev, src), cu(dev, dst), cu(dev, [count]), kc, vc, None if tk is None else cu(dev, tk))
            for got, old in ((kc, flat[0]), (vc, flat[1])):
                want = old.clone().view(layers, per + gap)
                was = old.view(layers, per + gap)[:, :per].view(layers, pages, Hkv, page, d)
                view = want[:, :per].view(layers, pages, Hkv, page, d)
                for e in range(min(count, n)):
                    if 0 <= src[e] < pages and 0 <= dst[e] < pages:
                        m = page if tk is None else min(max(int(tk[e]), 0), page)
                        view[:, dst[e], :, :m] = was[:, src[e], :, :m]
                assert dev.equal(got.view(layers, per + gap), want), (count, tk is None)
