"""sv_window_attn on the GPU against its definition in 64 bits (tolerances: cache_reference.window_tolerance).
Every slot that no row of its request sees holds NaN, and pages behind the window are not in the table."""
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


def make(torch, seed, k, ctx, Hq, Hkv, d, page, dtype, window, sinks, block=16, extra=2, spread=1.0):
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, ctx = np.array(k), np.array(ctx)
    R, n = len(k), np.array(k) + np.array(ctx)
    qo = np.concatenate([[0], np.cumsum(k)]).astype(np.int32)
    total, cols = min(int(qo[-1]) + extra, R * block), -(-int(n.max()) // page)
    table, at = np.full((R, cols), -1, np.int32), []
    seen = []
    for i in range(R):
        s = np.arange(n[i])
        s = s[(s < sinks) | (s > ctx[i] - window)]
        seen.append(s)
        at += [(i, c) for c in sorted(set((s // page).tolist()))]
    pages = len(at) + 1
    for (i, c), pg in zip(at, rng.permutation(pages)):
        table[i, c] = pg
    shape = (pages, Hkv, page, d)
    kc, vc = torch.full(shape, float("nan")), torch.full(shape, float("nan"))
    for i in range(R):
        pg, slot = torch.from_numpy(table[i, seen[i] // page]).long(), torch.from_numpy(seen[i] % page)
        for c in (kc, vc):
            c[pg, :, slot] = torch.randn((len(seen[i]), Hkv, d), generator=g) * spread
    q = torch.randn((total, Hq, d), generator=g) * spread
    return dict(torch=torch, R=R, qo=qo, kv=n.astype(np.int32), total=total, cols=cols, pages=pages, table=table, Hq=Hq,
                Hkv=Hkv, d=d, page=page, dtype=dtype, window=window, sinks=sinks, block=block, q=q.to(dt).cuda(),
                kc=kc.to(dt).cuda(), vc=vc.to(dt).cuda(), max_kv=int(n.max()), scale=0.0, split=0)


def call(s, stream=None, ws=None, out=None, lse=None):
    from paper_2607_25852_amd import binding as B
    torch = s["torch"]
    attn = B.attn_desc(s["R"], s["total"], s["block"], s["Hq"], s["Hkv"], s["d"], s["page"], s["cols"], s["pages"],
                       s["max_kv"], B.SV_BF16 if s["dtype"] == "bf16" else B.SV_F32, sm_scale=s["scale"],
                       kv_split=s["split"])
    w = B.window_desc(attn, s["window"], s["sinks"])
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    if ws is None:
        ws = torch.full((max(B.window_attn_workspace_size(w), 16),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full_like(s["q"], 7.0) if out is None else out
    lse = torch.full((s["total"], s["Hq"]), 7.0, device="cuda") if lse is None else lse
    B.window_attn(w, s["q"], s["kc"], s["vc"], cu(s["table"]), cu(s["qo"]), cu(s["kv"]), out, lse, ws, stream)
    torch.cuda.synchronize()
    return out, lse


def check(s):
    out, lse = call(s)
    f64 = lambda t: t.double().cpu().numpy()
    eo, el, absv, absz, count, defined = ref.window_attention(
        f64(s["q"]), f64(s["kc"]), f64(s["vc"]), s["table"], s["qo"], s["kv"], s["window"], s["sinks"], s["block"],
        s["max_kv"], s["scale"] or None)
    tol, tol_l = ref.window_tolerance(s["dtype"], s["d"], eo, el, absv, absz, count)
    go, gl = f64(out), f64(lse)
    assert (go[~defined] == 7.0).all() and (gl[~defined] == 7.0).all(), "rows that no request owns"
    empty = defined & (count == 0)
    assert (go[empty] == 0).all() and (gl[empty] == -np.inf).all(), "rows without a key"
    use = defined & (count > 0)
    # (where the definition gives NaN, a clamped length having moved a window onto unwritten slots, so must the call)
    bad = ~((np.abs(go - eo) <= tol) | (np.isnan(go) & np.isnan(eo)))[use]
    assert not bad.any(), ("out", int(bad.sum()), float(np.nanmax(np.abs(go - eo)[use])), np.argwhere(bad)[:3].tolist())
    bad = ~((np.abs(gl - el) <= tol_l) | (np.isnan(gl) & np.isnan(el)))[use]
    assert not bad.any(), ("lse", float(np.nanmax(np.abs(gl - el)[use])), np.argwhere(bad)[:3].tolist())
    return go, gl


MIX_K, MIX_CTX = [1, 5, 16, 3, 8, 1], [0, 700, 130, 64, 63, 300]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 0), (33, 4), (64, 0), (64, 64), (100, 70), (129, 200),
                                          (2 ** 31 - 1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (5, 2 ** 31 - 1)])
def test_windows_and_sinks(dev, dtype, window, sinks):
    say("window", dtype, window, sinks)
    check(make(dev, 1, MIX_K, MIX_CTX, 8, 2, 64, 16, dtype, window, sinks))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,page,k,ctx", [
    (4, 4, 128, 64, [1, 1, 1], [0, 1, 500]), (8, 1, 128, 64, [1, 2, 16], [10, 63, 999]),
    (64, 4, 128, 32, [16, 7], [65, 400]), (28, 4, 64, 1, [1, 9], [30, 70]), (16, 1, 64, 4096, [16, 13], [100, 5000]),
    (64, 1, 128, 128, [16, 3], [300, 77]), (32, 8, 64, 2, [3, 4], [200, 0]), (5, 5, 64, 8, [2, 1], [50, 0]),
    (64, 1, 64, 16, [16], [333])])
def test_heads_and_pages(dev, dtype, Hq, Hkv, d, page, k, ctx):
    say("window heads", dtype, Hq, Hkv, d, page)
    for window, sinks in ((90, 3), (257, 0)):
        check(make(dev, 2, k, ctx, Hq, Hkv, d, page, dtype, window, sinks))


@pytest.mark.parametrize("d", [4, 12, 100, 256])
def test_fp32_head_dims(dev, d):
    say("window fp32 d", d)
    check(make(dev, 3, [4, 1], [150, 20], 6, 2, d, 16, "f32", 70, 5))


@pytest.mark.parametrize("R,d", [(48, 64), (48, 36), (32, 128), (32, 100)])
def test_fp32_blocks_of_32_rows(dev, R, d):
    """So many blocks of 16 rows that those of 32 pass in fewer rounds; requests that fill 1 to 4 half blocks, one whose
    visible value is infinite, a missing page."""
    say("window fp32 rows", R, d)
    rng = np.random.default_rng(R + d)
    s = make(dev, 23, rng.integers(1, 17, R), rng.integers(0, 150, R), 32, 8, d, 16, "f32", 60, 3)
    clean = check(s)[0]
    k0, page = int(s["qo"][1]), int(s["table"][0, (int(s["kv"][0]) - 1) // 16])
    s["vc"][page, :, (int(s["kv"][0]) - 1) % 16] = float("inf")  # of the first request's last row alone
    got = call(s)[0].double().cpu().numpy()
    assert np.abs(got[:k0 - 1] - clean[:k0 - 1]).max(initial=0) < 1e-5 and (got[k0:] == clean[k0:]).all()
    assert not np.isfinite(got[k0 - 1]).any()
    s["vc"][page, :, (int(s["kv"][0]) - 1) % 16] = 1.0
    s["table"][1, int(s["kv"][1] - 1) // 16] = -1
    check(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_windows(dev, dtype):
    """Few rows over many keys: the window is divided. Splits given by the caller."""
    s = make(dev, 4, [1, 3], [9000, 6100], 4, 1, 128, 64, dtype, 6000, 130)
    for split in (0, 64, 512, 4096, 1 << 20):
        s["split"] = split
        say("window long", dtype, split)
        check(s)


@pytest.mark.parametrize("Hq,d,page,k,ctx,window", [
    (4, 64, 1, [5, 2], [2700, 1500], 2500), (4, 128, 1, [5, 2], [2700, 1500], 2500), (8, 128, 2, [16, 1], [3500, 2100], 3400),
    (16, 64, 1, [16, 9], [2300, 1100], 2200), (16, 128, 1, [16, 9], [2300, 1100], 2200), (2, 64, 8, [3], [9500], 9000),
    (2, 128, 16, [3], [17500], 17000)])
def test_lists_longer_than_the_staged_pages(dev, Hq, d, page, k, ctx, window):
    """One work item walks more page ids than are staged at a time; also with a page missing near the end."""
    s = make(dev, 21, k, ctx, Hq, 1, d, page, "bf16", window, 70)
    s["split"] = 1 << 20
    say("window staged pages", Hq, d, page)
    check(s)
    s["table"][0, (ctx[0] - 100) // page] = -1
    check(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_every_size(dev, dtype):
    """Large and growing scores (the maximum moves), scores below -1e30, a given scale."""
    say("window scores", dtype)
    s = make(dev, 5, [4, 16], [400, 333], 8, 2, 64, 16, dtype, 300, 4, spread=4.0)
    check(s)
    s["scale"] = 0.37
    check(s)
    s = make(dev, 6, [2, 3], [100, 33], 4, 2, 64, 16, dtype, 80, 2)
    s["q"].fill_(-2.0 ** 60)  # every score is -2^126 / 8 (an exact sum): the weights are even
    s["kc"].fill_(2.0 ** 60)
    out, lse = call(s)
    even = s["vc"].float().cpu()
    row = int(s["qo"][1])
    pos = np.arange(100 + 2)
    for r, (i, p) in enumerate([(0, 100), (0, 101), (1, 33), (1, 34), (1, 35)]):
        keys = np.arange(p + 1)
        keys = keys[(keys < 2) | (keys > p - 80)]
        v = even[s["table"][i, keys // 16], :, keys % 16].double().mean(0)  # [Hkv, d]
        got = out[r].double().cpu().view(2, 2, 64)
        tol = 2 * ref.BF16_HALF if dtype == "bf16" else 1e-5
        assert float((got - v[:, None]).abs().max()) <= tol * float(even[~even.isnan()].abs().max()), (i, p)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_missing_pages(dev, dtype):
    """A visible key on a page that does not exist is masked; a row with none left gives 0 and -inf."""
    s = make(dev, 7, [4, 4, 2, 3], [100, 100, 20, 90], 8, 2, 64, 16, dtype, 40, 4)
    s["table"][0, 5] = -1
    s["table"][1, :] = s["pages"]
    s["table"][2, 1] = -2 ** 31
    s["cols"] = 6  # columns behind the table
    s["table"] = s["table"][:, :6].copy()
    s["max_kv"] = 96
    say("window missing pages", dtype)
    check(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_requests_that_do_not_fit(dev, dtype):
    say("window malformed", dtype)
    s = make(dev, 8, [4, 4, 2, 3], [100, 50, 20, 90], 8, 2, 64, 16, dtype, 40, 4, block=8)
    s["kv"][1] = 3       # fewer keys than rows
    s["kv"][3] = 10 ** 6  # more than max_kv_len: clamped
    check(s)
    s["qo"][:] = [0, 4, 8, 20, 23]  # twelve rows in a block of eight; rows behind the batch
    check(s)
    s["qo"][:] = [0, 4, 4, 6, 9]  # a request without rows
    check(s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_nan_and_inf_of_other_rows_keys(dev, dtype):
    """A later draft's key and value, and those that only earlier rows see, hold NaN and infinity: the rows
    that do not see them are as without, the others are not finite."""
    say("window nan", dtype)
    for what in (float("nan"), float("inf")):
        s = make(dev, 9, [4, 2], [100, 40], 8, 2, 64, 16, dtype, 40, 4)
        clean = call(s)[0].float().cpu()
        for p in (103, 61):  # seen by row 3 alone; by row 0 alone (its first key)
            s["vc"][int(s["table"][0, p // 16]), :, p % 16] = what
        got = call(s)[0].float().cpu()
        near = lambda x, y: bool(((x - y).abs() <= 2.0 ** -6 * (y.abs() + 1)).all())
        assert near(got[1:3], clean[1:3]) and bool((got[4:6] == clean[4:6]).all())
        assert not bool(got[0].isfinite().any()) and not bool(got[3].isfinite().any())
        for p in (103, 61):
            s["vc"][int(s["table"][0, p // 16]), :, p % 16] = 1.0
            s["kc"][int(s["table"][0, p // 16]), :, p % 16] = float("nan")
        got = call(s)[0].float().cpu()
        assert bool(got[1:3].isfinite().all()) and bool((got[4:6] == clean[4:6]).all())
        assert not bool(got[0].isfinite().any()) and not bool(got[3].isfinite().any())
