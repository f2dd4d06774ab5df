"""sv_rope_append on the GPU against its definition in 64 bits.

Tolerance, per element: half a step of the storage type at the value, and 2^-20 of the sum of the absolute
products for the fp32 arithmetic (the fraction of a turn and its sine and cosine within 2^-21.5, three
roundings of 2^-24). Values, passed-through dims and everything that the call does not own are equal bit for bit."""
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


def make(torch, seed, k, ctx, Hq, Hkv, d, page, dtype, sections, order="blocks", pairing="halves", scale=1.0, pad=0,
         extra=3, far=0, fused=True):
    """pad: elements between the fused rows; extra: rows behind the last sequence; far: added to the positions"""
    rng = np.random.default_rng(seed)
    g = torch.Generator().manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    k, ctx = np.array(k), np.array(ctx)
    R, qo = len(k), np.concatenate([[0], np.cumsum(k)]).astype(np.int32)
    total, cols = int(qo[-1]) + extra, max(1, -(-int((ctx + k).max()) // page))
    pages = R * cols + 2
    table = rng.permutation(pages)[:R * cols].reshape(R, cols).astype(np.int32)
    width = (Hq + 2 * Hkv) * d + pad
    s = dict(torch=torch, k=k, ctx=ctx, qo=qo, total=total, cols=cols, pages=pages, table=table, Hq=Hq, Hkv=Hkv, d=d,
             page=page, dtype=dtype, sections=sections, order=order, pairing=pairing, scale=scale)
    if fused:
        qkv = torch.randn((total, width), generator=g).to(dt).cuda()
        s["q"], s["k_new"] = qkv[:, :Hq * d].view(total, Hq, d), qkv[:, Hq * d:(Hq + Hkv) * d].view(total, Hkv, d)
        s["v_new"], s["stride"] = qkv[:, (Hq + Hkv) * d:(Hq + 2 * Hkv) * d].view(total, Hkv, d), width
    else:
        s["q"], s["stride"] = torch.randn((total, Hq, d), generator=g).to(dt).cuda(), 0
        s["k_new"], s["v_new"] = (torch.randn((total, Hkv, d), generator=g).to(dt).cuda() for _ in range(2))
    s["positions"] = (rng.integers(0, 5000, (len(sections), total)) + far).astype(np.int32)
    s["inv_freq"] = 10000.0 ** (-np.arange(sum(sections)) / sum(sections))
    shape = (pages, Hkv, page, d)
    s["k_cache"], s["v_cache"] = (torch.randn(shape, generator=g).to(dt).cuda() for _ in range(2))
    s["q_out"] = torch.randn((total, Hq, d), generator=g).to(dt).cuda()
    return s


def desc_of(s):
    from paper_2607_25852_amd import binding as B
    return B.rope_desc(len(s["k"]), s["total"], s["Hq"], s["Hkv"], s["d"], s["sections"], s["page"], s["cols"],
                       s["pages"], B.SV_BF16 if s["dtype"] == "bf16" else B.SV_F32,
                       order=B.SV_ROPE_CYCLE if s["order"] == "cycle" else B.SV_ROPE_BLOCKS,
                       pairing=B.SV_ROPE_ADJACENT if s["pairing"] == "adjacent" else B.SV_ROPE_HALVES,
                       q_stride=s["stride"], k_stride=s["stride"], v_stride=s["stride"], scale=s["scale"])


def check(s, q_out=None):
    """Runs the call and compares all it writes and all it must not write."""
    from paper_2607_25852_amd import binding as B
    torch = s["torch"]
    cu = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
    f64 = lambda t: t.double().cpu().numpy()
    q, kn, vn = f64(s["q"]), f64(s["k_new"]), f64(s["v_new"])
    q_out = s["q_out"] if q_out is None else q_out
    before = f64(q_out), f64(s["k_cache"]), f64(s["v_cache"])
    B.rope_append(desc_of(s), s["q"], s["k_new"], s["v_new"], cu(s["positions"]), cu(s["inv_freq"]), cu(s["table"]),
                  cu(s["qo"]), cu(s["ctx"].astype(np.int32)), q_out, s["k_cache"], s["v_cache"])
    torch.cuda.synchronize()
    rows, slots = ref.rope_slots(s["qo"], s["ctx"], s["table"], s["page"], s["pages"], s["total"])
    turn = lambda x: ref.rotate(x, s["positions"], s["inv_freq"], s["sections"], s["order"], s["pairing"], s["scale"])
    (eq, mq), (ek, mk) = turn(q), turn(kn)
    want_q, tol_q = before[0].copy(), np.zeros_like(before[0])
    bound = lambda e, m: np.where(m > 0, ref.half_step(s["dtype"]) * np.abs(e) + 2.0 ** -20 * m + 1e-38, 0.0)
    want_q[rows], tol_q[rows] = eq[rows], bound(eq, mq)[rows]
    want_k, want_v, tol_k = before[1].copy(), before[2].copy(), np.zeros_like(before[1])
    for r, pg, slot in slots:
        want_k[pg, :, slot], tol_k[pg, :, slot], want_v[pg, :, slot] = ek[r], bound(ek, mk)[r], vn[r]
    for name, got, want, tol in (("q", f64(q_out), want_q, tol_q), ("k", f64(s["k_cache"]), want_k, tol_k),
                                 ("v", f64(s["v_cache"]), want_v, 0.0)):
        bad = ~(np.abs(got - want) <= tol)
        assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), float(np.abs(got - want)[bad].max()))
    return slots


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("order,pairing", [("blocks", "halves"), ("cycle", "halves"), ("blocks", "adjacent"),
                                           ("cycle", "adjacent")])
def test_axes_and_pairs(dev, dtype, order, pairing):
    say("rope", dtype, order, pairing)
    s = make(dev, 1, [1, 4, 1, 7], [0, 15, 16, 40], 8, 2, 128, 16, dtype, (24, 20, 20), order, pairing)
    assert len(check(s)) == 13


@pytest.mark.parametrize("d,sections,pairing,dtype", [
    (64, (32,), "halves", "bf16"), (64, (10, 5, 5), "adjacent", "bf16"), (64, (5, 4, 3), "halves", "bf16"),
    (8, (1,), "halves", "bf16"), (8, (4,), "adjacent", "bf16"), (4, (1, 1), "adjacent", "f32"), (256, (128,), "halves", "bf16"),
    (1024, (512,), "halves", "bf16"), (100, (7, 0, 9, 3), "halves", "f32"), (128, (0, 64), "halves", "bf16"),
    (72, (18, 9, 9), "halves", "bf16"), (128, (16,), "adjacent", "f32"), (1024, (300,), "adjacent", "f32")])
def test_parts_of_a_head(dev, d, sections, pairing, dtype):
    """Rotated parts of any size, whole 16-byte chunks or not, four axes, axes without a pair."""
    say("rope", d, sections, pairing, dtype)
    check(make(dev, 2, [3, 1, 2], [9, 0, 100], 6, 3, d, 8, dtype, sections, "blocks", pairing, pad=8))


@pytest.mark.parametrize("dtype,d", [("bf16", 24), ("f32", 12)])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
def test_every_count_of_pairs(dev, dtype, d, pairing):
    """Halves of whole 16-byte chunks, of parts of them, and both; what passes through likewise; in place too."""
    for pairs in range(1, d // 2 + 1):
        say("rope pairs", dtype, pairing, pairs)
        check(make(dev, 30 + pairs, [3, 1, 6], [9, 0, 30], 3, 2, d, 8, dtype, (pairs,), "blocks", pairing))
        s = make(dev, 60 + pairs, [2, 5], [0, 17], 5, 1, d, 16, dtype, (pairs,), "blocks", pairing, fused=False)
        check(s, q_out=s["q"])


@pytest.mark.parametrize("page", [1, 2, 64, 4096])
def test_pages(dev, page):
    say("rope page", page)
    check(make(dev, 3, [16, 1, 5], [60, 4095, 8], 4, 4, 64, page, "bf16", (32,)))


def test_prompts_and_many_requests(dev):
    """Prompts of many rows, requests without rows, and as many requests as need three steps of the search."""
    say("rope prompts")
    check(make(dev, 4, [700, 0, 1, 0, 0, 333, 64, 0], [0, 5, 17, 0, 3, 100, 64, 9], 8, 1, 64, 16, "bf16", (16, 8, 8),
               "cycle"))
    rng = np.random.default_rng(5)
    k = (rng.random(4200) < 0.3).astype(int)
    say("rope 4200 requests")
    check(make(dev, 5, k, rng.integers(0, 9, 4200), 1, 1, 8, 8, "f32", (4,)))


@pytest.mark.parametrize("dtype,n,Hq,Hkv,d,pairing", [("bf16", 5601, 30, 9, 128, "halves"),
                                                      ("f32", 3500, 38, 1, 128, "adjacent")])
def test_large_batches(dev, dtype, n, Hq, Hkv, d, pairing):
    """More than 64 MB of rows are read and written past the caches: the same bits as the rows in small batches."""
    from paper_2607_25852_amd import binding as B
    torch, page = dev, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    dt, code = (torch.bfloat16, B.SV_BF16) if dtype == "bf16" else (torch.float32, B.SV_F32)
    q, kn, vn = (torch.randn((n, h, d), generator=g, device="cuda").to(dt) for h in (Hq, Hkv, Hkv))
    assert sum(x.numel() * x.element_size() for x in (q, kn, vn)) > 64 << 20
    pos = torch.randint(0, 9000, (2, n), generator=g, device="cuda", dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(64, dtype=torch.float64, device="cuda") / 64)
    cols = -(-(n + 5) // page)
    table = torch.randperm(cols + 3, generator=g, device="cuda")[:cols].to(torch.int32)[None].contiguous()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    code_of = dict(order=B.SV_ROPE_BLOCKS, pairing=B.SV_ROPE_ADJACENT if pairing == "adjacent" else B.SV_ROPE_HALVES)
    res = []
    for step in (n, 700):
        say("rope large", dtype, pairing, step)
        out = torch.zeros_like(q)
        kc, vc = (torch.zeros((cols + 3, Hkv, page, d), dtype=dt, device="cuda") for _ in range(2))
        for r in range(0, n, step):
            m = min(step, n - r)
            desc = B.rope_desc(1, m, Hq, Hkv, d, (40, 24), page, cols, cols + 3, code, **code_of)
            B.rope_append(desc, q[r:r + m], kn[r:r + m], vn[r:r + m], pos[:, r:r + m].contiguous(), freq, table, i32(0, m),
                          i32(5 + r), out[r:r + m], kc, vc)
        res.append((out, kc, vc))
    for x, y in zip(*res):
        assert torch.equal(x, y) and bool(x.any())


def test_far_positions_and_scale(dev):
    """Positions around 2^31: the fraction of the turn is what counts. Negative positions turn back."""
    say("rope far")
    s = make(dev, 6, [5, 3], [7, 0], 4, 2, 128, 16, "f32", (24, 20, 20), scale=1.3, far=2 ** 31 - 6000)
    check(s)
    s = make(dev, 7, [5, 3], [7, 0], 4, 2, 128, 16, "f32", (24, 20, 20), scale=-0.5, far=-100000)
    check(s)


def test_in_place_and_single_rows(dev):
    say("rope in place")
    for pairing in ("halves", "adjacent"):
        for sections in ((32,), (9, 4)):
            s = make(dev, 8, [2, 1, 6], [3, 30, 14], 4, 2, 64, 16, "bf16", sections, "blocks", pairing, fused=False)
            check(s, q_out=s["q"])
    check(make(dev, 9, [1], [0], 1, 1, 8, 1, "bf16", (4,), extra=0))


def test_rows_and_pages_that_do_not_exist(dev):
    """Missing pages, ids out of range, positions behind the table, negative contexts: the query is
    rotated, nothing is written elsewhere. Requests with rows outside the batch stay untouched."""
    say("rope bad pages")
    s = make(dev, 10, [4, 4, 4, 4, 4], [14, 3, 0, 8, 30], 4, 2, 64, 8, "bf16", (16, 8, 8))
    s["table"][0, 2] = -1
    s["table"][1, 0] = s["pages"]
    s["table"][2, 0] = -2 ** 31
    s["ctx"][3] = -5
    s["ctx"][4] = s["cols"] * 8 - 2
    assert len(check(s)) == 2 + 0 + 0 + 0 + 2
    say("rope rows outside the batch")
    s = make(dev, 11, [3, 3], [1, 2], 4, 2, 64, 8, "bf16", (32,), extra=2)
    s["qo"][2] = 900  # the last request's rows end behind the batch
    check(s)
    s["qo"][:] = [-3, 2, 5]
    check(s)
