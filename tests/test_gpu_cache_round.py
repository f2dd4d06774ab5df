"""The paged cache's calls together, as a server uses them: prompts forked into samples, room for a block, the
partly filled pages copied, rotated keys appended, windowed attention, what is not needed given back, the cache
compacted, and the next block. Eagerly, as a replayed graph, on two streams, and in a cache above 4 GiB."""
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


P, HQ, HKV, D, B_, WINDOW, SINKS, LAYERS = 16, 8, 2, 64, 5, 70, 4, 2
SECTIONS = (16, 8, 8)


def cu(torch, x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).cuda()


class Server:
    """Device state of one windowed cache of two layers and the calls of a round."""

    def __init__(self, torch, seed, stream=None):
        from paper_2607_25852_amd import binding as B
        self.torch, self.B, self.stream = torch, B, stream
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.prompts, self.samples = 3, 3
        self.R = self.prompts * self.samples
        self.lens = rng.integers(1, 200, self.prompts).astype(np.int32)
        self.lens[0] = 3 * P  # a full last page: nothing to copy
        self.cols = 256 // P
        self.pages = 120
        table, refs = np.full((self.prompts, self.cols), -1, np.int32), np.zeros(self.pages, np.int32)
        ids = iter(rng.permutation(self.pages))
        for i in range(self.prompts):
            for c in range(-(-int(self.lens[i]) // P)):
                table[i, c] = next(ids)
                refs[table[i, c]] = 1
        self.host = dict(table=table, ref=refs)
        self.parent = np.repeat(np.arange(self.prompts), self.samples).astype(np.int32)
        bf = dict(dtype=torch.bfloat16, device="cuda")
        self.kc0, self.vc0 = (torch.randn((LAYERS, self.pages, HKV, P, D), generator=g).to(torch.bfloat16).cuda()
                              for _ in range(2))
        self.kc, self.vc = self.kc0.clone(), self.vc0.clone()
        self.k = rng.integers(1, B_ + 1, self.R).astype(np.int32)
        self.accepted = np.minimum(rng.integers(0, B_ + 1, self.R), self.k).astype(np.int32)
        self.qo_host = np.concatenate([[0], np.cumsum(self.k)]).astype(np.int32)
        total = self.R * B_
        self.qkv = torch.randn((LAYERS, total, (HQ + 2 * HKV) * D), generator=g).to(torch.bfloat16).cuda()
        self.positions = np.zeros((3, total), np.int32)
        for i in range(self.R):
            for j in range(self.k[i]):
                self.positions[:, self.qo_host[i] + j] = self.lens[self.parent[i]] + j - np.array([0, 3, 7])
        i32 = dict(dtype=torch.int32, device="cuda")
        self.table_in0, self.ref0 = cu(torch, table), cu(torch, refs)
        self.table_in, self.ref = self.table_in0.clone(), self.ref0.clone()
        self.lens_d, self.parent_d = cu(torch, self.lens), cu(torch, self.parent)
        self.table = torch.zeros((self.R, self.cols), **i32)
        self.ctx = torch.zeros(self.R, **i32)
        self.kv = cu(torch, self.lens[self.parent] + self.k)
        self.kept = cu(torch, self.lens[self.parent] + self.accepted)
        self.qo, self.pos = cu(torch, self.qo_host), cu(torch, self.positions)
        self.freq_host = 10000.0 ** (-np.arange(D // 2) * 2 / D)
        self.freq = cu(torch, self.freq_host, np.float64)
        self.src, self.dst, self.tok = (torch.zeros(self.pages, **i32) for _ in range(3))
        self.info = torch.zeros(4, **i32)
        self.moves = torch.zeros(2, **i32)
        self.msrc, self.mdst = (torch.zeros(self.pages, **i32) for _ in range(2))
        self.q = torch.zeros((LAYERS, total, HQ, D), **bf)
        self.out = torch.zeros((2, LAYERS, total, HQ, D), **bf)
        self.lse = torch.zeros((2, LAYERS, total, HQ), device="cuda")
        self.pd = B.pages_desc(self.R, self.cols, self.pages, P)
        self.cd = B.copy_desc(self.R, LAYERS, HKV, D, P, self.pages, B.SV_BF16)
        self.md = B.copy_desc(self.pages, LAYERS, HKV, D, P, self.pages, B.SV_BF16)
        w = (HQ + 2 * HKV) * D
        self.rd = B.rope_desc(self.R, total, HQ, HKV, D, SECTIONS, P, self.cols, self.pages, B.SV_BF16,
                              order=B.SV_ROPE_CYCLE, q_stride=w, k_stride=w, v_stride=w)
        self.wd = B.window_desc(B.attn_desc(self.R, total, B_, HQ, HKV, D, P, self.cols, self.pages, self.cols * P,
                                            B.SV_BF16, kv_split=64), WINDOW, SINKS)
        need = max(B.reserve_pages_workspace_size(self.pd), B.compact_pages_workspace_size(self.pd),
                   B.window_attn_workspace_size(self.wd))
        self.ws = torch.full((need,), 0x33, dtype=torch.uint8, device="cuda")  # one for all calls, in order

    def reset(self):
        for a, b in ((self.table_in, self.table_in0), (self.ref, self.ref0), (self.kc, self.kc0), (self.vc, self.vc0)):
            a.copy_(b)
        self.out.zero_()
        self.lse.zero_()

    def attend(self, n):
        B, total = self.B, self.R * B_
        for l in range(LAYERS):
            B.window_attn(self.wd, self.q[l], self.kc[l], self.vc[l], self.table, self.qo, self.kv, self.out[n, l],
                          self.lse[n, l], self.ws, self.stream)

    def round(self):
        B, s = self.B, self.stream
        B.fork_pages(self.pd, self.prompts, self.table_in, self.lens_d, self.parent_d, self.table, self.ctx, self.ref, s)
        B.reserve_pages(self.pd, self.table, self.ref, self.ctx, self.kv, self.src, self.dst, self.tok, self.info,
                        self.ws, s)
        B.copy_pages(self.cd, self.src, self.dst, self.info[2:3], self.kc, self.vc, self.tok, s)
        for l in range(LAYERS):
            x = self.qkv[l]
            total = x.shape[0]
            B.rope_append(self.rd, x[:, :HQ * D].view(total, HQ, D), x[:, HQ * D:(HQ + HKV) * D].view(total, HKV, D),
                          x[:, (HQ + HKV) * D:].view(total, HKV, D), self.pos, self.freq, self.table, self.qo, self.ctx,
                          self.q[l], self.kc[l], self.vc[l], s)
        self.attend(0)
        # moving pages changes nothing that attention sees
        B.compact_pages(self.pd, 0, self.table, self.ref, self.msrc, self.mdst, self.moves, self.ws, s)
        B.copy_pages(self.md, self.msrc, self.mdst, self.moves[:1], self.kc, self.vc, None, s)
        self.attend(1)
        B.release_pages(self.pd, self.table, self.ref, self.kept, WINDOW, SINKS, s)

    def results(self):
        return [x.clone() for x in (self.table, self.ref, self.info, self.moves, self.kc, self.vc, self.out, self.lse)]


def check(s):
    """The round's results against the definitions, request by request on dense keys and values."""
    total, rows = s.R * B_, int(s.qo_host[-1])
    t, r, ctx = ref.fork(s.host["table"], s.host["ref"], s.lens, s.parent, P)
    new = ctx + s.k
    t, r, copies, info = ref.reserve(t, r, ctx, new, P)
    assert s.info.tolist() == info and info[0] == s.R and info[2] == 4  # prompts 1 and 2: two samples copy
    t, r, moves, live = ref.compact(t, r)
    assert s.moves.tolist() == [len(moves), live]
    t, r = ref.release(t, r, ctx + s.accepted, P, WINDOW, SINKS)
    np.testing.assert_array_equal(s.table.cpu().numpy(), t)
    np.testing.assert_array_equal(s.ref.cpu().numpy(), r)
    bits = lambda x: x.view(s.torch.int16).cpu()
    assert bool((bits(s.out[0]) == bits(s.out[1])).all()) and bool((s.lse[0] == s.lse[1]).all())
    assert not bool(s.out[:, :, rows:].any())
    f64 = lambda x: x.double().cpu().numpy()
    for l in range(LAYERS):
        x = f64(s.qkv[l])
        parts = (x[:, :HQ * D].reshape(total, HQ, D), x[:, HQ * D:(HQ + HKV) * D].reshape(total, HKV, D),
                 x[:, (HQ + HKV) * D:].reshape(total, HKV, D))
        turn = lambda y: ref.rotate(y, s.positions, s.freq_host, SECTIONS, "cycle", "halves")
        eq, mq = turn(parts[0])
        got = f64(s.q[l])
        assert (np.abs(got - eq) <= ref.BF16_HALF * np.abs(eq) + 2.0 ** -20 * mq)[:rows].all()
        # attention on the rotated rows as stored: dense caches, one page per request
        from_bf = lambda y: f64(s.torch.from_numpy(y).to(s.torch.bfloat16))
        kn, vn = from_bf(turn(parts[1])[0]), parts[2]
        k0, v0 = f64(s.kc0[l]), f64(s.vc0[l])
        n = 512
        kd, vd = np.full((s.R, HKV, n, D), np.nan), np.full((s.R, HKV, n, D), np.nan)
        for i in range(s.R):
            for p in range(ctx[i]):
                pg = s.host["table"][s.parent[i], p // P]
                kd[i, :, p], vd[i, :, p] = k0[pg, :, p % P], v0[pg, :, p % P]
            for j in range(s.k[i]):
                kd[i, :, ctx[i] + j], vd[i, :, ctx[i] + j] = kn[s.qo_host[i] + j], vn[s.qo_host[i] + j]
        eo, el, absv, absz, count, defined = ref.window_attention(got, kd, vd, np.arange(s.R)[:, None], s.qo_host, new,
                                                                  WINDOW, SINKS, B_, n)
        assert defined[:rows].all() and not defined[rows:].any()
        tol, tol_l = ref.window_tolerance("bf16", D, eo, el, absv, absz, count)
        # (a key's rounding may differ by one step from the definition's where the two fall on either side of
        # a border: its score then moves by a step of the key, 2^-7 of the largest product)
        border = 2.0 ** -7 * absz / np.sqrt(D)
        assert (np.abs(f64(s.out[0, l]) - eo) <= tol + 2 * border[:, :, None] * absv)[:rows].all()
        assert (np.abs(f64(s.lse[0, l]) - el) <= tol_l + border)[:rows].all()


def test_round(dev):
    for seed in (1, 2, 3):
        say("cache round", seed)
        s = Server(dev, seed)
        s.round()
        dev.cuda.synchronize()
        check(s)


def test_replayed_round(dev):
    """Captured once, replayed with eager rounds and other work between: every replay equals the eager round."""
    s = Server(dev, 4)
    s.round()
    want = s.results()
    g, side = dev.cuda.CUDAGraph(), dev.cuda.Stream()
    side.wait_stream(dev.cuda.current_stream())
    with dev.cuda.stream(side):
        s.reset()
        s.round()
    dev.cuda.synchronize()
    say("cache round captured")
    with dev.cuda.graph(g):
        s.reset()
        s.round()
    for n in range(4):
        s.ws.fill_(n * 60)
        g.replay()
        dev.cuda.synchronize()
        for a, b in zip(s.results(), want):
            assert dev.equal(a, b), n
        s.reset()
        s.round()
        dev.cuda.synchronize()
        for a, b in zip(s.results(), want):
            assert dev.equal(a, b), n


def test_two_streams(dev):
    """Two servers at once on their own streams, given to the calls."""
    streams = [dev.cuda.Stream(), dev.cuda.Stream()]
    servers = [Server(dev, 5 + n, stream=s) for n, s in enumerate(streams)]
    dev.cuda.synchronize()
    want = []
    for s in servers:
        s.round()
        dev.cuda.synchronize()
        want.append(s.results())
    say("two cache rounds at once")
    for n in range(3):
        for s, st in zip(servers, streams):
            with dev.cuda.stream(st):
                s.reset()
        for s in servers:
            s.round()
        dev.cuda.synchronize()
        for s, w in zip(servers, want):
            for a, b in zip(s.results(), w):
                assert dev.equal(a, b), n


def test_cache_above_four_gib(dev):
    """Pages whose offsets pass 32 bits, in elements too: the last pages of a cache of 5.4 GB (2.7 G elements) per
    tensor against the same in the first pages."""
    from paper_2607_25852_amd import binding as B
    pages, Hkv, page, d, k, ctx = 41000, 8, 64, 128, 3, 150
    say("cache above 4 GiB")
    kc, vc = (dev.empty((pages, Hkv, page, d), dtype=dev.bfloat16, device="cuda") for _ in range(2))
    assert kc.numel() > 2 ** 31 and kc.numel() * 2 > 2 ** 32
    g = dev.Generator(device="cuda").manual_seed(1)
    rows = dev.randn((3, k, Hkv, d), generator=g, device="cuda").to(dev.bfloat16)
    old = dev.randn((2, 3, Hkv, page, d), generator=g, device="cuda").to(dev.bfloat16)
    qo, ctx_d, kv = cu(dev, [0, k]), cu(dev, [ctx]), cu(dev, [ctx + k])
    freq, pos = cu(dev, 10000.0 ** (-np.arange(64) / 64), np.float64), cu(dev, np.arange(ctx, ctx + k)[None])
    res = []
    for at in ([0, 1, 2], [pages - 1, pages - 3, pages - 2]):
        kc[at], vc[at] = old[0], old[1]
        table = cu(dev, [at])
        q, out = (dev.zeros((k, Hkv, d), dtype=dev.bfloat16, device="cuda") for _ in range(2))
        B.rope_append(B.rope_desc(1, k, Hkv, Hkv, d, (64,), page, 3, pages, B.SV_BF16), rows[0], rows[1], rows[2], pos,
                      freq, table, qo, ctx_d, q, kc, vc)
        w = B.window_desc(B.attn_desc(1, k, k, Hkv, Hkv, d, page, 3, pages, 192, B.SV_BF16), 100, 4)
        ws = dev.empty(max(B.window_attn_workspace_size(w), 16), dtype=dev.uint8, device="cuda")
        B.window_attn(w, q, kc, vc, table, qo, kv, out, None, ws)
        src, dst = cu(dev, at), cu(dev, [10 + at[0] % 7, 20, 30])
        kc[dst.long()], vc[dst.long()] = 0, 0
        B.copy_pages(B.copy_desc(3, 1, Hkv, d, page, pages, B.SV_BF16), src, dst, cu(dev, [3]), kc, vc)
        res.append((q, out, kc[at].clone(), vc[at].clone(), kc[dst.long()].clone(), vc[dst.long()].clone()))
    for a, b in zip(*res):
        assert dev.equal(a, b)
    assert dev.equal(res[0][2], res[0][4]) and dev.equal(res[0][3], res[0][5]) and bool(res[0][1].any())
