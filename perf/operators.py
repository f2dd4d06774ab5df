"""Performance cases of the paged cache's operators: rotary positions on the way into the cache,
attention with a sliding window and visible first tokens, and the bookkeeping and moves of pages.

Interface: own, listed(), draw(rng), prepare(case, seed), run(state), work(case), exact(case, seed).
With own = False run() computes the plain form in elementary torch operations, with own = True it
makes the library's calls.

A case is a dict of plain values:
  op      "rope"     sv_rope_append of a packed batch's projection rows
          "window"   sv_window_attn of a packed batch
          "step"     sv_reserve_pages for a round's positions, then sv_release_pages of what the
                     acceptance gave back and the window passed
          "fork"     sv_fork_pages of prompts into samples, sv_reserve_pages, sv_copy_pages
          "compact"  sv_compact_pages, then sv_copy_pages of the moved pages
  R, b    requests, positions per request
  keep    the share of the R*b positions that is in the batch, in permille (at least one each)
  rows    (instead of b and keep) the longest of R prompts, whose lengths run evenly down to rows / R
  ctx, ctx_lo, ctx_hi   committed context lengths: lognormal with median ctx and sigma 1
          clipped to [ctx_lo, ctx_hi], or uniform over [ctx_lo, ctx_hi] when ctx is 0
  Hq, Hkv, d, page, dtype   heads, head dim, page size and type of rows and caches
  window, sinks   keys a row sees: the last `window` and the first `sinks`
  sections, order, pairing   rotated pairs of each axis ("16,24,24"), their order, the partners of a pair
  pool, fill, layers, samples   pages of the cache, share in use (permille), layers, samples per prompt
The lengths and depths are those of the case, in a seeded order, so its work does not depend on the seed.
"""
import math
import random
import statistics

import numpy as np
import torch

own = False

HEADS64 = dict(Hq=64, Hkv=8, d=128, page=64)
MIXED = dict(ctx=4096, ctx_lo=512, ctx_hi=32768)


def listed():
    return [
        # The smallest: four users, one new token each, positions of text inside a video
        # conversation (time, height, width), keys and values into the cache.
        dict(name="rope_decode_c4", op="rope", R=4, b=1, keep=1000, ctx=8192, ctx_lo=512, ctx_hi=65536,
             dtype="bf16", sections="16,24,24", order="blocks", pairing="halves", window=1024, sinks=4, **HEADS64),
        # A full verify round of a text model: half of 64 requests' 16 positions, one axis.
        dict(name="rope_verify_c64", op="rope", R=64, b=16, keep=500, dtype="bf16", sections="64", order="blocks",
             pairing="halves", window=1024, sinks=4, **MIXED, **HEADS64),
        # Prompts of image and video tokens, ragged, 16-token pages, axes taken in turn.
        dict(name="rope_prompts_c5", op="rope", R=5, rows=4999, ctx=0, ctx_lo=0, ctx_hi=700, Hq=28, Hkv=4, d=128,
             page=16, dtype="bf16", sections="24,20,20", order="cycle", pairing="halves", window=1 << 20, sinks=0),
        # fp32 rows, a part of the head rotated, neighbouring dims as pairs.
        dict(name="rope_partial_f32_c27", op="rope", R=27, b=8, keep=700, ctx=0, ctx_lo=1000, ctx_hi=8191, Hq=32,
             Hkv=8, d=64, page=16, dtype="f32", sections="10,5,5", order="blocks", pairing="adjacent",
             window=1000, sinks=5),
        # One new token for each of four users: latency of a short window.
        dict(name="window_decode_c4", op="window", R=4, b=1, keep=1000, ctx=8192, ctx_lo=512, ctx_hi=65536,
             dtype="bf16", window=1024, sinks=4, **HEADS64),
        # A windowed layer of a full verify round.
        dict(name="window_verify_c64", op="window", R=64, b=16, keep=500, dtype="bf16", window=1024, sinks=4, **MIXED,
             **HEADS64),
        # 64-wide heads on 16-token pages, odd counts throughout.
        dict(name="window_page16_c27", op="window", R=27, b=8, keep=600, ctx=0, ctx_lo=100, ctx_hi=8191, Hq=32, Hkv=8,
             d=64, page=16, dtype="bf16", window=1000, sinks=5),
        # A wide window over 64K to 128K tokens, 16 query heads per kv-head. The largest.
        dict(name="window_long_c32", op="window", R=32, b=16, keep=520, ctx=0, ctx_lo=65536, ctx_hi=131072, Hq=64,
             Hkv=4, d=128, page=64, dtype="bf16", window=32768, sinks=64),
        # fp32 cache, blocks of five positions.
        dict(name="window_f32_c8", op="window", R=8, b=5, keep=1000, ctx=2048, ctx_lo=64, ctx_hi=16384, Hq=32, Hkv=8,
             d=128, page=64, dtype="f32", window=512, sinks=1),
        # A round's page bookkeeping: room for 64 blocks of 16, then the rejected positions' and
        # the window's dead pages back. No data moves; latency counts.
        dict(name="pages_step_c64", op="step", R=64, b=16, page=16, pool=24576, fill=700, window=1024, sinks=4,
             **MIXED),
        # Sixteen prompts into four samples each, eight layers: tables, counts, and copies of the
        # last, partly filled pages.
        dict(name="pages_fork_c16x4", op="fork", R=16, samples=4, b=16, layers=8, Hkv=8, d=128, page=64, dtype="bf16",
             ctx=2048, ctx_lo=300, ctx_hi=8000),
        # A cache of 16-token pages, six in ten in use, packed to its low end in two layers.
        dict(name="pages_compact_16k", op="compact", R=128, layers=2, Hkv=8, d=128, page=16, dtype="bf16", pool=16384,
             fill=600),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rope", "rope", "window", "window", "window", "step", "fork", "compact"))
    Hq, Hkv = rng.choice(((32, 8), (64, 8), (64, 4), (32, 4), (28, 4), (8, 1)))
    case = dict(op=op, R=_log_int(rng, 4, 64), Hkv=Hkv, d=rng.choice((64, 128, 128)),
                page=rng.choice((16, 32, 64, 64, 128)), dtype=rng.choice(("bf16", "bf16", "bf16", "f32")))
    if op in ("rope", "window"):
        case["Hq"] = Hq
        if op == "rope" and rng.random() < 0.4:
            case.update(R=rng.randint(1, 9), rows=_log_int(rng, 16, 2500), window=1 << 20, sinks=0, ctx=0, ctx_lo=0,
                        ctx_hi=rng.randint(1, 4000))
        else:
            case.update(b=rng.choice((1, 5, 8, 16, rng.randint(2, 16))), keep=rng.choice((250, 500, 750, 1000)),
                        window=_log_int(rng, 16, 8192), sinks=rng.choice((0, 1, 4, 64, rng.randint(2, 200))),
                        ctx=_log_int(rng, 64, 16384), ctx_lo=rng.choice((0, 1, 40)), ctx_hi=65536)
        if op == "rope":
            half = case["d"] // 2
            rot = rng.choice((half, half, half // 2, rng.randint(3, half)))
            axes = rng.randint(1, 3)
            rest = rot // 3 if axes > 1 else 0
            case.update(sections=",".join(str(n) for n in [rot - rest * (axes - 1)] + [rest] * (axes - 1)),
                        order=rng.choice(("blocks", "cycle")), pairing=rng.choice(("halves", "halves", "adjacent")))
        elif case["dtype"] == "f32":
            case.update(R=min(case["R"], 16), window=min(case["window"], 1024))
    elif op == "step":
        case.update(R=_log_int(rng, 4, 512), b=rng.choice((1, 5, 16)), pool=_log_int(rng, 40000, 100001),
                    fill=rng.choice((500, 700, 900)), window=rng.choice((0, 128, 1000)), sinks=rng.choice((0, 4, 70)),
                    ctx=1024, ctx_lo=1, ctx_hi=1200)
        for k in ("Hkv", "d", "dtype"):
            del case[k]
        case["page"] = max(case["page"], 32)
    elif op == "fork":
        case.update(R=rng.randint(1, 16), samples=rng.randint(2, 6), b=rng.choice((1, 5, 16)), layers=rng.randint(1, 4),
                    ctx=_log_int(rng, 64, 2048), ctx_lo=1, ctx_hi=5000)
    else:
        case.update(R=_log_int(rng, 8, 256), layers=rng.randint(1, 2), pool=_log_int(rng, 500, 4000),
                    fill=rng.choice((300, 600, 900)))
        case["R"] = min(case["R"], case["pool"] * case["fill"] // 4000)
    return case


# ---------------------------------------------------------------------------------------
# sizes that the case fixes
# ---------------------------------------------------------------------------------------
def _lengths(case):
    """Committed context lengths, in the case's own order."""
    R, out = case["R"], []
    for i in range(R):
        x = (i + 0.5) / R
        if case["ctx"]:
            v = case["ctx"] * math.exp(statistics.NormalDist().inv_cdf(x))
        else:
            v = case["ctx_lo"] + x * (case["ctx_hi"] - case["ctx_lo"])
        out.append(int(min(max(round(v), case["ctx_lo"]), case["ctx_hi"])))
    random.Random(1).shuffle(out)
    return out


def _depths(case):
    """Rows of each request in the batch, in the case's own order."""
    R = case["R"]
    if "rows" in case:
        return [max(1, round(case["rows"] * (i + 1) / R)) for i in range(R)]
    b = case["b"]
    k = [1] * R
    rng = random.Random(2)
    for _ in range(min(R * b, max(R, -(-case["keep"] * R * b // 1000))) - R):
        i = rng.randrange(R)
        while k[i] == b:
            i = (i + 1) % R
        k[i] += 1
    return k


def _esz(case):
    return 4 if case["dtype"] == "f32" else 2


def _sections(case):
    return [int(n) for n in case["sections"].split(",")]


def _axis(case):
    """The position axis of each rotated pair."""
    sec = _sections(case)
    pairs = sum(sec)
    if case["order"] == "blocks":
        return [a for a, n in enumerate(sec) for _ in range(n)]
    return [p % len(sec) if p // len(sec) < sec[p % len(sec)] else 0 for p in range(pairs)]


def _seen(L, k, window, sinks):
    """(keys any of the k rows after L sees, pairs of row and key)"""
    n = L + k
    lo = max(0, L - window + 1)
    head = min(sinks, lo)
    pairs = 0
    for p in range(L, n):
        w0 = max(0, p - window + 1)
        pairs += p + 1 - w0 + min(sinks, w0)
    return n - lo + head, pairs


# ---------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------
def _gen(seed, dev):
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    return g


def _order(n, seed):
    return np.random.default_rng(int(seed)).permutation(n)


def _i32(x, dev):
    return torch.tensor(np.ascontiguousarray(x), dtype=torch.int32, device=dev)


def _live_columns(L, n, window, sinks, P, cols):
    """[R, cols]: columns that hold a key which a row at position L or later sees, up to n tokens."""
    c = np.arange(cols)[None, :]
    L, n = np.asarray(L)[:, None], np.asarray(n)[:, None]
    return (c * P < n) & ((c * P < sinks) | ((c + 1) * P > L - window + 1))


def _batch(case, seed, dev):
    """The packed batch and the cache of a windowed layer: pages behind the window are given back."""
    R, P = case["R"], case["page"]
    perm = _order(R, seed)
    L, k = np.array(_lengths(case))[perm], np.array(_depths(case))[perm]
    qo = np.concatenate([[0], np.cumsum(k)])
    cols = -(-int((L + k).max()) // P)
    live = _live_columns(L, L + k, case["window"], case["sinks"], P, cols)
    pool = int(live.sum()) * 9 // 8 + 1
    table = np.full((R, cols), -1, np.int32)
    table[live] = _order(pool, seed + 1)[:int(live.sum())]
    K = int(qo[-1])
    total = K if "rows" in case else R * case["b"]
    return dict(case=case, K=K, total=total, L=L, k=k, pool=pool, cols=cols, table=_i32(table, dev), qo=_i32(qo, dev),
                ctx=_i32(L, dev), kv_lens=_i32(L + k, dev))


def _normal(shape, case, g, dev):
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    return torch.randn(shape, generator=g, device=dev, dtype=dt)


def _prepare_rope(case, seed, dev):
    s = _batch(case, seed, dev)
    g = _gen(seed, dev)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    A, rot = len(_sections(case)), 2 * sum(_sections(case))
    # the projection's rows: queries, keys and values of a token beside each other
    qkv = _normal((s["total"], (Hq + 2 * Hkv) * d), case, g, dev)
    s["q"] = qkv[:, :Hq * d].view(s["total"], Hq, d)
    s["k_new"] = qkv[:, Hq * d:(Hq + Hkv) * d].view(s["total"], Hkv, d)
    s["v_new"] = qkv[:, (Hq + Hkv) * d:].view(s["total"], Hkv, d)
    # positions: the prompts' rows are frames of 16 x 24 patches, other rows are text
    row = np.concatenate([np.arange(n) for n in s["k"]])
    base = np.repeat(s["L"], s["k"])
    if "rows" in case:
        pos = np.stack([base + row // 384, base + row // 24 % 16, base + row % 24])
    else:
        pos = np.stack([base + row] * 3)
    full = np.zeros((A, s["total"]), np.int32)
    full[:, :s["K"]] = pos[:A]
    s["positions"] = _i32(full, dev)
    s["inv_freq"] = 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
    s["axis"] = torch.tensor(_axis(case), device=dev)
    shape = (s["pool"], Hkv, case["page"], d)
    s["k_cache"], s["v_cache"] = _normal(shape, case, g, dev), _normal(shape, case, g, dev)
    s["q_out"] = torch.zeros((s["total"], Hq, d), dtype=s["q"].dtype, device=dev)
    if own:
        from paper_2607_25852_amd import binding as B
        s["desc"] = B.rope_desc(case["R"], s["total"], Hq, Hkv, d, _sections(case), case["page"], s["cols"], s["pool"],
                                B.SV_F32 if case["dtype"] == "f32" else B.SV_BF16,
                                order=B.SV_ROPE_CYCLE if case["order"] == "cycle" else B.SV_ROPE_BLOCKS,
                                pairing=B.SV_ROPE_ADJACENT if case["pairing"] == "adjacent" else B.SV_ROPE_HALVES,
                                q_stride=qkv.stride(0), k_stride=qkv.stride(0), v_stride=qkv.stride(0))
    return s


def _prepare_window(case, seed, dev):
    s = _batch(case, seed, dev)
    g = _gen(seed, dev)
    shape = (s["pool"], case["Hkv"], case["page"], case["d"])
    s["k_cache"], s["v_cache"] = _normal(shape, case, g, dev), _normal(shape, case, g, dev)
    s["q"] = _normal((s["total"], case["Hq"], case["d"]), case, g, dev)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros((s["total"], case["Hq"]), device=dev)
    if own:
        from paper_2607_25852_amd import binding as B
        attn = B.attn_desc(case["R"], s["total"], case["b"], case["Hq"], case["Hkv"], case["d"], case["page"],
                           s["cols"], s["pool"], int((s["L"] + s["k"]).max()),
                           B.SV_F32 if case["dtype"] == "f32" else B.SV_BF16)
        s["desc"] = B.window_desc(attn, case["window"], case["sinks"])
        s["ws"] = torch.empty(max(B.window_attn_workspace_size(s["desc"]), 256), dtype=torch.uint8, device=dev)
    return s


def _tables(ref, table, dev):
    """Reference counts and page table side by side in one buffer, and a copy a pass works on."""
    n, (R, cols) = len(ref), table.shape
    base = _i32(np.concatenate([ref, table.reshape(-1)]), dev)
    live = base.clone()
    return base, live, live[:n], live[n:].view(R, cols)


def _prepare_step(case, seed, dev):
    R, b, P, pool = case["R"], case["b"], case["page"], case["pool"]
    rng = np.random.default_rng(int(seed))
    perm = _order(R, seed)
    L = np.array(_lengths(case))[perm]
    accepted = np.array([1 + i % b for i in range(R)])[perm]
    cols = -(-(case["ctx_hi"] + b) // P)
    live = _live_columns(L, L, case["window"] or 1 << 30, case["sinks"], P, cols)
    n = int(live.sum())
    ids = rng.permutation(pool)
    table = np.full((R, cols), -1, np.int32)
    table[live] = ids[:n]
    ref = np.zeros(pool, np.int32)
    ref[ids[:max(n, pool * case["fill"] // 1000)]] = 1  # others are held by other batches
    s = dict(case=case, pages=pool, cols=cols, ctx=_i32(L, dev), new=_i32(L + b, dev), kept=_i32(L + accepted, dev))
    s["base"], s["live"], s["ref"], s["table"] = _tables(ref, table, dev)
    _copy_list(s, R, dev)
    if own:
        from paper_2607_25852_amd import binding as B
        s["desc"] = B.pages_desc(R, cols, pool, P)
        s["ws"] = torch.empty(B.reserve_pages_workspace_size(s["desc"]), dtype=torch.uint8, device=dev)
    return s


def _copy_list(s, n, dev):
    z = dict(dtype=torch.int32, device=dev)
    s.update(src=torch.zeros(n, **z), dst=torch.zeros(n, **z), tokens=torch.zeros(n, **z), info=torch.zeros(4, **z))


def _caches(s, case, seed, dev):
    g = _gen(seed, dev)
    shape = (case["layers"], s["pages"], case["Hkv"], case["page"], case["d"])
    s["k_cache"], s["v_cache"] = _normal(shape, case, g, dev), _normal(shape, case, g, dev)


def _prepare_fork(case, seed, dev):
    R, n, b, P = case["R"], case["samples"], case["b"], case["page"]
    L = np.array(_lengths(case))[_order(R, seed)]
    cols = -(-(int(L.max()) + b) // P)
    live = np.arange(cols)[None, :] * P < L[:, None]
    used = int(live.sum())
    pool = used + R * n * (b // P + 2) + 3
    table = np.full((R, cols), -1, np.int32)
    ids = _order(pool, seed)[:used]
    table[live] = ids
    ref = np.zeros(pool, np.int32)
    ref[ids] = 1
    s = dict(case=case, pages=pool, cols=cols, lens=_i32(L, dev), parent=_i32(np.repeat(np.arange(R), n), dev),
             ctx=torch.zeros(R * n, dtype=torch.int32, device=dev), new=_i32(np.repeat(L, n) + b, dev),
             forked=torch.zeros((R * n, cols), dtype=torch.int32, device=dev))
    s["base"], s["live"], s["ref"], s["table"] = _tables(ref, table, dev)
    _copy_list(s, R * n, dev)
    _caches(s, case, seed, dev)
    if own:
        from paper_2607_25852_amd import binding as B
        s["desc"] = B.pages_desc(R * n, cols, pool, P)
        s["cdesc"] = B.copy_desc(R * n, case["layers"], case["Hkv"], case["d"], P, pool,
                                 B.SV_F32 if case["dtype"] == "f32" else B.SV_BF16)
        s["ws"] = torch.empty(B.reserve_pages_workspace_size(s["desc"]), dtype=torch.uint8, device=dev)
    return s


def _compact_rows(case):
    """Columns each request uses; odd requests share the first half of the one before."""
    R, used = case["R"], case["pool"] * case["fill"] // 1000
    cols = max(1, used // R)
    return cols, cols // 2


def _prepare_compact(case, seed, dev):
    R, pool = case["R"], case["pool"]
    cols, shared = _compact_rows(case)
    ids = iter(_order(pool, seed).tolist())
    table = np.full((R, cols + 1), -1, np.int32)
    ref = np.zeros(pool, np.int32)
    for i in range(R):
        for c in range(cols):
            table[i, c] = table[i - 1, c] if i % 2 and c < shared else next(ids)
    np.add.at(ref, table[table >= 0], 1)
    s = dict(case=case, pages=pool, cols=cols + 1)
    s["base"], s["live"], s["ref"], s["table"] = _tables(ref, table, dev)
    _copy_list(s, pool, dev)
    _caches(s, case, seed, dev)
    if own:
        from paper_2607_25852_amd import binding as B
        s["desc"] = B.pages_desc(R, cols + 1, pool, case["page"])
        s["cdesc"] = B.copy_desc(pool, case["layers"], case["Hkv"], case["d"], case["page"], pool,
                                 B.SV_F32 if case["dtype"] == "f32" else B.SV_BF16)
        s["ws"] = torch.empty(B.compact_pages_workspace_size(s["desc"]), dtype=torch.uint8, device=dev)
    return s


PREPARE = dict(rope=_prepare_rope, window=_prepare_window, step=_prepare_step, fork=_prepare_fork,
               compact=_prepare_compact)


def prepare(case, seed):
    return PREPARE[case["op"]](case, int(seed), torch.device("cuda"))


# ---------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------
def _own_rope(s):
    from paper_2607_25852_amd import binding as B
    B.rope_append(s["desc"], s["q"], s["k_new"], s["v_new"], s["positions"], s["inv_freq"], s["table"], s["qo"],
                  s["ctx"], s["q_out"], s["k_cache"], s["v_cache"])
    return s["q_out"], s["k_cache"], s["v_cache"]


def _own_window(s):
    from paper_2607_25852_amd import binding as B
    B.window_attn(s["desc"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["qo"], s["kv_lens"], s["out"],
                  s["lse"], s["ws"])
    return s["out"], s["lse"]


def _own_step(s):
    from paper_2607_25852_amd import binding as B
    s["live"].copy_(s["base"])  # a pass starts from the same tables; a program carries them on
    B.reserve_pages(s["desc"], s["table"], s["ref"], s["ctx"], s["new"], s["src"], s["dst"], s["tokens"], s["info"],
                    s["ws"])
    B.release_pages(s["desc"], s["table"], s["ref"], s["kept"], s["case"]["window"], s["case"]["sinks"])
    return s["table"], s["ref"], s["info"]


def _own_fork(s):
    from paper_2607_25852_amd import binding as B
    s["live"].copy_(s["base"])
    B.fork_pages(s["desc"], s["case"]["R"], s["table"], s["lens"], s["parent"], s["forked"], s["ctx"], s["ref"])
    B.reserve_pages(s["desc"], s["forked"], s["ref"], s["ctx"], s["new"], s["src"], s["dst"], s["tokens"], s["info"],
                    s["ws"])
    B.copy_pages(s["cdesc"], s["src"], s["dst"], s["info"][2:3], s["k_cache"], s["v_cache"], s["tokens"])
    return (s["forked"], s["ref"], s["ctx"], s["src"], s["dst"], s["tokens"], s["info"], s["k_cache"], s["v_cache"])


def _own_compact(s):
    from paper_2607_25852_amd import binding as B
    s["live"].copy_(s["base"])
    B.compact_pages(s["desc"], 0, s["table"], s["ref"], s["src"], s["dst"], s["info"], s["ws"])
    B.copy_pages(s["cdesc"], s["src"], s["dst"], s["info"][:1], s["k_cache"], s["v_cache"])
    return s["table"], s["ref"], s["src"], s["dst"], s["info"][:2], s["k_cache"], s["v_cache"]


OWN = dict(rope=_own_rope, window=_own_window, step=_own_step, fork=_own_fork, compact=_own_compact)


# ---------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------
def _rotate(x, cos, sin, pairing):
    n = cos.shape[-1]
    a, b = (x[..., :n], x[..., n:2 * n]) if pairing == "halves" else (x[..., :2 * n:2], x[..., 1:2 * n:2])
    u, v = a * cos - b * sin, b * cos + a * sin
    both = torch.cat([u, v], -1) if pairing == "halves" else torch.stack([u, v], -1).flatten(-2)
    return torch.cat([both, x[..., 2 * n:]], -1)


def _plain_rope(s):
    case, K = s["case"], s["K"]
    ang = s["positions"][s["axis"], :K].t().double() * s["inv_freq"]  # far positions: the angle in 64 bits
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    s["q_out"][:K] = _rotate(s["q"][:K].float(), cos, sin, case["pairing"]).to(s["q"].dtype)
    k = _rotate(s["k_new"][:K].float(), cos, sin, case["pairing"]).to(s["q"].dtype)
    row = torch.arange(K, device=k.device)
    req = torch.searchsorted(s["qo"][1:], row, right=True)
    at = s["ctx"][req] + row - s["qo"][req]
    page, slot = s["table"][req, at // case["page"]].long(), (at % case["page"]).long()
    s["k_cache"][page, :, slot] = k
    s["v_cache"][page, :, slot] = s["v_new"][:K]
    return s["q_out"], s["k_cache"], s["v_cache"]


def _plain_window(s):
    case = s["case"]
    R, b, Hq, Hkv, d, P = (case[k] for k in ("R", "b", "Hq", "Hkv", "d", "page"))
    W, S, G = case["window"], case["sinks"], case["Hq"] // case["Hkv"]
    dev = s["q"].device
    W = min(W, int(s["kv_lens"].max()))
    T = S + W + b - 1
    some = max(1, (1 << 28) // (Hkv * T * max(d, G * b)))
    j = torch.arange(b, device=dev)
    for i in range(0, R, some):
        n = min(some, R - i)
        L, k = s["ctx"][i:i + n, None].long(), (s["qo"][i + 1:i + n + 1] - s["qo"][i:i + n])[:, None]
        lo = (L - W + 1).clamp(min=0)
        at = torch.cat([torch.arange(S, device=dev).expand(n, S), lo + torch.arange(W + b - 1, device=dev)], 1)
        first = (torch.arange(T, device=dev) < S)[None]  # the sinks' columns; the others begin at lo
        known = (at < L + k) & (~first | (at < lo))
        pos = (L + j)[:, :, None]
        seen = known[:, None] & (at[:, None] <= pos) & ((at[:, None] < S) | (at[:, None] > pos - W))  # [n, b, T]
        page = s["table"][i:i + n].gather(1, (at // P).clamp(max=s["cols"] - 1)).long()
        page, slot = page.clamp(min=0), at % P
        keys = s["k_cache"][page, :, slot].float().transpose(1, 2)    # [n, Hkv, T, d]
        vals = s["v_cache"][page, :, slot].float().transpose(1, 2).contiguous()
        rows = (s["qo"][i:i + n, None] + j).clamp(max=s["total"] - 1).long()  # [n, b]
        q = s["q"][rows].float().view(n, b, Hkv, G, d).permute(0, 2, 1, 3, 4).reshape(n, Hkv, b * G, d)
        z = torch.matmul(q, keys.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
        z = z.view(n, Hkv, b, G, T).masked_fill_(~seen[:, None, :, None], -math.inf)
        m = z.amax(-1, keepdim=True).clamp(min=-1e30)
        p = torch.exp(z - m)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.view(n, Hkv, b * G, T), vals).view(n, Hkv, b, G, d) / total
        use = (j < k)
        o = o.permute(0, 2, 1, 3, 4).reshape(n, b, Hq, d)[use]
        lse = (m + torch.log(total)).squeeze(-1).permute(0, 2, 1, 3).reshape(n, b, Hq)[use]
        s["out"][rows[use]] = o.to(s["out"].dtype)
        s["lse"][rows[use]] = lse
    return s["out"], s["lse"]


def _plain_reserve(s, table, ctx, new):
    P, cols, dev = s["case"]["page"], s["cols"], table.device
    ref = s["ref"]
    R = table.shape[0]
    c = torch.arange(cols, device=dev)
    inside = (c >= (ctx // P)[:, None]) & (c * P < new[:, None]) & (new > ctx)[:, None]
    pg = table.long()
    held = inside & (pg >= 0)
    shared = held & (ref[pg.clamp(min=0)] > 1)
    # of the entries that want to write a shared page, all but the last may have to leave it
    entry = torch.nonzero(shared.view(-1)).view(-1)
    page = pg.view(-1)[entry]
    writers = torch.zeros(s["pages"], dtype=torch.int64, device=dev).index_add_(0, page, torch.ones_like(page))
    last = torch.full_like(writers, -1).scatter_reduce_(0, page, entry, "amax")
    leave = shared.clone()
    leave.view(-1)[entry] = (writers[page] != ref[page]) | (last[page] != entry)
    want = (inside & ~held) | leave
    need = want.sum(1)
    upto = need.cumsum(0)
    free = torch.nonzero(ref == 0).view(-1)
    served = (upto <= free.numel()).long().cumprod(0).bool()
    want, leave = want & served[:, None], leave & served[:, None]
    rank = want.view(-1).cumsum(0) - 1
    take = free[rank.clamp(min=0, max=max(free.numel() - 1, 0))].view(R, cols) if free.numel() else torch.zeros_like(pg)
    part = leave & (c == (ctx // P)[:, None]) & (ctx % P > 0)[:, None]
    row = torch.nonzero(part.any(1)).view(-1)
    n = row.numel()
    s["src"][:n] = table[part]
    s["dst"][:n] = take[part].int()
    s["tokens"][:n] = (ctx % P)[row]
    ref.index_add_(0, pg[leave], torch.full_like(pg[leave], -1).int())
    ref[take[want]] = 1
    table.copy_(torch.where(want, take.int(), table))
    taken = want.sum()
    s["info"].copy_(torch.stack([served.sum(), taken, part.sum(), free.numel() - taken]))


def _plain_step(s):
    case = s["case"]
    P, W, S = case["page"], case["window"], case["sinks"]
    s["live"].copy_(s["base"])
    _plain_reserve(s, s["table"], s["ctx"], s["new"])
    n = s["kept"][:, None]
    c = torch.arange(s["cols"], device=n.device)
    stay = c * P < n
    if W:
        stay = stay & ((c * P < S) | ((c + 1) * P > n - W + 1))
    drop = ~stay & (s["table"] >= 0)
    gone = s["table"][drop].long()
    s["ref"].index_add_(0, gone, torch.full_like(gone, -1).int())
    s["table"].masked_fill_(drop, -1)
    return s["table"], s["ref"], s["info"]


def _plain_fork(s):
    P, dev = s["case"]["page"], s["ref"].device
    s["live"].copy_(s["base"])
    parent = s["parent"].long()
    s["ctx"].copy_(s["lens"][parent])
    old = s["table"]
    c = torch.arange(s["cols"], device=dev)
    s["forked"].copy_(torch.where(c * P < s["ctx"][:, None], old[parent], -1))
    for t, by in ((s["forked"], 1), (old, -1)):
        p = t[t >= 0].long()
        s["ref"].index_add_(0, p, torch.full_like(p, by).int())
    _plain_reserve(s, s["forked"], s["ctx"], s["new"])
    n = int(s["info"][2])
    src, dst = s["src"][:n].long(), s["dst"][:n].long()
    rows = (torch.arange(P, device=dev) < s["tokens"][:n, None])[None, :, None, :, None]
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, dst] = torch.where(rows, cache[:, src], cache[:, dst])
    return (s["forked"], s["ref"], s["ctx"], s["src"], s["dst"], s["tokens"], s["info"], s["k_cache"], s["v_cache"])


def _plain_compact(s):
    s["live"].copy_(s["base"])
    ref, table = s["ref"], s["table"]
    hole = torch.nonzero(ref == 0).view(-1)
    live = torch.nonzero(ref > 0).view(-1).flip(0)
    n = min(hole.numel(), live.numel())
    moves = int((hole[:n] < live[:n]).sum())
    hole, live = hole[:moves], live[:moves]
    s["src"][:moves], s["dst"][:moves] = live.int(), hole.int()
    s["info"][0], s["info"][1] = moves, (ref > 0).sum()
    to = torch.arange(s["pages"], device=ref.device)
    to[live] = hole
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), table))
    ref[hole] = ref[live]
    ref[live] = 0
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, hole] = cache[:, live]
    return table, ref, s["src"], s["dst"], s["info"][:2], s["k_cache"], s["v_cache"]


PLAIN = dict(rope=_plain_rope, window=_plain_window, step=_plain_step, fork=_plain_fork, compact=_plain_compact)


def run(state):
    return (OWN if own else PLAIN)[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------
# work: every input once, every output once
# ---------------------------------------------------------------------------------------
def work(case):
    op = case["op"]
    if op in ("rope", "window"):
        k, L = _depths(case), _lengths(case)
        K, Hq, Hkv, d, esz = sum(k), case["Hq"], case["Hkv"], case["d"], _esz(case)
        if op == "rope":
            return dict(bytes=K * ((2 * Hq + 4 * Hkv) * d * esz + 4 * len(_sections(case))) + 8 * sum(_sections(case)),
                        flops=K * (Hq + Hkv) * 6 * sum(_sections(case)))
        seen = [_seen(x, n, case["window"], case["sinks"]) for x, n in zip(L, k)]
        return dict(bytes=sum(t for t, _ in seen) * Hkv * 2 * d * esz + K * Hq * (2 * d * esz + 4),
                    flops=sum(p for _, p in seen) * Hq * 4 * d)
    if op == "step":
        # counts read, the round's columns and counts written
        return dict(bytes=4 * case["pool"] + case["R"] * 4 * (3 + 4 * (case["b"] // case["page"] + 2)), flops=0)
    page = case["Hkv"] * case["d"] * _esz(case)  # bytes of a token in one cache and layer
    if op == "fork":
        n, P, L = case["samples"], case["page"], _lengths(case)
        entries = sum(-(-x // P) for x in L)
        rows = sum(x % P for x in L) * (n - 1)
        return dict(bytes=4 * (1 + n) * entries + 8 * entries + rows * page * 2 * 2 * case["layers"], flops=0)
    pool, R = case["pool"], case["R"]
    cols, shared = _compact_rows(case)
    live = R * cols - (R // 2) * shared
    moves = live * (pool - live) // pool  # of random ids: free ones below `live`
    return dict(bytes=8 * pool + 8 * R * cols + moves * page * case["page"] * 2 * 2 * case["layers"], flops=0)


# ---------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_rope(case, s):
    K, P, n = s["K"], case["page"], sum(_sections(case))
    pos, f = s["positions"].double(), s["inv_freq"].double()
    q_out, kc, vc = (s[x].double() for x in ("q_out", "k_cache", "v_cache"))
    turned = {}
    for name in ("q", "k_new"):
        x = s[name][:K].double()
        y = x.clone()
        for p, a in enumerate(_axis(case)):
            i, j = (p, p + n) if case["pairing"] == "halves" else (2 * p, 2 * p + 1)
            t = (pos[a, :K] * f[p])[:, None]
            y[:, :, i] = x[:, :, i] * torch.cos(t) - x[:, :, j] * torch.sin(t)
            y[:, :, j] = x[:, :, i] * torch.sin(t) + x[:, :, j] * torch.cos(t)
        turned[name] = y
    q_out[:K] = turned["q"]
    table, r = s["table"].cpu().numpy(), 0
    for i in range(case["R"]):
        at = np.arange(s["L"][i], s["L"][i] + s["k"][i])
        page, slot = torch.tensor(table[i, at // P], device=kc.device).long(), torch.tensor(at % P, device=kc.device)
        kc[page, :, slot] = turned["k_new"][r:r + len(at)]
        vc[page, :, slot] = s["v_new"][r:r + len(at)].double()
        r += len(at)
    return q_out, kc, vc


def _exact_window(case, s):
    Hq, Hkv, d, P, W, S = (case[k] for k in ("Hq", "Hkv", "d", "page", "window", "sinks"))
    G = Hq // Hkv
    out, lse = s["out"].double(), s["lse"].double()
    table, r = s["table"].cpu().numpy(), 0
    for i in range(case["R"]):
        L, k = int(s["L"][i]), int(s["k"][i])
        lo = max(0, L - W + 1)
        at = np.concatenate([np.arange(min(S, lo)), np.arange(lo, L + k)])
        page = torch.tensor(table[i, at // P], device=out.device).long()
        slot, key = torch.tensor(at % P, device=out.device), torch.tensor(at, device=out.device)
        K = s["k_cache"][page, :, slot].double()  # [T, Hkv, d]
        V = s["v_cache"][page, :, slot].double()
        p = torch.arange(L, L + k, device=out.device)[:, None]
        hide = ~((key <= p) & ((key < S) | (key > p - W)))
        for h in range(Hkv):
            q = s["q"][r:r + k, h * G:(h + 1) * G].double()  # [k, G, d]
            z = (q.reshape(k * G, d) @ K[:, h].t()).view(k, G, -1) / math.sqrt(d)
            z.masked_fill_(hide[:, None], -math.inf)
            l = torch.logsumexp(z, -1)
            lse[r:r + k, h * G:(h + 1) * G] = l
            out[r:r + k, h * G:(h + 1) * G] = (torch.exp(z - l[..., None]).view(k * G, -1) @ V[:, h]).view(k, G, d)
        r += k
    return out, lse


def _exact_reserve(table, ref, ctx, new, P):
    """Request after request, column after column."""
    src, dst, tokens = [], [], []
    served = taken = 0
    free = [p for p in range(len(ref)) if ref[p] == 0]
    total = len(free)
    for i in range(len(ctx)):
        columns = range(ctx[i] // P, -(-new[i] // P)) if new[i] > ctx[i] else ()
        need = [c for c in columns if table[i][c] < 0 or ref[table[i][c]] > 1]
        if len(need) > len(free):
            break
        for c in need:
            old, page = table[i][c], free.pop(0)
            if old >= 0:
                ref[old] -= 1
                if c == ctx[i] // P and ctx[i] % P:
                    src.append(old), dst.append(page), tokens.append(ctx[i] % P)
            table[i][c], ref[page] = page, 1
        served, taken = served + 1, taken + len(need)
    return src, dst, tokens, [served, taken, len(src), total - taken]


def _padded(x, like):
    out = like.clone()
    out[:len(x)] = torch.tensor(x, dtype=torch.int32, device=like.device)
    return out


def _exact_step(case, s):
    P, W, S = case["page"], case["window"], case["sinks"]
    table, ref = s["table"].tolist(), s["ref"].tolist()
    *_, info = _exact_reserve(table, ref, s["ctx"].tolist(), s["new"].tolist(), P)
    for i, n in enumerate(s["kept"].tolist()):
        for c, page in enumerate(table[i]):
            dead = c * P >= n or (W and c * P >= S and (c + 1) * P <= n - W + 1)
            if page >= 0 and dead:
                ref[page] -= 1
                table[i][c] = -1
    return _padded(table, s["table"]), _padded(ref, s["ref"]), _padded(info, s["info"])


def _exact_fork(case, s):
    P = case["page"]
    old, ref, lens = s["table"].tolist(), s["ref"].tolist(), s["lens"].tolist()
    table, ctx = [], []
    for p in s["parent"].tolist():
        used = -(-lens[p] // P)
        table.append(old[p][:used] + [-1] * (s["cols"] - used))
        ctx.append(lens[p])
    for rows, by in ((table, 1), (old, -1)):
        for row in rows:
            for page in row:
                if page >= 0:
                    ref[page] += by
    src, dst, tokens, info = _exact_reserve(table, ref, ctx, s["new"].tolist(), P)
    kc, vc = s["k_cache"].clone(), s["v_cache"].clone()
    for a, b, n in zip(src, dst, tokens):
        kc[:, b, :, :n] = s["k_cache"][:, a, :, :n]
        vc[:, b, :, :n] = s["v_cache"][:, a, :, :n]
    return (_padded(table, s["forked"]), _padded(ref, s["ref"]), _padded(ctx, s["ctx"]), _padded(src, s["src"]),
            _padded(dst, s["dst"]), _padded(tokens, s["tokens"]), _padded(info, s["info"]), kc, vc)


def _exact_compact(case, s):
    table, ref = s["table"].tolist(), s["ref"].tolist()
    n = sum(1 for x in ref if x > 0)
    low, high, moved = 0, len(ref) - 1, {}
    while True:
        while low < len(ref) and ref[low] != 0:
            low += 1
        while high >= 0 and ref[high] == 0:
            high -= 1
        if low >= high:
            break
        ref[low], ref[high], moved[high] = ref[high], 0, low
    table = [[moved.get(p, p) for p in row] for row in table]
    kc, vc = s["k_cache"].clone(), s["v_cache"].clone()
    a, b = list(moved), list(moved.values())
    kc[:, b], vc[:, b] = s["k_cache"][:, a], s["v_cache"][:, a]
    return (_padded(table, s["table"]), _padded(ref, s["ref"]), _padded(a, s["src"]), _padded(b, s["dst"]),
            _padded([len(a), n], s["info"][:2]), kc, vc)


EXACT = dict(rope=_exact_rope, window=_exact_window, step=_exact_step, fork=_exact_fork, compact=_exact_compact)


def exact(case, seed):
    return EXACT[case["op"]](case, prepare(case, seed))
