"""Plain 64-bit definitions of the paged cache's operators (numpy loops), and inputs for their tests."""
import numpy as np

BF16_HALF, F32_HALF = 2.0 ** -8, 2.0 ** -24  # half a step, relative to the value


def half_step(dtype):
    return BF16_HALF if dtype == "bf16" else F32_HALF


def axes_of(sections, order):
    """Position axis of each rotated pair."""
    if order == "blocks":
        return [a for a, n in enumerate(sections) for _ in range(n)]
    n = len(sections)
    return [p % n if p // n < sections[p % n] else 0 for p in range(sum(sections))]


def rotate(x, positions, inv_freq, sections, order, pairing, scale=1.0):
    """x [rows, heads, d] float64, positions [axes, rows]: the rotated rows, and for each element the sum of
    the absolute products (what the fp32 rounding errors are relative to)."""
    y, mag = x.copy(), np.zeros_like(x)
    n = sum(sections)
    for p, a in enumerate(axes_of(sections, order)):
        i, j = (p, p + n) if pairing == "halves" else (2 * p, 2 * p + 1)
        t = positions[a].astype(np.float64) * inv_freq[p]
        c, s = np.cos(t)[:, None] * scale, np.sin(t)[:, None] * scale
        y[:, :, i] = x[:, :, i] * c - x[:, :, j] * s
        y[:, :, j] = x[:, :, j] * c + x[:, :, i] * s
        mag[:, :, i] = mag[:, :, j] = (np.abs(x[:, :, i]) + np.abs(x[:, :, j])) * abs(scale)
    return y, mag


def rope_slots(qo, ctx, table, page, num_pages, total):
    """(rows of sound requests, [(row, page, slot)] of those whose slot exists)"""
    rows, slots = [], []
    for i in range(len(ctx)):
        q0, q1 = int(qo[i]), int(qo[i + 1])
        if not (0 <= q0 < q1 <= total):
            continue
        for r in range(q0, q1):
            rows.append(r)
            s = int(ctx[i]) + r - q0
            if ctx[i] < 0 or s // page >= table.shape[1]:
                continue
            pg = int(table[i, s // page])
            if 0 <= pg < num_pages:
                slots.append((r, pg, s % page))
    return rows, slots


def window_attention(q, kc, vc, table, qo, kv_lens, window, sinks, block, max_kv_len, scale=None):
    """float64 arrays: q [total, Hq, d], caches [pages, Hkv, P, d]. Returns out, lse, the weighted sum of |V|,
    the largest sum of |q||K| of a row's keys, the keys of a row, and which rows are defined."""
    total, Hq, d = q.shape
    pages, Hkv, P, _ = kc.shape
    G = Hq // Hkv
    scale = scale or 1.0 / np.sqrt(d)
    out, lse = np.zeros_like(q), np.full((total, Hq), -np.inf)
    absv, absz, count = np.zeros_like(q), np.zeros((total, Hq)), np.zeros(total, int)
    defined = np.zeros(total, bool)
    for i in range(len(kv_lens)):
        q0, k = int(qo[i]), int(qo[i + 1]) - int(qo[i])
        n = min(int(kv_lens[i]), max_kv_len)
        if not (1 <= k <= block and q0 >= 0 and q0 + k <= total and n >= k):
            continue
        for j in range(k):
            p, r = n - k + j, q0 + j
            defined[r] = True
            s = np.arange(p + 1)
            s = s[(s < sinks) | (s > p - window)]
            col = s // P
            s, col = s[col < table.shape[1]], col[col < table.shape[1]]
            pg = table[i, col]
            ok = (pg >= 0) & (pg < pages)
            s, pg = s[ok], pg[ok]
            count[r] = len(s)
            if not len(s):
                continue
            for h in range(Hkv):
                K, V = kc[pg, h, s % P], vc[pg, h, s % P]
                for head in range(h * G, (h + 1) * G):
                    z = scale * (K @ q[r, head])
                    m = z.max()
                    lse[r, head] = m + np.log(np.exp(z - m).sum())
                    w = np.exp(z - lse[r, head])
                    out[r, head] = w @ V
                    absv[r, head] = w @ np.abs(V)
                    absz[r, head] = scale * (np.abs(K) @ np.abs(q[r, head])).max()
    return out, lse, absv, absz, count, defined


def window_tolerance(dtype, d, out, lse, absv, absz, count):
    """Bounds of |out - exact| and |lse - exact|. A score is a sum of d products in fp32: (d + 8) half steps
    of the sum of their absolute values (8: the scale, the maximum's subtraction, the exponential). The sum
    of n weights, the products with V and the merges of partial sums: (n + 64) half steps. In bf16 each
    weight is rounded before it meets V, and the result is rounded once."""
    dz = (d + 8) * F32_HALF * (absz + 1) + 2.0 ** -20
    n = (count + 64)[:, None] * F32_HALF
    tol = (2 * dz + 2 * n)[:, :, None] * absv + half_step(dtype) * np.abs(out)
    if dtype == "bf16":
        tol = tol + 1.01 * BF16_HALF * absv
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return tol + 1e-30, dz + n + 4 * F32_HALF * (finite + 1)


def fork(table, ref, lens, parent, page):
    ref = ref.copy()
    out = np.full((len(parent), table.shape[1]), -1, np.int32)
    lens_out = np.zeros(len(parent), np.int32)
    for i, p in enumerate(parent):
        if 0 <= p < len(table):
            lens_out[i] = max(lens[p], 0)
            used = -(-int(lens_out[i]) // page)
            out[i, :used] = table[p, :used]
    np.add.at(ref, out[out >= 0], 1)
    np.add.at(ref, table[table >= 0], -1)
    return out, ref, lens_out


def reserve(table, ref, ctx, new, page):
    table, ref = table.copy(), ref.copy()
    free = [p for p in range(len(ref)) if ref[p] == 0]
    copies, served, taken = [], 0, 0
    for i in range(len(ctx)):
        c, n = int(ctx[i]), int(new[i])
        columns = range(c // page, -(-n // page)) if n > c else range(0)
        if c < 0 or columns.stop > table.shape[1]:
            break
        need = [x for x in columns if table[i, x] < 0 or ref[table[i, x]] > 1]
        if len(need) > len(free) - taken:
            break
        for x in need:
            old, pg = table[i, x], free[taken]
            if old >= 0:
                ref[old] -= 1
                if x == c // page and c % page:
                    copies.append((old, pg, c % page))
            table[i, x], ref[pg] = pg, 1
            taken += 1
        served += 1
    return table, ref, copies, [served, taken, len(copies), len(free) - taken]


def release(table, ref, lens, page, window=0, sinks=0):
    table, ref = table.copy(), ref.copy()
    for i in range(len(table)):
        for c in range(table.shape[1]):
            first, past, n = c * page, (c + 1) * page, int(lens[i])
            if first >= n or (window and first >= sinks and past - 1 <= n - window):
                if table[i, c] >= 0:
                    ref[table[i, c]] -= 1
                table[i, c] = -1
    return table, ref


def compact(table, ref, max_moves=0):
    ref = ref.copy()
    live, moves = int((ref > 0).sum()), []
    lo, hi = 0, len(ref) - 1
    while not max_moves or len(moves) < max_moves:
        while lo < len(ref) and ref[lo] > 0:
            lo += 1
        while hi >= 0 and ref[hi] == 0:
            hi -= 1
        if lo >= hi:
            break
        ref[lo], ref[hi] = ref[hi], 0
        moves.append((hi, lo))
    to = np.arange(len(ref), dtype=np.int32)
    for s, d in moves:
        to[s] = d
    table = table.copy()
    table[table >= 0] = to[table[table >= 0]]
    return table, ref, moves, live


def random_tables(rng, R, cols, page, pages, share=0.4, others=0.3):
    """A consistent page table with shared prefixes, its counts and its lengths."""
    ids = rng.permutation(pages)
    table, ref = np.full((R, cols), -1, np.int32), np.zeros(pages, np.int32)
    lens, used = rng.integers(0, cols * page + 1, R).astype(np.int32), 0
    for i in range(R):
        near = rng.integers(0, i) if i and rng.random() < share else -1
        for c in range(-(-int(lens[i]) // page)):
            pg = table[near, c] if near >= 0 else -1
            if pg < 0:
                if used == pages:
                    lens[i] = c * page
                    break
                pg, used = ids[used], used + 1
            table[i, c] = pg
            ref[pg] += 1
    extra = int((pages - used) * others)
    ref[ids[used:used + extra]] = 1
    return table, ref, lens
