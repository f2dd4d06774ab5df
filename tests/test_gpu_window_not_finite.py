"""sv_window_attn where keys and values are not finite, or so large that scores are far from 0.

Rows that do not see such a key give the same bits as without it, in every division of the work; rows that do see
it are compared with the definition in 64 bits: NaN and infinities where it has them, the other elements within
cache_reference.window_tolerance."""
import numpy as np
import pytest

import cache_reference as ref
from gpu_util import say
from test_gpu_window import call, dev, make  # noqa: F401 (dev is a fixture)

pytestmark = pytest.mark.gpu

f64 = lambda t: t.double().cpu().numpy()  # noqa: E731


def slot(s, i, p):
    return int(s["table"][i, p // s["page"]]), p % s["page"]


def sees(s, i, keys):
    """[rows of request i]: whether the row sees one of the keys"""
    k = int(s["qo"][i + 1] - s["qo"][i])
    p = int(s["kv"][i]) - k + np.arange(k)[:, None]
    keys = np.array(keys)[None, :]
    return ((keys <= p) & ((keys < s["sinks"]) | (keys > p - s["window"]))).any(1)


def definition(s, r, i, head):
    """Row r of request i: out [d], lse, the weighted sums of finite |V|, the largest sum of |q||K|, keys. A key whose score is
    -inf has no weight."""
    k, n = int(s["qo"][i + 1] - s["qo"][i]), int(s["kv"][i])
    p = n - k + r - int(s["qo"][i])
    keys = np.arange(p + 1)
    keys = keys[(keys < s["sinks"]) | (keys > p - s["window"])]
    pg, at, h = s["table"][i, keys // s["page"]], keys % s["page"], head // (s["Hq"] // s["Hkv"])
    K, V, q = s["k64"][pg, h, at], s["v64"][pg, h, at], s["q64"][r, head]
    z = K @ q / np.sqrt(s["d"])
    if np.isnan(z).any() or (z == np.inf).any():
        return np.full(s["d"], np.nan), np.nan, np.zeros(s["d"]), 0.0, len(keys)
    use = z > -np.inf
    K, V, z = K[use], V[use], z[use]
    lse = z.max() + np.log(np.exp(z - z.max()).sum())
    w = np.exp(z - lse)[:, None]
    return ((w * V).sum(0), lse, (w * np.abs(np.where(np.isfinite(V), V, 0))).sum(0),
            (np.abs(K) @ np.abs(q)).max() / np.sqrt(s["d"]), len(keys))


def compare(s, touched, clean):
    """touched [total]: rows that see a changed key. The others keep the bits of `clean`."""
    out, lse = call(s)
    rows = ~touched
    assert bool((out[rows] == clean[0][rows]).all()) and bool((lse[rows] == clean[1][rows]).all())
    s.update(k64=f64(s["kc"]), v64=f64(s["vc"]), q64=f64(s["q"]))
    with np.errstate(invalid="ignore"):
        for r in np.nonzero(touched)[0]:
            i = int(np.searchsorted(s["qo"], r, side="right")) - 1
            for head in (0, s["Hq"] - 1):
                eo, el, absv, absz, count = definition(s, r, i, head)
                tol, tol_l = ref.window_tolerance(s["dtype"], s["d"], np.where(np.isfinite(eo), eo, 0)[None, None],
                                                  np.array([[el]]), absv[None, None], np.array([[absz]]), np.array([count]))
                for got, want, t in ((f64(out[r, head]), eo, tol[0, 0]), (f64(lse[r, head]), np.float64(el), tol_l[0, 0])):
                    same = (got == want) | (np.isnan(got) & np.isnan(want))
                    good = same | (np.isfinite(want) & (np.abs(got - want) <= t))
                    assert good.all(), (int(r), head, got[~good][:3], want[~good][:3])


# up to 32 rows on four waves, two waves per 32 rows, whole-tile waves, eight waves, fp32 of 16 and of 32 rows; whole
# lists and splits of a tile
LAYOUTS = [
    ("bf16", 4, 2, 64, 16, [16, 3], 0), ("bf16", 8, 4, 128, 64, [16, 5], 0), ("bf16", 8, 2, 64, 16, [16, 3], 64),
    ("bf16", 8, 2, 128, 64, [16, 5], 64), ("bf16", 32, 4, 128, 2, [16, 9], 0), ("bf16", 16, 2, 64, 1, [16, 9], 64),
    ("bf16", 16, 1, 128, 64, [16, 4], 0), ("bf16", 16, 1, 64, 32, [16, 4], 64), ("bf16", 16, 1, 128, 16, [16, 4], 64),
    ("f32", 4, 2, 64, 16, [16, 3], 0), ("f32", 8, 1, 128, 64, [16, 5], 64), ("f32", 3, 1, 100, 8, [7, 16], 0),
    ("f32", 2, 1, 256, 16, [16, 2], 64), ("f32", 6, 2, 36, 1, [5, 16], 64)]


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("dtype,Hq,Hkv,d,page,k,split", LAYOUTS)
def test_rows_that_do_not_see_it_keep_their_bits(dev, dtype, Hq, Hkv, d, page, k, split, what):  # noqa: F811
    say("window not finite", dtype, Hq, Hkv, d, page, split, what)
    s = make(dev, 41, k, [330, 290], Hq, Hkv, d, page, dtype, 200, 3)
    s["split"] = split
    clean = call(s)
    first, last = int(s["kv"][0]) - k[0], int(s["kv"][0]) - 1
    # keys of the last row alone, of the first alone, several of either kind
    for keys in ([last], [first - 199], [last - 1, last, first - 198], list(range(first + 1, last + 1))):
        touched = np.zeros(s["total"], bool)
        touched[:k[0]] = sees(s, 0, keys)
        assert touched.any() and not touched[:k[0]].all()
        for name, dims in (("vc", [d - 1]), ("vc", [0, d // 2 + 1]), ("vc", slice(None)), ("kc", [1])):
            keep = s[name].clone()
            for p in keys:
                pg, at = slot(s, 0, p)
                s[name][pg, :, at, dims] = what
            compare(s, touched, clean)
            s[name] = keep


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq", [2, 8, 16])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (4, 0), (5, 70), (16, 2), (17, 0), (1000, 0), (3, 500)])
@pytest.mark.parametrize("ctx", [0, 1, 60, 130])
def test_windows_shorter_than_a_block(dev, dtype, Hq, window, sinks, ctx):  # noqa: F811
    """Every key in turn that some rows of the block see, and all second ones; short requests among the first tokens."""
    say("window not finite, short", dtype, Hq, window, sinks, ctx)
    s = make(dev, 44, [16, 2], [ctx, 40], Hq, 1, 64, 16, dtype, window, sinks)
    clean = call(s)
    keep = s["vc"].clone()
    lo = max(0, ctx - window + 1)
    for keys in [[lo], [ctx], [ctx + 3], [ctx + 15], list(range(lo % 2, ctx + 16, 2))]:
        touched = np.zeros(s["total"], bool)
        touched[:16] = sees(s, 0, keys)
        for p in keys:
            if s["table"][0, p // 16] >= 0 and (p < sinks or p > ctx - window):
                pg, at = slot(s, 0, p)
                s["vc"][pg, :, at, 5] = float("inf")
        compare(s, touched, clean)
        s["vc"].copy_(keep)


@pytest.mark.parametrize("dtype,Hq,Hkv,d,page,k,split", LAYOUTS)
def test_a_value_that_all_rows_see(dev, dtype, Hq, Hkv, d, page, k, split):  # noqa: F811
    """In the first, a middle and the last part of a list, with those that only some rows see beside it."""
    say("window not finite, all rows", dtype, Hq, Hkv, d, page, split)
    s = make(dev, 42, k, [330, 290], Hq, Hkv, d, page, dtype, 200, 3)
    s["split"] = split
    clean = call(s)
    first, last = int(s["kv"][1]) - k[1], int(s["kv"][1]) - 1
    touched = np.zeros(s["total"], bool)
    touched[int(s["qo"][1]):int(s["qo"][2])] = True
    for p in (1, last - 199, first - 100, first):
        for what, dim in ((float("inf"), 2), (float("nan"), d - 2)):
            pg, at = slot(s, 1, p)
            keep = s["vc"].clone()
            s["vc"][pg, :, at, dim] = what
            pg, at = slot(s, 1, last)
            s["vc"][pg, :, at, dim] = what
            compare(s, touched, clean)
            s["vc"] = keep


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,k", [(2, [3, 1]), (8, [16, 4]), (16, [16, 4])])
@pytest.mark.parametrize("power", [10, 20, 26, 27, 28, 29, 30, 31, 32])  # (from 2^40 on the oracle's own lse is off by more than an fp32 result)
def test_scores_far_from_zero(dev, dtype, Hq, k, power):  # noqa: F811
    """Scores of a small whole number times a power of two, of one product each, so they are exact: the keys with the largest
    share the weight evenly. Whole lists: the partial results of splits carry their weight in an fp32 lse, which cannot
    hold it beside scores of this size. lse: the scale's, its product's and the change of base's roundings, 8 half steps."""
    say("window far scores", dtype, Hq, power)
    torch = dev
    for sign in (1.0, -1.0):
        s = make(dev, 43, k, [150, 90], Hq, 1, 64, 16, dtype, 100, 2)
        s["split"] = 1 << 20
        g = torch.Generator().manual_seed(power)
        s["q"].zero_()
        s["kc"].zero_()
        s["q"][:, :, 7] = sign * 2.0 ** (power // 2)
        s["kc"][..., 7] = (torch.randint(1, 6, s["kc"].shape[:3], generator=g) * 2.0 ** (power - power // 2)).to(s["kc"])
        out, lse = (f64(x) for x in call(s))
        eo, el, absv, absz, count, defined = ref.window_attention(
            f64(s["q"]), f64(s["kc"]), f64(s["vc"]), s["table"], s["qo"], s["kv"], s["window"], s["sinks"], s["block"],
            s["max_kv"])
        use = defined & (count > 0)
        tol, _ = ref.window_tolerance(dtype, 64, eo, el, absv, np.zeros_like(absz), count)
        assert (np.abs(out - eo) <= tol)[use].all(), float(np.abs(out - eo)[use].max())
        assert (np.abs(lse - el) <= 8 * ref.F32_HALF * np.abs(el) + 2.0 ** -18)[use].all()
