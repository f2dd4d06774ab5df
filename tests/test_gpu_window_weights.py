"""sv_window_attn in bf16: the weights' precision. Keys, values and queries are bf16 and their products exact in fp32, so
against 64 bits only fp32 sums, the weights' two bf16 parts and the result's own rounding are left.

Tolerance: cache_reference.window_tolerance without its bf16 weight term (1.01 * 2^-8 of the weighted sum of |V|),
and in its place the two parts': the upper half leaves less than 2^-7 of the weight, the rest is rounded to bf16
(2^-8 of it): 2^-15, and 2^-20 that the upper half leaves over."""
import numpy as np
import pytest

import cache_reference as ref
from gpu_util import say
from test_gpu_window import call, dev, make  # noqa: F401 (dev is a fixture)

pytestmark = pytest.mark.gpu


def compare(s, own_rounding=ref.BF16_HALF):
    f64 = lambda t: t.double().cpu().numpy()
    out, lse = (f64(x) for x in call(s))
    eo, el, absv, absz, count, defined = ref.window_attention(
        f64(s["q"]), f64(s["kc"]), f64(s["vc"]), s["table"], s["qo"], s["kv"], s["window"], s["sinks"], s["block"],
        s["max_kv"], s["scale"] or None)
    tol, tol_l = ref.window_tolerance("bf16", s["d"], eo, el, absv, absz, count)
    tol = tol - 1.01 * ref.BF16_HALF * absv + (2.0 ** -15 + 2.0 ** -20) * absv
    use = defined & (count > 0)
    bad = (np.abs(out - eo) > tol)[use]
    assert not bad.any(), (int(bad.sum()), bad.size, float((np.abs(out - eo) / absv)[use].max()))
    assert (np.abs(lse - el) <= tol_l)[use].all()
    return out, eo


# rows per kv-head and splits: up to 32 rows on four waves, two waves per 32 rows, whole-tile waves, eight waves
@pytest.mark.parametrize("Hq,Hkv,d,page,k,ctx,window,split", [
    (4, 4, 64, 16, [1, 3], [700, 90], 300, 0), (8, 2, 128, 64, [1, 5], [700, 130], 500, 0),
    (8, 2, 128, 64, [1, 5], [700, 130], 500, 64), (16, 4, 128, 64, [16, 9], [300, 700], 400, 0),
    (16, 2, 64, 16, [16, 9], [300, 700], 400, 64), (16, 1, 128, 32, [16, 4], [600, 90], 500, 0),
    (16, 1, 64, 64, [16, 4], [600, 90], 500, 128), (5, 1, 128, 1, [1], [40], 33, 0)])
def test_weights_keep_their_bits(dev, Hq, Hkv, d, page, k, ctx, window, split):  # noqa: F811
    say("window weights", Hq, Hkv, d, page, split)
    s = make(dev, 31, k, ctx, Hq, Hkv, d, page, "bf16", window, 4)
    s["split"] = split
    compare(s)


def test_infinite_values_stay_infinite(dev):  # noqa: F811
    """Even weights (zero queries) are exact in their upper half: an infinite value gives infinity all the same."""
    say("window infinite values")
    for k in ([1, 4], [16, 9]):
        s = make(dev, 32, k, [62, 100], 8, 2, 64, 16, "bf16", 64, 0)
        s["q"].zero_()
        key = int(s["kv"][0]) - int(k[0])  # the first row's own position: all rows of the request see it
        s["vc"][int(s["table"][0, key // 16]), :, key % 16, 5] = float("inf")
        s["vc"][int(s["table"][0, key // 16]), :, key % 16, 9] = -float("inf")
        out = call(s)[0].float().cpu()
        rows = slice(0, int(s["qo"][1]))
        assert bool((out[rows, :, 5] == float("inf")).all()) and bool((out[rows, :, 9] == -float("inf")).all())
        out[rows, :, 5] = out[rows, :, 9] = 0.0
        assert bool(out.isfinite().all())
