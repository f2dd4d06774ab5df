"""sv_window_attn where requests are taken in the order of their rows: the same bits as in a batch of 65 requests, which are
taken in their own order, with lists divided alike; some requests are compared with the definition in 64 bits. Equal
numbers of rows, requests without rows, with more than a block and with fewer keys than rows are among them."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_window import call, check, dev, make  # noqa: F401 (dev is a fixture)
from window_shapes import BY_ROWS, in_order

pytestmark = pytest.mark.gpu


def part(s, i, j, split):
    """Requests i .. j-1 of the batch, on the same caches."""
    a, b = int(s["qo"][i]), int(s["qo"][j])
    return {**s, "R": j - i, "qo": (s["qo"][i:j + 1] - a).astype(np.int32), "kv": s["kv"][i:j], "table": s["table"][i:j],
            "q": s["q"][a:b], "total": b - a, "split": split}


@pytest.mark.parametrize("shape,plan", BY_ROWS, ids=lambda x: "-".join(map(str, x)) if len(x) == 10 else "")
def test_requests_by_rows(dev, shape, plan):  # noqa: F811
    R, block, Hq, Hkv, d, dtype, max_kv, window, sinks, split = shape
    say("window by rows", shape)
    rng = np.random.default_rng(R + d)
    k = rng.choice([1, 2, block // 2, block - 1, block, block], R)
    ctx = rng.integers(1, 230, R)
    k[3], k[R - 2] = 0, 0
    k[7] = block + 1
    s = make(dev, 51, k, ctx, Hq, Hkv, d, 16, dtype, window, sinks, block=block)
    s["kv"][5] = max(int(k[5]) - 1, 0)
    cols = -(-max_kv // 16)
    s["table"] = np.concatenate([s["table"], np.full((R, cols - s["cols"]), -1, np.int32)], 1)
    s.update(cols=cols, max_kv=max_kv, split=split)
    out, lse = call(s)
    sound = [i for i in range(R) if 1 <= k[i] <= block and s["kv"][i] >= k[i]]
    assert len(sound) == R - 4
    owned = np.zeros(s["total"], bool)
    for i in sound:
        owned[int(s["qo"][i]):int(s["qo"][i + 1])] = True
    assert bool((out[~owned] == 7.0).all()) and bool((lse[~owned] == 7.0).all()), "rows that no request owns"
    more = 65 - R
    wide = {**s, "R": 65, "split": in_order(shape, plan)[0][-1],
            "qo": np.concatenate([s["qo"], np.full(more, s["qo"][-1], np.int32)]),
            "kv": np.concatenate([s["kv"], np.zeros(more, np.int32)]),
            "table": np.concatenate([s["table"], np.full((more, cols), -1, np.int32)])}
    o, l = call(wide)
    assert dev.equal(out, o) and dev.equal(lse, l), dev.nonzero((out != o).any(2).any(1)).flatten().tolist()
    for i in (sound[0], sound[len(sound) // 2]):
        check(part(s, i, i + 1, split))
        a, b = int(s["qo"][i]), int(s["qo"][i + 1])
        near = call(part(s, i, i + 1, split))[0].float()  # (maybe divided otherwise: two roundings of values below 4)
        assert float(near.abs().max()) < 4 and float((out[a:b].float() - near).abs().max()) <= 2 * 4 * 2.0 ** -8
