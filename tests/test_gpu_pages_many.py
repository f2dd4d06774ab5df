"""sv_copy_pages with more steps than workgroups: every workgroup takes several (exact). The scratch of sv_reserve_pages."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_pages import cu, dev  # noqa: F401 (dev is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,layers,Hkv,page,d,dtype", [
    (300, 2, 8, 64, 128, "bf16"),   # 8 pieces per page: 9600 steps for 2048 workgroups
    (701, 3, 3, 16, 72, "f32"),     # a piece that is not full: 4206 steps
    (2049, 1, 1, 8, 64, "bf16")])   # 4098 steps of 1 KB
def test_copies_of_many_steps(dev, n, layers, Hkv, page, d, dtype):  # noqa: F811
    from paper_2607_25852_amd import binding as B
    rng = np.random.default_rng(n)
    pages = 2 * n + 20
    dt = dev.bfloat16 if dtype == "bf16" else dev.float32
    shape = (layers, pages, Hkv, page, d)
    old = [dev.randn(shape, device="cuda").to(dt) for _ in range(2)]
    ids = rng.permutation(pages)
    src, dst = ids[:n].astype(np.int32), ids[n:2 * n].astype(np.int32)
    for e in rng.integers(0, n, 20):  # skipped, with others after them
        (src if e % 2 else dst)[e] = (-1, pages, 2 ** 31 - 1, -2 ** 31)[e % 4]
    tokens = rng.integers(-1, page + 2, n).astype(np.int32)
    desc = B.copy_desc(n, layers, Hkv, d, page, pages, B.SV_BF16 if dtype == "bf16" else B.SV_F32)
    for count in (n, n - 7, n + 3):
        for tk in (None, tokens):
            say("copy of many steps", n, layers, count, tk is None)
            kc, vc = (x.clone() for x in old)
            B.copy_pages(desc, cu(dev, src), cu(dev, dst), cu(dev, [count]), kc, vc, None if tk is None else cu(dev, tk))
            for got, was in ((kc, old[0]), (vc, old[1])):
                want = was.clone()
                for e in range(min(count, n)):
                    if 0 <= src[e] < pages and 0 <= dst[e] < pages:
                        m = page if tk is None else min(max(int(tk[e]), 0), page)
                        want[:, dst[e], :, :m] = was[:, src[e], :, :m]
                assert dev.equal(got, want), (count, tk is None)


@pytest.mark.parametrize("pages,kept", [(50, True), (4096, True), (4097, False)])
def test_scratch_of_reserve(dev, pages, kept):  # noqa: F811
    """Left as it was up to 4096 pages."""
    from paper_2607_25852_amd import binding as B
    say("reserve scratch", pages)
    d = B.pages_desc(3, 4, pages, 16)
    ws = dev.full((B.reserve_pages_workspace_size(d),), 0x77, dtype=dev.uint8, device="cuda")
    z = lambda n: dev.zeros(n, dtype=dev.int32, device="cuda")
    table, refs, info = dev.full((3, 4), -1, dtype=dev.int32, device="cuda"), z(pages), z(4)
    B.reserve_pages(d, table, refs, z(3), z(3) + 20, z(3), z(3), z(3), info, ws)
    assert info.tolist() == [3, 6, 0, pages - 6] and bool((ws == 0x77).all()) == kept
