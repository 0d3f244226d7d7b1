"""Weights where a key that every token sees holds an infinity: its product is
-inf and its weight 0, whatever rows a tile has beside the tokens' own."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()


import paper_2609_18703_gb300 as ro  # noqa: E402
from tests import step_reference as ref  # noqa: E402


@pytest.fixture
def ctx():
    c = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    yield c
    ro.ro_ctx_destroy(c)


# few rows, tiles (groups that fill one and that do not), rows of other pages
@pytest.mark.parametrize("news,heads,kv,page", [([1, 3], 4, 2, 16), ([1, 1], 9, 1, 16), ([300, 170], 4, 2, 16),
                                                ([300, 170], 14, 2, 16), ([300, 170], 6, 2, 32), ([70, 41], 43, 1, 16),
                                                ([30, 17], 3, 1, 5), ([30, 17], 100, 1, 5), ([1, 2], 4, 2, 5)])
@pytest.mark.parametrize("dtype,dim", [(torch.bfloat16, 128), (torch.float16, 64), (torch.bfloat16, 40)])
@pytest.mark.parametrize("window", [0, 400])
def test_weights_of_infinite_keys(ctx, news, heads, kv, page, dtype, dim, window):
    lens = [900, 700]
    c = ref.Cache(lens, kv, dim, page, dtype, 7, junk=0.0)
    g = torch.Generator().manual_seed(page)
    T = sum(news)
    q = torch.randn(T, heads, dim, generator=g).to(dtype)
    q[..., 0] = 1
    q = q.cuda()
    base = torch.as_tensor(np.concatenate([[0], np.cumsum(news)]).astype(np.int64)).cuda()
    length, past = torch.tensor(lens, dtype=torch.int32).cuda(), torch.rand(2, kv, 900, device="cuda")
    got = []
    for low in (-3000.0, -float("inf")):   # the product's weight is 0 either way
        for s, L in enumerate(lens):
            for j in (0, 3, 300, L - news[s] - 1):
                c.k[int(c.pages[c.base[s] + j // page]), :, j % page, 0] = low
        cache = ro.ro_cache(c.k.cuda(), c.v.cuda(), torch.as_tensor(c.base).cuda(), c.pages.cuda())
        out, lse = torch.zeros_like(q), torch.zeros(T, heads, device="cuda")
        score = torch.zeros(2, kv, 900, device="cuda")
        for st in (ro.ro_cache_attend(ctx, cache, base, max(news), length, 900, q, 0.125, window, 2, out, lse),
                   ro.ro_cache_weigh(ctx, cache, base, max(news), length, q, 0.125, window, 2, lse, 0.5, past, score),
                   ro.ro_ctx_sync(ctx)):
            assert st == ro.RO_OK, ro.ro_last_error(ctx)
        got.append((out, lse, score))
    assert not any(bool(torch.isnan(x).any()) for x in got[0])
    assert all(torch.equal(a, b) for a, b in zip(*got))
