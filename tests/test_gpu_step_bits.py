"""Equal calls give equal bits, whatever ran on the GPU between them."""
import math

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


def starts(n):
    return torch.as_tensor(np.concatenate([[0], np.cumsum(n)]).astype(np.int64)).cuda()


def step(ctx, c, news, q, window=0, sinks=0):
    """The chunks' attention and weights: out, lse, score."""
    cache = ro.ro_cache(c.k.cuda(), c.v.cuda(), torch.as_tensor(c.base).cuda(), c.pages.cuda())
    lens, base, scale = torch.as_tensor(c.lens, dtype=torch.int32).cuda(), starts(news), 1 / math.sqrt(q.shape[2])
    out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device="cuda")
    score = torch.zeros(len(news), c.k.shape[1], max(c.lens), device="cuda")
    for st in (ro.ro_cache_attend(ctx, cache, base, max(news), lens, max(c.lens), q, scale, window, sinks, out, lse),
               ro.ro_cache_weigh(ctx, cache, base, max(news), lens, q, scale, window, sinks, lse, 1.0, None, score),
               ro.ro_ctx_sync(ctx)):
        assert st == ro.RO_OK, ro.ro_last_error(ctx)
    return out, lse, score


@pytest.mark.parametrize("dtype,dim,heads,kv,page", [(torch.bfloat16, 128, 28, 4, 64), (torch.float16, 64, 14, 2, 16),
                                                     (torch.bfloat16, 64, 6, 2, 32), (torch.float16, 128, 12, 1, 20),
                                                     (torch.bfloat16, 80, 5, 1, 64)])
def test_groups_that_do_not_fill_a_tile(ctx, dtype, dim, heads, kv, page):
    """Rows of a tile that no token has hold what ran before: they must not reach the others' rounding."""
    news, lens = [300, 129, 40, 700], [900, 129, 600, 2500]
    g = torch.Generator().manual_seed(heads)
    c = ref.Cache(lens, kv, dim, page, dtype, 3, junk=0.0)
    q = torch.randn(sum(news), heads, dim, generator=g).to(dtype).cuda()
    before = ref.Cache([400] * 200, 1, dim, 16, dtype, 4, junk=0.0)
    rows = torch.randn(200 * 64, 4, dim, generator=g).to(dtype).cuda()
    got = []
    for size in (0.0, 1.0, 40.0, -300.0):   # what earlier calls leave in shared memory
        step(ctx, before, [64] * 200, rows * size)
        got.append(step(ctx, c, news, q))
        got.append(step(ctx, c, news, q, 256, 3))
    for a in got[2::2]:
        assert all(torch.equal(x, y) for x, y in zip(a, got[0]))
    for a in got[3::2]:
        assert all(torch.equal(x, y) for x, y in zip(a, got[1]))
