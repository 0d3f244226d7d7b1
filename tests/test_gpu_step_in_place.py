"""Outputs that may lie on an input, and those that may not."""
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

BF16 = torch.bfloat16


@pytest.fixture
def ctx():
    c = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)
    yield c
    ro.ro_ctx_destroy(c)


def ints(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x), dtype=dtype).cuda()


def views(heads=4):
    """Two views that start together: heads next to one another, and further apart."""
    flat = torch.randn(6 * 8 * 64, device="cuda").to(BF16)
    return flat, flat.as_strided((3, heads, 64), (heads * 64, 64, 1)), flat.as_strided((3, heads, 64), (8 * 64, 64, 1))


def setup():
    k = torch.zeros(4, 2, 16, 64, dtype=BF16, device="cuda")
    return ro.ro_cache(k, k.clone(), ints([0, 4], torch.int64), ints([0, 1, 2, 3])), ints([0, 3], torch.int64), ints([10])


def test_turned_in_place_only_where_it_lies(ctx):
    flat, near, far = views()
    cache, tok, lens = setup()
    before, pos, rope = flat.clone(), ints(np.zeros((3, 1))), ro.ro_rope([8])
    rows = torch.zeros(3, 2, 64, dtype=BF16, device="cuda")
    assert ro.ro_rotary(ctx, near, far, pos, rope) == ro.RO_E_INVAL
    assert "in place" in ro.ro_last_error(ctx)
    assert ro.ro_cache_append(ctx, cache, tok, ints([0, 0, 0]), lens, pos, rope, far, near, rows, rows) == ro.RO_E_INVAL
    assert torch.equal(flat, before)
    assert ro.ro_rotary(ctx, near, near, pos, rope) == ro.RO_OK
    assert ro.ro_cache_append(ctx, cache, tok, ints([0, 0, 0]), lens, pos, rope, far, far, rows, rows) == ro.RO_OK
    # one token: its stride does not count
    one = ro.ro_rotary(ctx, near[:1], far[:1], pos[:1], rope)
    assert one == ro.RO_OK and ro.ro_ctx_sync(ctx) == ro.RO_OK


def test_attention_does_not_overwrite_its_queries(ctx):
    cache, tok, lens = setup()
    q = torch.randn(3, 4, 64, device="cuda").to(BF16)
    before = q.clone()
    assert ro.ro_cache_attend(ctx, cache, tok, 3, lens, 10, q, 1.0, 0, 0, q) == ro.RO_E_INVAL
    assert ro.ro_ctx_sync(ctx) == ro.RO_OK and torch.equal(q, before)
    none = q[:0]
    assert ro.ro_cache_attend(ctx, cache, ints([0, 0], torch.int64), 0, lens, 10, none, 1.0, 0, 0, none) == ro.RO_OK


def test_scores_that_overlap(ctx):
    cache, tok, lens = setup()
    q, lse = torch.zeros(3, 4, 64, dtype=BF16, device="cuda"), torch.zeros(3, 4, device="cuda")
    flat = torch.rand(2 * 64 + 64, device="cuda")
    before = flat.clone()
    score, shifted = flat[:128].view(1, 2, 64), flat[64:].view(1, 2, 64)
    keep, n = torch.zeros(1, 2, 8, dtype=torch.int32, device="cuda"), ints([0])

    def weigh(past, out):
        return ro.ro_cache_weigh(ctx, cache, tok, 3, lens, q, 1.0, 0, 0, lse, 1.0, past, out)

    def evict(score, out):
        return ro.ro_cache_evict(ctx, cache, lens, score, 8, 0, 0, ints([0, 1], torch.int64), ints([3]), keep, n, out)

    assert weigh(score, shifted) == ro.RO_E_INVAL and weigh(shifted, score) == ro.RO_E_INVAL
    assert evict(score, shifted) == ro.RO_E_INVAL and evict(shifted, score) == ro.RO_E_INVAL
    assert evict(score, score) == ro.RO_E_INVAL
    assert ro.ro_ctx_sync(ctx) == ro.RO_OK and torch.equal(flat, before)
    assert weigh(score, score) == ro.RO_OK and evict(score, score.clone()) == ro.RO_OK and ro.ro_ctx_sync(ctx) == ro.RO_OK
