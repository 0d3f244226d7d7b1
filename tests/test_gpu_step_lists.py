"""Page lists whose offsets do not ascend: what lies past a list's end is not
read, the sequences concerned are left out and recorded, the others are whole."""
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


def ok(ctx, st):
    assert st == ro.RO_OK, ro.ro_last_error(ctx)


def i64(x):
    return torch.as_tensor(np.asarray(x, np.int64)).cuda()


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def caches(c):
    """The cache as it is, and with an offset past the list's end that its neighbours make ascend or not."""
    k, v = c.k.cuda(), c.v.cuda()
    bad = c.base.copy()
    bad[1] = bad[-1] + 1000                # sequence 0 runs past the list, sequence 1 backwards
    return ro.ro_cache(k, v, i64(c.base), c.pages.cuda()), ro.ro_cache(k, v, i64(bad), c.pages.cuda())


# few rows, many short sequences, tiles, rows by other pages, weights likewise
@pytest.mark.parametrize("seqs,top,new,heads,kv,page", [(4, 300, 1, 4, 2, 16), (400, 40, 1, 2, 2, 16), (4, 300, 50, 4, 2, 16),
                                                        (4, 300, 50, 4, 2, 5), (4, 300, 1, 4, 2, 5), (40, 300, 50, 4, 2, 16)])
@pytest.mark.parametrize("window", [0, 60])
def test_attend_and_weigh(ctx, seqs, top, new, heads, kv, page, window):
    lens, news = [top - s % 7 for s in range(seqs)], [new] * seqs
    c = ref.Cache(lens, kv, 64, page, torch.bfloat16, 5, junk=0.0)
    g = torch.Generator().manual_seed(1)
    q = torch.randn(seqs * new, heads, 64, generator=g).to(torch.bfloat16).cuda()
    base, length = i64(np.arange(seqs + 1) * new), i32(lens)
    got = []
    for cache in caches(c):
        out, lse = torch.full_like(q, 5.0), torch.zeros(q.shape[:2], device="cuda")
        score = torch.full((seqs, kv, top), -5.0, device="cuda")
        ok(ctx, ro.ro_cache_attend(ctx, cache, base, new, length, top, q, 0.125, window, 2, out, lse))
        first = ro.ro_ctx_sync(ctx)
        if got:
            lse = got[0][2]
        ok(ctx, ro.ro_cache_weigh(ctx, cache, base, new, length, q, 0.125, window, 2, lse, 1.0, None, score))
        assert ro.ro_ctx_sync(ctx) == first == (ro.RO_E_INVAL if got else ro.RO_OK)
        got.append((out, score, lse))
    good, bad = got
    assert bool((bad[0][:2 * new] == 5).all()) and bool((bad[1][:2] == -5).all())
    assert torch.equal(bad[0][2 * new:], good[0][2 * new:]) and torch.equal(bad[1][2:], good[1][2:])


def test_append(ctx):
    c = ref.Cache([40, 40, 40], 2, 64, 16, torch.bfloat16, 5, junk=0.0)
    c.k.zero_()
    _, bad = caches(c)
    x = torch.ones(9, 2, 64, dtype=torch.bfloat16, device="cuda")
    ok(ctx, ro.ro_cache_append(ctx, bad, i64([0, 3, 6, 9]), i32(np.repeat(range(3), 3)), i32(c.lens), None, None, None, None,
                               x, x))
    assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    k = bad._tensors[0]
    written = k[:, 0, :, 0].float()
    assert float(written.sum()) == 3   # sequence 2's
    assert float(written[c.pages[c.base[2] + 2].item(), 5:8].sum()) == 3


def test_evict(ctx):
    c = ref.Cache([40, 40, 40], 2, 64, 16, torch.bfloat16, 5, spare=6, junk=0.0)
    good, bad = caches(c)
    score = torch.rand(3, 2, 40, device="cuda")
    dst = c.free[:3].cuda()
    for cache, dst_base, held in ((bad, [0, 1, 2, 3], [0, 0, 10]), (good, [0, 500, 2, 3], [10, 10, 10])):
        k = cache._tensors[0]
        k[c.free.long().cuda()] = 0
        keep = torch.full((3, 2, 10), -1, dtype=torch.int32, device="cuda")
        n = torch.full((3,), 77, dtype=torch.int32, device="cuda")
        ok(ctx, ro.ro_cache_evict(ctx, cache, i32(c.lens), score, 10, 0, 0, i64(dst_base), dst, keep, n))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
        assert n.tolist() == held
        assert bool((k[c.free[:2].long().cuda()] == 0).all()) and not bool((k[c.free[2].item(), :, :10] == 0).all())
        for h in range(2):
            idx = ref.evict(40, score[2, h].cpu().numpy(), 10, 0, 0)
            assert np.array_equal(keep[2, h].cpu().numpy(), idx)
