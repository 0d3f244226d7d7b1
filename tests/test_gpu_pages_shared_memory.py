"""Outputs of page plans that share memory with a page list behind its first
entry, or with an array that changes in place: refused, or recorded where only
the GPU knows how long the list is.  Arrays beside one another are no overlap."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests.test_gpu_pages import Pool, _built, ctx, i32, i64, moves_of, ok  # noqa: E402,F401

REFS = [1, 0, 1, 0, 1, 0, 1, 1]


def setup():
    """A list of three entries at [8, 11) of an array, the rest of it free."""
    free = torch.zeros(96, dtype=torch.int32, device="cuda")
    pages = free[8:11]
    pages.copy_(i32([2, 4, 6]))
    t, n = moves_of(8)
    return free, pages, Pool(8, 1, 16, 32).caches(i64([0, 3]), pages)[0], i32(REFS), t, n


def test_compact_in_place(ctx):   # noqa: F811
    free, pages, cache, refs, t, n = setup()
    good = dict(cache=cache, d_pages_out=pages, d_refs=refs, d_refs_out=free[16:24], d_n_used=free[32:33], moves=ro.ro_moves(*t, n))

    def compact(**change):
        return ro.ro_cache_compact(ctx, *{**good, **change}.values())

    before = free.clone()
    for bad in (dict(d_n_used=free[9:10]), dict(d_n_used=free[10:11]), dict(d_refs_out=free[10:18]), dict(d_refs_out=free[1:9]),
                dict(moves=ro.ro_moves(free[4:12], t[1], t[2], n)), dict(moves=ro.ro_moves(*t, free[10:11])),
                dict(d_refs=free[9:17], d_refs_out=free[9:17]), dict(d_refs=free[16:24], d_n_used=free[17:18])):
        assert compact(**bad) == ro.RO_E_INVAL, bad
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert torch.equal(free, before)
    ok(ctx, compact(d_n_used=free[11:12], d_refs_out=free[0:8]))   # beside the list
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert free[11].item() == 5 and free[:8].tolist() == [1, 1, 1, 1, 1, 0, 0, 0] and pages.tolist() == [2, 4, 1]


def test_compact_into_another_array(ctx):   # noqa: F811
    for used, counts, out in ((9, 16, 40), (10, 16, 40), (32, 9, 40), (32, 16, 9), (32, 16, 10)):
        free, pages, cache, refs, t, n = setup()
        ok(ctx, ro.ro_cache_compact(ctx, cache, free[out:out + 3], refs, free[counts:counts + 8], free[used:used + 1],
                                    ro.ro_moves(*t, n)))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    free, pages, cache, refs, t, n = setup()
    # an output with room for more entries than the list has, right behind it
    ok(ctx, ro.ro_cache_compact(ctx, cache, free[11:75], refs, free[:8], free[75:76], ro.ro_moves(*t, n)))
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert free[11:14].tolist() == [2, 4, 1] and free[75].item() == 5 and pages.tolist() == [2, 4, 6]


def test_fork(ctx):   # noqa: F811
    def fork(free, cache, refs, t, n, pages=40, lens=48, counts=16, **change):
        a = dict(cache=cache, d_len=i32([40]), d_child_base=i64([0, 2]), d_child_parent=i32([0, 0]), d_dst_base=i64([0, 3, 6]),
                 d_dst_seq=i32([0, 0, 0, 1, 1, 1]), d_dst_pages=free[pages:pages + 6], d_len_out=free[lens:lens + 2],
                 d_refs=refs, d_refs_out=free[counts:counts + 8], moves=ro.ro_moves(*t, n))
        a.update(change)
        return ro.ro_cache_fork(ctx, *a.values())

    for bad in (dict(pages=9), dict(lens=9), dict(lens=10), dict(counts=10)):
        free, pages, cache, refs, t, n = setup()
        ok(ctx, fork(free, cache, refs, t, n, **bad))
        assert ro.ro_ctx_sync(ctx) == ro.RO_E_INVAL
    free, pages, cache, refs, t, n = setup()
    for bad in (dict(d_len=free[16:17]), dict(d_child_parent=free[18:20])):   # counts in place
        assert fork(free, cache, free[16:24], t, n, **bad) == ro.RO_E_INVAL
    ok(ctx, ro.ro_ctx_sync(ctx))
    ok(ctx, fork(free, cache, refs, t, n, pages=11, counts=0, lens=17))   # beside the list
    ok(ctx, ro.ro_ctx_sync(ctx))
    assert free[11:17].tolist() == [2, 4, 6, 2, 4, 1] and free[17:19].tolist() == [40, 40] and pages.tolist() == [2, 4, 6]
    assert free[:8].tolist() == [1, 1, 2, 0, 2, 0, 1, 1] and n.item() == 1
