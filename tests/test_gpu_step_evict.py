"""Eviction with the lengths cut in place: every head and every CTA of a
sequence chooses from the length it had."""
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


def i64(x):
    return torch.as_tensor(np.asarray(x, np.int64)).cuda()


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32)).cuda()


def starts(n):
    return np.concatenate([[0], np.cumsum(n)])


class Case:
    """Ragged sequences of heads of 8 dimensions whose keys name their slot, a page list and new pages."""

    def __init__(self, lens, kv, budget, page, seed):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.kv, self.budget, self.page = lens, kv, budget, page
        held, need = [-(-n // page) for n in lens], [-(-min(n, budget) // page) for n in lens]
        self.base, self.dst_base, self.old = starts(held), starts(need), sum(held)
        self.score = (torch.randn(len(lens), kv, max(lens) + 1, generator=g) * 2).exp()
        self.k = torch.randn(self.old + sum(need), kv, page, 8, generator=g).to(torch.bfloat16)
        self.dst = self.old + torch.randperm(sum(need), generator=g).int()

    def evict(self, ctx, len_in, len_out, sinks, recent):
        k, v = self.k.cuda(), (-self.k).cuda()
        cache = ro.ro_cache(k, v, i64(self.base), i32(np.arange(self.old)))
        keep = torch.full((len(self.lens), self.kv, self.budget), -1, dtype=torch.int32, device="cuda")
        out = torch.full_like(self.score, -7.0).cuda()
        st = ro.ro_cache_evict(ctx, cache, len_in, self.score.cuda(), self.budget, sinks, recent, i64(self.dst_base),
                               self.dst.cuda(), keep, len_out, out)
        assert st == ro.RO_OK, ro.ro_last_error(ctx)
        assert ro.ro_ctx_sync(ctx) == ro.RO_OK, ro.ro_last_error(ctx)
        return keep.cpu(), out.cpu(), k.cpu(), v.cpu()


# more (sequence, head) pairs than the GPU holds at once; several CTAs a pair
@pytest.mark.parametrize("seqs,top,kv,budget,sinks,recent,page", [(400, 300, 2, 50, 2, 16, 16), (500, 150, 3, 20, 0, 0, 5),
                                                                  (3, 30_000, 2, 700, 4, 100, 64),
                                                                  (19, 6000, 4, 999, 16, 0, 128)])
def test_lengths_cut_in_place(ctx, seqs, top, kv, budget, sinks, recent, page):
    lens = [int(x) for x in np.random.default_rng(top).integers(0, top + 1, seqs)]
    lens[0] = top
    c = Case(lens, kv, budget, page, seqs)
    length = i32(lens)
    keep, out, k, v = c.evict(ctx, length, length, sinks, recent)
    kept = [min(n, budget) for n in lens]
    assert length.tolist() == kept
    for s, n in enumerate(kept):
        for h in range(kv):
            idx = ref.evict(lens[s], c.score[s, h].numpy(), budget, sinks, recent)
            assert np.array_equal(keep[s, h, :n].numpy(), idx) and bool((keep[s, h, n:] == -1).all())
            j, d = torch.as_tensor(idx), torch.arange(n)
            assert torch.equal(out[s, h, :n], c.score[s, h, j])
            at = c.dst[c.dst_base[s] + d // page].long()
            rows = c.k[c.base[s] + j // page, h, j % page]
            assert torch.equal(k[at, h, d % page], rows) and torch.equal(v[at, h, d % page], -rows)
    other = torch.zeros_like(length)
    apart = c.evict(ctx, i32(lens), other, sinks, recent)
    assert other.tolist() == kept and all(torch.equal(a, b) for a, b in zip(apart, (keep, out, k, v)))


def test_lengths_that_overlap_otherwise_are_refused(ctx):
    c = Case([40, 30, 20], 1, 10, 16, 1)
    both = i32([40, 30, 20, 20])
    with pytest.raises(AssertionError, match="in place"):
        c.evict(ctx, both[:3], both[1:], 0, 0)
    assert both.tolist() == [40, 30, 20, 20]
    c.evict(ctx, both[:3], i32([0, 0, 0]), 0, 0)
