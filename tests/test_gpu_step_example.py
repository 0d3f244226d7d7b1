"""The example that runs the model-step operators beside the lineage path: every
video's assembled records against the same step in 64 bits."""
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


def test_every_video_against_64_bits():
    from examples import stream_frames as ex
    from tests import step_reference as ref
    counts, outs, held = ex.run(videos=9, frames=30, wave=7, seed=4)
    assert held == counts.tolist()
    _, records, place, weight = ex.inputs(9, 30, 4)
    qkv = (records @ weight).view(-1, ex.HEADS + 2 * ex.KV_HEADS, ex.DIM).cpu()
    turned = ref.turn(qkv, place.cpu(), [16, 8, 8], 10_000.0, False)
    starts = np.concatenate([[0], np.cumsum(counts)])
    for i, n in enumerate(counts):
        rows = slice(starts[i], starts[i] + n)
        k = turned[rows, ex.HEADS:ex.HEADS + ex.KV_HEADS]
        v = qkv[rows, ex.HEADS + ex.KV_HEADS:].double()
        for h in range(ex.HEADS):
            kh = h // (ex.HEADS // ex.KV_HEADS)
            x = turned[rows, h] @ k[:, kh].T / math.sqrt(ex.DIM)
            x = x.masked_fill(~torch.ones(n, n, dtype=torch.bool).tril(), -math.inf)
            p = torch.softmax(x, 1)
            want = p @ v[:, kh]
            # q and k are rounded to f16 once turned, a logit errs by their sum's size; weights and output are f16
            dx = 2 * 2.0 ** -11 * (turned[rows, h].abs() @ k[:, kh].abs().T).amax(1, keepdim=True) / math.sqrt(ex.DIM)
            tol = (2 * dx + 2.0 ** -10) * (p @ v[:, kh].abs()) + 2.0 ** -11 * want.abs() + 1e-6
            assert bool(((outs[i][:, h].double().cpu() - want).abs() <= tol).all())


def test_caches_stay_within_their_budget():
    from examples import stream_frames as ex
    counts, outs, held = ex.run(videos=20, frames=60, wave=16, budget=33, seed=5)
    assert held == np.minimum(counts, 33).tolist() and max(counts) > 33
    whole, full, _ = ex.run(videos=20, frames=60, wave=16, seed=5)
    for i in range(20):
        assert not bool(torch.isnan(outs[i]).any())
        n = min(int(counts[i]), 32)   # two waves fit the budget: the same until then
        assert torch.equal(outs[i][:n], full[i][:n])


def test_evictions_keep_the_heaviest(monkeypatch):
    """The slots that the example's evictions keep, against the definition on the scores that they saw."""
    from examples import stream_frames as ex
    from tests import step_reference as ref
    evict, cuts = ex.ro.ro_cache_evict, []

    def watched(ctx, cache, d_len, d_score, budget, sinks, recent, dst_base, dst_pages, d_keep, d_len_out, d_score_out):
        lens, score = d_len.cpu(), d_score.cpu()
        st = evict(ctx, cache, d_len, d_score, budget, sinks, recent, dst_base, dst_pages, d_keep, d_len_out, d_score_out)
        cuts.append((lens, score, budget, sinks, recent, d_keep.cpu(), d_len_out.cpu(), d_score_out.cpu()))
        return st

    monkeypatch.setattr(ex.ro, "ro_cache_evict", watched)
    ex.run(videos=200, frames=60, wave=16, budget=33, seed=5)
    assert len(cuts) > 3
    for lens, score, budget, sinks, recent, keep, held, kept_score in cuts:
        assert torch.equal(held, lens.clamp(max=budget)) and int(lens.max()) > budget
        for s in range(lens.numel()):
            n = int(held[s])
            for h in range(score.shape[1]):
                idx = ref.evict(int(lens[s]), score[s, h].numpy(), budget, sinks, recent)
                assert np.array_equal(keep[s, h, :n].numpy(), idx)
                assert torch.equal(kept_score[s, h, :n], score[s, h, torch.as_tensor(idx)])
