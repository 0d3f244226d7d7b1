"""Capped scores: what slots hold that nobody sees, and what ran before, does not
show in a single bit of the results."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

import paper_2609_18703_gb300 as ro  # noqa: E402
from tests import bias_reference as ref  # noqa: E402
from tests.test_gpu_biased import BF16, F16, _built, build, ctx, ok, starts  # noqa: E402,F401

FORMS = [dict(cap=30.0), dict(cap=30.0, docs=40), dict(cap=30.0, window=20, sinks=3), dict(cap=30.0, slopes=True, docs=25),
         dict(cap=30.0, docs=50, frame=9), dict(cap=100.0, window=9, sinks=2, docs=30, frame=4)]


@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("dtype,dim,page", [(BF16, 64, 16), (F16, 128, 64), (BF16, 128, 20), (F16, 64, 7)])
@pytest.mark.parametrize("lens,news", [([200, 77, 530], [120, 77, 300]), ([200, 77, 530], [2, 1, 2]),
                                       ([40 + s % 90 for s in range(300)], [s % 3 for s in range(300)])])
def test_unseen_slots_leave_no_trace(ctx, form, dtype, dim, page, lens, news):   # noqa: F811
    results = []
    for junk in (0.0, 1.0, 6e4, -300.0):
        case = build(lens, news, 2, dim, page, dtype, 4, FORMS[form], 17, pads=0.2, junk=junk)
        t = starts(news)
        for s, n in enumerate(news):
            first = None if case.first is None else case.first[t[s]:t[s + 1]]
            until = None if case.until is None else case.until[t[s]:t[s + 1]]
            used = ref.seen(lens[s], n, case.window, case.sinks, first, until).any(0) if n else torch.zeros(lens[s], dtype=torch.bool)
            for j in np.flatnonzero(~used.numpy()):
                at = int(case.c.pages[case.c.base[s] + j // page])
                case.c.k[at, :, j % page] = junk
                case.c.v[at, :, j % page] = junk
        case.device().call(ctx)
        ok(ctx, ro.ro_ctx_sync(ctx))
        results.append((case.out.clone(), case.lse.clone()))
    for out, lse in results[1:]:
        assert torch.equal(out, results[0][0]) and torch.equal(lse, results[0][1])
