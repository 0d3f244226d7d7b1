"""Attention over f16 caches where one token draws nearly all the weight: the
many light ones still count."""
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


# few rows: one CTA's, joined in a cluster, joined through memory, a warp alone; tiles unsplit and split; rows of other
# pages, unsplit and split
@pytest.mark.parametrize("lens,new,heads,kv,page,dim", [
    ([500], 1, 2, 1, 16, 64), ([777], 1, 4, 2, 16, 128), ([60_000], 1, 4, 2, 64, 64), ([300] * 400, 1, 2, 1, 16, 64),
    ([900, 700] * 80, 40, 6, 6, 16, 64), ([20_000], 40, 6, 2, 64, 128), ([700, 300], 1, 2, 1, 5, 64), ([700], 20, 2, 1, 5, 64),
    ([20_000], 20, 2, 1, 5, 64)])
@pytest.mark.parametrize("heavy", ["first", "middle"])
def test_light_weights_behind_a_heavy_token(ctx, lens, new, heads, kv, page, dim, heavy):
    c = ref.Cache(lens, kv, dim, page, torch.float16, 1, junk=0.0)
    g = torch.Generator().manual_seed(len(lens))
    # logits: 0 for the heavy token, -16.8 .. -18 (2^-24 .. 2^-26) for the others; values: 0 for it, 32 to 64 for the others
    c.k[..., 0] = -(16.8 + 1.2 * torch.rand(c.k.shape[:3], generator=g)).half()
    c.v[:] = (32 + 32 * torch.rand(c.v.shape, generator=g)).half()
    for s, L in enumerate(lens):
        at = 0 if heavy == "first" else (L - new) // 2
        page_at = int(c.pages[c.base[s] + at // page])
        c.k[page_at, :, at % page, 0] = 0
        c.v[page_at, :, at % page] = 0
    T = len(lens) * new
    q = torch.zeros(T, heads, dim, dtype=torch.float16)
    q[..., 0] = 1
    cache = ro.ro_cache(c.k.cuda(), c.v.cuda(), torch.as_tensor(c.base).cuda(), c.pages.cuda())
    out, lse = torch.zeros(T, heads, dim, dtype=torch.float16, device="cuda"), torch.zeros(T, heads, device="cuda")
    base = torch.as_tensor(np.arange(len(lens) + 1) * new).cuda()
    st = ro.ro_cache_attend(ctx, cache, base, new, torch.as_tensor(lens, dtype=torch.int32).cuda(), max(lens), q.cuda(), 1.0,
                            0, 0, out, lse)
    assert st == ro.RO_OK, ro.ro_last_error(ctx)
    assert ro.ro_ctx_sync(ctx) == ro.RO_OK
    for s in range(0, len(lens), max(1, len(lens) // 3)):
        for i in sorted({0, new - 1}):
            n = lens[s] - new + i + 1
            x, v = c.rows(c.k, s, n)[..., 0].double(), c.rows(c.v, s, n).double()
            for h in range(heads):
                kh = h // (heads // kv)
                p = torch.softmax(x[kh], 0)
                want = p @ v[kh]
                # a weight: one rounding to f16, and 2^-36 of the largest where f16 runs out of bits; 32-bit sums; the output
                tol = (2.0 ** -11 + 2.0 ** -11 + 2.0 ** -17) * want + 2.0 ** -36 * p.max() * v[kh].sum(0)
                err = (out[s * new + i, h].double().cpu() - want).abs()
                assert bool((err <= tol).all()), (float((err / want).max()), float((tol / want).min()))
                z = float(torch.logsumexp(x[kh], 0))
                assert abs(float(lse[s * new + i, h]) - z) < 2.0 ** -20 * 20
