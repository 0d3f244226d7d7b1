"""What the model step's calls keep on the GPU stays within the stated bound."""
import math

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


@pytest.mark.parametrize("new,heads,kv,slots", [(768, 16, 16, 400_000), (130, 8, 8, 500_000), (40, 12, 4, 300_000),
                                                (1, 32, 8, 400_000)])
def test_partial_results_of_a_long_sequence(new, heads, kv, slots):
    """Many runs of few pairs of row tiles; and they are joined right."""
    page, dim = 128, 128
    n = slots // page
    g = torch.Generator(device="cuda").manual_seed(new)
    pool = torch.randn(n, kv, page, dim, generator=g, device="cuda", dtype=torch.bfloat16)
    pages = torch.randperm(n, generator=g, device="cuda").int()
    cache = ro.ro_cache(pool, pool, torch.tensor([0, n], device="cuda"), pages)
    q = torch.randn(new, heads, dim, generator=g, device="cuda").bfloat16()
    out, lse = torch.zeros_like(q), torch.zeros(new, heads, device="cuda")
    tok, scale = torch.tensor([0, new], device="cuda"), 1 / math.sqrt(dim)
    ctx = ro.ro_ctx_create(0, torch.cuda.current_stream(), 1)

    def call(length):
        lens = torch.tensor([length], dtype=torch.int32, device="cuda")
        assert ro.ro_cache_attend(ctx, cache, tok, new, lens, length, q, scale, 0, 0, out, lse) == ro.RO_OK
        assert ro.ro_ctx_sync(ctx) == ro.RO_OK

    call(n * page // 100)   # loads the kernels, the join among them
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    call(n * page)
    torch.cuda.synchronize()
    # 1,024 runs of 256 rows (or 16,384 of 16) of dim + 2 floats, an eighth more, and the allocator's steps
    assert free - torch.cuda.mem_get_info()[0] <= 1024 * 256 * (dim + 2) * 4 * 9 // 8 + (8 << 20)
    for t in (0, new - 1):
        for h in (0, heads - 1):
            rows = pool[pages.long(), h // (heads // kv)].reshape(-1, dim)[: n * page - new + t + 1].double()
            x = scale * (rows @ q[t, h].double())
            p = torch.softmax(x, 0)
            # logits below 8 in 32 bits of 128 products; weights and output are bf16
            tol = 2.0 ** -8 * (p @ rows.abs()) + 2.0 ** -8 * (p @ rows).abs() + 1e-5
            assert bool(((out[t, h].double() - p @ rows).abs() <= tol).all())
            assert abs(float(lse[t, h]) - float(torch.logsumexp(x, 0))) < 1e-4
    ro.ro_ctx_destroy(ctx)


@pytest.mark.parametrize("new,heads,kv,slots,page", [(1, 8, 8, 20_000, 64), (64, 8, 2, 20_000, 64), (20, 2, 1, 9_000, 5)])
def test_graphs_outlive_the_growth_of_a_workspace(new, heads, kv, slots, page):
    """A captured call that splits its slots, replayed after calls that need larger workspaces."""
    dim, n = 64, -(-slots // page)
    g = torch.Generator(device="cuda").manual_seed(new)
    pool = torch.randn(n, kv, page, dim, generator=g, device="cuda").half()
    pages = torch.randperm(n, generator=g, device="cuda").int()
    stream = torch.cuda.Stream()
    ctx = ro.ro_ctx_create(0, stream, 1)

    def setup(seqs):
        cache = ro.ro_cache(pool, pool, torch.arange(seqs + 1, device="cuda") * n, pages.repeat(seqs))
        q = torch.randn(seqs * new, heads, dim, generator=g, device="cuda").half()
        tok = torch.arange(seqs + 1, device="cuda") * new
        lens = torch.full((seqs,), slots, dtype=torch.int32, device="cuda")
        out, lse = torch.zeros_like(q), torch.zeros(seqs * new, heads, device="cuda")
        torch.cuda.synchronize()

        def call():
            assert ro.ro_cache_attend(ctx, cache, tok, new, lens, slots, q, 0.125, 0, 0, out, lse) == ro.RO_OK, \
                ro.ro_last_error(ctx)
        return call, out, lse

    small, out, lse = setup(1)
    small()
    assert ro.ro_ctx_sync(ctx) == ro.RO_OK
    want = out.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        small()
    for seqs in (5, 40):
        large, large_out, large_lse = setup(seqs)
        large()
        assert ro.ro_ctx_sync(ctx) == ro.RO_OK
        taken = [torch.full((1 << 22,), 7, dtype=torch.uint8, device="cuda") for _ in range(8)]   # what was let go of
        first = large_out.clone(), large_lse.clone()
        for _ in range(2):
            out.zero_()
            lse.zero_()
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        assert all(bool((x == 7).all()) for x in taken)
        large()
        assert ro.ro_ctx_sync(ctx) == ro.RO_OK
        assert torch.equal(large_out, first[0]) and torch.equal(large_lse, first[1])
    ro.ro_ctx_destroy(ctx)
