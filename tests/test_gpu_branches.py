"""Biased attention, forks, sampling and compaction together: many samples of
many prompts on a pool they share, against each sample's own forward pass."""
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


from tests import step_reference as ref  # noqa: E402
from tests.test_gpu_sample import draw  # noqa: E402


def forward(tokens, model, cap):
    """Logits of the last token in 64 bits from the embeddings on, and a bound of what f16 steps may leave."""
    embed, into, back = (x.double().cpu() for x in model)
    from examples import branch_samples as ex
    H, K, D = ex.HEADS, ex.KV_HEADS, ex.DIM
    eps = 2.0 ** -11
    qkv = (embed[torch.as_tensor(tokens)] @ into).view(len(tokens), H + 2 * K, D)
    pos = torch.arange(len(tokens))[:, None]
    q, k = (ref.turn(x, pos, [D // 2], 10_000.0, False) for x in (qkv[:, :H], qkv[:, H:H + K]))
    v = qkv[:, H + K:]
    out, err = torch.zeros(H, D, dtype=torch.float64), torch.zeros(H, D, dtype=torch.float64)
    for h in range(H):
        g = h // (H // K)
        x = k[:, g] @ q[-1, h] / math.sqrt(D)
        # q and k rounded after the projection and after the turn: each product's four roundings, its sum in 32 bits
        dx = float((4.1 * eps * (k[:, g].abs() @ q[-1, h].abs()) / math.sqrt(D)).max())
        x = cap * torch.tanh(x / cap)
        p = torch.softmax(x, 0)
        out[h] = p @ v[:, g]
        err[h] = (2 * dx + 2.1 * eps) * (p @ v[:, g].abs()) + eps * out[h].abs()
    logits = out.view(-1) @ back
    return logits, err.view(-1) @ back.abs() + 1.1 * eps * logits.abs() + 1e-4


@pytest.mark.parametrize("prompts,samples,steps,seed", [(6, 3, 20, 1), (1, 40, 12, 2), (30, 1, 9, 3), (3, 2, 1, 4)])
def test_samples_of_prompts(prompts, samples, steps, seed):
    from examples import branch_samples as ex
    out, draws, last, used, model = ex.run(prompts, samples, steps, vocab=97, seed=seed)
    for logits, (t, k, p, m), u, got in draws:
        x, us = logits.double().cpu().numpy(), u.double().cpu().numpy()
        for r in range(len(got)):
            assert got[r] == draw(x[r], float(t[r]), int(k[r]), float(p[r]), float(m[r]), us[r])[0]
    for j, (n, logits) in last.items():
        want, tol = forward(out[j][:n], model, ex.CAP)
        off = (logits.double().cpu() - want).abs()
        assert bool((off <= tol).all()), (j, float((off - tol).max()))
    assert sum(len(x) for x in out) > 0 and used > 0
