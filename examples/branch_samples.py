"""Several samples of each of many prompts, on one paged cache that they share.

A prompt expands into its samples: they share the prompt's full pages and get
their own copy of the open one.  Each step the samples' tokens go through one
layer whose scores are capped, the next tokens are drawn from its logits, samples
that ended give their pages back, and the pool is closed up when it got sparse:

  ro_expand_noalloc       sequences -> pages, sequences -> tokens, prompts -> samples
  ro_cache_append         rotary by position, keys and values into the pages
  ro_cache_attend_biased  attention over what a sequence holds, capped scores
  ro_cache_fork           prompts -> samples; later samples -> those that go on
  ro_sample               each sample's next token, with settings of its own
  ro_cache_compact        the pages in use move together

    python examples/branch_samples.py [--prompts N] [--samples N] [--steps N]
"""
import argparse
import math
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_18703_gb300 as ro  # noqa: E402

HEADS, KV_HEADS, DIM, PAGE = 4, 2, 64, 16
CAP, END = 20.0, 0   # of the scores; the token that ends a sample


def check(ctx, status):
    if status != ro.RO_OK:
        raise ro.RoError("branch_samples", status, ro.ro_last_error(ctx))


def u32(x):
    return torch.as_tensor(np.asarray(x).astype(np.int64)).to(torch.int32).cuda()


def model(vocab, seed):
    """One layer: embedding, the fused projection, the way back to logits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")   # noqa: E731
    return (n(vocab, HEADS * DIM).half(), (n(HEADS * DIM, (HEADS + 2 * KV_HEADS) * DIM) / 12).half(),
            (n(HEADS * DIM, vocab) / 6).half())


class Server:
    """The pool, the running sequences' lists and lengths, and the calls on them."""

    def __init__(self, n_pages, vocab, seed):
        self.stream = torch.cuda.current_stream()
        self.ctx = ro.ro_ctx_create(torch.cuda.current_device(), self.stream, 1)
        self.embed, self.into, self.back = model(vocab, seed)
        self.k = torch.zeros(n_pages, KV_HEADS, PAGE, DIM, dtype=torch.float16, device="cuda")
        self.v = torch.zeros_like(self.k)
        self.rope = ro.ro_rope([DIM // 2])
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.n_used = torch.zeros(1, dtype=torch.int32, device="cuda")
        move = lambda: torch.zeros(n_pages, dtype=torch.int32, device="cuda")   # noqa: E731
        self.moves = ro.ro_moves(move(), move(), move(), torch.zeros(1, dtype=torch.int32, device="cuda"))
        # a sequence that holds nothing, whose continuations are the prompts
        self.lens = np.zeros(1, np.int64)
        self.base, self.pages = torch.zeros(2, dtype=torch.int64, device="cuda"), u32([0])

    def expand(self, counts):
        """offsets, parents of an expansion."""
        n, total = len(counts), int(np.sum(counts))
        base = torch.zeros(n + 1, dtype=torch.int64, device="cuda")
        parent, ordinal = (torch.zeros(max(total, 1), dtype=torch.int32, device="cuda") for _ in range(2))
        st, _, _ = ro.ro_expand_noalloc(u32(counts), n, base, parent, ordinal, total, stream=self.stream)
        check(self.ctx, st)
        return base, parent[:total]

    def cache(self):
        return ro.ro_cache(self.k, self.v, self.base, self.pages)

    def fork(self, kids, room):
        """Every sequence goes on in kids[s] continuations, each with room[c] tokens' pages."""
        child_base, child_parent = self.expand(kids)
        want = -(-np.asarray(room, np.int64) // PAGE)
        dst_base, dst_seq = self.expand(want) if len(want) else (torch.zeros(1, dtype=torch.int64, device="cuda"), child_parent)
        pages = torch.zeros(max(int(want.sum()), 1), dtype=torch.int32, device="cuda")
        length = torch.zeros(len(want), dtype=torch.int32, device="cuda")
        check(self.ctx, ro.ro_cache_fork(self.ctx, self.cache(), u32(self.lens), child_base, child_parent, dst_base, dst_seq,
                                         pages, length, self.refs, self.refs, self.moves))
        self.base, self.pages, self.lens = dst_base, pages, np.repeat(self.lens, kids)
        if len(want) == 0:                                           # nobody goes on
            self.lens, self.base = np.zeros(1, np.int64), torch.zeros(2, dtype=torch.int64, device="cuda")

    def compact(self):
        check(self.ctx, ro.ro_cache_compact(self.ctx, self.cache(), self.pages, self.refs, self.refs, self.n_used, self.moves))

    def step(self, tokens, news):
        """The next tokens of every sequence through the layer: logits of each one's last token."""
        T = int(np.sum(news))
        tok_base, tok_seq = self.expand(news)
        self.lens = self.lens + news
        length = u32(self.lens)
        place = u32(np.concatenate([np.arange(L - n, L) for L, n in zip(self.lens, news)]))[:, None]
        qkv = (self.embed[tokens.long()] @ self.into).view(T, HEADS + 2 * KV_HEADS, DIM)
        q = qkv[:, :HEADS]
        rows = torch.empty(T, HEADS, DIM, dtype=torch.float16, device="cuda")
        cache = self.cache()
        check(self.ctx, ro.ro_cache_append(self.ctx, cache, tok_base, tok_seq, length, place, self.rope, q, q,
                                           qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]))
        check(self.ctx, ro.ro_cache_attend_biased(self.ctx, cache, tok_base, int(np.max(news)), length, int(self.lens.max()),
                                                  q, 1 / math.sqrt(DIM), 0, 0, ro.ro_bias(CAP), rows))
        return rows[(tok_base[1:] - 1)].view(-1, HEADS * DIM) @ self.back

    def draw(self, logits, how, u):
        token, kept = (torch.zeros(logits.shape[0], dtype=torch.int32, device="cuda") for _ in range(2))
        logp = torch.zeros(logits.shape[0], device="cuda")
        check(self.ctx, ro.ro_sample(self.ctx, logits, how, u, token, logp, kept))
        return token


def run(prompts=8, samples=3, steps=24, vocab=600, seed=0):
    """Returns each sample's tokens (its prompt's first), the draws (logits, settings, random number, token), the
    logits of each sample's last step, pages in use at the end, and the model."""
    rng = np.random.default_rng(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    text = [rng.integers(1, vocab, int(n)) for n in rng.integers(1, 90, prompts)]
    room = lambda L: L + steps + 1   # noqa: E731
    per = lambda L: -(-room(L) // PAGE)   # noqa: E731
    s = Server(int(sum((samples + 1) * per(len(t)) for t in text)) + 8, vocab, seed)
    s.fork([prompts], [len(t) for t in text])                       # the prompts' first pages
    logits = s.step(u32(np.concatenate(text)), np.array([len(t) for t in text]))
    s.fork([samples] * prompts, [room(len(t)) for t in text for _ in range(samples)])
    of = np.repeat(np.arange(prompts), samples)
    logits = logits[torch.as_tensor(of, device="cuda")].contiguous()
    out = [list(text[p]) for p in of]
    alive = np.arange(len(of))
    settings = [rng.uniform(0.7, 1.2, len(of)).astype(np.float32), rng.integers(0, 60, len(of)),
                rng.uniform(0.8, 1.0, len(of)).astype(np.float32), rng.uniform(0.0, 0.05, len(of)).astype(np.float32)]
    draws, last = [], {}
    for i in range(steps):
        t, k, p, m = (x[alive] for x in settings)
        how = ro.ro_sampling(torch.tensor(t).cuda(), u32(k), torch.tensor(p).cuda(), torch.tensor(m).cuda())
        u = torch.rand(len(alive), generator=g, device="cuda")
        token = s.draw(logits, how, u)
        got = token.cpu().numpy()
        draws.append((logits, (t, k, p, m), u, got))
        go = got != END
        for j, x in zip(alive[go], got[go]):
            out[j].append(int(x))
        if not go.all():                                             # the others give their pages back
            s.fork(go.astype(np.int64), [per(len(text[of[j]])) * PAGE for j in alive[go]])
            alive, token = alive[go], token[torch.as_tensor(go, device="cuda")]
        if len(alive) == 0:
            break
        if i % 8 == 7:
            s.compact()
        logits = s.step(token, np.ones(len(alive), np.int64))
        for row, j in enumerate(alive):
            last[int(j)] = (len(out[j]), logits[row])
    s.compact()
    check(s.ctx, ro.ro_ctx_sync(s.ctx))
    refs = s.refs.cpu().numpy()
    ro.ro_ctx_destroy(s.ctx)
    used = int(s.n_used.item())
    assert (refs[:used] > 0).all() and (refs[used:] == 0).all()
    return out, draws, last, used, (s.embed, s.into, s.back)


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--prompts", type=int, default=8)
    ap.add_argument("--samples", type=int, default=3)
    ap.add_argument("--steps", type=int, default=24)
    a = ap.parse_args()
    out, draws, _, used, _ = run(a.prompts, a.samples, a.steps)
    print(f"{a.prompts} prompts, {len(out)} samples, {sum(len(d[3]) for d in draws)} tokens drawn; {used} pages in use at the end")


if __name__ == "__main__":
    main()
