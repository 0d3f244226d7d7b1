"""Frames of many videos through a Call's model step, on lineage arrays.

A microbatch of videos expands into frames.  Frames become ready in waves; each
wave is admitted and reserved (ro_batch_ready), its frames become one token
each (a record of fp16 x 256: 4 heads of 64), and the Call's step turns them:

  ro_expand_noalloc  videos -> the wave's tokens: token ranges and sequences
  ro_cache_append    rotary by (frame, row, column), keys and values into the
                     videos' pages; the pages are the children of another
                     expansion, videos -> pages
  ro_cache_attend    each token over its video's cache (window, first frames)
  ro_cache_weigh     the weight every cached frame gathered
  ro_cache_evict     caches past the budget are cut back to their heaviest
                     frames, in the other half of the pages

The attention's rows are the frames' results: committed out of the output
tensor (ro_gather_commit) and assembled per video in frame order (ro_assemble).

    python examples/stream_frames.py [--videos N] [--frames N] [--budget N]
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
RECORD = HEADS * DIM * 2   # bytes of a frame's result
SINKS, RECENT, WINDOW = 2, 16, 0


def check(ctx, status):
    if status != ro.RO_OK:
        raise ro.RoError("stream_frames", status, ro.ro_last_error(ctx))


def u32(x):
    return torch.as_tensor(np.asarray(x).astype(np.int32), device="cuda")


def inputs(videos, frames, seed):
    """Frames of each video (long-tailed), their records and places, and the step's projection."""
    rng = np.random.default_rng(seed)
    counts = np.clip(np.rint(rng.lognormal(math.log(frames), 0.6, videos)), 0, 4 * frames).astype(np.int64)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = int(counts.sum())
    records = torch.randn(n, HEADS * DIM, generator=g, device="cuda").half()
    weight = torch.randn(HEADS * DIM, (HEADS + 2 * KV_HEADS) * DIM, generator=g, device="cuda").half() / 16
    ordinal = np.concatenate([np.arange(c) for c in counts]) if n else np.zeros(0, np.int64)
    place = np.stack([ordinal, rng.integers(0, 24, n), rng.integers(0, 24, n)], 1)   # time, row, column
    return counts, records, u32(place), weight


def run(videos=64, frames=120, wave=24, budget=0, seed=0):
    """Returns (frames per video, each video's assembled records, cached frames per video at the end)."""
    counts, records, place, weight = inputs(videos, frames, seed)
    n, scale = records.shape[0], 1 / math.sqrt(DIM)
    budget = budget or int(counts.max())
    stream = torch.cuda.current_stream()
    ctx = ro.ro_ctx_create(torch.cuda.current_device(), stream, 1)
    rope = ro.ro_rope([16, 8, 8])

    # videos -> frames
    base = torch.zeros(videos + 1, dtype=torch.int64, device="cuda")
    parent, ordinal = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    st, _, _, xid = ro.ro_expand(ctx, -1, u32(counts), videos, None, base, parent, ordinal, n)
    check(ctx, st)
    # videos -> pages, twice over: a cache moves to the other half when it is cut back
    per = -(-(budget + wave) // PAGE)
    page_base = torch.zeros(videos + 1, dtype=torch.int64, device="cuda")
    page_of, page_ord = (torch.zeros(videos * per, dtype=torch.int32, device="cuda") for _ in range(2))
    st, n_pages, _ = ro.ro_expand_noalloc(u32([per] * videos), videos, page_base, page_of, page_ord, videos * per,
                                          stream=stream)
    check(ctx, st)
    halves = [u32(np.arange(n_pages) + h * n_pages) for h in (0, 1)]
    k = torch.zeros(2 * n_pages, KV_HEADS, PAGE, DIM, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    caches = [ro.ro_cache(k, v, page_base, h) for h in halves]
    half = 0

    length = torch.zeros(videos, dtype=torch.int32, device="cuda")
    score = torch.zeros(videos, KV_HEADS, per * PAGE, device="cuda")
    spare = torch.zeros_like(score)
    keep = torch.zeros(videos, KV_HEADS, budget, dtype=torch.int32, device="cuda")
    result = torch.zeros(n, HEADS, DIM, dtype=torch.float16, device="cuda")   # the arena of the frames' results
    batched, n_batched = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    status = torch.zeros(videos, dtype=torch.uint8, device="cuda")
    out_off = torch.zeros(videos + 1, dtype=torch.int64, device="cuda")
    out = torch.zeros(max(n * RECORD, 1), dtype=torch.uint8, device="cuda")
    starts = np.concatenate([[0], np.cumsum(counts)])
    lens = np.zeros(videos, np.int64)

    for w in range(-(-int(counts.max(initial=0)) // wave)):
        # the wave's frames, a video's together and in order
        first = np.minimum(w * wave, counts)
        new = np.minimum(counts - first, wave)
        cand = np.concatenate([np.arange(starts[i] + first[i], starts[i] + first[i] + new[i]) for i in range(videos)])
        T = cand.size
        st, got, _ = ro.ro_batch_ready(ctx, xid, 0, u32(cand), T, 256, True, batched, n, n_batched)
        check(ctx, st)
        frame = batched[:got].long()
        # videos -> the wave's tokens
        tok_base = torch.zeros(videos + 1, dtype=torch.int64, device="cuda")
        tok_seq, tok_ord = (torch.zeros(T, dtype=torch.int32, device="cuda") for _ in range(2))
        st, _, _ = ro.ro_expand_noalloc(u32(new), videos, tok_base, tok_seq, tok_ord, T, stream=stream)
        check(ctx, st)
        # the model step
        qkv = (records[frame] @ weight).view(T, HEADS + 2 * KV_HEADS, DIM)
        q = qkv[:, :HEADS]
        length += (tok_base[1:] - tok_base[:-1]).int()
        lens += new
        cache, rows = caches[half], torch.empty(T, HEADS, DIM, dtype=torch.float16, device="cuda")
        lse = torch.empty(T, HEADS, device="cuda")
        check(ctx, ro.ro_cache_append(ctx, cache, tok_base, tok_seq, length, place[frame], rope, q, q,
                                      qkv[:, HEADS:HEADS + KV_HEADS], qkv[:, HEADS + KV_HEADS:]))
        check(ctx, ro.ro_cache_attend(ctx, cache, tok_base, wave, length, int(lens.max()), q, scale, WINDOW, SINKS, rows,
                                      lse))
        check(ctx, ro.ro_cache_weigh(ctx, cache, tok_base, wave, length, q, scale, WINDOW, SINKS, lse, 1.0, score, score))
        if lens.max() > budget:
            check(ctx, ro.ro_cache_evict(ctx, cache, length, score, budget, SINKS, min(RECENT, budget - SINKS), page_base,
                                         halves[1 - half], keep, length, spare))
            half, score, spare = 1 - half, spare, score
            lens = np.minimum(lens, budget)
        result[frame] = rows
        # the frames' results, and the videos they complete
        reports = torch.full((T,), ro.RO_PRESENT, dtype=torch.uint8, device="cuda")
        st, _ = ro.ro_gather_commit(ctx, xid, T, None, batched, reports, u32([RECORD] * T), frame * RECORD, None,
                                    n * RECORD)
        check(ctx, st)
    listed = u32(np.arange(videos))
    st, total = ro.ro_assemble(ctx, xid, result.view(torch.uint8), n * RECORD, listed, videos, None, status, out_off, None,
                               out, n * RECORD)
    check(ctx, st)
    check(ctx, ro.ro_ctx_sync(ctx))
    ro.ro_ctx_destroy(ctx)
    at = out_off.tolist()
    assert total == n * RECORD and status.tolist() == [ro.RO_PRESENT] * videos
    videos_out = [out[at[i]:at[i] + int(counts[i]) * RECORD].view(torch.float16).view(-1, HEADS, DIM) for i in range(videos)]
    return counts, videos_out, length.tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--videos", type=int, default=64)
    ap.add_argument("--frames", type=int, default=120, help="median frames of a video")
    ap.add_argument("--budget", type=int, default=100, help="cached frames a video keeps")
    a = ap.parse_args()
    counts, outs, held = run(a.videos, a.frames, budget=a.budget)
    print(f"{a.videos} videos, {int(counts.sum())} frames, {sum(o.numel() * 2 for o in outs)} bytes assembled; "
          f"cached frames a video: at most {max(held)}")


if __name__ == "__main__":
    main()
