"""What the model-step binding looks at before it calls the library: sizes and
element types of every array, on the CPU, with stand-ins for GPU tensors and a
library that only notes that it was called."""
import pytest

torch = pytest.importorskip("torch")

import paper_2609_18703_gb300 as ro  # noqa: E402
from paper_2609_18703_gb300 import _binding  # noqa: E402

BF16, I32, I64, F32 = torch.bfloat16, torch.int32, torch.int64, torch.float32


class OnGpu:
    """A tensor as the binding sees one that lies on a GPU."""
    is_cuda = True

    def __init__(self, *shape, dtype=BF16):
        self._t = torch.zeros(*shape, dtype=dtype)

    def __getattr__(self, name):
        return getattr(self._t, name)


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or ro.RO_OK


SEQS, KV, HEADS, DIM, TOKENS, SLOTS, BUDGET = 3, 2, 4, 64, 5, 32, 8


def arguments():
    """Every operator's arguments by name, in the order of its call."""
    k = OnGpu(6, KV, 16, DIM)
    cache = ro.ro_cache(k, OnGpu(6, KV, 16, DIM), OnGpu(SEQS + 1, dtype=I64), OnGpu(6, dtype=I32))
    rows = lambda heads: OnGpu(TOKENS, heads, DIM)   # noqa: E731
    tok_base, length, rope = OnGpu(SEQS + 1, dtype=I64), OnGpu(SEQS, dtype=I32), ro.ro_rope([16, 16])
    pos, score = OnGpu(TOKENS, 2, dtype=I32), OnGpu(SEQS, KV, SLOTS, dtype=F32)
    return {
        "ro_rotary": dict(d_x=rows(HEADS), d_out=rows(HEADS), d_pos=pos, rope=rope),
        "ro_cache_append": dict(cache=cache, d_tok_base=tok_base, d_tok_seq=OnGpu(TOKENS, dtype=I32), d_len=length,
                                d_pos=pos, rope=rope, d_q=rows(HEADS), d_q_out=rows(HEADS), d_k=rows(KV), d_v=rows(KV)),
        "ro_cache_attend": dict(cache=cache, d_tok_base=tok_base, max_new=TOKENS, d_len=length, max_len=SLOTS,
                                d_q=rows(HEADS), scale=0.1, window=0, sinks=0, d_out=rows(HEADS),
                                d_lse=OnGpu(TOKENS, HEADS, dtype=F32)),
        "ro_cache_weigh": dict(cache=cache, d_tok_base=tok_base, max_new=TOKENS, d_len=length, d_q=rows(HEADS), scale=0.1,
                               window=0, sinks=0, d_lse=OnGpu(TOKENS, HEADS, dtype=F32), decay=1.0, d_past=score,
                               d_score=score),
        "ro_cache_evict": dict(cache=cache, d_len=length, d_score=score, budget=BUDGET, sinks=0, recent=0,
                               d_dst_base=OnGpu(SEQS + 1, dtype=I64), d_dst_pages=OnGpu(3, dtype=I32),
                               d_keep=OnGpu(SEQS, KV, BUDGET, dtype=I32), d_len_out=OnGpu(SEQS, dtype=I32)),
    }


@pytest.fixture
def library(monkeypatch):
    lib = Library()
    monkeypatch.setattr(_binding, "_lib", lib)
    return lib


@pytest.mark.parametrize("fn", sorted(arguments()))
def test_arguments_that_fit_are_passed(library, fn):
    assert getattr(ro, fn)(1, **arguments()[fn]) == ro.RO_OK and library.calls == [fn]


def test_longer_arrays_and_unsigned_types_are_passed(library):
    a = arguments()["ro_cache_attend"]
    a.update(d_tok_base=OnGpu(SEQS + 9, dtype=torch.uint64), d_len=OnGpu(SEQS + 4, dtype=torch.uint32))
    assert ro.ro_cache_attend(1, **a) == ro.RO_OK
    a = arguments()["ro_cache_append"]
    a.update(d_pos=None, rope=None)
    assert ro.ro_cache_append(1, **a) == ro.RO_OK
    a = arguments()["ro_cache_evict"]
    a.update(d_len=4096, d_len_out=8192)   # addresses are the caller's own affair
    assert ro.ro_cache_evict(1, **a) == ro.RO_OK and len(library.calls) == 3


SHORT = [(fn, name, n, dt) for fn, name, n, dt in (
    ("ro_cache_append", "d_tok_base", SEQS, I64), ("ro_cache_append", "d_len", SEQS - 1, I32),
    ("ro_cache_append", "d_tok_seq", TOKENS - 1, I32), ("ro_cache_attend", "d_tok_base", SEQS, I64),
    ("ro_cache_attend", "d_len", SEQS - 1, I32), ("ro_cache_weigh", "d_tok_base", SEQS, I64),
    ("ro_cache_weigh", "d_len", SEQS - 1, I32), ("ro_cache_evict", "d_len", SEQS - 1, I32),
    ("ro_cache_evict", "d_len_out", SEQS - 1, I32), ("ro_cache_evict", "d_dst_base", SEQS, I64))]


@pytest.mark.parametrize("fn,name,n,dtype", SHORT)
def test_arrays_too_short_are_refused(library, fn, name, n, dtype):
    a = arguments()[fn]
    a[name] = OnGpu(n, dtype=dtype)
    with pytest.raises(ValueError):
        getattr(ro, fn)(1, **a)
    assert library.calls == []


@pytest.mark.parametrize("fn,name", [(fn, n) for fn, a in sorted(arguments().items()) for n, x in a.items()
                                     if isinstance(x, OnGpu) and x.dtype is not BF16])
def test_elements_of_another_type_are_refused(library, fn, name):
    """The same size, another type: floats for integers, integers for floats."""
    a = arguments()[fn]
    a[name] = OnGpu(*a[name].shape, dtype={I32: F32, I64: torch.float64, F32: I32}[a[name].dtype])
    with pytest.raises(ValueError):
        getattr(ro, fn)(1, **a)
    assert library.calls == []


@pytest.mark.parametrize("base,pages", [(torch.float64, I32), (I64, F32), (I32, I32)])
def test_page_lists_of_another_type_are_refused(base, pages):
    k = OnGpu(6, KV, 16, DIM)
    with pytest.raises(ValueError):
        ro.ro_cache(k, k, OnGpu(SEQS + 1, dtype=base), OnGpu(6, dtype=pages))


@pytest.mark.parametrize("fn,name", [("ro_rotary", "d_out"), ("ro_cache_append", "d_q"), ("ro_cache_append", "d_v"),
                                     ("ro_cache_append", "d_k"), ("ro_cache_append", "d_q_out"), ("ro_cache_attend", "d_q"),
                                     ("ro_cache_attend", "d_out"), ("ro_cache_weigh", "d_q")])
def test_rows_of_another_shape_or_type_are_refused(library, fn, name):
    for change in (lambda s: OnGpu(s[0], s[1], s[2] + 8), lambda s: OnGpu(*s, dtype=torch.float16),
                   lambda s: OnGpu(s[0] + 1, s[1], s[2]), lambda s: OnGpu(s[0], s[1] * s[2])):
        a = arguments()[fn]
        a[name] = change(a[name].shape)
        with pytest.raises(ValueError):
            getattr(ro, fn)(1, **a)
    a = arguments()[fn]
    wide = {n: OnGpu(*x.shape[:2], DIM + 8) for n, x in a.items() if isinstance(x, OnGpu) and x.dtype is BF16}
    if fn != "ro_rotary":   # every row alike, but not the cache's
        a.update(wide)
        with pytest.raises(ValueError):
            getattr(ro, fn)(1, **a)
    assert library.calls == []
