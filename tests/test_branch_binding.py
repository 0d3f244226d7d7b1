"""The parts of biased attention, page operations and sampling that need no GPU:
struct layouts against the header, calls without a context, and what the binding
looks at before it calls the library."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2609_18703_gb300 as ro  # noqa: E402
from paper_2609_18703_gb300 import build  # noqa: E402
from tests.test_step_abi import test_struct_layout as check_layout  # noqa: E402
from tests.test_step_binding import BF16, F32, I32, I64, Library, OnGpu, library  # noqa: E402,F401

SEQS, KV, HEADS, DIM, TOKENS, PAGES, KIDS, ENTRIES, ROWS, VOCAB = 3, 2, 4, 64, 5, 6, 4, 7, 3, 50


@pytest.mark.parametrize("struct", ["ro_bias", "ro_moves", "ro_sampling"])
def test_struct_layouts(struct, tmp_path):
    check_layout(struct, tmp_path)


def test_calls_without_a_context_are_refused():
    build.build()
    lib = ro.load()
    for fn in ("ro_cache_attend_biased", "ro_cache_fork", "ro_cache_compact", "ro_cache_copy", "ro_sample"):
        f = getattr(lib, fn)
        args = [t() if t not in (ctypes.c_float,) else 0.0 for t in f.argtypes]
        assert f(*args) == ro.RO_E_INVAL


def moves(n=PAGES, count=1):
    return ro.ro_moves(OnGpu(n, dtype=I32), OnGpu(n, dtype=I32), OnGpu(n, dtype=I32), OnGpu(count, dtype=I32))


def arguments():
    cache = ro.ro_cache(OnGpu(PAGES, KV, 16, DIM), OnGpu(PAGES, KV, 16, DIM), OnGpu(SEQS + 1, dtype=I64), OnGpu(6, dtype=I32))
    i32 = lambda n: OnGpu(n, dtype=I32)   # noqa: E731
    f32 = lambda n: OnGpu(n, dtype=F32)   # noqa: E731
    return {
        "ro_cache_attend_biased": dict(cache=cache, d_tok_base=OnGpu(SEQS + 1, dtype=I64), max_new=TOKENS, d_len=i32(SEQS),
                                       max_len=32, d_q=OnGpu(TOKENS, HEADS, DIM), scale=0.1, window=0, sinks=0,
                                       bias=ro.ro_bias(1.0, f32(HEADS), i32(TOKENS), i32(TOKENS)),
                                       d_out=OnGpu(TOKENS, HEADS, DIM), d_lse=OnGpu(TOKENS, HEADS, dtype=F32)),
        "ro_cache_fork": dict(cache=cache, d_len=i32(SEQS), d_child_base=OnGpu(SEQS + 1, dtype=I64), d_child_parent=i32(KIDS),
                              d_dst_base=OnGpu(KIDS + 1, dtype=I64), d_dst_seq=i32(ENTRIES), d_dst_pages=i32(ENTRIES),
                              d_len_out=i32(KIDS), d_refs=i32(PAGES), d_refs_out=i32(PAGES), moves=moves()),
        "ro_cache_compact": dict(cache=cache, d_pages_out=i32(6), d_refs=i32(PAGES), d_refs_out=i32(PAGES), d_n_used=i32(1),
                                 moves=moves()),
        "ro_cache_copy": dict(cache=cache, moves=moves()),
        "ro_sample": dict(d_logits=OnGpu(ROWS, VOCAB, dtype=F32), how=ro.ro_sampling(f32(ROWS), i32(ROWS), f32(ROWS), f32(ROWS)),
                          d_u=f32(ROWS), d_token=i32(ROWS), d_logp=f32(ROWS), d_kept=i32(ROWS)),
    }


@pytest.mark.parametrize("fn", sorted(arguments()))
def test_arguments_that_fit_are_passed(library, fn):   # noqa: F811
    assert getattr(ro, fn)(1, **arguments()[fn]) == ro.RO_OK and library.calls == [fn]


def test_settings_may_be_left_out(library):   # noqa: F811
    a = arguments()["ro_sample"]
    a.update(how=None, d_logp=None, d_kept=None)
    assert ro.ro_sample(1, **a) == ro.RO_OK
    a.update(how=ro.ro_sampling())
    assert ro.ro_sample(1, **a) == ro.RO_OK
    a = arguments()["ro_cache_attend_biased"]
    a.update(bias=ro.ro_bias(), d_lse=None)
    assert ro.ro_cache_attend_biased(1, **a) == ro.RO_OK


SHORT = [("ro_cache_attend_biased", "d_tok_base", SEQS, I64), ("ro_cache_attend_biased", "d_len", SEQS - 1, I32),
         ("ro_cache_fork", "d_len", SEQS - 1, I32), ("ro_cache_fork", "d_child_base", SEQS, I64),
         ("ro_cache_fork", "d_dst_base", KIDS, I64), ("ro_cache_fork", "d_dst_pages", ENTRIES - 1, I32),
         ("ro_cache_fork", "d_len_out", KIDS - 1, I32), ("ro_cache_fork", "d_refs", PAGES - 1, I32),
         ("ro_cache_fork", "d_refs_out", PAGES - 1, I32), ("ro_cache_compact", "d_refs", PAGES - 1, I32),
         ("ro_cache_compact", "d_refs_out", PAGES - 1, I32), ("ro_cache_compact", "d_n_used", 0, I32),
         ("ro_sample", "d_u", ROWS - 1, F32), ("ro_sample", "d_token", ROWS - 1, I32), ("ro_sample", "d_logp", ROWS - 1, F32),
         ("ro_sample", "d_kept", ROWS - 1, I32)]


@pytest.mark.parametrize("fn,name,n,dtype", SHORT)
def test_arrays_too_short_are_refused(library, fn, name, n, dtype):   # noqa: F811
    a = arguments()[fn]
    a[name] = OnGpu(n, dtype=dtype)
    with pytest.raises(ValueError):
        getattr(ro, fn)(1, **a)
    assert library.calls == []


def test_descriptions_too_short_are_refused(library):   # noqa: F811
    a = arguments()
    for bias in (ro.ro_bias(1.0, OnGpu(HEADS - 1, dtype=F32)), ro.ro_bias(1.0, None, OnGpu(TOKENS - 1, dtype=I32)),
                 ro.ro_bias(1.0, None, None, OnGpu(TOKENS - 1, dtype=I32))):
        with pytest.raises(ValueError):
            ro.ro_cache_attend_biased(1, **dict(a["ro_cache_attend_biased"], bias=bias))
    for how in (ro.ro_sampling(OnGpu(ROWS - 1, dtype=F32)), ro.ro_sampling(None, OnGpu(ROWS - 1, dtype=I32))):
        with pytest.raises(ValueError):
            ro.ro_sample(1, **dict(a["ro_sample"], how=how))
    with pytest.raises(ValueError):
        ro.ro_cache_fork(1, **dict(a["ro_cache_fork"], moves=moves(KIDS - 1)))
    with pytest.raises(ValueError):
        ro.ro_cache_compact(1, **dict(a["ro_cache_compact"], moves=moves(PAGES // 2 - 1)))
    with pytest.raises(ValueError):
        moves(PAGES, 0)
    assert library.calls == []


@pytest.mark.parametrize("fn,name", [(fn, n) for fn, a in sorted(arguments().items()) for n, x in a.items()
                                     if isinstance(x, OnGpu) and x.dtype is not BF16 and n != "d_logits"])
def test_elements_of_another_type_are_refused(library, fn, name):   # noqa: F811
    a = arguments()[fn]
    a[name] = OnGpu(*a[name].shape, dtype={I32: F32, I64: torch.float64, F32: I32}[a[name].dtype])
    with pytest.raises(ValueError):
        getattr(ro, fn)(1, **a)
    assert library.calls == []


def test_descriptions_of_another_type_are_refused():
    for bad in (lambda: ro.ro_bias(1.0, OnGpu(4, dtype=I32)), lambda: ro.ro_bias(1.0, None, OnGpu(4, dtype=I64)),
                lambda: ro.ro_bias(1.0, None, None, OnGpu(4, dtype=F32)), lambda: ro.ro_sampling(OnGpu(4, dtype=I32)),
                lambda: ro.ro_sampling(None, OnGpu(4, dtype=I64)), lambda: ro.ro_sampling(None, None, OnGpu(4, dtype=torch.float64)),
                lambda: ro.ro_moves(OnGpu(4, dtype=I64), OnGpu(4, dtype=I32), OnGpu(4, dtype=I32), OnGpu(1, dtype=I32))):
        with pytest.raises(ValueError):
            bad()


def test_logits_of_another_layout_are_refused(library):   # noqa: F811
    a = arguments()["ro_sample"]
    for x in (OnGpu(ROWS, VOCAB, dtype=torch.float64), OnGpu(ROWS, VOCAB, dtype=I32)):
        with pytest.raises(ValueError):
            ro.ro_sample(1, **dict(a, d_logits=x))
    turned = OnGpu(VOCAB, ROWS, dtype=F32)
    turned._t = turned._t.t()
    with pytest.raises(ValueError):
        ro.ro_sample(1, **dict(a, d_logits=turned))
    assert library.calls == []
