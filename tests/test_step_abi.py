"""The binding's structs lie as the header's (compiled with the host compiler),
and the parts of the model-step operators that need no GPU."""
import ctypes
import os
import subprocess

import pytest

torch = pytest.importorskip("torch")

import paper_2609_18703_gb300 as ro  # noqa: E402
from paper_2609_18703_gb300 import build  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("struct", ["ro_rope", "ro_cache"])
def test_struct_layout(struct, tmp_path):
    cls = getattr(ro, struct)
    names = [n for n, _ in cls._fields_]
    src = tmp_path / "layout.c"
    lines = "".join(f'printf("%zu %zu\\n", offsetof({struct}, {n}), sizeof((({struct}*)0)->{n}));' for n in names)
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "rayorch_cache.h"\n'
                   f'int main(void) {{ {lines} printf("%zu 0\\n", sizeof({struct})); return 0; }}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    rows = [tuple(map(int, r.split())) for r in subprocess.check_output([str(exe)], text=True).splitlines()]
    assert rows[-1][0] == ctypes.sizeof(cls)
    for n, (off, size) in zip(names, rows):
        f = getattr(cls, n)
        assert (f.offset, f.size) == (off, size), n


def test_calls_without_a_context_are_refused():
    build.build()
    lib = ro.load()
    for fn in ("ro_rotary", "ro_cache_append", "ro_cache_attend", "ro_cache_weigh", "ro_cache_evict"):
        f = getattr(lib, fn)
        args = [t() if t not in (ctypes.c_float,) else 0.0 for t in f.argtypes]
        assert f(*args) == ro.RO_E_INVAL


def test_rope_takes_one_to_four_axes():
    r = ro.ro_rope([16, 24, 24], base=1e6, interleaved=True)
    assert (r.n_axes, list(r.pairs), r.interleaved, r.base) == (3, [16, 24, 24, 0], 1, 1e6)
    for bad in ([], [1] * 5):
        with pytest.raises(ValueError):
            ro.ro_rope(bad)


def test_cpu_tensors_are_refused():
    k = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        ro.ro_cache(k, k, torch.zeros(2, dtype=torch.int64), torch.zeros(2, dtype=torch.int32))
