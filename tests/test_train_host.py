"""Training entry points on the host (no GPU needed): exports, refusals, and the arithmetic of the checks and size
queries under the undefined-behaviour sanitizer."""
import ctypes
import itertools
import os
import re
import subprocess
import sys
import textwrap

import pytest
import torch

from test_host_sanitizer import sanitized_library  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "moegps_train.h")


def test_library_exports_every_training_call():
    from paper_2506_07366_amd import binding
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", src)))
    assert names == sorted(binding.EXPORTS_TRAIN)
    lib = binding.load_library()
    for n in names:
        assert hasattr(lib, n) and hasattr(binding, n), n


OK, INVALID, UNSUPPORTED = 0, -1, -2
P = 16  # a pointer that is never followed


def lib():
    from paper_2506_07366_amd import binding
    return binding.load_library()


@pytest.mark.parametrize("name", ["moe_checkpoint_store", "moe_checkpoint_load"])
def test_checkpoint_refusals(name):
    fn = getattr(lib(), name)

    def call(dtype=1, rows=4, d=64, a=P, b=P, c=P):
        if name.endswith("store"):
            return fn(a, dtype, rows, d, b, c, None)
        return fn(a, b, rows, d, c, dtype, None)

    assert call(dtype=2) == INVALID and call(rows=-1) == INVALID and call(d=0) == INVALID
    assert call(d=12) == UNSUPPORTED and call(dtype=0, d=2) == UNSUPPORTED
    assert call(rows=2**31) == UNSUPPORTED and call(d=2**22 + 8) == UNSUPPORTED
    assert call(a=None) == INVALID and call(b=None) == INVALID and call(c=None) == INVALID
    assert call(rows=0, a=None, b=None, c=None) == OK


def test_combine_backward_refusals():
    names = ("dout", "dtype", "T", "d", "k", "E", "row_of_assign", "topk_w", "topk_idx", "y", "scales", "dy", "dw", "dl")
    good = dict(dout=P, dtype=1, T=4, d=64, k=2, E=8, row_of_assign=P, topk_w=P, topk_idx=P, y=P, scales=None, dy=P, dw=P,
                dl=P)

    def call(**kw):
        a = {**good, **kw}
        return lib().moe_combine_backward(*(a[n] for n in names), None)

    assert call(dtype=7) == INVALID and call(T=-1) == INVALID and call(d=0) == INVALID and call(k=0) == INVALID
    assert call(k=17) == UNSUPPORTED and call(d=60) == UNSUPPORTED and call(T=2**30) == UNSUPPORTED
    assert call(E=1) == INVALID and call(E=2000) == UNSUPPORTED and call(topk_idx=None) == INVALID
    assert call(y=None) == INVALID                              # dw wanted, nothing to make it from
    assert call(y=None, scales=P) == INVALID
    assert call(dw=None) == INVALID and call(dw=None, dl=None) == INVALID
    for n in ("dout", "row_of_assign", "topk_w", "dy"):
        assert call(**{n: None}) == INVALID
    assert call(T=0, dout=None, dy=None) == OK


def test_python_checks_name_the_tensor():
    """Tensors of the wrong kind are refused before a pointer is taken (CPU tensors are never accepted)."""
    from paper_2506_07366_amd import binding as B
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(B.MoeGpsError, match="x must be a GPU tensor"):
        B.moe_checkpoint_store(x)
    with pytest.raises(B.MoeGpsError, match="unsupported dtype"):
        B.moe_checkpoint_store(x.half())
    with pytest.raises(B.MoeGpsError, match="dout must be a GPU tensor"):
        B.moe_combine_backward(x, None, torch.zeros(8, dtype=torch.int32), torch.zeros((4, 2)))


CHILD = textwrap.dedent('''
    import ctypes, itertools, sys
    lib = ctypes.CDLL(sys.argv[1])
    c_int, c_i64, vp = ctypes.c_int, ctypes.c_int64, ctypes.c_void_p
    I32 = [0, 1, -1, 2, 7, 64, 4096, 65536, 2**20, 2**24 + 1, 2**31 - 1, -2**31]
    I64 = I32 + [2**31, 2**40, 2**62, 2**63 - 1, -2**63]
    for dtype, rows, d in itertools.product([0, 1, 2], I64, I32):   # (no pointers: refused or empty)
        lib.moe_checkpoint_store.argtypes = [vp, c_int, c_i64, c_int, vp, vp, vp]
        lib.moe_checkpoint_load.argtypes = [vp, vp, c_i64, c_int, vp, c_int, vp]
        r = lib.moe_checkpoint_store(None, dtype, rows, d, None, None, None)
        assert r != 0 or rows == 0, (dtype, rows, d)
        assert lib.moe_checkpoint_load(None, None, rows, d, None, dtype, None) == r
    lib.moe_combine_backward.argtypes = [vp] + [c_int] * 5 + [vp] * 9
    for dtype, T, d, k, E in itertools.product([0, 1, 2], I32, I32, [0, 1, 2, 16, 17, 2**31 - 1], [0, 2, 1024, 2**31 - 1]):
        for dl in (None, 16):
            r = lib.moe_combine_backward(None, dtype, T, d, k, E, None, None, None, None, None, None, dl, dl, None)
            assert r != 0 or T == 0, (dtype, T, d, k, E)
    print("training checks ok", flush=True)
''')


def test_host_arithmetic_of_the_training_calls(sanitized_library, tmp_path):  # noqa: F811
    script = tmp_path / "child.py"
    script.write_text(CHILD)
    r = subprocess.run([sys.executable, str(script), sanitized_library], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, f"child ended with {r.returncode}\n{r.stdout[-1500:]}\n{r.stderr[-2000:]}"
    assert "training checks ok" in r.stdout
