"""Training entry points on the host (no GPU needed): exports, refusals, and the arithmetic of the checks and size
queries under the undefined-behaviour sanitizer."""
import os
import re
import subprocess
import sys
import textwrap

import pytest
import torch

from test_host_sanitizer import _hipcc

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


FFN_FIELDS = ("dtype", "T", "k", "d", "ffn", "E", "nseg", "relu", "x", "x_scales", "assign_of_row", "seg_offsets",
              "slot_expert", "packed", "packed_backward", "dy", "dx", "dW1", "dW3", "dW2", "workspace", "workspace_bytes")
FFN_GOOD = dict(dtype=1, T=4, k=2, d=64, ffn=64, E=8, nseg=16, relu=0, x=P, x_scales=0, assign_of_row=P, seg_offsets=P,
                slot_expert=P, packed=P, packed_backward=P, dy=P, dx=P, dW1=P, dW3=P, dW2=P, workspace=P, workspace_bytes=0)


def ffn_backward(**kw):
    from paper_2506_07366_amd import binding
    a = {**FFN_GOOD, **kw}
    return lib().moe_grouped_ffn_backward(binding._FFN_BACKWARD_ARGS.pack(*(a[n] for n in FFN_FIELDS)), None)


def test_ffn_backward_refusals():
    WORKSPACE = -3
    assert lib().moe_grouped_ffn_backward(None, None) == INVALID
    assert ffn_backward() == WORKSPACE                                     # all else is in order
    for field in ("T", "k", "d", "ffn", "E", "nseg"):
        assert ffn_backward(**{field: -1}) == INVALID
    assert ffn_backward(dtype=2) == INVALID
    for kw in (dict(k=17), dict(E=1025), dict(nseg=2049), dict(d=2**22 + 64), dict(ffn=2**22 + 1), dict(d=72),
               dict(dtype=0, d=66), dict(dtype=0, ffn=66), dict(T=2**30), dict(T=2**24, d=64, k=2), dict(d=2**22)):
        assert ffn_backward(**kw) == UNSUPPORTED, kw
    for field in ("x", "assign_of_row", "seg_offsets", "slot_expert", "packed", "packed_backward", "dy", "workspace", "dW1",
                  "dW3", "dW2"):
        assert ffn_backward(**{field: 0}) == INVALID, field
    assert ffn_backward(relu=1) == INVALID                                 # no third matrix in the ReLU form
    assert ffn_backward(relu=1, dW3=0) == WORKSPACE
    assert ffn_backward(dtype=0, packed_backward=0) == WORKSPACE           # fp32 reads the forward pass's form
    none = dict(dx=0, dW1=0, dW3=0, dW2=0, workspace_bytes=1 << 30)
    assert ffn_backward(**none) == OK                                      # nothing wanted, nothing enqueued
    assert ffn_backward(T=0, x=0, dy=0, dx=0, dW1=0, dW3=0, dW2=0, workspace_bytes=1 << 30) == OK


def test_ffn_backward_sizes():
    size = lib().moe_grouped_ffn_backward_workspace_bytes
    A, T, d, ffn = 8192, 4096, 4096, 14336
    assert size(T, 2, d, ffn, 8, 16, 1, 0) >= 2 * (T * d + 3 * A * ffn)
    assert size(T, 2, d, ffn, 8, 16, 1, 1) < size(T, 2, d, ffn, 8, 16, 1, 0)
    assert size(0, 2, d, ffn, 8, 16, 1, 0) > 0 and size(-1, 2, d, ffn, 8, 16, 1, 0) == 0
    assert size(T, 0, d, ffn, 8, 16, 1, 0) == 0 and size(T, 2, d, ffn, 8, 16, 2, 0) == 0
    packed = lib().moe_packed_weights_backward_bytes
    assert packed(8, d, ffn, 1, 0) == 3 * 8 * d * ffn * 2                  # whole tiles: no padding
    assert packed(8, d, ffn, 1, 1) == 2 * 8 * d * ffn * 2
    assert packed(1, 64, 8, 1, 0) == 2 * (256 * 64 + 256 * 128)
    assert packed(8, d, ffn, 0, 0) == 0 and packed(0, d, ffn, 1, 0) == 0
    pack = lib().moe_pack_weights_backward
    assert pack(P, P, P, 0, 8, 128, 128, None, None) == OK                 # fp32: nothing to do
    assert pack(P, P, P, 1, 8, 100, 128, P, None) == UNSUPPORTED and pack(P, P, P, 1, 2000, 128, 128, P, None) == UNSUPPORTED
    assert pack(None, P, P, 1, 8, 128, 128, P, None) == INVALID and pack(P, P, P, 3, 8, 128, 128, P, None) == INVALID


@pytest.fixture(scope="module")
def sanitized_training_library(tmp_path_factory):
    """The host pass alone of what the training calls need, trapping on undefined behaviour."""
    hipcc = _hipcc()
    if hipcc is None:
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("ubsan_train")
    flags = ["--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-Wno-unused-command-line-argument",
             "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fsanitize-trap=undefined"]
    objs, procs = [], []
    for name in ("api", "checkpoint", "combine_backward", "ffn_backward", "grouped_ffn"):
        objs.append(str(out / (name + ".o")))
        src = os.path.join(ROOT, "paper_2506_07366_amd", "csrc", name + ".hip")
        procs.append(subprocess.Popen([hipcc, *flags, "-c", src, "-o", objs[-1]], stdout=subprocess.PIPE,
                                      stderr=subprocess.PIPE, text=True))
    for p in procs:
        _, err = p.communicate()
        assert p.returncode == 0, err
    # the device code that the objects refer to and nothing here launches: empty
    undefined = subprocess.run(["nm", "-u", *objs], capture_output=True, text=True).stdout
    stub = out / "no_device_code.c"
    stub.write_text("".join(f"const char {n}[4096] = {{0}};\n" for n in sorted(set(re.findall(r"__hip_fatbin_\w+", undefined)))))
    path = str(out / "libtrain_ubsan.so")
    r = subprocess.run([hipcc, "-shared", "-fPIC", "-x", "c", str(stub), "-x", "none", *objs, "-o", path],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    return path


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
    c_sz = ctypes.c_size_t
    lib.moe_packed_weights_backward_bytes.restype = c_sz
    lib.moe_grouped_ffn_backward_workspace_bytes.restype = c_sz
    for E, d, ffn, dtype, relu in itertools.product(I32, I32, I32, [0, 1, 2], [0, 1]):
        lib.moe_packed_weights_backward_bytes(E, d, ffn, dtype, relu)
        r = lib.moe_pack_weights_backward(None, None, None, dtype, E, d, ffn, None, None)
        assert r != 0 or dtype == 0, (E, d, ffn)
    for T, d, ffn in itertools.product(I32, I32, I32):
        for k, E, nseg, dtype, relu in itertools.product([0, 1, 16, 2**31 - 1], [1, 1024, 2**31 - 1], [1, 2048, 2**31 - 1], [0, 1], [0, 1]):
            lib.moe_grouped_ffn_backward_workspace_bytes(T, k, d, ffn, E, nseg, dtype, relu)
    import struct
    lib.moe_grouped_ffn_backward.argtypes = [ctypes.c_char_p, vp]
    def call(*ints):
        return lib.moe_grouped_ffn_backward(struct.pack("@8i14Q", *ints, *[0] * 14), None)
    good = [1, 16, 2, 64, 64, 8, 16, 0]
    for i in range(8):
        for v in I32:
            assert call(*good[:i], v, *good[i + 1:]) != 0
    big = [1, 2**31 - 1, 16, 2**22, 2**22, 1024, 2048, 0]
    for fields in itertools.product([0, 1], repeat=8):
        assert call(*(b if f else g for f, g, b in zip(fields, good, big))) != 0
    print("training checks ok", flush=True)
''')


def test_host_arithmetic_of_the_training_calls(sanitized_training_library, tmp_path):
    script = tmp_path / "child.py"
    script.write_text(CHILD)
    r = subprocess.run([sys.executable, str(script), sanitized_training_library], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, f"child ended with {r.returncode}\n{r.stdout[-1500:]}\n{r.stderr[-2000:]}"
    assert "training checks ok" in r.stdout
