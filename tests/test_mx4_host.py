"""Weights in 4 bits, what the host side says: sizes, refusals (no GPU needed), and the oracle's own rounding."""
import ctypes
import re
import struct

import numpy as np
import pytest
import torch

import mx4_oracle as mx
from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl
from test_abi_exports import ROOT

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3
P = 16  # a pointer that nothing follows: the calls below end on the host


def test_library_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(f"{ROOT}/include/moegps_mx4.h").read(), flags=re.S)
    declared = sorted(set(re.findall(r"\b(moe_[a-z0-9_]+)\s*\(", src)))
    assert declared == sorted(B.EXPORTS_MX4)
    lib = B.load_library()
    for name in declared:
        assert hasattr(lib, name), name


def ffn_call(**kw):
    a = dict(dtype=1, d=64, ffn=100, E=4, nseg=5, seg_begin=0, seg_end=5, k=2, relu=0, reserved=0, A=8, rows_x=4, x=P, assign=P,
             offsets=P, slots=P, topk_w=0, packed=P, y=P, workspace=P, bytes=0)
    a.update(kw)
    return B.load_library().moe_grouped_ffn_mx4(B._FFN_MX4_ARGS.pack(*a.values()), None)


def product_call(**kw):
    a = dict(dtype=1, K=64, N=128, E=4, nseg=5, seg_begin=0, seg_end=5, k=2, A=8, rows_x=4, x=P, assign=P, offsets=P, slots=P,
             topk_w=0, packed=P, y=P, workspace=P, bytes=0)
    a.update(kw)
    return B.load_library().moe_grouped_product_mx4(B._PRODUCT_MX4_ARGS.pack(*a.values()), None)


@pytest.mark.parametrize("call,widths", [(ffn_call, ("d",)), (product_call, ("K", "N"))])
def test_refusals(call, widths):
    assert call() == WORKSPACE  # all else is in order
    assert call(dtype=0) == WORKSPACE
    for bad in (dict(dtype=2), dict(A=-1), dict(E=0), dict(nseg=0), dict(seg_begin=-1), dict(seg_end=6), dict(seg_begin=3, seg_end=2),
                dict(k=0), dict(rows_x=-1), dict(topk_w=P, assign=0), dict(offsets=0), dict(slots=0), dict(packed=0),
                dict(workspace=0), dict(x=0), dict(y=0)):
        assert call(**bad) == INVALID, bad
    for bad in (dict(nseg=2049), dict(E=1025), dict(A=2**31), dict(rows_x=2**31), dict(rows_x=2**25), dict(assign=0, A=2**25)):
        assert call(**bad) == UNSUPPORTED, bad
    for w in widths:
        assert call(**{w: 0}) == INVALID
        assert call(**{w: 2**22 + 64}) == UNSUPPORTED
        assert call(**{w: 60}) == UNSUPPORTED            # rows of 120 bytes
        assert call(**{w: 60, "dtype": 0}) == WORKSPACE  # of 240
        assert call(**{w: 62, "dtype": 0}) == UNSUPPORTED
    lib = B.load_library()
    assert lib.moe_grouped_ffn_mx4(None, None) == INVALID and lib.moe_grouped_product_mx4(None, None) == INVALID


def test_refusals_of_the_ffn_alone():
    assert ffn_call(relu=1) == WORKSPACE
    assert ffn_call(reserved=1) == INVALID
    assert ffn_call(ffn=0) == INVALID
    assert ffn_call(ffn=2**22 + 1) == UNSUPPORTED


def test_nothing_to_do():
    big = 1 << 30
    for call in (ffn_call, product_call):
        assert call(A=0, rows_x=0, x=0, y=0, bytes=big) == OK
        assert call(seg_begin=2, seg_end=2, bytes=big) == OK


def test_pack_refusals():
    lib = B.load_library()
    assert lib.moe_pack_weights_mx4(P, P, P, 2, 1, 64, 64, P, None) == INVALID
    assert lib.moe_pack_weights_mx4(0, P, P, 1, 1, 64, 64, P, None) == INVALID
    assert lib.moe_pack_weights_mx4(P, P, 0, 1, 1, 64, 64, P, None) == INVALID
    assert lib.moe_pack_weights_mx4(P, P, P, 1, 1, 64, 64, 0, None) == INVALID
    assert lib.moe_pack_weights_mx4(P, P, P, 1, 0, 64, 64, P, None) == INVALID
    assert lib.moe_pack_weights_mx4(P, P, P, 1, 1025, 64, 64, P, None) == UNSUPPORTED
    assert lib.moe_pack_weights_mx4(P, P, P, 1, 1, 2**22 + 1, 64, P, None) == UNSUPPORTED
    assert lib.moe_unpack_weights_mx4(P, 1, 64, 64, 1, P, P, P, 1, None) == INVALID  # the ReLU form has no W3
    assert lib.moe_unpack_weights_mx4(0, 1, 64, 64, 0, P, P, P, 1, None) == INVALID
    assert lib.moe_unpack_weights_mx4(P, 1, 64, 64, 0, 0, 0, 0, 1, None) == OK       # nothing wanted
    assert lib.moe_pack_matrix_mx4(P, 1, 1, 64, 0, P, None) == INVALID
    assert lib.moe_pack_matrix_mx4(0, 1, 1, 64, 64, P, None) == INVALID
    assert lib.moe_unpack_matrix_mx4(P, 1, 1, 64, 0, 1, None) == INVALID
    assert lib.moe_unpack_matrix_mx4(P, 1, 64, 64, P, 7, None) == INVALID


def test_sizes():
    lib = B.load_library()
    # 4.25 bits a weight where nothing is padded
    assert lib.moe_packed_matrix_mx4_bytes(3, 256, 64) == 3 * 256 * 64 * 17 // 32
    assert lib.moe_packed_weights_mx4_bytes(8, 4096, 14336, 0) == 8 * 3 * 4096 * 14336 * 17 // 32
    assert lib.moe_packed_weights_mx4_bytes(8, 4096, 14336, 1) == 8 * 2 * 4096 * 14336 * 17 // 32
    # one k-tile of one panel, with the scales of four
    assert lib.moe_packed_matrix_mx4_bytes(1, 1, 1) == 1024 + 256
    assert lib.moe_packed_matrix_mx4_bytes(1, 65, 33) == 2 * (2 * 1024 + 256)
    for bad in ((0, 64, 64), (1025, 64, 64), (1, 0, 64), (1, 64, 0), (1, 2**22 + 1, 64), (1, 64, 2**22 + 1)):
        assert lib.moe_packed_matrix_mx4_bytes(*bad) == 0
        assert lib.moe_packed_weights_mx4_bytes(*bad, 0) == 0
    assert lib.moe_packed_weights_mx4_bytes(1024, 2**22, 2**22, 0) == 1024 * 3 * 2**44 * 17 // 32
    assert lib.moe_grouped_ffn_mx4_workspace_bytes(100, 64, 100, 4, 1) >= 100 * 128 * 2
    assert lib.moe_grouped_ffn_mx4_workspace_bytes(100, 64, 100, 4, 0) >= 100 * 128 * 4
    assert lib.moe_grouped_product_mx4_workspace_bytes(100, 64, 128, 4, 1) >= 400
    for bad in ((-1, 64, 64, 1, 1), (2**31, 64, 64, 1, 1), (1, 0, 64, 1, 1), (1, 64, 0, 1, 1), (1, 64, 64, 0, 1), (1, 64, 64, 2049, 1),
                (1, 64, 64, 1, 2)):
        assert lib.moe_grouped_ffn_mx4_workspace_bytes(*bad) == 0
        assert lib.moe_grouped_product_mx4_workspace_bytes(*bad) == 0


def test_layer_step_refusals():
    lib = B.load_library()
    args = [1, 1, 4, 64, 100, 4, 2, 2, 3, 2, 0, 0] + [P] * 24

    def call(x_perm=0, **kw):
        a = list(args)
        a[12 + 16] = x_perm
        a[12 + 21] = a[12 + 23] = 1 << 30
        for name, v in kw.items():
            a[["mode", "dtype", "T", "d", "ffn", "E", "k", "G", "S", "c_max", "relu", "gate"].index(name)] = v
        return lib.moe_layer_step_mx4(B._STEP_ARGS.pack(*a), None)

    assert call(x_perm=P) == UNSUPPORTED
    assert call(x_perm=P, relu=1) == UNSUPPORTED
    assert call(d=60) == UNSUPPORTED
    assert call(mode=3) == INVALID
    assert call(T=0) == OK
    assert lib.moe_layer_step_mx4(None, None) == INVALID


# the Python side -------------------------------------------------------------
class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


def i32(n):
    return gpu(n, dtype=torch.int32)


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: 0)


def call_python(fn, **kw):
    T, k, d, E, n = 4, 2, 64, 3, 100 if fn is B.moe_grouped_ffn_mx4 else 128
    size = B.moe_packed_weights_mx4_bytes(E, d, n) if fn is B.moe_grouped_ffn_mx4 else B.moe_packed_matrix_mx4_bytes(E, d, n)
    a = dict(x=gpu(T, d), seg_offsets=i32(4), slot_expert=i32(3), packed=gpu(size, dtype=torch.uint8), assign_of_row=i32(T * k), k=k,
             topk_w=gpu(T, k, dtype=torch.float32), workspace=gpu(16, dtype=torch.uint8),
             out=gpu(T * k, d if fn is B.moe_grouped_ffn_mx4 else n))
    a.update(kw)
    x, so, se, packed = (a.pop(name) for name in ("x", "seg_offsets", "slot_expert", "packed"))
    return fn(x, so, se, packed, E, n, **a)


@pytest.mark.parametrize("fn", [B.moe_grouped_ffn_mx4, B.moe_grouped_product_mx4])
def test_python_refusals(fn):
    with pytest.raises(B.MoeGpsError, match="workspace too small"):  # all else is in order
        call_python(fn)
    for kw, text in ((dict(x=torch.zeros(4, 64, dtype=torch.bfloat16)), "x must be a GPU tensor"),
                     (dict(x=gpu(4, 64, dtype=torch.float16)), "unsupported dtype"),
                     (dict(x=gpu(64, 4).t()), "x must be contiguous"),
                     (dict(seg_offsets=i32(3)), "seg_offsets must have one entry more"),
                     (dict(slot_expert=gpu(3, dtype=torch.int64)), "slot_expert must be torch.int32"),
                     (dict(assign_of_row=i32(7)), "assign_of_row must have k entries"),
                     (dict(k=0), "assign_of_row must have k entries"),
                     (dict(assign_of_row=None), "topk_w goes with assign_of_row"),
                     (dict(topk_w=gpu(4, 1, dtype=torch.float32)), "topk_w must have one entry"),
                     (dict(packed=gpu(64, dtype=torch.uint8)), "packed must be the"),
                     (dict(out=gpu(8, 32)), "out must be"),
                     (dict(out=gpu(8, 64, dtype=torch.float32)), "out must be torch.bfloat16"),
                     (dict(workspace=torch.zeros(16, dtype=torch.uint8)), "workspace must be a GPU tensor")):
        with pytest.raises(B.MoeGpsError, match=text):
            call_python(fn, **kw)


def test_packed_for_the_other_form():
    with pytest.raises(B.MoeGpsError, match="packed must be the"):
        call_python(B.moe_grouped_ffn_mx4, relu=True)


def test_pack_python_refusals():
    W, W2 = gpu(2, 64, 100), gpu(2, 100, 64)
    with pytest.raises(B.MoeGpsError, match="weight shapes"):
        B.moe_pack_weights_mx4(W, W, W)
    with pytest.raises(B.MoeGpsError, match="W3 must be torch.bfloat16"):
        B.moe_pack_weights_mx4(W, W.float().as_subclass(OnGpu), W2)
    n = B.moe_packed_weights_mx4_bytes(2, 64, 100)
    with pytest.raises(B.MoeGpsError, match="out must hold"):
        B.moe_pack_weights_mx4(W, W, W2, out=gpu(n - 256, dtype=torch.uint8))
    with pytest.raises(B.MoeGpsError, match="packed must be the"):
        B.moe_unpack_weights_mx4(gpu(n, dtype=torch.uint8), 2, 64, 100, torch.bfloat16, relu=True)
    with pytest.raises(B.MoeGpsError, match="out must be"):
        B.moe_unpack_weights_mx4(gpu(n, dtype=torch.uint8), 2, 64, 100, torch.bfloat16, out=(W, W))
    with pytest.raises(B.MoeGpsError, match="packed must be the"):
        B.moe_unpack_matrix_mx4(gpu(n, dtype=torch.uint8), 2, 64, 64, torch.bfloat16)


def test_layer_refuses_what_it_cannot_do():
    from paper_2506_07366_amd.layer import MoELayer
    from paper_2506_07366_amd.training import MoETraining
    cfg = wl.CONFIGS["cfg1_tiny_f32"].replace(T=4)
    with pytest.raises(B.MoeGpsError, match="weights must be"):
        MoELayer(cfg, device="cpu", weights="int4")
    with pytest.raises(B.MoeGpsError, match="not trained"):
        MoETraining(MoELayer(cfg, device="cpu", weights="mx4"))


# the oracle ------------------------------------------------------------------
def test_oracle_codes():
    """Every code is its own, borders go to the even code, the scale is the smallest that cuts nothing off."""
    w = np.zeros((32, 1))
    w[:8, 0] = mx.CODES
    w[8:16, 0] = -mx.CODES
    assert np.array_equal(mx.quantise(w), w)
    w[16:23, 0] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    assert np.array_equal(mx.quantise(w)[16:23, 0], [0, 1, 1, 2, 2, 4, 4])
    for top, scale in ((6.0, 1.0), (6.0001, 2.0), (3.0, 0.5), (3.0001, 1.0), (12.0, 2.0), (1e-30, 2.0 ** -102)):
        g = np.full((32, 1), top)
        g[1] = top / 7.3
        q = mx.quantise(g)
        assert (q[0, 0] / scale) in (3.0, 4.0, 6.0) and (2 * q[1, 0] / scale) % 1 == 0, top
    assert np.array_equal(mx.quantise(np.zeros((5, 2))), np.zeros((5, 2)))
    g = np.ones((64, 2))
    g[3, 0], g[40, 1] = np.inf, np.nan
    q = mx.quantise(g)
    assert np.isnan(q[:32, 0]).all() and np.isnan(q[32:, 1]).all() and np.array_equal(q[32:, 0], g[32:, 0])


def test_oracle_bounds():
    rng = np.random.default_rng(0)
    w = rng.standard_normal((320, 50))
    q = mx.quantise(w)
    assert np.array_equal(mx.quantise(q), q)  # once is enough
    top = np.abs(w).reshape(10, 32, 50).max(1).repeat(32, 0)
    s = 2.0 ** np.ceil(np.log2(top / 6))
    assert (np.abs(q - w) <= np.maximum(0.2 * np.abs(w), s / 4) * (1 + 1e-12)).all()


@pytest.mark.parametrize("fn", [B.moe_grouped_ffn_mx4, B.moe_grouped_product_mx4])
@pytest.mark.parametrize("shape", [(4 * 64,), (4, 64, 2), (2, 4, 64)])
def test_rows_of_another_rank(fn, shape):
    """Only the first two sizes would be looked at, and less than all of x multiplied."""
    with pytest.raises(B.MoeGpsError, match="x must be \\[rows, width\\]"):
        call_python(fn, x=gpu(*shape))
