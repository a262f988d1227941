"""GPU parity of the training calls (through the C ABI) against the CPU oracle in 64 bits.

Roundings counted by the tolerances: u32 = 2^-24 for an fp32 operation, 2^-8 for a result stored as bf16."""
import numpy as np
import pytest
import torch

from oracle import checkpoint as ck
from oracle.backward import combine_backward
from paper_2506_07366_amd import binding as B
from gpu_util import dev_i32, to_host_f32

pytestmark = pytest.mark.gpu

U32, UBF = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
UNIT = {"f32": U32, "bf16": UBF}


def dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(DT[dtype])


def host(t):
    return t.detach().double().cpu().numpy()


# ---------------------------------------------------------------------------
# checkpoints: whole codes, so everything is equal
# ---------------------------------------------------------------------------
def check_checkpoint(x):
    codes, scales = B.moe_checkpoint_store(x)
    want_codes, want_scales = ck.store(host(x))
    got = codes.view(torch.uint8).cpu().numpy()
    np.testing.assert_array_equal(scales.cpu().numpy(), want_scales)
    nan = (want_codes & 0x7f) == 0x7f
    np.testing.assert_array_equal((got & 0x7f) == 0x7f, nan)
    np.testing.assert_array_equal(got[~nan], want_codes[~nan])
    back = host(B.moe_checkpoint_load(codes, scales, x.dtype))
    np.testing.assert_array_equal(back, ck.load(want_codes, want_scales))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,d", [(1, 8), (1, 4096), (3, 32), (7, 40), (129, 768), (65, 96), (5, 2056), (1000, 128),
                                    (33, 4104), (2, 16384)])
def test_checkpoint_codes(dtype, rows, d):
    rng = np.random.default_rng(rows * 7 + d)
    x = rng.normal(size=(rows, d)) * np.exp(4 * rng.normal(size=(rows, 1)))
    x[rng.random(x.shape) < 0.1] = 0
    x[rng.random((rows, d)) < 0.01] *= 100
    check_checkpoint(dev(x, dtype))


@pytest.mark.parametrize("d", [4, 12, 36, 1020])
def test_checkpoint_fp32_rows_of_half_a_piece(d):
    rng = np.random.default_rng(d)
    check_checkpoint(dev(rng.normal(size=(9, d)), "f32"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_checkpoint_borders_and_special_values(dtype):
    """Every midpoint between two codes at several scales; groups of zeros, tiny and huge values, infinities, NaN."""
    v = ck.e4m3_values()[:127]
    points = np.concatenate([v, (v[1:] + v[:-1]) / 2])
    x = np.zeros((64, 256))
    for r, e in enumerate((-130, -126, -60, -1, 0, 1, 60, 118)):
        for half in range(2):
            row = np.concatenate([points, [0.0] * 3])[:256]
            row = row.reshape(8, 32)
            row[:, 31] = 448.0                                   # holds the scale
            x[2 * r + half] = (1 - 2 * half) * row.reshape(-1) * 2.0 ** e
    x[20, :] = 3.38e38
    x[21, 3], x[22, 40], x[23, 64:96] = np.inf, -np.inf, np.nan
    x[21, 0], x[22, 32] = 1.0, -2.0
    x[24, ::2] = 1e-40
    check_checkpoint(dev(x, dtype))


def test_checkpoint_writes_nothing_else_and_empty_batches():
    x = dev(np.ones((5, 72)), "bf16")
    codes = torch.full((9, 72), 0x55, dtype=torch.uint8, device="cuda")
    scales = torch.full((9, 3), 0x55, dtype=torch.uint8, device="cuda")
    B.moe_checkpoint_store(x, out=(codes[2:7], scales[2:7]))
    assert torch.all(codes[:2] == 0x55) and torch.all(codes[7:] == 0x55)
    assert torch.all(scales[:2] == 0x55) and torch.all(scales[7:] == 0x55)
    back = torch.full((9, 72), -1.0, dtype=torch.bfloat16, device="cuda")
    B.moe_checkpoint_load(codes[2:7], scales[2:7], torch.bfloat16, out=back[2:7])
    assert torch.all(back[2:7] == 1) and torch.all(back[:2] == -1) and torch.all(back[7:] == -1)
    codes, scales = B.moe_checkpoint_store(x[:0])
    assert codes.shape == (0, 72) and B.moe_checkpoint_load(codes, scales, torch.bfloat16).shape == (0, 72)


# ---------------------------------------------------------------------------
# gradient of the combine
# ---------------------------------------------------------------------------
def combine_case(T, k, d, E, dtype, saved, seed):
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(T, k))
    w = np.exp(z - z.max(axis=1, keepdims=True))
    w = (w / w.sum(axis=1, keepdims=True)).astype(np.float32)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    rows = rng.permutation(T * k).astype(np.int32)
    dout, y = dev(rng.normal(size=(T, d)) * 1e-3, dtype), dev(rng.normal(size=(T * k, d)), dtype)
    if saved == "8bit":
        y = B.moe_checkpoint_store(y)
        y_host = ck.load(y[0].view(torch.uint8).cpu().numpy(), y[1].cpu().numpy())
    else:
        y_host = host(y)
    return dout, y, y_host, rows, torch.from_numpy(w).cuda(), w.astype(np.float64), idx


def check_combine(dtype, dy, dw, dl, dout, y_host, rows, w, idx, E):
    T, k = w.shape
    d = dout.shape[1]
    want_dy, want_dw, want_dl = combine_backward(host(dout), y_host, rows, w, idx, E)
    # one product in fp32, one rounding to the type
    u = U32 if dtype == "f32" else UBF + U32
    assert np.all(np.abs(host(dy) - want_dy) <= u * np.abs(want_dy) + 1e-38)
    # a sum of d products: a chain of at most d / 64 (+ 8: a whole piece) in a lane, then 6 + 16 additions, one for the scale
    size = np.abs(host(dout))[:, None, :] * np.abs(y_host[rows.reshape(T, k)])
    tol_w = (d / 64 + 8 + 24) * U32 * size.sum(axis=2)
    assert np.all(np.abs(host(dw) - want_dw) <= tol_w)
    if dl is not None:
        # the mean has k products, the difference and the product two more roundings
        tol = w * (tol_w + (w * tol_w).sum(1, keepdims=True)) + \
            (k + 3) * U32 * w * (np.abs(want_dw) + (w * np.abs(want_dw)).sum(1, keepdims=True))
        full = np.zeros((T, E))
        np.put_along_axis(full, idx.astype(np.int64), tol, axis=1)
        assert np.all(np.abs(host(dl) - want_dl) <= full)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("saved", ["plain", "8bit"])
@pytest.mark.parametrize("T,k,d,E", [(1, 8, 4096, 128), (1, 1, 8, 1), (5, 2, 64, 8), (33, 16, 520, 1024), (70, 3, 72, 9),
                                     (257, 4, 1032, 16), (1100, 2, 128, 8), (3, 5, 16384, 7), (19, 9, 2048, 64)])
def test_combine_backward(dtype, saved, T, k, d, E):
    dout, y, y_host, rows, w_dev, w, idx = combine_case(T, k, d, E, dtype, saved, T + k)
    dy, dw, dl = B.moe_combine_backward(dout, y, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=E)
    check_combine(dtype, dy, dw, dl, dout, y_host, rows, w, idx, E)
    again = B.moe_combine_backward(dout, y, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=E)
    assert all(torch.equal(a, b) for a, b in zip((dy, dw, dl), again))


@pytest.mark.parametrize("d", [4, 44, 1036])
def test_combine_backward_fp32_rows_of_half_a_piece(d):
    for saved in ("plain", "8bit"):
        dout, y, y_host, rows, w_dev, w, idx = combine_case(11, 3, d, 6, "f32", saved, d)
        out = B.moe_combine_backward(dout, y, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=6)
        check_combine("f32", *out, dout, y_host, rows, w, idx, 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_combine_backward_parts_and_places(dtype):
    """Without y only dy; without ids no dlogits; dy in the place of y; outputs that held something before."""
    T, k, d, E = 37, 3, 200, 11
    dout, y, y_host, rows, w_dev, w, idx = combine_case(T, k, d, E, dtype, "plain", 5)
    full = B.moe_combine_backward(dout, y, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=E)
    dy, dw, dl = B.moe_combine_backward(dout, None, dev_i32(rows), w_dev)
    assert torch.equal(dy, full[0]) and dw is None and dl is None
    dy, dw, dl = B.moe_combine_backward(dout, y, dev_i32(rows), w_dev)
    assert torch.equal(dy, full[0]) and torch.equal(dw, full[1]) and dl is None
    place = y.clone()
    dirty = (place, torch.full((T, k), float("nan"), device="cuda"), torch.full((T, E), float("nan"), device="cuda"))
    got = B.moe_combine_backward(dout, place, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=E, out=dirty)
    assert all(torch.equal(a, b) for a, b in zip(got, full))
    assert B.moe_combine_backward(dout[:0], y[:0], dev_i32([]), w_dev[:0], topk_idx=dev_i32(idx[:0]), E=E)[2].shape == (0, E)


def test_combine_backward_nan_stays_with_its_assignment():
    T, k, d, E = 4, 2, 96, 5
    dout, y, y_host, rows, w_dev, w, idx = combine_case(T, k, d, E, "bf16", "plain", 9)
    y[int(rows[2 * k + 1]), 7] = float("nan")
    kept = B.moe_checkpoint_store(y)
    for saved in (y, kept):
        dy, dw, dl = B.moe_combine_backward(dout, saved, dev_i32(rows), w_dev, topk_idx=dev_i32(idx), E=E)
        assert torch.isfinite(dy.float()).all()
        bad = torch.isnan(dw).cpu().numpy()
        assert bad.sum() == 1 and bad[2, 1]
        nan_rows = torch.isnan(dl).any(dim=1).cpu().tolist()
        assert nan_rows == [False, False, True, False]
        off = np.ones(E, bool)
        off[idx[2]] = False
        assert torch.all(dl[2][torch.from_numpy(off).cuda()] == 0)


def test_refusals_on_the_device():
    x = torch.zeros((4, 64), dtype=torch.bfloat16, device="cuda")
    w, rows = torch.zeros((4, 2), device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    y = torch.zeros((8, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.MoeGpsError, match="contiguous"):
        B.moe_checkpoint_store(x.t().contiguous().t())
    with pytest.raises(B.MoeGpsError, match="not supported"):
        B.moe_checkpoint_store(x[:, :12].contiguous())
    codes, scales = B.moe_checkpoint_store(x)
    with pytest.raises(B.MoeGpsError, match="scales must be"):
        B.moe_checkpoint_load(codes, scales[:, :1].contiguous(), torch.bfloat16)
    with pytest.raises(B.MoeGpsError, match="unsupported dtype"):
        B.moe_checkpoint_load(codes, scales, torch.float16)
    with pytest.raises(B.MoeGpsError, match="one entry per assignment"):
        B.moe_combine_backward(x, y, rows[:7].contiguous(), w)
    with pytest.raises(B.MoeGpsError, match="y_perm must be"):
        B.moe_combine_backward(x, y[:7], rows, w)
    with pytest.raises(B.MoeGpsError, match="y_perm must be torch.bfloat16"):
        B.moe_combine_backward(x, y.float(), rows, w)
    with pytest.raises(B.MoeGpsError, match="invalid argument"):
        B.moe_combine_backward(x, y, rows, w, topk_idx=rows.view(4, 2), E=1)
