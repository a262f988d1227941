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


# ---------------------------------------------------------------------------
# gradient of the grouped FFN
# ---------------------------------------------------------------------------
def ffn_case(rows_of_slot, slot_expert, E, k, d, ffn, dtype, relu, seed, x_scale=1.0):
    """Random tensors for the given segments; the rows are a random permutation of the assignments."""
    rng = np.random.default_rng(seed)
    A = int(sum(rows_of_slot))
    assert A % k == 0
    seg = np.concatenate([[0], np.cumsum(rows_of_slot)]).astype(np.int32)
    c = dict(E=E, k=k, d=d, ffn=ffn, dtype=dtype, relu=relu, seg=seg, slot_expert=np.asarray(slot_expert, np.int32),
             assign=rng.permutation(A).astype(np.int32))
    c["x"] = dev(rng.normal(size=(A // k, d)) * x_scale, dtype)
    c["dy"] = dev(rng.normal(size=(A, d)) * 1e-2, dtype)
    c["W1"] = dev(rng.normal(size=(E, d, ffn)) * d ** -0.5, dtype)
    c["W3"] = None if relu else dev(rng.normal(size=(E, d, ffn)) * d ** -0.5, dtype)
    c["W2"] = dev(rng.normal(size=(E, ffn, d)) * d ** -0.5, dtype)
    return c


def run_ffn(c, x=None, out=None, workspace=None):
    packed = B.moe_pack_weights_relu(c["W1"], c["W2"]) if c["relu"] else B.moe_pack_weights(c["W1"], c["W3"], c["W2"])
    back = B.moe_pack_weights_backward(c["W1"], c["W3"], c["W2"])
    return B.moe_grouped_ffn_backward(c["x"] if x is None else x, dev_i32(c["assign"]), c["k"], c["dy"], dev_i32(c["seg"]),
                                      dev_i32(c["slot_expert"]), packed, back, c["E"], c["ffn"], relu=c["relu"], out=out,
                                      workspace=workspace)


def ffn_reference(c, x):
    """(values, worst-case errors) of dx_perm, dW1, dW3, dW2 in 64 bits.  A sum of n products in fp32 is off by n * 2^-24 of the sum
    of their magnitudes at most; dh, h, da and db are rounded to the type once, results too; a, b and the exponential's and
    reciprocal's few units (times |a|) reach h, da and db through the derivatives, all of them 1.1 at most."""
    E, d, ffn, relu = c["E"], c["d"], c["ffn"], c["relu"]
    u = UNIT[c["dtype"]]
    gamma = lambda n: (n + 4) * U32
    dy_all, token = host(c["dy"]), c["assign"] // c["k"]
    W1, W2 = host(c["W1"]), host(c["W2"])
    W3 = None if relu else host(c["W3"])
    names = ("dx", "dW1", "dW3", "dW2")
    shapes = dict(dx=dy_all.shape, dW1=W1.shape, dW3=W1.shape, dW2=W2.shape)
    val, tol = {n: np.zeros(shapes[n]) for n in names}, {n: np.zeros(shapes[n]) for n in names}
    for e in range(E):
        r = np.concatenate([np.arange(c["seg"][s], c["seg"][s + 1]) for s in range(len(c["slot_expert"]))
                            if c["slot_expert"][s] == e] or [np.zeros(0, int)]).astype(int)
        n = len(r)
        xe, dy = x[token[r]], dy_all[r]
        a, dh = xe @ W1[e], dy @ W2[e].T
        ta, th = gamma(d) * (abs(xe) @ abs(W1[e])), u * abs(dh) + (1 + u) * gamma(d) * (abs(dy) @ abs(W2[e]).T)
        if relu:
            h, da = np.maximum(a, 0), np.where(a > 0, dh, 0)
            t_h = ta + u * abs(h)
            t_da = np.where(a > 0, th, 0) + u * abs(da) + np.where(abs(a) <= ta, abs(dh) + th, 0)  # either side of 0
            val["dx"][r], tol["dx"][r] = da @ W1[e].T, (t_da + gamma(ffn) * abs(da)) @ abs(W1[e]).T
        else:
            b = xe @ W3[e]
            tb = gamma(d) * (abs(xe) @ abs(W3[e]))
            s = 1 / (1 + np.exp(-a))
            f = s + a * s * (1 - s)
            ex = (np.abs(a) + 8) * 2.0 ** -22
            h, da, db = a * s * b, dh * b * f, dh * a * s
            t_h = abs(a * s) * tb + abs(b) * (1.1 * ta + ex * abs(a * s)) + u * abs(h)
            t_db = abs(a * s) * th + (abs(dh) + th) * (1.1 * ta + ex * abs(a * s)) + u * abs(db)
            t_da = abs(b * f) * th + (abs(dh) + th) * (abs(f) * tb + (abs(b) + tb) * (1.1 * ta + ex)) + u * abs(da)
            val["dx"][r] = da @ W1[e].T + db @ W3[e].T
            tol["dx"][r] = (t_da + gamma(2 * ffn) * abs(da)) @ abs(W1[e]).T + (t_db + gamma(2 * ffn) * abs(db)) @ abs(W3[e]).T
            val["dW3"][e], tol["dW3"][e] = xe.T @ db, abs(xe).T @ (t_db + gamma(n) * abs(db))
        val["dW1"][e], tol["dW1"][e] = xe.T @ da, abs(xe).T @ (t_da + gamma(n) * abs(da))
        val["dW2"][e], tol["dW2"][e] = h.T @ dy, (t_h + gamma(n) * abs(h)).T @ abs(dy)
    for n in names:
        tol[n] += u * (abs(val[n]) + tol[n]) + 1e-38
    return val, tol


def check_ffn(c, got, x=None):
    val, tol = ffn_reference(c, host(c["x"]) if x is None else x)
    # the roundings of a long sum's terms are independent: the error's norm is that of two roundings and the result's own, each
    # uniform within its half step, sqrt(3) / sqrt(3) of one
    norm = UNIT[c["dtype"]] if c["dtype"] == "bf16" else 64 * U32
    for name, t in zip(("dx", "dW1", "dW3", "dW2"), got):
        if t is None:
            continue
        g = host(t)
        err = np.abs(g - val[name])
        assert np.all(err <= tol[name]), (name, float((err - tol[name]).max()), np.argwhere(err > tol[name])[:4])
        size = np.linalg.norm(val[name])
        if not c["relu"] or c["dtype"] == "bf16":
            assert np.linalg.norm(g - val[name]) <= norm * size + 1e-30, (name, np.linalg.norm(g - val[name]) / max(size, 1e-300))


SEGMENTS = {  # rows of the slots, their experts, E
    "one_row": ([1], [0], 1),
    "two_experts": ([3, 5], [1, 0], 2),
    "empty_slots_and_experts": ([0, 7, 0, 1, 0], [2, 0, -1, 3, 2], 5),
    "replicas": ([17, 33, 16, 30], [1, 0, 1, 0], 2),
    "edges": ([31, 32, 33, 15, 64, 65], [0, 1, 2, 3, 4, 5], 6),
    "tall": ([300, 2, 258], [0, 1, 2], 4),
}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("segments", sorted(SEGMENTS))
@pytest.mark.parametrize("d,ffn", [(64, 64), (128, 100), (320, 264)])
def test_ffn_backward(dtype, relu, segments, d, ffn):
    rows, experts, E = SEGMENTS[segments]
    c = ffn_case(rows, experts, E, 1, d, ffn, dtype, relu, seed=len(rows) + d)
    got = run_ffn(c)
    check_ffn(c, got)
    if relu:
        assert got[2] is None
    again = run_ffn(c)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("d,ffn", [(64, 1), (64, 7), (128, 65), (192, 130), (64, 520), (576, 66)])
def test_ffn_backward_bf16_odd_widths(d, ffn):
    """Hidden widths that are no multiple of eight (gradients stored value by value), of 64 or of a tile."""
    c = ffn_case([9, 0, 40], [1, 2, 0], 3, 1, d, ffn, "bf16", False, seed=ffn)
    check_ffn(c, run_ffn(c))
    c = ffn_case([9, 0, 40], [1, 2, 0], 3, 1, d, ffn, "bf16", True, seed=ffn)
    check_ffn(c, run_ffn(c))


@pytest.mark.parametrize("d,ffn", [(64, 1), (64, 7), (128, 65), (192, 130), (64, 520), (576, 66)])
@pytest.mark.parametrize("rows", [[97, 0, 0, 128, 5], [65, 66, 1, 0, 161]])
def test_ffn_backward_bf16_odd_widths_of_many_rows(d, ffn, rows):
    """More than 32 rows per expert on average: the weights' gradients by large tiles.  Experts without rows and with few among them;
    the last of an expert's steps of 32 rows is first, second, third and fourth of four, whole and of one row."""
    for relu in (False, True):
        c = ffn_case(rows, [1, 4, 2, 0, 3], 5, 1, d, ffn, "bf16", relu, seed=ffn + rows[0])
        check_ffn(c, run_ffn(c))


def test_ffn_backward_is_the_same_on_either_side_of_the_tile_rule():
    """The gradients of an expert do not depend on how many other experts there are: 33 rows per expert on average, and fewer."""
    c = ffn_case([40, 26], [0, 1], 2, 1, 128, 200, "bf16", False, seed=21)
    got = run_ffn(c)
    wide = dict(c, E=9)
    for name in ("W1", "W3", "W2"):
        wide[name] = torch.cat([c[name], torch.zeros((7, *c[name].shape[1:]), dtype=torch.bfloat16, device="cuda")])
    many = run_ffn(wide)
    assert torch.equal(many[0], got[0])
    for a, b in zip(many[1:], got[1:]):
        assert torch.equal(a[:2], b) and torch.all(a[2:] == 0)


@pytest.mark.parametrize("d,ffn", [(4, 4), (12, 20), (132, 68)])
def test_ffn_backward_f32_narrow(d, ffn):
    for relu in (False, True):
        c = ffn_case([5, 0, 70], [1, 2, 0], 3, 1, d, ffn, "f32", relu, seed=ffn)
        check_ffn(c, run_ffn(c))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ffn_backward_of_tokens_with_several_experts(dtype):
    """k rows of a token, from the rows themselves and from a checkpoint of them."""
    rng = np.random.default_rng(7)
    k, T, E, d, ffn = 3, 150, 7, 256, 192
    sizes = rng.multinomial(T * k, rng.dirichlet(np.ones(9)))
    experts = [0, 1, 2, 3, 4, 5, 6, 2, 5]
    c = ffn_case(sizes.tolist(), experts, E, k, d, ffn, dtype, False, seed=3)
    check_ffn(c, run_ffn(c))
    kept = B.moe_checkpoint_store(c["x"])
    x = ck.load(kept[0].view(torch.uint8).cpu().numpy(), kept[1].cpu().numpy())
    got = run_ffn(c, x=kept)
    check_ffn(c, got, x)
    # the rows that the checkpoint stands for are exact in the type: the same bits
    plain = run_ffn(c, x=B.moe_checkpoint_load(*kept, DT[dtype]))
    assert all(torch.equal(a, b) for a, b in zip(got, plain))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ffn_backward_parts(dtype):
    """Only dx, only the weights' gradients, nothing; outputs and workspace that held NaN; rows of no expert."""
    rows, experts = [40, 5, 13], [0, -1, 1]
    c = ffn_case(rows, experts, 3, 2, 128, 72, dtype, False, seed=11)
    full = run_ffn(c)
    nan = lambda t: torch.full_like(t, float("nan"))
    dirty = tuple(nan(t) for t in full)
    ws = torch.full((B.moe_grouped_ffn_backward_workspace_bytes(29, 2, 128, 72, 3, 3, B.dtype_code(c["dy"])),), 0xff,
                    dtype=torch.uint8, device="cuda")
    got = run_ffn(c, out=dirty, workspace=ws)
    live = torch.ones(58, dtype=torch.bool, device="cuda")
    live[40:45] = False
    assert torch.equal(got[0][live], full[0][live]) and torch.isnan(got[0][~live]).all()
    assert all(torch.equal(a, b) for a, b in zip(got[1:], full[1:]))
    assert torch.all(got[1][2] == 0) and torch.all(got[3][2] == 0)
    only = run_ffn(c, out=(nan(full[0]), None, None, None))
    assert torch.equal(only[0][live], full[0][live])
    only = run_ffn(c, out=(None, *[nan(t) for t in full[1:]]))
    assert all(torch.equal(a, b) for a, b in zip(only[1:], full[1:]))
    assert run_ffn(c, out=(None, None, None, None)) == (None, None, None, None)
    with pytest.raises(B.MoeGpsError, match="invalid argument"):
        run_ffn(c, out=(full[0], full[1], None, full[3]))
    with pytest.raises(B.MoeGpsError, match="workspace too small"):
        run_ffn(c, workspace=ws[:-256])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_ffn_backward_of_an_empty_batch(dtype):
    c = ffn_case([0, 0], [0, 1], 2, 1, 64, 64, dtype, False, seed=1)
    got = run_ffn(c, out=(c["dy"], *(torch.full_like(c[w], 3.0) for w in ("W1", "W3", "W2"))))
    assert all(torch.all(t == 0) for t in got[1:])


def test_ffn_backward_against_differences():
    """fp32, in the direction of each gradient: a step that changes the loss by 2 eps |g|^2 (central difference of the library's own
    forward pass, whose fp32 sums are off by about 1e-6 of the loss's terms)."""
    c = ffn_case([20, 12, 31], [0, 1, 0], 2, 1, 64, 96, "f32", False, seed=5)
    got = run_ffn(c)
    x_perm = c["x"][torch.from_numpy(c["assign"].astype(np.int64)).cuda()]

    def loss(**changed):
        t = {**dict(x=x_perm, W1=c["W1"], W3=c["W3"], W2=c["W2"]), **changed}
        packed = B.moe_pack_weights(t["W1"], t["W3"], t["W2"])
        y = B.moe_grouped_ffn(t["x"], dev_i32(c["seg"]), dev_i32(c["slot_expert"]), packed, 2, 96)
        return float((y.double() * c["dy"].double()).sum())

    base = dict(x=x_perm, W1=c["W1"], W3=c["W3"], W2=c["W2"])
    for name, g in zip(("x", "W1", "W3", "W2"), got):
        n = float(g.double().norm())
        step = 1e-2 * float(base[name].double().norm()) / n
        up, down = (loss(**{name: base[name] + s * step * g}) for s in (1, -1))
        # third derivatives: (1e-2)^2 relative at most a few times; rounding: 1e-6 of the terms, against a change of 1e-2 of them
        assert abs((up - down) / (2 * step) - n * n) <= 2e-3 * n * n, name
