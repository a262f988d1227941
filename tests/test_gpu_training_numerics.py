"""What is kept in which precision on the way to the gradients, and where values that are not finite go."""
import numpy as np
import pytest
import torch

from paper_2506_07366_amd import binding as B
from gpu_util import dev_i32
from test_gpu_training import DT, ffn_case, run_ffn
from test_gpu_training_layer import host, make, step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("E", [1, 8])  # 40 rows: large tiles, small ones
def test_gradient_of_the_hidden_activation_is_not_rounded(dtype, E):
    """dh = 257 needs nine bits, one more than bf16 has.  With a = 48 (s is 1) and b = 3: da = 3 dh = 771 and db = 48 dh = 12336, in
    bf16 772 and 12352; from a rounded dh (256) they would be 768 and 12288.  Sums of one term or of equal ones, all exact."""
    n, d, ffn = 40, 64, 64
    t = lambda v: v.to(DT[dtype]).cuda()
    W1, W3 = t(torch.full((E, d, ffn), 48.0)), t(torch.full((E, d, ffn), 3.0))
    W2 = torch.zeros((E, ffn, d))
    W2[:, :, :2] = 1
    W2 = t(W2)
    dy = torch.zeros((n, d))
    dy[:, 0], dy[:, 1] = 256, 1
    packed, back = B.moe_pack_weights(W1, W3, W2), B.moe_pack_weights_backward(W1, W3, W2)
    dx, dW1, dW3, dW2 = B.moe_grouped_ffn_backward(
        t(torch.eye(n, d)), dev_i32(np.arange(n)), 1, t(dy), dev_i32([0, n]), dev_i32([0]), packed, back, E, ffn)
    da, db, dxv = (772, 12352, 145 * 2 ** 15) if dtype == "bf16" else (771, 12336, 64 * (771 * 48 + 12336 * 3))
    assert torch.all(dW1[0, :n] == da) and torch.all(dW3[0, :n] == db)
    assert torch.all(dW1[0, n:] == 0) and torch.all(dW3[0, n:] == 0)
    assert torch.all(dx == dxv)
    assert torch.all(dW2[0, :, 0] == n * 144 * 256) and torch.all(dW2[0, :, 1] == n * 144) and torch.all(dW2[0, :, 2:] == 0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["swiglu", "relu"])
def test_what_rows_kept_in_8_bits_cost(dtype, act):
    """Gradients from rows kept in 8 bits against those from the rows themselves.  A kept value is off by half a step, 2^-4 of it,
    at most; rounding errors are spread evenly within that and independent: their norm is u = 2^-4 / sqrt(3) of the rows' norm at
    most.  dtopk_w and dlogits are linear in y.  dW1 and dW3 are x times what depends on a = x W1 and b = x W3, dW2 depends on both, dx
    on da and db: three times u at most, to first order.  With ReLU an error moves a through 0 where |a| is of its size, u in
    the norm of a unit normal: a fraction u * sqrt(2 / pi) of the terms comes or goes, sqrt(u) of the norm."""
    c = make(600, 2, 8, 4, 3, 128, 72, dtype, act=act, mode=0, saved="plain")
    want = {n: host(v) for n, v in step(c).items() if v is not None}
    kept = make(600, 2, 8, 4, 3, 128, 72, dtype, act=act, mode=0, saved="8bit")
    got = {n: host(v) for n, v in step(kept).items() if v is not None}
    u = 2.0 ** -4 / 3 ** 0.5
    own = 2 * 2.0 ** -8 if dtype == "bf16" else 1e-4   # both sides' own roundings
    for n, w in want.items():
        size = np.linalg.norm(want["dtopk_w"]) if n == "dlogits" else np.linalg.norm(w)
        bound = u if n in ("dtopk_w", "dlogits") else 3 * u if act == "swiglu" else u + u ** 0.5
        err = np.linalg.norm(got[n] - w) / size
        assert err <= bound + own, (n, err)


def case_with(bad, where, dtype, relu, rows=(40, 30, 9)):
    """Three experts; one value of row 3 (expert 0), of its input or of its result's gradient, is not finite."""
    c = ffn_case(list(rows), [0, 1, 2], 3, 1, 128, 72, dtype, relu, seed=17)
    clean = run_ffn(c)
    row, at = 3, 17
    token = int(c["assign"][row])
    if where == "x":
        c["x"][token, at] = bad
    else:
        c["dy"][row, at] = bad
    return c, clean, run_ffn(c), row, at


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["x", "dy"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("rows", [(40, 30, 9), (40, 30, 70)])  # small tiles, large ones
def test_values_that_are_not_finite_stay_with_their_row_and_expert(dtype, where, bad, rows):
    c, clean, got, row, at = case_with(bad, where, dtype, False, rows)
    dx, dW1, dW3, dW2 = got
    others = torch.arange(dx.shape[0], device="cuda") != row
    assert torch.equal(dx[others], clean[0][others]) and not torch.isfinite(dx[row]).any()
    for g, before in zip(got[1:], clean[1:]):
        assert torch.equal(g[1:], before[1:])
    if where == "dy":  # h is as it was: one column of dW2 has it
        assert not torch.isfinite(dW2[0][:, at]).any()
        keep = torch.arange(dW2.shape[2], device="cuda") != at
        assert torch.equal(dW2[0][:, keep], clean[3][0][:, keep])
    else:
        assert not torch.isfinite(dW2[0]).any()
    assert not torch.isfinite(dW1[0]).any() and not torch.isfinite(dW3[0]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_sums_under_relu_count_as_zero(dtype):
    """As in the forward pass, max(a, 0) of a that is not a number is 0: the row adds nothing, but for its own NaN times 0."""
    c, clean, got, row, at = case_with(float("nan"), "x", dtype, True)
    dx, dW1, _, dW2 = got
    assert torch.all(dx[row] == 0)
    others = torch.arange(dx.shape[0], device="cuda") != row
    assert torch.equal(dx[others], clean[0][others])
    assert torch.isnan(dW1[0][at]).all()
    keep = torch.arange(dW1.shape[1], device="cuda") != at
    assert torch.isfinite(dW1[0][keep]).all() and torch.isfinite(dW2).all()
    assert torch.equal(dW1[1:], clean[1][1:]) and torch.equal(dW2[1:], clean[3][1:])
    # the forward pass of the same row: zeros
    y = B.moe_grouped_ffn(c["x"][torch.from_numpy(c["assign"].astype(np.int64)).cuda()], dev_i32(c["seg"]), dev_i32(c["slot_expert"]),
                          B.moe_pack_weights_relu(c["W1"], c["W2"]), 3, c["ffn"], relu=True)
    assert torch.all(y[row] == 0)
