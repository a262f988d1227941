"""Gradients of the weights where an expert's rows of the hidden activations are more than 2^32 bytes."""
import pytest
import torch

from paper_2506_07366_amd import binding as B

pytestmark = pytest.mark.gpu


def test_few_rows_on_average_all_of_one_expert():
    """1024 experts, 32 rows each on average and so made by small tiles, but one has all 32768, of 2 * 32896 values.  Only the rows
    whose place is past 2^32 bytes have inputs that are not zero, so the gradients of W1 and W3 are theirs alone.  Columns
    all over the width, in 64 bits; the error's norm is that of two roundings to bf16 (da and db, the result) at most, as in the
    tests of whole gradients."""
    E, T, d, ffn, busy = 1024, 32768, 64, 32896, 5
    past = T - (1 << 32) // (2 * ffn * 2)  # rows that begin past 2^32 bytes
    assert 32 * E == T and past > 100
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 120e9:
        pytest.skip("needs 100 GB")
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    normal = lambda *s: torch.randn(s, device="cuda", generator=gen)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((T, d), **bf16)
    x[T - past + 4:] = normal(past - 4, d).bfloat16()
    dy = (1e-2 * normal(T, d)).bfloat16()
    W = [torch.zeros(s, **bf16) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d))]
    for w in W:
        w[busy] = (d ** -0.5 * normal(*w.shape[1:])).bfloat16()
    own = [w[busy].double() for w in W]
    packed, back = B.moe_pack_weights(*W), B.moe_pack_weights_backward(*W)
    rows = torch.arange(T, dtype=torch.int32, device="cuda")
    seg = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    seg[busy + 1:] = T
    slots = torch.arange(E, dtype=torch.int32, device="cuda")
    _, dW1, dW3, dW2 = B.moe_grouped_ffn_backward(x, rows, 1, dy, seg, slots, packed, back, E, ffn, out=(None, *W))
    cols = torch.arange(7, ffn, 1231, device="cuda")
    live = slice(T - past, T)
    xd, dyd = x[live].double(), dy[live].double()
    a, b, dh = xd @ own[0][:, cols], xd @ own[1][:, cols], dyd @ own[2][cols].T.contiguous()
    s = torch.sigmoid(a)
    want = (xd.T @ (dh * b * s * (1 + a * (1 - s))), xd.T @ (dh * a * s), (a * s * b).T @ dyd)
    for name, got, w in zip(("dW1", "dW3", "dW2"), (dW1[busy][:, cols], dW3[busy][:, cols], dW2[busy][cols]), want):
        err = float((got.double() - w).norm() / w.norm())
        assert err <= 2.0 ** -8, (name, err)
    for g in (dW1, dW3, dW2):
        assert not torch.any(g[:busy]) and not torch.any(g[busy + 1:])
    del packed, back, W, dW1, dW3, dW2, g
    torch.cuda.empty_cache()
