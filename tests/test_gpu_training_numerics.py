"""What is kept in which precision on the way to the gradients."""
import numpy as np
import numpy as np
import pytest
import torch

from paper_2506_07366_amd import binding as B
from gpu_util import dev_i32
from test_gpu_training import DT

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
