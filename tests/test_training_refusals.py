"""What the training calls' Python side refuses before a pointer is taken (no GPU needed: host tensors that say they are on one,
and calls that never reach the device)."""
import pytest
import torch

from paper_2506_07366_amd import binding as B


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


E, D, FFN = 3, 128, 72
W1, W3, W2 = gpu(E, D, FFN), gpu(E, D, FFN), gpu(E, FFN, D)
PACKS = {
    "swiglu": (lambda out: B.moe_pack_weights(W1, W3, W2, out=out), lambda: B.moe_packed_weights_bytes(E, D, FFN, 1)),
    "relu": (lambda out: B.moe_pack_weights_relu(W1, W2, out=out),
             lambda: B.load_library().moe_packed_weights_relu_bytes(E, D, FFN, 1)),
    "backward": (lambda out: B.moe_pack_weights_backward(W1, W3, W2, out=out),
                 lambda: B.moe_packed_weights_backward_bytes(E, D, FFN, 1)),
}


@pytest.mark.parametrize("form", sorted(PACKS))
def test_packed_weights_into_a_buffer_of_another_size(form):
    pack, size = PACKS[form]
    for n in (size() - 256, size() + 256, 0):
        with pytest.raises(B.MoeGpsError, match="out must hold the packed weights"):
            pack(gpu(n, dtype=torch.uint8))
    with pytest.raises(B.MoeGpsError, match="out must be torch.uint8"):
        pack(gpu(size()))
    with pytest.raises(B.MoeGpsError, match="out must be a GPU tensor"):
        pack(torch.zeros(size(), dtype=torch.uint8))


def test_widths_whose_dx_sums_over_more_than_a_panel():
    """dx is a sum over the columns of da and db, 2^22 at most; the gradients of the weights are not concerned."""
    from test_train_host import UNSUPPORTED, ffn_backward
    WORKSPACE = -3  # all else is in order
    relu = dict(relu=1, dW3=0)
    assert ffn_backward(ffn=2**21) == WORKSPACE
    for ffn in (2**21 + 1, 2**21 + 64, 3 * 2**20, 2**22 - 64):
        assert ffn_backward(ffn=ffn) == UNSUPPORTED, ffn
        assert ffn_backward(ffn=ffn, dx=0) == WORKSPACE, ffn
        assert ffn_backward(ffn=ffn, **relu) == WORKSPACE, ffn
        assert ffn_backward(ffn=ffn, dtype=0) == (WORKSPACE if ffn % 4 == 0 else UNSUPPORTED), ffn
