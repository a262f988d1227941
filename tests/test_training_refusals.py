"""What the training calls' Python side refuses before a pointer is taken (no GPU needed: host tensors that say they are on one,
and calls that never reach the device)."""
import pytest
import torch

from paper_2506_07366_amd import binding as B


class OnGpu(torch.Tensor):
    is_cuda = True


def gpu(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture(autouse=True)
def no_stream(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: 0)


E, D, FFN = 3, 128, 200
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


def test_router_gradient_without_the_number_of_experts():
    """E belongs to topk_idx: without it there was an empty dlogits."""
    T, k = 4, 2
    args = (gpu(T, 64), gpu(T * k, 64), gpu(T * k, dtype=torch.int32), gpu(T, k, dtype=torch.float32))
    idx = gpu(T, k, dtype=torch.int32)
    with pytest.raises(B.MoeGpsError, match="E, the number of experts"):
        B.moe_combine_backward(*args, topk_idx=idx, out=(gpu(T * k, 64), gpu(T, k, dtype=torch.float32),
                                                         gpu(T, 0, dtype=torch.float32)))


def ffn_backward_call(dtype=torch.bfloat16, relu=False, **kw):
    T, k = 4, 2
    code = 1 if dtype == torch.bfloat16 else 0
    lib = B.load_library()
    size = lib.moe_packed_weights_relu_bytes if relu else lib.moe_packed_weights_bytes
    a = dict(x=gpu(T, D, dtype=dtype), assign_of_row=gpu(T * k, dtype=torch.int32), k=k, dy_perm=gpu(T * k, D, dtype=dtype),
             seg_offsets=gpu(E + 1, dtype=torch.int32), slot_expert=gpu(E, dtype=torch.int32),
             packed=gpu(size(E, D, FFN, code), dtype=torch.uint8),
             packed_backward=gpu(B.moe_packed_weights_backward_bytes(E, D, FFN, code, relu), dtype=torch.uint8), E=E, ffn=FFN,
             relu=relu, workspace=gpu(1, dtype=torch.uint8),
             out=(gpu(T * k, D, dtype=dtype), gpu(E, D, FFN, dtype=dtype), None if relu else gpu(E, D, FFN, dtype=dtype),
                  gpu(E, FFN, D, dtype=dtype)))
    a.update(kw)
    return B.moe_grouped_ffn_backward(**a)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("relu", [False, True])
def test_weights_that_were_packed_for_something_else(dtype, relu):
    """The kernels read as many bytes as the form has: of another shape's or form's they would read others, or past them."""
    code = 1 if dtype == torch.bfloat16 else 0
    lib = B.load_library()
    byte = lambda n: gpu(n, dtype=torch.uint8)
    with pytest.raises(B.MoeGpsError, match="workspace too small"):  # all else is in order
        ffn_backward_call(dtype, relu)
    other = lib.moe_packed_weights_bytes if relu else lib.moe_packed_weights_relu_bytes
    for n in (other(E, D, FFN, code), other(E, D, FFN + 64, code), 0):
        with pytest.raises(B.MoeGpsError, match="packed must be"):
            ffn_backward_call(dtype, relu, packed=byte(n))
    if code == 1:
        for n in (B.moe_packed_weights_backward_bytes(E, D, FFN, 1, not relu), 0):
            with pytest.raises(B.MoeGpsError, match="packed_backward must be"):
                ffn_backward_call(dtype, relu, packed_backward=byte(n))
    for name in ("packed", "workspace"):
        with pytest.raises(B.MoeGpsError, match=f"{name} must be a GPU tensor"):
            ffn_backward_call(dtype, relu, **{name: torch.zeros(1 << 20, dtype=torch.uint8)})
    with pytest.raises(B.MoeGpsError, match="out must be"):
        ffn_backward_call(dtype, relu, out=(None, None, None))
