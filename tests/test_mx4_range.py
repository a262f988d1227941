"""How far a weight in 4 bits may be off at the ends of the range, and which values of such a format are held as they are."""
import numpy as np
import pytest
import torch

import mx4_oracle as mx
from paper_2506_07366_amd import binding as B

CODES = np.concatenate([mx.CODES, -mx.CODES])
TOP = 3 * 2.0 ** 126  # the largest value that is held
CUT = 3.5 * 2.0 ** 126


def every_scale():
    """A group of every byte from 2 to 253 (as columns, K = 32) with all of its codes that are not above TOP, and one with a few small ones."""
    cols = []
    for b in range(2, 254):
        s = 2.0 ** (b - 127)
        v = CODES[np.abs(CODES) * s <= TOP]
        cols.append(np.resize(v, 32) * s)
        cols.append(np.resize([0.5, 0.0, -1.5], 32) * s)
    return np.stack(cols, 1)


def test_bounds_of_the_oracle():
    rng = np.random.default_rng(0)
    for top in (2.0 ** 128 * (1 - 2.0 ** -24), CUT * (1 + 2.0 ** -20), CUT, 2.0 ** 126, 1.0, 2.0 ** -100, 2.0 ** -120):
        w = rng.uniform(-1, 1, (32, 400)) * top
        w[0] = top
        q = mx.quantise(w)
        s = 2.0 ** np.clip(np.ceil(np.log2(top / 6)), -125, 126)
        size, off = np.abs(w), np.abs(q - w)
        large = size >= CUT
        assert (off[~large] <= np.maximum(0.2 * size, s / 4)[~large]).all(), top
        assert (off[large] <= 0.25 * size[large]).all() and (np.abs(q[large]) == TOP).all()
        assert (size[large] > 0).any() == (top >= CUT)
    # (the looser bound is needed: a fifth does not hold there)
    assert 2.0 ** 128 * (1 - 2.0 ** -24) - TOP > 0.2 * 2.0 ** 128


def test_values_of_the_format_in_the_oracle():
    w = every_scale()
    assert np.array_equal(mx.quantise(w), w)
    # what smaller bytes than 2 have besides, no multiples of 2^-126, and what is larger
    small = np.full((32, 3), [2.0 ** -128, 2.0 ** -127, 1.5 * 2.0 ** -126])
    assert not (mx.quantise(small) == small).any()
    assert (mx.quantise(np.full((32, 1), CUT)) == TOP).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_of_the_format(dtype):
    """Held as they are, whatever the byte: to the bit, there and back."""
    W = torch.from_numpy(every_scale()).to(dtype)[None]
    assert np.array_equal(W[0].double().numpy(), every_scale())
    back = B.moe_unpack_matrix_mx4(B.moe_pack_matrix_mx4(W.cuda()), 1, 32, W.shape[2], dtype)
    assert torch.equal(back.cpu(), W)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_weights(dtype):
    """Finite weights up to the type's largest: as the oracle holds them, a quarter off at most from 3.5 * 2^126 on."""
    rng = np.random.default_rng(1)
    top = float(torch.finfo(dtype).max)
    W = torch.from_numpy(rng.uniform(-1, 1, (64, 48)) * top).to(dtype)
    W[::16] = top
    back = B.moe_unpack_matrix_mx4(B.moe_pack_matrix_mx4(W[None].cuda()), 1, 64, 48, dtype).double().cpu().numpy()[0]
    w = W.double().numpy()
    assert np.array_equal(back, mx.quantise(w))
    large = np.abs(w) >= CUT
    assert large.any() and (np.abs(back - w) <= np.where(large, 0.25, 1.0) * np.abs(w)).all()
