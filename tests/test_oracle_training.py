"""Pins of the training oracle: gradients against central differences of the forward oracle, the 8-bit format against
its definition by hand and against torch's cast.  No GPU needed."""
import numpy as np
import pytest
import torch

from oracle import checkpoint, combine, grouped_ffn
from oracle.backward import combine_backward, grouped_ffn_backward


def differences(f, x, eps=1e-6):
    """Gradient of the scalar f at x, by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        x0 = x[i]
        x[i] = x0 + eps
        up = f()
        x[i] = x0 - eps
        down = f()
        x[i] = x0
        g[i] = (up - down) / (2 * eps)
    return g


@pytest.mark.parametrize("relu", [False, True])
def test_ffn_gradients_are_those_of_the_forward_oracle(relu):
    rng = np.random.default_rng(1)
    d, ffn, E = 3, 4, 3
    W1, W2 = rng.normal(size=(E, d, ffn)), rng.normal(size=(E, ffn, d))
    W3 = None if relu else rng.normal(size=(E, d, ffn))
    slot_expert, seg = np.array([0, 2, -1, 0]), np.array([0, 2, 5, 5, 6])  # expert 0 twice, expert 1 without rows
    x, c = rng.normal(size=(6, d)), rng.normal(size=(6, d))
    loss = lambda: float(np.sum(c * grouped_ffn(x, seg, slot_expert, W1, W3, W2)))
    got = grouped_ffn_backward(x, c, seg, slot_expert, W1, W3, W2)
    for g, v in zip(got, (x, W1, W3, W2)):
        if v is not None:
            np.testing.assert_allclose(g, differences(loss, v), rtol=1e-6, atol=1e-8)
    assert np.all(got[1][1] == 0) and np.all(got[3][1] == 0)


def test_combine_gradients_are_those_of_the_forward_oracle():
    rng = np.random.default_rng(2)
    T, k, d, E = 3, 2, 4, 5
    logits, y, c = rng.normal(size=(T, E)), rng.normal(size=(T * k, d)), rng.normal(size=(T, d))
    rows = rng.permutation(T * k)
    idx = np.argsort(-logits, axis=1)[:, :k]

    def weights():
        z = np.take_along_axis(logits, idx, axis=1)
        z = np.exp(z - z.max(axis=1, keepdims=True))
        return z / z.sum(axis=1, keepdims=True)

    loss = lambda: float(np.sum(c * combine(y, rows, weights(), T, k)))
    dy, dw, dlogits = combine_backward(c, y, rows, weights(), idx, E)
    np.testing.assert_allclose(dy, differences(loss, y), rtol=1e-6, atol=1e-8)
    np.testing.assert_allclose(dlogits, differences(loss, logits), rtol=1e-6, atol=1e-8)
    w = weights()
    np.testing.assert_allclose(dw, differences(lambda: float(np.sum(c * combine(y, rows, w, T, k))), w), rtol=1e-6, atol=1e-8)


def test_codes_against_the_library_cast():
    """Every code, every border between two of them and points on either side, against torch's cast on the CPU."""
    v = checkpoint.e4m3_values()
    assert v[0x7e] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and np.isnan(v[0x7f])
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(table, v)
    pos = v[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    points = np.concatenate([pos, mid, mid * (1 + 1e-6), mid * (1 - 1e-6), np.random.default_rng(0).uniform(0, 448, 4096)])
    points = np.concatenate([points, -points]).astype(np.float32)
    want = torch.from_numpy(points).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(checkpoint.nearest_code(points), want)


def test_scales_at_their_borders():
    """448 * 2^e is held with the scale 2^e, the next number above it with twice that."""
    top = np.float32(448 * 2.0 ** 3)
    x = np.zeros((6, 40), np.float32)
    x[0, 5], x[1, 5], x[2, 5] = top, np.nextafter(top, np.float32(np.inf)), -top
    x[3, 39] = 1e-45                                   # the last group holds eight values; below every normal number
    x[4, 0], x[4, 1] = np.inf, 2.0
    x[5, :] = np.float32(3.4028235e38)
    codes, scales = checkpoint.store(x)
    assert scales[:, 0].tolist() == [130, 131, 130, 127, 127 - 7, 247]
    assert scales[3, 1] == 1 and codes[3, 39] == 0
    back = checkpoint.load(codes, scales)
    assert back[0, 5] == top and back[1, 5] == top and back[2, 5] == -top
    assert np.all(back[5] == 240 * 2.0 ** 120)         # not 2^128
    assert np.isnan(back[4, 0]) and back[4, 1] == 2.0 and np.all(back[4, 2:] == 0)
    rng = np.random.default_rng(3)
    x = rng.normal(size=(64, 96)) * np.exp(3 * rng.normal(size=(64, 1)))
    codes, scales = checkpoint.store(x)
    back = checkpoint.load(codes, scales)
    scale = np.repeat(2.0 ** (scales.astype(float) - 127), 32, axis=1)
    assert np.all(np.abs(back - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * scale))
