"""Weights in 4 bits and the products with them, from their definition in 64 bits (numpy, on the host)."""
import numpy as np

GROUP = 32
CODES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(w):
    """[..., K, N] float64 -> the values that its 4-bit form stands for."""
    w = np.asarray(w, np.float64)
    out = np.empty_like(w)
    K = w.shape[-2]
    for k0 in range(0, K, GROUP):
        g = w[..., k0:k0 + GROUP, :]
        with np.errstate(invalid="ignore"):
            top = np.abs(g).max(axis=-2, keepdims=True)  # (NaN if there is one)
        bad = ~np.isfinite(top)
        t = np.where(bad | (top == 0), 1.0, top)
        e = np.ceil(np.log2(t / 6.0))
        # (the logarithm may be off by a rounding: settled by comparing)
        e = np.where(6.0 * 2.0 ** (e - 1) >= t, e - 1, np.where(6.0 * 2.0 ** e < t, e + 1, e))
        e = np.where(top == 0, 0, np.clip(e, 2 - 127, 253 - 127))
        s = 2.0 ** e
        a = np.abs(np.where(bad, 0.0, g)) / s
        a = np.where(e == 126, np.minimum(a, 3.0), a)
        # nearest code, of two as near the one with the even number
        d = np.abs(a[..., None] - CODES)
        near = d == d.min(axis=-1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)
        pick = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
        v = np.copysign(CODES[pick], g) * s
        out[..., k0:k0 + GROUP, :] = np.where(bad, np.nan, v)
    return out


def silu(a):
    with np.errstate(over="ignore"):
        return a / (1.0 + np.exp(-a))


def rows_of_experts(seg_offsets, slot_expert, E, seg_begin=0, seg_end=None):
    """expert -> its rows, in the segments [seg_begin, seg_end)."""
    seg_end = len(slot_expert) if seg_end is None else seg_end
    rows = {}
    for i in range(seg_begin, seg_end):
        e = int(slot_expert[i])
        if 0 <= e < E and seg_offsets[i + 1] > seg_offsets[i]:
            rows.setdefault(e, []).extend(range(seg_offsets[i], seg_offsets[i + 1]))
    return rows


def product(x, W, u_sum):
    """x [r, K] times W [K, N]: result, and how far sums in 32 bits may be from it: K + 8 roundings of u_sum each, of
    the sum of magnitudes."""
    return x @ W, (W.shape[0] + 8) * u_sum * (np.abs(x) @ np.abs(W))


def ffn(x, W1, W3, W2, u_sum, u_hidden):
    """The experts' FFN (W3 None: ReLU): result, and the bound of what sums in 32 bits and a hidden activation rounded by u_hidden
    may make of it.  |silu'| <= 1.1; exponential, reciprocal and products of the activation: 16 roundings."""
    a, da = product(x, W1, u_sum)
    if W3 is None:
        h, dh = np.maximum(a, 0), da
    else:
        b, db = product(x, W3, u_sum)
        h = silu(a) * b
        dh = 1.1 * da * (np.abs(b) + db) + np.abs(silu(a)) * db + 16 * u_sum * np.abs(h)
    dh = dh + u_hidden * (np.abs(h) + dh)
    y, dy = product(h, W2, u_sum)
    return y, dh @ np.abs(W2) * (1 + (W2.shape[0] + 8) * u_sum) + dy
