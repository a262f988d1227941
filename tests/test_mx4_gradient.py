"""The gradient of a batch through experts that stay in 4 bits: the formula in 64 bits over the held values, with bounds for 32 bits; against
differences (no GPU needed), and the library's backward pass of the unpacked values against the formula."""
import numpy as np
import pytest
import torch

import mx4_oracle as mx
from gpu_util import Case
from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl

U = 2.0 ** -23
CFG = wl.CONFIGS["cfg1_tiny_f32"].replace(T=16, mode=wl.MODE_NONE)


class Inputs:
    def __init__(self, relu):
        self.cfg = CFG.replace(act="relu" if relu else "swiglu")
        rng = np.random.default_rng(2)
        c = self.cfg
        shapes = ((c.E, c.d, c.ffn), (c.E, c.d, c.ffn), (c.E, c.ffn, c.d))
        self.W = [(0.2 * rng.standard_normal(s)).astype(np.float32) for s in shapes]
        self.held = [mx.quantise(w) for w in self.W]
        if relu:
            self.W[1] = self.held[1] = None
        self.case = Case(c)
        self.x = np.asarray(self.case.x, np.float64)
        self.dout = rng.standard_normal((c.T, c.d)).astype(np.float32)
        self.v = rng.standard_normal((c.T, c.d))

    def sides(self):
        """expert, its tokens, their gate weights"""
        for e in range(self.cfg.E):
            t, j = np.nonzero(self.case.idx == e)
            if len(t):
                yield e, t, self.case.w[t, j].astype(np.float64)[:, None]


def loss(i, x, W):
    """sum of out * dout"""
    total = 0.0
    for e, t, g in i.sides():
        a = x[t] @ W[0][e]
        h = np.maximum(a, 0) if W[1] is None else mx.silu(a) * (x[t] @ W[1][e])
        total += (g * (h @ W[2][e]) * i.dout[t]).sum()
    return total


def gradient(i, W, wrong=None):
    """dx and its bound: K + 8 roundings of U for a sum of K products, 16 for an activation, 2^-20 for a gate weight (a few
    roundings of the softmax); |silu'| <= 1.1, |silu''| <= 0.5.  ReLU's gradient may be either side's where the sum's bound reaches 0.
    `wrong`: a mistake to plant."""
    dx, tol = np.zeros_like(i.x), np.zeros_like(i.x)
    for e, t, g in i.sides():
        W1, W3, W2 = (None if w is None else w[e] for w in W)
        dy = (1.0 if wrong == "no gate weight" else g) * i.dout[t].astype(np.float64)
        ddy = 2.0 ** -20 * np.abs(dy)
        a, da = mx.product(i.x[t], W1, U)
        dh, ddh = mx.product(dy, W2.T, U)
        ddh = ddh + ddy @ np.abs(W2.T)
        if W3 is None:
            on = a > 0
            ga, dga = dh * on, ddh * on + (np.abs(dh) + ddh) * (np.abs(a) <= da)
            r, dr = mx.product(ga, W1.T, U)
            dr = dr + dga @ np.abs(W1.T)
        else:
            b, db = mx.product(i.x[t], W3, U)
            s = 1 / (1 + np.exp(-a))
            slope = s if wrong == "slope" else s * (1 + a * (1 - s))
            ga, gb = dh * b * slope, dh * a * s
            dga = 1.1 * ddh * (np.abs(b) + db) + np.abs(dh) * (1.1 * db + 0.5 * (np.abs(b) + db) * da) + 16 * U * np.abs(dh * b) * 1.1
            dgb = ddh * (np.abs(a * s) + 1.1 * da) + np.abs(dh) * 1.1 * da + 16 * U * np.abs(gb)
            r1, dr1 = mx.product(ga, W1.T, U)
            r3, dr3 = mx.product(gb, W3.T, U)
            r = r1 if wrong == "no W3" else r3 if wrong == "no W1" else r1 + r3
            # (one sum of both)
            dr = 2 * (dr1 + dr3) + dga @ np.abs(W1.T) + dgb @ np.abs(W3.T)
        dx[t] += r
        tol[t] += dr * (1 + 16 * U) + U * np.abs(r)
    return dx, tol + U * np.abs(dx)


@pytest.mark.parametrize("relu", [False, True])
def test_the_formula_against_differences(relu):
    i = Inputs(relu)
    dx, _ = gradient(i, i.held)
    h = 1e-6 if not relu else 1e-9  # (short enough that hardly a ReLU sum changes its sign)
    slope = (loss(i, i.x + h * i.v, i.held) - loss(i, i.x - h * i.v, i.held)) / (2 * h)
    want = (dx * i.v).sum()
    size = (np.abs(dx) * np.abs(i.v)).sum()
    assert abs(slope - want) <= 1e-5 * size and abs(want) > 1e-3 * size, (slope, want, size)


WRONG = ["sign", "half", "no gate weight", "weights of before"]


@pytest.mark.parametrize("relu,wrong", [(r, w) for r in (False, True) for w in WRONG] + [(False, w) for w in ("slope", "no W3", "no W1")])
def test_the_bound_is_narrow(relu, wrong):
    """Far below the gradient itself, and another gradient is outside for most values."""
    i = Inputs(relu)
    dx, tol = gradient(i, i.held)
    assert np.linalg.norm(tol) < 0.02 * np.linalg.norm(dx)
    other = {"sign": -dx, "half": dx / 2}.get(wrong)
    if other is None:
        W = i.held if wrong != "weights of before" else [None if w is None else w.astype(np.float64) for w in i.W]
        other = gradient(i, W, wrong)[0]
    assert (np.abs(other - dx) > 2 * tol).mean() > 0.8, wrong


@pytest.mark.gpu
@pytest.mark.parametrize("relu", [False, True])
def test_the_backward_pass(relu):
    from paper_2506_07366_amd.layer import MoELayer
    from paper_2506_07366_amd.training import MoETraining
    i = Inputs(relu)
    c = i.cfg
    four = MoELayer(c, weights="mx4")
    four.set_weights(*(None if w is None else torch.from_numpy(w).cuda() for w in i.W))
    held = B.moe_unpack_weights_mx4(four.packed, c.E, c.d, c.ffn, torch.float32, relu=relu)
    plain = MoELayer(c)
    train = MoETraining(plain, saved="plain")
    train.set_weights(*held)
    x = i.case.dev_x()
    plain.step(i.case.dev_logits(), x, mode=wl.MODE_NONE)
    train.save(x)
    got = train.backward(torch.from_numpy(i.dout).cuda())["dx"].double().cpu().numpy()
    dx, tol = gradient(i, i.held)
    assert np.array_equal(i.x, x.double().cpu().numpy())
    assert (np.abs(got - dx) <= tol).all(), (np.abs(got - dx) / tol).max()
