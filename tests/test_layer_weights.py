"""Weights that a layer refuses: what is packed is opaque bytes, as many of them for a shape as for others (no GPU needed)."""
import pytest
import torch

from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl
from paper_2506_07366_amd.layer import MoELayer

CFG = wl.CONFIGS["cfg1_tiny_f32"].replace(T=4)
E, D, F = CFG.E, CFG.d, CFG.ffn
ASKED = ["moe_pack_weights", "moe_pack_weights_relu", "moe_pack_weights_mx4"]


@pytest.fixture
def packed(monkeypatch):
    """The calls that lay weights out, as a list of what reaches them."""
    calls = []
    for name in ASKED:
        monkeypatch.setattr(B, name, lambda *a, _name=name, **k: calls.append(_name) or torch.empty(256, dtype=torch.uint8))
    return calls


def weights(e=E, d=D, f=F):
    return [torch.zeros(s) for s in ((e, d, f), (e, d, f), (e, f, d))]


@pytest.mark.parametrize("form", ["plain", "mx4"])
@pytest.mark.parametrize("act", ["swiglu", "relu"])
def test_shapes_of_another_layer(form, act, packed):
    layer = MoELayer(CFG.replace(act=act), device="cpu", weights=form)
    W1, W3, W2 = weights()
    t = lambda w: w.transpose(1, 2).contiguous()
    # one half of the widths for the other, fewer experts that are as much wider: as many bytes
    cases = [("W1", [t(W1), t(W3), t(W2)]), ("W1", weights(E // 2, D, 2 * F)), ("W1", weights(E, D // 2, 2 * F)),
             ("W1", [t(W1), W3, W2]), ("W2", [W1, W3, t(W2)]), ("W2", [W1, W3, weights(E + 1)[2]])]
    if act == "swiglu":
        cases.append(("W3", [W1, t(W3), W2]))
    for name, bad in cases:
        with pytest.raises(B.MoeGpsError, match=f"{name} must be \\[{E}, "):
            layer.set_weights(*bad)
    assert not packed and layer.packed is None
    if act == "swiglu":
        with pytest.raises(B.MoeGpsError, match="W3"):
            layer.set_weights(W1, None, W2)
    assert not packed
    layer.set_weights(W1, None if act == "relu" else W3, W2)
    assert len(packed) == 1 and layer.packed is not None


@pytest.mark.parametrize("form", ["plain", "mx4"])
def test_a_relu_layer_does_not_look_at_w3(form, packed):
    layer = MoELayer(CFG.replace(act="relu"), device="cpu", weights=form)
    W1, _, W2 = weights()
    layer.set_weights(W1, torch.zeros(3), W2)
    assert len(packed) == 1
