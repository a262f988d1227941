"""What a training step keeps from one call to the next: the routing of the saved batch, both layouts of the weights, the
places that a recorded graph reads."""
import numpy as np
import pytest
import torch

from paper_2506_07366_amd.layer import MoELayer
from paper_2506_07366_amd.training import MoETraining
from test_gpu_training_layer import make, step

pytestmark = pytest.mark.gpu


def clones(grads):
    return {n: None if v is None else v.clone() for n, v in grads.items()}


def same(got, want):
    for n, v in want.items():
        assert (got[n] is None) == (v is None) and (v is None or torch.equal(got[n], v)), n


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,k,E,G,S,mode", [(1, 2, 8, 4, 3, 1), (200, 2, 8, 4, 3, 1), (555, 3, 4, 2, 3, 0)])
def test_several_batches_under_way(dtype, T, k, E, G, S, mode):
    """Rows kept in 8 bits, with the routing that belongs to them: the layer's next step may come before the gradients of this one."""
    c = make(T, k, E, G, S, 128, 72, dtype, mode=mode)
    layer, first = c["layer"], c["train"]
    second = MoETraining(layer)
    second.set_weights(c["W1"], c["W3"], c["W2"])
    batches = []
    for i, train in enumerate((first, second)):
        b = dict(c, train=train, x=c["x"].roll(i, dims=1), logits=c["logits"].roll(3 * i, dims=1).contiguous(),
                 hist_pred=c["hist_pred"].roll(2 * i), dout=c["dout"].roll(i, dims=1))
        batches.append((b, clones(step(b))))
    for b, _ in batches:
        layer.step(b["logits"], b["x"], hist_pred=b["hist_pred"])
        b["train"].save(b["x"])
    for b, want in batches:
        same(b["train"].backward(b["dout"]), want)


@pytest.mark.parametrize("dtype,act", [("f32", "swiglu"), ("bf16", "swiglu"), ("bf16", "relu")])
def test_weights_set_on_the_layer(dtype, act):
    """Weights that are set on the layer, not on the object beside it, are those of its gradients too."""
    c = make(150, 2, 8, 4, 3, 128, 72, dtype, act=act, mode=0)
    step(c)
    W = [None if c[n] is None else c[n].flip(0).contiguous() for n in ("W1", "W3", "W2")]
    c["layer"].set_weights(*W)
    got = clones(step(c))
    other = MoETraining(MoELayer(c["cfg"]))
    other.set_weights(*W)
    same(got, step(dict(c, layer=other.layer, train=other)))


@pytest.mark.parametrize("dtype,act", [("f32", "swiglu"), ("bf16", "swiglu"), ("bf16", "relu")])
def test_graph_of_a_step_and_weights_that_change(dtype, act):
    """A recorded training step reads the weights set last: they are laid out in the same place every time."""
    c = make(100, 2, 8, 4, 3, 128, 72, dtype, act=act)
    train, layer = c["train"], c["layer"]
    step(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(c)
    at = (layer.packed.data_ptr(), train.packed_backward.data_ptr())
    size = layer.packed.numel() + train.packed_backward.numel()
    for i in range(3):
        W = [None if c[n] is None else (-0.5 * c[n]).roll(i + 1, dims=0).contiguous() for n in ("W1", "W3", "W2")]
        train.set_weights(*W)
        # (first: nothing is replayed that would read freed memory)
        assert (layer.packed.data_ptr(), train.packed_backward.data_ptr()) == at
        torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # what takes the place of anything freed
        graph.replay()
        torch.cuda.synchronize()
        replayed = clones(got)
        other = MoETraining(MoELayer(c["cfg"]))
        other.set_weights(*W)
        same(replayed, step(dict(c, layer=other.layer, train=other)))


def test_layouts_that_came_from_elsewhere_are_not_written_over():
    """A layer that reads another one's weights gets buffers of its own when its weights are set."""
    c = make(40, 2, 8, 4, 3, 128, 72, "bf16")
    want = clones(step(c))
    other = MoETraining(MoELayer(c["cfg"]))
    other.layer.packed, other.packed_backward = c["layer"].packed, c["train"].packed_backward
    shared = dict(c, layer=other.layer, train=other)
    same(step(shared), want)
    other.set_weights(*[2 * c[n] for n in ("W1", "W3", "W2")])
    step(shared)
    same(step(c), want)


def test_graph_of_two_batches_under_way():
    """Both steps and both saves, then both backward passes, as one graph."""
    c = make(100, 2, 8, 4, 3, 128, 72, "bf16")
    layer = c["layer"]
    batches = [dict(c, train=t, x=c["x"] + 0, logits=c["logits"].roll(i, dims=1).contiguous())
               for i, t in enumerate((c["train"], MoETraining(layer)))]

    def both():
        for b in batches:
            layer.step(b["logits"], b["x"], hist_pred=b["hist_pred"])
            b["train"].save(b["x"])
        return [b["train"].backward(b["dout"]) for b in batches]

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for i in range(4):
        for b in batches:
            b["x"].mul_(-0.5 if i % 2 else 2.0)
            b["logits"].copy_(b["logits"].roll(1, dims=1))
        want = [clones(step(b)) for b in batches]  # (one after the other, each with its gradients)
        for g in got:
            for v in g.values():
                v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            same(g, w)
