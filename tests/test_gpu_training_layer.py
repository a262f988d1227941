"""Training of the whole layer (MoETraining): its gradients against the oracle's in 64 bits, against differences of the layer's own
outputs, on another stream and from a HIP graph."""
import numpy as np
import pytest
import torch

from oracle import checkpoint as ck
from oracle.backward import combine_backward, grouped_ffn_backward
from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl
from paper_2506_07366_amd.layer import MoELayer, to_device
from paper_2506_07366_amd.training import MoETraining, example

pytestmark = pytest.mark.gpu

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def make(T, k, E, G, S, d, ffn, dtype, act="swiglu", mode=1, saved="8bit", seed=3, gather=False):
    cfg = wl.MoEConfig("train", T=T, d=d, ffn=ffn, E=E, k=k, G=G, S=S, dtype=dtype, mode=mode, seed=seed, act=act)
    rng = np.random.default_rng([seed, T, E])
    dev = lambda a: to_device(wl.to_storage(a.astype(np.float32), dtype), dtype)
    c = dict(cfg=cfg, x=dev(rng.normal(size=(T, d))), dout=dev(rng.normal(size=(T, d)) * 1e-2),
             logits=torch.from_numpy((rng.normal(size=(T, E)) - 0.3 * np.arange(E)).astype(np.float32)).cuda(),
             W1=dev(rng.normal(size=(E, d, ffn)) * d ** -0.5), W2=dev(rng.normal(size=(E, ffn, d)) * ffn ** -0.5),
             W3=None if act == "relu" else dev(rng.normal(size=(E, d, ffn)) * d ** -0.5))
    c["hist_pred"] = torch.from_numpy(rng.integers(0, 50, E).astype(np.int32)).cuda()
    c["layer"] = MoELayer(cfg, fused_gather=gather)
    c["train"] = MoETraining(c["layer"], saved=saved)
    c["train"].set_weights(c["W1"], c["W3"], c["W2"])
    return c


def step(c):
    c["layer"].step(c["logits"], c["x"], hist_pred=c["hist_pred"])
    c["train"].save(c["x"])
    return c["train"].backward(c["dout"])


def host(t):
    return t.detach().double().cpu().numpy()


def reference(c):
    """From the layer's routing, permutation and results, which have tests of their own."""
    layer, cfg = c["layer"], c["cfg"]
    p = layer.perm
    ints = lambda t: t.cpu().numpy().astype(np.int64)
    kept = lambda t: (host(t) if c["train"].saved == "plain" else ck.load(*ck.store(host(t))))
    x, y = kept(c["x"]), kept(layer.y_perm)
    rows, assign = ints(p["row_of_assign"]), ints(p["assign_of_row"])
    dy, dw, dl = combine_backward(host(c["dout"]), y, rows, host(layer.topk_w), ints(layer.topk_idx), cfg.E)
    W3 = None if c["W3"] is None else host(c["W3"])
    dxp, dW1, dW3, dW2 = grouped_ffn_backward(x[assign // cfg.k], dy, ints(p["seg_offsets"]), ints(layer.slot_expert),
                                              host(c["W1"]), W3, host(c["W2"]))
    return dict(dx=dxp[rows.reshape(cfg.T, cfg.k)].sum(axis=1), dtopk_w=dw, dlogits=dl, dW1=dW1, dW3=dW3, dW2=dW2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("saved", ["8bit", "plain"])
@pytest.mark.parametrize("T,k,E,G,S,act,mode,gather", [
    (1, 2, 8, 4, 3, "swiglu", 1, False),      # one token: most experts have no rows
    (37, 1, 5, 2, 3, "relu", 0, False),
    (200, 2, 8, 4, 3, "swiglu", 1, True),     # replicas; no x_perm
    (300, 4, 6, 3, 4, "relu", 1, False),
    (555, 3, 4, 2, 3, "swiglu", 1, False),    # more than 32 rows per expert
])
def test_layer_gradients(dtype, saved, T, k, E, G, S, act, mode, gather):
    c = make(T, k, E, G, S, 128, 72, dtype, act=act, mode=mode, saved=saved, gather=gather)
    got = step(c)
    want = reference(c)
    assert (got["dW3"] is None) == (act == "relu")
    # of a norm: dy is rounded once, what follows from it in the FFN gives that error once more (each of its roundings is within
    # half a step, their rms a third of that squared), dx is rounded again and summed over k rows.  fp32: sums of up to 128 + 72 terms
    # or of an expert's rows, their roundings independent
    tol = 3 * UNIT["bf16"] if dtype == "bf16" else 128 * UNIT["f32"]
    for name, w in want.items():
        if w is None:
            continue
        g = host(got[name])
        t = 64 * UNIT["f32"] if name in ("dtopk_w", "dlogits") else tol
        # dlogits: differences of products, against the size of what is subtracted
        size = np.linalg.norm(want["dtopk_w"]) if name == "dlogits" else np.linalg.norm(w)
        assert np.linalg.norm(g - w) <= t * size + 1e-30, (name, np.linalg.norm(g - w) / size)
    again = {n: None if v is None else v.clone() for n, v in got.items()}
    for n, v in step(c).items():
        assert v is None or torch.equal(v, again[n])


def test_layer_gradients_against_differences():
    """fp32, from the layer's own outputs: the change of <dout, out> along each gradient, steps of 1e-2 of what is changed (logits: as
    far as no token changes its experts)."""
    c = make(64, 2, 4, 2, 2, 64, 96, "f32", mode=0, saved="plain", seed=8)
    got = {n: v.clone() for n, v in step(c).items()}
    layer = c["layer"]
    ids = layer.topk_idx.clone()

    def loss(**changed):
        t = {**c, **changed}
        layer.set_weights(t["W1"], t["W3"], t["W2"])
        layer.step(t["logits"], t["x"])
        assert torch.equal(layer.topk_idx, ids)
        return float((layer.out.double() * c["dout"].double()).sum())

    for name, grad in (("x", "dx"), ("W1", "dW1"), ("W3", "dW3"), ("W2", "dW2"), ("logits", "dlogits")):
        g = got[grad]
        n = float(g.double().norm())
        h = 1e-2 * float(c[name].double().norm()) / n
        if name == "logits":  # the smallest gap between a selected logit and one that is not, and a tenth of it
            top = torch.topk(c["logits"], 3, dim=1).values
            h = min(h, 0.1 * float((top[:, 1] - top[:, 2]).min()) / float(g.abs().max()))
        up, down = (loss(**{name: c[name] + s * h * g}) for s in (1, -1))
        # (third derivatives: 1e-4 a few times over; fp32 outputs: 1e-6 of <|dout|, |out|>, divided by the step)
        noise = 2e-6 * float((layer.out.double() * c["dout"].double()).abs().sum()) / h
        assert abs((up - down) / (2 * h) - n * n) <= 2e-3 * n * n + noise, name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_on_another_stream(dtype):
    c = make(150, 2, 8, 4, 3, 128, 72, dtype)
    want = {n: v.clone() for n, v in step(c).items()}
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for v in c["train"].backward(c["dout"]).values():
            v.zero_()
        c["layer"].out.zero_()
        got = {n: v.clone() for n, v in step(c).items()}
    side.synchronize()
    assert all(torch.equal(got[n], want[n]) for n in want)


@pytest.mark.parametrize("dtype,T", [("f32", 100), ("bf16", 100), ("bf16", 700)])
def test_captured_training_step(dtype, T):
    """The whole step as a graph, replayed on other inputs with eager work between the replays."""
    c = make(T, 2, 8, 4, 3, 128, 72, dtype)
    step(c)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(c)
    for i in range(4):
        c["x"].mul_(-0.5 if i % 2 else 2.0)
        c["logits"].copy_(c["logits"].roll(1, dims=1))
        c["dout"].neg_()
        want = {n: v.clone() for n, v in step(c).items()}
        torch.cuda.synchronize()
        for v in got.values():
            v.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), i


def test_training_refusals():
    cfg = wl.CONFIGS["cfg1_tiny_f32"]
    layer = MoELayer(cfg)
    with pytest.raises(B.MoeGpsError, match="saved must be"):
        MoETraining(layer, saved="4bit")
    with pytest.raises(B.MoeGpsError, match="fused_weights"):
        MoETraining(MoELayer(cfg, fused_weights=True))
    train = MoETraining(layer)
    dout = torch.zeros((cfg.T, cfg.d), device="cuda")
    with pytest.raises(B.MoeGpsError, match="set_weights"):
        train.backward(dout)
    zeros = lambda *s: torch.zeros(s, device="cuda")
    train.set_weights(zeros(cfg.E, cfg.d, cfg.ffn), zeros(cfg.E, cfg.d, cfg.ffn), zeros(cfg.E, cfg.ffn, cfg.d))
    with pytest.raises(B.MoeGpsError, match=r"save\(\) first"):
        train.backward(dout)
    layer.step(zeros(cfg.T, cfg.E), dout, mode=wl.MODE_NONE)
    with pytest.raises(B.MoeGpsError, match="out codes must be"):
        train.save(dout[:5])
    train.save(dout)
    with pytest.raises(B.MoeGpsError, match="must be"):
        train.backward(dout[:5])


def test_example_learns():
    """Losses of plain gradient descent on a smooth loss with a small step: lower at the end than at the start, and finite."""
    losses = example(steps=20)
    assert np.all(np.isfinite(losses)) and losses[-1] < 0.9 * losses[0]
