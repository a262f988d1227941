"""Training of the layer: what its backward pass keeps, and the gradients.

``MoETraining`` stands beside a ``MoELayer``.  After a step, ``save`` keeps what the backward pass reads, the input rows
and the experts' results, in 8 bits (``moe_checkpoint_store``) or as they are; ``backward`` runs

    moe_combine_backward      dy_perm, gradients of the gate weights and of the router logits
    moe_grouped_ffn_backward  dx_perm, gradients of the expert weights (hidden activations worked out again)
    moe_combine               dx

with no host synchronisation; buffers are allocated once, those of the weights with the first ``set_weights``, so ``save`` and
``backward`` can be recorded into a HIP graph after one eager run, which then reads the weights set last.  Laying changed weights out takes
2.5 ms for 8 bf16 experts of 4096 x 14336, whose gradient takes 7 at 4096 tokens.  The paper trains nothing; the plan only says where a
row is computed and has no gradient.

``python -m paper_2506_07366_amd.training`` fits a small layer to another one's outputs.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding as B
from .layer import MoELayer, torch_dtype


class MoETraining:
    def __init__(self, layer: MoELayer, saved: str = "8bit"):
        """saved: "8bit" keeps x and y_perm as checkpoints (1.03 bytes a value) and a copy of the step's routing, apart from the
        layer's buffers: several layers, or several objects with a micro-batch of one layer each, can be under way; "plain" reads
        all of it where it is: x and the layer are left alone until backward.

        "8bit" is for memory, at a price, in fp32 layers too: a kept value is off by 2.5 % (rms; 6 % at most), and the gradients by as
        much as these errors make, independent from value to value.  Of their norm, normal inputs: dtopk_w 2.5 %, dlogits
        0.8 % (of dtopk_w's norm); dx 3 %, dW1 4 to 5 %, dW3 and dW2 4 % with SwiGLU; dx and dW1 13 %, dW2 2.7 % with ReLU, where an
        error moves sums through 0.  "plain" has none of them."""
        if saved not in ("8bit", "plain"):
            raise B.MoeGpsError(f"saved must be '8bit' or 'plain', got {saved!r}")
        if layer.fused_weights:
            raise B.MoeGpsError("a layer with fused_weights keeps y_perm with the gate weights applied: its gradient needs "
                                "the rows without them")
        if layer.mx4:
            raise B.MoeGpsError("weights in 4 bits are not trained")
        self.layer = layer
        layer.in_training = True
        self.saved = saved
        c = layer.cfg
        dt = torch_dtype(c)
        self._dtype = dt
        like = dict(dtype=dt, device=layer.dev)
        groups = -(-c.d // B.CHECKPOINT_GROUP)
        keep = lambda rows: (torch.empty((rows, c.d), dtype=torch.float8_e4m3fn, device=layer.dev),
                             torch.empty((rows, groups), dtype=torch.uint8, device=layer.dev))
        self._kept = (keep(c.T), keep(c.A)) if saved == "8bit" else None
        self._kept_routing = tuple(torch.empty_like(t) for t in self._live_routing()) if saved == "8bit" else None
        self._x = self._y = self._routing = None
        self.dy_perm = torch.empty((c.A, c.d), **like)
        self.dx_perm = torch.empty((c.A, c.d), **like)
        self.dx = torch.empty((c.T, c.d), **like)
        self.dtopk_w = torch.empty((c.T, c.k), dtype=torch.float32, device=layer.dev)
        self.dlogits = torch.empty((c.T, c.E), dtype=torch.float32, device=layer.dev)
        self.dW1 = torch.empty((c.E, c.d, c.ffn), **like)
        self.dW3 = None if c.act == "relu" else torch.empty((c.E, c.d, c.ffn), **like)
        self.dW2 = torch.empty((c.E, c.ffn, c.d), **like)
        dcode = B.MOE_DTYPE_F32 if c.dtype == "f32" else B.MOE_DTYPE_BF16
        self.workspace = torch.empty(
            B.moe_grouped_ffn_backward_workspace_bytes(c.T, c.k, c.d, c.ffn, c.E, c.nseg, dcode, c.act == "relu"),
            dtype=torch.uint8, device=layer.dev)

    @property
    def packed_backward(self) -> Optional[torch.Tensor]:
        """The layer's: whoever sets its weights, both layouts are of the same ones."""
        return self.layer.packed_backward

    @packed_backward.setter
    def packed_backward(self, packed: Optional[torch.Tensor]) -> None:
        self.layer.packed_backward = packed

    def set_weights(self, W1: torch.Tensor, W3: Optional[torch.Tensor], W2: torch.Tensor) -> None:
        """Lays the weights out for both passes, whenever they have changed; in the same buffers every time, in stream order."""
        self.layer.set_weights(W1, W3, W2)

    def _live_routing(self) -> tuple:
        """What backward reads of the layer's last step besides its rows: all of it 32-bit values."""
        layer, p = self.layer, self.layer.perm
        return (layer.topk_w, layer.topk_idx, p["row_of_assign"], p["assign_of_row"], p["seg_offsets"], layer.slot_expert)

    def save(self, x: torch.Tensor) -> None:
        """Keeps what the backward pass of the layer's last step reads; x: the step's input rows."""
        if self._kept is None:
            self._x, self._y, self._routing = x, self.layer.y_perm, self._live_routing()
            return
        kept_x, kept_y = self._kept
        self._x = B.moe_checkpoint_store(x, out=kept_x)
        self._y = B.moe_checkpoint_store(self.layer.y_perm, out=kept_y)
        # (one launch for all of them, and as tensors of one type)
        torch._foreach_copy_([t.view(torch.int32) for t in self._kept_routing],
                             [t.view(torch.int32) for t in self._live_routing()])
        self._routing = self._kept_routing

    def backward(self, dout: torch.Tensor) -> dict:
        """Gradients of the saved step from that of its output: dx, dtopk_w, dlogits and those of the expert weights, in this
        object's buffers.  The weights are those that the layer has now: they are set for the next step after this."""
        if self.packed_backward is None:
            raise B.MoeGpsError("set_weights() first")
        if self._x is None:
            raise B.MoeGpsError("save() first")
        layer, c = self.layer, self.layer.cfg
        topk_w, topk_idx, row_of_assign, assign_of_row, seg_offsets, slot_expert = self._routing
        B.moe_combine_backward(dout, self._y, row_of_assign, topk_w, topk_idx=topk_idx, E=c.E,
                               out=(self.dy_perm, self.dtopk_w, self.dlogits))
        B.moe_grouped_ffn_backward(self._x, assign_of_row, c.k, self.dy_perm, seg_offsets, slot_expert, layer.packed,
                                   self.packed_backward, c.E, c.ffn, relu=c.act == "relu", workspace=self.workspace,
                                   out=(self.dx_perm, self.dW1, self.dW3, self.dW2))
        B.moe_combine(self.dx_perm, row_of_assign, None, c.T, c.k, out=self.dx)
        return dict(dx=self.dx, dtopk_w=self.dtopk_w, dlogits=self.dlogits, dW1=self.dW1, dW3=self.dW3, dW2=self.dW2)


def example(steps: int = 30, lr: float = 0.5) -> list:
    """Fits the experts of a small fp32 layer to the outputs of another one; returns the losses."""
    import numpy as np
    from . import workloads as wl
    from .layer import to_device

    cfg = wl.CONFIGS["cfg1_tiny_f32"]
    logits = torch.from_numpy(wl.gen_logits(cfg)).cuda()
    x = to_device(wl.to_storage(wl.gen_x(cfg), cfg.dtype), cfg.dtype)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1)
    scale = (cfg.d ** -0.5, cfg.d ** -0.5, cfg.ffn ** -0.5)
    shapes = ((cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.ffn, cfg.d))
    draw = lambda: [s * torch.randn(n, device="cuda", generator=gen) for s, n in zip(scale, shapes)]
    layer = MoELayer(cfg)
    train = MoETraining(layer)
    layer.set_weights(*draw())
    target = layer.step(logits, x, mode=wl.MODE_NONE).clone()
    W = draw()
    losses = []
    for _ in range(steps):
        train.set_weights(*W)
        out = layer.step(logits, x, mode=wl.MODE_NONE)
        train.save(x)
        err = out - target
        losses.append(0.5 * err.square().sum(dim=1).mean())
        g = train.backward(err / cfg.T)
        for w, name in zip(W, ("dW1", "dW3", "dW2")):
            w -= lr * g[name]
    return [float(v) for v in torch.stack(losses).cpu().numpy().astype(np.float64)]


if __name__ == "__main__":
    for i, loss in enumerate(example()):
        print(f"step {i}: loss {loss:.4f}")
