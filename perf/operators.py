"""What training adds to the layer, as a set of timed cases with plain forms to hold the results against.

Three operators.  A case is one pass of one of them on data that is resident in device memory:

  op = "checkpoint"        a batch of rows kept as 8-bit codes with a power-of-two scale for every 32 values
                           of a row (store), and given back (load)
  op = "combine_backward"  gradient of the way back from the experts, out[t] = sum_j w[t, j] y[row(t, j)]:
                           rows of dy in expert order, gradients of the gate weights and of the router logits
  op = "ffn_backward"      gradient of the experts' products, y = (silu(x W1) * (x W3)) W2 or max(x W1, 0) W2:
                           rows of dx in expert order and the gradients of all weight matrices.  The hidden
                           activations are worked out again from x

Other fields of a case:

  rows, width, dtype    of the rows that are kept ("checkpoint")
  shape                 name in ``paper_2506_07366_amd.workloads.CONFIGS``: widths, experts, ranks and slots,
                        data type, form of the experts (the other two)
  tokens                tokens of the batch
  saved                 the activation that the backward pass reads (y, or x), as the forward pass left it:
                        "plain" in the layer's type, "8bit" as a checkpoint
  alpha                 Dirichlet concentration of the expert popularity (shapes with Zipf popularity keep it)

Inputs are drawn on the device from the seed alone: activations N(0, 1) with some loud channels and rows,
weights N(0, 0.02), gradients N(0, 1e-3), router logits N(0, 1) + log popularity.  Spare expert slots hold second copies
of the busiest experts, which share their rows.
"""
import math

import numpy as np
import torch

from paper_2506_07366_amd import workloads as wl

own = False

# tokens each shape is trained at
RANGES = {
    "cfg1_tiny_f32": (1, 4096),
    "mid_bf16": (1, 4096),
    "cfg2_mixtral_dist": (1, 4096),
    "cfg4_finegrained": (16, 16384),
    "cfg5_decode_m1": (1, 8192),
    "cfg6_switch_relu": (16, 16384),
    "cfg7_llama_moe": (16, 8192),
}
MOST_COMBINED = 32768 * 8 * 4096        # elements of y of the largest combine_backward
MOST_KEPT = 262144 * 4096               # elements of the largest checkpoint
MOST_TOKENS_COMBINED = 32768
GROUP = 32                              # values that share a scale
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    keep = lambda name, rows, width, dtype: dict(name=name, op="checkpoint", rows=rows, width=width, dtype=dtype)
    back = lambda name, op, shape, tokens, saved, alpha=0.5: dict(name=name, op=op, shape=shape, tokens=tokens,
                                                                  saved=saved, alpha=alpha)
    return [
        # the input rows of a short batch: launches
        keep("keep_128", 128, 4096, "bf16"),
        # an odd number of fp32 rows of a narrow model
        keep("keep_f32_1001", 1001, 768, "f32"),
        # the expert results of a long prefill-sized training batch, 2 GiB
        keep("keep_262144", 262144, 4096, "bf16"),
        # one token of fine-tuning on a single sequence's end: latency
        back("back_one_token", "combine_backward", "cfg5_decode_m1", 1, "plain", 1.0),
        # the training batch of the few-large-experts layer, results kept in 8 bits
        back("back_mixtral_8bit", "combine_backward", "cfg2_mixtral_dist", 4096, "8bit"),
        # the largest batch, eight experts a token
        back("back_32768_8bit", "combine_backward", "cfg5_decode_m1", MOST_TOKENS_COMBINED, "8bit", 1.0),
        # the small fp32 layer that gradients are checked on
        back("ffn_tiny_f32", "ffn_backward", "cfg1_tiny_f32", 256, "plain"),
        # a micro-batch over many small experts: a few rows each, weights and their gradients are all the traffic
        back("ffn_128_of_many", "ffn_backward", "cfg5_decode_m1", 128, "8bit", 1.0),
        # a ragged batch of odd length on few large experts
        back("ffn_mixtral_1001", "ffn_backward", "cfg2_mixtral_dist", 1001, "plain"),
        # ReLU experts, top-1, narrow model, a full batch
        back("ffn_switch_relu", "ffn_backward", "cfg6_switch_relu", 16384, "8bit"),
        # fine-grained experts with Zipf popularity, a full batch
        back("ffn_finegrained", "ffn_backward", "cfg4_finegrained", 16384, "8bit"),
        # a full batch on few large experts: the benchmark's layer
        back("ffn_mixtral_8bit", "ffn_backward", "cfg2_mixtral_dist", 4096, "8bit"),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("checkpoint", "combine_backward", "ffn_backward", "ffn_backward"))
    if op == "checkpoint":
        dtype = rng.choice(("bf16", "bf16", "f32"))
        width = rng.choice((128, 512, 768, 2048, 4096, 4 * rng.randint(1, 1024)))
        return dict(op=op, rows=_spread(rng, 1, min(262144, MOST_KEPT // width // (2 if dtype == "f32" else 1))),
                    width=width if dtype == "f32" else (width + 7) // 8 * 8, dtype=dtype)
    shape = rng.choice(sorted(RANGES))
    lo, hi = RANGES[shape]
    cfg = wl.CONFIGS[shape]
    if op == "combine_backward":
        hi = min(MOST_TOKENS_COMBINED, MOST_COMBINED // (cfg.k * cfg.d))
    return dict(op=op, shape=shape, tokens=_spread(rng, lo, hi), saved=rng.choice(("plain", "8bit")),
                alpha=rng.choice((0.1, 0.5, 1.0, 10.0)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _config(case, seed):
    return wl.CONFIGS[case["shape"]].replace(T=case["tokens"], alpha=case["alpha"], seed=seed)


def _normal(gen, shape, dtype, scale):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=gen)


def _activations(gen, rows, width, dtype):
    """N(0, 1), every row at a level of its own, a few channels ten times as loud."""
    x = _normal(gen, (rows, width), dtype, 1.0)
    level = torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=gen))
    loud = torch.where(torch.rand((1, width), device="cuda", generator=gen) < 0.01, 10.0, 1.0)
    return x.mul_(level.to(dtype)).mul_(loud.to(dtype))


def _to_codes(x):
    """Rows as a checkpoint holds them: e4m3 codes and the biased exponents of the scales, one for every 32 values."""
    rows, width = x.shape
    groups = -(-width // GROUP)
    v = torch.nn.functional.pad(x.float(), (0, groups * GROUP - width)).view(rows, groups, GROUP)
    # the smallest power of two that brings the largest magnitude to 448 = 1.75 * 2^8 or below
    mantissa, exponent = torch.frexp(v.abs().amax(dim=2))  # mantissa in [0.5, 1)
    e = exponent - 9 + (mantissa > 0.875)
    biased = torch.where(mantissa == 0, 127, (e + 127).clamp(1, 254))
    codes = torch.ldexp(v, (127 - biased).unsqueeze(2)).to(torch.float8_e4m3fn)
    return codes.view(rows, groups * GROUP)[:, :width].contiguous(), biased.to(torch.uint8)


def _from_codes(codes, scales):
    rows, width = codes.shape
    exponent = (scales.int() - 127).repeat_interleave(GROUP, dim=1)[:, :width]
    return torch.ldexp(codes.float(), exponent)


def _dispatch(cfg, logits):
    """A batch in expert order: gate weights and ids, both permutations, segments of the slots, rows of an expert."""
    top, idx = torch.topk(logits, cfg.k, dim=1)
    weights = torch.softmax(top, dim=1)
    of = idx.reshape(-1)
    count = torch.bincount(of, minlength=cfg.E)
    count_host = count.cpu().numpy()
    # slots: every expert at home, spare ones hold a second copy of the busiest experts
    home = -(-cfg.E // cfg.G)
    slot_expert = np.full(cfg.nseg, -1, np.int32)
    slots = np.full((cfg.E, 2), -1, np.int64)
    for e in range(cfg.E):
        slots[e, 0] = (e // home) * cfg.S + e % home
        slot_expert[slots[e, 0]] = e
    slots[:, 1] = slots[:, 0]
    for slot, e in zip(np.flatnonzero(slot_expert < 0), np.argsort(-count_host, kind="stable")):
        slot_expert[slot] = e
        slots[e, 1] = slot
    # the first half of an expert's assignments goes home, the rest to the copy
    order = torch.argsort(of, stable=True)
    first = torch.cumsum(count, 0) - count
    rank = torch.empty_like(of)
    rank[order] = torch.arange(cfg.A, device="cuda") - first[of[order]]
    slots = torch.from_numpy(slots).cuda()
    segment = torch.where(2 * rank < count[of], slots[of, 0], slots[of, 1])
    assign_of_row = torch.argsort(segment, stable=True)
    row_of_assign = torch.empty_like(assign_of_row)
    row_of_assign[assign_of_row] = torch.arange(cfg.A, device="cuda")
    seg_offsets = torch.zeros(cfg.nseg + 1, dtype=torch.int64, device="cuda")
    seg_offsets[1:] = torch.cumsum(torch.bincount(segment, minlength=cfg.nseg), 0)
    return dict(topk_w=weights, topk_idx=idx.to(torch.int32), assign_of_row=assign_of_row.to(torch.int32),
                row_of_assign=row_of_assign.to(torch.int32), seg_offsets=seg_offsets.to(torch.int32),
                slot_expert=torch.from_numpy(slot_expert).cuda(), rows_of_expert=count_host.tolist())


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    if case["op"] == "checkpoint":
        return dict(op=case["op"], x=_activations(gen, case["rows"], case["width"], DTYPES[case["dtype"]]))
    cfg = _config(case, seed)
    dt = DTYPES[cfg.dtype]
    bias = torch.from_numpy(np.log(wl.expert_popularity(cfg)).astype(np.float32)).cuda()
    logits = torch.randn((cfg.T, cfg.E), device="cuda", generator=gen) + bias
    state = dict(op=case["op"], cfg=cfg, **_dispatch(cfg, logits))
    if case["op"] == "combine_backward":
        state["dout"] = _normal(gen, (cfg.T, cfg.d), dt, 1e-3)
        saved = _normal(gen, (cfg.A, cfg.d), dt, 0.3)
    else:
        state["dy"] = _normal(gen, (cfg.A, cfg.d), dt, 1e-3)
        state["W1"] = _normal(gen, (cfg.E, cfg.d, cfg.ffn), dt, 0.02)
        state["W3"] = None if cfg.act == "relu" else _normal(gen, (cfg.E, cfg.d, cfg.ffn), dt, 0.02)
        state["W2"] = _normal(gen, (cfg.E, cfg.ffn, cfg.d), dt, 0.02)
        saved = _activations(gen, cfg.T, cfg.d, dt)
    state["saved"] = _to_codes(saved) if case["saved"] == "8bit" else saved
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        from paper_2506_07366_amd import binding as B
        if case["op"] == "checkpoint":
            rows, width = state["x"].shape
            state["kept"] = (torch.empty((rows, width), dtype=torch.float8_e4m3fn, device="cuda"),
                             torch.empty((rows, -(-width // GROUP)), dtype=torch.uint8, device="cuda"))
            state["back"] = torch.empty_like(state["x"])
            return state
        cfg = state["cfg"]
        if case["op"] == "combine_backward":
            state["out"] = (torch.empty((cfg.A, cfg.d), dtype=state["dout"].dtype, device="cuda"),
                            torch.empty((cfg.T, cfg.k), dtype=torch.float32, device="cuda"),
                            torch.empty((cfg.T, cfg.E), dtype=torch.float32, device="cuda"))
            return state
        # weights are laid out when they are set, as for the forward pass, and serve every micro-batch until the next
        # change; the gradients go to buffers that the program keeps
        if cfg.act == "relu":
            state["packed"] = B.moe_pack_weights_relu(state["W1"], state["W2"])
        else:
            state["packed"] = B.moe_pack_weights(state["W1"], state["W3"], state["W2"])
        state["packed_backward"] = B.moe_pack_weights_backward(state["W1"], state["W3"], state["W2"])
        state["out"] = (torch.empty_like(state["dy"]),) + tuple(
            None if state[w] is None else torch.empty_like(state[w]) for w in ("W1", "W3", "W2"))
        state["workspace"] = torch.empty(
            B.moe_grouped_ffn_backward_workspace_bytes(cfg.T, cfg.k, cfg.d, cfg.ffn, cfg.E, cfg.nseg,
                                                       B.dtype_code(state["dy"]), cfg.act == "relu"),
            dtype=torch.uint8, device="cuda")
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_checkpoint(s):
    return _from_codes(*_to_codes(s["x"])).to(s["x"].dtype)


def _plain_combine_backward(s):
    cfg = s["cfg"]
    row = s["row_of_assign"].long().view(cfg.T, cfg.k)
    w = s["topk_w"]
    dout = s["dout"].float()
    y = _from_codes(*s["saved"]) if isinstance(s["saved"], tuple) else s["saved"].float()
    dy = torch.empty((cfg.A, cfg.d), dtype=s["dout"].dtype, device="cuda")
    dy[row] = (dout.unsqueeze(1) * w.unsqueeze(2)).to(dy.dtype)
    dw = (dout.unsqueeze(1) * y[row]).sum(dim=2)
    dlogits = torch.zeros((cfg.T, cfg.E), device="cuda")
    dlogits.scatter_(1, s["topk_idx"].long(), w * (dw - (w * dw).sum(dim=1, keepdim=True)))
    return dict(dy=dy, dtopk_w=dw, dlogits=dlogits)


def _plain_ffn_backward(s):
    cfg = s["cfg"]
    W1, W3, W2 = s["W1"], s["W3"], s["W2"]
    x = _from_codes(*s["saved"]) if isinstance(s["saved"], tuple) else s["saved"].float()
    lengths = s["seg_offsets"].diff().long()
    expert_of_row = s["slot_expert"].long().repeat_interleave(lengths, output_size=cfg.A)
    rows_of = torch.argsort(expert_of_row, stable=True).split(s["rows_of_expert"])
    dx = torch.empty_like(s["dy"])
    grads = [torch.empty_like(W) if W is not None else None for W in (W1, W3, W2)]
    for e in range(cfg.E):
        rows = rows_of[e]
        xe = x[s["assign_of_row"][rows].long() // cfg.k]
        dye = s["dy"][rows].float()
        w1, w2 = W1[e].float(), W2[e].float()
        dh = dye @ w2.t()
        if W3 is None:
            # (which side of 0 a sum is on: in 64 bits)
            a = (xe.double() @ W1[e].double()).float()
            h = a.clamp(min=0)
            da = torch.where(a > 0, dh, 0.0)
            dx[rows] = (da @ w1.t()).to(dx.dtype)
        else:
            w3 = W3[e].float()
            g, u = xe @ w1, xe @ w3
            sig = 1 / (1 + torch.exp(-g))
            h = g * sig * u
            da = dh * u * sig * (1 + g * (1 - sig))
            db = dh * g * sig
            dx[rows] = (da @ w1.t() + db @ w3.t()).to(dx.dtype)
            grads[1][e] = (xe.t() @ db).to(W3.dtype)
        grads[0][e] = (xe.t() @ da).to(W1.dtype)
        grads[2][e] = (h.t() @ dye).to(W2.dtype)
    return _ffn_outputs(dx, *grads)


def _ffn_outputs(dx, dW1, dW3, dW2):
    out = dict(dx=dx, dW1=dW1, dW2=dW2)
    if dW3 is not None:
        out["dW3"] = dW3
    return out


def run(state):
    if not own:
        return {"checkpoint": _plain_checkpoint, "combine_backward": _plain_combine_backward,
                "ffn_backward": _plain_ffn_backward}[state["op"]](state)
    from paper_2506_07366_amd import binding as B
    if state["op"] == "checkpoint":
        codes, scales = B.moe_checkpoint_store(state["x"], out=state["kept"])
        return B.moe_checkpoint_load(codes, scales, state["x"].dtype, out=state["back"])
    cfg = state["cfg"]
    if state["op"] == "combine_backward":
        dy, dw, dlogits = B.moe_combine_backward(state["dout"], state["saved"], state["row_of_assign"], state["topk_w"],
                                                 topk_idx=state["topk_idx"], E=cfg.E, out=state["out"])
        return dict(dy=dy, dtopk_w=dw, dlogits=dlogits)
    return _ffn_outputs(*B.moe_grouped_ffn_backward(
        state["saved"], state["assign_of_row"], cfg.k, state["dy"], state["seg_offsets"], state["slot_expert"],
        state["packed"], state["packed_backward"], cfg.E, cfg.ffn, relu=cfg.act == "relu",
        workspace=state["workspace"], out=state["out"]))


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _kept(saved):
    """What a checkpoint stands for."""
    if not isinstance(saved, tuple):
        return saved.double()
    codes, scales = saved
    scale = 2.0 ** (scales.double() - 127.0)
    return codes.double() * scale[:, torch.arange(codes.shape[1], device="cuda") // GROUP]


def _exact_checkpoint(s):
    """The nearest multiple (ties to the even one) of the step that 4 significant bits have at a value's size."""
    x = s["x"].double()
    group = torch.arange(x.shape[1], device="cuda") // GROUP
    top = torch.zeros((x.shape[0], int(group[-1]) + 1), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(1, group.expand(x.shape[0], -1), x.abs(), "amax")
    scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)).clamp(-126, 127))[:, group]
    v = x / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.where(x == 0, 0.0, torch.round(v / step) * step * scale)


def _exact_combine_backward(s):
    cfg = s["cfg"]
    y, dout, w = _kept(s["saved"]), s["dout"].double(), s["topk_w"].double()
    assign = s["assign_of_row"].long()
    token = assign // cfg.k
    dw = torch.empty(cfg.A, dtype=torch.float64, device="cuda")
    dw[assign] = torch.einsum("rd,rd->r", dout[token], y)
    dw = dw.view(cfg.T, cfg.k)
    dlogits = torch.zeros((cfg.T, cfg.E), dtype=torch.float64, device="cuda")
    mean = (w * dw).sum(1)
    for j in range(cfg.k):  # (ids of a token are distinct)
        dlogits[torch.arange(cfg.T, device="cuda"), s["topk_idx"][:, j].long()] = w[:, j] * (dw[:, j] - mean)
    return dict(dy=dout[token] * w.reshape(-1)[assign].unsqueeze(1), dtopk_w=dw, dlogits=dlogits)


def _exact_ffn_backward(s):
    cfg = s["cfg"]
    x, dy = _kept(s["saved"]), s["dy"]
    offsets = s["seg_offsets"].tolist()
    segments = {}
    for i, e in enumerate(s["slot_expert"].tolist()):
        segments.setdefault(e, []).append(torch.arange(offsets[i], offsets[i + 1], device="cuda"))
    out = dict(dx=torch.zeros(dy.shape, dtype=torch.float64, device="cuda"))
    for name in ("W1", "W3", "W2"):
        if s[name] is not None:
            out["d" + name] = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
    for e in range(cfg.E):
        r = torch.cat(segments[e])
        xe, dye = x[s["assign_of_row"][r].long().div(cfg.k, rounding_mode="floor")], dy[r].double()
        w1, w2 = s["W1"][e].double(), s["W2"][e].double()
        a, dh = xe @ w1, dye @ w2.T
        if cfg.act == "relu":
            on = (a > 0).double()
            out["dW2"][e] = (a * on).T @ dye
            out["dW1"][e] = xe.T @ (dh * on)
            out["dx"][r] = (dh * on) @ w1.T
            continue
        w3 = s["W3"][e].double()
        b, p = xe @ w3, torch.sigmoid(a)
        out["dW2"][e] = (a * p * b).T @ dye
        da = dh * b * (p + a * p * (1 - p))
        db = dh * (a * p)
        out["dW1"][e], out["dW3"][e] = xe.T @ da, xe.T @ db
        out["dx"][r] = da @ w1.T + db @ w3.T
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    return {"checkpoint": _exact_checkpoint, "combine_backward": _exact_combine_backward,
            "ffn_backward": _exact_ffn_backward}[s["op"]](s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _experts_with_rows(cfg):
    """Experts that a batch touches, averaged over a few popularities of the shape's kind."""
    n = []
    for seed in range(4):
        c = cfg.replace(T=min(cfg.T, 1024), seed=1000 + seed)
        n.append(np.unique(np.argpartition(-wl.gen_logits(c), c.k - 1, axis=1)[:, :c.k]).size)
    return float(np.mean(n))


def work(case):
    kept = lambda rows, width: rows * (width + math.ceil(width / GROUP))
    if case["op"] == "checkpoint":
        rows, width = case["rows"], case["width"]
        size = 4 if case["dtype"] == "f32" else 2
        return {"bytes": 2 * (rows * width * size + kept(rows, width)), "flops": 0.0}
    cfg = _config(case, 0)
    size = 4 if cfg.dtype == "f32" else 2
    if case["op"] == "combine_backward":
        y = kept(cfg.A, cfg.d) if case["saved"] == "8bit" else cfg.A * cfg.d * size
        small = 4 * (4 * cfg.A + cfg.T * cfg.E)  # ids, rows, weights and their gradients; dlogits
        return {"bytes": cfg.T * cfg.d * size + y + cfg.A * cfg.d * size + small, "flops": 3.0 * cfg.A * cfg.d}
    matrices = 2 if cfg.act == "relu" else 3
    x = kept(cfg.T, cfg.d) if case["saved"] == "8bit" else cfg.T * cfg.d * size
    weights = (_experts_with_rows(cfg) + cfg.E) * matrices * cfg.d * cfg.ffn * size  # read; gradients of all written
    # hidden activations again, then two products for each of the forward's
    flops = 2.0 * cfg.A * cfg.d * cfg.ffn * (matrices - 1 + 2 * matrices)
    return {"bytes": x + 2 * cfg.A * cfg.d * size + weights + 4 * cfg.A, "flops": flops}
