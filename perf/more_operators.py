"""Experts whose weights are kept in 4 bits, as a set of timed cases with plain forms to hold the results against.

Three operators.  A case is one pass of one of them on data that is resident in device memory:

  op = "weights"   an FFN's expert weights brought to 4 bits (pack) and given back (unpack)
  op = "product"   one matrix per expert: y[r] = w[r] (x[r] W_e) for the rows r of expert e, ragged numbers of rows
  op = "ffn"       the experts' FFN, y[r] = w[r] (silu(x[r] W1_e) * (x[r] W3_e)) W2_e or w[r] max(x[r] W1_e, 0) W2_e

A weight in 4 bits is code * 2^(b - 127): 32 neighbours along the dimension that is summed over share the byte b, the smallest with
no magnitude of theirs above 6 * 2^(b - 127); a code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, the nearest, ties to
the one with the even last bit.

Other fields of a case:

  dtype                 of the activations, and of the weights before and after ("f32", "bf16")
  d, ffn                model width and hidden width; a "product" takes d to ffn
  experts, topk         experts of the layer, experts of a token
  act                   "swiglu" or "relu" ("weights", "ffn")
  tokens                tokens of the batch ("product", "ffn")
  gather                True: the rows are those of the tokens, read through the permutation, and results carry
                        their gate weights; False: permuted rows in place, no gate weights
  alpha                 Dirichlet concentration of the expert popularity

Inputs are drawn on the device from the seed alone: activations N(0, 1) with some loud channels and rows, weights
N(0, 0.02) with some loud rows, router logits N(0, 1) + log popularity.  Spare expert slots hold second copies of the busiest
experts, which share their rows.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32                 # weights that share a scale
VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
MOST_WEIGHTS = 8 * 3 * 4096 * 14336        # of the largest "weights" case
MOST_FLOPS = 6 * 4096 * 2 * 4096 * 14336   # of the largest products


def listed():
    shape = lambda dtype, d, ffn, experts, topk, act="swiglu": dict(dtype=dtype, d=d, ffn=ffn, experts=experts, topk=topk,
                                                                    act=act)
    tiny = shape("f32", 128, 256, 8, 2)
    many = shape("bf16", 4096, 1536, 128, 8)
    large = shape("bf16", 4096, 14336, 8, 2)
    fine = shape("bf16", 2048, 1408, 64, 6)
    cut = shape("bf16", 4096, 688, 16, 4)
    narrow = shape("bf16", 768, 2048, 64, 1, "relu")
    batch = lambda name, op, s, tokens, gather=True, alpha=0.5: dict(s, name=name, op=op, tokens=tokens, gather=gather, alpha=alpha)
    return [
        # the weights of a small fp32 layer: launches
        dict(tiny, name="weights_tiny_f32", op="weights"),
        # a layer's weights as a checkpoint is loaded
        dict(large, name="weights_mixtral", op="weights"),
        # one projection for one token, eight experts of it: latency
        batch("product_one_token", "product", many, 1, alpha=1.0),
        # one projection of a ragged prompt batch of odd length
        batch("product_8191", "product", cut, 8191, gather=False),
        # one token of a generation, the whole FFN: latency
        batch("ffn_one_token", "ffn", many, 1, alpha=1.0),
        # the small fp32 layer
        batch("ffn_tiny_f32", "ffn", tiny, 256, gather=False),
        # a decode batch on few large experts
        batch("ffn_mixtral_16", "ffn", large, 16),
        # a decode batch on many small experts, the benchmark's
        batch("ffn_decode_128", "ffn", many, 128, alpha=1.0),
        # ReLU experts, top-1, narrow model, a prompt of odd length
        batch("ffn_relu_4001", "ffn", narrow, 4001, gather=False),
        # a short prompt: between bytes and arithmetic
        batch("ffn_fine_777", "ffn", fine, 777),
        # a full batch of fine-grained experts
        batch("ffn_fine_16384", "ffn", fine, 16384),
        # a full batch on few large experts: the benchmark's layer
        batch("ffn_mixtral_4096", "ffn", large, 4096),
    ]


def _spread(rng, lo, hi):
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(("weights", "product", "ffn", "ffn", "ffn"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    # widths up to the largest layer's; rows are multiples of 16 bytes, the hidden width is anything
    piece = 8 if dtype == "bf16" else 4
    d = piece * _spread(rng, 64 // piece, 4096 // piece) if rng.random() < 0.5 else rng.choice((128, 768, 2048, 4096))
    ffn = _spread(rng, 64, 14336) if op != "product" else 8 * _spread(rng, 8, 1792)
    act = rng.choice(("swiglu", "swiglu", "relu"))
    matrices = 3 if act == "swiglu" else 2
    most = MOST_WEIGHTS // (matrices * d * ffn) // (2 if dtype == "f32" else 1)
    experts = _spread(rng, 1, max(1, min(256, most)))
    topk = _spread(rng, 1, min(8, experts))
    case = dict(op=op, dtype=dtype, d=d, ffn=ffn, experts=experts, topk=topk, act=act)
    if op == "weights":
        return case
    # an fp32 product is three bf16 ones
    flops = 2.0 * topk * d * ffn * (matrices if op == "ffn" else 1) * (3 if dtype == "f32" else 1)
    tokens = _spread(rng, 1, max(1, min(32768, int(MOST_FLOPS / flops))))
    return dict(case, tokens=tokens, gather=rng.random() < 0.5, alpha=rng.choice((0.1, 0.5, 1.0, 10.0)))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(gen, shape, dtype, scale):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=gen)


def _activations(gen, rows, width, dtype):
    """N(0, 1), every row at a level of its own, a few channels ten times as loud."""
    x = _normal(gen, (rows, width), dtype, 1.0)
    level = torch.exp(0.5 * torch.randn((rows, 1), device="cuda", generator=gen))
    loud = torch.where(torch.rand((1, width), device="cuda", generator=gen) < 0.01, 10.0, 1.0)
    return x.mul_(level.to(dtype)).mul_(loud.to(dtype))


def _weights(gen, experts, k, n, dtype):
    """N(0, 0.02), a few rows five times as loud."""
    loud = torch.where(torch.rand((experts, k, 1), device="cuda", generator=gen) < 0.005, 5.0, 1.0)
    return _normal(gen, (experts, k, n), dtype, 0.02).mul_(loud.to(dtype))


def _to_codes(w):
    """[K, N] -> codes [K, N] (sign in bit 3) and biased exponents [ceil(K / 32), N]."""
    k, n = w.shape
    groups = -(-k // GROUP)
    v = torch.nn.functional.pad(w.float(), (0, 0, 0, groups * GROUP - k)).view(groups, GROUP, n)
    # the smallest power of two that brings the largest magnitude to 6 = 0.75 * 2^3 or below
    mantissa, exponent = torch.frexp(v.abs().amax(dim=1))  # mantissa in [0.5, 1)
    e = exponent - 3 + (mantissa > 0.75)
    biased = torch.where(mantissa == 0, 127, (e + 127).clamp(2, 253))
    a = torch.ldexp(v, (127 - biased).unsqueeze(1))
    m = a.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    # (a border belongs to the neighbour whose last bit is 0)
    for border, below in ((0.25, True), (0.75, False), (1.25, True), (1.75, False), (2.5, True), (3.5, False), (5.0, True)):
        code += m > border if below else m >= border
    code += (a < 0).to(torch.uint8) * 8
    return code.view(groups * GROUP, n)[:k].contiguous(), biased.to(torch.uint8)


def _from_codes(codes, scales):
    """fp32 values of codes [K, N]."""
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device="cuda")
    exponent = (scales.int() - 127).repeat_interleave(GROUP, dim=0)[:codes.shape[0]]
    return torch.ldexp(table[codes.int()], exponent)


def _kept(gen, experts, k, n, dtype):
    """Weights as a 4-bit checkpoint holds them: codes and scales of every expert."""
    w = _weights(gen, experts, k, n, dtype)
    pairs = [_to_codes(w[e]) for e in range(experts)]
    return torch.stack([c for c, _ in pairs]), torch.stack([s for _, s in pairs])


def _dense(kept, dtype):
    """Values of codes and scales in dtype, where they are exact: what a program that holds a 4-bit checkpoint makes of it, once, for
    moe_pack_weights_mx4.  Two codes are one look-up; a scale's byte is the exponent field of its power of two."""
    codes, scales = kept
    whole = codes.shape[1] // GROUP
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), device="cuda", dtype=dtype)
    pair = torch.arange(16 * 256, device="cuda")
    pairs = table[torch.stack((pair % 16, pair // 256), dim=1)]
    two = torch.int32 if dtype == torch.bfloat16 else torch.int64
    w = pairs.view(two).view(-1).index_select(0, codes.view(-1).view(torch.int16).int()).view(dtype).view(codes.shape)
    scale = (scales.short() << 7).view(dtype) if dtype == torch.bfloat16 else (scales.int() << 23).view(dtype)
    w[:, :whole * GROUP].unflatten(1, (whole, GROUP)).mul_(scale[:, :whole].unsqueeze(2))
    w[:, whole * GROUP:].mul_(scale[:, whole:])
    return w


def _dispatch(case, gen, seed):
    """A batch in expert order: gate weights, the permutation, segments of the slots, rows of an expert."""
    E, T, k = case["experts"], case["tokens"], case["topk"]
    popularity = np.random.default_rng(seed).dirichlet(np.full(E, case["alpha"]))
    bias = torch.from_numpy(np.log(np.maximum(popularity, 1e-30)).astype(np.float32)).cuda()
    logits = torch.randn((T, E), device="cuda", generator=gen) + bias
    top, idx = torch.topk(logits, k, dim=1)
    of = idx.reshape(-1)
    count = torch.bincount(of, minlength=E)
    count_host = count.cpu().numpy()
    # a slot for every expert, and one in four besides for second copies of the busiest
    spare = -(-E // 4)
    slot_expert = np.full(E + spare, -1, np.int32)
    slot_expert[:E] = np.arange(E)
    copy = np.arange(E)
    for slot, e in zip(range(E, E + spare), np.argsort(-count_host, kind="stable")):
        slot_expert[slot] = e
        copy[e] = slot
    # the first half of an expert's assignments goes home, the rest to the copy
    order = torch.argsort(of, stable=True)
    first = torch.cumsum(count, 0) - count
    rank = torch.empty_like(of)
    rank[order] = torch.arange(T * k, device="cuda") - first[of[order]]
    segment = torch.where(2 * rank < count[of], of, torch.from_numpy(copy).cuda()[of])
    assign_of_row = torch.argsort(segment, stable=True)
    seg_offsets = torch.zeros(E + spare + 1, dtype=torch.int64, device="cuda")
    seg_offsets[1:] = torch.cumsum(torch.bincount(segment, minlength=E + spare), 0)
    return dict(topk_w=torch.softmax(top, dim=1), assign_of_row=assign_of_row.to(torch.int32),
                seg_offsets=seg_offsets.to(torch.int32), slot_expert=torch.from_numpy(slot_expert).cuda(),
                rows_of_expert=count_host.tolist())


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    E, d, ffn, dt = case["experts"], case["d"], case["ffn"], DTYPES[case["dtype"]]
    relu = case["act"] == "relu"
    shapes = dict(W1=(d, ffn), W3=(d, ffn), W2=(ffn, d))
    if relu:
        del shapes["W3"]
    if case["op"] == "weights":
        return dict(case=case, **{name: _weights(gen, E, k, n, dt) for name, (k, n) in shapes.items()})
    if case["op"] == "product":
        shapes = dict(W1=(d, ffn))
    state = dict(case=case, **_dispatch(case, gen, seed))
    state.update({name: _kept(gen, E, k, n, dt) for name, (k, n) in shapes.items()})
    state["x"] = _activations(gen, case["tokens"], d, dt)
    if not case["gather"]:
        state["x"] = state["x"][state["assign_of_row"].long() // case["topk"]]
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    if own:
        from paper_2506_07366_amd import binding as B
        E, d, ffn, dt = case["experts"], case["d"], case["ffn"], DTYPES[case["dtype"]]
        relu = case["act"] == "relu"
        if case["op"] == "weights":
            state["packed"] = torch.empty(B.moe_packed_weights_mx4_bytes(E, d, ffn, relu), dtype=torch.uint8, device="cuda")
            state["back"] = tuple(torch.empty_like(state[w]) if w in state else None for w in ("W1", "W3", "W2"))
            return state
        # weights are packed once, as a layer is loaded; results go to buffers that the program keeps
        A = case["tokens"] * case["topk"]
        code, nseg = B.dtype_code(state["x"]), state["slot_expert"].numel()
        if case["op"] == "product":
            state["packed"] = B.moe_pack_matrix_mx4(_dense(state["W1"], dt))
            size = B.moe_grouped_product_mx4_workspace_bytes(A, d, ffn, nseg, code)
        else:
            state["packed"] = B.moe_pack_weights_mx4(*(_dense(state[w], dt) if w in state else None for w in ("W1", "W3", "W2")))
            size = B.moe_grouped_ffn_mx4_workspace_bytes(A, d, ffn, nseg, code)
        state["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        state["out"] = torch.empty((A, ffn if case["op"] == "product" else d), dtype=dt, device="cuda")
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_weights(s):
    out = {}
    for name in ("W1", "W3", "W2"):
        if name in s:
            out[name] = torch.empty_like(s[name])
            for e in range(s[name].shape[0]):
                out[name][e] = _from_codes(*_to_codes(s[name][e])).to(out[name].dtype)
    return out


def _rows_by_expert(s):
    A = s["assign_of_row"].numel()
    expert_of_row = s["slot_expert"].long().repeat_interleave(s["seg_offsets"].diff().long(), output_size=A)
    return torch.argsort(expert_of_row, stable=True).split(s["rows_of_expert"])


def _plain_products(s):
    case = s["case"]
    rows_of = _rows_by_expert(s)
    gate = s["topk_w"].reshape(-1)
    out = torch.empty((s["assign_of_row"].numel(), case["ffn"] if case["op"] == "product" else case["d"]), dtype=s["x"].dtype,
                      device="cuda")
    for e, rows in enumerate(rows_of):
        if rows.numel() == 0:
            continue
        assign = s["assign_of_row"][rows].long()
        xe = s["x"][assign // case["topk"] if case["gather"] else rows].float()
        w = {name: _from_codes(s[name][0][e], s[name][1][e]) for name in ("W1", "W3", "W2") if name in s}
        y = xe @ w["W1"]
        if case["op"] == "ffn":
            y = y.clamp(min=0) if "W3" not in w else y / (1 + torch.exp(-y)) * (xe @ w["W3"])
            y = y @ w["W2"]
        out[rows] = (y * gate[assign].unsqueeze(1) if case["gather"] else y).to(out.dtype)
    return out


def run(state):
    case = state["case"]
    if not own:
        return _plain_weights(state) if case["op"] == "weights" else _plain_products(state)
    from paper_2506_07366_amd import binding as B
    relu = case["act"] == "relu"
    if case["op"] == "weights":
        packed = B.moe_pack_weights_mx4(state["W1"], state.get("W3"), state["W2"], out=state["packed"])
        back = B.moe_unpack_weights_mx4(packed, case["experts"], case["d"], case["ffn"], state["W1"].dtype, relu=relu,
                                        out=state["back"])
        return {name: w for name, w in zip(("W1", "W3", "W2"), back) if w is not None}
    rows = dict(workspace=state["workspace"], out=state["out"])
    if case["gather"]:
        rows.update(assign_of_row=state["assign_of_row"], k=case["topk"], topk_w=state["topk_w"])
    if case["op"] == "product":
        return B.moe_grouped_product_mx4(state["x"], state["seg_offsets"], state["slot_expert"], state["packed"], case["experts"],
                                         case["ffn"], **rows)
    return B.moe_grouped_ffn_mx4(state["x"], state["seg_offsets"], state["slot_expert"], state["packed"], case["experts"],
                                 case["ffn"], relu=relu, **rows)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_back(w):
    """[K, N]: the nearest multiple (ties to the even one) of the step that 2 significant bits have at a value's size."""
    group = torch.arange(w.shape[0], device="cuda") // GROUP
    x = w.double()
    top = torch.zeros((int(group[-1]) + 1, w.shape[1]), dtype=torch.float64, device="cuda")
    top.scatter_reduce_(0, group.unsqueeze(1).expand(-1, w.shape[1]), x.abs(), "amax")
    scale = torch.exp2(torch.ceil(torch.log2(top / 6.0)).clamp(-125, 126))[group]
    v = x / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=1.0))) - 1)
    return torch.where(x == 0, 0.0, torch.round(v / step) * step * scale)


def _exact_value(codes, scales):
    c = codes.long()
    size, odd = (c & 7) >> 1, (c & 1).double()
    value = torch.where(size == 0, 0.5 * odd, (1.0 + 0.5 * odd) * 2.0 ** (size - 1).double())
    value = value * (1.0 - 2.0 * (c >> 3).double())
    return value * (2.0 ** (scales.double() - 127.0))[torch.arange(c.shape[0], device="cuda") // GROUP]


def _exact_products(s):
    case = s["case"]
    offsets, slots = s["seg_offsets"].tolist(), s["slot_expert"].tolist()
    width = case["ffn"] if case["op"] == "product" else case["d"]
    out = torch.zeros((offsets[-1], width), dtype=torch.float64, device="cuda")
    for e in range(case["experts"]):
        r = [torch.arange(offsets[i], offsets[i + 1], device="cuda") for i, of in enumerate(slots) if of == e]
        r = torch.cat(r)
        if len(r) == 0:
            continue
        a = s["assign_of_row"][r].long()
        x = s["x"][a.div(case["topk"], rounding_mode="floor") if case["gather"] else r].double()
        y = x @ _exact_value(s["W1"][0][e], s["W1"][1][e])
        if case["op"] == "ffn":
            if case["act"] == "relu":
                y = torch.relu(y)
            else:
                y = y * torch.sigmoid(y) * (x @ _exact_value(s["W3"][0][e], s["W3"][1][e]))
            y = y @ _exact_value(s["W2"][0][e], s["W2"][1][e])
        if case["gather"]:
            y = y * s["topk_w"].double().view(-1, 1)[a]
        out[r] = y
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["op"] != "weights":
        return _exact_products(s)
    out = {}
    for name in ("W1", "W3", "W2"):
        if name in s:
            out[name] = torch.empty(s[name].shape, dtype=torch.float64, device="cuda")
            for e in range(case["experts"]):
                out[name][e] = _exact_back(s[name][e])
    return out


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def _experts_with_rows(case):
    """Experts that a batch touches, averaged over a few popularities of the case's kind."""
    E, k = case["experts"], case["topk"]
    n = []
    for seed in range(8):
        rng = np.random.default_rng(1000 + seed)
        bias = np.log(np.maximum(rng.dirichlet(np.full(E, case["alpha"])), 1e-30))
        logits = rng.standard_normal((min(case["tokens"], 1024), E)) + bias
        n.append(np.unique(np.argpartition(-logits, k - 1, axis=1)[:, :k]).size)
    return float(np.mean(n))


def work(case):
    d, ffn = case["d"], case["ffn"]
    size = 4 if case["dtype"] == "f32" else 2
    in4 = lambda k, n: k * n / 2 + math.ceil(k / GROUP) * n
    first = 1 if case["op"] == "product" or case["act"] == "relu" else 2
    kept = first * in4(d, ffn) + (0 if case["op"] == "product" else in4(ffn, d))
    if case["op"] == "weights":
        return {"bytes": 2 * case["experts"] * (kept + (first + 1) * d * ffn * size), "flops": 0.0}
    A = case["tokens"] * case["topk"]
    rows = case["tokens"] if case["gather"] else A
    matrices = first if case["op"] == "product" else first + 1
    small = 4 * A * (2 if case["gather"] else 0)  # ids and gate weights
    out = ffn if case["op"] == "product" else d
    return {"bytes": _experts_with_rows(case) * kept + (rows * d + A * out) * size + small,
            "flops": 2.0 * A * d * ffn * matrices}
