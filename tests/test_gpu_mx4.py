"""Experts with weights in 4 bits against the definition in 64 bits: packing and back, ragged products, the FFN, the layer.

Tolerances.  What is held in 4 bits has to be equal.  A product's sum of K exact products is off by at most a rounding of 2^-23 of the sum of
magnitudes for every addition (K, and a handful of parts that are joined); a result in bf16 is rounded by 2^-8 of itself at most, one in
fp32 and every multiplication with a gate weight by 2^-24; the FFN's hidden activation is rounded like a result (mx4_oracle.ffn)."""
import ctypes

import numpy as np
import pytest
import torch

import mx4_oracle as mx
from gpu_util import Case
from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl
from paper_2506_07366_amd.layer import MoELayer
from paper_2506_07366_amd.training import MoETraining

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U_SUM = 2.0 ** -23


def u_of(dtype):
    return torch.finfo(dtype).eps / 2


def host(t):
    return t.detach().double().cpu().numpy()


def normal(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(dtype).cuda()


# ---------------------------------------------------------------------------
# weights to 4 bits and back
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("E,K,N", [(1, 1, 1), (2, 32, 32), (3, 33, 31), (1, 64, 256), (2, 65, 257), (1, 300, 130), (4, 96, 7), (1, 257, 514)])
def test_matrix_there_and_back(dtype, E, K, N):
    rng = np.random.default_rng(K * 1000 + N)
    W = normal(rng, (E, K, N), dtype) * torch.from_numpy(np.exp2(rng.integers(-8, 9, (E, K, N))).astype(np.float32)).to(dtype).cuda()
    packed = B.moe_pack_matrix_mx4(W)
    for out_type in (BF16, F32):
        back = B.moe_unpack_matrix_mx4(packed, E, K, N, out_type)
        assert np.array_equal(host(back), mx.quantise(host(W)))
        # what is held is held exactly (not byte by byte: a group whose largest weight was 3.4 s holds 3 s, which s / 2 does for)
        assert torch.equal(B.moe_unpack_matrix_mx4(B.moe_pack_matrix_mx4(back), E, K, N, out_type), back)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("E,d,ffn", [(1, 8, 1), (2, 64, 64), (3, 136, 65), (2, 72, 200), (1, 512, 333)])
def test_weights_there_and_back(dtype, relu, E, d, ffn):
    rng = np.random.default_rng(d + ffn)
    W1, W3, W2 = (normal(rng, s, dtype, 0.02) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d)))
    if relu:
        W3 = None
    packed = B.moe_pack_weights_mx4(W1, W3, W2)
    assert packed.numel() == B.moe_packed_weights_mx4_bytes(E, d, ffn, relu)
    back = B.moe_unpack_weights_mx4(packed, E, d, ffn, dtype, relu=relu)
    for w, b in zip((W1, W3, W2), back):
        assert (w is None) == (b is None)
        if w is not None:
            assert np.array_equal(host(b), mx.quantise(host(w)))
    again = torch.full_like(packed, 0xa5)
    B.moe_pack_weights_mx4(*back, out=again)
    for a, b in zip(B.moe_unpack_weights_mx4(again, E, d, ffn, dtype, relu=relu), back):
        assert a is b is None or torch.equal(a, b)
    only = torch.full_like(W2, 7.0)
    B.moe_unpack_weights_mx4(packed, E, d, ffn, dtype, relu=relu, out=(None, None, only))
    assert torch.equal(only, back[2])
    if not relu:
        only = torch.full_like(W1, 7.0)
        B.moe_unpack_weights_mx4(packed, E, d, ffn, dtype, out=(None, only, None))
        assert torch.equal(only, back[1])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_at_borders_and_ends(dtype):
    """Borders between codes (one in a group sets the scale), the largest and the smallest values, groups without a finite value."""
    cols = []
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    eps = torch.finfo(dtype).eps
    for e in (-100, -3, 0, 50):
        for f in (1.0, 1 + eps, 1 - eps / 2):
            g = np.zeros(32)
            g[0] = 6.0
            g[1:8], g[8:15] = borders * f, -borders * f
            cols.append(g * 2.0 ** e)
    top = float(torch.finfo(dtype).max)
    tiny = float(torch.finfo(dtype).tiny)
    for t in (top, top / 4 * 3, top / 2, tiny, tiny / 2, tiny / 4, tiny * 3, 0.0):
        g = np.linspace(-1, 1, 32) * t
        cols.append(g)
        cols.append(-g * 0.9)
    for bad in (np.inf, -np.inf, np.nan):
        g = np.linspace(-1, 1, 32)
        g[5] = bad
        cols.append(g)
    W = torch.from_numpy(np.stack(cols, 1)).to(dtype)[None]
    back = B.moe_unpack_matrix_mx4(B.moe_pack_matrix_mx4(W.cuda()), 1, 32, W.shape[2], dtype)
    ref = mx.quantise(W.double().numpy())
    assert np.array_equal(host(back), ref, equal_nan=True)
    assert np.isfinite(ref[0, :, :-3]).all() and np.isnan(ref[0, :, -3:]).all()


def test_a_weight_panel_further_than_32_bits():
    """Experts behind the 2^31st byte of their weights, packed and as they are."""
    E, K, N = 130, 4096, 4096
    W = torch.zeros((E, K, N), dtype=BF16, device="cuda")
    assert W.numel() * 2 > 2 ** 32
    rng = np.random.default_rng(1)
    W[0, :64, :64] = normal(rng, (64, 64), BF16)
    W[-1, -64:, -64:] = normal(rng, (64, 64), BF16)
    packed = B.moe_pack_matrix_mx4(W)
    x = normal(rng, (2, K), BF16)
    se = torch.tensor([0, E - 1], dtype=torch.int32, device="cuda")
    so = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    y = host(B.moe_grouped_product_mx4(x, so, se, packed, E, N))
    W = B.moe_unpack_matrix_mx4(packed, E, K, N, BF16, out=W)
    for r, e in ((0, 0), (1, E - 1)):
        ref, tol = mx.product(host(x[r:r + 1]), host(W[e]), U_SUM)
        assert (np.abs(y[r] - ref[0]) <= tol[0] + u_of(BF16) * (np.abs(ref[0]) + tol[0])).all()
        assert np.abs(ref).max() > 0


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
@pytest.fixture(params=[-1, 0, 1, 2], ids=["auto", "tall", "split", "wide"])
def form(request):
    """The form of bf16 products: by the rule, tall tiles, K split between wavefronts, eight panels side by side."""
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, request.param)
    yield request.param
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, -1)


class Batch:
    """Rows of segments: lengths of the segments and the experts that their slots hold (-1: none)."""

    def __init__(self, rng, lengths, experts, E, gather, k=2):
        self.E = E
        self.so = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
        self.se = np.array(experts, np.int32)
        self.A = int(self.so[-1])
        self.k = k if gather else 1
        while self.A % self.k:
            self.k -= 1
        self.assign = rng.permutation(self.A).astype(np.int32) if gather else None
        self.gate = rng.random(self.A).astype(np.float32) if gather else None
        self.rows_x = self.A // self.k

    def kwargs(self):
        dev = lambda a: torch.from_numpy(a).cuda()
        kw = dict(seg_offsets=dev(self.so), slot_expert=dev(self.se))
        if self.assign is not None:
            kw.update(assign_of_row=dev(self.assign), k=self.k, topk_w=dev(self.gate).view(self.rows_x, self.k))
        return kw

    def rows(self, x, of):
        return x[self.assign[of] // self.k] if self.assign is not None else x[of]

    def check(self, got, one, dtype, untouched, seg_begin=0, seg_end=None):
        """one(expert, rows of this expert) -> (result, bound)"""
        seen = np.zeros(self.A, bool)
        for e, of in mx.rows_of_experts(self.so, self.se, self.E, seg_begin, seg_end).items():
            ref, tol = one(e, np.array(of))
            if self.gate is not None:
                g = self.gate[self.assign[of]].astype(np.float64)[:, None]
                ref, tol = ref * g, tol * g + 2.0 ** -24 * np.abs(ref * g)
            tol = tol + u_of(dtype) * (np.abs(ref) + tol)
            bad = ~(np.abs(got[of] - ref) <= tol)
            assert not bad.any(), (e, np.argwhere(bad)[:4], got[of][bad][:4], ref[bad][:4], tol[bad][:4])
            seen[of] = True
        assert (got[~seen] == untouched).all()


# rows of the segments, experts of their slots
RAGGED = [
    ([1], [0]),
    ([0, 1, 0], [1, 0, 2]),
    ([16, 17, 15, 0, 1], [0, 1, 2, 3, 0]),
    ([32, 33, 31, 5, 3], [3, 1, -1, 1, 0]),
    ([64, 65, 0, 63, 2], [0, 1, 2, 3, 1]),
    ([100, 7, 129, 1], [2, 2, 0, 1]),
    ([256, 257, 40], [1, 0, 1]),
    ([600, 3, 511], [0, 1, 0]),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,N", [(8, 8), (64, 32), (72, 40), (128, 256), (200, 264), (512, 136), (1544, 72)])
@pytest.mark.parametrize("gather", [False, True])
def test_product(dtype, K, N, gather, form):
    rng = np.random.default_rng(K + N)
    E = 4
    W = normal(rng, (E, K, N), dtype, 0.05)
    packed = B.moe_pack_matrix_mx4(W)
    Wq = mx.quantise(host(W))
    for lengths, experts in RAGGED:
        b = Batch(rng, lengths, experts, E, gather)
        x = normal(rng, (b.rows_x, K), dtype)
        out = torch.full((b.A, N), 7.0, dtype=dtype, device="cuda")
        y = B.moe_grouped_product_mx4(x, packed=packed, E=E, N=N, out=out, **b.kwargs())
        b.check(host(y), lambda e, of: mx.product(b.rows(host(x), of), Wq[e], U_SUM), dtype, 7.0)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("d,ffn", [(8, 1), (64, 64), (136, 65), (72, 200), (512, 100), (256, 1030)])
@pytest.mark.parametrize("gather", [False, True])
def test_ffn(dtype, relu, d, ffn, gather, form):
    rng = np.random.default_rng(d + ffn)
    E = 4
    W1, W3, W2 = (normal(rng, s, dtype, 0.1) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d)))
    if relu:
        W3 = None
    packed = B.moe_pack_weights_mx4(W1, W3, W2)
    Q = [None if w is None else mx.quantise(host(w)) for w in (W1, W3, W2)]
    for lengths, experts in RAGGED:
        b = Batch(rng, lengths, experts, E, gather)
        x = normal(rng, (b.rows_x, d), dtype)
        out = torch.full((b.A, d), 7.0, dtype=dtype, device="cuda")
        y = B.moe_grouped_ffn_mx4(x, packed=packed, E=E, ffn=ffn, relu=relu, out=out, **b.kwargs())
        b.check(host(y), lambda e, of: mx.ffn(b.rows(host(x), of), *(None if q is None else q[e] for q in Q), U_SUM, u_of(dtype)),
                dtype, 7.0)


def test_slot_ranges(form):
    """A rank's share: rows of the range's segments alone, with the bits that a call over all slots gives them."""
    rng = np.random.default_rng(5)
    E, d, ffn = 4, 128, 96
    W = [normal(rng, s, BF16, 0.1) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d))]
    packed = B.moe_pack_weights_mx4(*W)
    for lengths, experts in (([5, 40, 0, 70, 9], [0, 1, 2, 1, 0]), ([300, 200, 1, 90], [0, 1, 0, 1])):
        b = Batch(rng, lengths, experts, E, True)
        x = normal(rng, (b.rows_x, d), BF16)
        whole = B.moe_grouped_ffn_mx4(x, packed=packed, E=E, ffn=ffn, **b.kwargs())
        pieces = torch.full_like(whole, 7.0)
        for i in range(len(lengths)):
            alone = torch.full_like(whole, 7.0)
            B.moe_grouped_ffn_mx4(x, packed=packed, E=E, ffn=ffn, seg_begin=i, seg_end=i + 1, out=alone, **b.kwargs())
            lo, hi = b.so[i], b.so[i + 1]
            assert (alone[:lo] == 7).all() and (alone[hi:] == 7).all()
            pieces[lo:hi] = alone[lo:hi]
        # (an expert's rows may be cut into other M-tiles: the order of a sum depends on the form of the product, not on those)
        assert torch.equal(pieces, whole)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [3, 40, 300])
def test_infinities_and_nan_stay_where_they_are(dtype, rows, form):
    rng = np.random.default_rng(rows)
    E, K, N = 2, 136, 72
    W = normal(rng, (E, K, N), dtype, 0.1)
    W[1, 40, 5] = float("inf")
    packed = B.moe_pack_matrix_mx4(W)
    so = torch.tensor([0, rows, 2 * rows], dtype=torch.int32, device="cuda")
    se = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    x = normal(rng, (2 * rows, K), dtype)
    clean = B.moe_grouped_product_mx4(x, so, se, packed, E, N)
    nan = torch.isnan(clean)
    assert nan[rows:, 5].all() and nan.sum() == rows  # the weights' column of their expert
    bad = x.clone()
    bad[0, 3], bad[rows - 1, K - 1], bad[rows + 1, 0] = float("inf"), float("nan"), -float("inf")
    y = B.moe_grouped_product_mx4(bad, so, se, packed, E, N)
    keep = torch.ones(2 * rows, dtype=torch.bool, device="cuda")
    keep[[0, rows - 1, rows + 1]] = False
    same = (y == clean) | (torch.isnan(y) & nan)
    assert same[keep].all()
    Wq = torch.from_numpy(mx.quantise(host(W)))
    with np.errstate(invalid="ignore"):
        ref = host(bad)[[0, rows - 1]] @ Wq[0].numpy()
    got = host(y)[[0, rows - 1]]
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])


def test_hidden_rows_past_32_bits(form):
    """Hidden activations of more than 2^32 bytes: what their last rows make."""
    rng = np.random.default_rng(6)
    E, d, ffn, A = 2, 64, 65600, 33000
    assert A * ffn * 2 > 2 ** 32
    W = [normal(rng, s, BF16, 0.1) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d))]
    packed = B.moe_pack_weights_mx4(*W)
    x = normal(rng, (A, d), BF16)
    so = torch.tensor([0, 200, A], dtype=torch.int32, device="cuda")
    se = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    y = B.moe_grouped_ffn_mx4(x, so, se, packed, E, ffn)
    for e, rows in ((0, slice(0, 3)), (1, slice(A - 5, A))):
        Q = [mx.quantise(host(w[e])) for w in W]
        ref, tol = mx.ffn(host(x[rows]), *Q, U_SUM, u_of(BF16))
        assert (np.abs(host(y[rows]) - ref) <= tol + u_of(BF16) * (np.abs(ref) + tol)).all()


def test_rows_that_end_inside_a_k_tile(form):
    """What a workgroup has left of other experts' rows, all NaN, is not taken for the end of a row."""
    rng = np.random.default_rng(4)
    E, K, N, rows = 16, 72, 10240, 16
    W = normal(rng, (E, K, N), BF16, 0.1)
    packed = B.moe_pack_matrix_mx4(W)
    x = normal(rng, (E * rows, K), BF16)
    so = torch.arange(0, E * rows + 1, rows, dtype=torch.int32, device="cuda")
    se = torch.arange(E, dtype=torch.int32, device="cuda")
    clean = B.moe_grouped_product_mx4(x, so, se, packed, E, N)
    bad = x.clone().view(E, rows, K)
    bad[::2] = float("nan")
    y = B.moe_grouped_product_mx4(bad.view(-1, K), so, se, packed, E, N).view(E, rows, N)
    assert torch.isnan(y[::2]).all() and torch.equal(y[1::2], clean.view(E, rows, N)[1::2])


def test_fp32_rows_of_any_size():
    """Parts of an fp32 value: every exponent, and values with all 24 bits."""
    rng = np.random.default_rng(8)
    K, N, rows = 128, 32, 64
    W = normal(rng, (1, K, N), F32, 0.05)
    x = torch.from_numpy((rng.standard_normal((rows, K)) * np.exp2(rng.integers(-60, 60, (rows, 1)))).astype(np.float32)).cuda()
    x[1] = 3.0e38 / 128
    x[2] = 2.0 ** -126
    x[3, ::2] = 1 + 2.0 ** -23
    packed = B.moe_pack_matrix_mx4(W)
    so = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
    se = torch.tensor([0], dtype=torch.int32, device="cuda")
    y = host(B.moe_grouped_product_mx4(x, so, se, packed, 1, N))
    ref, tol = mx.product(host(x), mx.quantise(host(W))[0], U_SUM)
    assert (np.abs(y - ref) <= tol + 2.0 ** -24 * np.abs(ref) + 2.0 ** -126).all()


# ---------------------------------------------------------------------------
# streams, graphs, repeats
# ---------------------------------------------------------------------------
def small_ffn(dtype=BF16, lengths=(30, 0, 75, 11), d=256, ffn=192, seed=3):
    rng = np.random.default_rng(seed)
    E = 3
    W = [normal(rng, s, dtype, 0.1) for s in ((E, d, ffn), (E, d, ffn), (E, ffn, d))]
    b = Batch(rng, list(lengths), [0, 1, 2, 0], E, True)
    x = normal(rng, (b.rows_x, d), dtype)
    return W, b, x, dict(E=E, ffn=ffn)


@pytest.mark.parametrize("lengths", [(1, 0, 1, 0), (30, 0, 75, 11), (700, 0, 301, 5)])
def test_same_bits_every_time_and_on_another_stream(lengths, form):
    W, b, x, kw = small_ffn(lengths=lengths)
    packed = B.moe_pack_weights_mx4(*W)
    first = B.moe_grouped_ffn_mx4(x, packed=packed, **kw, **b.kwargs())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        packed2 = B.moe_pack_weights_mx4(*W)
        other = B.moe_grouped_ffn_mx4(x, packed=packed2, **kw, **b.kwargs())
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(packed, packed2) and torch.equal(first, other)
    for _ in range(3):
        assert torch.equal(B.moe_grouped_ffn_mx4(x, packed=packed, **kw, **b.kwargs()), first)


def test_two_graphs_that_share_a_workspace():
    W, b, x, kw = small_ffn()
    packed = B.moe_pack_weights_mx4(*W)
    args = b.kwargs()
    x2 = x.flip(0).contiguous()
    ws = torch.empty(B.moe_grouped_ffn_mx4_workspace_bytes(b.A, x.shape[1], kw["ffn"], len(b.se), 1), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros((b.A, x.shape[1]), dtype=BF16, device="cuda") for _ in range(2)]
    refs = [B.moe_grouped_ffn_mx4(v, packed=packed, **kw, **args) for v in (x, x2)]
    torch.cuda.synchronize()
    graphs = []
    for v, out in zip((x, x2), outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.moe_grouped_ffn_mx4(v, packed=packed, workspace=ws, out=out, **kw, **args)
        graphs.append(g)
    for _ in range(3):
        for g, out, ref in zip(graphs, outs, refs):
            out.zero_()
            ws.fill_(0xa5)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref)


# ---------------------------------------------------------------------------
# the layer
# ---------------------------------------------------------------------------
CFGS = [
    wl.CONFIGS["cfg1_tiny_f32"],
    wl.CONFIGS["mid_bf16"],
    wl.CONFIGS["mid_bf16"].replace(T=1, mode=wl.MODE_NONE),
    wl.CONFIGS["mid_bf16"].replace(T=7, act="relu", k=1),
    wl.CONFIGS["mid_bf16"].replace(T=3000, mode=wl.MODE_TOKEN, d=192, ffn=200),
    wl.CONFIGS["cfg5_decode_m1"].replace(T=33, d=256, ffn=128),
]


@pytest.mark.parametrize("i", range(len(CFGS)))
@pytest.mark.parametrize("fused_weights", [False, True])
def test_layer(i, fused_weights):
    """The whole step with weights in 4 bits: as one call and as single steps the same bits; as an fp64 layer of the held weights within
    the bounds; and captured."""
    cfg = CFGS[i]
    case = Case(cfg)
    dt = F32 if cfg.dtype == "f32" else BF16
    rng = np.random.default_rng(cfg.T)
    W1, W3, W2 = (normal(rng, s, dt, 0.05) for s in ((cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.ffn, cfg.d)))
    layer = MoELayer(cfg, fused_weights=fused_weights, weights="mx4")
    layer.set_weights(W1, W3, W2)
    logits, x = case.dev_logits(), case.dev_x()
    kw = dict(hist_pred=case.dev_hist_plan() if cfg.mode == wl.MODE_DISTRIBUTION else None, pred_idx=case.dev_pred_idx())
    out = layer.step(logits, x, **kw).clone()

    class Single(MoELayer):
        pass
    single = Single(cfg, fused_weights=fused_weights, weights="mx4")
    single.set_weights(W1, W3, W2)
    assert torch.equal(single.step(logits, x, **kw), out)
    assert torch.equal(single.y_perm, layer.y_perm)

    Q = [mx.quantise(host(w)) for w in (W1, W3, W2)]
    if cfg.act == "relu":
        Q[1] = None
    xs = host(x)
    ref, tol = np.zeros((cfg.T, cfg.d)), np.zeros((cfg.T, cfg.d))
    u = u_of(dt)
    for e in range(cfg.E):
        t, j = np.nonzero(case.idx == e)
        if len(t) == 0:
            continue
        y, dy = mx.ffn(xs[t], *(None if q is None else q[e] for q in Q), U_SUM, u)
        g = case.w[t, j].astype(np.float64)[:, None]
        # a row is rounded before the combine, with its gate weight (a few roundings of the softmax, 2^-20) or without
        np.add.at(ref, t, g * y)
        np.add.at(tol, t, g * (dy + u * (np.abs(y) + dy) + 2.0 ** -20 * np.abs(y)))
    tol = tol + u * (np.abs(ref) + tol)
    assert (np.abs(host(out) - ref) <= tol).all()

    graph = layer.capture(logits, x, **kw)
    for _ in range(3):
        layer.out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(layer.out, out)


def test_gradient_through_experts_in_4_bits():
    """Experts that stay as they are: the plain backward pass of their values, against differences of the 4-bit layer."""
    cfg = wl.CONFIGS["cfg1_tiny_f32"].replace(T=16)
    rng = np.random.default_rng(2)
    W = [normal(rng, s, F32, 0.2) for s in ((cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.d, cfg.ffn), (cfg.E, cfg.ffn, cfg.d))]
    case = Case(cfg)
    logits, x = case.dev_logits(), case.dev_x()
    four = MoELayer(cfg, weights="mx4")
    four.set_weights(*W)
    held = B.moe_unpack_weights_mx4(four.packed, cfg.E, cfg.d, cfg.ffn, F32)
    plain = MoELayer(cfg)
    train = MoETraining(plain, saved="plain")
    train.set_weights(*held)
    plain.step(logits, x, mode=wl.MODE_NONE)
    train.save(x)
    dout = normal(rng, (cfg.T, cfg.d), F32)
    dx = train.backward(dout)["dx"]
    v = normal(rng, (cfg.T, cfg.d), F32)
    v = v / v.norm()
    f = lambda s: float((four.step(logits, x + s * v, mode=wl.MODE_NONE).double() * dout.double()).sum())
    h = 2.0 ** -6
    slope = (f(h) - f(-h)) / (2 * h)
    want = float((dx.double() * v.double()).sum())
    # differences of fp32 results: (K + 8) 2^-23 of their sum of magnitudes, over 2 h; curvature h^2 / 6 of a third derivative
    size = float((four.step(logits, x, mode=wl.MODE_NONE).double().abs() * dout.double().abs()).sum())
    third = abs(f(2 * h) - 2 * f(h) + 2 * f(-h) - f(-2 * h)) / (2 * h ** 3)
    noise = (cfg.d + cfg.ffn + 16) * 2.0 ** -23 * size / h
    assert abs(slope - want) <= noise + h * h / 6 * (third + 4 * noise / (h * h)) * 2, (slope, want, noise)
    assert abs(want) > 10 * noise / (cfg.d + cfg.ffn)


def test_workspace_that_is_too_small():
    W, b, x, kw = small_ffn()
    packed = B.moe_pack_weights_mx4(*W)
    n = B.moe_grouped_ffn_mx4_workspace_bytes(b.A, x.shape[1], kw["ffn"], len(b.se), 1)
    with pytest.raises(B.MoeGpsError, match="workspace too small"):
        B.moe_grouped_ffn_mx4(x, packed=packed, workspace=torch.empty(n - 256, dtype=torch.uint8, device="cuda"), **kw, **b.kwargs())


def test_nothing_to_do():
    W, b, x, kw = small_ffn()
    packed = B.moe_pack_weights_mx4(*W)
    so, se = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    y = B.moe_grouped_ffn_mx4(x[:0], so, se, packed, kw["E"], kw["ffn"])
    assert y.shape == (0, x.shape[1])
    y = B.moe_grouped_ffn_mx4(x[:1], so, se, packed, kw["E"], kw["ffn"])  # a row that no segment has
    assert (y == 0).all()
