"""Weights in 4 bits: long sums, the buffers that their loops go round in, far offsets, narrow fp32 rows, rows of no expert.

Sums that are exact in fp32, in whatever order: rows of small whole numbers, weights that are codes times a few powers of two, so
that no partial sum has more than 24 bits.  A k-tile that is read twice, too late, from another row or with another group's scale makes another
number, and a result has to be the exact one, rounded once."""
import numpy as np
import pytest
import torch

import mx4_oracle as mx
from gpu_util import Case
from paper_2506_07366_amd import binding as B
from paper_2506_07366_amd import workloads as wl
from paper_2506_07366_amd.layer import MoELayer

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
U_SUM = 2.0 ** -23


@pytest.fixture(params=[-1, 0, 1, 2], ids=["auto", "tall", "split", "wide"])
def form(request):
    """The form of bf16 products: by the rule, tall tiles, K split between wavefronts, eight panels side by side."""
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, request.param)
    yield request.param
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, -1)


@pytest.fixture(params=[(-1, BF16), (0, BF16), (1, BF16), (2, BF16), (-1, F32)], ids=["auto", "tall", "split", "wide", "fp32"])
def dtype(request):
    """The forms, and fp32 rows, which have one of their own: the type of the rows."""
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, request.param[0])
    yield request.param[1]
    B.moe_grouped_ffn_set_option(B.FFN_OPT_STREAM, -1)


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def codes(gen, shape, dtype, scales=2):
    """Codes times 2^-1 .. 2^(scales - 2), a power of two for 32 neighbours of a column (multiples of 1 / 4, 6 * 2^(scales - 2) at most)."""
    E, K, N = shape
    table = torch.tensor(list(mx.CODES) + list(-mx.CODES), device="cuda")
    w = table[torch.randint(0, 16, shape, device="cuda", generator=gen)]
    s = torch.exp2(torch.randint(-1, scales - 1, (E, -(-K // 32), N), device="cuda", generator=gen).double())
    return (w * s.repeat_interleave(32, dim=1)[:, :K]).to(dtype)


def whole(gen, shape, dtype, most=2):
    return torch.randint(-most, most + 1, shape, device="cuda", generator=gen).to(dtype)


def segments(lengths, experts):
    so = torch.tensor([0, *lengths], device="cuda").cumsum(0).to(torch.int32)
    return so, torch.tensor(experts, dtype=torch.int32, device="cuda")


def rounded(y, dtype):
    """64-bit values that fp32 holds, rounded once."""
    assert torch.equal(y.float().double(), y)
    return y.float().to(dtype)


def rows_of(lengths, experts, E):
    return mx.rows_of_experts(np.concatenate([[0], np.cumsum(lengths)]), experts, E)


# steps of 256 along K in a share of it (an eighth): none or 1, 1, 2, 2 or 3, 3 or 4, 7
LONG = [520, 2048, 4096, 4680, 6152, 14336]
# rows of an M-tile: 8 and fewer, 9 to 16, two sixteens, two tiles (of one expert, whose weights then are read twice) and more
ROWS = [([5, 8, 9, 16, 17, 32], [0, 1, 2, 3, 4, 5]), ([1, 33, 70, 1], [0, 1, 2, 3]), ([300, 8, 7], [0, 1, 2]), ([1, 1, 1], [5, 3, 0])]


@pytest.mark.parametrize("K", LONG)
def test_products(K, dtype):
    E, N = 6, 72
    gen = generator(K)
    W = codes(gen, (E, K, N), dtype, scales=4)
    packed = B.moe_pack_matrix_mx4(W)
    assert torch.equal(B.moe_unpack_matrix_mx4(packed, E, K, N, dtype), W)
    for lengths, experts in ROWS:
        x = whole(gen, (sum(lengths), K), dtype)
        y = B.moe_grouped_product_mx4(x, *segments(lengths, experts), packed, E, N)
        for e, of in rows_of(lengths, experts, E).items():
            assert torch.equal(y[of], rounded(x[of].double() @ W[e].double(), dtype)), (lengths, e)


@pytest.mark.parametrize("K", LONG)
def test_first_products(K, dtype):
    """SwiGLU experts whose gate sums are all above 17, where 1 + exp(-a) is 1 in fp32 and silu(a) is a, and whose second matrix picks a
    hidden value for every column: the product of two exact sums, rounded to fp32 and to the rows' type, times a power of two."""
    E, ffn = 6, 72
    gen = generator(K)
    W1, W3 = codes(gen, (E, K, ffn), dtype).abs(), codes(gen, (E, K, ffn), dtype)
    pick = torch.randint(0, ffn, (E, K), device="cuda", generator=gen)
    W2 = torch.zeros((E, ffn, K), dtype=dtype, device="cuda")
    W2.scatter_(1, pick.unsqueeze(1), torch.exp2(torch.randint(-1, 2, (E, 1, K), device="cuda", generator=gen).float()).to(dtype))
    packed = B.moe_pack_weights_mx4(W1, W3, W2)
    for lengths, experts in ROWS:
        x = whole(gen, (sum(lengths), K), dtype).abs()
        y = B.moe_grouped_ffn_mx4(x, *segments(lengths, experts), packed, E, ffn)
        for e, of in rows_of(lengths, experts, E).items():
            a, b = (x[of].double() @ w[e].double() for w in (W1, W3))
            assert a.min() > 17
            h = (rounded(a, F32) * rounded(b, F32)).to(dtype)
            assert torch.equal(y[of], h[:, pick[e]] * W2[e].sum(0)), (lengths, e)


@pytest.mark.parametrize("ffn", LONG + [4097, 14300])
def test_second_products(ffn, dtype):
    """ReLU experts whose hidden activations are whole numbers up to 32, which bf16 holds."""
    E, d = 6, 16
    gen = generator(ffn)
    W1, W2 = whole(gen, (E, d, ffn), dtype), codes(gen, (E, ffn, d), dtype)
    packed = B.moe_pack_weights_mx4(W1, None, W2)
    for lengths, experts in ROWS:
        x = whole(gen, (sum(lengths), d), dtype, most=1)
        y = B.moe_grouped_ffn_mx4(x, *segments(lengths, experts), packed, E, ffn, relu=True)
        for e, of in rows_of(lengths, experts, E).items():
            h = (x[of].double() @ W1[e].double()).clamp(min=0)
            assert h.max() <= 32
            assert torch.equal(y[of], rounded(h @ W2[e].double(), dtype)), (lengths, e)


@pytest.mark.parametrize("lengths", [[1, 16, 17, 32, 33, 48, 64, 65, 96, 100], [127, 128, 129, 130, 160, 161, 192, 200, 224, 1],
                                     [225, 240, 241, 255, 256, 3, 2, 0, 250, 251], [256, 300, 512, 600, 1, 0, 40, 7, 9, 100]])
def test_weights_that_no_cache_keeps(lengths, form):
    """More than 128 MiB of them: tiles that are the only ones of their experts read them past the caches."""
    E, K, N = 40, 4096, 2048
    assert B.moe_packed_matrix_mx4_bytes(E, K, N) > 128 << 20
    gen = generator(7)
    W = codes(gen, (E, K, N), BF16)
    packed = B.moe_pack_matrix_mx4(W)
    experts = [0, 39, 7, 20, 33, 12, 1, 38, 25, 16]
    x = whole(gen, (sum(lengths), K), BF16)
    y = B.moe_grouped_product_mx4(x, *segments(lengths, experts), packed, E, N)
    for e, of in rows_of(lengths, experts, E).items():
        assert torch.equal(y[of], rounded(x[of].double() @ W[e].double(), BF16)), e


# ---------------------------------------------------------------------------
# far offsets
# ---------------------------------------------------------------------------
def test_packed_weights_past_32_bits(form):
    """Packed weights of more than 2^32 bytes: experts on both sides of the 2^31st and the 2^32nd, in either type of rows, and back."""
    E, K, N = 512, 4096, 4096
    assert B.moe_packed_matrix_mx4_bytes(E, K, N) > 2 ** 32
    of_bytes = lambda n: n * E // B.moe_packed_matrix_mx4_bytes(E, K, N)
    some = [0, of_bytes(2 ** 31), of_bytes(2 ** 31) + 1, of_bytes(2 ** 32), of_bytes(2 ** 32) + 1, E - 1]
    gen = generator(1)
    W = torch.zeros((E, K, N), dtype=BF16, device="cuda")
    for e in some:
        W[e] = codes(gen, (1, K, N), BF16)[0]
    packed = B.moe_pack_matrix_mx4(W)
    lengths = [3] * len(some)
    for dtype in (BF16, F32) if form == -1 else (BF16,):
        x = whole(gen, (sum(lengths), K), dtype)
        y = B.moe_grouped_product_mx4(x, *segments(lengths, some), packed, E, N)
        for e, of in rows_of(lengths, some, E).items():
            assert torch.equal(y[of], rounded(x[of].double() @ W[e].double(), dtype)), (dtype, e)
    if form == -1:
        assert torch.equal(B.moe_unpack_matrix_mx4(packed, E, K, N, BF16), W)


@pytest.mark.parametrize("gather", [False, True])
def test_as_many_values_of_x_as_there_may_be(gather, dtype):
    """2^31 - 4096 values of x (bf16: 2^32 bytes less 8192): its first and last rows, in place and through the permutation."""
    E, K, N = 2, 4096, 40
    rows = (2 ** 31 - 64) // K
    gen = generator(3)
    W = codes(gen, (E, K, N), dtype)
    packed = B.moe_pack_matrix_mx4(W)
    x = torch.zeros((rows, K), dtype=dtype, device="cuda")
    x[:50], x[-300:] = whole(gen, (50, K), dtype), whole(gen, (300, K), dtype)
    kw = {}
    of = torch.arange(rows, device="cuda")
    if gather:  # (back to front)
        of = of.flip(0)
        kw = dict(assign_of_row=of.to(torch.int32), k=1)
    so, se = segments([200, rows - 250, 50], [0, 1, 0])
    y = B.moe_grouped_product_mx4(x, so, se, packed, E, N, **kw)
    expert = torch.ones(rows, dtype=torch.long, device="cuda")
    expert[:200] = expert[-50:] = 0
    loud = torch.cat([torch.arange(50, device="cuda"), torch.arange(rows - 300, rows, device="cuda")])
    at = torch.argsort(of)[loud]  # places of those rows
    for e in range(E):
        mine = expert[at] == e
        assert mine.any()
        assert torch.equal(y[at[mine]], rounded(x[loud[mine]].double() @ W[e].double(), dtype))


def test_second_matrices_past_32_bits(form):
    """An FFN whose second matrices lie behind the 2^32nd byte."""
    E, d, ffn = 640, 2048, 4096
    assert E * B.moe_packed_matrix_mx4_bytes(1, d, ffn) > 2 ** 31 and B.moe_packed_weights_mx4_bytes(E, d, ffn, True) > 2 ** 32
    gen = generator(2)
    some = [0, 300, 511, 512, E - 1]
    W1, W2 = (torch.zeros(s, dtype=BF16, device="cuda") for s in ((E, d, ffn), (E, ffn, d)))
    for e in some:
        W1[e, :16] = whole(gen, (16, ffn), BF16)
        W2[e] = codes(gen, (1, ffn, d), BF16)[0]
    packed = B.moe_pack_weights_mx4(W1, None, W2)
    lengths = [2, 5, 9, 1, 20]
    x = whole(gen, (sum(lengths), d), BF16, most=1)
    y = B.moe_grouped_ffn_mx4(x, *segments(lengths, some), packed, E, ffn, relu=True)
    for e, of in rows_of(lengths, some, E).items():
        h = (x[of].double() @ W1[e].double()).clamp(min=0)
        assert torch.equal(y[of], rounded(h @ W2[e].double(), BF16)), e


def test_fp32_hidden_rows_past_32_bits():
    """Hidden activations of more than 2^31 fp32 values: what the rows around the 2^31st value and the last ones make."""
    E, d, ffn, A = 2, 16, 65600, 33000
    assert A * ffn > 2 ** 31
    gen = generator(6)
    W1, W2 = whole(gen, (E, d, ffn), F32), codes(gen, (E, ffn, d), F32)
    packed = B.moe_pack_weights_mx4(W1, None, W2)
    x = whole(gen, (A, d), F32, most=1)
    y = B.moe_grouped_ffn_mx4(x, *segments([200, A - 200], [0, 1]), packed, E, ffn, relu=True)
    edge = 2 ** 31 // 65600
    for e, rows in ((0, slice(0, 200)), (1, slice(edge - 40, edge + 40)), (1, slice(A - 70, A))):
        h = (x[rows].double() @ W1[e].double()).clamp(min=0)
        # (sums of 65600 values of up to 32 times 6: multiples of a quarter below 2^24 of them as they come out here)
        ref = h @ W2[e].double()
        size = h @ W2[e].double().abs()
        assert ref.abs().max() > 0
        assert ((y[rows].double() - ref).abs() <= (ffn + 8) * U_SUM * size).all()


# ---------------------------------------------------------------------------
# narrow fp32 rows, rows of no expert
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("K,N", [(4, 4), (12, 20), (36, 44), (100, 12), (260, 68)])
def test_fp32_rows_of_a_multiple_of_four(K, N):
    E = 3
    gen = generator(K)
    W = codes(gen, (E, K, N), F32)
    packed = B.moe_pack_matrix_mx4(W)
    W1, W2 = whole(gen, (E, K, 20), F32), codes(gen, (E, 20, K), F32)
    packed_ffn = B.moe_pack_weights_mx4(W1, None, W2)
    for lengths, experts in (([1], [2]), ([7, 16, 40], [0, 2, 1]), ([65, 3, 130], [1, 0, 1])):
        x = whole(gen, (sum(lengths), K), F32)
        so_se = segments(lengths, experts)
        out = torch.full((x.shape[0] + 1, N), 7.0, device="cuda")  # (what lies behind the last row stays)
        y = B.moe_grouped_product_mx4(x, *so_se, packed, E, N, out=out[:-1])
        z = B.moe_grouped_ffn_mx4(x, *so_se, packed_ffn, E, 20, relu=True)
        assert (out[-1] == 7).all()
        for e, of in rows_of(lengths, experts, E).items():
            assert torch.equal(y[of], rounded(x[of].double() @ W[e].double(), F32))
            assert torch.equal(z[of], rounded((x[of].double() @ W1[e].double()).clamp(min=0) @ W2[e].double(), F32))


@pytest.mark.parametrize("T,E,k,G,S", [(1, 8, 2, 4, 3), (40, 16, 4, 4, 5), (3000, 16, 8, 4, 5)])
@pytest.mark.parametrize("mode", [wl.MODE_NONE, wl.MODE_DISTRIBUTION])
def test_tokens_of_no_expert(T, E, k, G, S, mode):
    """Tokens whose logits are NaN: in one call and in single steps the same bits, and the others get what they get without them."""
    cfg = wl.MoEConfig("nan", T=T, d=64, ffn=72, E=E, k=k, G=G, S=S, dtype="bf16", mode=mode, seed=65)
    gen = generator(66)
    W = [torch.randn(s, device="cuda", generator=gen).mul_(0.1).to(BF16) for s in ((E, 64, 72), (E, 64, 72), (E, 72, 64))]
    logits = torch.randn((T, E), device="cuda", generator=gen)
    x = torch.randn((T, 64), device="cuda", generator=gen).to(BF16)
    hist = torch.randint(1, 9, (E,), device="cuda", generator=gen, dtype=torch.int32)
    kw = dict(hist_pred=hist if mode == wl.MODE_DISTRIBUTION else None)

    class Single(MoELayer):
        pass
    for fused in (False, True):
        layers = [cls(cfg, fused_weights=fused, weights="mx4") for cls in (MoELayer, Single)]
        for layer in layers:
            layer.set_weights(*W)
        clean = layers[0].step(logits, x, **kw).clone()
        bad = logits.clone()
        lost = sorted({0, T // 2, T - 1})
        bad[lost] = float("nan")
        one, single = (layer.step(bad, x, **kw).clone() for layer in layers)
        keep = [t for t in range(T) if t not in lost]
        assert torch.equal(one[keep], clean[keep]) and torch.equal(single[keep], clean[keep])
