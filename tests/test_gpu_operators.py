"""Routing from logits (and its gradient), 8-bit products and 8-bit experts against plain evaluations in 64 bits.

Tolerances come from the roundings that the operators make: 2^-24 for an fp32 operation, half a unit in the last place of the
output type for the final rounding, and for the experts the possible move of single codes of the gated activation, whose
32-bit sums may fall on the other side of a tie than the 64-bit ones.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}    # relative rounding, generous by <= 2


@pytest.fixture(scope="module")
def mok():
    from paper_2609_36070_b200 import mok
    yield mok
    assert mok.mok_i8_status() == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


# ------------------------------------------------------------------------------------------------------------- gate

def scores64(logits, score):
    z = logits.double()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    return torch.nan_to_num(s, nan=0.0)          # softmax of a row that is masked completely


def choices64(logits, bias, score, G, top_groups, group_top):
    """Choice values of the experts, -inf outside the chosen groups, and the smallest gap that the groups were decided by."""
    s = scores64(logits, score)
    c = s if bias is None else s + bias.double()
    T, E = c.shape
    gap = torch.full((T,), math.inf, dtype=torch.float64, device=c.device)
    if G > 1:
        v = c.view(T, G, E // G).topk(group_top, -1).values.sum(-1)
        o = v.sort(dim=-1, descending=True, stable=True)
        if top_groups < G:
            gap = o.values[:, top_groups - 1] - o.values[:, top_groups]
        keep = torch.zeros(T, G, dtype=torch.bool, device=c.device).scatter_(1, o.indices[:, :top_groups], True)
        c = c.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    return s, c, gap


def weights64(s, idx, renorm, scale):
    w = s.gather(1, idx.long())
    if renorm:
        t = w.sum(-1, keepdim=True)
        w = torch.where(t > 0, w / t, torch.zeros_like(w))
    return w * scale


GATES = [  # T, E, k, score, groups, topk_groups, group_top, bias, renorm, scale, dtype
    (1, 1, 1, "sigmoid", 1, 1, 1, False, True, 1.0, torch.float32),
    (1, 8, 8, "softmax", 1, 1, 1, False, True, 1.0, torch.float32),
    (5, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, torch.float32),
    (1000, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, torch.bfloat16),
    (333, 60, 4, "softmax", 1, 1, 1, False, False, 1.0, torch.float32),
    (333, 60, 6, "softmax", 4, 2, 1, False, True, 1.0, torch.float16),
    (200, 33, 7, "softmax", 3, 2, 2, True, False, 2.0, torch.float32),
    (200, 510, 32, "sigmoid", 15, 7, 2, True, True, 1.0, torch.float32),
    (64, 512, 32, "sigmoid", 32, 32, 2, False, False, 1.0, torch.float32),
    (64, 512, 16, "softmax", 32, 1, 1, True, True, 1.0, torch.bfloat16),
    (40000, 32, 2, "softmax", 1, 1, 1, False, True, 1.0, torch.bfloat16),
    (17, 31, 31, "sigmoid", 1, 1, 1, True, True, 1.0, torch.float32),
    (1001, 512, 10, "sigmoid", 16, 5, 2, True, True, 1.0, torch.float32),
    # enough tokens for four of them in a warp: with and without lists, groups of several sizes, rows that are not aligned
    (3001, 256, 8, "sigmoid", 8, 4, 2, True, True, 2.5, torch.float32),
    (2500, 160, 6, "softmax", 8, 3, 1, False, False, 16.0, torch.bfloat16),
    (2401, 510, 17, "sigmoid", 1, 1, 1, True, True, 1.0, torch.float16),
    (2402, 512, 16, "sigmoid", 32, 12, 2, True, True, 1.0, torch.float32),
    (2403, 60, 5, "softmax", 5, 2, 2, True, True, 1.0, torch.float32),
    (2404, 64, 8, "sigmoid", 16, 4, 2, False, True, 1.0, torch.float32),
    (5000, 37, 9, "softmax", 1, 1, 1, True, False, 1.0, torch.bfloat16),
    (2405, 24, 3, "sigmoid", 2, 1, 2, True, True, 1.0, torch.float32),
    (2406, 8, 8, "softmax", 1, 1, 1, False, True, 1.0, torch.float32),
    (515, 384, 8, "softmax", 4, 3, 2, True, True, 1.0, torch.float16),
    (515, 320, 6, "sigmoid", 5, 1, 1, False, True, 1.0, torch.bfloat16),
    (130, 128, 32, "softmax", 4, 4, 1, False, False, 1.0, torch.float32),
]


@pytest.mark.parametrize("T,E,k,score,G,tg,gt,with_bias,renorm,scale,dtype", GATES)
def test_gate(mok, T, E, k, score, G, tg, gt, with_bias, renorm, scale, dtype):
    g = gen(T + E)
    wide = randn(g, T, E + 3).mul(1.5).to(dtype)
    logits = wide[:, 2:2 + E]                                          # rows of a wider buffer, not 16-byte aligned
    bias = randn(g, E) * 0.05 if with_bias else None
    idx, w = mok.mok_gate(logits, k, bias=bias, score=score, n_groups=G, topk_groups=tg, group_top=gt, renormalise=renorm,
                          scale=scale)
    assert idx.dtype == torch.int32 and w.dtype == torch.float32 and idx.shape == w.shape == (T, k)
    s, c, gap = choices64(logits, bias, score, G, tg, gt)
    assert ((idx >= 0) & (idx < E)).all()
    assert (idx.sort(-1).values.diff(dim=-1) > 0).all()                # distinct
    # fp32 scores decide the groups of the other tokens; where logits are compared, equal ones included, all is decided
    clear = gap > 1e-6 if bias is not None or (G > 1 and gt == 2) else torch.ones_like(gap, dtype=torch.bool)
    assert clear.float().mean() > 0.97
    mine, best = c.gather(1, idx.long())[clear], c.sort(dim=-1, descending=True).values[:, :k][clear]
    assert (mine - best).abs().max() <= 1e-6                           # scores are below 1, each good to a few 2^-24
    ref = weights64(s, idx, renorm, scale)
    assert ((w.double() - ref).abs() <= 16 * UNIT[torch.float32] * ref.abs() * 8 + 1e-30).all()


@pytest.mark.parametrize("T", [257, 2600])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_gate_ties_go_to_the_lowest_id(mok, dtype, T):
    g = gen(3)
    logits = torch.randint(-3, 4, (T, 96), generator=g, device="cuda").to(dtype)        # seven values: ties everywhere
    logits[0] = 0.0
    logits[1, ::2] = -0.0                                               # equal to +0
    logits[1, 1::2] = 0.0
    for score in ("softmax", "sigmoid"):
        idx, _ = mok.mok_gate(logits, 8, score=score)
        ref = logits.float().add(0.0).sort(dim=-1, descending=True, stable=True).indices[:, :8]
        assert torch.equal(idx.long(), ref)
        # equal groups as well: every group has the same two best
        tied = torch.zeros(T, 96, device="cuda", dtype=dtype)
        for k, G in ((4, 6), (8, 3), (7, 32)):
            idx, _ = mok.mok_gate(tied, k, score=score, n_groups=G, topk_groups=3, group_top=2)
            assert torch.equal(idx, torch.arange(k, device="cuda", dtype=torch.int32).expand(T, k))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("T,k", [(8, 4), (2408, 4), (2408, 6)])
def test_gate_masked_and_broken_rows(mok, score, renorm, with_bias, T, k):
    E = 40
    logits = randn(gen(1), T, E)
    bias = torch.zeros(E, device="cuda") if with_bias else None
    logits[0] = -math.inf                                               # nothing left
    logits[1, 3:] = -math.inf                                           # fewer experts than k
    logits[2, ::2] = torch.finfo(torch.float32).min                     # a mask of the lowest value
    logits[3, 5] = math.nan
    logits[4] = math.nan
    logits[5, 7] = math.inf
    logits[6] = torch.finfo(torch.float32).min
    clean = mok.mok_gate(torch.cat([logits[7:], logits[7:14]])[:T], k, bias=bias, score=score, renormalise=renorm)
    idx, w = mok.mok_gate(logits, k, bias=bias, score=score, renormalise=renorm)
    assert ((idx >= 0) & (idx < E)).all() and (idx.sort(-1).values.diff(dim=-1) > 0).all()
    assert torch.equal(idx[0], torch.arange(k, device="cuda", dtype=torch.int32)) and (w[0] == 0).all()
    assert idx[1, :3].sort().values.tolist() == [0, 1, 2] and (w[1, 3:] == 0).all() and torch.isfinite(w[1]).all()
    assert (idx[2] % 2 == 1).all() and torch.isfinite(w[2]).all()
    assert torch.equal(idx[7:], clean[0][:T - 7]) and torch.equal(w[7:], clean[1][:T - 7])      # other rows are not touched
    if score == "softmax" and renorm:
        assert (w[6] - 1 / k).abs().max() < 1e-6                        # a uniform row, however low
    if score == "sigmoid":
        assert idx[5, 0] == 7 and 5 not in idx[3].tolist()


GRADS = [(1, 8, 2, torch.float32), (257, 60, 4, torch.float32), (300, 256, 8, torch.float32), (300, 256, 8, torch.bfloat16),
         (65, 511, 32, torch.float16), (9, 3, 3, torch.float32)]


@pytest.mark.parametrize("T,E,k,dtype", GRADS)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gate_backward(mok, T, E, k, dtype, score, renorm):
    g = gen(E + k)
    logits = randn(g, T, E + 5).to(dtype)[:, 1:1 + E]
    idx, _ = mok.mok_gate(logits, k, score=score, renormalise=renorm)
    dw = randn(g, T, k)
    d = mok.mok_gate_backward(logits, idx, dw, score=score, renormalise=renorm, scale=1.7)
    z = logits.double().requires_grad_()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    w = s.gather(1, idx.long())
    ref, = torch.autograd.grad((w / w.sum(-1, keepdim=True) if renorm else w) * 1.7, z, dw.double())
    assert d.dtype == dtype and d.shape == (T, E)
    # sums of up to 32 products and the difference g - mean: 64 roundings of the token's largest |g|
    room = 64 * UNIT[torch.float32] * 1.7 * dw.abs().max(-1, keepdim=True).values.double()
    assert ((d.double() - ref).abs() <= UNIT[dtype] * ref.abs() + room).all()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gate_gradient_against_differences(mok, score, renorm):
    """(L(l + h v) - L(l - h v)) / 2h of the operator's own forward, L = sum dw * w, along a direction v that leaves the
    selection as it is; h = 1/64: the third derivatives of these weights are below 1, so the difference is good to h^2 / 6
    of |dw| |v|, and rounding adds 2^-23 / h of it."""
    g = gen(11)
    T, E, k, h = 50, 24, 4, 1.0 / 64
    logits = randn(g, T, E)
    logits.scatter_add_(1, logits.topk(k, -1).indices, torch.full((T, k), 2.0, device="cuda"))   # clear of the others
    order = logits.topk(k, -1)
    logits.scatter_(1, order.indices, order.values + torch.arange(k, 0, -1, device="cuda") * 0.5)
    v, dw = torch.rand(T, E, generator=g, device="cuda") * 2 - 1, randn(g, T, k)
    f = [mok.mok_gate(logits + sign * h * v, k, score=score, renormalise=renorm) for sign in (1, -1)]
    idx, _ = mok.mok_gate(logits, k, score=score, renormalise=renorm)
    assert torch.equal(f[0][0], idx) and torch.equal(f[1][0], idx)
    diff = ((f[0][1] - f[1][1]).double() * dw).sum(-1) / (2 * h)
    d = mok.mok_gate_backward(logits, idx, dw, score=score, renormalise=renorm)
    along = (d.double() * v).sum(-1)
    assert ((along - diff).abs() <= (h * h / 6 * 2 + 2.0 ** -23 / h) * dw.abs().sum(-1) * 2).all()


@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("G,k", [(1, 4), (2, 4), (4, 4), (4, 6)])
def test_gate_masked_experts_whatever_their_bias(mok, T, G, k):
    """An expert whose logit is -inf is not chosen for a token that has k others, however large its bias."""
    E = 64
    logits = randn(gen(21), T, E)
    masked = torch.rand(T, E, generator=gen(22), device="cuda") < 0.5
    logits[masked] = -math.inf
    bias = torch.where(masked.float().mean(0) > 0.5, 10.0, 0.0)
    for score in ("softmax", "sigmoid"):
        idx, w = mok.mok_gate(logits, k, bias=bias, score=score, n_groups=G, topk_groups=G, group_top=2)
        assert not masked.gather(1, idx.long()).any() and torch.isfinite(w).all()


def test_gate_backward_ignores_dropped_ids(mok):
    logits, dw = randn(gen(2), 6, 16), randn(gen(3), 6, 3)
    idx, _ = mok.mok_gate(logits, 3, score="sigmoid")
    full = mok.mok_gate_backward(logits, idx, dw, score="sigmoid", renormalise=False)
    idx[:, 1] = torch.tensor([-1, 16, 1 << 30, -(1 << 30), 16, -1], device="cuda", dtype=torch.int32)
    part = mok.mok_gate_backward(logits, idx, dw, score="sigmoid", renormalise=False)
    assert (part != full).sum() == 6 and (part[part != full] == 0).all()
    idx[:] = -1
    for renorm in (True, False):
        for score in ("sigmoid", "softmax"):
            assert (mok.mok_gate_backward(logits, idx, dw, score=score, renormalise=renorm) == 0).all()


# --------------------------------------------------------------------------------------------------------- 8-bit rows

def codes64(x):
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    return torch.where(amax > 0, (x * 127 / amax).round(), torch.zeros_like(x)), (amax / 127).squeeze(-1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("rows,K,pitch,skip", [(1, 1, 0, 0), (3, 7, 0, 0), (5, 16, 8, 0), (9, 130, 3, 1), (2, 2048, 0, 0),
                                               (1200, 256, 8, 8), (1201, 2048, 0, 0), (4, 16384, 0, 0), (3, 20000, 0, 0),
                                               (1, 7168, 0, 0), (1500, 72, 0, 0)])
def test_quantize(mok, dtype, rows, K, pitch, skip):
    g = gen(K)
    x = (randn(g, rows, K + pitch + skip) * torch.rand(rows, 1, generator=g, device="cuda")).to(dtype)[:, skip:skip + K]
    codes, scales = mok.mok_i8_quantize(x)
    assert codes.shape == (rows, (K + 15) // 16 * 16) and (codes[:, K:] == 0).all()
    ref, s = codes64(x)
    if dtype == torch.float32:                          # the rule is fp32 arithmetic: the same operations one by one
        amax = x.abs().amax(-1, keepdim=True)
        ref = torch.where(amax > 0, (x * 127.0 / amax).round(), torch.zeros_like(x))
    assert torch.equal(codes[:, :K].double(), ref.double())
    assert ((scales.double() - s).abs() <= UNIT[torch.float32] * s).all()


def test_quantize_special_rows(mok):
    for dtype in (torch.bfloat16, torch.float32):
        big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).tiny
        for K in (24, 9):                               # both kernels
            x = randn(gen(5), 7, K).to(dtype)
            clean = mok.mok_i8_quantize(x[6:])
            x[0] = 0.0
            x[1, 3] = math.nan
            x[2, 4] = -math.inf
            x[3] = big * torch.linspace(-1, 1, K, device="cuda").to(dtype)
            x[4] = tiny
            x[5, :] = -0.0
            codes, scales = mok.mok_i8_quantize(x)
            assert (codes[0] == 0).all() and scales[0] == 0 and (codes[5] == 0).all() and scales[5] == 0
            assert (codes[1] == 0).all() and math.isnan(scales[1]) and (codes[2] == 0).all() and scales[2] == math.inf
            ref, s = codes64(x[3:4])
            assert (codes[3, :K].double() - ref).abs().max() <= (1 if dtype == torch.float32 else 0) and codes[3].abs().max() == 127
            assert (codes[4, :K] == 127).all()
            assert torch.equal(codes[6:], clean[0]) and torch.equal(scales[6:], clean[1])


def test_codes_of_ties_are_even(mok):
    x = torch.zeros(1, 16, device="cuda")
    x[0, 0] = 127.0
    x[0, 1:9] = torch.tensor([0.5, 1.5, 2.5, -0.5, -1.5, 126.5, -125.5, 3.5], device="cuda")
    codes, _ = mok.mok_i8_quantize(x.bfloat16())
    assert codes[0, 1:9].tolist() == [0, 2, 2, 0, -2, 126, -126, 4]


# ------------------------------------------------------------------------------------------------------- 8-bit product

def weights(mok, g, *shape):
    codes = torch.randint(-127, 128, (*shape[:-1], (shape[-1] + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
    return mok.I8Weights(codes, (torch.rand(*shape[:-1], generator=g, device="cuda") + 0.5) * 1e-3)     # (bytes past K: garbage)


def product64(codes, scales, w, bias, K):
    y = codes[:, :K].double() @ w.codes[:, :K].double().t()
    assert y.abs().max() < 2 ** 31
    return y * scales.double()[:, None] * w.scales.double() + (0 if bias is None else bias.double())


def check_product(out, ref, bias, dtype):
    room = 4 * UNIT[torch.float32] * (ref.abs() + (0 if bias is None else bias.double().abs()))
    assert ((out.double() - ref).abs() <= UNIT[dtype] * ref.abs() + room + 1e-30).all()


PRODUCTS = [(1, 1, 1), (1, 16, 8), (2, 15, 7), (1, 7168, 300), (3, 128, 33), (7, 130, 257), (16, 256, 256), (17, 1000, 100),
            (31, 2048, 512), (33, 512, 1030), (64, 640, 384), (65, 300, 200), (127, 4096, 129), (129, 96, 65), (255, 1024, 255),
            (257, 777, 513), (1000, 144, 72), (700, 2880, 720)]


@pytest.mark.parametrize("M,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype,out_dtype,with_bias", [(torch.bfloat16, torch.bfloat16, False), (torch.float16, torch.float32, True),
                                                       (torch.float32, torch.float16, True)])
def test_linear(mok, M, K, N, dtype, out_dtype, with_bias):
    g = gen(M * K + N)
    x = randn(g, M, K + 4).to(dtype)[:, 2:2 + K]
    w = weights(mok, g, N, K)
    bias = randn(g, N) if with_bias else None
    out = mok.mok_i8_linear(x, w, bias=bias, out_dtype=out_dtype)
    codes, scales = mok.mok_i8_quantize(x)
    assert out.dtype == out_dtype and out.shape == (M, N)
    check_product(out, product64(codes, scales, w, bias, K), bias, out_dtype)
    again = mok.mok_i8_matmul(codes, scales, w, K=K, bias=bias, out_dtype=out_dtype)
    assert torch.equal(out, again)
    assert mok.mok_i8_status() == 0


def test_linear_rows_do_not_depend_on_the_batch(mok):
    """Integer sums are exact, so a token's row has the same bits in a batch of any size, whatever kernel serves it."""
    g = gen(8)
    K, N = 1040, 520
    x, w = randn(g, 600, K).bfloat16(), weights(mok, g, N, K)
    whole = mok.mok_i8_linear(x, w, out_dtype=torch.float32)
    for M in (1, 5, 16, 40, 100, 128, 200, 256, 400):
        assert torch.equal(mok.mok_i8_linear(x[:M], w, out_dtype=torch.float32), whole[:M]), M


@pytest.mark.parametrize("M,K,N", [(1, 16384, 128), (1, 300, 2000), (2, 640, 1), (5, 384, 300), (9, 900, 2300), (16, 14336, 130), (24, 5000, 640),
                                   (40, 1100, 4100), (48, 2048, 1024), (63, 900, 300), (64, 7168, 256), (64, 24000, 64),
                                   (64, 128, 128), (33, 127, 20000),
                                   (65, 4096, 4096), (100, 2000, 1000), (128, 7168, 2048), (129, 1024, 500), (200, 4096, 4100),
                                   (256, 2048, 7168), (256, 130, 300), (255, 14336, 512)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear_few_tokens(mok, M, K, N, dtype):
    """The shapes by which a product of few tokens is split over K, quantised in the kernel or before it."""
    g = gen(M + K + N)
    x, w = randn(g, M, K).to(dtype), weights(mok, g, N, K)
    out = mok.mok_i8_linear(x, w, out_dtype=torch.float32)
    codes, scales = mok.mok_i8_quantize(x)
    check_product(out, product64(codes, scales, w, None, K), None, torch.float32)
    assert torch.equal(out, mok.mok_i8_matmul(codes, scales, w, K=K, out_dtype=torch.float32))


def test_linear_largest_sums_and_poisoned_rows(mok):
    K = 131072
    codes = torch.full((3, K), 127, device="cuda", dtype=torch.int8)
    codes[1] = -127
    w = mok.I8Weights(torch.full((20, K), 127, device="cuda", dtype=torch.int8), torch.ones(20, device="cuda"))
    out = mok.mok_i8_matmul(codes, torch.ones(3, device="cuda"), w, out_dtype=torch.float32)
    total = 127 * 127 * K
    assert (out[0].double() - total).abs().max() <= total * UNIT[torch.float32]
    assert torch.equal(out[1], -out[0])
    x = randn(gen(1), 40, 512)
    w = weights(mok, gen(2), 64, 512)
    clean = mok.mok_i8_linear(x, w)
    x[7, 100], x[9, 3], x[11] = math.nan, math.inf, 0.0
    out = mok.mok_i8_linear(x, w)
    assert torch.isnan(out[7]).all() and torch.isnan(out[9]).all() and (out[11] == 0).all()
    rest = [r for r in range(40) if r not in (7, 9, 11)]
    assert torch.equal(out[rest], clean[rest])


# ------------------------------------------------------------------------------------------------------- 8-bit experts

def experts64(x, idx, w, gu, dn, add=None):
    """The layer in 64 bits and how far the operator may be from it."""
    T, H = x.shape
    E, I = gu.codes.shape[0], gu.codes.shape[1] // 2
    out = torch.zeros(T, H, dtype=torch.float64, device=x.device) if add is None else add.double().clone()
    room = torch.zeros_like(out)
    q, s = codes64(x)
    for e in range(E):
        t, slot = torch.nonzero(idx == e, as_tuple=True)
        if not len(t):
            continue
        z = (q[t] @ gu.codes[e, :, :H].double().t()) * s[t, None] * gu.scales[e].double()
        hq, hs = codes64(torch.nn.functional.silu(z[:, :I]) * z[:, I:])
        y = (hq @ dn.codes[e, :, :I].double().t()) * hs[:, None] * dn.scales[e].double()
        f = w[t, slot].double()[:, None]
        out.index_add_(0, t, f * y)
        # fp16 of a row's sums, and three codes of the gated activation on the other side of a tie
        room.index_add_(0, t, f.abs() * (2.0 ** -11 * y.abs() + 3 * 127 * hs[:, None] * dn.scales[e].double()))
    return out, room


def routes(g, T, E, k):
    top = randn(g, T, E).topk(k, -1)
    return top.indices.int().contiguous(), top.values.softmax(-1)


EXPERTS = [(1, 8, 8, 1, 1), (1, 256, 128, 8, 2), (3, 64, 264, 4, 4), (16, 256, 136, 64, 8), (50, 520, 200, 7, 3), (200, 128, 1032, 4, 2),
           (300, 264, 384, 3, 2), (1000, 256, 256, 2, 1), (2500, 136, 72, 16, 4), (700, 72, 8200, 2, 2),
           (4200, 72, 64, 300, 8), (6000, 64, 40, 8, 4), (130, 2048, 768, 128, 8), (129, 384, 512, 1, 1), (112, 384, 72, 1, 1)]


@pytest.mark.parametrize("T,H,I,E,k", EXPERTS)
@pytest.mark.parametrize("dtype,with_add", [(torch.bfloat16, False), (torch.float16, True)])
def test_experts(mok, T, H, I, E, k, dtype, with_add):
    g = gen(T + H + I)
    x = randn(g, T, H + 8).to(dtype)[:, 4:4 + H]
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    idx, w = routes(g, T, E, k)
    add = randn(g, T, H).to(dtype) if with_add else None
    out = mok.mok_i8_experts(x, idx, w, gu, dn, add=add)
    ref, room = experts64(x, idx, w, gu, dn, add)
    assert out.dtype == dtype and out.shape == (T, H)
    assert ((out.double() - ref).abs() <= UNIT[dtype] * ref.abs() + room).all()
    # in norm: the final rounding and the rows' fp16, uniform in the last place
    assert (out.double() - ref).norm() <= (UNIT[dtype] + 2.0 ** -11) * ref.norm()
    assert mok.mok_i8_status() == 0
    assert torch.equal(out, mok.mok_i8_experts(x, idx, w, gu, dn, add=add))


def test_experts_dropped_routes_and_lonely_experts(mok):
    g = gen(4)
    T, H, I, E, k = 90, 128, 136, 6, 3
    x = randn(g, T, H).bfloat16()
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    idx, w = routes(g, T, E, k)
    idx[:, 1] = -1
    idx[5:9] = torch.tensor([E, -7, 1 << 30], device="cuda", dtype=torch.int32)          # tokens without any route
    w[:, 1] = math.nan                                                                   # (the weight of a dropped slot is not read)
    out = mok.mok_i8_experts(x, idx, w, gu, dn)
    ref, room = experts64(x, idx, w, gu, dn)
    assert (out[5:9] == 0).all() and ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()
    idx[:] = 4                                                                           # everything on one expert, ids repeated
    w = torch.rand(T, k, generator=g, device="cuda")
    out = mok.mok_i8_experts(x, idx, w, gu, dn)
    ref, room = experts64(x, idx, w, gu, dn)
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()
    idx[:] = -1
    add = randn(g, T, H).bfloat16()
    assert torch.equal(mok.mok_i8_experts(x, idx, w, gu, dn, add=add), add)


def test_experts_poisoned_token_and_zero_weights(mok):
    g = gen(6)
    T, H, I, E, k = 40, 64, 64, 4, 2
    x = randn(g, T, H).bfloat16()
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    idx, w = routes(g, T, E, k)
    clean = mok.mok_i8_experts(x, idx, w, gu, dn)
    x[3, 5], x[17, 0] = math.nan, math.inf
    out = mok.mok_i8_experts(x, idx, w, gu, dn)
    rest = [t for t in range(T) if t not in (3, 17)]
    assert torch.isnan(out[3]).all() and torch.isnan(out[17]).all() and torch.equal(out[rest], clean[rest])
    dn.scales.zero_()
    x[3, 5], x[17, 0] = 0.0, 0.0
    assert (mok.mok_i8_experts(x, idx, w, gu, mok.I8Weights(dn.codes, dn.scales)) == 0).all()


def test_experts_weights_beyond_four_gigabytes(mok):
    """Matrices whose offsets pass 32 bits: only the last experts are used."""
    E, H, I, k, T = 160, 7168, 2048, 2, 24
    g = gen(9)
    gu = mok.I8Weights(torch.empty(E, 2 * I, H, device="cuda", dtype=torch.int8), torch.full((E, 2 * I), 1e-3, device="cuda"))
    dn = mok.I8Weights(torch.empty(E, H, I, device="cuda", dtype=torch.int8), torch.full((E, H), 1e-3, device="cuda"))
    for e in range(E - 3, E):
        gu.codes[e] = torch.randint(-127, 128, (2 * I, H), generator=g, device="cuda", dtype=torch.int8)
        dn.codes[e] = torch.randint(-127, 128, (H, I), generator=g, device="cuda", dtype=torch.int8)
    x = randn(g, T, H).bfloat16()
    local, w = routes(g, T, 3, k)
    out = mok.mok_i8_experts(x, local + (E - 3), w, gu, dn)
    last = [mok.I8Weights(m.codes[E - 3:].clone(), m.scales[E - 3:].clone()) for m in (gu, dn)]
    ref, room = experts64(x, local, w, *last)
    assert ((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + room).all()
    assert torch.equal(out, mok.mok_i8_experts(x, local, w, *last))


# ------------------------------------------------------------------------------------- streams, graphs, refusals

def test_other_streams_and_graph_capture(mok):
    g = gen(12)
    logits, x = randn(g, 64, 16), randn(g, 64, 256).bfloat16()
    gu, dn, lin = weights(mok, g, 16, 2 * 128, 256), weights(mok, g, 16, 256, 128), weights(mok, g, 512, 256)

    def calls(**kw):
        idx, w = mok.mok_gate(logits, 4, score="sigmoid", **kw)
        d = mok.mok_gate_backward(logits, idx, w, score="sigmoid", **kw)
        return idx, w, d, mok.mok_i8_linear(x, lin, **kw), mok.mok_i8_experts(x, idx, w, gu, dn, **kw)

    ref = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)                   # the side stream is busy: the results must be ordered behind it
        fresh = x.clone()
    out = mok.mok_i8_linear(fresh, lin, stream=side)
    others = calls(stream=side)
    side.synchronize()
    assert torch.equal(out, ref[3]) and all(torch.equal(a, b) for a, b in zip(ref, others))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = calls()
    logits.copy_(randn(g, 64, 16))
    x.copy_(randn(g, 64, 256))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(captured, calls()))


def test_empty_batches(mok):
    logits = torch.empty(0, 16, device="cuda")
    idx, w = mok.mok_gate(logits, 2)
    assert idx.shape == w.shape == (0, 2) and mok.mok_gate_backward(logits, idx, w).shape == (0, 16)
    x = torch.empty(0, 32, device="cuda", dtype=torch.bfloat16)
    g = gen(1)
    assert mok.mok_i8_linear(x, weights(mok, g, 24, 32)).shape == (0, 24)
    idx = torch.empty(0, 2, device="cuda", dtype=torch.int32)
    out = mok.mok_i8_experts(x, idx, torch.empty(0, 2, device="cuda"), weights(mok, g, 4, 16, 32), weights(mok, g, 4, 32, 8))
    assert out.shape == (0, 32)


def test_refusals(mok):
    E = mok.MokError
    g = gen(1)
    logits = randn(g, 4, 16)
    for bad in (dict(k=17), dict(k=0), dict(k=2, n_groups=3), dict(k=9, n_groups=4, topk_groups=2), dict(k=1, n_groups=16, topk_groups=1),
                dict(k=1, n_groups=2, topk_groups=3), dict(k=1, n_groups=2, topk_groups=1, group_top=3)):
        with pytest.raises(E) as err:
            mok.mok_gate(logits, **bad)
        assert err.value.status == mok.MOK_ERR_SHAPE, bad
    with pytest.raises(E):
        mok.mok_gate(torch.zeros(2, 513, device="cuda"), 1)
    for call in (lambda: mok.mok_gate(logits.cpu(), 2), lambda: mok.mok_gate(logits.double(), 2),
                 lambda: mok.mok_gate(logits.t(), 2), lambda: mok.mok_gate(logits, 2, bias=torch.zeros(15, device="cuda")),
                 lambda: mok.mok_gate(logits, 2, bias=torch.zeros(16)),
                 lambda: mok.mok_gate_backward(logits, torch.zeros(4, 2, device="cuda", dtype=torch.int64), randn(g, 4, 2)),
                 lambda: mok.mok_gate_backward(logits, torch.zeros(4, 2, device="cuda", dtype=torch.int32), randn(g, 4, 3))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        mok.mok_gate(logits, 2, score="tanh")
    for call in (lambda: mok.mok_gate(logits), lambda: mok.mok_gate(logits, 2, groups=2), lambda: mok.mok_gate(logits, 2, k=2),
                 lambda: mok.mok_gate([1.0], 1), lambda: mok.mok_gate(logits, 2, score=3)):
        with pytest.raises(TypeError):
            call()
    x, w = randn(g, 4, 32).bfloat16(), weights(mok, g, 24, 32)
    with pytest.raises(ValueError):
        mok.mok_i8_linear(randn(g, 4, 33).bfloat16(), w)                                    # weights narrower than x
    with pytest.raises(ValueError):
        mok.mok_i8_linear(x, w, bias=torch.zeros(23, device="cuda"))
    with pytest.raises(E) as err:
        mok.mok_i8_matmul(torch.zeros(4, 24, device="cuda", dtype=torch.int8), torch.ones(4, device="cuda"),
                          mok.I8Weights(w.codes[:, :24].contiguous(), w.scales))
    assert err.value.status == mok.MOK_ERR_ALIGN                                            # rows of 24 bytes
    with pytest.raises(E) as err:
        mok.mok_i8_linear(randn(g, 300, 32).bfloat16(), w, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert err.value.status == mok.MOK_ERR_WORKSPACE
    idx, tw = routes(g, 4, 4, 2)
    gu, dn = weights(mok, g, 4, 16, 32), weights(mok, g, 4, 32, 8)
    with pytest.raises(E) as err:
        mok.mok_i8_experts(x, idx, tw, gu, dn, workspace=torch.empty(512, dtype=torch.uint8, device="cuda"))
    assert err.value.status == mok.MOK_ERR_WORKSPACE
    for call in (lambda: mok.mok_i8_experts(x.float(), idx, tw, gu, dn), lambda: mok.mok_i8_experts(x, idx.long(), tw, gu, dn),
                 lambda: mok.mok_i8_experts(x, idx, tw, dn, gu), lambda: mok.mok_i8_experts(x, idx, tw, gu, dn, add=x[:3])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(E) as err:
        mok.mok_i8_experts(randn(g, 4, 28).bfloat16(), idx, tw, weights(mok, g, 4, 16, 28), weights(mok, g, 4, 28, 8))
    assert err.value.status == mok.MOK_ERR_SHAPE                                            # H not a multiple of 8
