"""Routing and 8-bit operators where they can go wrong: precision of small channels, masked groups, signed zeros, extreme
logits, aligned rows of every width, buffers wider than the rows, other streams.  Plain evaluations in 64 bits.

Roundings: 2^-24 of the value for an fp32 operation; half a unit in the last place for the final one."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module")
def mok():
    from paper_2609_36070_b200 import mok
    yield mok
    assert mok.mok_i8_status() == 0


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


# ------------------------------------------------------------------------------------------------------ 8-bit experts

def codes64(x):
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    return torch.where(amax > 0, (x * 127 / amax).round(), torch.zeros_like(x)), (amax / 127).squeeze(-1)


def weights(mok, g, *shape, scales=None):
    codes = torch.randint(-127, 128, (*shape[:-1], (shape[-1] + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
    if scales is None:
        scales = (torch.rand(*shape[:-1], generator=g, device="cuda") + 0.5) * 1e-3
    return mok.I8Weights(codes, scales)


def experts64(x, idx, w, gu, dn):
    T, H = x.shape
    E, I = gu.codes.shape[0], gu.codes.shape[1] // 2
    out = torch.zeros(T, H, dtype=torch.float64, device=x.device)
    q, s = codes64(x)
    for e in range(E):
        t, slot = torch.nonzero(idx == e, as_tuple=True)
        if len(t):
            z = (q[t] @ gu.codes[e, :, :H].double().t()) * s[t, None] * gu.scales[e].double()
            hq, hs = codes64(torch.nn.functional.silu(z[:, :I]) * z[:, I:])
            y = (hq @ dn.codes[e, :, :I].double().t()) * hs[:, None] * dn.scales[e].double()
            out.index_add_(0, t, w[t, slot].double()[:, None] * y)
    return out


def routes(g, T, E, k):
    top = randn(g, T, E).topk(k, -1)
    return top.indices.int().contiguous(), top.values.softmax(-1)


# few rows per expert and many (both products), batches of all three schedules
@pytest.mark.parametrize("T,H,I,E,k", [(40, 256, 128, 8, 2), (900, 256, 192, 4, 2), (9000, 136, 64, 8, 4)])
def test_experts_small_and_negative_channel_scales(mok, T, H, I, E, k):
    """Output channels whose scales span ten orders of magnitude, some negative: every column keeps its own precision."""
    g = gen(T)
    x = randn(g, T, H).bfloat16()
    scales = 10.0 ** (-10 * torch.rand(E, H, generator=g, device="cuda"))
    scales = torch.where(torch.rand(E, H, generator=g, device="cuda") < 0.3, -scales, scales)
    scales[:, 3] = -1.0
    scales[:, 5] = 1e-10
    scales[:, 7] = 0.0
    scales[1] = -scales[1].abs()                          # a matrix without any positive scale
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I, scales=scales)
    idx, w = routes(g, T, E, k)
    out = mok.mok_i8_experts(x, idx, w, gu, dn).double()
    ref = experts64(x, idx, w, gu, dn)
    assert (out[:, 7] == 0).all()
    # one bf16 rounding moves a value by 2^-8 of it at most, and by less than half of that in the mean square; a code of the
    # hidden row on the other side of a tie (one value in 2^14) moves a column by some 2^-7 / sqrt(I) of one of its T values
    assert ((out - ref).norm(dim=0) <= 2.0 ** -8 * ref.norm(dim=0)).all()


@pytest.mark.parametrize("T,H,I,E,k", [(64, 256, 64, 8, 2), (1000, 256, 64, 4, 2), (9000, 136, 64, 8, 4)])
def test_experts_round_once(mok, T, H, I, E, k):
    """fp16 outputs are the rounded 64-bit ones but for what 32-bit sums move across a rounding boundary.  Each output carries
    some ten roundings of 2^-24 where the unit is 2^-11: one in 400 moves.  A hidden value is good to about 2^-21 of itself, 127
    times that of a code: less than one row in 100 has a code on the other side of a tie.  A row with a second rounding to 11
    bits would move every fourth output."""
    g = gen(T + 1)
    x = randn(g, T, H).half()
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    dn.scales.mul_(20)                                     # (normal numbers of fp16)
    idx, w = routes(g, T, E, k)
    out = mok.mok_i8_experts(x, idx, w, gu, dn)
    ref = experts64(x, idx, w, gu, dn)
    assert ref.abs().max() < 6e4
    assert (out != ref.half()).double().mean() <= 0.02


def test_experts_broken_channel_and_zero_weight(mok):
    """A channel whose scale is NaN is NaN for its expert's tokens, and no other channel is; a weight of 0 on a row that is NaN
    gives NaN."""
    g = gen(3)
    T, H, I, E = 48, 64, 64, 4
    x = randn(g, T, H).bfloat16()
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    idx = (torch.arange(T, device="cuda") % E)[:, None].int().contiguous()
    w = torch.ones(T, 1, device="cuda")
    clean = mok.mok_i8_experts(x, idx, w, gu, dn)
    dn.scales[2, 9] = math.nan
    out = mok.mok_i8_experts(x, idx, w, gu, mok.I8Weights(dn.codes, dn.scales))
    bad = torch.zeros(T, H, dtype=torch.bool, device="cuda")
    bad[2::4, 9] = True
    assert torch.equal(torch.isnan(out), bad) and torch.equal(out[~bad], clean[~bad])
    w[2] = 0.0
    out = mok.mok_i8_experts(x, idx, w, gu, mok.I8Weights(dn.codes, dn.scales))
    assert torch.isnan(out[2, 9]) and (out[2, :9] == 0).all() and (out[2, 10:] == 0).all()


# --------------------------------------------------------------------------------------------------------------- gate
# T = 33 is served by the kernel with a warp per token, T = 2433 by the one with four tokens per warp.

@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("E", [40, 64, 160, 256])
def test_gate_zeros_of_both_signs_are_equal(mok, T, dtype, E):
    """Few zeros of both signs decide the k-th place: fewer than the lists hold, in the same and in different pieces of four."""
    g = gen(E)
    logits = torch.full((T, E), -1.0, device="cuda")
    at = torch.rand(T, E, generator=g, device="cuda").argsort(-1)
    zeros = torch.where(torch.randint(0, 2, (T, 20), generator=g, device="cuda") > 0, -0.0, 0.0)
    logits.scatter_(1, at[:, :20], zeros)
    above = torch.randint(0, 7, (T, 1), generator=g, device="cuda") > torch.arange(6, device="cuda")
    logits.scatter_(1, at[:, 20:26], torch.where(above, randn(g, T, 6).abs() + 0.5, torch.full((T, 6), -2.0, device="cuda")))
    logits[0] = -1.0                                       # every piece has a zero of both signs, the positive one later
    logits[0, 0:32:4], logits[0, 1:32:4] = -0.0, 0.0
    logits[1] = -1.0
    logits[1, 0:24:4], logits[1, 1], logits[1, 24], logits[1, 28] = 1.0, -0.0, 0.0, 0.0
    logits = logits.to(dtype)
    for k in (3, 5, 8, 16):
        idx, _ = mok.mok_gate(logits, k, score="sigmoid")
        ref = logits.float().add(0.0).sort(dim=-1, descending=True, stable=True).indices[:, :k]     # (-0 + 0 is +0)
        assert torch.equal(idx.long(), ref), k


@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("k", [1, 2, 8])
def test_gate_weights_of_subnormal_scores(mok, T, k):
    """Sigmoid scores of logits around -88 are subnormal numbers of 32 bits, good to 2^-149: their renormalised weights are
    finite and right to that."""
    E = 16
    logits = -87.5 - 1.2 * torch.rand(T, E, generator=gen(k), device="cuda")               # scores of 3e-39 .. 1e-38
    for scale in (1.0, 2.5, 40.0):
        idx, w = mok.mok_gate(logits, k, score="sigmoid", scale=scale)
        s = torch.sigmoid(logits.double()).gather(1, idx.long())
        ref = scale * s / s.sum(-1, keepdim=True)
        # a score is off by 2^-22 of itself (exponential, quotient) and half of 2^-149; so is the sum, k times
        off = 2.0 ** -22 + 2.0 ** -150 / s.min()
        assert ((w.double() - ref).abs() <= 4 * off * ref).all()


@pytest.mark.parametrize("k", [1, 2, 8])
def test_gate_gradient_of_subnormal_scores(mok, k):
    T, E = 300, 16
    logits = -87.5 - 1.2 * torch.rand(T, E, generator=gen(k), device="cuda")
    idx, _ = mok.mok_gate(logits, k, score="sigmoid")
    dw = randn(gen(k + 1), T, k)
    d = mok.mok_gate_backward(logits, idx, dw, score="sigmoid", scale=2.5)
    s = torch.sigmoid(logits.double()).gather(1, idx.long())
    r, g = s / s.sum(-1, keepdim=True), 2.5 * dw.double()
    ref = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    ref.scatter_(1, idx.long(), r * (1 - s) * (g - (g * r).sum(-1, keepdim=True)))
    # r is off by 4 (2^-22 + 2^-150 / s) of itself, as the weights are, and multiplies differences of the largest |g|
    off = 4 * (2.0 ** -22 + 2.0 ** -150 / s.min())
    assert ((d.double() - ref).abs() <= 4 * off * g.abs().amax(-1, keepdim=True)).all()


@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("E,k", [(40, 8), (64, 3), (60, 16), (256, 8), (300, 20)])
def test_gate_order_of_extreme_logits(mok, T, dtype, E, k):
    """+inf, finite values down to the type's lowest, -inf, NaN: in this order, equals by their ids, for tokens that have fewer
    ordinary experts than k."""
    g = gen(E + k)
    kind = torch.randint(0, 40, (T, E), generator=g, device="cuda")
    low = torch.finfo(dtype).min
    logits = torch.full((T, E), -math.inf, device="cuda")
    for at, v in ((0, 1.0), (1, -2.0), (2, low), (3, low / 2), (4, math.nan), (5, -low)):
        logits[kind == at] = v
    logits[T // 2:][kind[T // 2:] >= 20] = low             # half of the tokens: mostly the lowest value
    logits[3:6] = -math.inf
    logits[3, E - 1], logits[4, 1], logits[5, E // 2] = low, low, 0.0
    logits[6:9] = math.nan
    logits[6, E - 1], logits[7, 1] = -math.inf, low
    logits[9, :] = low
    logits[9, 5] = -math.inf
    logits = logits.to(dtype)
    idx, _ = mok.mok_gate(logits, k, score="sigmoid")
    order = logits.double()
    order = torch.where(torch.isnan(order), -1e40, torch.where(order == -math.inf, -1e39, order))
    assert torch.equal(idx.long(), order.sort(dim=-1, descending=True, stable=True).indices[:, :k])


@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("score,with_bias", [("sigmoid", False), ("sigmoid", True), ("softmax", False)])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("E,G,top_groups,k", [(64, 8, 4, 6), (64, 16, 5, 8), (160, 8, 3, 3), (60, 5, 2, 5), (54, 6, 3, 4)])
def test_gate_groups_with_masked_experts(mok, T, score, with_bias, group_top, E, G, top_groups, k):
    """Groups of which a token may use no, one, two or more experts: the value of a group is that of its usable ones."""
    g = gen(E + G)
    gs = E // G
    logits = randn(g, T, E)
    usable = torch.randint(0, 5, (T, G), generator=g, device="cuda")                       # 4: all
    place = torch.rand(T, G, gs, generator=g, device="cuda").argsort(-1)
    masked = ((place >= usable[..., None]) & (usable < 4)[..., None]).view(T, E)
    logits[masked] = -math.inf
    if score == "sigmoid":                                                                 # (a NaN breaks a whole softmax)
        logits[masked & (torch.rand(T, E, generator=g, device="cuda") < 0.2)] = math.nan
    logits[0] = -math.inf                                                                  # the seventh expert alone is left
    logits[0, 7] = -3.0
    logits[1, :gs] = -math.inf
    logits[1, gs:] = randn(g, E - gs)
    logits[1, -gs:] = -math.inf                                                            # one left of the last group ...
    logits[1, -2] = 4.0
    logits[1, gs:2 * gs] = -math.inf                                                       # ... and none of the first two
    bias = randn(g, E) * 0.1 if with_bias else None
    idx, w = mok.mok_gate(logits, k, bias=bias, score=score, n_groups=G, topk_groups=top_groups, group_top=group_top)
    z = logits.double()
    dead = torch.isnan(z) | (z == -math.inf)
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    c = (s if bias is not None or group_top == 2 else z) + (0 if bias is None else bias.double())
    c = torch.where(dead, -1e30, c)
    best = c.view(T, G, gs).topk(min(2, gs), -1).values
    value = torch.where((best[..., 1] > -1e29) & (group_top == 2), best.sum(-1), best[..., 0])
    order = value.sort(dim=-1, descending=True, stable=True)
    clear = (order.values[:, top_groups - 1] - order.values[:, top_groups] > 1e-6) | (order.values[:, top_groups] < -1e29)
    keep = torch.zeros(T, G, dtype=torch.bool, device="cuda").scatter_(1, order.indices[:, :top_groups], True)
    c = torch.where(torch.isnan(z), -2e30, c).masked_fill(~keep.repeat_interleave(gs, 1), -math.inf)
    order = c.sort(dim=-1, descending=True, stable=True)
    gaps = order.values[:, :k] - order.values[:, 1:k + 1]
    clear &= ((gaps > 1e-6) | (order.values[:, :k] < -1e29)).all(-1)
    assert clear.float().mean() > 0.97 and clear[:2].all()
    assert torch.equal(idx.long()[clear], order.indices[:, :k][clear])
    alive = (~dead).any(-1)
    assert not dead.gather(1, idx.long())[alive, 0].any()                                  # no masked expert before a usable one


@pytest.mark.parametrize("score,with_bias,renorm", [("sigmoid", True, True), ("sigmoid", False, False), ("softmax", False, True),
                                                    ("softmax", True, False), ("softmax", False, False)])
@pytest.mark.parametrize("E,G,top_groups,k,dtype", [(8, 1, 1, 2, torch.float32), (60, 1, 1, 4, torch.float16), (64, 8, 3, 6, torch.bfloat16),
                                                    (160, 8, 3, 6, torch.float32), (256, 8, 4, 8, torch.float32), (256, 1, 1, 8, torch.bfloat16),
                                                    (384, 1, 1, 10, torch.float32), (384, 4, 2, 32, torch.bfloat16), (511, 1, 1, 17, torch.float32),
                                                    (512, 16, 5, 16, torch.float32)])
@pytest.mark.parametrize("pitch", [0, 3])
def test_gate_gives_a_token_the_same_bits_in_any_batch(mok, score, with_bias, renorm, E, G, top_groups, k, dtype, pitch):
    g = gen(E + k)
    T = 2900
    logits = (randn(g, T, E + pitch) * 2).to(dtype)[:, :E]
    logits[5:40][torch.rand(35, E, generator=g, device="cuda") < 0.7] = -math.inf
    logits[40:60][torch.rand(20, E, generator=g, device="cuda") < 0.7] = torch.finfo(dtype).min
    logits[60] = -math.inf
    logits[61, 3] = math.nan
    logits[62, 3] = math.inf
    logits[63:90] -= 80.0
    bias = randn(g, E) * 0.1 if with_bias else None
    kw = dict(bias=bias, score=score, n_groups=G, topk_groups=top_groups, group_top=2, renormalise=renorm, scale=1.7)
    idx, w = mok.mok_gate(logits, k, **kw)
    for some in (slice(0, 1), slice(0, 100), slice(900, 2900)):
        i, v = mok.mok_gate(logits[some], k, **kw)
        assert torch.equal(i, idx[some]) and ((v == w[some]) | (torch.isnan(v) & torch.isnan(w[some]))).all()
    assert torch.isfinite(w[63:]).all() and (w[60] == 0).all()


# ------------------------------------------------------------------------------------------------- what a call leaves

@pytest.mark.parametrize("dependent", [False, True])
def test_calls_leave_the_threads_launch_mode(mok, dependent):
    """The layer's serial_launches sets how the later entry points that read the mode launch; these operators put it back."""
    import ctypes
    from paper_2609_36070_b200 import build
    mode = ctypes.c_bool.in_dll(ctypes.CDLL(build.LIB), "_ZN3mok5g_pdlE")
    g = gen(1)
    logits, x = randn(g, 12, 16), randn(g, 12, 64).bfloat16()
    gu, dn = weights(mok, g, 16, 32, 64), weights(mok, g, 16, 64, 16)
    lin = mok.I8Weights(gu.codes[0], gu.scales[0])
    before = mode.value
    try:
        for call in (lambda: mok.mok_gate(logits, 2), lambda: mok.mok_i8_quantize(x), lambda: mok.mok_i8_linear(x, lin),
                     lambda: mok.mok_gate_backward(logits, *mok.mok_gate(logits, 2)),
                     lambda: mok.mok_i8_experts(x, *mok.mok_gate(logits, 2), gu, dn)):
            mode.value = dependent
            call()
            assert mode.value == dependent
    finally:
        mode.value = before


def test_weights_quantised_on_another_stream(mok):
    """Codes, scales and the largest scales all belong to the stream that is named."""
    g = gen(2)
    W = randn(g, 5, 64, 96)
    ref = mok.I8Weights.quantize(W)
    side = torch.cuda.Stream()
    for n in range(3):
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)                   # the stream is busy when the call is made
            late = W.clone()
        q = mok.I8Weights.quantize(late, stream=side)
        side.synchronize()
        assert torch.equal(q.codes, ref.codes) and torch.equal(q.scales, ref.scales) and torch.equal(q.max, ref.scales.amax(-1))
        del q, late
        torch.full((5,), 7.0, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [1, 3, 1300])
@pytest.mark.parametrize("K,stride", [(16, 64), (16, 48), (20, 64), (20, 24), (24, 48), (7, 16), (7, 7), (2048, 2080), (2056, 2096), (17000, 17040)])
def test_quantised_rows_of_a_wider_buffer(mok, dtype, rows, K, stride):
    """Codes as a column range of a wider buffer: what follows the next multiple of 16 columns is not written."""
    import ctypes
    from paper_2609_36070_b200 import build
    f = ctypes.CDLL(build.LIB).mok_i8_quantize
    f.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong, ctypes.c_int, ctypes.c_longlong, ctypes.c_void_p,
                  ctypes.c_longlong, ctypes.c_void_p, ctypes.c_void_p]
    x = randn(gen(K), rows, K).to(dtype)
    want, _ = mok.mok_i8_quantize(x)
    buffer = torch.full((rows + 2, stride), 77, dtype=torch.int8, device="cuda")           # (a row before and one behind)
    scales = torch.empty(rows, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert f(x.data_ptr(), 2 if dtype == torch.float32 else 0, rows, K, K, buffer[1].data_ptr(), stride, scales.data_ptr(), stream) == 0
    end = min(stride, (K + 15) // 16 * 16)
    assert torch.equal(buffer[1:-1, :K], want[:, :K]) and (buffer[1:-1, K:end] == 0).all()
    assert (buffer[1:-1, end:] == 77).all() and (buffer[0] == 77).all() and (buffer[-1] == 77).all()


def test_gate_of_the_largest_number_of_tokens(mok):
    """2^31 - 1 tokens: the step past the last one does not fit 32 bits (two experts in two groups: a warp per token)."""
    T = 2 ** 31 - 1
    logits = torch.zeros(T, 2, dtype=torch.bfloat16, device="cuda")
    logits[-1, 1] = logits[T // 2, 1] = logits[0, 1] = 1.0
    idx, w = mok.mok_gate(logits, 1, n_groups=2, group_top=1, renormalise=False)
    torch.cuda.synchronize()
    at = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    assert idx[at, 0].tolist() == [1, 0, 1, 0, 1]
    assert (w[at, 0].double() - torch.tensor([1.0, 0.0, 1.0, 0.0, 1.0], device="cuda", dtype=torch.float64).sigmoid()).abs().max() < 1e-6


def test_gate_refuses_k_before_it_allocates(mok):
    logits = torch.zeros(1 << 16, 8, device="cuda")
    for k in (9, 1 << 30, 2 ** 31 - 1, 0, -1):
        with pytest.raises(mok.MokError) as e:
            mok.mok_gate(logits, k)
        assert e.value.status == mok.MOK_ERR_SHAPE
    for k in (2 ** 31, -2 ** 31 - 1):
        with pytest.raises(ValueError):
            mok.mok_gate(logits, k)


def test_matmul_refuses_a_contraction_out_of_range(mok):
    g = gen(1)
    w = weights(mok, g, 24, 32)
    codes, scales = torch.zeros(1, 16, dtype=torch.int8, device="cuda"), torch.ones(1, device="cuda")
    for K in (-2 ** 32 + 32, 2 ** 32 + 16, 2 ** 31, 2 ** 63 - 1, 33, 17):
        with pytest.raises(ValueError):
            mok.mok_i8_matmul(codes, scales, w, K=K)
    for K in (0, -1, -2 ** 31):
        with pytest.raises(mok.MokError) as e:
            mok.mok_i8_matmul(codes, scales, w, K=K)
        assert e.value.status == mok.MOK_ERR_SHAPE


@pytest.mark.parametrize("K", [16, 100, 2049])
def test_products_of_single_rows(mok, K):
    """One token's codes, or one channel's, need no pitch of whole 16 bytes."""
    g = gen(K)
    for M, N in ((1, 40), (1, 1), (300, 1)):
        codes = torch.randint(-127, 128, (M, K if M == 1 else (K + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
        wide = torch.randint(-127, 128, (N, K if N == 1 else (K + 15) // 16 * 16), generator=g, device="cuda", dtype=torch.int8)
        s, ws = torch.rand(M, generator=g, device="cuda"), torch.rand(N, generator=g, device="cuda")
        out = mok.mok_i8_matmul(codes, s, mok.I8Weights(wide, ws), K=K, out_dtype=torch.float32)
        ref = (codes[:, :K].double() @ wide[:, :K].double().t()) * s.double()[:, None] * ws.double()
        assert ((out.double() - ref).abs() <= 4 * UNIT[torch.float32] * ref.abs()).all()


# ------------------------------------------------------------------------------ aligned rows of every width, large batches

@pytest.mark.parametrize("T", [70, 2500])
@pytest.mark.parametrize("E,G,top_groups,k", [(28, 1, 1, 6), (64, 1, 1, 6), (128, 1, 1, 8), (160, 8, 3, 6), (192, 1, 1, 12), (256, 8, 4, 8),
                                              (256, 1, 1, 8), (256, 1, 1, 2), (256, 1, 1, 20), (320, 10, 4, 9), (384, 1, 1, 8), (384, 4, 2, 8),
                                              (512, 1, 1, 10), (512, 16, 6, 8)])
@pytest.mark.parametrize("dtype,score,with_bias,renorm", [(torch.float32, "sigmoid", True, True), (torch.bfloat16, "softmax", False, True),
                                                          (torch.float16, "softmax", True, False), (torch.float32, "softmax", False, False)])
def test_gate_of_aligned_rows(mok, T, E, G, top_groups, k, dtype, score, with_bias, renorm):
    g = gen(E + k)
    logits = (randn(g, T, E) * 1.5).to(dtype)
    bias = randn(g, E) * 0.05 if with_bias else None
    idx, w = mok.mok_gate(logits, k, bias=bias, score=score, n_groups=G, topk_groups=top_groups, group_top=2, renormalise=renorm, scale=2.5)
    z = logits.double()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    by_score = with_bias or G > 1
    c = s + bias.double() if with_bias else s if by_score else z
    grouped = torch.ones(T, dtype=torch.bool, device="cuda")                               # tokens whose groups fp32 cannot mistake
    if G > 1:
        value = c.view(T, G, E // G).topk(2, -1).values.sum(-1)
        order = value.sort(dim=-1, descending=True, stable=True)
        grouped = order.values[:, top_groups - 1] - order.values[:, top_groups] > 1e-6
        keep = torch.zeros(T, G, dtype=torch.bool, device="cuda").scatter_(1, order.indices[:, :top_groups], True)
        c = c.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    order = c.sort(dim=-1, descending=True, stable=True)
    assert grouped.float().mean() > 0.97
    assert (c.gather(1, idx.long()) - order.values[:, :k])[grouped].abs().max() <= 1e-6
    clear = grouped                                        # logits are compared as they are, fp32 decides closer scores
    if by_score:
        clear = grouped & (order.values[:, :k] - order.values[:, 1:k + 1] > 1e-6).all(-1)
    assert torch.equal(idx.long()[clear], order.indices[:, :k][clear])
    ref = s.gather(1, idx.long())
    ref = 2.5 * (ref / ref.sum(-1, keepdim=True) if renorm else ref)
    # exponentials, sums of up to 512 terms in lanes of 16 and a tree, quotients: less than 64 roundings
    assert ((w.double() - ref).abs() <= 64 * UNIT[torch.float32] * ref).all()


@pytest.mark.parametrize("T,E,k", [(300, 64, 4), (301, 128, 8), (302, 256, 8), (303, 384, 6), (304, 512, 16), (200_001, 8, 2), (160_000, 36, 4)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("score,renorm", [("softmax", False), ("softmax", True), ("sigmoid", True), ("sigmoid", False)])
def test_gate_gradient_of_aligned_rows(mok, T, E, k, dtype, score, renorm):
    g = gen(E + k)
    logits = randn(g, T, E).to(dtype)
    idx, _ = mok.mok_gate(logits, k, score=score, renormalise=renorm)
    dw = randn(g, T, k)
    d = mok.mok_gate_backward(logits, idx, dw, score=score, renormalise=renorm, scale=1.7)
    z = logits.double().requires_grad_()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    w = s.gather(1, idx.long())
    ref, = torch.autograd.grad((w / w.sum(-1, keepdim=True) if renorm else w) * 1.7, z, dw.double())
    # as for rows of any alignment: 64 roundings of the token's largest |g|
    room = 64 * UNIT[torch.float32] * 1.7 * dw.abs().amax(-1, keepdim=True).double()
    assert ((d.double() - ref).abs() <= UNIT[dtype] * ref.abs() + room).all()


@pytest.mark.parametrize("M,K,N", [(2049, 256, 520), (2305, 130, 1000), (4100, 384, 72), (7000, 64, 300), (16384, 512, 256)])
@pytest.mark.parametrize("dtype,out_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32)])
def test_linear_of_many_rows(mok, M, K, N, dtype, out_dtype):
    """Row tiles past the first group of 2048 rows, with and without a bias."""
    g = gen(M)
    x, w, bias = randn(g, M, K).to(dtype), weights(mok, g, N, K), randn(g, N)
    codes, scales = mok.mok_i8_quantize(x)
    for b in (None, bias):
        out = mok.mok_i8_linear(x, w, bias=b, out_dtype=out_dtype)
        ref = (codes[:, :K].double() @ w.codes[:, :K].double().t()) * scales.double()[:, None] * w.scales.double()
        room = 4 * UNIT[torch.float32] * ref.abs()
        if b is not None:
            ref, room = ref + b.double(), room + 4 * UNIT[torch.float32] * b.double().abs()
        assert ((out.double() - ref).abs() <= UNIT[out_dtype] * ref.abs() + room).all()


# ------------------------------------------------------------------------------------------------------ bounded waits

def test_waits_of_the_products_run_out(mok):
    """Products whose loads never come end with a status, and the next calls are as before: few tokens (quantised in the kernel,
    and codes), pairs of CTAs, experts with few and with many rows, of all tile sizes."""
    g = gen(5)
    lin, wide = weights(mok, g, 640, 512), weights(mok, g, 4096, 1024)
    gu, dn = weights(mok, g, 4, 128, 512), weights(mok, g, 4, 512, 64)
    x = {T: randn(g, T, 512).bfloat16() for T in (3, 100, 150, 600)}
    many = randn(g, 1500, 1024).bfloat16()
    r = {T: routes(g, T, 4, 2) for T in x}

    def calls():
        yield lambda: mok.mok_i8_linear(x[3], lin)
        yield lambda: mok.mok_i8_linear(x[150], lin)
        yield lambda: mok.mok_i8_linear(many, wide)
        for T in (3, 100, 150, 600):
            yield lambda: mok.mok_i8_experts(x[T], *r[T], gu, dn)

    good = [call() for call in calls()]
    assert mok.mok_i8_status() == mok.MOK_OK
    try:
        for call in calls():
            mok.mok_i8_starve(20_000)
            call()
            assert mok.mok_i8_status() == mok.MOK_ERR_TIMEOUT
            assert mok.mok_i8_status() == mok.MOK_OK       # read once
    finally:
        mok.mok_i8_starve(0)
    assert all(torch.equal(a, call()) for a, call in zip(good, calls()))
    assert mok.mok_i8_status() == mok.MOK_OK


@pytest.mark.parametrize("H,I,E,k", [(256, 64, 4, 2), (136, 200, 16, 4)])
def test_experts_give_a_token_the_same_bits_in_any_batch(mok, H, I, E, k):
    g = gen(H)
    T = 9000
    x, (idx, w) = randn(g, T, H).half(), routes(g, T, E, k)
    idx[::7, 0] = -1
    gu, dn = weights(mok, g, E, 2 * I, H), weights(mok, g, E, H, I)
    whole = mok.mok_i8_experts(x, idx, w, gu, dn)
    for n in (1, 40, 100, 300, 900, 4000):
        assert torch.equal(mok.mok_i8_experts(x[:n], idx[:n].contiguous(), w[:n].contiguous(), gu, dn), whole[:n]), n


@pytest.mark.parametrize("K,N", [(1040, 520), (256, 2000)])
def test_linear_gives_a_token_the_same_bits_in_any_batch(mok, K, N):
    g = gen(K)
    x, w, bias = randn(g, 6000, K).bfloat16(), weights(mok, g, N, K), randn(g, N)
    for b in (None, bias):
        whole = mok.mok_i8_linear(x, w, bias=b, out_dtype=torch.float32)
        for n in (1, 16, 40, 128, 256, 400, 2500):
            assert torch.equal(mok.mok_i8_linear(x[:n], w, bias=b, out_dtype=torch.float32), whole[:n]), n


@pytest.mark.parametrize("T", [33, 2433])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("E,G", [(40, 1), (64, 8)])
def test_gate_nan_rows_are_not_taken_for_masked_ones(mok, T, score, with_bias, E, G):
    """A NaN reaches its token's weights and gradients, also where nothing but NaN and masks is left."""
    k = 6
    logits = randn(gen(E), T, E)
    logits[0] = math.nan
    logits[1], logits[1, 1::2] = math.nan, -math.inf
    logits[2, 11] = math.nan
    logits[3] = -math.inf
    bias = torch.zeros(E, device="cuda") if with_bias else None
    for renorm in (True, False):
        kw = dict(score=score, renormalise=renorm)
        idx, w = mok.mok_gate(logits, k, bias=bias, n_groups=G, topk_groups=G, **kw)
        assert torch.equal(idx[0], torch.arange(k, device="cuda", dtype=torch.int32)) and torch.isnan(w[0]).all()
        assert (w[3] == 0).all() and torch.isfinite(w[4:]).all()
        every = torch.arange(k, device="cuda", dtype=torch.int32).expand(T, k).contiguous()
        d = mok.mok_gate_backward(logits, every, torch.ones(T, k, device="cuda") * torch.arange(k, device="cuda"), **kw)
        assert torch.isnan(d[0, 1:k]).all() and torch.isfinite(d[3:]).all()
        if score == "softmax" and not renorm:
            assert torch.isnan(w[2]).all() and torch.isnan(d[:3]).all()
