"""The join between two blocks and its gradients against an evaluation in 64 bits (join_reference.py, which derives the bounds)."""
import pytest
import torch

import join_reference as ref

pytestmark = pytest.mark.gpu
BF, HF, FF = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def mok():
    from paper_2609_36070_b200 import mok
    return mok


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def half(t):
    return torch.finfo(t).eps / 2


def make(seed, T, H, dtype, stream, vectors, before, after, gate, shift, pad=0):
    """Inputs by name; rows of buffers that are `pad` elements wider, starting at an element that is not aligned."""
    g = gen(seed)
    def matrix(t, scale=1.0):
        return (randn(g, T, H + pad) * scale).to(t)[:, pad // 2:pad // 2 + H] if pad else (randn(g, T, H) * scale).to(t)
    large = torch.where(torch.rand(H + pad, generator=g, device="cuda") < 0.05, 10.0, 2.0)
    d = {"x": matrix(stream, large), "y": matrix(dtype), "d_sum": matrix(stream), "d_normed": matrix(dtype) if before else None}
    rule = {"before": before, "after": after}
    for end, norm in (("before", before), ("after", after)):
        rule[end + "_weight"] = (1 + 0.2 * randn(g, H)).to(vectors) if norm else None
        rule[end + "_bias"] = (0.3 * randn(g, H)).to(vectors) if norm and shift else None
    rule["gate"] = {None: None, "channel": (0.3 * randn(g, H)).to(vectors), "token": torch.sigmoid(randn(g, T, 1)).to(dtype),
                    "full": matrix(dtype)}[gate]
    return d, rule


def wide(rule):
    return {k: v.double() if torch.is_tensor(v) else v for k, v in rule.items()}


def near(got, want, bound, what):
    if want is None:
        assert got is None, what
        return
    far = ((got.double() - want).abs() / bound.expand_as(want)).max().item() if want.numel() else 0.0
    assert far <= 1, (what, far)


def check(mok, d, rule, scale=1.0, eps=1e-6, p=0.0, seed=0, offset=0, grad=True):
    T, H = d["y"].shape
    more = dict(scale=scale, eps=eps, p=p)
    keys = dict(seed=seed, offset=offset)
    mask = ref.kept(T, H, p, seed, offset, "cuda") if p > 0 else None
    total, normed = mok.mok_block_join(d["x"], d["y"], **rule, **more, **keys)
    assert total.dtype == d["x"].dtype and (normed is None or normed.dtype == d["y"].dtype)
    want, bound, want_n, bound_n = ref.forward_bounds(d["x"].double(), d["y"].double(), half(total.dtype), half(d["y"].dtype), mask=mask, **wide(rule), **more)
    near(total, want, bound, "sum")
    near(normed, want_n, bound_n, "normed")
    if not grad:
        return total, normed
    got = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, **more, **keys)
    want, bound = ref.backward_bounds(d["d_sum"].double(), None if d["d_normed"] is None else d["d_normed"].double(), total.double(), d["y"].double(),
                                      half(total.dtype), half(d["y"].dtype), mask=mask, **wide(rule), **more)
    for name, a, b, c in zip(("dx", "dy", "dgate", "dbefore_weight", "dbefore_bias", "dafter_weight", "dafter_bias"), got, want, bound):
        near(a, b, c, name)
    again = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, **more, **keys)
    for a, b in zip(got, again):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))         # the same bits on every run
    return total, normed


RULES = [  # before, after, gate, shift, scale, p
    ("rms", None, None, False, 1.0, 0.0), ("rms", "rms", None, False, 0.5, 0.0), ("layer", "layer", "channel", True, 1.0, 0.1),
    (None, "rms", "full", True, -2.0, 0.5), ("layer", None, "token", False, 1.0, 0.0), ("rms", "layer", "full", True, 0.25, 0.9),
    (None, None, None, False, 1.0, 0.3), ("layer", "rms", "channel", False, 1.0, 0.0), (None, "layer", "token", True, 1.0, 0.0),
]


@pytest.mark.parametrize("dtype,stream,vectors", [(BF, BF, FF), (HF, HF, BF), (FF, FF, FF), (BF, FF, BF), (HF, FF, HF)])
@pytest.mark.parametrize("before,after,gate,shift,scale,p", RULES)
@pytest.mark.parametrize("T,H", [(5, 64), (37, 257), (700, 1000), (33, 2880)])
def test_types_and_rules(mok, T, H, before, after, gate, shift, scale, p, dtype, stream, vectors):
    d, rule = make(T + H, T, H, dtype, stream, vectors, before, after, gate, shift)
    check(mok, d, rule, scale=scale, p=p, seed=0x123456789ABCDEF, offset=77)


@pytest.mark.parametrize("T,H", [(1, 1), (1, 8), (3, 5), (2, 7), (9, 8), (1, 8192), (3, 8191), (601, 256), (600, 264), (700, 4096), (700, 4104), (650, 7168),
                                 (1, 2048), (4097, 16), (3000, 512), (3001, 520), (200, 8192), (601, 2047)])
@pytest.mark.parametrize("before,after,gate,shift", [("rms", "rms", None, False), ("layer", "layer", "channel", True), ("layer", "layer", "full", True)])
def test_sizes(mok, T, H, before, after, gate, shift):
    d, rule = make(T * H, T, H, BF, BF, FF, before, after, gate, shift)
    check(mok, d, rule, eps=1e-3, p=0.2, seed=3)


@pytest.mark.parametrize("pad", [16, 2, 5])
@pytest.mark.parametrize("H", [512, 500])
def test_rows_of_wider_buffers(mok, pad, H):
    d, rule = make(pad, 700, H, BF, FF, FF, "rms", "layer", "full", True, pad=pad)
    check(mok, d, rule, scale=0.5)
    # aligned copies of the same rows: other code adds up a row's elements in another order, so both are held to the same bound
    check(mok, {k: v.contiguous() for k, v in d.items()}, {k: v.contiguous() if torch.is_tensor(v) else v for k, v in rule.items()}, scale=0.5)


def test_a_mean_that_is_large_beside_the_spread(mok):
    """Two-pass statistics: a mean of 100 beside a spread of 0.1 loses no more than the input's own bits."""
    d, rule = make(1, 40, 1024, FF, FF, FF, "layer", "layer", None, True)
    d["x"], d["y"] = 100 + 0.1 * d["x"], 100 + 0.1 * d["y"]
    check(mok, d, rule)


def test_rows_of_zeros_and_constants(mok):
    d, rule = make(2, 6, 320, BF, BF, FF, "rms", "layer", None, True)
    d["x"][0], d["y"][0], d["y"][1] = 0, 0, 3.0
    total, normed = check(mok, d, rule, eps=1e-5)
    assert torch.isfinite(normed).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("H", [256, 1000, 1001])
def test_a_broken_row_breaks_no_other(mok, bad, H):
    d, rule = make(3, 300, H, BF, BF, FF, "layer", "rms", "token", False)
    clean = mok.mok_block_join(d["x"], d["y"], **rule)
    back = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], clean[0], d["y"], **rule)
    y = d["y"].clone()
    y[7, H - 1] = bad
    others = torch.arange(300, device="cuda") != 7
    broken = mok.mok_block_join(d["x"], y, **rule)
    for a, b in zip(clean, broken):
        assert torch.equal(a[others], b[others]) and b[7].isnan().any()
    broken = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], clean[0], y, **rule)
    assert torch.equal(back[0], broken[0])                               # (y has no part in dx)
    assert torch.equal(back[1][others], broken[1][others]) and broken[1][7].isnan().any()


@pytest.mark.parametrize("H", [64, 1030])
def test_dropout_alone(mok, H):
    T = 500
    y = torch.ones(T, H, device="cuda")
    for p, seed, offset in ((0.5, 1, 0), (0.1, -1, 1 << 40), (0.999, 1 << 63, 5)):
        out = mok.mok_block_join(None, y, p=p, seed=seed, offset=offset)[0]
        mask = ref.kept(T, H, p, seed % (1 << 64), offset, "cuda")
        assert torch.equal(out != 0, mask) and torch.allclose(out[mask], torch.tensor(1 / (1 - p), device="cuda"), rtol=1e-6)
        back = mok.mok_block_join_backward(y, None, None, y, p=p, seed=seed, offset=offset)[1]
        assert torch.equal(back, out)
        where = torch.tensor([seed if seed < 1 << 63 else seed - (1 << 64), offset], device="cuda")
        assert torch.equal(mok.mok_block_join(None, y, p=p, seed=where)[0], out)
    assert torch.equal(mok.mok_block_join(None, y, p=0.0)[0], y)
    y[0, 0] = float("nan")
    assert (mok.mok_block_join(None, y, p=1.0)[0] == 0).all()


def test_the_norm_alone(mok):
    """Before the first block: x is handed through, normed may be of a narrower type."""
    d, rule = make(4, 50, 640, BF, FF, FF, "rms", None, None, False)
    total, normed = mok.mok_block_join(d["x"], before="rms", before_weight=rule["before_weight"], dtype=BF)
    assert total is d["x"] and normed.dtype == BF
    _, _, want, bound = ref.forward_bounds(d["x"].double(), None, 0.0, half(BF), before="rms", before_weight=rule["before_weight"].double())
    near(normed, want, bound, "normed")
    got = mok.mok_block_join_backward(None, d["d_normed"], d["x"], before="rms", before_weight=rule["before_weight"])
    want, bound = ref.backward_bounds(None, d["d_normed"].double(), d["x"].double(), None, half(FF), half(BF), before="rms",
                                      before_weight=rule["before_weight"].double())
    assert got[0].dtype == FF and got[1] is None and got[2] is None
    near(got[0], want[0], bound[0], "dx")
    near(got[3], want[3], bound[3], "dbefore_weight")


def test_in_place(mok):
    """sum over x and normed over y, through the C entry point."""
    import ctypes
    from paper_2609_36070_b200 import build
    lib = ctypes.CDLL(build.LIB)
    d, rule = make(5, 650, 1024, BF, BF, FF, "rms", "rms", None, False)
    ref_sum, ref_normed = mok.mok_block_join(d["x"], d["y"], **rule)
    x, y = d["x"].clone(), d["y"].clone()
    from test_join_abi import Join
    a = Join(x=x.data_ptr(), y=y.data_ptr(), before_weight=rule["before_weight"].data_ptr(), after_weight=rule["after_weight"].data_ptr(), x_stride=1024,
             y_stride=1024, sum_stride=1024, normed_stride=1024, T=650, H=1024, type=0, x_type=0, vector_type=2, before=1, after=1, scale=1.0, eps=1e-6,
             sum=x.data_ptr(), normed=y.data_ptr(), stream=torch.cuda.current_stream().cuda_stream)
    assert lib.mok_block_join(ctypes.byref(a)) == 0
    assert torch.equal(x, ref_sum) and torch.equal(y, ref_normed)


def test_no_rows(mok):
    x, w = torch.empty(0, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda")
    total, normed = mok.mok_block_join(x, x, before="rms", before_weight=w)
    assert total.shape == normed.shape == (0, 64)
    got = mok.mok_block_join_backward(x, x, x, x, before="rms", before_weight=w)
    assert got[0].shape == (0, 64) and (got[3] == 0).all()


def test_capture_replay_and_streams(mok):
    """A captured step reads its seed from the device: every replay drops other elements, and the gradient finds the same."""
    d, rule = make(6, 300, 512, BF, BF, FF, "rms", "rms", None, False)
    seed = torch.tensor([11, 0], device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mok.mok_block_join(d["x"], d["y"], **rule, p=0.5, seed=seed)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        total, normed = mok.mok_block_join(d["x"], d["y"], **rule, p=0.5, seed=seed)
        back = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, p=0.5, seed=seed)
        seed[1] += 1
    for i in range(3):
        g.replay()
        want = mok.mok_block_join(d["x"], d["y"], **rule, p=0.5, seed=11, offset=i)
        assert torch.equal(total, want[0]) and torch.equal(normed, want[1])
        for a, b in zip(back, mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, p=0.5, seed=11, offset=i)):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, p=0.5, seed=11, offset=2, stream=s) for s in streams * 4]
    torch.cuda.synchronize()
    for o in outs:
        for a, b in zip(o, back):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))


def test_offsets_past_32_bits(mok):
    """Rows that lie more than 2^31 elements into their buffers."""
    T, H = 300000, 7168
    x = torch.zeros(T, H, device="cuda", dtype=BF)
    x[-1], x[0] = 2.0, 1.0
    total, normed = mok.mok_block_join(x, x, before="rms")
    assert (total[-1] == 4).all() and (total[0] == 2).all() and (normed[-1] == 1).all() and total[1:-1].abs().max() == 0
    del normed
    dx, dy, *_ = mok.mok_block_join_backward(x, x, total, x, before="rms")
    assert torch.equal(dx, dy) and dx[-1].float().sub(2).abs().max() < 1e-2


@pytest.mark.parametrize("T", [40, 700])
@pytest.mark.parametrize("H", [264, 1032, 1031, 2056])
def test_an_infinite_weight_stays_in_its_column(mok, H, T):
    """The last threads of a row hold pieces past its end, which multiply zeros with the weight: they may not reach the statistics."""
    d, rule = make(7, T, H, BF, FF, FF, "rms", "rms", None, False)
    rule["after_weight"][0] = float("inf")
    total, normed = mok.mok_block_join(d["x"], d["y"], **rule)
    assert total[:, 0].isinf().all() and torch.isfinite(total[:, 1:]).all()
    assert normed[:, 0].isnan().all() and (normed[:, 1:] == 0).all()             # 1 / sqrt(inf) = 0


@pytest.mark.parametrize("T", [3, 150])
def test_the_widest_rows_with_every_vector(mok, T):
    """fp32 rows of the largest width with both biases and a channel gate: more than shared memory holds, so rows are read in place."""
    d, rule = make(8, T, 8192, FF, FF, FF, "layer", "layer", "channel", True)
    check(mok, d, rule, scale=0.5, p=0.25, seed=5)


def test_two_graphs_share_a_workspace(mok):
    """Backward passes of different sizes, captured with one workspace and replayed in turn."""
    sets = [make(s, T, H, BF, BF, FF, "rms", "layer", "channel", True) for s, T, H in ((1, 700, 512), (2, 90, 2048), (3, 1, 64))]
    ws = torch.empty(max(mok.mok_join_bwd_workspace_bytes(*d["y"].shape) for d, _ in sets) + 256, dtype=torch.uint8, device="cuda")
    calls = []
    for d, rule in sets:
        total, _ = mok.mok_block_join(d["x"], d["y"], **rule)
        want = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule, workspace=ws)
        calls.append((g, got, want, total))
    for i in (0, 1, 2, 1, 0, 2, 0):
        g, got, want, _ = calls[i]
        for t in got:
            t.zero_()
        g.replay()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_results_that_are_not_wanted_and_rows_between_others(mok):
    """Through the C entry point: any of the results may be left out, and rows of wider buffers leave the columns beside them alone."""
    import ctypes
    from paper_2609_36070_b200 import build
    from test_join_abi import Join, JoinBackward
    lib = ctypes.CDLL(build.LIB)
    T, H = 200, 520
    d, rule = make(9, T, H, BF, BF, FF, "rms", "layer", "full", True)
    total, _ = mok.mok_block_join(d["x"], d["y"], **rule)
    want = mok.mok_block_join_backward(d["d_sum"], d["d_normed"], total, d["y"], **rule)
    ws = torch.empty(mok.mok_join_bwd_workspace_bytes(T, H) + 256, dtype=torch.uint8, device="cuda")
    at = lambda t: t.data_ptr()
    forward = Join(x=at(total), y=at(d["y"]), gate=at(rule["gate"]), before_weight=at(rule["before_weight"]), before_bias=at(rule["before_bias"]),
                   after_weight=at(rule["after_weight"]), after_bias=at(rule["after_bias"]), x_stride=H, y_stride=H, gate_stride=H, T=T, H=H, type=0, x_type=0,
                   vector_type=2, before=1, after=2, gate_kind=3, scale=1.0, eps=1e-6)
    names = ("dx", "dy", "dgate", "d_before_weight", "d_before_bias", "d_after_weight", "d_after_bias")
    for wanted in (names[:1], names[1:2], names[2:3], names[3:4], names[5:], names[:2] + names[6:], ()):
        for pad in (0, 24, 3):
            buffers = {n: torch.full((T, H + pad), 7.0, device="cuda", dtype=BF) if n in names[:3] else torch.full((H,), 7.0, device="cuda") for n in wanted}
            b = JoinBackward(forward=forward, d_sum=at(d["d_sum"]), d_normed=at(d["d_normed"]), d_sum_stride=H, d_normed_stride=H, dx_stride=H + pad,
                             dy_stride=H + pad, dgate_stride=H + pad, workspace=at(ws) + -at(ws) % 256, workspace_bytes=ws.numel() - 256,
                             stream=torch.cuda.current_stream().cuda_stream, **{n: at(t) for n, t in buffers.items()})
            assert lib.mok_block_join_backward(ctypes.byref(b)) == 0
            for n, t in buffers.items():
                i = names.index(n)
                got = t[:, :H] if i < 3 else t
                # unaligned rows are added up in another order.  A rounded result moves by a step at most, 2^-7 of it, and by what the sums over
                # a row differ, below 1e-4; sums over the rows by twice (T + 170) 2^-24 of their magnitudes, which are below 1.5 T
                atol = 1e-4 if i < 3 else 2 * (T + 170) * 2.0 ** -24 * 1.5 * T
                assert torch.equal(got, want[i]) or pad == 3 and torch.allclose(got.float(), want[i].float(), rtol=2.0 ** -7, atol=atol), (n, pad)
                assert i >= 3 or (t[:, H:] == 7).all()


@pytest.mark.parametrize("dtype,stream", [(BF, BF), (HF, FF)])
@pytest.mark.parametrize("before,after,gate,shift,p", [("rms", "rms", "token", False, 0.0), ("layer", "layer", "full", True, 0.1), ("rms", None, "channel", True, 0.0)])
@pytest.mark.parametrize("T,H", [(4000, 264), (3000, 512), (2500, 520), (2300, 768), (1500, 1152), (1300, 1536), (900, 2304), (700, 3584), (700, 3592), (650, 4096), (650, 4095),
                                 (600, 5760), (40, 4096), (5, 512), (300, 512), (3000, 511)])
def test_widths_where_the_shape_of_a_block_changes(mok, T, H, before, after, gate, shift, p, dtype, stream):
    d, rule = make(T * H, T, H, dtype, stream, FF, before, after, gate, shift)
    check(mok, d, rule, scale=0.5, p=p, seed=21)


@pytest.mark.parametrize("dtype,stream,vectors", [(BF, BF, FF), (HF, FF, HF), (FF, FF, BF)])
@pytest.mark.parametrize("before,after,gate,shift", [("rms", "rms", None, False), ("rms", None, None, False), ("layer", "rms", "full", True),
                                                     ("layer", "layer", "channel", True), (None, "layer", "token", False)])
@pytest.mark.parametrize("T,H,pad", [(2, 1, 0), (9, 3, 4), (700, 9, 0), (3000, 15, 2), (5000, 33, 0), (1, 250, 1), (9, 249, 0), (2500, 242, 0), (600, 256, 1),
                                     (601, 512, 6), (3000, 505, 0), (3000, 506, 0), (333, 1022, 0), (1500, 2049, 0), (40, 7161, 0), (40, 7162, 0), (300, 8185, 0), (20, 8186, 0), (300, 4100, 3)])
def test_rows_that_begin_anywhere(mok, T, H, pad, before, after, gate, shift, dtype, stream, vectors):
    """Rows of any width, one behind the other or `pad` elements apart, in buffers that lie on 256 bytes."""
    d, rule = make(T + H, T, H + pad, dtype, stream, vectors, before, after, gate, shift)
    d = {k: None if v is None else v[:, :H] for k, v in d.items()}
    rule = {k: v[:, :H] if torch.is_tensor(v) and v.dim() == 2 and v.shape[1] > 1 else v[:H].clone() if torch.is_tensor(v) and v.dim() == 1 else v
            for k, v in rule.items()}
    check(mok, d, rule, scale=0.5, p=0.0 if gate is None else 0.25, seed=9, offset=1 << 33)


@pytest.mark.parametrize("before,after", [("rms", "rms"), ("rms", None), (None, "rms"), ("layer", "rms"), ("layer", "layer")])
@pytest.mark.parametrize("T,H", [(1, 2047), (5, 264), (40, 1025), (700, 520), (601, 2047), (333, 2880), (300, 505), (200, 8185), (150, 8192)])
@pytest.mark.parametrize("stream", [BF, FF])
def test_gradients_of_biases_that_are_not_there(mok, T, H, before, after, stream):
    """Through the C entry point: a NULL bias stands for zeros, and has a gradient like any other; with every other result, and alone."""
    import ctypes
    from paper_2609_36070_b200 import build
    from test_join_abi import Join, JoinBackward
    lib = ctypes.CDLL(build.LIB)
    d, rule = make(T + H, T, H, BF, stream, FF, before, after, None, False)
    zeros = {n + "_bias": torch.zeros(H, device="cuda") for n, norm in (("before", before), ("after", after)) if norm}
    want, bound = ref.backward_bounds(d["d_sum"].double(), None if before is None else d["d_normed"].double(), d["x"].double(), d["y"].double(), half(stream),
                                      half(BF), **wide({**rule, **zeros}))
    names = ("dx", "dy", "dgate", "d_before_weight", "d_before_bias", "d_after_weight", "d_after_bias")
    there = [n for n, w in zip(names, want) if w is not None]
    kinds = {None: 0, "rms": 1, "layer": 2}
    at = lambda t: None if t is None else t.data_ptr()
    forward = Join(x=at(d["x"]), y=at(d["y"]), before_weight=at(rule["before_weight"]), after_weight=at(rule["after_weight"]), x_stride=H, y_stride=H, T=T,
                   H=H, type=0, x_type=2 if stream == FF else 0, vector_type=2, before=kinds[before], after=kinds[after], scale=1.0, eps=1e-6)
    need = mok.mok_join_bwd_workspace_bytes(T, H)
    ws = torch.full((need + 512,), 0x5A, device="cuda", dtype=torch.uint8)
    first = -ws.data_ptr() % 256
    for wanted in (there, [n for n in there if n.endswith("bias")]):
        outs = {n: torch.full((T, H) if n in ("dx", "dy") else (H,), float("nan"), device="cuda", dtype={"dx": stream, "dy": BF}.get(n, FF)) for n in wanted}
        b = JoinBackward(forward=forward, d_sum=at(d["d_sum"]), d_normed=at(d["d_normed"]), d_sum_stride=H, d_normed_stride=H, dx_stride=H, dy_stride=H,
                         workspace=ws.data_ptr() + first, workspace_bytes=need, stream=torch.cuda.current_stream().cuda_stream,
                         **{n: at(t) for n, t in outs.items()})
        assert lib.mok_block_join_backward(ctypes.byref(b)) == 0
        for n, t in outs.items():
            near(t, want[names.index(n)], bound[names.index(n)], n)
        assert (ws[:first] == 0x5A).all() and (ws[first + need:] == 0x5A).all()


@pytest.mark.parametrize("before,after,gate,shift", [("rms", "rms", None, False), ("layer", "layer", "full", True)])
@pytest.mark.parametrize("H", [520, 2047, 4096])
def test_numbers_of_rows_where_the_code_changes(mok, H, before, after, gate, shift):
    """592 rows and one more run in other code: both are held to the bound, and a row's bits stay while only the others' contents change."""
    d, rule = make(H, 593, H, BF, BF, FF, before, after, gate, shift)
    for T in (592, 593):
        part = {k: v[:T] for k, v in d.items()}
        some = {k: v[:T] if k == "gate" and v is not None else v for k, v in rule.items()}
        total, normed = check(mok, part, some, scale=0.5)
        others = torch.ones(T, dtype=torch.bool, device="cuda")
        others[::7] = False
        new = {k: torch.where(others[:, None], v.flip(0), v) for k, v in part.items()}
        if gate:
            some["gate"] = torch.where(others[:, None], some["gate"].flip(0), some["gate"])
        again = mok.mok_block_join(new["x"], new["y"], **some, scale=0.5)
        assert torch.equal(again[0][~others], total[~others]) and torch.equal(again[1][~others], normed[~others])
