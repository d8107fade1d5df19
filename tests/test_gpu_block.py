"""Blocks around the expert layer, as a network runs them: a stack forwards for few and for many tokens, its gradients against
autograd in 64 bits, a captured decoding step, and the 8-bit layer in the same place."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def stack(seed, T, H=256, I=128, I_s=64, E=8, k=2, n=2, p=0.0, bias=True):
    from paper_2609_36070_b200.block import ExpertBlock
    g = gen(seed)
    def r(*s, std=1.0, dtype=BF):
        return (torch.randn(*s, generator=g, device="cuda") * std).to(dtype)
    blocks = []
    for _ in range(n):
        blocks.append(ExpertBlock(r(E, H, std=H ** -0.5, dtype=torch.float32), r(E, 2 * I, H, std=H ** -0.5), r(E, H, I, std=I ** -0.5),
                                  r(2 * I_s, H, std=H ** -0.5), r(H, I_s, std=I_s ** -0.5), k=k, router_bias=r(E, std=0.1, dtype=torch.float32) if bias else None,
                                  before="rms", before_weight=1 + r(H, std=0.1, dtype=torch.float32), after="layer",
                                  after_weight=1 + r(H, std=0.1, dtype=torch.float32), after_bias=r(H, std=0.1, dtype=torch.float32),
                                  gate=0.5 + r(H, std=0.1, dtype=torch.float32), scale=0.7, p=p))
    return blocks, r(T, H), r(T, H)


def layer64(b, normed, idx, w):
    W_gu, W_d, W_sgu, W_sd = b["experts"]
    def ffn(x, gu, dn):
        gate, up = (x @ gu.t()).chunk(2, -1)
        return (torch.nn.functional.silu(gate) * up) @ dn.t()
    rows = [ffn(normed, W_sgu, W_sd)]
    for e in range(W_gu.shape[0]):
        share = (w * (idx == e)).sum(-1, keepdim=True)
        rows.append(share * ffn(normed, W_gu[e], W_d[e]))
    return sum(rows)


def run64(blocks, leaves, x, normed, saved, masks, p):
    """The same stack in 64 bits on the routes that were taken; leaves: per block the weights in 64 bits."""
    import join_reference as ref
    for b, l, s, m in zip(blocks, leaves, saved, masks):
        logits = normed @ l["W_router"].t() + l["router_bias"]
        idx = s.topk_idx.long()
        w = torch.softmax(logits.gather(1, idx), -1)
        y = layer64(l, normed, idx, w)
        x, normed = ref.join(x, y, "rms", l["before_weight"], None, "layer", l["after_weight"], l["after_bias"], l["gate"], 0.7, 1e-6, m, p)
    return x, normed


@pytest.mark.parametrize("T,p", [(1, 0.0), (16, 0.0), (64, 0.2), (200, 0.0), (333, 0.2)])
def test_stack_forwards_and_backwards(T, p):
    import join_reference as ref
    from paper_2609_36070_b200 import mok
    blocks, x, normed = stack(T, T, p=p)
    total, out, saved = x, normed, []
    for i, b in enumerate(blocks):
        total, out, s = b(total, out, seed=9, offset=i, save=True)
        saved.append(s)
    masks = [ref.kept(T, x.shape[1], p, 9, i, "cuda") if p else None for i in range(len(blocks))]
    leaves = [{**{n: getattr(b, n).double().requires_grad_() for n in ("W_router", "router_bias")},
               **{n: b.rule[n].double().requires_grad_() for n in ("before_weight", "after_weight", "after_bias", "gate")},
               "experts": [w.double().requires_grad_() for w in b.experts]} for b in blocks]
    x64, n64 = x.double().requires_grad_(), normed.double().requires_grad_()
    want, want_n = run64(blocks, leaves, x64, n64, saved, masks, p)
    # bf16 roundings on the way through two blocks: h, the rows, y, the sum, normed; each half a step (2^-9 of a value on average less),
    # about ten of them in the 2-norm
    tol = 10 * 2.0 ** -8
    assert (total.double() - want).norm() <= tol * want.norm() and (out.double() - want_n).norm() <= tol * want_n.norm()
    d_x, d_n = (torch.randn(T, x.shape[1], generator=gen(5), device="cuda").to(BF) for _ in range(2))
    names = ["W_router", "router_bias", "before_weight", "after_weight", "after_bias", "gate"]
    grads = torch.autograd.grad([want, want_n], [x64, n64] + [l[n] for l in leaves for n in names] + [w for l in leaves for w in l["experts"]],
                                [d_x.double(), d_n.double()])
    got = []
    dx, dn = d_x, d_n
    for b, s in zip(blocks[::-1], saved[::-1]):
        dx, dn, g = b.backward(s, dx, dn)
        got.insert(0, g)
    flat = [dx, dn] + [g[n] for g in got for n in names] + [g[n] for g in got for n in ("W_gate_up", "W_down", "W_shared_gate_up", "W_shared_down")]
    for i, (a, want) in enumerate(zip(flat, grads)):
        # gradients pass the same roundings again, backwards; the router's are differences of nearly equal numbers, a few times larger
        scale = 4 if i >= 2 and (i - 2) % len(names) < 2 and i < 2 + len(names) * len(blocks) else 1
        assert (a.double() - want).norm() <= scale * 2.5 * tol * want.norm() + 1e-9, i


def test_a_decoding_step_in_a_graph():
    from paper_2609_36070_b200 import mok
    blocks, x, normed = stack(3, 16, n=3)
    ws = blocks[0].workspace(16)
    def step():
        total, out = x, normed
        for b in blocks:
            total, out = b(total, out, ws)
        return total, out
    want = step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for seed in (1, 2):
        x.copy_(torch.randn(16, 256, generator=gen(seed), device="cuda"))
        graph.replay()
        want = step()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and mok.mok_read_status(ws) == 0


def test_few_and_many_tokens_agree():
    """The 64 tokens of the one-launch layer beside the same tokens through the layer for many: each rounds h and its output to bf16."""
    blocks, x, normed = stack(4, 65, n=1)
    few, many = blocks[0].layer(normed[:64]), blocks[0].layer(normed)[:64]
    assert (few.double() - many.double()).norm() <= 4 * 2.0 ** -8 * many.double().norm()


def test_the_8_bit_layer_in_a_block():
    from paper_2609_36070_b200 import mok
    from paper_2609_36070_b200.int8_layer import Int8Layer
    g = gen(6)
    W = [torch.randn(*s, generator=g, device="cuda") * 0.05 for s in ((8, 256, 128), (8, 128, 128))]
    layer = Int8Layer(torch.randn(8, 128, generator=g, device="cuda"), *W, k=2)
    x = torch.randn(20, 128, generator=g, device="cuda")
    normed = torch.randn(20, 128, generator=g, device="cuda").to(BF)
    got = layer.block(x, normed, before="rms", after="layer", scale=0.5)
    want = mok.mok_block_join(x, layer(normed), before="rms", after="layer", scale=0.5)
    assert got[0].dtype == torch.float32 and got[1].dtype == BF and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("train", [False, True])
def test_command(train):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    cmd = [sys.executable, "-m", "paper_2609_36070_b200.block", "--config", "tiny", "--tokens", "32", "--steps", "3"] + (["--train"] if train else [])
    done = subprocess.run(cmd, cwd=root, capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]
    assert "us per step" in done.stdout


@pytest.mark.parametrize("T", [20, 100])
def test_rows_of_wider_buffers(T):
    """The layer's input as columns of a wider buffer: the same as in rows of its own, in both layers and in the gradients."""
    blocks, x, normed = stack(7, T, n=1)
    wide = torch.full((T, 256 + 40), 3.0, device="cuda", dtype=BF)
    wide[:, 8:8 + 256] = normed
    d_x, d_n = (torch.randn(T, 256, generator=gen(s), device="cuda").to(BF) for s in (1, 2))
    results = []
    for n in (normed, wide[:, 8:8 + 256]):
        total, out, saved = blocks[0](x, n, save=True)
        dx, dn, g = blocks[0].backward(saved, d_x, d_n)
        results.append([total, out, dx, dn] + [g[k] for k in sorted(g)])
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("T", [20, 100])
def test_types_that_the_layer_does_not_take(T):
    """They are refused for any number of tokens: the layer for many tokens reads bf16 whatever it is given."""
    from paper_2609_36070_b200.block import ExpertBlock
    blocks, x, normed = stack(7, T, n=1)
    b = blocks[0]
    for bad in (normed.float(), normed.half(), normed[:, :128], normed[0], normed.cpu()):
        with pytest.raises(ValueError):
            b(x, bad)
    half = ExpertBlock(b.W_router, *(w.half() for w in b.experts), k=2, before="rms")
    if T > 64:
        with pytest.raises(ValueError):
            half(x.half(), normed.half())
    else:
        _, _, saved = half(x.half(), normed.half(), save=True)
        with pytest.raises(ValueError):
            half.backward(saved, None, normed.half())


@pytest.mark.parametrize("T", [10, 70])
def test_a_seed_on_the_device(T):
    """Seed and offset in a tensor: the mask of the same integers, other masks on the replays of a captured step, and gradients by the same."""
    blocks, x, normed = stack(8, T, n=1, p=0.3)
    b = blocks[0]
    want = b(x, normed, seed=5, offset=7, save=True)
    d_x, d_n = (torch.randn(T, 256, generator=gen(s), device="cuda").to(BF) for s in (1, 2))
    want_back = b.backward(want[2], d_x, d_n)
    seed = torch.tensor([5, 7], device="cuda")
    got = b(x, normed, seed=seed, save=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    back = b.backward(got[2], d_x, d_n)
    assert torch.equal(back[0], want_back[0]) and torch.equal(back[1], want_back[1])
    ws = b.workspace(T)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = b(x, normed, ws, seed=seed)
        seed[1] += 1
    for offset in (7, 8):
        graph.replay()
        assert torch.equal(got[0], b(x, normed, seed=5, offset=offset)[0])
    with pytest.raises(ValueError):
        b(x, normed, seed=seed, offset=3)


@pytest.mark.parametrize("T", [40, 200])
def test_gradients_of_the_router(T):
    """From the gradient of the routes' weights, which the layer's own tests hold, to those of the router: fp32 products of up to 256 terms
    after a softmax, so 1e-5 of the norm; and the input's, with a rounding to bf16 (2^-8 of each element at most)."""
    from paper_2609_36070_b200 import mok
    blocks, x, normed = stack(9, T, n=1)
    b = blocks[0]
    d_x, d_n = (torch.randn(T, 256, generator=gen(s), device="cuda").to(BF) for s in (1, 2))
    _, _, saved = b(x, normed, save=True)
    _, dn, grads = b.backward(saved, d_x, d_n)
    d_y = mok.mok_block_join_backward(d_x, d_n, saved.sum, saved.y, **b.rule)[1]
    g = mok.mok_moe_backward(saved.normed, *b.experts, saved.topk_idx, saved.topk_w, d_y)
    leaves = [t.double().requires_grad_() for t in (b.W_router, b.router_bias, saved.normed)]
    logits = leaves[2] @ leaves[0].t() + leaves[1]
    w = torch.softmax(logits.gather(1, saved.topk_idx.long()), -1)
    assert (w - saved.topk_w).abs().max() < 1e-5
    want = torch.autograd.grad(w, leaves, g["dw"].double())
    for name, ref in zip(("W_router", "router_bias"), want):
        assert (grads[name].double() - ref).norm() <= 1e-5 * ref.norm(), name
    ref = want[2] + g["dx"].double()
    assert (dn.double() - ref).norm() <= (2.0 ** -8 + 1e-5) * ref.norm()


def test_no_rows():
    """Gradients of an empty batch are zeros, also in memory that held something else."""
    from paper_2609_36070_b200 import mok
    blocks, x, normed = stack(10, 1, n=1, p=0.1)
    b, none = blocks[0], normed[:0]
    W = b.experts
    def poison():
        used = [torch.full(s, float("nan"), device="cuda", dtype=BF) for w in W for s in [w.shape] * 3]
        del used
    poison()
    total, out, saved = b(x[:0], none, save=True)
    dx, dn, grads = b.backward(saved, x[:0], none)
    assert total.shape == out.shape == dx.shape == dn.shape == (0, 256)
    names = {"W_router", "router_bias", "W_gate_up", "W_down", "W_shared_gate_up", "W_shared_down", "gate", "before_weight", "after_weight", "after_bias"}
    assert set(grads) == names and all((g == 0).all() for g in grads.values())
    poison()
    idx, w = torch.empty(1, 0, dtype=torch.int32, device="cuda"), torch.empty(1, 0, device="cuda")
    ws = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    grads = mok.mok_ep_expert_bwd(0, [0], [0], idx, w, *W, 8, 2, 256, none, idx, w, none, ws)
    assert len(grads) == 4 and all((g == 0).all() for g in grads.values())


@pytest.mark.parametrize("T", [10, 100])
def test_parameters(T):
    """Weights that require gradients: all of a block is outside of autograd, and its gradients hold no graph."""
    blocks, x, normed = stack(11, T, n=1)
    b = blocks[0]
    want = b.backward(b(x, normed, save=True)[2], x, normed)
    b.W_router, b.router_bias = torch.nn.Parameter(b.W_router), torch.nn.Parameter(b.router_bias)
    b.experts = tuple(torch.nn.Parameter(w) for w in b.experts)
    total, out, saved = b(x, normed, save=True)
    d_x, d_normed, grads = b.backward(saved, x, normed)
    assert not any(t.requires_grad for t in (total, out, d_x, d_normed, *grads.values()))
    assert torch.equal(d_x, want[0]) and torch.equal(d_normed, want[1]) and all(torch.equal(g, want[2][n]) for n, g in grads.items())


def test_a_training_step_in_a_graph():
    """Forwards and backwards of two blocks, captured: other masks on every replay, and the gradients of each."""
    blocks, x, normed = stack(12, 100, n=2, p=0.2)
    seed = torch.tensor([3, 0], device="cuda")
    def step():
        total, out, saved = x, normed, []
        for b in blocks:
            total, out, s = b(total, out, seed=seed, save=True)
            saved.append(s)
        d_x, d_n, grads = x, normed, []
        for b, s in zip(blocks[::-1], saved[::-1]):
            d_x, d_n, g = b.backward(s, d_x, d_n)
            grads += g.values()
        return [total, out, d_x, d_n, *grads]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for offset in (0, 1, 1 << 40):
        seed[1] = offset
        graph.replay()
        for a, b in zip(got, step()):
            assert torch.equal(a, b)
