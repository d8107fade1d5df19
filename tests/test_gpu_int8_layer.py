"""The 8-bit layer put together from routing, shared and routed experts, and the router's gradients, in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def codes64(x):
    x = x.double()
    amax = x.abs().amax(-1, keepdim=True)
    return (x * 127 / amax).round() * (amax / 127)


def dequantised(w, K):
    return w.codes[..., :K].double() * w.scales.double()[..., None]


def expert64(x, gu, dn):
    z = codes64(x) @ gu.t()
    g, u = z.chunk(2, -1)
    return codes64(torch.nn.functional.silu(g) * u) @ dn.t()


@pytest.mark.parametrize("T", [1, 7, 300])
@pytest.mark.parametrize("shared", [False, True])
def test_layer(T, shared):
    from paper_2609_36070_b200 import mok
    from paper_2609_36070_b200.int8_layer import Int8Layer
    g = gen(T)
    H, I, I_s, E, k = 256, 136, 200, 16, 3
    x = randn(g, T, H).bfloat16()
    W = [randn(g, *s) * 0.05 for s in ((E, 2 * I, H), (E, H, I), (2 * I_s, H), (H, I_s))]
    bias = randn(g, E) * 0.05
    layer = Int8Layer(randn(g, E, H) * 0.1, *W[:2], *(W[2:] if shared else (None, None)), k=k, score="sigmoid", bias=bias,
                      n_groups=4, topk_groups=2, scale=1.5)
    ws = layer.workspace(T)
    out = layer(x, ws)
    assert out.dtype == torch.bfloat16 and out.shape == (T, H)
    logits, idx, w = layer.route(x)
    s = torch.sigmoid(logits.double()).gather(1, idx.long())
    assert ((w.double() - 1.5 * s / s.sum(-1, keepdim=True)).abs() <= 1e-6).all()
    gu, dn = dequantised(layer.gate_up, H), dequantised(layer.down, I)
    ref = torch.zeros(T, H, dtype=torch.float64, device="cuda")
    if shared:
        ref += expert64(x, dequantised(layer.shared[0], H)[0], dequantised(layer.shared[1], I_s)[0])
    for t in range(T):
        for j in range(k):
            e = int(idx[t, j])
            ref[t] += w[t, j].double() * expert64(x[t:t + 1], gu[e], dn[e])[0]
    # two bf16 roundings (the shared expert's output is one of the sums' terms), fp16 rows, single codes of the activation
    assert (out.double() - ref).norm() <= (2 * 2.0 ** -8 + 2.0 ** -11) * ref.norm()
    assert torch.equal(out, layer(x)) and mok.mok_i8_status() == 0


@pytest.mark.parametrize("score,renorm", [("sigmoid", True), ("softmax", True), ("softmax", False)])
def test_router_gradients_follow_the_layers_backward(score, renorm):
    """dL/dW_router of L = sum(dout * layer(x)) through topk_w: the router-weight gradient of the layer's backward pass, then
    the routing's; against differences of L in the weights' direction, both sides through the bf16 expert layer."""
    from paper_2609_36070_b200 import mok
    from paper_2609_36070_b200.int8_layer import router_gradients
    g = gen(5)
    T, H, I, E, k = 64, 64, 64, 8, 2
    x, dout = randn(g, T, H).bfloat16(), randn(g, T, H).bfloat16()
    W_r = randn(g, E, H) * 0.2
    W_gu, W_d = (randn(g, E, 2 * I, H) * 0.1).bfloat16(), (randn(g, E, H, I) * 0.1).bfloat16()
    logits = x.float() @ W_r.t()
    idx, w = mok.mok_gate(logits, k, score=score, renormalise=renorm)
    dw = mok.mok_moe_backward(x, W_gu, W_d, None, None, idx, w, dout, weight_grads=False)["dw"]
    dW, dx, d = router_gradients(x, W_r, logits, idx, dw, score=score, renormalise=renorm)
    z = logits.double().requires_grad_()
    s = torch.sigmoid(z) if score == "sigmoid" else torch.softmax(z, -1)
    c = s.gather(1, idx.long())
    ref, = torch.autograd.grad(c / c.sum(-1, keepdim=True) if renorm else c, z, dw.double())
    room = 64 * 2.0 ** -24 * dw.abs().max().double()
    assert ((d.double() - ref).abs() <= 4 * 2.0 ** -24 * ref.abs() + room).all()
    assert (dW.double() - ref.t() @ x.double()).norm() <= 1e-5 * dW.double().norm()     # fp32 sums over 64 tokens
    assert (dx.double() - ref @ W_r.double()).norm() <= 1e-5 * dx.double().norm()
    # L is linear in the weights: dw is the expert outputs' inner product with dout (a bf16 evaluation of it)
    y = torch.zeros(T, k, dtype=torch.float64, device="cuda")
    for t in range(T):
        for j in range(k):
            e = int(idx[t, j])
            a, b = (W_gu[e].double() @ x[t].double()).chunk(2)
            y[t, j] = (W_d[e].double() @ (torch.nn.functional.silu(a) * b)) @ dout[t].double()
    assert (dw.double() - y).norm() <= 1e-2 * y.norm()
