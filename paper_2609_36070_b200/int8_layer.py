"""An expert layer on 8-bit weights: routing from logits, routed experts and shared expert in 8-bit integers.

`Int8Layer` is the layer of `mok_moe_forward_ex` as a serving program with a quantised checkpoint runs it: the router's
projection, `mok_gate` (softmax or sigmoid scores, balance bias, groups, scaled weights), `mok_i8_experts` for the shared
expert (one expert that every token meets) and for the routed ones, whose combine adds the shared expert's output.
`router_gradients` is the training side of the same routing: from the router-weight gradient that `mok_moe_backward` returns
to the gradients of the router's weights and of its input.

    python -m paper_2609_36070_b200.int8_layer --config qwen3_30b_a3b --tokens 512

times the layer and says how far its output is from the bf16 layer on the same routes.
"""
import argparse

import torch

from . import mok


class Int8Layer:
    """W_router fp32 [E, H]; W_gate_up [E, 2I, H] (gate rows, then up rows), W_down [E, H, I], shared [2 I_s, H] and [H, I_s]
    in any floating-point type: quantised here, once, with a scale for each output channel."""

    def __init__(self, W_router, W_gate_up, W_down, W_shared_gate_up=None, W_shared_down=None, *, k, score="softmax", bias=None,
                 n_groups=1, topk_groups=1, group_top=2, renormalise=True, scale=1.0):
        self.W_router, self.bias = W_router, bias
        self.gate_up, self.down = mok.I8Weights.quantize(W_gate_up), mok.I8Weights.quantize(W_down)
        self.shared = None
        if W_shared_gate_up is not None:
            self.shared = mok.I8Weights.quantize(W_shared_gate_up[None]), mok.I8Weights.quantize(W_shared_down[None])
        self.k = k
        self.routing = dict(score=score, n_groups=n_groups, topk_groups=topk_groups, group_top=group_top,
                            renormalise=renormalise, scale=scale)

    def route(self, x):
        """(logits [T, E], topk_idx, topk_w) of the tokens x [T, H]."""
        logits = x.float() @ self.W_router.t()
        return (logits, *mok.mok_gate(logits, self.k, bias=self.bias, **self.routing))

    def __call__(self, x, workspace=None):
        """out [T, H] of x (bf16 or fp16); workspace: from `workspace`, kept between calls."""
        _, idx, w = self.route(x)
        add = None
        if self.shared is not None:
            everyone = torch.zeros((len(x), 1), dtype=torch.int32, device=x.device)
            add = mok.mok_i8_experts(x, everyone, torch.ones((len(x), 1), device=x.device), *self.shared, workspace=workspace)
        return mok.mok_i8_experts(x, idx, w, self.gate_up, self.down, add=add, workspace=workspace)

    def workspace(self, T):
        """Scratch for calls of up to T tokens."""
        E, two_i, _ = self.gate_up.codes.shape
        H = self.down.codes.shape[1]
        need = [mok.mok_i8_experts_workspace_bytes(T, H, two_i // 2, E, self.k)]
        if self.shared is not None:
            need.append(mok.mok_i8_experts_workspace_bytes(T, H, self.shared[0].codes.shape[1] // 2, 1, 1))
        return torch.empty(max(need) + 256, dtype=torch.uint8, device=self.gate_up.codes.device)


def router_gradients(x, W_router, logits, topk_idx, dw, *, score="softmax", renormalise=True, scale=1.0):
    """(dW_router [E, H], dx [T, H] through the router, dlogits [T, E]) from dL/dtopk_w, all fp32 for fp32 logits."""
    d = mok.mok_gate_backward(logits, topk_idx, dw, score=score, renormalise=renormalise, scale=scale)
    return d.t() @ x.to(d.dtype), d @ W_router.to(d.dtype), d


def main():
    from . import inputs
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="tiny", choices=inputs.CONFIG_ORDER)
    ap.add_argument("--tokens", type=int, default=0, help="0: the configuration's")
    ap.add_argument("--steps", type=int, default=20)
    a = ap.parse_args()
    cfg = inputs.CONFIGS[a.config]
    T = a.tokens or cfg.T
    g = torch.Generator(device="cuda").manual_seed(cfg.seed)

    def normal(*shape, std=0.02):
        return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()

    x, W_r = normal(T, cfg.H, std=1.0), torch.randn(cfg.E, cfg.H, generator=g, device="cuda") * 0.02
    W_gu, W_d = normal(cfg.E, 2 * cfg.I, cfg.H), normal(cfg.E, cfg.H, cfg.I)
    W_sgu, W_sd = (normal(2 * cfg.I_s, cfg.H), normal(cfg.H, cfg.I_s)) if cfg.I_s else (None, None)
    layer = Int8Layer(W_r, W_gu, W_d, W_sgu, W_sd, k=cfg.k)
    ws = layer.workspace(T)
    for _ in range(3):
        out = layer(x, ws)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for _ in range(a.steps):
        out = layer(x, ws)
    end.record()
    end.synchronize()
    assert mok.mok_i8_status() == mok.MOK_OK
    ref = mok.mok_moe_forward(x, W_r, W_gu, W_d, W_sgu, W_sd, cfg.k)
    far = ((out.float() - ref.float()).norm() / ref.float().norm()).item()
    print(f"{a.config}: {T} tokens, {begin.elapsed_time(end) / a.steps * 1e3:.1f} us per call, "
          f"{far:.4f} from the bf16 layer (2-norm)")


if __name__ == "__main__":
    main()
