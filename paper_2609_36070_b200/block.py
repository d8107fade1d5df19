"""A block of a network around the expert layer: norm, layer, norm, gate, dropout and residual.

The residual stream x and the layer's input `normed` go from block to block:

    y = layer(normed);   x, normed = x + scale * drop(gate * norm_after(y)), norm_before_of_the_next_block(x)

`ExpertBlock` runs the layer as `mok_moe_few` for up to 64 tokens (a decoding step: one launch) and as `mok_moe_forward_ex` above,
and everything between two layers as one `mok_block_join`.  `ExpertBlock.backward` is the training side: the gradients of the join,
of the layer (`mok_moe_backward`, which recomputes its activations) and of the router.  All of it is outside of autograd.

    python -m paper_2609_36070_b200.block --config qwen3_30b_a3b --tokens 16 --blocks 4

times a stack of blocks, forwards and (--train) backwards.
"""
import argparse

import torch

from . import mok
from .int8_layer import router_gradients


class Saved:
    """What the backward pass of a block needs of its forward pass."""
    __slots__ = ("normed", "y", "sum", "topk_idx", "topk_w", "seed", "offset")

    def __init__(self, **fields):
        for name in self.__slots__:
            setattr(self, name, fields[name])


def _check_weight(name, t, shape, dtype, device):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor {list(shape)} of {dtype} on {device}, got shape {list(t.shape)}, strides "
                         f"{list(t.stride())}, {t.dtype} on {t.device}")


class ExpertBlock:
    """W_router fp32 [E, H], W_gate_up bf16 [E, 2I, H], W_down bf16 [E, H, I], shared [2 I_s, H] and [H, I_s] or None.  (The experts may be
    fp16 where up to 64 tokens are all that the block is called with, forwards.)

    after, after_weight, after_bias: the norm of the layer's output; gate, scale, p: how it is added to the residual stream;
    before, before_weight, before_bias: the norm in front of the NEXT block's layer (all of them as in `mok_block_join`)."""

    def __init__(self, W_router, W_gate_up, W_down, W_shared_gate_up=None, W_shared_down=None, *, k, router_bias=None, before="rms",
                 before_weight=None, before_bias=None, after=None, after_weight=None, after_bias=None, gate=None, scale=1.0, eps=1e-6, p=0.0):
        self.W_router, self.router_bias, self.k = W_router, router_bias, k
        self.experts = (W_gate_up, W_down, W_shared_gate_up, W_shared_down)
        if W_gate_up.dim() != 3 or W_gate_up.dtype not in (torch.bfloat16, torch.float16):
            raise ValueError(f"W_gate_up: expected [E, 2I, H] of bfloat16, got shape {list(W_gate_up.shape)} of {W_gate_up.dtype}")
        if (W_shared_gate_up is None) != (W_shared_down is None):
            raise ValueError("W_shared_gate_up, W_shared_down: expected both or neither")
        _, H, I, I_s, E, _ = self.sizes(0)
        shapes = dict(W_gate_up=(E, 2 * I, H), W_down=(E, H, I), W_shared_gate_up=(2 * I_s, H), W_shared_down=(H, I_s))
        for (name, shape), t in zip(shapes.items(), self.experts):
            if t is not None:
                _check_weight(name, t, shape, W_gate_up.dtype, W_gate_up.device)
        _check_weight("W_router", W_router, (E, H), torch.float32, W_gate_up.device)
        if router_bias is not None:
            _check_weight("router_bias", router_bias, (E,), torch.float32, W_gate_up.device)
        self.rule = dict(before=before, before_weight=before_weight, before_bias=before_bias, after=after, after_weight=after_weight,
                         after_bias=after_bias, gate=gate, scale=scale, eps=eps, p=p)

    def sizes(self, T):
        W_gate_up, _, W_shared_gate_up, _ = self.experts
        E, two_i, H = W_gate_up.shape
        return T, H, two_i // 2, 0 if W_shared_gate_up is None else W_shared_gate_up.shape[0] // 2, E, self.k

    def workspace(self, T):
        """Scratch for calls of up to T tokens."""
        need = mok.mok_workspace_bytes(*self.sizes(T))
        few = mok.mok_few_workspace_bytes(*self.sizes(min(T, mok.MOK_FEW_MAX_TOKENS)))
        if need == 0 or few == 0:
            raise mok.MokError(mok.MOK_ERR_SHAPE)
        return torch.empty(max(need, few) + 256, dtype=torch.uint8, device=self.W_router.device)

    def check_input(self, normed, many):
        """many: for the layer of many tokens or the gradients, which read bf16 whatever they are given."""
        W = self.experts[0]
        if normed.dim() != 2 or normed.shape[1] != W.shape[2] or normed.dtype != W.dtype or normed.device != W.device:
            raise ValueError(f"normed: expected [T, {W.shape[2]}] of {W.dtype} on {W.device}, got shape {list(normed.shape)} of {normed.dtype} "
                             f"on {normed.device}")
        if many and W.dtype != torch.bfloat16:
            raise ValueError(f"more than {mok.MOK_FEW_MAX_TOKENS} tokens, and gradients, are for experts of bfloat16, these are of {W.dtype}")

    def layer(self, normed, workspace=None, routes=False):
        """The expert layer's output; with routes also topk_idx and topk_w."""
        self.check_input(normed, len(normed) > mok.MOK_FEW_MAX_TOKENS)
        if workspace is None:
            workspace = self.workspace(len(normed))
        if len(normed) <= mok.MOK_FEW_MAX_TOKENS:
            return mok.mok_moe_few(normed, self.W_router, self.router_bias, *self.experts, self.k, workspace, stages=routes)
        # (mok_moe_forward_ex takes rows one behind the other, and runs on the current device; mok_moe_few takes any, and finds theirs)
        with torch.cuda.device(normed.device):
            out = mok.mok_moe_forward_ex(normed.contiguous(), self.W_router, self.router_bias, *self.experts, self.k, workspace, stages=routes)
        return (out[0], out[1]["topk_idx"], out[1]["topk_w"]) if routes else out

    def __call__(self, x, normed, workspace=None, seed=0, offset=None, save=False):
        """(x, normed) for the next block, from this block's; with save also what `backward` needs.  seed, offset: of the dropout, integers
        (None: 0), or seed an int64 tensor [2] of both on the device and no offset."""
        y, idx, w = self.layer(normed, workspace, True) if save else (self.layer(normed, workspace), None, None)
        total, after = mok.mok_block_join(x, y, **self.rule, seed=seed, offset=offset)
        if not save:
            return total, after
        return total, after, Saved(normed=normed, y=y, sum=total, topk_idx=idx, topk_w=w, seed=seed, offset=offset)

    @torch.no_grad()
    def backward(self, saved, d_x, d_normed):
        """From the gradients of the block's two outputs (d_x may be None: 0) those of its two inputs and of its weights: (d_x, d_normed,
        {name: gradient}).  A seed tensor has to hold what it held in the forward pass."""
        self.check_input(saved.normed, True)
        d_sum, d_y, d_gate, *vectors = mok.mok_block_join_backward(d_x, d_normed, saved.sum, saved.y, **self.rule, seed=saved.seed,
                                                                   offset=saved.offset)
        with torch.cuda.device(saved.normed.device):
            g = mok.mok_moe_backward(saved.normed.contiguous(), *self.experts, saved.topk_idx, saved.topk_w, d_y)
        logits = saved.normed.float() @ self.W_router.t()
        if self.router_bias is not None:
            logits += self.router_bias
        d_router, d_in, d_logits = router_gradients(saved.normed, self.W_router, logits, saved.topk_idx, g["dw"])
        grads = {"W_router": d_router, "W_gate_up": g["dW_gate_up"], "W_down": g["dW_down"]}
        if self.router_bias is not None:
            grads["router_bias"] = d_logits.sum(0)
        if self.experts[2] is not None:
            grads["W_shared_gate_up"], grads["W_shared_down"] = g["dW_shared_gate_up"], g["dW_shared_down"]
        grads.update((n, v) for n, v in zip(("gate", "before_weight", "before_bias", "after_weight", "after_bias"), (d_gate, *vectors)) if v is not None)
        return d_sum, (g["dx"].float() + d_in).to(saved.normed.dtype), grads


def main():
    from . import inputs
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--config", default="tiny", choices=inputs.CONFIG_ORDER)
    ap.add_argument("--tokens", type=int, default=0, help="0: the configuration's")
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--train", action="store_true", help="forwards and backwards")
    a = ap.parse_args()
    cfg = inputs.CONFIGS[a.config]
    T = a.tokens or cfg.T
    g = torch.Generator(device="cuda").manual_seed(cfg.seed)

    def normal(*shape, std=0.02, dtype=torch.bfloat16):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    blocks = []
    for _ in range(a.blocks):
        shared = (normal(2 * cfg.I_s, cfg.H), normal(cfg.H, cfg.I_s)) if cfg.I_s else (None, None)
        blocks.append(ExpertBlock(normal(cfg.E, cfg.H, dtype=torch.float32), normal(cfg.E, 2 * cfg.I, cfg.H), normal(cfg.E, cfg.H, cfg.I), *shared,
                                  k=cfg.k, before_weight=torch.ones(cfg.H, device="cuda"), after="rms",
                                  after_weight=torch.ones(cfg.H, device="cuda"), scale=0.5, p=0.1 if a.train else 0.0))
    x, ws = normal(T, cfg.H, std=1.0), blocks[0].workspace(T)
    first = torch.ones(cfg.H, device="cuda")

    def step(i):
        total, normed = mok.mok_block_join(x, before="rms", before_weight=first)
        saved = []
        for n, b in enumerate(blocks):
            out = b(total, normed, ws, seed=n, offset=i, save=a.train)
            total, normed = out[:2]
            saved += out[2:]
        if a.train:
            d_x, d_normed = None, torch.ones_like(normed)
            for b, s in zip(blocks[::-1], saved[::-1]):
                d_x, d_normed, _ = b.backward(s, d_x, d_normed)
        return total

    for i in range(3):
        step(i)
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    begin.record()
    for i in range(a.steps):
        step(i)
    end.record()
    end.synchronize()
    assert mok.mok_read_status(ws) == mok.MOK_OK
    print(f"{a.config}: {T} tokens, {a.blocks} blocks, {'forwards and backwards' if a.train else 'forwards'}: "
          f"{begin.elapsed_time(end) / a.steps * 1e3:.1f} us per step")


if __name__ == "__main__":
    main()
