"""Weights that a block does not take are refused when it is made (CPU): its two layers would read them as what they should be."""
import pytest
import torch


def weights(E=4, H=64, I=32, I_s=16, dtype=torch.bfloat16):
    return [torch.zeros(E, H)] + [torch.zeros(s, dtype=dtype) for s in ((E, 2 * I, H), (E, H, I), (2 * I_s, H), (H, I_s))]


def test_weights_are_checked():
    from paper_2609_36070_b200.block import ExpertBlock
    ExpertBlock(*weights(), k=2, router_bias=torch.zeros(4))
    ExpertBlock(*weights()[:3], k=2)
    ExpertBlock(*weights(dtype=torch.float16), k=2)
    for i, bad in ((0, torch.zeros(4, 64, dtype=torch.bfloat16)), (0, torch.zeros(4, 63)), (0, torch.zeros(64, 4).t()), (1, torch.zeros(4, 64, 64)),
                   (1, torch.zeros(4, 63, 64, dtype=torch.bfloat16)), (1, torch.zeros(64, 64, dtype=torch.bfloat16)),
                   (2, torch.zeros(4, 64, 32, dtype=torch.float16)), (2, torch.zeros(4, 64, 24, dtype=torch.bfloat16)),
                   (2, torch.zeros(4, 32, 64, dtype=torch.bfloat16).transpose(1, 2)), (3, torch.zeros(32, 64)), (3, None), (4, None),
                   (4, torch.zeros(16, 64, dtype=torch.bfloat16))):
        with pytest.raises(ValueError):
            ExpertBlock(*[bad if j == i else w for j, w in enumerate(weights())], k=2)
    for bad in (torch.zeros(4, dtype=torch.bfloat16), torch.zeros(3), torch.zeros(8)[::2]):
        with pytest.raises(ValueError):
            ExpertBlock(*weights(), k=2, router_bias=bad)


def test_the_layer_runs_on_its_tensors_device(monkeypatch):
    """The entry points for many tokens and for gradients launch on the current device, whichever holds the tensors: the block makes it theirs."""
    from paper_2609_36070_b200 import block, mok
    current, met = [], []

    class Device:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            current.append(self.device)

        def __exit__(self, *_):
            current.pop()

    def forward(x, *_, stages=False, **__):
        met.append(("forward", list(current)))
        return x, {"topk_idx": torch.zeros(len(x), 2, dtype=torch.int32), "topk_w": torch.zeros(len(x), 2)}

    def backward(x, *_, **__):
        met.append(("backward", list(current)))
        return {n: torch.zeros(1, 64) for n in ("dx", "dw", "dW_gate_up", "dW_down", "dW_shared_gate_up", "dW_shared_down")}

    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(mok, "mok_moe_forward_ex", forward)
    monkeypatch.setattr(mok, "mok_moe_backward", backward)
    monkeypatch.setattr(mok, "mok_block_join", lambda x, y, **_: (x, y))
    monkeypatch.setattr(mok, "mok_block_join_backward", lambda d_x, *_, **__: (d_x, d_x, None, None, None, None, None))
    monkeypatch.setattr(block, "router_gradients", lambda *_: (torch.zeros(4, 64), torch.zeros(1, 64), torch.zeros(1, 4)))
    b = block.ExpertBlock(*weights(), k=2)
    x = torch.zeros(65, 64, dtype=torch.bfloat16)
    _, _, saved = b(x, x, save=True)
    b.backward(saved, x, x)
    assert met == [("forward", [x.device]), ("backward", [x.device])]
