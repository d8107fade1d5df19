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
