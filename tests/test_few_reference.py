"""The 64-bit form of the layer of a few tokens, by which its errors are judged in the 2-norm: it takes the two roundings to 16 bits, and
nothing that is off as a product without its last columns is.  CPU only."""
import pytest
import torch

import few_reference as ref
from test_gpu_few import SHAPES


def layer(seed, T, H, I, E, k, I_s, dtype):
    """The layer of test_gpu_few.py with at most 16 experts (which differ in nothing but their numbers), and random routes."""
    E = min(E, max(16, k))
    g = torch.Generator().manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g)
    d = {"x": randn(T, H).to(dtype), "gu": (randn(E, 2 * I, H) * H ** -0.5).to(dtype), "dn": (randn(E, H, I) * I ** -0.5).to(dtype), "sgu": None, "sdn": None}
    if I_s:
        d["sgu"], d["sdn"] = (randn(2 * I_s, H) * H ** -0.5).to(dtype), (randn(H, I_s) * I_s ** -0.5).to(dtype)
    idx = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    return d, idx, torch.softmax(randn(T, k), -1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("T,H,I,E,k,I_s", SHAPES)
def test_roundings_are_taken_and_lost_columns_are_not(T, H, I, E, k, I_s, dtype):
    d, idx, w = layer(T + H + I, T, H, I, E, k, I_s, dtype)
    want = ref.layer(d, idx, w)
    rows, together = ref.off(ref.layer(d, idx, w, roundings=True)[0], *want)
    assert rows <= 1 and together <= 1
    g = torch.Generator().manual_seed(5)
    for wrong in (ref.layer(d, idx, w, drop_H=8)[0], ref.layer(d, idx, w, drop_I=8)[0], 1.02 * want[0],
                  want[0] + 0.02 * torch.randn(T, H, generator=g, dtype=torch.float64) * want[0].norm() / (T * H) ** 0.5):
        assert max(ref.off(wrong, *want)) > 1
