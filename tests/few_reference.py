"""The layer of a few tokens in 64 bits, for the tests, with the errors in the 2-norm that its two roundings to 16 bits make.

The gated activation h and the output are rounded to the type, by at most u = eps / 2 relatively.  The rounding of an output moves a
row by at most u of its norm.  The roundings of h are independent and spread over +-u at most, so that each has a standard
deviation of at most u / sqrt(3): a row y = W_down h then moves by sqrt(sum_ij (W_ij h_j)^2) u / sqrt(3) on average over them, and by
four times that hardly ever.  (fp16 is spaced absolutely by 2^-24 below 2^-14: 2^-25 beside u |h_j|.)  fp32 arithmetic adds far less:
a term of a product passes through some tens of roundings of 2^-24 that are independent as well, 1e-6 of a row.
"""
import torch


def rounded(v, t):
    return v.to(t).double()


def layer(d, idx, w, add=None, roundings=False, drop_H=0, drop_I=0):
    """(out, rows, all) in 64 bits for routes idx, w; d: x, gu, dn, sgu, sdn.  rows: how far the roundings move each row of it, as a
    2-norm; all: all rows together, where the errors add up as squares and half as much again is allowed for their scatter.  roundings:
    with h and out rounded to the type; drop_H, drop_I: without the last columns of the first or the second product."""
    x, t = d["x"].double(), d["x"].dtype
    u, tiny = torch.finfo(t).eps / 2, 2.0 ** -25 if t == torch.float16 else 0.0
    out = torch.zeros_like(x) if add is None else add.double()
    var = torch.zeros(len(x), dtype=torch.float64, device=x.device)
    parts = [(torch.arange(len(x), device=x.device), None, d["sgu"], d["sdn"])] if d["sgu"] is not None else []
    for e in idx.unique().tolist():
        parts.append((*torch.nonzero(idx == e, as_tuple=True), d["gu"][e], d["dn"][e]))
    for tokens, slot, gate_up, down in parts:
        half, H, gate_up, down = len(gate_up) // 2, x.shape[1] - drop_H, gate_up.double(), down.double()
        rows = x[tokens][:, :H]
        h = torch.nn.functional.silu(rows @ gate_up[:half, :H].t()) * (rows @ gate_up[half:, :H].t())
        if roundings:
            h = rounded(h, t)
        I = half - drop_I
        share = torch.ones_like(x[tokens, :1]) if slot is None else w[tokens, slot].double()[:, None]
        out.index_add_(0, tokens, share * (h[:, :I] @ down[:, :I].t()))
        step = u * h.abs() + tiny
        var.index_add_(0, tokens, (share.square() * (step.square() @ down.square().sum(0)[:, None]))[:, 0] / 3)
    size = out.norm(dim=-1)
    last = u * size + tiny * x.shape[1] ** 0.5
    moved = last + 4 * var.sqrt() + 1e-5 * size, 1.5 * (last.square() / 3 + var).sum().sqrt() + 1e-5 * size.norm()
    return (rounded(out, t) if roundings else out, *moved)


def off(got, out, rows, all_rows):
    """How far `got` is from out beside what it may be: the worst row, and all rows together."""
    far = (got.double() - out).norm(dim=-1)
    return (far / rows).max().item(), (far.norm() / all_rows).item()
