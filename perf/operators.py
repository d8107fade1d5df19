"""Cases and plain forms of the routing and 8-bit operators of an expert layer.

Three operators, measured on the sizes that they meet in a serving or training program:

  gate           routing scores -> experts: softmax or sigmoid of the router's logits, a balance bias that only decides the
                 selection, expert groups, top-k, renormalised and scaled weights; and its gradient with respect to the logits
  i8 linear      out = quantise(x) W8^T, with one scale for each token (found in the call) and one for each output channel
  i8 experts     out[t] = sum_s w[t, s] f_{idx[t, s]}(x[t]),  f_e(x) = W_down_e (silu(W_gate_e x) .* (W_up_e x)), all three
                 products in 8-bit integers, x and the gated activation quantised for each token

`run` computes them with elementary torch operations in 32 bits (own = False) or calls the library (own = True).
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}


# ---------------------------------------------------------------------------------------------------------- cases

def _gate(name, T, E, k, score="sigmoid", groups=1, top_groups=1, group_top=2, bias=False, renorm=True, scale=1.0,
          dtype="f32", grad=False):
    return {"name": name, "op": "gate", "T": T, "E": E, "k": k, "score": score, "groups": groups, "top_groups": top_groups,
            "group_top": group_top, "bias": bias, "renorm": renorm, "scale": scale, "type": dtype, "grad": grad}


def _linear(name, M, K, N, dtype="bf16", out="bf16", bias=False, coded=False, pitch=0):
    return {"name": name, "op": "linear", "M": M, "K": K, "N": N, "type": dtype, "out": out, "bias": bias, "coded": coded,
            "pitch": pitch}


def _experts(name, T, H, I, E, k, dtype="bf16"):
    return {"name": name, "op": "experts", "T": T, "H": H, "I": I, "E": E, "k": k, "type": dtype}


def listed():
    return [
        # one decoding step of 16 sequences, group-limited sigmoid routing with a balance bias: pure latency
        _gate("gate decode", 16, 256, 8, groups=8, top_groups=4, bias=True, scale=2.5),
        # a long prompt batch through the same router
        _gate("gate prompt", 32768, 256, 8, groups=8, top_groups=4, bias=True, scale=2.5),
        # softmax routing of a training batch, logits as a 16-bit router produces them
        _gate("gate softmax bf16", 16384, 128, 8, score="softmax", dtype="bf16"),
        # an odd number of tokens and experts, weights left as the softmax gives them: the dense gradient
        _gate("gate gradient softmax", 8191, 60, 4, score="softmax", renorm=False, grad=True),
        # the training batch of the first router: only the chosen experts have a gradient
        _gate("gate gradient sigmoid", 32768, 256, 8, scale=2.5, grad=True),
        # one token through a shared expert's gate/up projection: reading the weights once is all there is
        _linear("linear one token", 1, 7168, 4096),
        # a decoding batch through the shared expert's down projection
        _linear("linear decode batch", 48, 2048, 7168),
        # an odd prompt through a projection whose width fills no tile, half precision in, 32 bits out, rows of a wider buffer
        _linear("linear ragged", 1003, 2880, 2880, dtype="f16", out="f32", bias=True, pitch=40),
        # a prompt batch through the gate/up projection, activations that are already 8-bit codes
        _linear("linear prompt codes", 8192, 7168, 4096, coded=True),
        # one decoding step of 16 sequences: most experts see one row, or none
        _experts("experts decode", 16, 2048, 768, 128, 8),
        # an odd chunk of a prompt on one of four devices' experts: about a hundred rows for each
        _experts("experts chunk", 777, 2880, 2880, 32, 4),
        # a prompt batch on every expert of the layer: about a thousand rows for each
        _experts("experts prompt", 16384, 2048, 768, 128, 8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A layer's width: multiples of 80 fill few tiles exactly, the others are the usual powers of two."""
    if rng.random() < 0.3:
        return 1 << rng.randint(int(math.log2(lo)) + 1, int(math.log2(hi)))
    return max(80, _log(rng, lo, hi) // 80 * 80)


def _case(c):
    return {key: v for key, v in c.items() if key != "name"}


def draw(rng):
    op = rng.choice(["gate", "gate", "linear", "linear", "experts"])
    if op == "gate":
        grad = rng.random() < 0.4
        E = rng.choice([8, 16, 60, 64, 72, 96, 128, 160, 256, 384, 512, rng.randint(9, 300)])
        T = min(_log(rng, 1, 65536), (32768 * 256) // E)
        divisors = [g for g in (2, 4, 8, 16) if E % g == 0 and E // g >= 2]
        groups, top_groups = 1, 1
        if divisors and not grad and rng.random() < 0.5:
            groups = rng.choice(divisors)
            top_groups = rng.randint(1, groups)
        k = rng.randint(1, max(1, min(16, top_groups * (E // groups) // 2)))
        return _case(_gate("", T, E, k, rng.choice(["sigmoid", "softmax"]), groups, top_groups, rng.choice([1, 2]),
                           not grad and rng.random() < 0.5, rng.random() < 0.7, rng.choice([1.0, 2.5]),
                           rng.choice(["f32", "f32", "bf16"]), grad))
    if op == "linear":
        M, K, N = _log(rng, 1, 16384), _width(rng, 256, 14336), _width(rng, 128, 16384)
        if M > 16 and rng.random() < 0.5:
            M |= 1
        most = 8192 * 7168 * 4096
        while M * K * N > most:
            M, N = max(1, M // 2), max(80, N // 160 * 80)
        pitch = rng.choice([0, 0, 8, 24])
        return _case(_linear("", M, K, N, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.choice(["bf16", "bf16", "f16", "f32"]),
                             rng.random() < 0.3, rng.random() < 0.3, pitch))
    T, H, I = _log(rng, 1, 16384), _width(rng, 256, 4096), _width(rng, 128, 4096)
    E = rng.choice([4, 8, 16, 32, 64, 128])
    k = rng.randint(1, min(8, E))
    while E * 3 * H * I > 128 * 3 * 2048 * 768:
        E = max(4, E // 2)
        k = min(k, E)
        if E == 4:
            H, I = max(80, H // 160 * 80), max(80, I // 160 * 80)
    while T * k * H * I > 16384 * 8 * 2048 * 768:
        T = max(1, T // 2)
    return _case(_experts("", T, H, I, E, k, rng.choice(["bf16", "bf16", "f16"])))


# --------------------------------------------------------------------------------------------------------- inputs

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)


def _draw_logits(case, g, offset, T):
    return (_normal(g, T, case["E"]) * 1.2 + offset).to(_TYPES[case["type"]])


def _close(case, logits, bias):
    """Tokens whose selection or order hangs on less than 3e-6 of a score: which expert such a token gets is decided by the
    last bits of an exponential, so that two right programs can differ there."""
    s = _scores64(case, logits)
    c = s if bias is None else s + bias.double()
    bad = torch.zeros(len(c), dtype=torch.bool, device=c.device)
    if case["groups"] > 1:
        value = c.view(len(c), case["groups"], -1).sort(-1, descending=True).values[..., :case["group_top"]].sum(-1)
        best = value.sort(-1, descending=True)
        if case["top_groups"] < case["groups"]:
            bad |= best.values[:, case["top_groups"] - 1] - best.values[:, case["top_groups"]] < 3e-6
        keep = torch.zeros_like(value, dtype=torch.bool).scatter_(1, best.indices[:, :case["top_groups"]], True)
        c = c.masked_fill(~keep.repeat_interleave(case["E"] // case["groups"], 1), -math.inf)
    top = c.sort(-1, descending=True).values[:, :case["k"] + 1]
    return bad | (top[:, :-1] - top[:, 1:] < 3e-6).any(-1)


def _routes(g, T, E, k):
    """Experts of every token as a router with some favourites gives them, and weights that sum to one."""
    value = _normal(g, T, E) + _normal(g, E) * 0.3
    top = value.topk(k, -1)
    return top.indices.int(), top.values.softmax(-1)


def _activations(g, rows, width, dtype, pitch=0):
    """Hidden states: normal, with a few channels that are much larger than the others."""
    x = _normal(g, rows, width + pitch) * torch.where(torch.rand(width + pitch, generator=g, device="cuda") < 0.01, 12.0, 1.0)
    return x.to(_TYPES[dtype])[:, :width]


def _weights(g, *shape):
    """8-bit weights as a checkpoint holds them: codes [.., N, K] in rows of whole 16 bytes, a scale for each channel, and the
    largest scale of each matrix."""
    K = shape[-1]
    codes = torch.zeros(*shape[:-1], (K + 15) // 16 * 16, dtype=torch.int8, device="cuda")
    codes[..., :K] = _normal(g, *shape).mul_(36).round_().clamp_(-127, 127)
    scales = (torch.rand(*shape[:-1], generator=g, device="cuda") + 0.5) * (0.02 / 36)
    return codes, scales, scales.amax(-1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    st = {"case": case}
    if case["op"] == "gate":
        offset = _normal(g, case["E"]) * 0.5
        # a bias as repeated steps of a fixed size leave it
        st["bias"] = (_normal(g, case["E"]) * 30).round() * 1e-3 if case["bias"] else None
        logits = _draw_logits(case, g, offset, case["T"])
        if case["bias"] or (case["groups"] > 1 and case["group_top"] == 2):
            for _ in range(8):
                bad = _close(case, logits, st["bias"])
                logits = torch.where(bad[:, None], _draw_logits(case, g, offset, case["T"]), logits)
        st["logits"] = logits
        if case["grad"]:
            st["idx"] = logits.float().sort(dim=-1, descending=True, stable=True).indices[:, :case["k"]].int().contiguous()
            st["dw"] = _normal(g, case["T"], case["k"])
    elif case["op"] == "linear":
        x = _activations(g, case["M"], case["K"], case["type"], case["pitch"])
        st["weights"] = _weights(g, case["N"], case["K"])
        st["bias"] = _normal(g, case["N"]) if case["bias"] else None
        if case["coded"]:
            code, scale = _quantise(x)
            st["codes"] = torch.zeros(case["M"], (case["K"] + 15) // 16 * 16, dtype=torch.int8, device="cuda")
            st["codes"][:, :case["K"]] = code.to(torch.int8)
            st["scales"] = scale
        else:
            st["x"] = x
    else:
        st["x"] = _activations(g, case["T"], case["H"], case["type"])
        st["gate_up"] = _weights(g, case["E"], 2 * case["I"], case["H"])
        st["down"] = _weights(g, case["E"], case["H"], case["I"])
        st["idx"], st["w"] = _routes(g, case["T"], case["E"], case["k"])
    return st


# ----------------------------------------------------------------------------------------------------- plain forms

def _plain_scores(score, logits):
    if score == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-logits))
    e = torch.exp(logits - logits.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_gate(st):
    case, logits, bias = st["case"], st["logits"].float(), st["bias"]
    T, E, k, G = case["T"], case["E"], case["k"], case["groups"]
    s = _plain_scores(case["score"], logits)
    # the scores rise with the logits: without a bias and without sums of scores the logits themselves decide
    choice = logits if bias is None and (G == 1 or case["group_top"] == 1) else s if bias is None else s + bias
    if G > 1:
        value = choice.view(T, G, E // G).sort(-1, descending=True).values[..., :case["group_top"]].sum(-1)
        best = value.sort(dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros(T, G, dtype=torch.bool, device=logits.device).scatter_(1, best, True)
        choice = torch.where(keep[:, :, None], choice.view(T, G, E // G), -math.inf).view(T, E)
    idx = choice.sort(dim=-1, descending=True, stable=True).indices[:, :k]
    w = s.gather(1, idx)
    if case["renorm"]:
        total = w.sum(-1, keepdim=True)
        w = torch.where(total > 0, w / total, torch.zeros_like(w))
    return idx.int(), w * case["scale"]


def _plain_gate_backward(st):
    case, logits, idx, dw = st["case"], st["logits"].float(), st["idx"].long(), st["dw"]
    s = _plain_scores(case["score"], logits)
    ds = dw * case["scale"]
    if case["renorm"]:
        mine = s.gather(1, idx)
        total = mine.sum(-1, keepdim=True)
        ds = (ds - (ds * mine).sum(-1, keepdim=True) / total) / total
    ds = torch.zeros_like(s).scatter_(1, idx, ds)
    if case["score"] == "sigmoid":
        return (ds * s * (1.0 - s)).to(st["logits"].dtype)
    return (s * (ds - (ds * s).sum(-1, keepdim=True))).to(st["logits"].dtype)


def _quantise(x):
    """Rows -> codes (as 32-bit numbers) and a scale for each row: code = round(127 x / amax), ties to the even code."""
    x = x.float()
    amax = x.abs().amax(-1, keepdim=True)
    code = torch.where(amax > 0, (x * 127.0 / amax).round(), torch.zeros_like(x))
    return code, (amax / 127.0).squeeze(-1)


def _plain_linear(st):
    case = st["case"]
    code, scale = (st["codes"][:, :case["K"]].float(), st["scales"]) if case["coded"] else _quantise(st["x"])
    w, ws, _ = st["weights"]
    y = (code @ w[:, :case["K"]].float().t()) * scale[:, None] * ws
    return (y if st["bias"] is None else y + st["bias"]).to(_TYPES[case["out"]])


def _plain_experts(st):
    case, x, w = st["case"], st["x"], st["w"]
    T, H, I, E, k = (case[n] for n in ("T", "H", "I", "E", "k"))
    gu, gu_s, _ = st["gate_up"]
    dn, dn_s, _ = st["down"]
    code, scale = _quantise(x)
    # the routes sorted by expert, every expert's rows padded to the fullest one's
    expert = st["idx"].long().view(-1)
    order = expert.sort(dim=0, stable=True).indices
    counts = torch.bincount(expert, minlength=E)
    place = torch.arange(T * k, device=x.device) - (counts.cumsum(0) - counts)[expert[order]]
    C = int(counts.max())
    row = expert[order] * C + place
    rows = torch.zeros(E * C, H, device=x.device).index_copy_(0, row, code[order // k])
    row_scale = torch.zeros(E * C, device=x.device).index_copy_(0, row, scale[order // k])
    y = torch.bmm(rows.view(E, C, H), gu[..., :H].float().transpose(1, 2)) * row_scale.view(E, C, 1) * gu_s[:, None]
    gate, up = y[..., :I], y[..., I:]
    h, h_scale = _quantise(gate / (1.0 + torch.exp(-gate)) * up)
    y = torch.bmm(h, dn[..., :I].float().transpose(1, 2)) * h_scale[..., None] * dn_s[:, None]
    at = torch.empty_like(row).index_copy_(0, order, row)
    return (y.view(E * C, H)[at].view(T, k, H) * w[..., None]).sum(1).to(x.dtype)


# ------------------------------------------------------------------------------------------------------------ runs

def run(st):
    case = st["case"]
    if not own:
        if case["op"] == "gate":
            return _plain_gate_backward(st) if case["grad"] else _plain_gate(st)
        return _plain_linear(st) if case["op"] == "linear" else _plain_experts(st)
    from paper_2609_36070_b200 import mok
    if case["op"] == "gate":
        if case["grad"]:
            return mok.mok_gate_backward(st["logits"], st["idx"], st["dw"], score=case["score"], renormalise=case["renorm"],
                                         scale=case["scale"])
        return mok.mok_gate(st["logits"], case["k"], bias=st["bias"], score=case["score"], n_groups=case["groups"],
                            topk_groups=case["top_groups"], group_top=case["group_top"], renormalise=case["renorm"],
                            scale=case["scale"])
    if case["op"] == "linear":
        weights = mok.I8Weights(*st["weights"])
        if case["coded"]:
            return mok.mok_i8_matmul(st["codes"], st["scales"], weights, K=case["K"], bias=st["bias"],
                                     out_dtype=_TYPES[case["out"]])
        return mok.mok_i8_linear(st["x"], weights, bias=st["bias"], out_dtype=_TYPES[case["out"]])
    return mok.mok_i8_experts(st["x"], st["idx"], st["w"], mok.I8Weights(*st["gate_up"]), mok.I8Weights(*st["down"]))


def work(case):
    if case["op"] == "gate":
        T, E, k, b = case["T"], case["E"], case["k"], _BYTES[case["type"]]
        if not case["grad"]:
            return {"bytes": T * E * b + T * k * 8 + (4 * E if case["bias"] else 0), "flops": 4 * T * E}
        dense = case["score"] == "softmax" and not case["renorm"]
        return {"bytes": T * E * b + T * k * 8 + T * (E if dense else k) * b, "flops": (6 * E if dense else 12 * k) * T}
    if case["op"] == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        moved = M * K * (1 if case["coded"] else _BYTES[case["type"]]) + N * K + M * N * _BYTES[case["out"]] + 4 * N
        return {"bytes": moved + (4 * M if case["coded"] else 0) + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    T, H, I, E, k = (case[n] for n in ("T", "H", "I", "E", "k"))
    met = E * (1.0 - (1.0 - k / E) ** T)        # experts that get at least one row
    return {"bytes": 2 * 2 * T * H + 8 * T * k + met * (3 * H * I + 4 * (2 * I + H)), "flops": 6 * T * k * H * I}


# -------------------------------------------------------------------------------------------- the same in 64 bits

def _scores64(case, logits):
    z = logits.double()
    return torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, -1)


def _codes64(x):
    x = x.double()
    amax = x.abs().max(-1, keepdim=True).values
    return torch.nan_to_num((x * 127 / amax).round(), nan=0.0), amax / 127


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "gate" and not case["grad"]:
        s = _scores64(case, st["logits"])
        c = st["logits"].double() if st["bias"] is None else s + st["bias"].double()
        if case["groups"] > 1:
            by = (c if case["group_top"] == 1 or st["bias"] is not None else s).unflatten(1, (case["groups"], -1))
            value = by.topk(case["group_top"], -1).values.sum(-1)
            rank = value.argsort(dim=-1, descending=True, stable=True).argsort(-1)
            c = c.unflatten(1, (case["groups"], -1)).masked_fill((rank >= case["top_groups"])[..., None], -math.inf).flatten(1)
        idx = c.argsort(dim=-1, descending=True, stable=True)[:, :case["k"]]
        w = torch.take_along_dim(s, idx, 1)
        return idx.int(), (w / w.sum(-1, keepdim=True) if case["renorm"] else w) * case["scale"]
    if case["op"] == "gate":
        z = st["logits"].double().requires_grad_()
        w = torch.take_along_dim(torch.sigmoid(z) if case["score"] == "sigmoid" else torch.softmax(z, -1), st["idx"].long(), 1)
        w = (w / w.sum(-1, keepdim=True) if case["renorm"] else w) * case["scale"]
        return torch.autograd.grad(w, z, st["dw"].double())[0]
    if case["op"] == "linear":
        q, s = (st["codes"][:, :case["K"]].double(), st["scales"].double()[:, None]) if case["coded"] else _codes64(st["x"])
        w, ws, _ = st["weights"]
        y = (q * s) @ (w[:, :case["K"]].double() * ws.double()[:, None]).t()
        return y if st["bias"] is None else y + st["bias"].double()
    I = case["I"]
    out = torch.zeros(case["T"], case["H"], dtype=torch.float64, device="cuda")
    q, s = _codes64(st["x"])
    for e in range(case["E"]):
        t, slot = torch.nonzero(st["idx"] == e, as_tuple=True)
        if len(t):
            z = (q[t] @ st["gate_up"][0][e, :, :case["H"]].double().t()) * s[t] * st["gate_up"][1][e].double()
            hq, hs = _codes64(torch.nn.functional.silu(z[:, :I]) * z[:, I:])
            y = (hq @ st["down"][0][e, :, :I].double().t()) * hs * st["down"][1][e].double()
            out.index_add_(0, t, y * st["w"][t, slot].double()[:, None])
    return out
