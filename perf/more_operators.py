"""The measured calls of the 8-bit expert operators and of the whole layer for a
few tokens: what a server of an MoE layer runs when its weights are kept in
8-bit floating point, and what it runs for each decode step.

    rows      activations [T,K] in blocks of 1 x 128: e4m3 codes and a power of two
    weights   weights [E,N,K] in blocks of 128 x 128
    product   y = a W^T of quantised activations and weights, dense or on the rows
              of each expert; the activations are quantised within the call
    ffn       a layer's experts forward on those products
    layer     router, Top-K, experts and join for 1 to 64 tokens, weights bf16 or
              in blocks of 128

A block's exponent byte e is the least from 3 on whose 448 * 2^(e - 127) holds the
block's largest value; codes are rounded to nearest even.  E experts, k of them
per token, T tokens, H the hidden size, F the experts' inner size (128 experts,
k = 8, F = 768 and H = 1024 or 2048 are the library's models), R = T k routed
rows.  Routing is uneven (a bias per expert); weights are N(0, 0.02).
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128


def _case(name, op, **sizes):
    return {**({"name": name} if name else {}), "op": op, **sizes}


def listed():
    return [
        # a micro-batch's hidden states (4 x 4096 tokens) on their way into 8-bit products, read back once
        _case("rows", "rows", T=16384, K=2048),
        # one layer's up projections on loading a model, read back once
        _case("weights", "weights", E=128, N=1536, K=2048, gated=True),
        # one token through a dense map: latency
        _case("product_token", "product", T=1, K=2048, N=4096, E=1, k=0, skew=0.0),
        # a dense map of a long prefill
        _case("product_dense", "product", T=16384, K=2048, N=4096, E=1, k=0, skew=0.0),
        # odd sizes: few experts, ragged rows, gathered tokens, a last block that is not full
        _case("product_odd", "product", T=5003, K=1008, N=520, E=24, k=3, skew=1.0),
        # the experts of a prefill of 4 x 4096 tokens: the largest
        _case("ffn", "ffn", T=16384, H=2048, F=768, E=128, k=8, skew=0.3),
        # a short prompt with an inner size off the blocks' width, a collapsing router
        _case("ffn_odd", "ffn", T=301, H=1008, F=208, E=40, k=5, skew=1.0),
        # a decode step of one token, weights as trained
        _case("layer_token", "layer", T=1, H=2048, F=768, E=128, k=8, skew=0.3, eight=False, softmax=False),
        # the same with weights in 8 bits
        _case("layer_token8", "layer", T=1, H=2048, F=768, E=128, k=8, skew=0.3, eight=True, softmax=False),
        # a few sequences on a small layer of odd sizes, softmax gate
        _case("layer_odd", "layer", T=7, H=1000, F=208, E=40, k=5, skew=1.0, eight=False, softmax=True),
        # a serving batch: most experts are read for one or a few tokens each
        _case("layer_batch", "layer", T=48, H=1024, F=768, E=128, k=8, skew=0.3, eight=False, softmax=False),
        # the largest batch of the call, weights in 8 bits
        _case("layer_batch8", "layer", T=64, H=2048, F=768, E=128, k=8, skew=0.3, eight=True, softmax=False),
    ]


def draw(rng):
    """A case of the ranges above: tokens on a logarithmic scale, sizes in the steps the operators take."""
    op = rng.choice(["rows", "weights", "product", "product", "ffn", "layer", "layer", "layer"])

    def size(lo, hi, step):
        return step * max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)))

    if op == "rows":
        return _case(None, op, T=size(1, 32768, 1), K=size(64, 4096, 16))
    if op == "weights":
        return _case(None, op, E=rng.choice([1, 8, 24, 64, 128]), N=size(64, 1536, 32), K=size(64, 2048, 16),
                     gated=rng.random() < 0.5)
    E, k = rng.choice([8, 16, 24, 40, 64, 96, 128]), rng.choice([1, 2, 3, 4, 5, 6, 8])
    skew = rng.choice([0.0, 0.3, 1.0])
    if op == "product":
        dense = rng.random() < 0.4
        return _case(None, op, T=size(1, 16384, 1), K=size(128, 2048, 16), N=size(64, 1536, 8),
                     E=1 if dense else E, k=0 if dense else k, skew=skew)
    if op == "ffn":
        return _case(None, op, T=size(1, 12288, 1), H=size(128, 2048, 16), F=size(64, 768, 16), E=E, k=k, skew=skew)
    eight = rng.random() < 0.5
    return _case(None, op, T=size(1, 64, 1), H=size(128, 3000, 16 if eight else 8), F=size(64, 896, 16), E=E, k=k,
                 skew=skew, eight=eight, softmax=rng.random() < 0.3)


# ---------------------------------------------------------------- inputs

def _pad(v, rows):
    """v [..., N, K] as [..., N / rows, rows, K / BLOCK, BLOCK], filled up with zeros."""
    n, k = v.shape[-2:]
    v = torch.nn.functional.pad(v, (0, -k % BLOCK, 0, -n % rows))
    return v.reshape(*v.shape[:-2], v.shape[-2] // rows, rows, v.shape[-1] // BLOCK, BLOCK)


def _quantise(v, rows):
    """Blocks of `rows` x 128 of v [..., N, K]: e4m3 codes and exponent bytes."""
    n, k = v.shape[-2:]
    b = _pad(v.float(), rows)
    most = b.abs().amax((-3, -1), keepdim=True)
    m, x = torch.frexp(most)                       # most = m 2^x with m in [0.5, 1); 448 = 0.875 2^9
    e = (x - 9 + (m > 0.875).to(x.dtype) + 127).clamp_(min=3)
    e = torch.where(most == 0, torch.full_like(e, 3), e)
    codes = torch.ldexp(b, 127 - e).to(torch.float8_e4m3fn)
    codes = codes.reshape(*v.shape[:-2], b.shape[-4] * rows, b.shape[-2] * BLOCK)[..., :n, :k].contiguous()
    return codes, e.squeeze(-1).squeeze(-2).to(torch.uint8)


def _values(q, rows):
    codes, e = q
    n, k = codes.shape[-2:]
    b = torch.ldexp(_pad(codes.float(), rows), (e.to(torch.int32) - 127).unsqueeze(-2).unsqueeze(-1))
    return b.reshape(*codes.shape[:-2], b.shape[-4] * rows, b.shape[-2] * BLOCK)[..., :n, :k]


def _halves(w):
    """w [E, 2 F, K], gate and up rows with blocks of their own, as [E, 2, F, K]."""
    return w.reshape(w.shape[0], 2, -1, w.shape[2])


def _quantise_weights(w, gated):
    codes, e = _quantise(_halves(w) if gated else w, BLOCK)
    return codes.reshape(w.shape), e.reshape(w.shape[0], -1, e.shape[-1])


def _weight_values(q, gated):
    codes, e = q
    if gated:
        e = e.reshape(e.shape[0], 2, -1, e.shape[-1])
    return _values((_halves(codes) if gated else codes, e), BLOCK).reshape(codes.shape)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(scale)

    c, op = case, case["op"]
    s = {"case": case}
    if op == "rows":
        # rows of different size, as hidden states are
        s["x"] = randn(c["T"], c["K"]) * torch.exp(torch.randn(c["T"], 1, generator=g, device="cuda")).bfloat16()
        return s
    if op == "weights":
        s["w"] = randn(c["E"], c["N"], c["K"], scale=0.02)
        return s
    T, E, k = c["T"], c["E"], c["k"]
    if op == "product":
        s["x"] = randn(T, c["K"])
        s["w"] = _quantise_weights(randn(E, c["N"], c["K"], scale=0.02), False)
    else:
        H, F = c["H"], c["F"]
        s["x"] = randn(T, H)
        s["w1"], s["w2"] = randn(E, 2 * F, H, scale=0.02), randn(E, H, F, scale=0.02)
        if op == "ffn" or c["eight"]:
            s["w1"], s["w2"] = _quantise_weights(s["w1"], True), _quantise_weights(s["w2"], False)
    if op == "layer":
        # hidden states share a direction, so that the router's logits have a bias per expert
        s["wr"] = randn(E, H, scale=0.02)
        s["x"] += randn(1, H) * (c["skew"] / 2)
        return s
    if k:
        z = torch.randn(T, E, generator=g, device="cuda")
        z += torch.randn(E, generator=g, device="cuda") * c["skew"]
        top, ids = torch.topk(z, k, dim=1)
        gates = torch.sigmoid(top)
        s["combine"] = (gates / gates.sum(1, keepdim=True)).contiguous()
        ids = ids.reshape(-1)
        order = torch.argsort(ids, stable=True)
        pos = torch.empty(T * k, dtype=torch.int32, device="cuda")
        pos[order] = torch.arange(T * k, dtype=torch.int32, device="cuda")
        counts = torch.bincount(ids, minlength=E)
        s["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        s["offsets"][1:] = torch.cumsum(counts, 0)
        s["rows"], s["pos"], s["largest"] = (order // k).to(torch.int32), pos.reshape(T, k), int(counts.max())
    return s


# ---------------------------------------------------------------- plain forms

def _product(s, a, w):
    """a [R, K] times the weights [E, N, K] of each row's expert."""
    off = s["offsets"].long()
    r = torch.arange(a.shape[0], device=a.device)
    e = torch.searchsorted(off[1:].contiguous(), r, right=True)
    box = torch.zeros(w.shape[0], s["largest"], a.shape[1], dtype=torch.float32, device=a.device)
    box[e, r - off[e]] = a
    return torch.bmm(box, w.transpose(1, 2))[e, r - off[e]]


def _swiglu(z):
    gate, up = z.chunk(2, dim=-1)
    return gate / (1 + torch.exp(-gate)) * up


def _route(s):
    c = s["case"]
    z = s["x"].double() @ s["wr"].double().T       # values next to the border of the Top-K
    top, ids = torch.sort(z, dim=1, descending=True, stable=True)
    top, ids = top[:, :c["k"]], ids[:, :c["k"]]
    if c["softmax"]:
        p = torch.exp(top - top[:, :1])
    else:
        p = 1 / (1 + torch.exp(-top))
    return ids, p / p.sum(1, keepdim=True)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "rows":
        return {"values": _values(_quantise(s["x"], 1), 1).bfloat16()}
    if op == "weights":
        return {"values": _weight_values(_quantise_weights(s["w"], c["gated"]), c["gated"]).bfloat16()}
    if op == "product":
        a, w = _values(_quantise(s["x"], 1), 1), _weight_values(s["w"], False)
        y = _product(s, a[s["rows"].long()], w) if c["k"] else a @ w[0].T
        return {"y": y.bfloat16()}
    if op == "ffn":
        a, w1, w2 = _values(_quantise(s["x"], 1), 1), _weight_values(s["w1"], True), _weight_values(s["w2"], False)
        act = _swiglu(_product(s, a[s["rows"].long()], w1))
        y = _product(s, _values(_quantise(act, 1), 1), w2)
        return {"out": (y[s["pos"].long()] * s["combine"].unsqueeze(-1)).sum(1).bfloat16()}
    ids, combine = _route(s)
    x = s["x"].float()
    if c["T"] * c["k"] <= c["E"]:
        # the chosen experts' weights, once for each choice
        pick = ids.reshape(-1)
        x = x.repeat_interleave(c["k"], dim=0).unsqueeze(1)
    else:
        # all experts for all tokens
        pick = torch.arange(c["E"], device=x.device)
    if c["eight"]:
        w1 = _weight_values(tuple(t[pick] for t in s["w1"]), True)
        w2 = _weight_values(tuple(t[pick] for t in s["w2"]), False)
    else:
        w1, w2 = s["w1"][pick].float(), s["w2"][pick].float()
    y = _swiglu(x @ w1.transpose(1, 2)) @ w2.transpose(1, 2)
    if c["T"] * c["k"] <= c["E"]:
        y = y.reshape(c["T"], c["k"], -1)
    else:
        y = y[ids, torch.arange(c["T"], device=x.device).unsqueeze(1)]
    combine = combine.float()
    return {"out": (y * combine.unsqueeze(-1)).sum(1).bfloat16(), "ids": ids.to(torch.int32), "combine": combine}


# ---------------------------------------------------------------- the library's calls

def _own(s):
    from paper_2609_32398_gb300 import doloss as dl
    from paper_2609_32398_gb300 import experts8 as e8
    from paper_2609_32398_gb300 import layer

    c, op = s["case"], s["case"]["op"]
    if op == "rows":
        return {"values": e8.quantise_rows(s["x"]).values()}
    if op == "weights":
        return {"values": e8.quantise_weights(s["w"], gated=c["gated"]).values()}
    if op == "product":
        a, w = e8.quantise_rows(s["x"]), e8.Blocks(*s["w"])
        return {"y": e8.matmul(a, w, s["offsets"], s["rows"]) if c["k"] else e8.matmul(a, w)}
    if op == "ffn":
        return {"out": e8.expert_ffn(s["x"], e8.Blocks(*s["w1"], gated=True), e8.Blocks(*s["w2"]), s["combine"],
                                     s["offsets"], s["rows"], s["pos"])}
    w1, w2 = s["w1"], s["w2"]
    if c["eight"]:
        w1, w2 = e8.Blocks(*w1, gated=True), e8.Blocks(*w2)
    out, ids, combine = layer.moe_layer(s["x"], s["wr"], w1, w2, c["k"],
                                        dl.GATE_SOFTMAX if c["softmax"] else dl.GATE_SIGMOID_NORM)
    return {"out": out, "ids": ids, "combine": combine}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- work and 64 bits

def work(case):
    """Each input read once and each output written once.  Of the weights, the experts that balanced routing
    reaches: E (1 - (1 - k/E)^T) of them."""
    c, op = case, case["op"]
    if op == "rows":  # the codes written and read back
        return {"bytes": c["T"] * c["K"] * (2 + 2 * (1 + 1 / BLOCK) + 2), "flops": c["T"] * c["K"] * 2}
    if op == "weights":
        return {"bytes": c["E"] * c["N"] * c["K"] * 6, "flops": c["E"] * c["N"] * c["K"] * 2}
    T, E, k = c["T"], c["E"], c["k"]
    R = T * k if k else T
    used = E * (1 - (1 - k / E) ** T) if k else 1
    index = 4 * R + 4 * (E + 1) if k else 0
    if op == "product":
        return {"bytes": 2 * T * c["K"] + used * c["N"] * c["K"] + index + 2 * R * c["N"],
                "flops": 2 * R * c["N"] * c["K"]}
    H, F = c["H"], c["F"]
    if op == "ffn":
        return {"bytes": 4 * T * H + used * 3 * F * H + 2 * index + 4 * R, "flops": 6 * R * H * F}
    return {"bytes": used * 3 * F * H * (1 if c["eight"] else 2) + 2 * E * H + 4 * T * H + 8 * R,
            "flops": 6 * R * H * F + 2 * T * E * H}


def _rounded(v, rows):
    """The values that v's blocks of rows x 128 stand for, in 64 bits: the grid of e4m3 by its definition."""
    n, k = v.shape[-2:]
    b = _pad(v.double(), rows)
    most = b.abs().amax((-3, -1), keepdim=True)
    least = torch.full_like(most, 2.0 ** -124)
    scale = torch.maximum(torch.exp2(torch.ceil(torch.log2(torch.clamp(most / 448, min=1e-300)))), least)
    scale = torch.where(most <= 448 * scale / 2, torch.maximum(scale / 2, least), scale)   # log2 may round
    scale = torch.where(most > 448 * scale, scale * 2, scale)
    u = b / scale
    step = torch.exp2(torch.clamp(torch.frexp(u)[1].double() - 4, min=-9.0))
    u = torch.round(u / step) * step * scale
    return u.reshape(*v.shape[:-2], u.shape[-4] * rows, u.shape[-2] * BLOCK)[..., :n, :k]


def _stands_for(codes, e):
    """The 64-bit values of weights [N, K] in blocks of 128 x 128."""
    scale = torch.pow(2.0, e.double() - 127).repeat_interleave(BLOCK, 0).repeat_interleave(BLOCK, 1)
    return codes.double() * scale[:codes.shape[0], :codes.shape[1]]


def exact(case, seed):
    s = prepare(case, seed)
    c, op = case, case["op"]
    if op == "rows":
        return {"values": _rounded(s["x"], 1)}
    if op == "weights":
        w = s["w"]
        out = torch.empty(w.shape, dtype=torch.float64, device=w.device)
        parts = 2 if c["gated"] else 1
        n = w.shape[1] // parts
        for e in range(w.shape[0]):
            for p in range(parts):
                out[e, p * n:(p + 1) * n] = _rounded(w[e, p * n:(p + 1) * n], BLOCK)
        return {"values": out}

    def weights(name, e):
        w = s[name]
        if not isinstance(w, tuple):
            return w[e].double()
        codes, x = w[0][e], w[1][e]
        if name != "w1":
            return _stands_for(codes, x)
        n, m = codes.shape[0] // 2, x.shape[0] // 2
        return torch.cat([_stands_for(codes[:n], x[:m]), _stands_for(codes[n:], x[m:])])

    def act_of(z):
        n = z.shape[1] // 2
        return z[:, :n] * torch.sigmoid(z[:, :n]) * z[:, n:]

    if op == "layer":
        x = s["x"].double()
        z = x @ s["wr"].double().T
        k, T = c["k"], c["T"]
        ids = torch.empty(T, k, dtype=torch.int32, device=x.device)
        left = z.clone()
        for q in range(k):
            ids[:, q] = left.argmax(1).to(torch.int32)
            left[torch.arange(T, device=x.device), ids[:, q].long()] = -math.inf
        chosen = torch.gather(z, 1, ids.long())
        combine = torch.softmax(chosen, 1) if c["softmax"] else torch.sigmoid(chosen) / torch.sigmoid(chosen).sum(1, True)
        out = torch.zeros_like(x)
        for e in range(c["E"]):
            t, q = torch.nonzero(ids == e, as_tuple=True)
            if t.numel():
                y = act_of(x[t] @ weights("w1", e).T) @ weights("w2", e).T
                out.index_add_(0, t, y * combine[t, q].unsqueeze(1))
        return {"out": out, "ids": None, "combine": combine}
    a = _rounded(s["x"], 1)
    if op == "product" and not c["k"]:
        return {"y": a @ weights("w", 0).T}
    bounds, rows = s["offsets"].tolist(), s["rows"].long()
    out = torch.empty(rows.numel(), c["N"] if op == "product" else c["H"], dtype=torch.float64, device=a.device)
    for e in range(c["E"]):
        i, j = bounds[e], bounds[e + 1]
        if i == j:
            continue
        if op == "product":
            out[i:j] = a[rows[i:j]] @ weights("w", e).T
        else:
            out[i:j] = _rounded(act_of(a[rows[i:j]] @ weights("w1", e).T), 1) @ weights("w2", e).T
    if op == "product":
        return {"y": out}
    total = torch.zeros(c["T"], c["H"], dtype=torch.float64, device=a.device)
    for q in range(c["k"]):
        total += out[s["pos"][:, q].long()] * s["combine"][:, q:q + 1].double()
    return {"out": total}
