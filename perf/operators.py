"""The measured calls of the expert operators: the products of an MoE layer's
experts on the dispatch order that the router's `routing()` gives, their
8-bit activation checkpoints and their gradients.

Each case is one call that a user's program makes between the router and the
rest of the layer:

    up          act = silu(X W1g^T) * (X W1u^T) on the rows of each expert,
                with `checkpoint` also the pre-activations kept in 8 bits
    matmul      Y = A W^T (or A W) on the rows of each expert
    join        the same products, summed per token over its k rows
    up_grad     the gradient through the down projection and the activation,
                from the 8-bit checkpoint
    weight_grad dW = P^T Q over the rows of each expert, fp32
    ffn         the whole expert layer forward, as a server calls it

E experts, k of them per token, T tokens, H the hidden size, F the experts'
inner size (128 experts, k = 8, F = 768 and H = 1024 or 2048 are the
library's models; 64 experts its c2 layer), R = T k routed rows.  Routing is
uneven (a bias per expert), so groups are ragged; weights are N(0, 0.02) as
in the library's router recipes.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 16      # values that share one exponent in an 8-bit checkpoint


def _case(name, op, T, H, F, E, k, skew=0.3, **more):
    c = {"op": op, "T": T, "H": H, "F": F, "E": E, "k": k, "skew": skew, **more}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token through one layer's experts: eight of them are read, latency is all of it
        _case("ffn_token", "ffn", 1, 2048, 768, 128, 8),
        # a serving batch: most experts are read for one or a few rows each
        _case("ffn_batch", "ffn", 48, 1024, 768, 128, 8),
        # a long prefill or a large micro-batch, forward only (16 x 4096 tokens, the library's c3): the largest
        _case("up_long", "up", 65536, 2048, 768, 128, 8, checkpoint=False),
        # the forward half of a training micro-batch (4 x 4096 tokens) with its 8-bit checkpoint, read back once
        _case("up_checkpoint", "up", 16384, 2048, 768, 128, 8, checkpoint=True),
        # a shared product without activation on odd sizes: few experts, ragged rows, gathered tokens
        _case("matmul_odd", "matmul", 5003, 1000, 520, 24, 3, skew=1.0, transposed=False, gather=True),
        # the same through the weights' other side, rows in dispatch order (an input gradient before its join)
        _case("matmul_back", "matmul", 8192, 1024, 768, 64, 8, transposed=True, gather=False),
        # the down projection of a training micro-batch and the weighted join per token
        _case("down_join", "join", 16384, 2048, 768, 128, 8, transposed=False, weighted=True),
        # the gradient of the layer's input: dZ through W1, joined without weights; a collapsing router
        _case("input_grad", "join", 7001, 1024, 1536, 128, 8, skew=1.0, transposed=True, weighted=False),
        # the backward half of the same micro-batch, from the checkpoint
        _case("up_grad", "up_grad", 16384, 2048, 768, 128, 8),
        # a short ragged window with an inner size off the tiles' width
        _case("up_grad_odd", "up_grad", 1531, 1016, 208, 40, 5, skew=1.0),
        # dW1 of the micro-batch: the tokens are gathered again, nothing was kept of them
        _case("w1_grad", "weight_grad", 16384, 2048, 1536, 128, 8, gather="q"),
        # dW2 of a smaller layer: the outputs' gradient is the gathered side
        _case("w2_grad", "weight_grad", 4095, 1024, 768, 64, 8, gather="p"),
    ]


def draw(rng):
    """A case of the ranges above: T from 1 to 32768 on a logarithmic scale, sizes in the steps the operators take."""
    op = rng.choice(["up", "up", "matmul", "join", "up_grad", "weight_grad", "ffn"])
    T = int(round(math.exp(rng.uniform(0.0, math.log(4096 if op == "ffn" else 32768)))))
    E = rng.choice([8, 16, 24, 40, 64, 96, 128])
    k = rng.choice([1, 2, 3, 4, 5, 6, 8])
    H = 8 * int(round(math.exp(rng.uniform(math.log(16), math.log(256)))))
    F = 16 * int(round(math.exp(rng.uniform(math.log(4), math.log(56)))))
    skew = rng.choice([0.0, 0.3, 1.0])
    if op == "up":
        return _case(None, op, T, H, F, E, k, skew, checkpoint=rng.random() < 0.5)
    if op == "matmul":
        return _case(None, op, T, H, F, E, k, skew, transposed=rng.random() < 0.5, gather=rng.random() < 0.5)
    if op == "join":
        return _case(None, op, T, H, F, E, k, skew, transposed=rng.random() < 0.5, weighted=rng.random() < 0.5)
    if op == "weight_grad":
        return _case(None, op, T, H, F, E, k, skew, gather=rng.choice(["p", "q"]))
    return _case(None, op, T, H, F, E, k, skew)


# ---------------------------------------------------------------- inputs

def _draws(case, seed):
    """The inputs of one case: tensors on the GPU, and the largest group as the host knows it."""
    T, H, F, E, k = (case[n] for n in ("T", "H", "F", "E", "k"))
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def randn(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16).mul_(scale)

    z = torch.randn(T, E, generator=g, device="cuda")
    z += torch.randn(E, generator=g, device="cuda") * case["skew"]
    top, ids = torch.topk(z, k, dim=1)
    gates = torch.sigmoid(top)
    combine = gates / gates.sum(1, keepdim=True)
    ids = ids.reshape(-1)
    order = torch.argsort(ids, stable=True)
    pos = torch.empty(T * k, dtype=torch.int32, device="cuda")
    pos[order] = torch.arange(T * k, dtype=torch.int32, device="cuda")
    counts = torch.bincount(ids, minlength=E)
    offsets = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = torch.cumsum(counts, 0)
    s = {"case": case, "rows": (order // k).to(torch.int32), "offsets": offsets, "pos": pos.reshape(T, k),
         "combine": combine.contiguous(), "largest": int(counts.max())}
    R, op = T * k, case["op"]
    if op in ("up", "ffn"):
        s["x"] = randn(T, H)
        s["w1"] = randn(E, 2 * F, H, scale=0.02)
    if op in ("ffn", "up_grad"):
        s["w2"] = randn(E, H, F, scale=0.02)
    if op == "matmul":
        # A W^T with W [E, F, H], or A W with W [E, H, F]
        s["a"] = randn(T if case["gather"] else R, H)
        s["w"] = randn(E, H, F, scale=0.02) if case["transposed"] else randn(E, F, H, scale=0.02)
    if op == "join":
        # rows of F values to H per token: A W^T with W [E, H, F], or A W with W [E, F, H]
        s["a"] = randn(R, F)
        s["w"] = randn(E, F, H, scale=0.02) if case["transposed"] else randn(E, H, F, scale=0.02)
    if op == "up_grad":
        s["dout"] = randn(T, H, scale=1.0 / 64)
        s["codes"], s["exponents"] = _quantise(torch.randn(R, 2 * F, generator=g, device="cuda"))
    if op == "weight_grad":
        # dW [E, P columns, Q columns]; the gathered side is a matrix of tokens
        token, row = randn(T, H), randn(R, F, scale=1.0 / 64)
        s["p"], s["q"] = (token, row) if case["gather"] == "p" else (row, token)
    return s


def prepare(case, seed):
    return _draws(case, seed)


def _quantise(z):
    """Blocks of 16 neighbours in 8 bits: codes in [-127, 127] and a power of two, 2^(e - 127), the least that
    holds the block's largest value."""
    b = z.float().reshape(z.shape[0], -1, BLOCK)
    most = b.abs().amax(-1)
    m, x = torch.frexp(most)                       # most = m 2^x with m in [0.5, 1)
    e = (x - 7 + (m > 127.0 / 128.0).to(x.dtype) + 127).clamp_(min=1)
    e = torch.where(most == 0, torch.ones_like(e), e)
    codes = torch.round(torch.ldexp(b, (127 - e).unsqueeze(-1)))
    return codes.to(torch.int8).reshape(z.shape), e.to(torch.uint8)


def _values(codes, exponents):
    b = codes.float().reshape(codes.shape[0], -1, BLOCK)
    return torch.ldexp(b, (exponents.to(torch.int32) - 127).unsqueeze(-1)).reshape(codes.shape)


# ---------------------------------------------------------------- plain forms

def _groups(s):
    """The expert of each routed row and the row's place among the expert's."""
    off = s["offsets"].long()
    r = torch.arange(s["rows"].numel(), device=off.device)
    e = torch.searchsorted(off[1:].contiguous(), r, right=True)
    return e, r - off[e]


def _boxed(s, a, e, slot):
    box = torch.zeros(s["case"]["E"], s["largest"], a.shape[1], dtype=torch.float32, device=a.device)
    box[e, slot] = a.float()
    return box


def _product(s, a, w, transposed=False):
    """a [R, K] times the weights of each row's expert: w [E, N, K], or [E, K, N] where transposed."""
    e, slot = _groups(s)
    w = w.float()
    return torch.bmm(_boxed(s, a, e, slot), w if transposed else w.transpose(1, 2))[e, slot]


def _swiglu(z):
    gate, up = z.chunk(2, dim=1)
    return gate / (1 + torch.exp(-gate)) * up


def _join(s, y, weights):
    picked = y[s["pos"].reshape(-1).long()].reshape(*s["pos"].shape, -1)
    return (picked if weights is None else picked * weights.unsqueeze(-1)).sum(1)


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    rows = s["rows"].long()
    if op == "up":
        z = _product(s, s["x"][rows], s["w1"])
        act = _swiglu(z).bfloat16()
        return {"act": act, "values": _values(*_quantise(z)).bfloat16()} if c["checkpoint"] else {"act": act}
    if op == "ffn":
        act = _swiglu(_product(s, s["x"][rows], s["w1"]))
        return {"out": _join(s, _product(s, act, s["w2"]), s["combine"]).bfloat16()}
    if op == "matmul":
        a = s["a"][rows] if c["gather"] else s["a"]
        return {"y": _product(s, a, s["w"], c["transposed"]).bfloat16()}
    if op == "join":
        y = _product(s, s["a"], s["w"], c["transposed"])
        return {"out": _join(s, y, s["combine"] if c["weighted"] else None).bfloat16()}
    if op == "up_grad":
        gate, up = _values(s["codes"], s["exponents"]).chunk(2, dim=1)
        sig = 1 / (1 + torch.exp(-gate))
        act = gate * sig * up
        g = _product(s, s["dout"][rows], s["w2"], True)
        w = torch.empty(rows.numel(), 1, device=g.device)
        w[s["pos"].reshape(-1).long(), 0] = s["combine"].reshape(-1)
        dz = torch.cat([g * w * up * sig * (1 + gate * (1 - sig)), g * w * gate * sig], dim=1)
        dcombine = (g * act).sum(1)[s["pos"].long()]
        return {"dz": dz.bfloat16(), "act": (act * w).bfloat16(), "dcombine": dcombine}
    p = s["p"][rows] if c["gather"] == "p" else s["p"]
    q = s["q"][rows] if c["gather"] == "q" else s["q"]
    e, slot = _groups(s)
    return {"dw": torch.bmm(_boxed(s, p, e, slot).transpose(1, 2), _boxed(s, q, e, slot))}


# ---------------------------------------------------------------- the library's calls

def _own(s):
    from paper_2609_32398_gb300 import experts as ex

    c, op = s["case"], s["case"]["op"]
    rows, offsets, pos = s["rows"], s["offsets"], s["pos"]
    if op == "up":
        act, kept = ex.expert_up(s["x"], s["w1"], offsets, rows, checkpoint=c["checkpoint"])
        return {"act": act, "values": kept.values()} if c["checkpoint"] else {"act": act}
    if op == "ffn":
        with torch.no_grad():
            return {"out": ex.expert_ffn(s["x"], s["w1"], s["w2"], s["combine"], offsets, rows, pos)}
    if op == "matmul":
        return {"y": ex.grouped_matmul(s["a"], s["w"], offsets, rows if c["gather"] else None,
                                       transposed=c["transposed"])}
    if op == "join":
        return {"out": ex.grouped_matmul_join(s["a"], s["w"], offsets, pos, s["combine"] if c["weighted"] else None,
                                              transposed=c["transposed"])}
    if op == "up_grad":
        dz, act, dcombine = ex.expert_up_backward(s["dout"], s["w2"], ex.Checkpoint(s["codes"], s["exponents"]),
                                                  s["combine"], offsets, rows, pos)
        return {"dz": dz, "act": act, "dcombine": dcombine}
    return {"dw": ex.grouped_weight_grad(s["p"], s["q"], offsets, rows if c["gather"] == "p" else None,
                                         rows if c["gather"] == "q" else None)}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- work and 64 bits

def work(case):
    """Each input read once and each output written once.  Of the weights, the experts that balanced routing
    reaches: E (1 - (1 - k/E)^T) of them."""
    T, H, F, E, k, op = (case[n] for n in ("T", "H", "F", "E", "k", "op"))
    R = T * k
    used = E * (1 - (1 - k / E) ** T)
    index = 4 * R + 4 * (E + 1)
    if op == "up":
        b = 2 * T * H + 2 * used * 2 * F * H + index + 2 * R * F
        if case["checkpoint"]:  # written, read back, and the values written
            b += 2 * R * 2 * F * (1 + 1 / BLOCK) + 2 * R * 2 * F
        return {"bytes": b, "flops": 2 * R * H * 2 * F}
    if op == "ffn":
        return {"bytes": 2 * used * 3 * F * H + 2 * 2 * T * H + 2 * index + 4 * R, "flops": 2 * R * H * 3 * F}
    if op == "matmul":
        return {"bytes": 2 * (T if case["gather"] else R) * H + 2 * used * F * H + index + 2 * R * F,
                "flops": 2 * R * H * F}
    if op == "join":
        return {"bytes": 2 * R * F + 2 * used * F * H + index + (4 * R if case["weighted"] else 0) + 2 * T * H,
                "flops": 2 * R * H * F}
    if op == "up_grad":
        return {"bytes": 2 * T * H + 2 * used * H * F + R * 2 * F * (1 + 1 / BLOCK) + 2 * index + 8 * R
                + 2 * R * 2 * F + 2 * R * F, "flops": 2 * R * H * F}
    return {"bytes": 2 * T * H + 2 * R * F + index + 4 * E * H * F, "flops": 2 * R * H * F}


def exact(case, seed):
    s = _draws(case, seed)
    T, H, F, E, k, op = (case[n] for n in ("T", "H", "F", "E", "k", "op"))
    rows, pos, R = s["rows"].long(), s["pos"].long(), T * k
    bounds = s["offsets"].tolist()

    def of_each(n, value):
        """value(expert, first row, end row) for every expert with rows, in one [R, n] matrix."""
        out = torch.zeros(R, n, dtype=torch.float64, device="cuda")
        for e in range(E):
            if bounds[e] < bounds[e + 1]:
                out[bounds[e]:bounds[e + 1]] = value(e, bounds[e], bounds[e + 1])
        return out

    def joined(y, weights):
        out = torch.zeros(T, y.shape[1], dtype=torch.float64, device="cuda")
        for q in range(k):
            out += y[pos[:, q]] * (1.0 if weights is None else weights[:, q:q + 1].double())
        return out

    if op in ("up", "ffn"):
        z = of_each(2 * F, lambda e, a, b: s["x"][rows[a:b]].double() @ s["w1"][e].double().T)
        act = z[:, :F] * torch.sigmoid(z[:, :F]) * z[:, F:]
        if op == "up":
            # the checkpoint stands for the pre-activations themselves
            return {"act": act, "values": z} if case["checkpoint"] else {"act": act}
        return {"out": joined(of_each(H, lambda e, a, b: act[a:b] @ s["w2"][e].double().T), s["combine"])}
    if op in ("matmul", "join"):
        def rows_of(e, a, b):
            left = (s["a"][rows[a:b]] if op == "matmul" and case["gather"] else s["a"][a:b]).double()
            w = s["w"][e].double()
            return left @ (w if case["transposed"] else w.T)
        if op == "matmul":
            return {"y": of_each(F, rows_of)}
        return {"out": joined(of_each(H, rows_of), s["combine"] if case["weighted"] else None)}
    if op == "up_grad":
        scale = torch.pow(2.0, s["exponents"].double() - 127).repeat_interleave(BLOCK, dim=1)
        z = s["codes"].double() * scale
        gate, up = z[:, :F], z[:, F:]
        sig = torch.sigmoid(gate)
        g = of_each(F, lambda e, a, b: s["dout"][rows[a:b]].double() @ s["w2"][e].double())
        w = torch.zeros(R, 1, dtype=torch.float64, device="cuda")
        w[pos.reshape(-1), 0] = s["combine"].reshape(-1).double()
        act = gate * sig * up
        dz = torch.cat([w * g * up * (sig + gate * sig * torch.sigmoid(-gate)), w * g * gate * sig], dim=1)
        return {"dz": dz, "act": w * act, "dcombine": (g * act).sum(1)[pos]}
    p_of = (lambda a, b: s["p"][rows[a:b]]) if case["gather"] == "p" else (lambda a, b: s["p"][a:b])
    q_of = (lambda a, b: s["q"][rows[a:b]]) if case["gather"] == "q" else (lambda a, b: s["q"][a:b])
    dw = torch.zeros(E, s["p"].shape[1], s["q"].shape[1], dtype=torch.float64, device="cuda")
    for e in range(E):
        a, b = bounds[e], bounds[e + 1]
        dw[e] = p_of(a, b).double().T @ q_of(a, b).double()
    return {"dw": dw}
