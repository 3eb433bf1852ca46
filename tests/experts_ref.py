"""The expert operators in 64 bits on the CPU, written from their formulas, with
the sums of magnitudes that the tests' error bounds are made of."""
import torch


def groups(counts):
    off = torch.zeros(len(counts) + 1, dtype=torch.int64)
    off[1:] = torch.cumsum(torch.tensor(counts), 0)
    return off


def each(offsets, n, rows, value):
    out = torch.zeros(rows, n, dtype=torch.float64)
    for e in range(len(offsets) - 1):
        a, b = int(offsets[e]), int(offsets[e + 1])
        if a < b:
            out[a:b] = value(e, a, b)
    return out


def product(a, w, offsets, rows=None, transposed=False):
    """(y, the same sum of magnitudes): a [T,K], w [E,N,K] or [E,K,N]."""
    a, w = a.double(), w.double()
    a = a if rows is None else a[rows.long()]
    n = w.shape[2] if transposed else w.shape[1]
    side = (lambda m: m) if transposed else (lambda m: m.T)
    y = each(offsets, n, a.shape[0], lambda e, i, j: a[i:j] @ side(w[e]))
    m = each(offsets, n, a.shape[0], lambda e, i, j: a[i:j].abs() @ side(w[e].abs()))
    return y, m


def swiglu(z):
    F = z.shape[1] // 2
    g, u = z[:, :F], z[:, F:]
    return g * torch.sigmoid(g) * u


def quantise(z):
    """The 8-bit format by its definition: per block of 16, the least e in 1..250
    with max |z| <= 127 * 2^(e - 127), by trying them all."""
    b = z.double().reshape(z.shape[0], -1, 16)
    top = b.abs().amax(-1)
    e = torch.full(top.shape, 250, dtype=torch.int64)
    for x in range(249, 0, -1):
        e[top <= 127.0 * 2.0 ** (x - 127)] = x
    codes = torch.round(b / torch.pow(2.0, (e - 127).double()).unsqueeze(-1))
    return codes.to(torch.int8).reshape(z.shape), e.to(torch.uint8)


def values(codes, exponents):
    b = codes.double().reshape(codes.shape[0], -1, 16)
    return (b * torch.pow(2.0, exponents.double() - 127).unsqueeze(-1)).reshape(codes.shape)


def up_backward(dout, w2, z, combine, offsets, rows, pos):
    """dz, w act, dcombine, and the magnitudes of g's terms, for z [R,2F]."""
    F = z.shape[1] // 2
    gate, up = z[:, :F].double(), z[:, F:].double()
    s = torch.sigmoid(gate)
    act = gate * s * up
    g, gm = product(dout, w2, offsets, rows, transposed=True)
    w = torch.zeros(g.shape[0], 1, dtype=torch.float64)
    w[pos.reshape(-1).long(), 0] = combine.double().reshape(-1)
    dz = torch.cat([w * g * up * s * (1 + gate * (1 - s)), w * g * gate * s], 1)
    return dz, w * act, (g * act).sum(1)[pos.long()], g, gm, w, act


def dispatch(ids, E):
    """offsets, rows, pos of expert ids [T,k], the pairs by expert then token."""
    T, k = ids.shape
    flat = ids.reshape(-1)
    order = torch.argsort(flat, stable=True)
    pos = torch.empty(T * k, dtype=torch.int64)
    pos[order] = torch.arange(T * k)
    counts = torch.bincount(flat, minlength=E)
    return groups(counts.tolist()), (order // k), pos.reshape(T, k)


def ffn(x, w1, w2, combine, offsets, rows, pos):
    """The whole layer, differentiable in 64 bits (no rounding, no checkpoint)."""
    a = x[rows.long()]
    parts = []
    for e in range(len(offsets) - 1):
        i, j = int(offsets[e]), int(offsets[e + 1])
        parts.append(swiglu(a[i:j] @ w1[e].T) @ w2[e].T)
    y = torch.cat(parts)
    return (y[pos.reshape(-1).long()].reshape(*pos.shape, -1) * combine.unsqueeze(-1)).sum(1)
