"""The 8-bit block format in 64 bits on the CPU, from its definition: e4m3 codes and one
exponent byte for a block of 128 columns of one row, or of 128 x 128."""
import torch

GRID = None


def grid():
    """The 127 finite magnitudes of e4m3 by their codes: 2^-9 m for exponent field 0,
    (8 + m) 2^(x - 10) for x = 1..15 (15, 7 is the NaN)."""
    global GRID
    if GRID is None:
        v = [m * 2.0 ** -9 for m in range(8)]
        v += [(8 + m) * 2.0 ** (x - 10) for x in range(1, 16) for m in range(8)]
        GRID = torch.tensor(v[:-1], dtype=torch.float64)
    return GRID


def code_values(codes):
    """64-bit values of codes (uint8): the sign bit, then the grid; 127 is the NaN."""
    c = codes.to(torch.int64)
    table = torch.cat([grid(), torch.tensor([float("nan")], dtype=torch.float64)])
    return torch.where(c >= 128, -1.0, 1.0).double() * table[c & 127]


def _blocks(v, rows):
    n, k = v.shape
    b = torch.zeros(-(-n // rows) * rows, -(-k // 128) * 128, dtype=torch.float64)
    b[:n, :k] = v
    return b.reshape(b.shape[0] // rows, rows, b.shape[1] // 128, 128).transpose(1, 2)


def _back(b, n, k):
    x, y = b.shape[:2]
    return b.transpose(1, 2).reshape(x * b.shape[2], y * 128)[:n, :k]


def quantise(v, rows):
    """v [N,K] -> (codes uint8 [N,K], exponents uint8): the least e >= 3 by trying them all,
    codes by the nearest value of the grid, ties to the even code.  `rows` rows share a block."""
    b = _blocks(v.double(), rows)
    top = b.abs().nan_to_num(nan=float("inf")).amax((-1, -2))
    e = torch.full(top.shape, 255, dtype=torch.int64)
    for x in range(247, 2, -1):
        e[top <= 448.0 * 2.0 ** (x - 127)] = x
    u = b.abs() * torch.pow(2.0, (127 - e).double()).unsqueeze(-1).unsqueeze(-1)
    g = grid()
    hi = torch.searchsorted(g, u.nan_to_num(nan=0.0, posinf=0.0).contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = u - g[lo], g[hi] - u
    c = torch.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo)
    c = c + 128 * torch.signbit(b)
    bad = (e == 255).unsqueeze(-1).unsqueeze(-1)
    c = torch.where(bad, torch.full_like(c, 127), c)
    return _back(c, *v.shape).to(torch.uint8), e.to(torch.uint8)


def values(codes, exponents, rows):
    """64-bit values of codes [N,K] (uint8) under exponents [ceil(N / rows), ceil(K / 128)]."""
    n, k = codes.shape
    s = torch.pow(2.0, exponents.double() - 127)
    s = torch.where(exponents == 255, float("nan"), s)
    s = s.repeat_interleave(rows, 0)[:n].repeat_interleave(128, 1)[:, :k]
    return code_values(codes) * s


def weights(w, gated=False):
    """codes, exponents and values of weights [E,N,K]."""
    halves = 2 if gated else 1
    E, N, K = w.shape
    n = N // halves
    q = [quantise(w[e, h * n:(h + 1) * n], 128) for e in range(E) for h in range(halves)]
    v = torch.stack([values(c, x, 128) for c, x in q]).reshape(E, N, K)
    codes = torch.stack([c for c, _ in q]).reshape(E, N, K)
    return codes, torch.stack([x for _, x in q]).reshape(E, -1, -(-K // 128)), v
