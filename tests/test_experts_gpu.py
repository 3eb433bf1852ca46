"""The expert operators against 64 bits (tests/experts_ref.py).

Bounds, for U = 2^-24: a product of bf16 values is exact in fp32 and K of them
summed in fp32 are within 2 K U of the sum of magnitudes (twice the classic
bound); a result rounded to bf16 is within 2^-9 of itself (2^-8 taken); __expf
and the divide of sigma are within 2^-18 of it for |z| < 30.  What follows from
them is written at each check."""
import pytest
import torch

import experts_ref as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = 2.0 ** -8
FN = 2.0 ** -18


@pytest.fixture(scope="module")
def ex():
    from paper_2609_32398_gb300 import doloss, experts

    doloss.lib()
    return experts


def rnd(seed, *shape, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).bfloat16()


def gpu(*ts):
    return [None if t is None else (t.to(torch.int32) if t.dtype == torch.int64 else t).contiguous().cuda()
            for t in ts]


def ok(ex):
    torch.cuda.synchronize()
    st = ex.device_status()
    from paper_2609_32398_gb300 import doloss as dl
    assert st == 0, dl.status_string(st)


def within(got, want, bound):
    got = got.double().cpu()
    assert got.shape == want.shape
    off = (got - want).abs() - bound
    assert torch.isfinite(got).all()
    assert (off <= 1e-30).all(), float(off.max())


def ragged(E, total, seed):
    """Group sizes with empty groups, groups of one, and one long group."""
    g = torch.Generator().manual_seed(seed)
    p = torch.rand(E, generator=g) ** 4
    p[:: 3] = 0
    p[E // 2] += 2
    c = torch.floor(p / p.sum() * total).long()
    c[E // 2] += total - c.sum()
    return c.tolist()


# counts of each expert's rows, K, N
PRODUCTS = [([1], 8, 8), ([0, 3, 0, 0, 1], 64, 64), ([17, 0, 130, 16], 72, 136), ([255, 256, 257, 0, 1], 200, 264),
            ([1] * 40, 520, 24), ([700], 128, 512), (ragged(24, 2000, 3), 1000, 520), ([5, 300, 33], 2048, 96),
            ([0, 0, 9], 16, 1032), (ragged(128, 3000, 5), 256, 128)]


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,K,N", PRODUCTS)
def test_grouped_matmul(ex, counts, K, N, gather, transposed):
    off = ref.groups(counts)
    R, E = sum(counts), len(counts)
    T = 37 if gather else R
    a, w = rnd(R, T, K), rnd(R + 1, E, *((K, N) if transposed else (N, K)), scale=0.1)
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R)) if gather else None
    y, m = ref.product(a, w, off, rows, transposed)
    ga, gw, go, gr = gpu(a, w, off, rows)
    got = ex.grouped_matmul(ga, gw, go, gr, transposed=transposed)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())


@pytest.mark.parametrize("counts,H,F", [([1], 64, 16), ([0, 3, 0, 1], 72, 48), ([255, 256, 257, 0, 1], 200, 160),
                                        ([1] * 40, 520, 32), ([700], 128, 272), (ragged(24, 2000, 3), 1000, 208),
                                        (ragged(128, 1500, 9), 256, 64), ([2, 4, 0, 1, 1], 2048, 768)])
@pytest.mark.parametrize("checkpoint", [False, True])
def test_expert_up(ex, counts, H, F, checkpoint):
    off = ref.groups(counts)
    R, E, T = sum(counts), len(counts), 53
    x, w1 = rnd(R + H, T, H), rnd(R + F, E, 2 * F, H, scale=0.5 / H ** 0.5 * 2)
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R))
    z, m = ref.product(x, w1, off, rows)
    act = ref.swiglu(z)
    gx, gw, go, gr = gpu(x, w1, off, rows)
    got, kept = ex.expert_up(gx, gw, go, gr, checkpoint=checkpoint)
    ok(ex)
    d = 2 * H * U * m
    dg, du, gate, up = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    # |silu'| <= 1.1 and |silu(g)| <= |g|; the second-order term is dg du
    within(got, act, 1.1 * dg * up + gate * du + 2 * dg * du + (BF + FN) * act.abs())
    if checkpoint:
        # half a step, a step being at most 2/127 of the block's largest value
        top = (z.abs() + d).reshape(R, -1, 16).amax(-1, keepdim=True).expand(R, 2 * F // 16, 16).reshape(R, 2 * F)
        vals = kept.values()
        within(vals, z, top / 127 + d)
        assert torch.equal(vals.cpu().double(), ref.values(kept.codes.cpu(), kept.exponents.cpu()))
        # every block uses its range: the largest code is at least 63
        codes = kept.codes.cpu().int().reshape(R, -1, 16).abs().amax(-1)
        assert ((codes >= 63) & (codes <= 127)).all()


def test_checkpoint_format_is_exact(ex):
    """Blocks whose product is known exactly (one-hot rows times the weights): codes
    and exponents equal the definition's, at powers of two, at 127/128 of them,
    at ties, at zeros, at the ends of the range, and with NaN and infinities."""
    F, H, R = 64, 64, 64
    w = rnd(1, 1, 2 * F, H)
    w[0, :16, 0] = torch.tensor([1.984375 * 2.0 ** -i for i in range(16)]).bfloat16()
    w[0, :16, 1] = torch.tensor([1.9921875, 1.0, -1.0] + [2.0 ** -7 * (2 * i + 1) for i in range(13)]).bfloat16()
    w[0, :16, 2] = 0
    w[0, :16, 3] = torch.tensor([3e38] + [1e37] * 15).bfloat16()
    w[0, :16, 4] = torch.tensor([2.0 ** -120, 2.0 ** -126] + [2.0 ** -124] * 14).bfloat16()
    w[0, :16, 5] = torch.tensor([127.0] + [0.5 + i for i in range(15)]).bfloat16()
    # from here on every value of the block is a huge multiple, so that zero times it stays finite
    x = torch.eye(R, H).bfloat16()
    off = ref.groups([R])
    gx, gw, go = gpu(x, w, off)
    _, kept = ex.expert_up(gx, gw, go, checkpoint=True)
    ok(ex)
    codes, exps = ref.quantise(w[0].double().T.contiguous())
    assert torch.equal(kept.exponents.cpu(), exps)
    assert torch.equal(kept.codes.cpu(), codes)
    bad = x.clone()
    bad[3, 0] = float("nan")
    bad[4, 1] = float("inf")
    (gb,) = gpu(bad)
    _, kept = ex.expert_up(gb, gw, go, checkpoint=True)
    ok(ex)
    vals = kept.values().cpu()
    assert torch.isnan(vals[3]).all() and (kept.exponents[3] == 255).all()
    assert torch.isnan(vals[4, :16]).all()
    keep = [r for r in range(R) if r not in (3, 4)]
    assert torch.equal(vals[keep].double(), ref.values(codes, exps)[keep])


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("T,k,E,K,N", [(1, 1, 1, 8, 8), (1, 8, 128, 96, 264), (3, 2, 40, 64, 72), (300, 5, 24, 136, 520),
                                       (77, 12, 16, 48, 128), (2, 8, 64, 768, 2048)])
def test_grouped_matmul_join(ex, T, k, E, K, N, transposed, weighted):
    g = torch.Generator().manual_seed(T + N)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, _, pos = ref.dispatch(ids, E)
    a, w = rnd(T, T * k, K), rnd(N, E, *((K, N) if transposed else (N, K)), scale=0.1)
    c = torch.rand(T, k, generator=g) if weighted else None
    y, m = ref.product(a, w, off, None, transposed)
    cw = (c if weighted else torch.ones(T, k)).double().unsqueeze(-1)
    out = (y[pos] * cw).sum(1)
    bound = ((2 * K * U * m[pos] + (BF + 4 * k * U) * y[pos].abs()) * cw).sum(1) * (1 + BF) + BF * out.abs()
    ga, gw, go, gp, gc = gpu(a, w, off, pos, c)
    got = ex.grouped_matmul_join(ga, gw, go, gp, gc, transposed=transposed)
    ok(ex)
    within(got, out, bound)


@pytest.mark.parametrize("T,k,E,H,F", [(1, 1, 1, 8, 16), (1, 8, 128, 96, 64), (40, 3, 5, 72, 48), (700, 2, 9, 200, 272),
                                       (333, 5, 40, 1016, 208), (600, 1, 2, 128, 32)])
def test_expert_up_backward(ex, T, k, E, H, F):
    g = torch.Generator().manual_seed(T + F)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, rows, pos = ref.dispatch(ids, E)
    dout, w2 = rnd(1, T, H, scale=0.1), rnd(2, E, H, F, scale=0.1)
    combine = torch.rand(T, k, generator=g)
    codes, exps = ref.quantise(torch.randn(T * k, 2 * F, generator=g) * 2)
    z = ref.values(codes, exps)
    dz, act, dc, gr, gm, w, a1 = ref.up_backward(dout, w2, z, combine, off, rows, pos)
    gd, gw, gc, go, grw, gp, gco, gex = gpu(dout, w2, combine, off, rows, pos, codes, exps)
    kept = ex.Checkpoint(gco, gex)
    got_z, got_a, got_c = ex.expert_up_backward(gd, gw, kept, gc, go, grw, gp)
    ok(ex)
    d = 2 * H * U * gm
    gate, up = z[:, :F], z[:, F:].abs()
    s = torch.sigmoid(gate)
    slope = torch.cat([w * up * s * (1 + gate.abs() * (1 - s)), w * gate.abs() * s], 1)
    gg = torch.cat([gr, gr], 1).abs()
    # the gate's factor 1 + z (1 - s) is a difference where z < 0: its error is that of its terms
    within(got_z, dz, slope * torch.cat([d, d], 1) * 1.01 + 4 * FN * slope * gg + BF * dz.abs())
    within(got_a, act, (BF + 2 * FN) * act.abs())
    mag = (gr * a1).abs()
    bound = ((d * a1.abs()) * 1.01 + (2 * F * U + 2 * FN) * mag).sum(1)[pos]
    within(got_c, dc, bound)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("side", ["none", "p", "q"])
@pytest.mark.parametrize("counts,M,N", [([1], 8, 8), ([0, 3, 0, 0, 1], 64, 64), ([17, 0, 130, 16], 72, 136),
                                        ([255, 256, 257, 0, 1], 200, 264), (ragged(24, 2000, 3), 96, 520),
                                        ([64, 128, 63, 65, 0], 512, 40)])
def test_grouped_weight_grad(ex, counts, M, N, side, accumulate):
    off = ref.groups(counts)
    R, E, T = sum(counts), len(counts), 29
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R))
    p, q = rnd(M, T if side == "p" else R, M), rnd(N, T if side == "q" else R, N)
    pr, qr = (rows if side == "p" else None), (rows if side == "q" else None)
    pd, qd = (p[rows] if side == "p" else p).double(), (q[rows] if side == "q" else q).double()
    want = torch.stack([pd[int(off[e]):int(off[e + 1])].T @ qd[int(off[e]):int(off[e + 1])] for e in range(E)])
    mag = torch.stack([pd[int(off[e]):int(off[e + 1])].abs().T @ qd[int(off[e]):int(off[e + 1])].abs()
                       for e in range(E)])
    n = torch.tensor(counts, dtype=torch.float64).reshape(-1, 1, 1)
    base = torch.randn(E, M, N, generator=torch.Generator().manual_seed(7)) if accumulate else None
    gp, gq, go, gpr, gqr, gb = gpu(p, q, off, pr, qr, base)
    got = ex.grouped_weight_grad(gp, gq, go, gpr, gqr, out=gb, accumulate=accumulate)
    ok(ex)
    bound = 2 * n * U * mag
    if accumulate:
        want = want + base.double()
        bound = bound + 2 * U * (want.abs() + bound)
    within(got, want, bound)


def test_rows_past_the_groups_are_not_written(ex):
    counts, cap, K, N = [3, 0, 40], 64, 64, 48
    off = ref.groups(counts)
    a, w = rnd(1, cap, K), rnd(2, 3, N, K)
    ga, gw, go = gpu(a, w, off)
    from paper_2609_32398_gb300 import doloss as dl
    y = torch.full((cap, N), 7.0, dtype=torch.bfloat16, device="cuda")
    st = dl.lib().do_grouped_matmul(ga.data_ptr(), gw.data_ptr(), None, go.data_ptr(), cap, K, N, 3, cap, 0,
                                    y.data_ptr(), None, dl._stream(ga))
    assert st == 0
    torch.cuda.synchronize()
    want, m = ref.product(a[:43], w, off)
    within(y[:43], want, 2 * K * U * m + BF * want.abs())
    assert (y[43:] == 7).all()


def test_nan_stays_in_its_rows(ex):
    """A NaN row, the infinities of another expert's rows, and the weights of an
    expert without rows reach no other result."""
    counts, K, N = [5, 300, 0, 20], 136, 264
    off = ref.groups(counts)
    R = sum(counts)
    a, w, q = rnd(1, R, K), rnd(2, 4, N, K), rnd(3, R, 72)
    clean_y, m = ref.product(a, w, off)
    dirty = a.clone()
    dirty[7] = float("nan")
    dirty[304] = float("inf")
    wd = w.clone()
    wd[2] = float("nan")
    ga, gw, go, gq = gpu(dirty, wd, off, q)
    got = ex.grouped_matmul(ga, gw, go).cpu()
    keep = [r for r in range(R) if r not in (7, 304)]
    within(got[keep], clean_y[keep], (2 * K * U * m + BF * clean_y.abs())[keep])
    assert torch.isnan(got[7]).all() and not torch.isfinite(got[304]).any()
    dw = ex.grouped_weight_grad(ga, gq, go).cpu()
    assert torch.isfinite(dw[[0, 2, 3]]).all() and (dw[2] == 0).all() and torch.isnan(dw[1]).all()
    want = a[:5].double().T @ q[:5].double()
    within(dw[0], want, 10 * U * (a[:5].double().abs().T @ q[:5].double().abs()))
    ok(ex)


def test_rows_outside_the_matrix_are_zero_and_recorded(ex):
    counts, K, N, T = [3, 5], 64, 40, 9
    off = ref.groups(counts)
    a, w = rnd(1, T, K), rnd(2, 2, N, K)
    rows = torch.tensor([0, -1, 8, 9, 1, 2, 2 ** 31 - 1, 3])
    ga, gw, go, gr = gpu(a, w, off, rows)
    got = ex.grouped_matmul(ga, gw, go, gr)
    torch.cuda.synchronize()
    assert ex.device_status() == 1
    good = [0, 2, 4, 5, 7]
    r2 = rows.clone()
    r2[[1, 3, 6]] = 0
    y, m = ref.product(a, w, off, r2)
    within(got[good], y[good], (2 * K * U * m + BF * y.abs())[good])
    assert (got[[1, 3, 6]] == 0).all()
    assert ex.device_status() == 0


def test_positions_outside_the_rows_are_left_out(ex):
    T, k, E, K, N = 4, 2, 3, 32, 24
    ids = torch.tensor([[0, 1], [1, 2], [0, 2], [2, 1]])
    off, _, pos = ref.dispatch(ids, E)
    a, w, c = rnd(1, T * k, K), rnd(2, E, N, K), torch.rand(T, k, generator=torch.Generator().manual_seed(1))
    y, m = ref.product(a, w, off)
    p2 = pos.clone()
    p2[0, 1], p2[3, 0] = -5, 2 ** 31 - 1
    c2 = c.clone().double()
    c2[0, 1] = c2[3, 0] = 0
    ga, gw, go, gp, gc = gpu(a, w, off, p2, c)
    got = ex.grouped_matmul_join(ga, gw, go, gp, gc)
    torch.cuda.synchronize()
    assert ex.device_status() == 1
    out = (y[pos] * c2.unsqueeze(-1)).sum(1)
    bound = ((2 * K * U * m[pos] + 2 * BF * y[pos].abs()) * c2.unsqueeze(-1)).sum(1) + BF * out.abs()
    within(got, out, bound)


def test_results_are_the_same_on_every_run_and_stream(ex):
    counts, H, F = ragged(24, 900, 4), 136, 64
    off = ref.groups(counts)
    R = sum(counts)
    x, w1 = rnd(1, R, H), rnd(2, 24, 2 * F, H, scale=0.1)
    gx, gw, go = gpu(x, w1, off)
    a0, k0 = ex.expert_up(gx, gw, go, checkpoint=True)
    d0 = ex.grouped_weight_grad(gx, a0, go)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        a1, k1 = ex.expert_up(gx, gw, go, checkpoint=True)
        d1 = ex.grouped_weight_grad(gx, a1, go)
    side.synchronize()
    assert torch.equal(a0, a1) and torch.equal(k0.codes, k1.codes) and torch.equal(k0.exponents, k1.exponents)
    assert torch.equal(d0, d1)
    ok(ex)


def layer(seed, T, k, E, H, F):
    g = torch.Generator().manual_seed(seed)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, rows, pos = ref.dispatch(ids, E)
    combine = torch.softmax(torch.randn(T, k, generator=g), 1)
    return (rnd(seed, T, H), rnd(seed + 1, E, 2 * F, H, scale=1 / H ** 0.5), rnd(seed + 2, E, H, F, scale=1 / F ** 0.5),
            combine, off, rows, pos)


@pytest.mark.parametrize("T,k,E,H,F", [(1, 2, 4, 64, 32), (300, 4, 16, 128, 80), (65, 1, 8, 72, 48)])
def test_layer_and_its_gradients(ex, T, k, E, H, F):
    """expert_ffn against the 64-bit layer and its autograd.  Norms: each bf16
    rounding adds 2^-9 of a vector's norm at most and the checkpoint's error is
    at most 2^-7 of each block's largest value (about 1.2% of a normal vector's
    norm with F-independent factors below 3), so 2% for the output and 6% for
    the gradients hold every entry's share."""
    x, w1, w2, c, off, rows, pos = layer(T, T, k, E, H, F)
    dref = [t.double().requires_grad_() for t in (x, w1, w2, c)]
    out = ref.ffn(*dref, off, rows, pos)
    dout = rnd(5, T, H)
    grads = torch.autograd.grad(out, dref, dout.double())
    gx, gw1, gw2, gc, go, gr, gp, gd = gpu(x, w1, w2, c, off, rows, pos, dout)
    leaves = [t.requires_grad_() for t in (gx, gw1, gw2, gc)]
    got = ex.expert_ffn(*leaves, go, gr, gp)
    assert got.dtype == torch.bfloat16
    with torch.no_grad():
        assert torch.equal(ex.expert_ffn(gx, gw1, gw2, gc, go, gr, gp), got)
    g2 = torch.autograd.grad(got, leaves, gd)
    ok(ex)
    rel = lambda a, b: float((a.double().cpu() - b).norm() / b.norm())
    assert rel(got.detach(), out.detach()) < 0.02
    for a, b in zip(g2, grads):
        assert rel(a, b) < 0.06
    # the weights' gradients into fp32 buffers, twice
    bufs = (torch.zeros(E, 2 * F, H, device="cuda"), torch.zeros(E, H, F, device="cuda"))
    for _ in range(2):
        got = ex.expert_ffn(*leaves, go, gr, gp, main_grads=bufs)
        got.backward(gd)
    ok(ex)
    assert rel(bufs[0], 2 * grads[1]) < 0.06 and rel(bufs[1], 2 * grads[2]) < 0.06
    assert gw1.grad is None and gw2.grad is None


def test_combine_gradient_against_differences(ex):
    """The layer is linear in the combine weights: a central difference of the
    output along any direction is the directional derivative up to the outputs'
    rounding (2^-8 of each of k rows' magnitudes, both sides, over 2 h), and the
    checkpoint's error (2% of the norm of the terms)."""
    T, k, E, H, F = 40, 3, 8, 128, 64
    x, w1, w2, c, off, rows, pos = layer(11, T, k, E, H, F)
    gx, gw1, gw2, gc, go, gr, gp = gpu(x, w1, w2, c, off, rows, pos)
    gc.requires_grad_()
    out = ex.expert_ffn(gx, gw1, gw2, gc, go, gr, gp)
    dout = rnd(9, T, H).cuda()
    (dc,) = torch.autograd.grad(out, gc, dout)
    h = 0.25
    with torch.no_grad():
        for q in range(k):
            v = torch.zeros_like(gc)
            v[:, q] = 1
            hi = ex.expert_ffn(gx, gw1, gw2, (gc + h * v).contiguous(), go, gr, gp).double()
            lo = ex.expert_ffn(gx, gw1, gw2, (gc - h * v).contiguous(), go, gr, gp).double()
            diff = ((hi - lo) / (2 * h) * dout.double()).sum(1)
            noise = 2.0 ** -8 * ((hi.abs() + lo.abs()) / (2 * h) * dout.double().abs()).sum(1)
            got = dc[:, q].double()
            scale = float(diff.norm()) / T ** 0.5
            assert ((got - diff).abs() <= 2 * noise + 0.1 * scale).all()
    ok(ex)


def test_router_to_experts_training_step(ex):
    """The library's router, the layer and the DO-loss in one backward pass."""
    from paper_2609_32398_gb300 import doloss as dl

    T, H, F, E, k = 200, 64, 32, 16, 4
    x = rnd(1, T, H).cuda()
    wr = (torch.randn(E, H, generator=torch.Generator().manual_seed(2)) * 0.3).cuda().requires_grad_()
    w1, w2 = rnd(3, E, 2 * F, H, scale=0.1).cuda().requires_grad_(), rnd(4, E, H, F, scale=0.1).cuda().requires_grad_()
    z = x.float() @ wr.T
    ids, combine, route = dl.route(z, k)
    off, rows, pos = ex.dispatch_of(route)
    out = ex.expert_ffn(x, w1, w2, combine, off, rows, pos)
    loss = out.float().square().mean() + 1e-2 * dl.do_loss(z, k)
    loss.backward()
    ok(ex)
    ro, rr, rp = ref.dispatch(ids.cpu().long(), E)
    assert torch.equal(off.cpu().long(), ro) and torch.equal(rows.cpu().long(), rr)
    assert torch.equal(pos.cpu().long(), rp)
    want = ref.ffn(x.cpu().double(), w1.detach().cpu().double(), w2.detach().cpu().double(),
                   combine.detach().cpu().double(), ro, rr, rp)
    assert float((out.detach().cpu().double() - want).norm() / want.norm()) < 0.02
    for t in (wr, w1, w2):
        assert t.grad is not None and torch.isfinite(t.grad).all() and float(t.grad.abs().max()) > 0
