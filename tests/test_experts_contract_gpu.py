"""What the expert operators promise beside their formulas: routed rows and choices
that are left out, with the workspace of any content; gradients that are whole or
refused; checks of shapes; captures; the variants of every size; the layer entry by entry.
Bounds as in test_experts_gpu.py."""
import pytest
import torch

import experts_ref as ref
from test_experts_gpu import BF, FN, U, ex, gpu, layer, ok, rnd, within  # noqa: F401

pytestmark = pytest.mark.gpu


def raw(name, *args):
    """A call of the C ABI on the current stream: tensors by their address, a NULL for None."""
    from paper_2609_32398_gb300 import doloss as dl

    st = getattr(dl.lib(), name)(*[a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args],
                                 torch.cuda.current_stream().cuda_stream)
    assert st == 0, dl.status_string(st)


def of_nans(name, *sizes):
    """A workspace of that call that holds NaNs, and its size."""
    from paper_2609_32398_gb300 import doloss as dl

    n = getattr(dl.lib(), name)(*sizes)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda"), n


def recorded(status):
    from paper_2609_32398_gb300 import doloss as dl

    return dl.lib().do_device_status(status.data_ptr(), torch.cuda.current_stream().cuda_stream)


def word():
    return torch.zeros(64, dtype=torch.int32, device="cuda")


def chosen(seed, T, k, E):
    g = torch.Generator().manual_seed(seed)
    return torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])


def gradient_bounds(one, z, w2, F, H):
    """Bounds of dz, w act and dcombine by row, from ref.up_backward's results."""
    dz, act, _, g, gm, w, a = one
    d = 2 * H * U * gm
    gate, up = z[:, :F], z[:, F:].abs()
    s = torch.sigmoid(gate)
    slope = torch.cat([w * up * s * (1 + gate.abs() * (1 - s)), w * gate.abs() * s], 1)
    gg = torch.cat([g, g], 1).abs()
    return (slope * torch.cat([d, d], 1) * 1.01 + 4 * FN * slope * gg + BF * dz.abs(), (BF + 2 * FN) * act.abs(),
            ((d * a.abs()) * 1.01 + (2 * F * U + 2 * FN) * (g * a).abs()).sum(1))


@pytest.mark.parametrize("T,k", [(1, 8), (2, 8), (40, 3)])
@pytest.mark.parametrize("first", [5, 9])
@pytest.mark.parametrize("transposed", [False, True])
def test_join_with_the_offsets_of_a_slice(ex, T, k, first, transposed):  # noqa: F811
    """Offsets that begin above zero: choices before them are left out and recorded, whatever
    the workspace held."""
    E, K, N = 12, 72, 136
    off, _, pos = ref.dispatch(chosen(T + first, T, k, E), E)
    a, w = rnd(T, T * k, K), rnd(2, E, *((K, N) if transposed else (N, K)), scale=0.1)
    c = torch.rand(T, k, generator=torch.Generator().manual_seed(first))
    lo = int(off[first])
    assert lo > 0
    y, m = ref.product(a, w, off, None, transposed)
    cw = (c.double() * (pos >= lo)).unsqueeze(-1)
    out = (y[pos] * cw).sum(1)
    ga, gw, go, gp, gc = gpu(a, w[first:], off[first:], pos, c)
    ws, n = of_nans("do_grouped_matmul_join_workspace_size", T, k, N)
    got, status = torch.empty(T, N, dtype=torch.bfloat16, device="cuda"), word()
    raw("do_grouped_matmul_join", ga, gw, go, gp, gc, T, k, K, N, E - first, int(transposed), got, status, ws, n)
    assert recorded(status) == 1
    within(got, out, ((2 * (K + 2 * k) * U * m[pos]) * cw).sum(1) + BF * out.abs())


@pytest.mark.parametrize("R", [9, 16, 17, 90])
@pytest.mark.parametrize("gather", [False, True])
def test_products_with_the_offsets_of_a_slice(ex, R, gather):  # noqa: F811
    """Rows before offsets[0] are not written."""
    E, first, K, N, F, T = 6, 2, 72, 40, 48, 11
    g = torch.Generator().manual_seed(R)
    off = ref.groups(torch.bincount(torch.randint(0, E, (R,), generator=g), minlength=E).tolist())
    lo = int(off[first])
    assert 0 < lo < R
    a, w, w1 = rnd(1, T if gather else R, K), rnd(2, E, N, K, scale=0.2), rnd(3, E, 2 * F, K, scale=0.2)
    rows = torch.randint(0, T, (R,), generator=g) if gather else None
    y, m = ref.product(a, w, off, rows)
    z, mz = ref.product(a, w1, off, rows)
    act = ref.swiglu(z)
    ga, gw, gw1, go, gr = gpu(a, w[first:], w1[first:], off[first:], rows)
    got = torch.full((R, N), 7.0, dtype=torch.bfloat16, device="cuda")
    up = torch.full((R, F), 7.0, dtype=torch.bfloat16, device="cuda")
    raw("do_grouped_matmul", ga, gw, gr, go, a.shape[0], K, N, E - first, R, 0, got, None)
    raw("do_expert_up", ga, gw1, gr, go, a.shape[0], K, F, E - first, R, up, None, None, None)
    assert (got[:lo] == 7).all() and (up[:lo] == 7).all()
    within(got[lo:], y[lo:], (2 * K * U * m + BF * y.abs())[lo:])
    d = 2 * K * U * mz
    dg, du, gate, u = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    within(up[lo:], act[lo:], (1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs())[lo:])


@pytest.mark.parametrize("T,k,F", [(1, 8, 48), (40, 3, 208)])
def test_gradient_with_the_offsets_of_a_slice(ex, T, k, F):  # noqa: F811
    E, first, H = 12, 6, 72
    off, rows, pos = ref.dispatch(chosen(T, T, k, E), E)
    R, lo = T * k, int(off[first])
    assert 0 < lo < R
    dout, w2 = rnd(1, T, H, scale=0.1), rnd(2, E, H, F, scale=0.1)
    c = torch.rand(T, k, generator=torch.Generator().manual_seed(k))
    codes, exps = ref.quantise(torch.randn(R, 2 * F, generator=torch.Generator().manual_seed(F)) * 2)
    z = ref.values(codes, exps)
    one = ref.up_backward(dout, w2, z, c, off, rows, pos)
    bz, ba, bc = gradient_bounds(one, z, w2, F, H)
    gd, gw, gco, gex, gc, grw, go, gp = gpu(dout, w2[first:], codes, exps, c, rows, off[first:], pos)
    ws, n = of_nans("do_expert_up_backward_workspace_size", T, k, F)
    dz = torch.full((R, 2 * F), 7.0, dtype=torch.bfloat16, device="cuda")
    act = torch.full((R, F), 7.0, dtype=torch.bfloat16, device="cuda")
    dc, status = torch.empty(T, k, device="cuda"), word()
    raw("do_expert_up_backward", gd, gw, gco, gex, gc, grw, go, gp, T, k, H, F, E - first, dz, act, dc, status, ws, n)
    assert recorded(status) == 1
    assert (dz[:lo] == 7).all() and (act[:lo] == 7).all()
    within(dz[lo:], one[0][lo:], bz[lo:])
    within(act[lo:], one[1][lo:], ba[lo:])
    kept = pos >= lo
    within(dc, torch.where(kept, one[2], 0.0), torch.where(kept, bc[pos], 0.0))


def test_a_choice_left_out_of_the_gradient(ex):  # noqa: F811
    """A position outside the rows: the routed row that it should have named has no weight, so
    that its dz and act are zeros, and nothing else changes."""
    T, k, E, H, F = 40, 3, 5, 72, 208
    off, rows, pos = ref.dispatch(chosen(1, T, k, E), E)
    R = T * k
    dout, w2, x = rnd(1, T, H, scale=0.1), rnd(2, E, H, F, scale=0.1), rnd(3, T, H)
    c = torch.rand(T, k, generator=torch.Generator().manual_seed(k))
    codes, exps = ref.quantise(torch.randn(R, 2 * F, generator=torch.Generator().manual_seed(F)) * 2)
    bad = pos.clone()
    gone = [int(pos[0, 1]), int(pos[31, 0])]
    bad[0, 1], bad[31, 0] = -5, 2 ** 31 - 1
    gd, gw, gco, gex, gc, grw, go, gp, gb, gx = gpu(dout, w2, codes, exps, c, rows, off, pos, bad, x)

    def run(p, status):
        ws, n = of_nans("do_expert_up_backward_workspace_size", T, k, F)
        dz = torch.full((R, 2 * F), 7.0, dtype=torch.bfloat16, device="cuda")
        act, dc = torch.full((R, F), 7.0, dtype=torch.bfloat16, device="cuda"), torch.empty(T, k, device="cuda")
        raw("do_expert_up_backward", gd, gw, gco, gex, gc, grw, go, p, T, k, H, F, E, dz, act, dc, status, ws, n)
        return dz, act, dc

    status = word()
    dz, act, dc = run(gp, status)
    assert recorded(status) == 0
    want = [t.clone() for t in (dz, act, dc)]
    want[0][gone] = 0
    want[1][gone] = 0
    want[2][0, 1] = want[2][31, 0] = 0
    got = run(gb, status)
    assert recorded(status) == 1
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for grad in (lambda z, a: ex.grouped_weight_grad(z, gx, go, None, grw),
                 lambda z, a: ex.grouped_weight_grad(gd, a, go, grw, None)):
        assert torch.equal(grad(*got[:2]), grad(*want[:2]))
    ok(ex)


def test_a_second_derivative_is_refused(ex):  # noqa: F811
    """The layer has no second derivative: a graph through its gradient raises instead of
    leaving its terms out."""
    x, w1, w2, c, off, rows, pos = layer(3, 20, 2, 4, 64, 32)
    gx, gw1, gw2, gc, go, gr, gp = gpu(x, w1, w2, c, off, rows, pos)
    leaves = [t.requires_grad_() for t in (gx, gw1, gw2, gc)]
    out = ex.expert_ffn(*leaves, go, gr, gp).float().sum()
    (dx,) = torch.autograd.grad(out, gx, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        (out + dx.float().square().sum()).backward()
    ok(ex)


def test_shapes_are_checked_alike_with_and_without_gradients(ex):  # noqa: F811
    T, k, E, H, F = 20, 2, 4, 64, 32
    x, w1, w2, c, off, rows, pos = layer(5, T, k, E, H, F)
    gx, gw1, gw2, gc, go, gr, gp = gpu(x, w1, w2, c, off, rows, pos)
    good = dict(x=gx, w1=gw1, w2=gw2, combine=gc, offsets=go, rows=gr, pos=gp)
    bad = [dict(pos=gp.T.contiguous()), dict(combine=gc.T.contiguous()), dict(combine=gc.reshape(-1)),
           dict(w2=rnd(1, E, H + 8, F).cuda()), dict(w2=rnd(1, E + 1, H, F).cuda()), dict(w1=rnd(1, E, 2 * F, H + 8).cuda()),
           dict(x=rnd(1, T + 1, H).cuda()), dict(rows=gr[:-1])]
    for train in (False, True):
        for t in (gx, gw1, gw2, gc):
            t.requires_grad_(train)
        for change in bad:
            with pytest.raises(ValueError):
                ex.expert_ffn(**{**good, **change})
    # the positions in one dimension are the same memory
    flat = {**good, "pos": gp.reshape(-1)}
    want = ex.expert_ffn(**good)
    assert torch.equal(ex.expert_ffn(**flat), want)
    with torch.no_grad():
        assert torch.equal(ex.expert_ffn(**flat), ex.expert_ffn(**good))
    codes, exps = ref.quantise(torch.randn(T * k, 2 * F, generator=torch.Generator().manual_seed(1)))
    kept = ex.Checkpoint(*gpu(codes, exps))
    with torch.no_grad(), pytest.raises(ValueError):
        ex.expert_up_backward(gx, gw2, kept, gc, go, gr, gp.T.contiguous())
    ok(ex)


def test_buffers_of_the_weights_gradients_are_checked_in_the_forward_call(ex):  # noqa: F811
    T, k, E, H, F = 20, 2, 4, 64, 32
    x, w1, w2, c, off, rows, pos = layer(5, T, k, E, H, F)
    args = gpu(x, w1, w2, c, off, rows, pos)
    bufs = (torch.zeros(E, 2 * F, H, device="cuda"), torch.zeros(E, H, F, device="cuda"))
    for train in (False, True):
        for t in args[:4]:
            t.requires_grad_(train)
        for bad in (bufs[::-1], (bufs[0], bufs[1].half()), bufs[:1], (bufs[0], bufs[1].cpu()), (None, bufs[1]),
                    (bufs[0].transpose(1, 2).contiguous().transpose(1, 2), bufs[1])):
            with pytest.raises(ValueError):
                ex.expert_ffn(*args, main_grads=bad)
        ex.expert_ffn(*args, main_grads=bufs)
    ok(ex)


def test_a_layer_without_choices_has_gradients(ex):  # noqa: F811
    """k = 0: zeros, and zeros for gradients."""
    T, E, H, F = 6, 4, 64, 32
    x, w1, w2 = rnd(1, T, H), rnd(2, E, 2 * F, H), rnd(3, E, H, F)
    none = torch.zeros(T, 0, dtype=torch.int64)
    gx, gw1, gw2, gc, go, gr, gp = gpu(x, w1, w2, torch.zeros(T, 0), torch.zeros(E + 1, dtype=torch.int64),
                                       none.reshape(-1), none)
    leaves = [t.requires_grad_() for t in (gx, gw1, gw2, gc)]
    out = ex.expert_ffn(*leaves, go, gr, gp)
    assert out.shape == (T, H) and (out == 0).all()
    for g, t in zip(torch.autograd.grad(out, leaves, torch.ones_like(out)), leaves):
        assert g.shape == t.shape and (g == 0).all()
    ok(ex)


@pytest.mark.parametrize("frozen", [0, 1])
def test_a_frozen_weight_takes_no_gradient(ex, frozen):  # noqa: F811
    """Weights that require no gradient leave their buffer of main_grads as it was."""
    x, w1, w2, c, off, rows, pos = layer(7, 30, 2, 4, 64, 32)
    gx, gw1, gw2, gc, go, gr, gp = gpu(x, w1, w2, c, off, rows, pos)
    for t in (gx, gw1, gw2, gc):
        t.requires_grad_()
    full = [torch.full(w.shape, 2.0, device="cuda") for w in (gw1, gw2)]
    ex.expert_ffn(gx, gw1, gw2, gc, go, gr, gp, main_grads=tuple(full)).float().sum().backward()
    (gw1, gw2)[frozen].requires_grad_(False)
    bufs = [torch.full(w.shape, 2.0, device="cuda") for w in (gw1, gw2)]
    ex.expert_ffn(gx, gw1, gw2, gc, go, gr, gp, main_grads=tuple(bufs)).float().sum().backward()
    assert (bufs[frozen] == 2.0).all()
    assert torch.equal(bufs[1 - frozen], full[1 - frozen]) and not (full[1 - frozen] == 2.0).all()
    ok(ex)


def test_the_first_call_of_a_capture_is_refused_in_words(ex, monkeypatch):  # noqa: F811
    """The device's status word is made by the first call, which a capture cannot hold: it is
    refused before anything is captured, and the capture goes on."""
    x, w = rnd(1, 20, 64), rnd(2, 1, 40, 64)
    gx, gw, go = gpu(x, w, ref.groups([20]))
    want = ex.grouped_matmul(gx, gw, go)
    ok(ex)
    with monkeypatch.context() as m:
        m.setattr(ex, "_flags", {})
        m.setattr(ex, "_flag_ptrs", {})
        graph, other = torch.cuda.CUDAGraph(), torch.zeros(8, device="cuda")
        with torch.cuda.graph(graph):
            with pytest.raises(RuntimeError, match="capture"):
                ex.grouped_matmul(gx, gw, go)
            other += 1
        graph.replay()
        torch.cuda.synchronize()
        assert (other == 1).all()
        assert ex.device_status() == 0        # makes the word
        with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
            got = ex.grouped_matmul(gx, gw, go)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        ok(ex)


@pytest.mark.parametrize("T,k,N", [(3100, 8, 1032), (2100, 12, 1032), (1600, 4, 4104), (3100, 4, 2056), (300, 4, 4104),
                                   (90, 9, 2056)])
@pytest.mark.parametrize("weighted", [False, True])
def test_wide_and_long_joins(ex, T, k, N, weighted):  # noqa: F811
    """Both sides of the 25,165,824 values up to which joined rows are kept in fp32, columns
    past 2048 and more than eight choices."""
    E, K = 24, 16
    off, _, pos = ref.dispatch(chosen(T + N, T, k, E), E)
    a, w = rnd(T, T * k, K), rnd(N, E, N, K, scale=0.3)
    c = torch.rand(T, k, generator=torch.Generator().manual_seed(T)) if weighted else None
    y, m = ref.product(a, w, off)
    cw = (c if weighted else torch.ones(T, k)).double()
    out, bound = torch.zeros(T, N, dtype=torch.float64), torch.zeros(T, N, dtype=torch.float64)
    rounded = BF if T * k * N > (96 << 20) // 4 else 0.0     # of each row, before the sum
    for q in range(k):
        out += y[pos[:, q]] * cw[:, q:q + 1]
        bound += (2 * (K + 2 * k) * U * m[pos[:, q]] + rounded * y[pos[:, q]].abs()) * cw[:, q:q + 1]
    ga, gw, go, gp, gc = gpu(a, w, off, pos, c)
    got = ex.grouped_matmul_join(ga, gw, go, gp, gc)
    ok(ex)
    within(got, out, bound * (1 + BF) + BF * out.abs())


@pytest.mark.parametrize("K", [8, 264, 512, 520, 776, 1024, 1032, 2048, 2056, 4104])
@pytest.mark.parametrize("R", [1, 7, 16])
@pytest.mark.parametrize("gather", [False, True])
def test_products_of_few_rows(ex, K, R, gather):  # noqa: F811
    """Few rows with contractions at the edges of every variant, and odd numbers of columns."""
    E, N, F, T = 5, 104, 112, 6
    g = torch.Generator().manual_seed(K + R)
    off = ref.groups(torch.bincount(torch.randint(0, E, (R,), generator=g), minlength=E).tolist())
    a, w, w1 = rnd(K, T if gather else R, K), rnd(R, E, N, K, scale=0.1), rnd(R + 1, E, 2 * F, K, scale=1 / K ** 0.5)
    rows = torch.randint(0, T, (R,), generator=g) if gather else None
    y, m = ref.product(a, w, off, rows)
    z, mz = ref.product(a, w1, off, rows)
    act = ref.swiglu(z)
    ga, gw, gw1, go, gr = gpu(a, w, w1, off, rows)
    got = ex.grouped_matmul(ga, gw, go, gr)
    up, _ = ex.expert_up(ga, gw1, go, gr)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())
    d = 2 * K * U * mz
    dg, du, gate, u = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    within(up, act, 1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs())


@pytest.mark.parametrize("K", [768, 776, 1536, 4104])
@pytest.mark.parametrize("T,k", [(1, 1), (1, 5), (2, 8), (1, 16)])
def test_joins_of_few_rows_over_long_contractions(ex, K, T, k):  # noqa: F811
    E, N = 20, 72
    off, _, pos = ref.dispatch(chosen(K, T, k, E), E)
    a, w, c = rnd(T, T * k, K), rnd(2, E, N, K, scale=0.1), torch.rand(T, k, generator=torch.Generator().manual_seed(K))
    y, m = ref.product(a, w, off)
    cw = c.double().unsqueeze(-1)
    out = (y[pos] * cw).sum(1)
    ga, gw, go, gp, gc = gpu(a, w, off, pos, c)
    got = ex.grouped_matmul_join(ga, gw, go, gp, gc)
    ok(ex)
    within(got, out, ((2 * (K + 2 * k) * U * m[pos]) * cw).sum(1) + BF * out.abs())


@pytest.mark.parametrize("T,k,E,H,F", [(60, 3, 8, 136, 80), (300, 2, 5, 72, 208), (2, 8, 16, 264, 48)])
def test_every_entry_of_the_layers_gradients(ex, T, k, E, H, F):  # noqa: F811
    """The layer's output and gradients entry by entry, in 64 bits from its own checkpoint: which
    operand goes into which product, with which rounding.  dz and w act are bf16, dW and the
    joined rows (few here) fp32, dx is rounded once."""
    x, w1, w2, c, off, rows, pos = layer(T + F, T, k, E, H, F)
    dout = rnd(T, T, H)
    gx, gw1, gw2, gc, go, gr, gp, gd = gpu(x, w1, w2, c, off, rows, pos, dout)
    _, kept = ex.expert_up(gx, gw1, go, gr, checkpoint=True)
    zk = ref.values(kept.codes.cpu(), kept.exponents.cpu())
    leaves = [t.requires_grad_() for t in (gx, gw1, gw2, gc)]
    out = ex.expert_ffn(*leaves, go, gr, gp)
    dx, dw1, dw2, dc = torch.autograd.grad(out, leaves, gd)
    ok(ex)
    # the output: act from the exact z, rounded to bf16
    z, mz = ref.product(x, w1, off, rows)
    act = ref.swiglu(z)
    d = 2 * H * U * mz
    dg, du, gate, u = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    ba = 1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs()
    cw = c.double().unsqueeze(-1)
    y = ref.each(off, H, T * k, lambda e, i, j: act[i:j] @ w2[e].double().T)
    by = ref.each(off, H, T * k, lambda e, i, j: (ba[i:j] + 2 * (F + 2 * k) * U * act[i:j].abs()) * 1.01
                  @ w2[e].double().abs().T)
    want = (y[pos] * cw).sum(1)
    within(out.detach(), want, (by[pos] * cw).sum(1) + BF * want.abs())
    # the gradients, from the checkpoint's z
    one = ref.up_backward(dout, w2, zk, c, off, rows, pos)
    dz, wact = one[0], one[1]
    bz, bw, bc = gradient_bounds(one, zk, w2, F, H)
    within(dc, one[2], bc[pos])
    xr, dr = x[rows].double(), dout[rows].double()
    w1d = w1.double()
    for e in range(E):
        i, j = int(off[e]), int(off[e + 1])
        n = max(j - i, 1)
        # the returned gradients have the leaves' type: one more rounding to bf16
        g1, g2 = dz[i:j].T @ xr[i:j], dr[i:j].T @ wact[i:j]
        e1 = (bz[i:j] + 2 * n * U * dz[i:j].abs()).T * 1.01 @ xr[i:j].abs()
        e2 = dr[i:j].abs().T @ (bw[i:j] + 2 * n * U * wact[i:j].abs()) * 1.01
        within(dw1[e], g1, e1 * (1 + BF) + BF * g1.abs())
        within(dw2[e], g2, e2 * (1 + BF) + BF * g2.abs())
    v = ref.each(off, H, T * k, lambda e, i, j: dz[i:j] @ w1d[e])
    bv = ref.each(off, H, T * k, lambda e, i, j: (bz[i:j] + 2 * (2 * F + 2 * k) * U * dz[i:j].abs()) * 1.01
                  @ w1d[e].abs())
    want = v[pos].sum(1)
    within(dx, want, bv[pos].sum(1) * (1 + BF) + BF * want.abs())


def test_weight_gradient_of_a_collapsed_router(ex):  # noqa: F811
    """131072 rows of one expert.  A step of 16 rows is one addition to the fp32 accumulator:
    each of its 17 terms loses at most a unit in the last of 24 bits of the largest, so 2 * 17 U of
    the partial sum's and the step's magnitudes (the running error bound)."""
    n, M, N = 131072, 64, 48
    p, q = rnd(1, n, M), rnd(2, n, N)
    gp, gq, go = gpu(p, q, ref.groups([n, 0]))
    dw = ex.grouped_weight_grad(gp, gq, go)
    ok(ex)
    ps, qs = p.double().reshape(-1, 16, M), q.double().reshape(-1, 16, N)
    steps = torch.bmm(ps.transpose(1, 2), qs)
    mags = torch.bmm(ps.abs().transpose(1, 2), qs.abs())
    sums = torch.cumsum(steps, 0)
    within(dw[0], sums[-1], 34 * U * (sums.abs() + mags).sum(0))
    assert (dw[1] == 0).all()


@pytest.mark.parametrize("n", [16384, 131072])
@pytest.mark.parametrize("positive", [False, True])
def test_long_weight_gradients_keep_fp32s_precision(ex, n, positive):  # noqa: F811
    """However many rows an expert has, an accumulator takes at most 2048 of them: 128 additions of
    16 rows, each losing at most a unit in the last place (2^-23) of the partial sum.  Those grow as
    the root of the rows, or with them where all terms are positive, so that an accumulator is off by
    128 * 2/3 * 2^-23 of its value at most, and the fp32 sum of the n / 2048 of them by another
    n / 2048 * 2/3 * 2^-24."""
    p, q = rnd(n, n, 64), rnd(n + 1, n, 48)
    if positive:
        p, q = p.abs(), q.abs()
    gp, gq, go = gpu(p, q, ref.groups([0, n]))
    want = p.double().T @ q.double()
    tolerance = 2 / 3 * (128 * 2.0 ** -23 + n / 2048 * 2.0 ** -24)
    dw = ex.grouped_weight_grad(gp, gq, go)
    ok(ex)
    assert float((dw[1].double().cpu() - want).norm() / want.norm()) <= tolerance
    assert (dw[0] == 0).all()
    # added to a gradient of the same size: the sum is twice as large, and so may the error be
    total = ex.grouped_weight_grad(gp, gq, go, out=dw.clone(), accumulate=True)
    ok(ex)
    assert float((total[1].double().cpu() - 2 * want).norm() / (2 * want).norm()) <= tolerance
    for _ in range(3):
        assert torch.equal(ex.grouped_weight_grad(gp, gq, go), dw)
        assert torch.equal(ex.grouped_weight_grad(gp, gq, go, out=dw.clone(), accumulate=True), total)


@pytest.mark.parametrize("n", [2047, 2048, 2049, 2111, 4096, 4097, 6145])
@pytest.mark.parametrize("side", ["none", "p", "q"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_weight_gradients_at_the_accumulators_edges(ex, n, side, accumulate):  # noqa: F811
    """Groups of one accumulator, of several, and of none in turn, on more tiles than pairs."""
    counts, M, N, T = [3, n, 0, n + 64, 1, 2 * n], 264, 520, 37
    off = ref.groups(counts)
    R = sum(counts)
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(n))
    p, q = rnd(n, T if side == "p" else R, M), rnd(n + 1, T if side == "q" else R, N)
    base = torch.randn(6, M, N, generator=torch.Generator().manual_seed(7)) if accumulate else None
    gp, gq, go, gr, gb = gpu(p, q, off, rows, base)
    got = ex.grouped_weight_grad(gp, gq, go, gr if side == "p" else None, gr if side == "q" else None, out=gb,
                                 accumulate=accumulate)
    ok(ex)
    pd, qd = (p[rows] if side == "p" else p).double(), (q[rows] if side == "q" else q).double()
    for e, m in enumerate(counts):
        i, j = int(off[e]), int(off[e + 1])
        want, mag = pd[i:j].T @ qd[i:j], pd[i:j].abs().T @ qd[i:j].abs()
        bound = 2 * m * U * mag
        if accumulate:
            want = want + base[e].double()
            bound = bound + 4 * U * (want.abs() + base[e].abs().double() + bound)
        within(got[e], want, bound)
