"""The expert operators where they can go wrong: group sizes at the tiles' edges,
many experts, both sides of the few-row kernels' line, results past 2^31 values,
blocks of zeros and of NaNs, windows without rows, and graph replays.  Bounds as
in test_experts_gpu.py."""
import pytest
import torch

import experts_ref as ref
from test_experts_gpu import BF, FN, U, ex, gpu, ok, rnd, within  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [15, 16, 17, 31, 32, 33, 127, 129, 239, 240, 241, 255, 256, 257, 272, 511, 512, 513, 769])
@pytest.mark.parametrize("gather", [False, True])
def test_group_sizes_at_the_tiles_edges(ex, n, gather):  # noqa: F811
    counts, K, N = [n, 1, n + 1, 0, 2], 72, 272
    off = ref.groups(counts)
    R, T = sum(counts), 50
    a = rnd(n, T if gather else R, K)
    w, w1 = rnd(n + 1, 5, N, K, scale=0.2), rnd(n + 2, 5, 2 * 144, K, scale=0.2)
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(n)) if gather else None
    y, m = ref.product(a, w, off, rows)
    z, mz = ref.product(a, w1, off, rows)
    act = ref.swiglu(z)
    q = rnd(n + 3, R, 40)
    ga, gw, gw1, go, gr, gq = gpu(a, w, w1, off, rows, q)
    got = ex.grouped_matmul(ga, gw, go, gr)
    up, kept = ex.expert_up(ga, gw1, go, gr, checkpoint=True)
    dw = ex.grouped_weight_grad(ga, gq, go, gr, None)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())
    d = 2 * K * U * mz
    dg, du, gate, u = d[:, :144], d[:, 144:], z[:, :144].abs(), z[:, 144:].abs()
    within(up, act, 1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs())
    top = (z.abs() + d).reshape(R, -1, 16).amax(-1, keepdim=True).expand(R, 18, 16).reshape(R, 288)
    within(kept.values(), z, top / 127 + d)
    ad = (a if rows is None else a[rows]).double()
    for e in range(5):
        i, j = int(off[e]), int(off[e + 1])
        within(dw[e], ad[i:j].T @ q[i:j].double(), 2 * (j - i) * U * (ad[i:j].abs().T @ q[i:j].double().abs()))


@pytest.mark.parametrize("R", [16, 17, 24, 25, 900])
@pytest.mark.parametrize("gather", [False, True])
def test_many_experts_and_both_sides_of_the_few_row_line(ex, R, gather):  # noqa: F811
    E, K, N = 1024, 136, 72
    g = torch.Generator().manual_seed(R)
    picks = torch.sort(torch.randint(0, E, (R,), generator=g))[0]
    picks[-1] = E - 1
    off = ref.groups(torch.bincount(picks, minlength=E).tolist())
    a = rnd(1, 11 if gather else R, K)
    w, w1 = rnd(2, E, N, K, scale=0.2), rnd(3, E, 2 * 48, K, scale=0.2)
    rows = torch.randint(0, 11, (R,), generator=g) if gather else None
    y, m = ref.product(a, w, off, rows)
    z, mz = ref.product(a, w1, off, rows)
    act = ref.swiglu(z)
    ga, gw, gw1, go, gr = gpu(a, w, w1, off, rows)
    got = ex.grouped_matmul(ga, gw, go, gr)
    up, _ = ex.expert_up(ga, gw1, go, gr)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())
    d = 2 * K * U * mz
    dg, du, gate, u = d[:, :48], d[:, 48:], z[:, :48].abs(), z[:, 48:].abs()
    within(up, act, 1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs())
    dw = ex.grouped_weight_grad(ga, up, go, gr, None)
    ok(ex)
    e = E - 1
    i, j = int(off[e]), int(off[e + 1])
    ad = (a if rows is None else a[rows]).double()
    ud = up.double().cpu()
    within(dw[e], ad[i:j].T @ ud[i:j], 2 * (j - i) * U * (ad[i:j].abs().T @ ud[i:j].abs()))


@pytest.mark.parametrize("T,k", [(1, 16), (2, 12), (24, 1), (25, 1), (3, 5), (2, 8), (3, 4), (1, 17)])
def test_join_of_few_rows(ex, T, k):  # noqa: F811
    E, K, N = 40, 776, 136
    g = torch.Generator().manual_seed(T + k)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, _, pos = ref.dispatch(ids, E)
    a, w, c = rnd(T, T * k, K), rnd(2, E, N, K, scale=0.1), torch.rand(T, k, generator=g)
    y, m = ref.product(a, w, off)
    cw = c.double().unsqueeze(-1)
    out = (y[pos] * cw).sum(1)
    ga, gw, go, gp, gc = gpu(a, w, off, pos, c)
    got = ex.grouped_matmul_join(ga, gw, go, gp, gc)
    ok(ex)
    # the rows stay in fp32 here: one rounding
    bound = ((2 * (K + 2 * k) * U * m[pos]) * cw).sum(1) + BF * out.abs()
    within(got, out, bound)


def test_results_past_two_to_the_31_values(ex):  # noqa: F811
    """R N > 2^31: rows at the far end of the result are the right ones."""
    counts, K, N = [700_000, 1, 400_000], 8, 2056
    R = sum(counts)
    assert R * N > 2 ** 31
    off = ref.groups(counts)
    ga = torch.randn(R, K, generator=torch.Generator("cuda").manual_seed(1), device="cuda").bfloat16()
    w = rnd(2, 3, N, K)
    gw, go = gpu(w, off)
    got = ex.grouped_matmul(ga, gw, go)
    ok(ex)
    for r, e in ((0, 0), (699_999, 0), (700_000, 1), (700_001, 2), (R - 300, 2), (R - 1, 2)):
        a = ga[r].double().cpu()
        want, m = w[e].double() @ a, w[e].double().abs() @ a.abs()
        within(got[r], want, 2 * K * U * m + BF * want.abs())


def test_a_checkpoint_past_two_to_the_31_values(ex):  # noqa: F811
    T, k, H, F = 550_000, 2, 8, 1024
    R = T * k
    assert R * 2 * F > 2 ** 31
    g = torch.Generator("cuda").manual_seed(3)
    counts = [R - 70_001, 0, 70_001]
    off = ref.groups(counts)
    rows = torch.arange(R, device="cuda", dtype=torch.int32) % T
    pos = torch.arange(R, device="cuda", dtype=torch.int32).reshape(k, T).T.contiguous()
    x = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    w1, w2 = rnd(4, 3, 2 * F, H, scale=0.5), rnd(5, 3, H, F, scale=0.5)
    c = torch.rand(T, k, generator=g, device="cuda")
    dout = torch.randn(T, H, generator=g, device="cuda").bfloat16()
    gw1, gw2, go = gpu(w1, w2, off)
    act, kept = ex.expert_up(x, gw1, go, rows, checkpoint=True)
    dz, wa, dc = ex.expert_up_backward(dout, gw2, kept, c, go, rows, pos)
    ok(ex)
    for r in (0, 1_000_000, R - 70_001, R - 2, R - 1):
        e = 0 if r < counts[0] else 2
        t, q = r % T, r // T
        z = w1[e].double() @ x[t].double().cpu()
        m = w1[e].double().abs() @ x[t].double().cpu().abs()
        d = 2 * H * U * m
        a = ref.swiglu(z.unsqueeze(0))[0]
        within(act[r], a, 1.1 * d[:F] * z[F:].abs() + z[:F].abs() * d[F:] + 2 * d[:F] * d[F:] + (BF + FN) * a.abs())
        zk = ref.values(kept.codes[r:r + 1].cpu(), kept.exponents[r:r + 1].cpu())
        one = ref.up_backward(dout[t:t + 1].cpu(), w2[e:e + 1], zk, c[t:t + 1, q:q + 1].cpu(), ref.groups([1]),
                              torch.zeros(1, dtype=torch.int64), torch.zeros(1, 1, dtype=torch.int64))
        want, gw, gm, a1 = one[0], one[3], one[4], one[6]
        gate, up = zk[:, :F], zk[:, F:].abs()
        s = torch.sigmoid(gate)
        slope = torch.cat([up * s * (1 + gate.abs() * (1 - s)), gate.abs() * s], 1) * float(c[t, q])
        gd = 2 * H * U * gm
        within(dz[r:r + 1], want, slope * torch.cat([gd, gd], 1) * 1.01 + 4 * FN * slope * torch.cat([gw, gw], 1).abs()
               + BF * want.abs())
        within(wa[r:r + 1], one[1], (BF + 2 * FN) * one[1].abs())
        bound = (gd * a1.abs() * 1.01 + (2 * F * U + 2 * FN) * (gw * a1).abs()).sum()
        assert abs(float(dc[t, q]) - float(one[2])) <= float(bound)


def test_weight_gradients_past_two_to_the_31_values(ex):  # noqa: F811
    E, M, N, R = 520, 2048, 2048, 12
    assert E * M * N > 2 ** 31
    counts = [3] + [0] * (E - 2) + [9]
    off = ref.groups(counts)
    p, q = rnd(1, R, M), rnd(2, R, N)
    gp, gq, go = gpu(p, q, off)
    dw = ex.grouped_weight_grad(gp, gq, go)
    ok(ex)
    for e, i, j in ((0, 0, 3), (E - 1, 3, 12)):
        want = p[i:j].double().T @ q[i:j].double()
        within(dw[e], want, 2 * (j - i) * U * (p[i:j].double().abs().T @ q[i:j].double().abs()))
    assert float(dw[1:E - 1].abs().max()) == 0.0


def test_blocks_of_zeros_and_of_nans(ex):  # noqa: F811
    """A row of zeros keeps exponent 1 and codes 0; a NaN block of a checkpoint makes
    its own 16 columns and its own row's combine gradient NaN, nothing else."""
    T, k, E, H, F = 40, 1, 2, 64, 48
    off, rows, pos = ref.dispatch((torch.arange(T) % E).reshape(T, 1), E)
    x, w1, w2 = rnd(1, T, H), rnd(2, E, 2 * F, H, scale=0.2), rnd(3, E, H, F, scale=0.2)
    x[5] = 0
    dout, c = rnd(4, T, H), torch.rand(T, k, generator=torch.Generator().manual_seed(1))
    gx, gw1, gw2, go, gr, gp, gd, gc = gpu(x, w1, w2, off, rows, pos, dout, c)
    act, kept = ex.expert_up(gx, gw1, go, gr, checkpoint=True)
    ok(ex)
    r = int(pos[5, 0])
    assert (kept.codes[r] == 0).all() and (kept.exponents[r] == 1).all() and (act[r] == 0).all()
    clean = ex.expert_up_backward(gd, gw2, kept, gc, go, gr, gp)
    n = int(pos[7, 0])
    kept.exponents[n, 1] = 255       # gate columns 16 .. 31
    dz, a, dc = ex.expert_up_backward(gd, gw2, kept, gc, go, gr, gp)
    ok(ex)
    for got, was, cols in ((dz, clean[0], list(range(16, 32)) + list(range(F + 16, F + 32))),
                           (a, clean[1], list(range(16, 32)))):
        mark = torch.zeros_like(got, dtype=torch.bool)
        mark[n, cols] = True
        assert torch.isnan(got[mark]).all()
        assert torch.equal(got[~mark], was[~mark])
    assert torch.isnan(dc[7, 0])
    dc[7, 0] = clean[2][7, 0]
    assert torch.equal(dc, clean[2])


def test_a_window_without_rows(ex):  # noqa: F811
    """offsets of zeros: nothing is written, joins give zeros (and say so), weight
    gradients are zero or unchanged."""
    T, k, E, H, F = 30, 2, 4, 64, 32
    from paper_2609_32398_gb300 import doloss as dl

    off = torch.zeros(E + 1, dtype=torch.int64)
    x, w1, w2 = rnd(1, T, H), rnd(2, E, 2 * F, H), rnd(3, E, H, F)
    rows, pos = torch.zeros(T * k, dtype=torch.int64), torch.arange(T * k).reshape(T, k)
    gx, gw1, gw2, go, gr, gp = gpu(x, w1, w2, off, rows, pos)
    act = torch.full((T * k, F), 3.0, dtype=torch.bfloat16, device="cuda")
    assert dl.lib().do_expert_up(gx.data_ptr(), gw1.data_ptr(), gr.data_ptr(), go.data_ptr(), T, H, F, E, T * k,
                                 act.data_ptr(), None, None, None, dl._stream(gx)) == 0
    torch.cuda.synchronize()
    assert (act == 3).all()
    out = ex.grouped_matmul_join(act, gw2, go, gp, None)
    torch.cuda.synchronize()
    assert (out == 0).all() and ex.device_status() == 1
    dw = ex.grouped_weight_grad(act, act, go)
    assert (dw == 0).all()
    keep = torch.randn(E, F, F, device="cuda")
    assert torch.equal(ex.grouped_weight_grad(act, act, go, out=keep.clone(), accumulate=True), keep)
    ok(ex)


def test_graph_replays_give_the_same_results(ex):  # noqa: F811
    T, k, E, H, F = 120, 4, 16, 128, 64
    g = torch.Generator().manual_seed(2)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, rows, pos = ref.dispatch(ids, E)
    x, w1, w2 = rnd(1, T, H), rnd(2, E, 2 * F, H, scale=0.1), rnd(3, E, H, F, scale=0.1)
    c, dout = torch.rand(T, k, generator=g), rnd(4, T, H)
    gx, gw1, gw2, go, gr, gp, gc, gd = gpu(x, w1, w2, off, rows, pos, c, dout)

    def step():
        out = ex.expert_ffn(gx, gw1, gw2, gc, go, gr, gp)
        _, kept = ex.expert_up(gx, gw1, go, gr, checkpoint=True)
        dz, a, dc = ex.expert_up_backward(gd, gw2, kept, gc, go, gr, gp)
        return (out, dz, a, dc, ex.grouped_weight_grad(dz, gx, go, None, gr),
                ex.grouped_matmul_join(dz, gw1, go, gp, None, transposed=True))

    plain = [t.clone() for t in step()]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        caught = step()
    for _ in range(3):
        for t in caught:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(caught, plain):
            assert torch.equal(a, b)
    ok(ex)


def test_checkpoint_values_over_the_whole_range(ex):  # noqa: F811
    """Every code with exponents from the least to the greatest that the format has; a
    code above 64 at the greatest stands for more than bf16 holds and reads as infinity."""
    codes = torch.arange(-127, 129).clamp(max=127).to(torch.int8).reshape(1, 256).repeat(10, 1)
    exps = torch.tensor([1, 2, 3, 100, 127, 200, 231, 232, 240, 249], dtype=torch.uint8).reshape(10, 1).repeat(1, 16)
    gc, gexp = gpu(codes, exps)
    got = ex.Checkpoint(gc, gexp).values()
    ok(ex)
    assert torch.equal(got.cpu(), ref.values(codes, exps).bfloat16())


@pytest.mark.parametrize("gather", [False, True])
def test_short_steps_leave_no_warp_behind(ex, gather):  # noqa: F811
    """Many experts of one to three rows: steps in which most loading warps have nothing
    to load.  The same results, and no wait that runs out, over many runs."""
    E, K, N = 500, 512, 1024
    g = torch.Generator().manual_seed(5)
    counts = torch.randint(0, 4, (E,), generator=g).tolist()
    off = ref.groups(counts)
    R = sum(counts)
    a, q, w = rnd(1, 40 if gather else R, K), rnd(2, R, N), rnd(3, E, N, K, scale=0.1)
    rows = torch.randint(0, 40, (R,), generator=g) if gather else None
    ga, gq, gw, go, gr = gpu(a, q, w, off, rows)
    dw = ex.grouped_weight_grad(ga, gq, go, gr, None)
    y = ex.grouped_matmul(ga, gw, go, gr)
    ok(ex)
    want, m = ref.product(a, w, off, rows)
    within(y, want, 2 * K * U * m + BF * want.abs())
    ad = (a if rows is None else a[rows]).double()
    for e in range(0, E, 37):
        i, j = int(off[e]), int(off[e + 1])
        within(dw[e], ad[i:j].T @ q[i:j].double(), 2 * max(j - i, 1) * U * (ad[i:j].abs().T @ q[i:j].double().abs()))
    for _ in range(100):
        assert torch.equal(ex.grouped_weight_grad(ga, gq, go, gr, None), dw)
        assert torch.equal(ex.grouped_matmul(ga, gw, go, gr), y)
    ok(ex)


@pytest.mark.parametrize("n", [63, 65, 128, 129, 255, 256, 257, 513])
@pytest.mark.parametrize("blocks", [1, 9, 20, 40])
def test_tile_widths_follow_the_number_of_tiles(ex, n, blocks):  # noqa: F811
    """Few tiles are divided and many are not: group sizes at the edges of each width, with
    one to forty tiles of weights, through every epilogue."""
    counts, K, F, T = [n, 0, 1, n + 1], 72, 128 * blocks - 16, 31
    off, R = ref.groups(counts), 2 * n + 2
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(n))
    a, w = rnd(n, T, K), rnd(n + blocks, 4, 2 * F, K, scale=0.2)
    z, mz = ref.product(a, w, off, rows)
    act = ref.swiglu(z)
    ga, gw, go, gr = gpu(a, w, off, rows)
    got = ex.grouped_matmul(ga, gw, go, gr)
    up, kept = ex.expert_up(ga, gw, go, gr, checkpoint=True)
    ok(ex)
    within(got, z, 2 * K * U * mz + BF * z.abs())
    d = 2 * K * U * mz
    dg, du, gate, u = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    within(up, act, 1.1 * dg * u + gate * du + 2 * dg * du + (BF + FN) * act.abs())
    top = (z.abs() + d).reshape(R, -1, 16).amax(-1, keepdim=True).expand(R, F // 8, 16).reshape(R, 2 * F)
    within(kept.values(), z, top / 127 + d)


@pytest.mark.parametrize("T,E", [(63, 2), (128, 1), (129, 3), (515, 2)])
@pytest.mark.parametrize("F", [48, 1296, 5120])
def test_tile_widths_of_the_gradient(ex, T, E, F):  # noqa: F811
    H, k, g = 72, 1, torch.Generator().manual_seed(T + F)
    ids = torch.randint(0, E, (T, k), generator=g)
    off, rows, pos = ref.dispatch(ids, E)
    dout, w2 = rnd(1, T, H, scale=0.1), rnd(2, E, H, F, scale=0.1)
    combine = torch.rand(T, k, generator=g)
    codes, exps = ref.quantise(torch.randn(T * k, 2 * F, generator=g) * 2)
    z = ref.values(codes, exps)
    dz, act, dc, gr, gm, w, a1 = ref.up_backward(dout, w2, z, combine, off, rows, pos)
    gd, gw, gc, go, grw, gp, gco, gex = gpu(dout, w2, combine, off, rows, pos, codes, exps)
    got_z, got_a, got_c = ex.expert_up_backward(gd, gw, ex.Checkpoint(gco, gex), gc, go, grw, gp)
    ok(ex)
    d = 2 * H * U * gm
    gate, up = z[:, :F], z[:, F:].abs()
    s = torch.sigmoid(gate)
    slope = torch.cat([w * up * s * (1 + gate.abs() * (1 - s)), w * gate.abs() * s], 1)
    gg = torch.cat([gr, gr], 1).abs()
    within(got_z, dz, slope * torch.cat([d, d], 1) * 1.01 + 4 * FN * slope * gg + BF * dz.abs())
    within(got_a, act, (BF + 2 * FN) * act.abs())
    bound = ((d * a1.abs()) * 1.01 + (2 * F * U + 2 * FN) * (gr * a1).abs()).sum(1)[pos]
    within(got_c, dc, bound)
