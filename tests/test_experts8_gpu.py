"""The 8-bit expert operators against 64 bits (tests/blocks_ref.py, tests/experts_ref.py).

Bounds, for U = 2^-24: the product of two codes is exact in fp32 and a power of two
changes nothing, so that K of them summed in fp32 are within 2 K U of the sum of magnitudes
(twice the classic bound); a result rounded to bf16 is within 2^-8 of itself; sigma is within
2^-18 of itself for |z| < 30; a code is within 2^-4 of its value, or 2^-10 of its block's
scale where that is more, and the scale is below top / 224 unless it is the least."""
import pytest
import torch

import blocks_ref as br
import experts_ref as ref
from test_experts_gpu import BF, FN, U, gpu, ok, ragged, rnd, within

pytestmark = pytest.mark.gpu
E4 = 2.0 ** -4


@pytest.fixture(scope="module")
def ex():
    from paper_2609_32398_gb300 import doloss, experts

    doloss.lib()
    return experts


@pytest.fixture(scope="module")
def e8():
    from paper_2609_32398_gb300 import experts8

    return experts8


def blocks(e8, codes, exponents, gated=False):
    return e8.Blocks(codes.view(torch.float8_e4m3fn).contiguous().cuda(), exponents.contiguous().cuda(), gated)


def edges(x):
    """Rows of x at the format's edges: zeros, one value, powers of two, ties, the ends of
    the range, NaN and infinities."""
    n = x.shape[1]
    x[0] = 0
    x[1] = 0
    x[1, n // 2] = 448
    x[2] = 1.75 * 2.0 ** 5                       # exactly 448 of the next scale down
    x[3, 0], x[3, 1:] = 448, 2.0 ** -10          # half of the least code
    x[4, 0], x[4, 1:8] = 448, torch.tensor([17., 19., 21., -17., 9.5, 8.5, 2.5])  # ties among the codes
    x[5] = 3.38e38
    x[6] = 1e-38
    x[7] = 2.0 ** -133                           # bf16's least number
    x[8, n - 1] = float("nan")
    x[9, 0] = float("inf")
    x[10, n // 3] = -float("inf")
    return x


@pytest.mark.parametrize("M,K", [(1, 16), (12, 48), (11, 128), (67, 144), (33, 1008), (300, 2048), (1025, 256)])
def test_rows_are_quantised_by_the_definition(e8, M, K):
    x = rnd(M + K, M, K) * torch.exp(2 * torch.randn(M, 1, generator=torch.Generator().manual_seed(M))).bfloat16()
    if M > 10:
        edges(x)
    codes, exps = br.quantise(x, 1)
    got = e8.quantise_rows(x.cuda())
    assert torch.equal(got.exponents.cpu(), exps)
    bad = (exps == 255).repeat_interleave(128, 1)[:, :K]
    got_codes = got.codes.cpu().view(torch.uint8)
    assert torch.equal(got_codes[~bad], codes[~bad]) and bool(((got_codes[bad] & 127) == 127).all())
    want = br.values(codes, exps, 1)
    v = got.values().cpu().double()
    # values are bf16: the codes of what lies past (2 - 1/16) 2^127 stand for 2^128, its infinity
    assert bool(torch.isnan(v[bad]).all()) and torch.equal(v[~bad], want.float().bfloat16().double()[~bad])
    off = (want - x.double()).abs()[~bad]
    assert bool((off <= torch.maximum(E4 * x.double().abs(), torch.pow(2.0, exps.double() - 137)
                                      .repeat_interleave(128, 1)[:, :K])[~bad]).all())


@pytest.mark.parametrize("E,N,K,gated", [(1, 8, 16, False), (3, 40, 144, False), (2, 128, 128, False),
                                         (2, 272, 1008, True), (1, 24, 16, True), (5, 520, 272, False),
                                         (2, 1536, 256, True)])
def test_weights_are_quantised_by_the_definition(e8, E, N, K, gated):
    w = rnd(N + K, E, N, K, scale=0.02)
    w[0, N // 2, K // 2] = float("nan")
    w[E - 1, N - 1, K - 1] = 7.0
    codes, exps, want = br.weights(w, gated)
    got = e8.quantise_weights(w.cuda(), gated=gated)
    assert torch.equal(got.exponents.cpu(), exps) and got.gated == gated
    bad = torch.isnan(want)
    assert torch.equal(got.codes.cpu().view(torch.uint8)[~bad], codes[~bad])
    v = got.values().cpu().double()
    assert bool(torch.isnan(v[bad]).all()) and torch.equal(v[~bad], want[~bad])


def test_values_over_all_codes_and_exponents(e8):
    """Every code under every exponent: bf16 of the 64-bit value (NaN codes and exponent 255:
    NaN), rounded to nearest where it lies below bf16's numbers."""
    codes = torch.arange(256, dtype=torch.int64).to(torch.uint8).repeat(256, 1)
    exps = torch.arange(256, dtype=torch.int64).to(torch.uint8).reshape(256, 1).repeat(1, 2)
    got = blocks(e8, codes, exps).values().cpu()
    want = br.values(codes, exps, 1).float().bfloat16()     # exact in fp32 but for e < 3 below 2^-149
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


# counts of each expert's rows, K, N
PRODUCTS = [([1], 16, 8), ([0, 3, 0, 0, 1], 64, 64), ([17, 0, 130, 16], 80, 136), ([239, 240, 241, 0, 1], 208, 264),
            ([1] * 40, 528, 24), ([700], 128, 512), (ragged(24, 2000, 3), 1008, 520), ([5, 300, 33], 2048, 96),
            ([0, 0, 9], 16, 1032), (ragged(128, 3000, 5), 256, 128), ([481, 2], 640, 256)]


def operands(e8, R, T, E, N, K, gated=False, scale=0.1):
    x, w = rnd(R, T, K), rnd(R + 1, E, N, K, scale=scale)
    codes, exps = br.quantise(x, 1)
    wc, wx, wv = br.weights(w, gated)
    return br.values(codes, exps, 1), wv, blocks(e8, codes, exps), blocks(e8, wc, wx, gated)


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,K,N", PRODUCTS)
def test_matmul(ex, e8, counts, K, N, gather):
    off = ref.groups(counts)
    R, E = sum(counts), len(counts)
    T = 37 if gather else R
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R)) if gather else None
    a, w, ga, gw = operands(e8, R, T, E, N, K)
    y, m = ref.product(a, w, off, rows)
    go, gr = gpu(off, rows)
    got = e8.matmul(ga, gw, go, gr)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())


@pytest.mark.parametrize("R,K,N", [(1, 2048, 264), (2, 16, 8), (16, 144, 1032), (17, 512, 264), (100, 1008, 520),
                                   (1000, 256, 2048)])
def test_dense_matmul(ex, e8, R, K, N):
    a, w, ga, gw = operands(e8, R, R, 1, N, K)
    y, m = ref.product(a, w, ref.groups([R]))
    got = e8.matmul(ga, gw)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())


UPS = [([1], 64, 16), ([0, 3, 0, 1], 80, 48), ([239, 240, 241, 0, 1], 208, 160), ([1] * 40, 528, 32),
       ([700], 128, 272), (ragged(24, 2000, 3), 1008, 208), (ragged(128, 1500, 9), 256, 64), ([2, 4, 0, 1, 1], 2048, 768)]


def top_of(v):
    """The largest of each 128 columns."""
    pad = torch.zeros(v.shape[0], -v.shape[1] % 128, dtype=torch.float64)
    return torch.cat([v, pad], 1).reshape(v.shape[0], -1, 128).amax(-1)


def exponent_of(top):
    e = torch.full(top.shape, 255, dtype=torch.int64)
    for x in range(247, 2, -1):
        e[top <= 448.0 * 2.0 ** (x - 127)] = x
    return e


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("counts,H,F", UPS)
def test_expert_up(ex, e8, counts, H, F, gather):
    off = ref.groups(counts)
    R, E = sum(counts), len(counts)
    T = 53 if gather else R
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R)) if gather else None
    a, w, ga, gw = operands(e8, R + H, T, E, 2 * F, H, True, scale=1.0 / H ** 0.5)
    z, m = ref.product(a, w, off, rows)
    act = ref.swiglu(z)
    go, gr = gpu(off, rows)
    got = e8.expert_up(ga, gw, go, gr)
    v = got.values()
    ok(ex)
    d = 2 * H * U * m
    dg, du, gate, up = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
    err = 1.1 * dg * up + gate * du + 2 * dg * du + FN * act.abs()
    top = top_of(act.abs() + err)
    least = (top / 224 * 2.0 ** -10).repeat_interleave(128, 1)[:, :F]
    within(v, act, err + torch.maximum(E4 * (act.abs() + err), least))
    # the exponent is that of the block's largest value, which is known up to its error.  (Not
    # of what the codes stand for: a largest value just above 448 of one scale is a code of 224
    # of the next, which is 448 of the lower one again.)
    assert bool((got.exponents.cpu() >= exponent_of(top_of(act.abs() - err))).all())
    assert bool((got.exponents.cpu() <= exponent_of(top)).all())


def test_the_activations_blocks_where_their_largest_value_is(ex, e8):
    """The largest value of a block of 128 in either half of it (two CTAs share a block) and at
    its ends: one-hot rows choose columns of the weights, which are known exactly."""
    F, H = 256, 64
    w = torch.zeros(1, 2 * F, H)
    for h in range(16):
        w[0, :F, h] = 16.0                                  # sigma(16) is 1 to 2^-23
        w[0, F:, h] = 1.0
        w[0, F + (0, 63, 64, 127, 128, 191, 192, 255)[h % 8], h] = 240.0 if h < 8 else -240.0
    wc, wx, wv = br.weights(w, True)
    x = torch.eye(64, H)
    codes, exps = br.quantise(x, 1)
    go, = gpu(ref.groups([64]))
    got = e8.expert_up(blocks(e8, codes, exps), blocks(e8, wc, wx, True), go)
    ok(ex)
    act = ref.swiglu(x.double() @ wv[0].T).float()
    want_codes, want = br.quantise(act, 1)
    assert torch.equal(got.exponents.cpu(), want)
    v, wanted = got.values().cpu().double(), br.values(want_codes, want, 1)
    assert bool(((v - wanted).abs() <= E4 * act.double().abs()).all())


FFNS = [(1, 1, 1, 16, 16), (1, 8, 128, 2048, 768), (5, 3, 24, 272, 208), (301, 5, 40, 1008, 208), (64, 2, 8, 512, 64),
        (1000, 8, 16, 256, 128)]


def layer(e8, T, k, E, H, F, seed):
    g = torch.Generator().manual_seed(seed)
    x, w1, w2 = rnd(seed, T, H), rnd(seed + 1, E, 2 * F, H, scale=H ** -0.5), rnd(seed + 2, E, H, F, scale=F ** -0.5)
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    combine = torch.rand(T, k, generator=g) + 0.1
    combine = combine / combine.sum(1, keepdim=True)
    off, rows, pos = ref.dispatch(ids, E)
    return x, w1, w2, combine, off, rows, pos


@pytest.mark.parametrize("T,k,E,H,F", FFNS)
def test_expert_ffn(ex, e8, T, k, E, H, F):
    """Against 64 bits with the activations quantised where the kernel's are: a value at a
    code's border may fall on either side, so that each is allowed a step of its own, 2^-3 of
    it, where its error reaches the border; the bound is that of the unquantised activation."""
    x, w1, w2, combine, off, rows, pos = layer(e8, T, k, E, H, F, T + H)
    c, xe = br.quantise(x, 1)
    a = br.values(c, xe, 1)
    c1, x1, v1 = br.weights(w1, True)
    c2, x2, v2 = br.weights(w2)
    z, _ = ref.product(a, v1, off, rows)
    act = ref.swiglu(z)
    y, _ = ref.product(act, v2, off)
    _, m = ref.product(act.abs() + act.abs().amax(1, keepdim=True) / 224 * 2.0 ** -6, v2, off)
    cw = combine.double().unsqueeze(-1)
    want = (y[pos] * cw).sum(1)
    room = (m[pos] * cw).sum(1)
    gx, gc, go, gr, gp = gpu(x, combine, off, rows, pos)
    got = e8.expert_ffn(gx, blocks(e8, c1, x1, True), blocks(e8, c2, x2), gc, go, gr, gp)
    ok(ex)
    within(got, want, (E4 + 2 * (H + F) * U + 2.0 ** -9) * room + BF * want.abs())
    # and against its pieces, which the tests above hold to their definitions
    act8 = e8.expert_up(e8.quantise_rows(gx), blocks(e8, c1, x1, True), go, gr)
    y8 = e8.matmul(act8, blocks(e8, c2, x2), go).cpu().double()
    pieces = (y8[pos] * cw).sum(1)
    m8 = (y8.abs()[pos] * cw).sum(1)
    within(got, pieces, BF * m8 + BF * pieces.abs() + 2 * (F + k) * U * room)


def test_nans_and_infinities_stay_in_their_rows(ex, e8):
    T, k, E, H, F = 40, 2, 8, 272, 144
    x, w1, w2, combine, off, rows, pos = layer(e8, T, k, E, H, F, 5)
    gx, gc, go, gr, gp = gpu(x, combine, off, rows, pos)
    q1, q2 = e8.quantise_weights(w1.cuda(), True), e8.quantise_weights(w2.cuda())
    clean = e8.expert_ffn(gx, q1, q2, gc, go, gr, gp)
    bad = gx.clone()
    bad[3, 5], bad[17, 271] = float("nan"), float("inf")
    got = e8.expert_ffn(bad, q1, q2, gc, go, gr, gp)
    ok(ex)
    touched = torch.zeros(T, dtype=torch.bool)
    touched[[3, 17]] = True
    assert bool(torch.isnan(got[touched.cuda()]).all())
    assert torch.equal(got[~touched.cuda()], clean[~touched.cuda()])


@pytest.mark.parametrize("gather", [False, True])
def test_rows_outside_of_groups_are_left(ex, e8, gather):
    """Offsets of a slice of the experts: rows before and behind it keep what they held."""
    K, N, E, R, T = 272, 136, 3, 90, 41
    a, w, ga, gw = operands(e8, R, T if gather else R, E, N, K)
    off = torch.tensor([7, 20, 20, 63])
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(R)) if gather else None
    go, gr = gpu(off, rows)
    from paper_2609_32398_gb300 import doloss as dl
    y = torch.full((R, N), 3.0, dtype=torch.bfloat16, device="cuda")
    dl._check("do_grouped_matmul8", dl.lib().do_grouped_matmul8(
        ga.codes.data_ptr(), ga.exponents.data_ptr(), gw.codes.data_ptr(), gw.exponents.data_ptr(), dl._ptr(gr),
        go.data_ptr(), ga.codes.shape[0], K, N, E, R, y.data_ptr(), None, torch.cuda.current_stream().cuda_stream))
    want, m = ref.product(a, w, off, rows)
    torch.cuda.synchronize()
    assert bool((y[:7] == 3).all()) and bool((y[63:] == 3).all())
    within(y[7:63], want[7:63], (2 * K * U * m + BF * want.abs())[7:63])


def test_a_row_outside_the_matrix_counts_as_zeros_and_is_recorded(ex, e8):
    from paper_2609_32398_gb300 import doloss as dl
    a, w, ga, gw = operands(e8, 20, 20, 2, 64, 144)
    rows = torch.arange(20)
    rows[4], rows[11] = -1, 20
    go, gr = gpu(ref.groups([9, 11]), rows)
    got = e8.matmul(ga, gw, go, gr)
    torch.cuda.synchronize()
    assert ex.device_status() == 1      # DO_ERR_INVALID_ARG
    good = torch.ones(20, dtype=torch.bool)
    good[[4, 11]] = False
    assert bool((got[~good.cuda()] == 0).all())
    y, m = ref.product(a, w, ref.groups([9, 11]))
    within(got[good.cuda()], y[good], (2 * 144 * U * m + BF * y.abs())[good])


def test_operands_of_other_makers(ex, e8):
    """Exponents anywhere in the range, unaligned ones among them (a slice of rows)."""
    M, K, N = 37, 144, 72
    g = torch.Generator().manual_seed(1)
    codes = torch.randint(0, 256, (M, K), generator=g).to(torch.uint8)
    codes[(codes & 127) == 127] = 0
    exps = torch.randint(60, 190, (M, 2), generator=g).to(torch.uint8)
    wc = torch.randint(0, 256, (1, N, K), generator=g).to(torch.uint8)
    wc[(wc & 127) == 127] = 0
    wx = torch.randint(60, 190, (1, 1, 2), generator=g).to(torch.uint8)
    a, w = br.values(codes, exps, 1), br.values(wc[0], wx[0], 128).unsqueeze(0)
    full = blocks(e8, codes, exps)
    part = e8.Blocks(full.codes[1:], full.exponents[1:])
    got = e8.matmul(part, blocks(e8, wc, wx))
    ok(ex)
    y, m = ref.product(a[1:], w, ref.groups([M - 1]))
    within(got, y, 2 * K * U * m + BF * y.abs())


def test_graph_replays_and_streams(ex, e8):
    """The layer captured once and replayed on other inputs, two graphs of one pool, and a call
    on a side stream give what eager calls give."""
    T, k, E, H, F = 130, 4, 16, 272, 208
    x, w1, w2, combine, off, rows, pos = layer(e8, T, k, E, H, F, 9)
    gx, gc, go, gr, gp = gpu(x, combine, off, rows, pos)
    q1, q2 = e8.quantise_weights(w1.cuda(), True), e8.quantise_weights(w2.cuda())
    want = e8.expert_ffn(gx, q1, q2, gc, go, gr, gp)
    want2 = e8.expert_ffn(-gx, q1, q2, gc, go, gr, gp)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = e8.expert_ffn(gx, q1, q2, gc, go, gr, gp)
    side.synchronize()
    assert torch.equal(on_side, want)
    buf = gx.clone()
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(e8.expert_ffn(buf, q1, q2, gc, go, gr, gp))
        graphs.append(graph)
    for graph, out in zip(graphs, outs):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    buf.copy_(-gx)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want2)
    ok(ex)


def test_empty_calls(ex, e8):
    x = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    q = e8.quantise_rows(x)
    assert q.codes.shape == (0, 64) and q.exponents.shape == (0, 1) and q.values().shape == (0, 64)
    w = e8.quantise_weights(rnd(1, 2, 32, 64).cuda(), True)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert e8.expert_up(q, w, off).codes.shape == (0, 16)
    w2 = e8.quantise_weights(rnd(1, 2, 64, 16).cuda())
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    empty = torch.empty(0, 2, device="cuda")
    assert e8.expert_ffn(x, w, w2, empty, off, none, none).shape == (0, 64)
    ok(ex)


@pytest.mark.parametrize("gather", [False, True])
def test_many_tiles_a_pair(ex, e8, gather):
    """Tiles in long succession on each pair of CTAs, whose halves of a block's largest value cross
    on the way: the same bits from thirty calls, and those of 64 bits."""
    E, H, F, R = 16, 256, 768, 32000
    counts = [2000 + 61 * (e % 5) - 122 for e in range(E)]
    R = sum(counts)
    T = 4001 if gather else R
    off = ref.groups(counts)
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(1)) if gather else None
    x, w = rnd(1, T, H).cuda(), rnd(2, E, 2 * F, H, scale=H ** -0.5).cuda()
    a, q = e8.quantise_rows(x), e8.quantise_weights(w, True)
    go, gr = gpu(off, rows)
    got = e8.expert_up(a, q, go, gr)
    for _ in range(30):
        again = e8.expert_up(a, q, go, gr)
        assert torch.equal(again.exponents, got.exponents)
        assert torch.equal(again.codes.view(torch.uint8), got.codes.view(torch.uint8))
    ok(ex)
    av, wv, v = a.values().double(), q.values().double(), got.values().double()
    for e in range(E):
        i, j = int(off[e]), int(off[e + 1])
        ar = av[gr[i:j].long()] if gather else av[i:j]
        z, m = ar @ wv[e].T, ar.abs() @ wv[e].abs().T
        act, d = ref.swiglu(z), 2 * H * U * m
        dg, du, gate, up = d[:, :F], d[:, F:], z[:, :F].abs(), z[:, F:].abs()
        err = 1.1 * dg * up + gate * du + 2 * dg * du + FN * act.abs()
        top = (act.abs() + err).reshape(j - i, -1, 128).amax(-1)
        least = (top / 224 * 2.0 ** -10).repeat_interleave(128, 1)
        off_by = (v[i:j] - act).abs() - err - torch.maximum(E4 * (act.abs() + err), least)
        assert bool((off_by <= 0).all()), (e, float(off_by.max()))


@pytest.mark.parametrize("shift", [0, 1, 2])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("K", [128, 256, 384, 512, 640, 768, 1040])
def test_exponents_of_any_alignment(ex, e8, K, gather, shift):
    """Rows of one to nine exponent bytes that begin on any byte, of rows and of weights: they are read
    as words, halves or bytes."""
    counts, N = [70, 0, 3, 255], 144
    off = ref.groups(counts)
    R, E = sum(counts), len(counts)
    T = 40 if gather else R
    rows = torch.randint(0, T, (R,), generator=torch.Generator().manual_seed(K)) if gather else None
    a, w, ga, gw = operands(e8, K, T, E, N, K)
    y, m = ref.product(a, w, off, rows)

    def moved(q):
        big = torch.full((q.exponents.numel() + 16,), 255, dtype=torch.uint8, device="cuda")
        view = big[shift:shift + q.exponents.numel()]
        view.copy_(q.exponents.reshape(-1))
        return e8.Blocks(q.codes, view.view(q.exponents.shape), q.gated)

    go, gr = gpu(off, rows)
    got = e8.matmul(moved(ga), moved(gw), go, gr)
    ok(ex)
    within(got, y, 2 * K * U * m + BF * y.abs())


def test_past_two_to_the_31_values(ex, e8):
    """More than 2^31 values in the rows, in their codes and in a product, checked at both ends."""
    M, K, N = (1 << 20) + 37, 2064, 2056
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).random_(0, 20000)      # bit patterns of finite numbers
    x[:, 7] = 1
    q = e8.quantise_rows(x)
    ends = [0, 1, M - 300, M - 1]
    for r in ends:
        codes, exps = br.quantise(x[r:r + 1].cpu(), 1)
        assert torch.equal(q.exponents[r:r + 1].cpu(), exps)
        assert torch.equal(q.codes[r:r + 1].cpu().view(torch.uint8), codes)
    v = q.values()
    for r in ends:
        want = br.values(q.codes[r:r + 1].cpu().view(torch.uint8), q.exponents[r:r + 1].cpu(), 1)
        assert torch.equal(v[r:r + 1].cpu().double(), want.float().bfloat16().double())
    del v, x
    # rows of 16 columns times 2056: results past 2^31
    small = e8.quantise_rows(rnd(3, 61, 16).cuda())
    w = e8.quantise_weights(rnd(4, 1, N, 16).cuda())
    rows = torch.arange(M, dtype=torch.int32, device="cuda") % 61
    off = torch.tensor([0, M], dtype=torch.int32, device="cuda")
    y = e8.matmul(small, w, off, rows)
    ok(ex)
    want = small.values().double() @ w.values()[0].double().T
    m = small.values().double().abs() @ w.values()[0].double().abs().T
    for r in (*ends, M - 61):
        assert bool(((y[r].double() - want[r % 61]).abs() <= 2 * 16 * U * m[r % 61] + BF * want[r % 61].abs()).all())
    assert torch.equal(y[M - 61 * 3:M - 61 * 2], y[M - 61 * 2:M - 61])
