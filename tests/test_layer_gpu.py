"""The whole layer for a few tokens against 64 bits.

Bounds, for U = 2^-24: the choice is that of the 64-bit logits, whose gaps in these inputs are far
above the kernel's 2^-40 or zero; combine is within 16 U of itself for |z| < 8 (an
exponential of a rounded argument, two additions and a division); a projection summed in fp32 is within
2 K U of the sum of magnitudes, an activation is rounded to bf16 (2^-8 of itself), sigma
within 2^-18 for |z| < 30, and the result is rounded to bf16."""
import pytest
import torch

import blocks_ref as br
import experts_ref as ref
from test_experts8_gpu import blocks
from test_experts_gpu import BF, FN, U, ok, rnd, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ex():
    from paper_2609_32398_gb300 import doloss, experts

    doloss.lib()
    return experts


@pytest.fixture(scope="module")
def layer():
    from paper_2609_32398_gb300 import layer

    return layer


@pytest.fixture(scope="module")
def e8():
    from paper_2609_32398_gb300 import experts8

    return experts8


def reference(x, wr, v1, v2, k, softmax):
    """out, its bound, ids, combine in 64 bits for expert weights of values v1 and v2."""
    T, H = x.shape
    E, F = v1.shape[0], v1.shape[1] // 2
    z = x.double() @ wr.double().T
    ids = torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k]
    chosen = torch.gather(z, 1, ids)
    combine = torch.softmax(chosen, 1)
    if not softmax:
        # sigmoids over their sum, with e^(their largest) taken out
        top = chosen.amax(1, keepdim=True).clamp(max=0)
        s = torch.exp(torch.clamp(chosen, max=0) - top) / (1 + torch.exp(-chosen.abs()))
        combine = s / s.sum(1, keepdim=True)
    out, room = torch.zeros(T, H, dtype=torch.float64), torch.zeros(T, H, dtype=torch.float64)
    for t in range(T):
        for q in range(k):
            e = int(ids[t, q])
            w1, w2 = v1[e].double(), v2[e].double()
            zz, m = w1 @ x[t].double(), w1.abs() @ x[t].double().abs()
            act = ref.swiglu(zz[None])[0]
            d = 2 * H * U * m
            dg, du, g, u = d[:F], d[F:], zz[:F].abs(), zz[F:].abs()
            err = 1.1 * dg * u + g * du + 2 * dg * du + (BF + FN) * act.abs()
            c = combine[t, q]
            out[t] += c * (w2 @ act)
            room[t] += c * (w2.abs() @ (err + (2 * F + 2 * k + 16) * U * act.abs()))
    return out, room + BF * out.abs(), ids, combine


def make(T, k, E, H, F, seed, skew=0.3):
    x, wr = rnd(seed, T, H) + (rnd(seed + 1, 1, H) * skew).bfloat16(), rnd(seed + 2, E, H, scale=H ** -0.5)
    return x, wr, rnd(seed + 3, E, 2 * F, H, scale=H ** -0.5), rnd(seed + 4, E, H, F, scale=F ** -0.5)


def run(layer, e8, x, wr, w1, w2, k, gate, eight):
    if eight:
        c1, x1, v1 = br.weights(w1, True)
        c2, x2, v2 = br.weights(w2)
        g1, g2 = blocks(e8, c1, x1, True), blocks(e8, c2, x2)
    else:
        v1, v2, g1, g2 = w1, w2, w1.cuda(), w2.cuda()
    return v1, v2, layer.moe_layer(x.cuda(), wr.cuda(), g1, g2, k, gate)


# T, k, E, H, F
SIZES = [(1, 1, 1, 16, 16), (1, 8, 128, 2048, 768), (2, 2, 8, 272, 48), (3, 3, 5, 128, 16), (7, 5, 40, 1008, 208),
         (8, 8, 8, 512, 64), (9, 4, 33, 144, 272), (16, 2, 128, 256, 128), (33, 6, 24, 528, 80), (48, 8, 128, 512, 96),
         (64, 8, 16, 272, 64), (64, 1, 300, 64, 32), (64, 2, 2, 1040, 144), (5, 32, 40, 160, 32), (4, 3, 1024, 48, 16),
         (2, 2, 4, 2992, 896), (64, 32, 64, 96, 32), (8, 1, 5, 1040, 272), (4, 2, 3, 144, 400), (13, 3, 20, 1024, 128),
         (40, 1, 9, 512, 64), (41, 1, 9, 512, 64), (64, 4, 8, 512, 48), (50, 8, 8, 272, 272), (64, 2, 9, 144, 16)]


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,k,E,H,F", SIZES)
def test_layer(ex, layer, e8, T, k, E, H, F, eight):
    x, wr, w1, w2 = make(T, k, E, H, F, T + H)
    gate = (T + k) % 2
    v1, v2, (out, ids, combine) = run(layer, e8, x, wr, w1, w2, k, gate, eight)
    ok(ex)
    want, bound, want_ids, want_c = reference(x, wr, v1, v2, k, gate == 1)
    assert torch.equal(ids.cpu().long(), want_ids)
    within(combine, want_c, 16 * U * want_c + 1e-30)
    within(out, want, bound)


@pytest.mark.parametrize("H", [8, 24, 1000])
def test_columns_that_are_not_whole_pieces(ex, layer, e8, H):
    x, wr, w1, w2 = make(7, 2, 6, H, 16, H)
    v1, v2, (out, ids, combine) = run(layer, e8, x, wr, w1, w2, 2, 0, False)
    ok(ex)
    want, bound, want_ids, _ = reference(x, wr, v1, v2, 2, False)
    assert torch.equal(ids.cpu().long(), want_ids)
    within(out, want, bound)


@pytest.mark.parametrize("eight,H,F", [(False, 4096, 4096), (True, 8192, 32), (True, 64, 8192), (False, 4088, 16)])
def test_the_widest_rows(ex, layer, e8, eight, H, F):
    for T in (11, 1):
        x, wr, w1, w2 = make(T, 2, 2, H, F, H + F)
        v1, v2, (out, ids, _) = run(layer, e8, x, wr, w1, w2, 2, 1, eight)
        ok(ex)
        want, bound, want_ids, _ = reference(x, wr, v1, v2, 2, True)
        assert torch.equal(ids.cpu().long(), want_ids)
        within(out, want, bound)


@pytest.mark.parametrize("T", [1, 9])
def test_equal_logits_go_to_the_lower_expert(ex, layer, e8, T):
    """Experts in equal pairs, and tokens of zeros: all logits equal, weights 1/k."""
    k, E, H, F = 5, 40, 264, 16
    x, wr, w1, w2 = make(T, k, E, H, F, 3)
    wr[1::2] = wr[::2]
    x[T // 2] = 0
    _, _, (_, ids, combine) = run(layer, e8, x, wr, w1, w2, k, 0, False)
    ok(ex)
    z = x.double() @ wr.double().T
    assert torch.equal(ids.cpu().long(), torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k])
    assert torch.equal(ids[T // 2].cpu(), torch.arange(k, dtype=torch.int32))
    within(combine[T // 2], torch.full((k,), 0.2, dtype=torch.float64), torch.full((k,), 4 * U, dtype=torch.float64))


def test_the_choice_does_not_hang_on_fp32(ex, layer, e8):
    """Logits that differ by 2^-30 of their terms: fp32 sums would not tell them apart."""
    E, H, k, F = 6, 2048, 3, 16
    x = torch.ones(2, H).bfloat16()
    wr = rnd(1, 1, H).repeat(E, 1)
    for e in range(E):
        wr[e, 7 * e] = wr[0, 7 * e]
        wr[e, 100] = 2.0 ** -30 * (1 + (5 * e) % E)
    x[1] = -x[1]
    _, _, (_, ids, _) = run(layer, e8, x, wr, *make(2, k, E, H, F, 1)[2:], k, 0, False)
    ok(ex)
    z = x.double() @ wr.double().T
    assert torch.equal(ids.cpu().long(), torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k])


@pytest.mark.parametrize("scale", [-40.0, 40.0, -120.0, 1e-6])
def test_weights_of_extreme_logits(ex, layer, e8, scale):
    """Sigmoids that all underflow or saturate: the weights are still those of the formula."""
    E, H, k, F = 16, 64, 4, 16
    x, wr, w1, w2 = make(3, k, E, H, F, 5)
    x = x.abs()
    wr = (torch.sign(torch.tensor(scale)) * rnd(7, E, H).abs() * abs(scale) / H * 1.25).bfloat16()
    for gate in (0, 1):
        _, _, (_, ids, combine) = run(layer, e8, x, wr, w1, w2, k, gate, False)
        ok(ex)
        _, _, want_ids, want = reference(x, wr, w1, w2, k, gate == 1)
        assert torch.equal(ids.cpu().long(), want_ids)
        z = (x.double() @ wr.double().T).abs().amax()
        within(combine, want, (16 + 4 * z) * U * want + 1e-30)


@pytest.mark.parametrize("eight", [False, True])
def test_nans_and_infinities_stay_in_their_tokens(ex, layer, e8, eight):
    """(the router's weights leave the bad columns out, so that the logits are finite)"""
    T, k, E, H, F = 20, 2, 8, 272, 80
    x, wr, w1, w2 = make(T, k, E, H, F, 11)
    wr[:, 5] = 0
    x[:, 5] = 1
    _, _, (clean, ids, _) = run(layer, e8, x, wr, w1, w2, k, 0, eight)
    bad = x.clone()
    bad[3, 5], bad[17, 5] = 3.0e38, -3.0e38       # past fp32 in the products
    w = w1.clone()
    w[:, :, 5] = 100.0
    _, _, (clean, ids, _) = run(layer, e8, x, wr, w, w2, k, 0, eight)
    _, _, (got, got_ids, _) = run(layer, e8, bad, wr, w, w2, k, 0, eight)
    ok(ex)
    touched = torch.zeros(T, dtype=torch.bool)
    touched[[3, 17]] = True
    assert torch.equal(got_ids, ids)
    assert torch.equal(got[~touched.cuda()], clean[~touched.cuda()])
    assert not bool(torch.isfinite(got[touched.cuda()]).all())


def test_tokens_of_any_size(ex, layer, e8):
    """Rows over the whole range of bf16 through 8-bit weights: the scale of their blocks follows."""
    T, k, E, H, F = 12, 2, 4, 272, 48
    x, wr, w1, w2 = make(T, k, E, H, F, 13)
    w1[:, F:] *= 0.001
    for t, p in enumerate([-126, -100, -60, -30, -10, 0, 10, 20, 30, 40, 50, 60]):
        x[t] *= 2.0 ** p
    x[5, 10] = 2.0 ** 40      # one block of a row far above the others
    v1, v2, (out, ids, combine) = run(layer, e8, x, wr, w1, w2, k, 1, True)
    ok(ex)
    want, bound, want_ids, _ = reference(x, wr, v1, v2, k, True)
    # tiny tokens: results below bf16's normal numbers are within its least step
    within(out, want, bound + 2.0 ** -133)
    assert torch.equal(ids.cpu().long(), want_ids)


def test_weights_of_other_makers(ex, layer, e8):
    """Exponents off the least possible, among them 0; a NaN block reaches its expert's tokens only."""
    T, k, E, H, F = 8, 1, 4, 144, 144
    x, wr, w1, w2 = make(T, k, E, H, F, 17, skew=0.0)
    c1, x1, v1 = br.weights(w1, True)
    c2, x2, v2 = br.weights(w2)
    x2 = x2.clone()
    x2[0] = 0
    v2 = torch.stack([br.values(c2[e], x2[e], 128) for e in range(E)])
    out, ids, _ = layer.moe_layer(x.cuda(), wr.cuda(), blocks(e8, c1, x1, True), blocks(e8, c2, x2), k)
    ok(ex)
    want, bound, want_ids, _ = reference(x, wr, v1, v2, k, False)
    within(out, want, bound + 2.0 ** -133)
    x1 = x1.clone()
    x1[2] = 255
    bad, ids, _ = layer.moe_layer(x.cuda(), wr.cuda(), blocks(e8, c1, x1, True), blocks(e8, c2, x2), k)
    ok(ex)
    hit = (ids.cpu() == 2).any(1)
    assert bool(torch.isnan(bad[hit.cuda()]).all()) and torch.equal(bad[~hit.cuda()], out[~hit.cuda()])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,k,E", [(1, 4, 32), (40, 4, 32), (60, 4, 8)])
def test_replays_streams_and_repeats(ex, layer, e8, T, k, E, eight):
    """The same bits from a hundred calls, from a side stream next to another call, and from two
    graphs replayed in turn, one of them on other inputs."""
    H, F = 528, 208
    x, wr, w1, w2 = make(T, k, E, H, F, 23)
    gx, gr, g1, g2 = x.cuda(), wr.cuda(), w1.cuda(), w2.cuda()
    if eight:
        g1, g2 = e8.quantise_weights(g1, True), e8.quantise_weights(g2)
    want = layer.moe_layer(gx, gr, g1, g2, k)
    want2 = layer.moe_layer(-gx, gr, g1, g2, k)
    for _ in range(100):
        assert all(torch.equal(a, b) for a, b in zip(layer.moe_layer(gx, gr, g1, g2, k), want))
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    got = []
    for i in range(12):
        with torch.cuda.stream(streams[i % 3]):
            got.append(layer.moe_layer(gx if i % 2 else -gx, gr, g1, g2, k))
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(o, want if i % 2 else want2))
    buf, graphs, outs = gx.clone(), [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(layer.moe_layer(buf, gr, g1, g2, k))
        graphs.append(graph)
    for i in (0, 1, 0, 1):
        buf.copy_(gx if i else -gx)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[i], want if i else want2))
    ok(ex)


def test_the_layers_calls_agree(ex, layer, e8):
    """One layer three ways: this call, router and experts' own calls in bf16, and in 8 bits, on one
    choice of experts."""
    from paper_2609_32398_gb300 import doloss as dl
    T, k, E, H, F = 24, 4, 16, 528, 208
    x, wr, w1, w2 = (t.cuda() for t in make(T, k, E, H, F, 29))
    out, ids, combine = layer.moe_layer(x, wr, w1, w2, k)
    z = (x.double() @ wr.double().T).float()
    r = dl.routing(z, k)
    assert torch.equal(r.expert_ids[0].sort(1)[0], ids.sort(1)[0])
    a = ex.expert_ffn(x, w1, w2, r.combine[0], *ex.dispatch_of(r))
    q1, q2 = e8.quantise_weights(w1, True), e8.quantise_weights(w2)
    b = e8.expert_ffn(x, q1, q2, r.combine[0], *ex.dispatch_of(r))
    c, ids8, _ = layer.moe_layer(x, wr, q1, q2, k)
    ok(ex)
    assert torch.equal(ids8, ids)
    def off(p, q):
        return float((p.double() - q.double()).norm() / q.double().norm())
    # bf16: two roundings of each side.  8-bit weights: a code is off by at most 2^-4 of
    # its value, two projections' worth; the activations' codes come on top
    assert off(out, a) < 4 * BF and off(c, out) < 2 * 2.0 ** -4 and off(b, out) < 4 * 2.0 ** -4


@pytest.mark.parametrize("T", [1, 30])
def test_views_into_larger_tensors(ex, layer, e8, T):
    """Tokens and weights that begin anywhere on a 16-byte border, and other data around them."""
    k, E, H, F = 3, 7, 264, 48
    x, wr, w1, w2 = (t.cuda() for t in make(T, k, E, H, F, 31))
    want = layer.moe_layer(x, wr, w1, w2, k)

    def shifted(t):
        big = torch.full((t.numel() + 72,), float("nan"), dtype=t.dtype, device="cuda")
        big[8:8 + t.numel()] = t.reshape(-1)
        return big[8:8 + t.numel()].view(t.shape)

    got = layer.moe_layer(shifted(x), shifted(wr), shifted(w1), shifted(w2), k)
    ok(ex)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_two_layers_share_a_workspace_in_turn(ex, layer, e8):
    """The C call on one workspace of any content, for a small and then a large call."""
    from paper_2609_32398_gb300 import doloss as dl
    L = dl.lib()
    ws = torch.full((1 << 24,), 255, dtype=torch.uint8, device="cuda")
    for T, k, E, H, F in ((1, 2, 4, 64, 16), (50, 8, 16, 512, 96), (3, 1, 4, 64, 16), (64, 8, 8, 512, 96), (20, 8, 64, 512, 96)):
        x, wr, w1, w2 = (t.cuda() for t in make(T, k, E, H, F, 37))
        want = layer.moe_layer(x, wr, w1, w2, k)
        out = torch.empty_like(want[0])
        ids, combine = torch.empty_like(want[1]), torch.empty_like(want[2])
        assert L.do_moe_layer_workspace_size(T, k, H, F) <= ws.numel()
        assert 0 == L.do_moe_layer(x.data_ptr(), wr.data_ptr(), w1.data_ptr(), None, w2.data_ptr(), None, T, H, F, E, k, 0,
                                   out.data_ptr(), ids.data_ptr(), combine.data_ptr(), None, ws.data_ptr(), ws.numel(),
                                   torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(ids, want[1]) and torch.equal(combine, want[2])


def test_empty_call(layer):
    x, wr, w1, w2 = (t.cuda() for t in make(1, 2, 4, 64, 16, 1))
    out, ids, combine = layer.moe_layer(x[:0], wr, w1, w2, 2)
    assert out.shape == (0, 64) and ids.shape == (0, 2) and combine.shape == (0, 2)
