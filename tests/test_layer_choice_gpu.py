"""The choice of experts of the layer for a few tokens against exact sums.

The router keeps each lane's running sum and the sum of its rounding errors, every error exact.  With
U = 2^-24, A the sum of the products' magnitudes and n = 4 ceil(H / 256) + 6 additions on the
way of a product, the sum of the errors is at most n U A at any time.  Where all products are
multiples of g and n A U <= 2^24 g it is therefore a multiple of g below 2^24 g, which fp32 holds
exactly: the logits are the exact ones, equal ones are equal, and the choice is that of
integers.  The inputs here are made so, and every test checks that they are."""
import pytest
import torch

from test_experts_gpu import U, ok, rnd

pytestmark = pytest.mark.gpu

F, K_MOST = 16, 32


@pytest.fixture(scope="module")
def ex():
    from paper_2609_32398_gb300 import doloss, experts

    doloss.lib()
    return experts


@pytest.fixture(scope="module")
def layer():
    from paper_2609_32398_gb300 import layer

    return layer


def whole(x, wr, g):
    """The logits over g as whole numbers, by 64-bit integers; the inputs keep to the bound above."""
    p = x.double().unsqueeze(1) * wr.double().unsqueeze(0)            # 16 bits each: exact
    q = p / g
    assert torch.equal(q, q.round()) and bool((q.abs() < 2.0 ** 53).all())
    n = 4 * -(-x.shape[1] // 256) + 6
    assert bool((n * U * p.abs().sum(-1) <= 2.0 ** 24 * g).all())
    return q.to(torch.int64).sum(-1)


def chosen(ex, layer, x, wr, k):
    E, H = wr.shape
    w1, w2 = torch.zeros(E, 2 * F, H).bfloat16(), torch.zeros(E, H, F).bfloat16()
    _, ids, _ = layer.moe_layer(x.cuda(), wr.cuda(), w1.cuda(), w2.cuda(), k)
    ok(ex)
    return ids.cpu().long()


def first(z, k):
    return torch.sort(z, dim=1, descending=True, stable=True)[1][:, :k]


@pytest.mark.parametrize("T", [1, 13])
def test_products_larger_than_the_sum_so_far(ex, layer, T):
    """1/2, then 2^-24, then 3/2 in one lane: what is lost of 2 + 2^-24 is an error of the sum
    before, not of the product."""
    H, E = 64, 4
    x = torch.ones(T, H).bfloat16()
    wr = torch.zeros(E, H).bfloat16()
    wr[:, 0], wr[:, 4] = 0.5, 1.5
    wr[1, 2], wr[3, 2] = 2.0 ** -24, 2.0 ** -23
    assert torch.equal(chosen(ex, layer, x, wr, E), torch.tensor([3, 1, 0, 2]).expand(T, E))
    assert torch.equal(first(whole(x, wr, 2.0 ** -25), E), torch.tensor([3, 1, 0, 2]).expand(T, E))


@pytest.mark.parametrize("T", [1, 8, 9, 61, 64])
@pytest.mark.parametrize("H,E", [(64, 33), (264, 8), (1000, 40), (2048, 128), (4096, 300)])
def test_rows_of_the_same_columns_in_any_order(ex, layer, T, H, E):
    """Experts whose rows are one row's columns in other orders, half of them with a column moved by a
    few of the least steps; large columns of both signs among them, which cancel but for little.
    The tokens have one magnitude in all columns, so that an order does not change a logit."""
    g = torch.Generator().manual_seed(H + T)
    base = (torch.randint(-2 ** 8, 2 ** 8 + 1, (H,), generator=g).double() * 2.0 ** -30).bfloat16()   # small ones
    mid = torch.arange(0, H, 3)
    base[mid] = (torch.randint(-2 ** 7, 2 ** 7 + 1, (len(mid),), generator=g).double() * 2.0 ** -14).bfloat16()
    large = torch.arange(1, H, 9)
    base[large] = (torch.randint(1, 2 ** 7 + 1, (len(large),), generator=g).double() * 2.0 ** -6).bfloat16()
    base[large[1::2]] = -base[large[::2]][:len(large[1::2])]
    wr = torch.stack([base[torch.randperm(H, generator=g)] for _ in range(E)])
    for e in range(0, E, 2):
        at = int(torch.nonzero(wr[e].abs().double() <= 2.0 ** -23)[e % 5])
        wr[e, at] = float(wr[e, at]) + 2.0 ** -30 * ((7 * e) % 9 - 4)      # at most 2^7 + 4 steps: 8 bits, or even
    x = torch.where(torch.rand(T, 1, generator=g) < 0.5, -1.0, 1.0).expand(T, H).bfloat16().contiguous()
    x *= (2.0 ** torch.randint(-3, 4, (T, 1), generator=g).float()).bfloat16()
    k = min(E, K_MOST)
    want = torch.stack([first(whole(x[t:t + 1], wr, 2.0 ** -30 * float(x[t, 0].abs())), k)[0] for t in range(T)])
    assert torch.equal(chosen(ex, layer, x, wr, k), want)


@pytest.mark.parametrize("T", [3, 20])
def test_differences_of_two_pow_minus_38(ex, layer, T):
    """Random rows beside a large column, each with a copy in another order that is 2^-38 of the
    largest product away."""
    H, E = 1024, 24
    g = torch.Generator().manual_seed(T)
    wr = (torch.randint(-2 ** 7, 2 ** 7 + 1, (E, H), generator=g).double() * 2.0 ** -24).bfloat16()
    wr[:, 17] = (torch.randint(2 ** 6, 2 ** 7, (E,), generator=g).double() * 2.0 ** -6).bfloat16()
    for e in range(0, E, 2):
        wr[e, 20 * e] = 0
        wr[e + 1] = wr[e]
        wr[e + 1, 20 * e] = 2.0 ** -37 if e % 4 == 0 else -2.0 ** -37
        wr[e + 1] = wr[e + 1, torch.randperm(H, generator=g)]
    x = torch.where(torch.rand(T, 1, generator=g) < 0.5, -1.0, 1.0).expand(T, H).bfloat16().contiguous()
    z = whole(x, wr, 2.0 ** -37)
    assert bool((z[:, 1::2] != z[:, ::2]).all())
    assert torch.equal(chosen(ex, layer, x, wr, E), first(z, E))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("T,k,E", [(1, 4, 6), (7, 4, 256), (7, 32, 257), (20, 8, 40), (20, 5, 1000), (64, 2, 300)])
@pytest.mark.parametrize("eight", [False, True])
def test_a_token_that_is_not_finite(ex, layer, T, k, E, bad, eight):
    """Its experts are k different ones all the same, its weights and results are NaN, and every
    other token's stay as they were, to the bit."""
    from paper_2609_32398_gb300 import experts8 as e8

    H, hit = 272, [T // 2, T - 1]
    x, wr = rnd(T, T, H).cuda(), rnd(E, E, H, scale=H ** -0.5).cuda()
    w1, w2 = rnd(1, E, 2 * F, H, scale=H ** -0.5).cuda(), rnd(2, E, H, F, scale=F ** -0.5).cuda()
    if eight:
        w1, w2 = e8.quantise_weights(w1, True), e8.quantise_weights(w2)
    broken = x.clone()
    broken[hit, [5, 200][:len(hit)]] = bad
    good = torch.ones(T, dtype=torch.bool)
    good[hit] = False
    for gate in (0, 1):
        want = layer.moe_layer(x, wr, w1, w2, k, gate)
        out, ids, combine = layer.moe_layer(broken, wr, w1, w2, k, gate)
        ok(ex)
        for a, b in zip((out, ids, combine), want):
            assert torch.equal(a[good.cuda()], b[good.cuda()])
        chosen = ids.cpu().sort(1)[0]
        assert bool((chosen >= 0).all()) and bool((chosen < E).all()) and bool((chosen.diff(dim=1) > 0).all())
        assert bool(torch.isnan(combine[~good.cuda()]).all()) and bool(torch.isnan(out[~good.cuda()]).all())
