"""The layer for a few tokens on tokens and weights over the range of bf16, against 64 bits, by the
bounds of test_layer_gpu.py (which are relative to the magnitudes that are summed)."""
import pytest
import torch

import blocks_ref as br
import experts_ref as ref
from test_experts8_gpu import blocks
from test_experts_gpu import BF, FN, U, ok
from test_layer_gpu import e8, ex, layer, make, reference, run, within  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("T,k,E,H,F", [(1, 4, 8, 272, 48), (4, 2, 4, 528, 144), (8, 1, 5, 1040, 272), (12, 2, 4, 272, 48)])
@pytest.mark.parametrize("p", [-80, -20, 60, 100, 118])
def test_tokens_of_any_size(ex, layer, e8, p, T, k, E, H, F, eight):  # noqa: F811
    """Tokens of 2^p, up rows and a router of 2^-p: the gate's sums, the activations and the results are
    of 2^p (up to 2^122), which fp32 holds.  The kernels for few and for many rows."""
    x, wr, w1, w2 = make(T, k, E, H, F, T + p + 200)
    x, wr = x * 2.0 ** p, wr * 2.0 ** -p
    w1[:, F:] *= 2.0 ** -p
    v1, v2, (out, ids, _) = run(layer, e8, x, wr, w1, w2, k, 1, eight)
    ok(ex)
    want, bound, want_ids, _ = reference(x, wr, v1, v2, k, True)
    assert torch.equal(ids.cpu().long(), want_ids)
    within(out, want, bound)


@pytest.mark.parametrize("T,k,E,H,F", [(1, 4, 8, 272, 48), (4, 2, 4, 528, 144), (12, 2, 4, 272, 48)])
@pytest.mark.parametrize("d", [-70, -5, 3, 9, 11, 12, 40, 110])
def test_exponents_of_any_size(ex, layer, e8, d, T, k, E, H, F):  # noqa: F811
    """Blocks 2^d as large as ordinary ones, tokens 2^-d: exponent bytes from 40 to 230."""
    x, wr, w1, w2 = make(T, k, E, H, F, T + d + 100)
    c1, x1, v1 = br.weights(w1, True)
    c2, x2, v2 = br.weights(w2)
    x, wr = x * 2.0 ** -d, wr * 2.0 ** d
    x1, x2 = (x1.int() + d).to(torch.uint8), (x2.int() + d).to(torch.uint8)
    out, ids, _ = layer.moe_layer(x.cuda(), wr.cuda(), blocks(e8, c1, x1, True), blocks(e8, c2, x2), k, 1)
    ok(ex)
    want, bound, want_ids, _ = reference(x, wr, v1 * 2.0 ** d, v2 * 2.0 ** d, k, True)
    assert torch.equal(ids.cpu().long(), want_ids)
    within(out, want, bound)


@pytest.mark.parametrize("T,grain", [(1, 0.0), (8, 0.0), (9, 2.0 ** -11), (40, 2.0 ** -11)])
def test_activations_between_products_with_codes(ex, layer, e8, T, grain):  # noqa: F811
    """Results that are the differences of two activations a few hundredths apart, so that what the
    activations lose between the projections shows: nothing of their fp32 for up to eight routed rows, a
    rounding to 11 bits for more (and bits below 2^-39 of the largest)."""
    E, H, F = 3, 272, 144
    x, wr, w1, w2 = make(T, 1, E, H, F, 41)
    x[:, 0] = 1
    for rows in (slice(0, F), slice(F, 2 * F)):
        w1[:, rows][:, 1::2] = w1[:, rows][:, ::2]
    w1[:, F + 1::2, 0] += 2.0 ** -6
    w2[:] = 0
    for h in range(F // 2):
        w2[:, h, 2 * h], w2[:, h, 2 * h + 1] = 1, -1
    v1, _, (out, ids, combine) = run(layer, e8, x, wr, w1, w2, 1, 1, True)
    ok(ex)
    assert bool((combine == 1).all())
    e = ids.cpu().long()[:, 0]
    xd, v = x.double(), v1.double()[e]                        # [T, 2F, H]
    z, m = torch.einsum("tfh,th->tf", v, xd), torch.einsum("tfh,th->tf", v.abs(), xd.abs())
    act, d = ref.swiglu(z), 2 * H * U * m
    g, u, dg, du = z[:, :F].abs(), z[:, F:].abs(), d[:, :F], d[:, F:]
    err = 1.1 * dg * u + g * du + 2 * dg * du + (grain + FN + 2 * U) * act.abs() + 2.0 ** -39 * act.abs().amax(1, True)
    want, room = act[:, ::2] - act[:, 1::2], err[:, ::2] + err[:, 1::2]
    assert float((want.abs() / act[:, ::2].abs()).median()) < 0.1
    within(out[:, :F // 2], want, room + BF * want.abs())
    assert not bool(out[:, F // 2:].any())
