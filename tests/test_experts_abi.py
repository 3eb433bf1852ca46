"""The expert operators' refusals, on the host and before any launch, and their
binding's checks of tensors."""
import ctypes

import pytest
import torch

import experts_ref as ref

INV, UNS, WS = 1, 2, 6


@pytest.fixture(scope="module")
def dl():
    from paper_2609_32398_gb300 import build, doloss

    build.build()
    return doloss


fake, odd8, odd2 = (ctypes.c_void_p(a) for a in (0x10000, 0x10008, 0x10002))
big = 1 << 40


def test_expert_up_validates_on_the_host(dl):
    f = dl.lib().do_expert_up
    #      X     W1    rows  off   T   H   F   E  R   act   codes exps  status stream
    good = [fake, fake, fake, fake, 16, 64, 32, 4, 16, fake, None, None, None, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)

    for i in (0, 1, 3, 9):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 9):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (2, 3, 12):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (4, 5, 6, 7, 8):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_10=fake) == INV and call(_11=fake) == INV      # codes and exponents go together
    assert call(_10=odd8, _11=fake) == INV
    assert call(_2=None, _8=17) == INV                          # rows of X themselves, and too few
    assert call(_5=60) == UNS                                   # H % 8
    assert call(_6=24) == UNS                                   # F % 16
    assert call(_7=1025) == UNS
    assert call(_8=2 ** 31 - 1) == UNS
    assert call(_4=2 ** 31 - 1) == UNS


def test_grouped_matmul_validates_on_the_host(dl):
    f = dl.lib().do_grouped_matmul
    #      A     W     rows  off   T   K   N   E  R   tr Y     status stream
    good = [fake, fake, fake, fake, 16, 64, 40, 4, 16, 0, fake, None, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)

    for i in (0, 1, 3, 10):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 10):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (4, 5, 6, 7, 8):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_9=2) == INV and call(_9=-1) == INV
    assert call(_2=None, _8=17) == INV
    assert call(_5=68) == UNS and call(_6=44) == UNS and call(_7=1025) == UNS
    assert call(_6=(1 << 20) + 8) == UNS


def test_grouped_matmul_join_validates_on_the_host(dl):
    L = dl.lib()
    f = L.do_grouped_matmul_join
    n = L.do_grouped_matmul_join_workspace_size(8, 2, 40)
    assert n >= 2 * 16 * 40
    for bad in ((0, 2, 40), (8, 0, 40), (8, 2, 0), (1 << 30, 4, 40)):
        assert L.do_grouped_matmul_join_workspace_size(*bad) == 0
    #      A     W     off   pos   wts   T  k  K   N   E  tr out   status ws    bytes stream
    good = [fake, fake, fake, fake, fake, 8, 2, 64, 40, 4, 0, fake, None, fake, n, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)

    for i in (0, 1, 2, 3, 11):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 11):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (2, 3, 4, 12):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (5, 6, 7, 8, 9):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_10=3) == INV
    assert call(_5=1 << 30) == UNS and call(_7=60) == UNS and call(_8=44) == UNS
    assert call(_13=None) == WS and call(_14=n - 1) == WS and call(_13=odd8) == WS


def test_expert_up_backward_validates_on_the_host(dl):
    L = dl.lib()
    f = L.do_expert_up_backward
    n = L.do_expert_up_backward_workspace_size(8, 2, 48)
    assert n >= 4 * 16 * 2
    assert L.do_expert_up_backward_workspace_size(8, 2, 0) == 0
    #      dout  W2    codes exps  comb  rows  off   pos   T  k  H   F   E  dz    act   dcomb status ws    bytes stream
    good = [fake] * 8 + [8, 2, 64, 48, 4, fake, fake, fake, None, fake, n, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)

    for i in list(range(8)) + [13, 14, 15]:
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 2, 13, 14):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (4, 5, 6, 7, 15, 16):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (8, 9, 10, 11, 12):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_10=60) == UNS and call(_11=40) == UNS and call(_12=2000) == UNS
    assert call(_17=None) == WS and call(_18=n - 1) == WS


def test_grouped_weight_grad_validates_on_the_host(dl):
    f = dl.lib().do_grouped_weight_grad
    #      P     Q     pr    qr    off   Tp  Tq  M   N   E  R   acc dW    status stream
    good = [fake, fake, fake, None, fake, 5, 16, 64, 40, 4, 16, 0, fake, None, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)

    for i in (0, 1, 4, 12):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 12):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (5, 6, 7, 8, 9, 10):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_6=15) == INV                                   # q has no row ids and too few rows
    assert call(_2=None) == INV                                 # nor p
    assert call(_11=2) == INV
    assert call(_7=60) == UNS and call(_8=44) == UNS and call(_9=1025) == UNS


def test_expert_ffn_and_values_validate_on_the_host(dl):
    L = dl.lib()
    n = L.do_expert_ffn_workspace_size(8, 2, 64, 48)
    assert n > 2 * 16 * 48 and L.do_expert_ffn_workspace_size(8, 2, 64, 0) == 0
    #      X W1 W2 comb rows off pos  T  k  H   F   E  out   status ws    bytes stream
    good = [fake] * 7 + [8, 2, 64, 48, 4, fake, None, fake, n, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return L.do_expert_ffn(*a)

    for i in list(range(7)) + [12]:
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 2, 12):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (7, 8, 9, 10, 11):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_9=60) == UNS and call(_10=40) == UNS
    assert call(_14=None) == WS and call(_15=n - 1) == WS
    v = L.do_checkpoint_values
    assert v(None, fake, 4, 32, fake, None) == INV and v(fake, None, 4, 32, fake, None) == INV
    assert v(fake, fake, 0, 32, fake, None) == INV and v(odd8, fake, 4, 32, fake, None) == INV
    assert v(fake, fake, 4, 40, fake, None) == UNS


def test_binding_refuses_tensors_that_the_library_cannot_read(dl):
    """Tensors of the CPU, of other types and of other shapes raise before the call."""
    from paper_2609_32398_gb300 import experts as ex

    x, w1, w2 = torch.zeros(4, 64).bfloat16(), torch.zeros(2, 32, 64).bfloat16(), torch.zeros(2, 64, 16).bfloat16()
    off, rows = torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    pos, c = torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1)
    kept = ex.Checkpoint(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8))
    for call in (lambda: ex.expert_up(x, w1, off, rows), lambda: ex.grouped_matmul(x, w1, off),
                 lambda: ex.grouped_matmul_join(x, w1, off, pos, c), lambda: kept.values(),
                 lambda: ex.expert_up_backward(x, w2, kept, c, off, rows, pos),
                 lambda: ex.grouped_weight_grad(x, x, off), lambda: ex.expert_ffn(x, w1, w2, c, off, rows, pos)):
        with pytest.raises(ValueError):
            call()


def test_reference_gradients_against_differences():
    """The formulas that the GPU tests compare with: up_backward's dz and dcombine
    are the derivatives of the layer, by central differences in 64 bits."""
    g = torch.Generator().manual_seed(3)
    T, k, E, H, F = 5, 2, 3, 4, 16
    ids = torch.stack([torch.randperm(E, generator=g)[:k] for _ in range(T)])
    off, rows, pos = ref.dispatch(ids, E)
    w2 = torch.randn(E, H, F, generator=g).double()
    z = torch.randn(T * k, 2 * F, generator=g).double()
    c = torch.rand(T, k, generator=g).double()
    dout = torch.randn(T, H, generator=g).double()

    def value(z, c):
        y, _ = ref.product(ref.swiglu(z), w2, off)
        return float(((y[pos.reshape(-1)].reshape(T, k, H) * c.unsqueeze(-1)).sum(1) * dout).sum())

    dz, act, dc = ref.up_backward(dout, w2, z, c, off, rows, pos)[:3]
    h = 1e-5
    for _ in range(40):
        i, j = int(torch.randint(T * k, (1,), generator=g)), int(torch.randint(2 * F, (1,), generator=g))
        d = torch.zeros_like(z)
        d[i, j] = h
        assert abs((value(z + d, c) - value(z - d, c)) / (2 * h) - float(dz[i, j])) < 1e-6 * (1 + abs(float(dz[i, j])))
    for t in range(T):
        for q in range(k):
            d = torch.zeros_like(c)
            d[t, q] = h
            assert abs((value(z, c + d) - value(z, c - d)) / (2 * h) - float(dc[t, q])) < 1e-6 * (1 + abs(float(dc[t, q])))
    # and the whole layer's autograd agrees with them through W2's operand
    w2r = w2.clone().requires_grad_()
    y = torch.cat([ref.swiglu(z)[int(off[e]):int(off[e + 1])] @ w2r[e].T for e in range(E)])
    ((y[pos.reshape(-1)].reshape(T, k, H) * c.unsqueeze(-1)).sum(1) * dout).sum().backward()
    for e in range(E):
        a, b = int(off[e]), int(off[e + 1])
        assert torch.allclose(w2r.grad[e], dout[rows[a:b]].T @ act[a:b], atol=1e-12)
