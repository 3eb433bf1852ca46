"""The refusals of the whole layer's call, on the host and before any launch, and its
binding's checks of tensors."""
import ctypes

import pytest
import torch

INV, UNS, WS = 1, 2, 6
fake, odd8, odd2 = (ctypes.c_void_p(a) for a in (0x10000, 0x10008, 0x10002))


@pytest.fixture(scope="module")
def dl():
    from paper_2609_32398_gb300 import build, doloss

    build.build()
    return doloss


def test_moe_layer_validates_on_the_host(dl):
    L = dl.lib()
    n = L.do_moe_layer_workspace_size(8, 2, 64, 48)
    assert n >= 2 * 16 * 48 + 4 * 16 * 64
    for bad in ((0, 2, 64, 48), (8, 0, 64, 48), (8, 2, 0, 48), (8, 2, 64, 0), (65, 2, 64, 48), (8, 33, 64, 48)):
        assert L.do_moe_layer_workspace_size(*bad) == 0
    #       X     Wr    W1    w1x   W2    w2x   T  H   F   E  k  gate out  ids   comb  status ws    bytes stream
    good = [fake, fake, fake, None, fake, None, 8, 64, 48, 4, 2, 0, fake, fake, fake, None, fake, n, None]

    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return L.do_moe_layer(*a)

    for i in (0, 1, 2, 4, 12, 13, 14):
        assert call(**{f"_{i}": None}) == INV
    assert call(_3=fake) == INV and call(_5=fake) == INV       # both exponents or neither
    for i in (0, 1, 2, 4, 12):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (13, 14, 15):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (6, 7, 8, 9, 10):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_10=5) == INV and call(_11=2) == INV and call(_11=-1) == INV
    assert call(_6=65) == UNS and call(_7=60) == UNS and call(_8=24) == UNS and call(_9=1025) == UNS
    assert call(_9=40, _10=33) == UNS and call(_7=4104) == UNS and call(_8=4112) == UNS
    assert call(_3=fake, _5=fake, _7=72) == UNS and call(_3=fake, _5=fake, _7=8208) == UNS
    assert call(_16=None) == WS and call(_16=odd8) == WS and call(_17=n - 1) == WS


def test_the_binding_checks_its_tensors():
    from paper_2609_32398_gb300 import experts8 as e8, layer

    x, wr = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, 64, dtype=torch.bfloat16)
    w1, w2 = torch.zeros(2, 32, 64, dtype=torch.bfloat16), torch.zeros(2, 64, 16, dtype=torch.bfloat16)
    q1 = e8.Blocks(w1.to(torch.float8_e4m3fn), torch.zeros(2, 2, 1, dtype=torch.uint8), True)
    with pytest.raises(ValueError, match="CUDA"):
        layer.moe_layer(x, wr, w1, w2, 2)
    with pytest.raises(ValueError, match="both"):
        layer.moe_layer(x, wr, q1, w2, 2)
    for i in range(4):
        a = [x, wr, w1, w2]
        a[i] = a[i].clone().requires_grad_()
        with pytest.raises(RuntimeError, match="not differentiable"):
            layer.moe_layer(*a, 2)
        with torch.no_grad(), pytest.raises(ValueError, match="CUDA"):
            layer.moe_layer(*a, 2)
