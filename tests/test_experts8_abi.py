"""The 8-bit expert operators' refusals, on the host and before any launch, and their
binding's checks of tensors; orders in their sources that no run shows until it hangs."""
import ctypes
import os
import re

import pytest
import torch

import paper_2609_32398_gb300

INV, UNS, WS = 1, 2, 6
fake, odd8, odd2 = (ctypes.c_void_p(a) for a in (0x10000, 0x10008, 0x10002))


@pytest.fixture(scope="module")
def dl():
    from paper_2609_32398_gb300 import build, doloss

    build.build()
    return doloss


def caller(f, good):
    def call(**at):
        a = list(good)
        for i, v in at.items():
            a[int(i[1:])] = v
        return f(*a)
    return call


def test_quantisation_validates_on_the_host(dl):
    #                                         X     M  K   codes exps  stream
    call = caller(dl.lib().do_quantise_rows, [fake, 4, 64, fake, fake, None])
    for i in (0, 3, 4):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 3):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (1, 2):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_2=72) == UNS and call(_2=(1 << 17) + 16) == UNS and call(_1=2 ** 31 - 1) == UNS
    #                                            W     E  N   K   g  codes exps  stream
    call = caller(dl.lib().do_quantise_weights, [fake, 4, 24, 64, 0, fake, fake, None])
    for i in (0, 5, 6):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 5):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (1, 2, 3):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_4=2) == INV and call(_2=25, _4=1) == INV
    assert call(_1=1025) == UNS and call(_3=72) == UNS and call(_2=(1 << 18) + 2) == UNS
    #                                        codes exps  pl N   K   rows values stream
    call = caller(dl.lib().do_block_values, [fake, fake, 2, 24, 64, 128, fake, None])
    for i in (0, 1, 6):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 6):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (2, 3, 4):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_5=2) == INV and call(_5=0) == INV
    assert call(_4=72) == UNS and call(_2=1 << 40) == UNS and call(_2=1 << 30, _3=1 << 30, _4=1 << 17) == UNS


def test_grouped_matmul8_validates_on_the_host(dl):
    #                                           A     ax    W     wx    rows  off   T   K   N   E  R   Y     status stream
    call = caller(dl.lib().do_grouped_matmul8, [fake, fake, fake, fake, fake, fake, 16, 64, 40, 4, 16, fake, None, None])
    for i in (0, 1, 2, 3, 5, 11):
        assert call(**{f"_{i}": None}) == INV            # (no offsets: E = 1 only)
    for i in (0, 2, 11):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (4, 5, 12):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (6, 7, 8, 9, 10):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_4=None, _10=17) == INV
    assert call(_7=72) == UNS and call(_8=44) == UNS and call(_9=1025) == UNS
    assert call(_6=2 ** 31 - 1) == UNS and call(_10=2 ** 31 - 1) == UNS and call(_8=(1 << 17) + 8) == UNS


def test_expert_up8_validates_on_the_host(dl):
    #                                      X     xx    W1    wx    rows  off   T   H   F   E  R   act   ae    status stream
    call = caller(dl.lib().do_expert_up8, [fake, fake, fake, fake, fake, fake, 16, 64, 32, 4, 16, fake, fake, None, None])
    for i in (0, 1, 2, 3, 5, 11, 12):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 2, 11):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (4, 5, 13):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (6, 7, 8, 9, 10):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_4=None, _10=17) == INV
    assert call(_7=72) == UNS and call(_8=24) == UNS and call(_9=1025) == UNS


def test_expert_ffn8_validates_on_the_host(dl):
    L = dl.lib()
    n = L.do_expert_ffn8_workspace_size(8, 2, 64, 48)
    assert n >= 8 * 64 + 16 * 48 + 4 * 16 * 64
    for bad in ((0, 2, 64, 48), (8, 0, 64, 48), (8, 2, 0, 48), (8, 2, 64, 0), (1 << 30, 4, 64, 48)):
        assert L.do_expert_ffn8_workspace_size(*bad) == 0
    #      X     W1    w1x   W2    w2x   comb  rows  off   pos   T  k  H   F   E  out   status ws    bytes stream
    good = [fake] * 9 + [8, 2, 64, 48, 4, fake, None, fake, n, None]
    call = caller(L.do_expert_ffn8, good)
    for i in (*range(9), 14):
        assert call(**{f"_{i}": None}) == INV
    for i in (0, 1, 3, 14):
        assert call(**{f"_{i}": odd8}) == INV
    for i in (5, 6, 7, 8, 15):
        assert call(**{f"_{i}": odd2}) == INV
    for i in (9, 10, 11, 12, 13):
        assert call(**{f"_{i}": 0}) == INV
    assert call(_9=1 << 30, _10=4) == UNS and call(_11=72) == UNS and call(_12=24) == UNS and call(_13=1025) == UNS
    assert call(_16=None) == WS and call(_17=n - 1) == WS and call(_16=odd8) == WS


def test_the_binding_checks_its_tensors():
    from paper_2609_32398_gb300 import experts8 as e8

    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(2, 24, 64, dtype=torch.bfloat16)
    codes, exps = torch.zeros(4, 64, dtype=torch.float8_e4m3fn), torch.zeros(4, 1, dtype=torch.uint8)
    off = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        e8.quantise_rows(x)
    with pytest.raises(ValueError, match="CUDA"):
        e8.quantise_weights(w)
    with pytest.raises(ValueError, match="CUDA"):
        e8.Blocks(codes, exps).values()
    with pytest.raises(ValueError, match="CUDA"):
        e8.matmul(e8.Blocks(codes, exps), e8.Blocks(codes.reshape(1, 4, 64), exps.reshape(1, 4, 1)))
    with pytest.raises(ValueError, match="Blocks"):
        e8.matmul(x, w, off)
    with pytest.raises(ValueError, match="offsets"):
        e8.expert_up(e8.Blocks(codes, exps), e8.Blocks(codes, exps, True), None)
    with pytest.raises(ValueError, match="CUDA"):
        e8.expert_ffn(x, w, w, torch.zeros(4, 1), off, off, off)
    # with a graph being recorded, an operand that wants a gradient is refused
    for f in (e8.quantise_rows, e8.quantise_weights):
        with pytest.raises(RuntimeError, match="not differentiable"):
            f((x if f is e8.quantise_rows else w).clone().requires_grad_())
    with pytest.raises(RuntimeError, match="not differentiable"):
        e8.expert_ffn(x.clone().requires_grad_(), None, None, torch.zeros(4, 1), off, off, off)
    with pytest.raises(RuntimeError, match="not differentiable"):
        e8.expert_ffn(x, None, None, torch.zeros(4, 1, requires_grad=True), off, off, off)


def source(name):
    with open(os.path.join(os.path.dirname(paper_2609_32398_gb300.__file__), "csrc", name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def test_tensor_memory_is_taken_after_the_kernel_before():
    """As for the bf16 products: a dependent that took all of the tensor memory and then waited
    for the kernel before would be waited for by it in turn."""
    code = source("experts8_product.cu")
    waits = [m.start() for m in re.finditer(r"\bpdl_wait\(\)", code)]
    takes = [m.start() for m in re.finditer(r"\bpair_tmem_alloc\(", code)]
    assert len(waits) == 1 and len(takes) == 1 and waits[0] < takes[0]


@pytest.mark.parametrize("name", ["experts_product.cu", "experts8_product.cu"])
def test_no_tile_is_empty(name):
    """The tiles of a group, by the arithmetic of the kernels' tile table: for every length of
    a group and every limit, the tiles add up to it and none is empty (an MMA of width 0 is an
    illegal instruction)."""
    widest = int(re.search(r"kTileN = (\d+);", source(name)).group(1))
    limits = re.search(r"int next_cap\(int cap\) { return cap > (\d+) \? (\d+) : (\d+); }", source("experts_tiles.cuh"))
    caps = [widest, int(limits.group(2)), int(limits.group(3))]
    assert int(limits.group(1)) == caps[1] and widest <= 256
    for cap in caps:
        for n in range(1, 2000):
            tiles = -(-n // cap)
            width = (-(-n // tiles) + 15) & ~15
            rows = [min(width, n - j * width) for j in range(tiles)]
            assert width <= cap and min(rows) >= 1 and sum(rows) == n


@pytest.mark.parametrize("call", ["values", "matmul", "expert_up", "weights", "gated weights"])
def test_codes_that_want_a_gradient_are_refused(call):
    from paper_2609_32398_gb300 import experts8

    def blocks(*size, gated=False, grad=False):
        exps = [*size[:-2], 2 if gated else size[-2] if len(size) == 2 else 1, 1]
        codes = torch.zeros(size).to(torch.float8_e4m3fn)
        return experts8.Blocks(codes.requires_grad_(grad), torch.zeros(exps, dtype=torch.uint8), gated)

    b = blocks(4, 64, grad=True)
    w = blocks(2, 64, 64, grad=True)
    g = blocks(2, 128, 64, gated=True, grad=True)
    run = {"values": b.values,
           "matmul": lambda: experts8.matmul(b, w),
           "expert_up": lambda: experts8.expert_up(b, g, torch.zeros(3, dtype=torch.int32)),
           "weights": lambda: w.check("w2", 3, False, 0),
           "gated weights": lambda: g.check("w1", 3, True, 0)}[call]
    with pytest.raises(RuntimeError, match="gradient"):
        run()
    with torch.no_grad(), pytest.raises(ValueError):  # on the CPU, which is refused next
        w.check("w2", 3, False, -1)
