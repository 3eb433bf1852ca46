"""What the expert operators' binding refuses on the host, before it touches a tensor's
memory or a device."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

from paper_2609_32398_gb300 import experts as ex

T, k, E, H, F = 4, 1, 2, 64, 16


def operands():
    """One of each operand, on the CPU: a call that gets past the checks tested here is
    refused as not being on a GPU, by a ValueError."""
    return dict(x=torch.zeros(T, H).bfloat16(), w1=torch.zeros(E, 2 * F, H).bfloat16(),
                w2=torch.zeros(E, H, F).bfloat16(), a=torch.zeros(T * k, F).bfloat16(), combine=torch.zeros(T, k),
                offsets=torch.zeros(E + 1, dtype=torch.int32), rows=torch.zeros(T * k, dtype=torch.int32),
                pos=torch.zeros(T, k, dtype=torch.int32))


# the layer's forward pieces, and their operands that have derivatives
CALLS = {
    "expert_up": (lambda o: ex.expert_up(o["x"], o["w1"], o["offsets"], o["rows"]), ("x", "w1")),
    "grouped_matmul": (lambda o: ex.grouped_matmul(o["a"], o["w2"], o["offsets"]), ("a", "w2")),
    "grouped_matmul_join": (lambda o: ex.grouped_matmul_join(o["a"], o["w2"], o["offsets"], o["pos"], o["combine"]),
                            ("a", "w2", "combine")),
}
EACH = [(name, operand) for name, (_, has) in CALLS.items() for operand in has]


@pytest.mark.parametrize("name,operand", EACH)
def test_a_call_that_leaves_no_graph_refuses_operands_that_want_one(name, operand):
    """Of the forward calls only expert_ffn is an autograd node: the others raise where a
    gradient would be lost."""
    o = operands()
    o[operand].requires_grad_()
    with pytest.raises(RuntimeError, match="expert_ffn"):
        CALLS[name][0](o)
    with torch.no_grad(), pytest.raises(ValueError):    # as without a gradient: not on a GPU
        CALLS[name][0](o)
    o[operand] = o[operand].detach()
    with pytest.raises(ValueError):
        CALLS[name][0](o)


LAYER = {**CALLS, "expert_ffn": (lambda o: ex.expert_ffn(o["x"], o["w1"], o["w2"], o["combine"], o["offsets"],
                                                         o["rows"], o["pos"]), ("x", "w1", "w2", "combine"))}


@pytest.mark.parametrize("name,operand", [(name, operand) for name, (_, has) in LAYER.items() for operand in has])
def test_forward_mode_derivatives_are_refused(name, operand):
    """A dual tensor needs no requires_grad: its tangent would be lost."""
    with fwd.dual_level():
        o = operands()
        o[operand] = fwd.make_dual(o[operand], torch.ones_like(o[operand]))
        with pytest.raises(RuntimeError, match="forward-mode"):
            LAYER[name][0](o)
        with torch.no_grad(), pytest.raises(RuntimeError, match="forward-mode"):   # which does not turn it off
            LAYER[name][0](o)
        o[operand] = fwd.unpack_dual(o[operand]).primal
        with pytest.raises(ValueError):
            LAYER[name][0](o)


class Elsewhere:
    """Stands for a tensor of device 1: all that may be asked of it before it is refused."""

    requires_grad = False

    def get_device(self):
        return 1


def test_tensors_of_a_device_that_is_not_current_are_refused(monkeypatch):
    """The streams and kernels of a call are the current device's: a tensor of another one is
    refused before anything is launched or read of it."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = Elsewhere()
    kept = ex.Checkpoint(t, t)
    for call in (lambda: ex.expert_up(t, t, t, t), lambda: ex.grouped_matmul(t, t, t),
                 lambda: ex.grouped_matmul_join(t, t, t, t, t), lambda: kept.values(),
                 lambda: ex.expert_up_backward(t, t, kept, t, t, t, t), lambda: ex.grouped_weight_grad(t, t, t),
                 lambda: ex.expert_ffn(t, t, t, t, t, t, t)):
        with pytest.raises(ValueError, match="current device"):
            call()


def test_importing_the_module_leaves_forked_children_their_gpu():
    """Nothing asks the driver for devices at import: a process may fork workers after it."""
    import os
    import subprocess
    import sys

    code = ("import os, torch, paper_2609_32398_gb300.experts\n"
            "pid = os.fork()\n"
            "if pid == 0:\n"
            "    os._exit(3 if torch.cuda._is_in_bad_fork() else 0)\n"
            "sys_exit = os.waitstatus_to_exitcode(os.waitpid(pid, 0)[1])\n"
            "raise SystemExit(sys_exit)\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    assert subprocess.run([sys.executable, "-c", code], cwd=root, timeout=300).returncode == 0


@pytest.mark.parametrize("d", [1000, 1021, 1023])
def test_tiles_that_a_reciprocal_cannot_divide_are_refused(d):
    """An expert's tiles are divided by its d weight tiles with ceil(2^32 / d), which is exact
    while a tile's number times (that d - 2^32) stays below 2^32.  Calls that could reach past it
    (1023 weight tiles, 1,055,232 rows, 276 GB of results) are refused before any launch."""
    from paper_2609_32398_gb300 import build, doloss as dl

    build.build()
    magic = 0xffffffff // d + 1
    last = (2 ** 32 - 1) // (magic * d - 2 ** 32)
    assert all(i * magic >> 32 == i // d for i in range(last - 3 * d, last + 1))
    assert any(i * magic >> 32 != i // d for i in range(last + 1, last + 3 * d))
    R, F = 256 * (last // d + 2), 128 * d
    fake = 0x10000
    assert dl.lib().do_expert_up(fake, fake, fake, fake, 1, 8, F, 1, R, fake, None, None, None, None) == 2
    n = dl.lib().do_expert_ffn_workspace_size(R, 1, 8, F)
    assert dl.lib().do_expert_ffn(*[fake] * 7, R, 1, 8, F, 1, fake, None, fake, n, None) == 2
