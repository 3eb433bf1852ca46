"""The experts of an MoE layer on the router's dispatch order: grouped products
with ragged groups, the SwiGLU up projection with its 8-bit activation
checkpoint, the gradients, and the layer as one autograd node.

Argument marshalling over libdoloss.so (include/doloss.h); torch supplies
device memory and the current stream.  There is no CPU fallback, and the tensors
of a call are on the current device.

Layouts: tokens x [T,H], expert weights w1 [E,2F,H] (gate rows, then up rows)
and w2 [E,H,F], all bf16; offsets [E+1], rows [T*k] and pos [T,k] int32 and
combine [T,k] fp32 as `doloss.routing()` writes them for one layer
(`dispatch_of(route, l)`).  H and the columns of every matrix are multiples of
8, F a multiple of 16.

    ids, combine, route = dl.route(z, k)
    offsets, rows, pos = dispatch_of(route)
    out = expert_ffn(x, w1, w2, combine, offsets, rows, pos)    # differentiable

The other calls are the pieces of its forward and backward pass and leave no graph:
the forward ones raise where an operand requires a gradient and one is recorded.
"""
from __future__ import annotations

import threading

import torch
import torch.autograd.forward_ad as fwd

from . import doloss as dl

_flags_lock = threading.Lock()
_flags: dict[int, torch.Tensor] = {}
_flag_ptrs: dict[int, int] = {}


def _status(device: int) -> int:
    """Address of the device's status word, which every call on it may set.  It is made by the
    first call, which therefore cannot be captured."""
    p = _flag_ptrs.get(device)
    if p is None:
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the first call of this module on a device makes its status word, outside of a graph "
                               "capture: call device_status() before the capture")
        with _flags_lock:
            f = torch.zeros(64, dtype=torch.int32, device=f"cuda:{device}")
            torch.cuda.synchronize(device)  # cleared for every stream
            _flags.setdefault(device, f)
            p = _flag_ptrs.setdefault(device, _flags[device].data_ptr())
    return p


def device_status(device="cuda") -> int:
    """Synchronizes the current stream, returns and clears what the calls of this
    module recorded on the device, on any stream: 0, DO_ERR_TIMEOUT (a bounded
    wait ran out: results of calls since the last poll may be wrong) or
    DO_ERR_INVALID_ARG (a row or position outside its matrix, left out).  There is
    one word a device, which a poll clears for everybody.  A call before the first
    graph capture makes it."""
    t = torch.empty(0, device=device)
    return int(dl.lib().do_device_status(_status(_device(t)), dl._stream(t)))


def _device(t: torch.Tensor) -> int:
    """The device of a call's tensors (-1: the CPU), which has to be the current one: streams
    and launches are the current device's."""
    dev = t.get_device()
    if dev > 0 or (dev == 0 and not dl._only_device):
        dl._check_current(dev)
    return dev


# (not torch.cuda.is_available(): asking the driver here would leave the children of a later
# fork without their GPU)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _bf16(name: str, t: torch.Tensor, dim: int, device: int) -> None:
    if t.dtype is not torch.bfloat16 or t.dim() != dim or not t.is_contiguous() or t.get_device() != device \
            or device < 0:
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor of {dim} dimensions, "
                         "all tensors on one device")


def _index(name: str, t, n: int, device: int) -> None:
    if t is not None and (t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous()
                          or t.get_device() != device):
        raise ValueError(f"{name} must be a contiguous CUDA int32 tensor of {n} values, "
                         "all tensors on one device")


def _no_tangent(name: str, *tensors) -> None:
    """Forward-mode derivatives are refused: a kernel would drop the tangent."""
    if any(t is not None and fwd.unpack_dual(t).tangent is not None for t in tensors):
        raise RuntimeError(f"{name} has no forward-mode derivative")


def _no_graph(name: str, a: torch.Tensor, w: torch.Tensor, weights=None) -> None:
    """The pieces of the layer are no autograd nodes: where a graph is being recorded,
    operands that want one are refused instead of being detached."""
    if fwd._current_level >= 0:
        _no_tangent(name, a, w, weights)
    if ((a.requires_grad or w.requires_grad or (weights is not None and weights.requires_grad))
            and torch.is_grad_enabled()):
        raise RuntimeError(f"{name} is not differentiable: call it under torch.no_grad(), or take expert_ffn, "
                           "whose gradients are")


def _fp32(name: str, t, shape: tuple, device: int) -> None:
    if t is not None and (t.dtype is not torch.float32 or t.shape != shape or not t.is_contiguous()
                          or t.get_device() != device):
        raise ValueError(f"{name} must be a contiguous CUDA float32 tensor of shape {list(shape)}, "
                         "all tensors on one device")


def _positions(pos: torch.Tensor, T: int, k: int, device: int) -> torch.Tensor:
    """pos as [T, k], which a flat one of T*k values is too."""
    _index("pos", pos, T * k, device)
    if pos.shape == (T, k):
        return pos
    if pos.dim() != 1:
        raise ValueError(f"pos must be [T, k], here {[T, k]}")
    return pos.view(T, k)


class Checkpoint:
    """Pre-activations [R, 2F] kept in 8 bits: codes int8 [R, 2F] and exponents
    uint8 [R, 2F/16]; the value of a code is code * 2^(e - 127), e the exponent
    of its block of 16 columns (255: the block held a NaN or an infinity)."""

    __slots__ = ("codes", "exponents")

    def __init__(self, codes: torch.Tensor, exponents: torch.Tensor):
        self.codes = codes
        self.exponents = exponents

    def check(self, R: int, F: int, device: int) -> None:
        c, e = self.codes, self.exponents
        if (c.dtype is not torch.int8 or e.dtype is not torch.uint8 or c.shape != (R, 2 * F)
                or e.numel() * 16 != c.numel() or c.get_device() != device or e.get_device() != device
                or device < 0 or not (c.is_contiguous() and e.is_contiguous())):
            raise ValueError("a checkpoint holds contiguous CUDA codes int8 [R,2F] and exponents "
                             "uint8 [R,2F/16], all tensors on one device")

    def values(self) -> torch.Tensor:
        """The values it stands for, bf16 [R, 2F] (7 significant bits: exact)."""
        codes = self.codes
        dev = _device(codes)
        R, n = codes.shape
        self.check(R, n // 2, dev)
        out = codes.new_empty((R, n), dtype=torch.bfloat16)
        if R:
            dl._check("do_checkpoint_values", dl.lib().do_checkpoint_values(
                codes.data_ptr(), self.exponents.data_ptr(), R, n, out.data_ptr(), _raw_stream(dev)))
        return out


def dispatch_of(route: "dl.Routing", layer: int = 0):
    """(offsets [E+1], rows [T*k], pos [T,k]) of one layer of a Routing."""
    if route.offsets is None:
        raise ValueError("the routing was made without its dispatch order")
    return route.offsets[layer], route.rows[layer], route.pos[layer]


def expert_up(x: torch.Tensor, w1: torch.Tensor, offsets: torch.Tensor,
              rows: torch.Tensor | None = None, checkpoint: bool = False):
    """do_expert_up: act [R,F] bf16 = silu(z_gate) * z_up with z = x[rows] W1^T
    of each row's expert, and with `checkpoint` the Checkpoint of z (else None).
    rows [R] None: the R rows of x are in dispatch order.  Not differentiable."""
    _no_graph("expert_up", x, w1)
    dev = _device(x)
    _bf16("x", x, 2, dev)
    _bf16("w1", w1, 3, dev)
    T, H = x.shape
    E, F2, Hw = w1.shape
    if Hw != H or F2 % 2:
        raise ValueError("w1 must be [E, 2F, H] for x [T, H]")
    R = T if rows is None else rows.numel()
    _index("offsets", offsets, E + 1, dev)
    _index("rows", rows, R, dev)
    F = F2 // 2
    act = x.new_empty((R, F))
    kept = None
    if checkpoint:
        kept = Checkpoint(x.new_empty((R, F2), dtype=torch.int8),
                          x.new_empty((R, F2 // 16), dtype=torch.uint8))
    if R:
        dl._check("do_expert_up", dl.lib().do_expert_up(
            x.data_ptr(), w1.data_ptr(), dl._ptr(rows), offsets.data_ptr(), T, H, F, E, R,
            act.data_ptr(), kept.codes.data_ptr() if kept else None,
            kept.exponents.data_ptr() if kept else None, _status(dev), _raw_stream(dev)))
    return act, kept


def _weights(a, w, transposed):
    E = w.shape[0]
    N, K = (w.shape[2], w.shape[1]) if transposed else (w.shape[1], w.shape[2])
    if K != a.shape[1]:
        raise ValueError("w must be [E, N, K], or [E, K, N] where transposed, for a [., K]")
    return E, N, K


def grouped_matmul(a: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor,
                   rows: torch.Tensor | None = None, transposed: bool = False) -> torch.Tensor:
    """do_grouped_matmul: y [R,N] bf16, row r = a[rows[r]] (or a[r]) times the
    weights of its expert: w [E,N,K] (y = a w^T), or [E,K,N] where transposed
    (y = a w).  Not differentiable."""
    _no_graph("grouped_matmul", a, w)
    dev = _device(a)
    _bf16("a", a, 2, dev)
    _bf16("w", w, 3, dev)
    E, N, K = _weights(a, w, transposed)
    T = a.shape[0]
    R = T if rows is None else rows.numel()
    _index("offsets", offsets, E + 1, dev)
    _index("rows", rows, R, dev)
    y = a.new_empty((R, N))
    if R:
        dl._check("do_grouped_matmul", dl.lib().do_grouped_matmul(
            a.data_ptr(), w.data_ptr(), dl._ptr(rows), offsets.data_ptr(), T, K, N, E, R,
            int(bool(transposed)), y.data_ptr(), _status(dev), _raw_stream(dev)))
    return y


def grouped_matmul_join(a: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, pos: torch.Tensor,
                        weights: torch.Tensor | None = None, transposed: bool = False) -> torch.Tensor:
    """do_grouped_matmul_join: out [T,N] bf16, the products of grouped_matmul on
    the rows a [T*k,K] in dispatch order, summed per token over its rows
    pos [T,k] with weights [T,k] fp32 (None: one each).  The products are kept in
    fp32 up to T k N = 25165824 values and rounded to bf16 before the sum beyond.
    Not differentiable."""
    _no_graph("grouped_matmul_join", a, w, weights)
    dev = _device(a)
    _bf16("a", a, 2, dev)
    _bf16("w", w, 3, dev)
    E, N, K = _weights(a, w, transposed)
    if pos.dim() != 2 or pos.numel() != a.shape[0]:
        raise ValueError("pos must be [T, k] for a [T*k, K]")
    T, k = pos.shape
    _index("offsets", offsets, E + 1, dev)
    _index("pos", pos, T * k, dev)
    _fp32("weights", weights, (T, k), dev)
    if k == 0:
        return a.new_zeros((T, N))
    out = a.new_empty((T, N))
    if T:
        L = dl.lib()
        n = L.do_grouped_matmul_join_workspace_size(T, k, N)
        ws = a.new_empty(n, dtype=torch.uint8)
        dl._check("do_grouped_matmul_join", L.do_grouped_matmul_join(
            a.data_ptr(), w.data_ptr(), offsets.data_ptr(), pos.data_ptr(), dl._ptr(weights), T, k,
            K, N, E, int(bool(transposed)), out.data_ptr(), _status(dev), ws.data_ptr(),
            n, _raw_stream(dev)))
    return out


def expert_up_backward(dout: torch.Tensor, w2: torch.Tensor, kept: Checkpoint,
                       combine: torch.Tensor, offsets: torch.Tensor, rows: torch.Tensor,
                       pos: torch.Tensor):
    """do_expert_up_backward: the gradient dout [T,H] of the layer's output
    through the join, the down projection w2 [E,H,F] and the activation, from
    the 8-bit checkpoint.  Returns (dz [R,2F] bf16, act [R,F] bf16 times each
    row's combine weight, the operand of dW2, dcombine [T,k] fp32)."""
    dev = _device(dout)
    _bf16("dout", dout, 2, dev)
    _bf16("w2", w2, 3, dev)
    T, H = dout.shape
    E, Hw, F = w2.shape
    if Hw != H:
        raise ValueError("w2 must be [E, H, F] for dout [T, H]")
    if combine.dim() != 2:
        raise ValueError("combine must be [T, k]")
    k = combine.shape[1]
    R = T * k
    _fp32("combine", combine, (T, k), dev)
    _index("offsets", offsets, E + 1, dev)
    _index("rows", rows, R, dev)
    pos = _positions(pos, T, k, dev)
    kept.check(R, F, dev)
    dz = dout.new_empty((R, 2 * F))
    act = dout.new_empty((R, F))
    dcombine = combine.new_empty((T, k))
    if R:
        L = dl.lib()
        n = L.do_expert_up_backward_workspace_size(T, k, F)
        ws = dout.new_empty(n, dtype=torch.uint8)
        dl._check("do_expert_up_backward", L.do_expert_up_backward(
            dout.data_ptr(), w2.data_ptr(), kept.codes.data_ptr(), kept.exponents.data_ptr(),
            combine.data_ptr(), rows.data_ptr(), offsets.data_ptr(), pos.data_ptr(), T, k, H, F, E,
            dz.data_ptr(), act.data_ptr(), dcombine.data_ptr(), _status(dev), ws.data_ptr(),
            n, _raw_stream(dev)))
    return dz, act, dcombine


def grouped_weight_grad(p: torch.Tensor, q: torch.Tensor, offsets: torch.Tensor,
                        p_rows: torch.Tensor | None = None, q_rows: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """do_grouped_weight_grad: dw [E,M,N] fp32, dw[e] = sum over the expert's rows
    r of p[p_rows[r]]^T q[q_rows[r]] (p [.,M], q [.,N] bf16; rows None: r itself).
    With accumulate it is added to `out`."""
    dev = _device(p)
    _bf16("p", p, 2, dev)
    _bf16("q", q, 2, dev)
    sizes = {t.numel() for t in (p_rows, q_rows) if t is not None}
    sizes |= {t.shape[0] for t, r in ((p, p_rows), (q, q_rows)) if r is None}
    if len(sizes) != 1:
        raise ValueError("p and q must have one row (or row index) for each routed row")
    R = sizes.pop()
    E, M, N = offsets.numel() - 1, p.shape[1], q.shape[1]
    _index("offsets", offsets, E + 1, dev)
    _index("p_rows", p_rows, R, dev)
    _index("q_rows", q_rows, R, dev)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the out to add to")
        out = p.new_empty((E, M, N), dtype=torch.float32)
    _fp32("out", out, (E, M, N), dev)
    if R == 0:
        return out if accumulate else out.zero_()
    dl._check("do_grouped_weight_grad", dl.lib().do_grouped_weight_grad(
        p.data_ptr(), q.data_ptr(), dl._ptr(p_rows), dl._ptr(q_rows), offsets.data_ptr(),
        p.shape[0], q.shape[0], M, N, E, R, int(bool(accumulate)), out.data_ptr(),
        _status(dev), _raw_stream(dev)))
    return out


class _ExpertFFN(torch.autograd.Function):
    """The experts of one layer as an autograd node.  The forward keeps its inputs
    and the 8-bit checkpoint of the pre-activations; nothing of the routed rows is
    kept in bf16."""

    @staticmethod
    def forward(ctx, x, w1, w2, combine, offsets, rows, pos, main_grads):
        act, kept = expert_up(x, w1, offsets, rows, checkpoint=True)
        out = grouped_matmul_join(act, w2, offsets, pos, combine)
        ctx.save_for_backward(x, w1, w2, combine, offsets, rows, pos, kept.codes, kept.exponents)
        ctx.main_grads = main_grads
        return out

    @staticmethod
    def backward(ctx, dout):
        args = (dout.contiguous(), *ctx.saved_tensors, ctx.main_grads, ctx.needs_input_grad)
        # under create_graph the gradients get a graph too, whose only node raises
        grads = (_ExpertFFNGrad.apply if torch.is_grad_enabled() else _expert_ffn_grad)(*args)
        return (*grads, None, None, None, None)


def _expert_ffn_grad(dout, x, w1, w2, combine, offsets, rows, pos, codes, exponents, main_grads, need):
    """(dx, dw1, dw2, dcombine) of the layer, None where not needed."""
    dz, act, dcombine = expert_up_backward(dout, w2, Checkpoint(codes, exponents), combine, offsets, rows, pos)
    dw1 = dw2 = dx = None
    add = main_grads is not None
    to1, to2 = main_grads if add else (None, None)
    if need[1]:
        dw1 = grouped_weight_grad(dz, x, offsets, None, rows, out=to1, accumulate=add)
    if need[2]:
        dw2 = grouped_weight_grad(dout, act, offsets, rows, None, out=to2, accumulate=add)
    if add:  # nothing else is returned for them
        dw1 = dw2 = None
    if need[0]:
        dx = grouped_matmul_join(dz, w1, offsets, pos, None, transposed=True)
    return dx, dw1, dw2, dcombine


class _ExpertFFNGrad(torch.autograd.Function):
    """The layer's gradients as a node without a derivative: the kernels leave no graph, so
    that second-order terms through x, the weights, combine or dout would be left out."""

    @staticmethod
    def forward(ctx, *args):
        return _expert_ffn_grad(*args)

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("expert_ffn has no second derivative")


def expert_ffn(x: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor, combine: torch.Tensor,
               offsets: torch.Tensor, rows: torch.Tensor, pos: torch.Tensor,
               main_grads: tuple[torch.Tensor, torch.Tensor] | None = None) -> torch.Tensor:
    """The experts of one MoE layer: out[t] = sum_q combine[t,q] W2_e (silu(g) * u)
    with (g, u) = W1_e x[t], e the q-th expert of token t; out [T,H] bf16.
    Differentiable once in x, w1, w2 and combine (a second derivative raises); the
    backward pass works from 8-bit pre-activations.  main_grads: (dw1 [E,2F,H],
    dw2 [E,H,F]) fp32 buffers that the gradients of the weights that require one are
    added to instead of being returned.  The activations are rounded to bf16 between
    the two products, and the second one's rows before their sum as in
    grouped_matmul_join."""
    if fwd._current_level >= 0:
        _no_tangent("expert_ffn", x, w1, w2, combine)
    dev = _device(x)
    _bf16("x", x, 2, dev)
    _bf16("w1", w1, 3, dev)
    _bf16("w2", w2, 3, dev)
    T, H = x.shape
    E, F2, Hw = w1.shape
    F = F2 // 2
    if Hw != H or F2 % 2 or w2.shape != (E, H, F) or combine.dim() != 2:
        raise ValueError("w1 must be [E, 2F, H], w2 [E, H, F] and combine [T, k] for x [T, H]")
    k = combine.shape[1]
    _fp32("combine", combine, (T, k), dev)
    _index("offsets", offsets, E + 1, dev)
    _index("rows", rows, T * k, dev)
    pos = _positions(pos, T, k, dev)
    if main_grads is not None:
        if len(main_grads) != 2 or any(b is None for b in main_grads):
            raise ValueError("main_grads must be a pair of buffers, of w1 and of w2")
        _fp32("main_grads[0]", main_grads[0], w1.shape, dev)
        _fp32("main_grads[1]", main_grads[1], w2.shape, dev)
    if ((x.requires_grad or w1.requires_grad or w2.requires_grad or combine.requires_grad)
            and torch.is_grad_enabled()):
        return _ExpertFFN.apply(x, w1, w2, combine, offsets, rows, pos, main_grads)
    if k == 0:
        return x.new_zeros((T, H))
    out = x.new_empty((T, H))
    if T:
        L = dl.lib()
        n = L.do_expert_ffn_workspace_size(T, k, H, F)
        ws = x.new_empty(n, dtype=torch.uint8)
        dl._check("do_expert_ffn", L.do_expert_ffn(
            x.data_ptr(), w1.data_ptr(), w2.data_ptr(), combine.data_ptr(), rows.data_ptr(),
            offsets.data_ptr(), pos.data_ptr(), T, k, H, F, E, out.data_ptr(), _status(dev),
            ws.data_ptr(), n, _raw_stream(dev)))
    return out
