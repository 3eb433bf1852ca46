"""The experts of an MoE layer on the router's dispatch order: grouped products
with ragged groups, the SwiGLU up projection with its 8-bit activation
checkpoint, the gradients, and the layer as one autograd node.

Argument marshalling over libdoloss.so (include/doloss.h); torch supplies
device memory and the current stream.  There is no CPU fallback.

Layouts: tokens x [T,H], expert weights w1 [E,2F,H] (gate rows, then up rows)
and w2 [E,H,F], all bf16; offsets [E+1], rows [T*k] and pos [T,k] int32 and
combine [T,k] fp32 as `doloss.routing()` writes them for one layer
(`dispatch_of(route, l)`).  H and the columns of every matrix are multiples of
8, F a multiple of 16.

    ids, combine, route = dl.route(z, k)
    offsets, rows, pos = dispatch_of(route)
    out = expert_ffn(x, w1, w2, combine, offsets, rows, pos)    # differentiable
"""
from __future__ import annotations

import threading

import torch

from . import doloss as dl

_flags_lock = threading.Lock()
_flags: dict[int, torch.Tensor] = {}


def _status(t: torch.Tensor) -> torch.Tensor:
    """The device's status word, which every call on it may set (see device_status)."""
    f = _flags.get(t.device.index)
    if f is None:
        with _flags_lock:
            f = _flags.get(t.device.index)
            if f is None:
                f = torch.zeros(64, dtype=torch.int32, device=t.device)
                torch.cuda.synchronize(t.device)  # cleared for every stream
                _flags[t.device.index] = f
    return f


def device_status(device="cuda") -> int:
    """Synchronizes the current stream, returns and clears what the calls of this
    module recorded on the device: 0, DO_ERR_TIMEOUT or DO_ERR_INVALID_ARG (a
    row or position outside its matrix, left out)."""
    f = _status(torch.empty(0, device=device))
    return int(dl.lib().do_device_status(f.data_ptr(), dl._stream(f)))


def _bf16(name: str, t: torch.Tensor, dim: int) -> None:
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != dim or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous CUDA bfloat16 tensor of {dim} dimensions")


def _index(name: str, t, n: int) -> None:
    if t is not None and (t.dtype != torch.int32 or not t.is_cuda or t.numel() != n
                          or not t.is_contiguous()):
        raise ValueError(f"{name} must be a contiguous CUDA int32 tensor of {n} values")


def _same_device(a: torch.Tensor, *others) -> None:
    for t in others:
        if t is not None and t.device != a.device:
            raise ValueError("all tensors must be on one device")


class Checkpoint:
    """Pre-activations [R, 2F] kept in 8 bits: codes int8 [R, 2F] and exponents
    uint8 [R, 2F/16]; the value of a code is code * 2^(e - 127), e the exponent
    of its block of 16 columns (255: the block held a NaN or an infinity)."""

    __slots__ = ("codes", "exponents")

    def __init__(self, codes: torch.Tensor, exponents: torch.Tensor):
        self.codes = codes
        self.exponents = exponents

    def check(self, R: int, F: int) -> None:
        c, e = self.codes, self.exponents
        if (c.dtype != torch.int8 or e.dtype != torch.uint8 or tuple(c.shape) != (R, 2 * F)
                or e.numel() * 16 != c.numel() or not (c.is_cuda and e.is_cuda)
                or not (c.is_contiguous() and e.is_contiguous())):
            raise ValueError("a checkpoint holds contiguous CUDA codes int8 [R,2F] and exponents "
                             "uint8 [R,2F/16]")

    def values(self) -> torch.Tensor:
        """The values it stands for, bf16 [R, 2F] (7 significant bits: exact)."""
        R, n = self.codes.shape
        self.check(R, n // 2)
        out = torch.empty(R, n, dtype=torch.bfloat16, device=self.codes.device)
        if R:
            dl._check("do_checkpoint_values", dl.lib().do_checkpoint_values(
                self.codes.data_ptr(), self.exponents.data_ptr(), R, n, out.data_ptr(),
                dl._stream(out)))
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
    rows [R] None: the R rows of x are in dispatch order."""
    _bf16("x", x, 2)
    _bf16("w1", w1, 3)
    T, H = x.shape
    E, F2, Hw = w1.shape
    if Hw != H or F2 % 2:
        raise ValueError("w1 must be [E, 2F, H] for x [T, H]")
    _same_device(x, w1, offsets, rows)
    R = T if rows is None else rows.numel()
    _index("offsets", offsets, E + 1)
    _index("rows", rows, R)
    F = F2 // 2
    act = torch.empty(R, F, dtype=torch.bfloat16, device=x.device)
    kept = None
    if checkpoint:
        kept = Checkpoint(torch.empty(R, F2, dtype=torch.int8, device=x.device),
                          torch.empty(R, F2 // 16, dtype=torch.uint8, device=x.device))
    if R:
        dl._check("do_expert_up", dl.lib().do_expert_up(
            x.data_ptr(), w1.data_ptr(), dl._ptr(rows), offsets.data_ptr(), T, H, F, E, R,
            act.data_ptr(), kept.codes.data_ptr() if kept else None,
            kept.exponents.data_ptr() if kept else None, _status(x).data_ptr(), dl._stream(x)))
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
    (y = a w)."""
    _bf16("a", a, 2)
    _bf16("w", w, 3)
    E, N, K = _weights(a, w, transposed)
    _same_device(a, w, offsets, rows)
    T = a.shape[0]
    R = T if rows is None else rows.numel()
    _index("offsets", offsets, E + 1)
    _index("rows", rows, R)
    y = torch.empty(R, N, dtype=torch.bfloat16, device=a.device)
    if R:
        dl._check("do_grouped_matmul", dl.lib().do_grouped_matmul(
            a.data_ptr(), w.data_ptr(), dl._ptr(rows), offsets.data_ptr(), T, K, N, E, R,
            int(bool(transposed)), y.data_ptr(), _status(a).data_ptr(), dl._stream(a)))
    return y


def grouped_matmul_join(a: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, pos: torch.Tensor,
                        weights: torch.Tensor | None = None, transposed: bool = False) -> torch.Tensor:
    """do_grouped_matmul_join: out [T,N] bf16, the products of grouped_matmul on
    the rows a [T*k,K] in dispatch order, summed per token over its rows
    pos [T,k] with weights [T,k] fp32 (None: one each)."""
    _bf16("a", a, 2)
    _bf16("w", w, 3)
    E, N, K = _weights(a, w, transposed)
    _same_device(a, w, offsets, pos, weights)
    if pos.dim() != 2 or pos.numel() != a.shape[0]:
        raise ValueError("pos must be [T, k] for a [T*k, K]")
    T, k = pos.shape
    _index("offsets", offsets, E + 1)
    _index("pos", pos, T * k)
    if weights is not None and (weights.dtype != torch.float32 or weights.shape != pos.shape
                                or not weights.is_contiguous()):
        raise ValueError("weights must be a contiguous float32 tensor shaped like pos")
    out = torch.empty(T, N, dtype=torch.bfloat16, device=a.device)
    if T:
        L = dl.lib()
        ws = torch.empty(int(L.do_grouped_matmul_join_workspace_size(T, k, N)), dtype=torch.uint8,
                         device=a.device)
        dl._check("do_grouped_matmul_join", L.do_grouped_matmul_join(
            a.data_ptr(), w.data_ptr(), offsets.data_ptr(), pos.data_ptr(), dl._ptr(weights), T, k,
            K, N, E, int(bool(transposed)), out.data_ptr(), _status(a).data_ptr(), ws.data_ptr(),
            ws.numel(), dl._stream(a)))
    return out


def expert_up_backward(dout: torch.Tensor, w2: torch.Tensor, kept: Checkpoint,
                       combine: torch.Tensor, offsets: torch.Tensor, rows: torch.Tensor,
                       pos: torch.Tensor):
    """do_expert_up_backward: the gradient dout [T,H] of the layer's output
    through the join, the down projection w2 [E,H,F] and the activation, from
    the 8-bit checkpoint.  Returns (dz [R,2F] bf16, act [R,F] bf16 times each
    row's combine weight, the operand of dW2, dcombine [T,k] fp32)."""
    _bf16("dout", dout, 2)
    _bf16("w2", w2, 3)
    T, H = dout.shape
    E, Hw, F = w2.shape
    if Hw != H:
        raise ValueError("w2 must be [E, H, F] for dout [T, H]")
    if combine.dim() != 2 or combine.shape[0] != T or combine.dtype != torch.float32 \
            or not combine.is_contiguous():
        raise ValueError("combine must be a contiguous float32 tensor of shape [T, k]")
    k = combine.shape[1]
    R = T * k
    _same_device(dout, w2, combine, offsets, rows, pos, kept.codes, kept.exponents)
    _index("offsets", offsets, E + 1)
    _index("rows", rows, R)
    _index("pos", pos, R)
    kept.check(R, F)
    dz = torch.empty(R, 2 * F, dtype=torch.bfloat16, device=dout.device)
    act = torch.empty(R, F, dtype=torch.bfloat16, device=dout.device)
    dcombine = torch.empty(T, k, dtype=torch.float32, device=dout.device)
    if R:
        L = dl.lib()
        ws = torch.empty(int(L.do_expert_up_backward_workspace_size(T, k, F)), dtype=torch.uint8,
                         device=dout.device)
        dl._check("do_expert_up_backward", L.do_expert_up_backward(
            dout.data_ptr(), w2.data_ptr(), kept.codes.data_ptr(), kept.exponents.data_ptr(),
            combine.data_ptr(), rows.data_ptr(), offsets.data_ptr(), pos.data_ptr(), T, k, H, F, E,
            dz.data_ptr(), act.data_ptr(), dcombine.data_ptr(), _status(dout).data_ptr(),
            ws.data_ptr(), ws.numel(), dl._stream(dout)))
    return dz, act, dcombine


def grouped_weight_grad(p: torch.Tensor, q: torch.Tensor, offsets: torch.Tensor,
                        p_rows: torch.Tensor | None = None, q_rows: torch.Tensor | None = None,
                        out: torch.Tensor | None = None, accumulate: bool = False) -> torch.Tensor:
    """do_grouped_weight_grad: dw [E,M,N] fp32, dw[e] = sum over the expert's rows
    r of p[p_rows[r]]^T q[q_rows[r]] (p [.,M], q [.,N] bf16; rows None: r itself).
    With accumulate it is added to `out`."""
    _bf16("p", p, 2)
    _bf16("q", q, 2)
    _same_device(p, q, offsets, p_rows, q_rows, out)
    sizes = {t.numel() for t in (p_rows, q_rows) if t is not None}
    sizes |= {t.shape[0] for t, r in ((p, p_rows), (q, q_rows)) if r is None}
    if len(sizes) != 1:
        raise ValueError("p and q must have one row (or row index) for each routed row")
    R = sizes.pop()
    E, M, N = offsets.numel() - 1, p.shape[1], q.shape[1]
    _index("offsets", offsets, E + 1)
    _index("p_rows", p_rows, R)
    _index("q_rows", q_rows, R)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs the out to add to")
        out = torch.empty(E, M, N, dtype=torch.float32, device=p.device)
    if tuple(out.shape) != (E, M, N) or out.dtype != torch.float32 or not out.is_contiguous():
        raise ValueError("out must be a contiguous float32 tensor of shape [E, M, N]")
    if R == 0:
        return out if accumulate else out.zero_()
    dl._check("do_grouped_weight_grad", dl.lib().do_grouped_weight_grad(
        p.data_ptr(), q.data_ptr(), dl._ptr(p_rows), dl._ptr(q_rows), offsets.data_ptr(),
        p.shape[0], q.shape[0], M, N, E, R, int(bool(accumulate)), out.data_ptr(),
        _status(p).data_ptr(), dl._stream(p)))
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
        x, w1, w2, combine, offsets, rows, pos, codes, exponents = ctx.saved_tensors
        dout = dout.contiguous()
        dz, act, dcombine = expert_up_backward(dout, w2, Checkpoint(codes, exponents), combine,
                                               offsets, rows, pos)
        need = ctx.needs_input_grad
        dw1 = dw2 = dx = None
        if ctx.main_grads is not None:
            grouped_weight_grad(dz, x, offsets, None, rows, out=ctx.main_grads[0], accumulate=True)
            grouped_weight_grad(dout, act, offsets, rows, None, out=ctx.main_grads[1], accumulate=True)
        else:
            if need[1]:
                dw1 = grouped_weight_grad(dz, x, offsets, None, rows)
            if need[2]:
                dw2 = grouped_weight_grad(dout, act, offsets, rows, None)
        if need[0]:
            dx = grouped_matmul_join(dz, w1, offsets, pos, None, transposed=True)
        return dx, dw1, dw2, dcombine, None, None, None, None


def expert_ffn(x: torch.Tensor, w1: torch.Tensor, w2: torch.Tensor, combine: torch.Tensor,
               offsets: torch.Tensor, rows: torch.Tensor, pos: torch.Tensor,
               main_grads: tuple[torch.Tensor, torch.Tensor] | None = None) -> torch.Tensor:
    """The experts of one MoE layer: out[t] = sum_q combine[t,q] W2_e (silu(g) * u)
    with (g, u) = W1_e x[t], e the q-th expert of token t; out [T,H] bf16.
    Differentiable in x, w1, w2 and combine; the backward pass works from 8-bit
    pre-activations.  main_grads: (dw1 [E,2F,H], dw2 [E,H,F]) fp32 buffers that
    the weights' gradients are added to instead of being returned."""
    if torch.is_grad_enabled() and any(t.requires_grad for t in (x, w1, w2, combine)):
        return _ExpertFFN.apply(x, w1, w2, combine, offsets, rows, pos, main_grads)
    act, _ = expert_up(x, w1, offsets, rows)
    return grouped_matmul_join(act, w2, offsets, pos, combine)
