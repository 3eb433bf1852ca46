"""The experts of an MoE layer with weights and activations in 8 bits: e4m3 codes and
a power of two for each block of 128, forward only, on the dispatch order of
`experts`.

Argument marshalling over libdoloss.so (include/doloss.h), by the rules of
`experts`: torch supplies device memory and the current stream, there is no CPU
fallback, the tensors of a call are on the current device, and what the calls
record on the device is read by `experts.device_status`.

Layouts: rows [M,K] have blocks of 1 x 128, weights [E,N,K] of 128 x 128, and a
gated w1 [E,2F,H] has its gate rows and its up rows blocked apart.  The inner size
of a product is a multiple of 16, N of 8.

    w1, w2 = quantise_weights(w1, gated=True), quantise_weights(w2)   # once
    out = expert_ffn(x, w1, w2, combine, offsets, rows, pos)          # x [T,H] bf16

or its pieces:

    act = expert_up(quantise_rows(x), w1, offsets, rows)              # in blocks again
    y = matmul(act, w2, offsets)                                      # [R,H] bf16

A dense map is matmul(a, w) with w [1,N,K] and no offsets.  Nothing here is
differentiable: an operand that wants a gradient while a graph is recorded is refused.
"""
from __future__ import annotations

import functools

import torch
import torch.autograd.forward_ad as fwd

from . import doloss as dl
from .experts import _bf16, _device, _flag_ptrs, _fp32, _index, _no_tangent, _positions, _raw_stream, _status

BLOCK = 128
_E4M3, _U8, _BF16 = torch.float8_e4m3fn, torch.uint8, torch.bfloat16


def _blocks(n: int) -> int:
    return (n + BLOCK - 1) // BLOCK


@functools.lru_cache(maxsize=256)
def _exponent_shape(name: str, size: torch.Size, gated: bool) -> tuple:
    if len(size) == 2:
        return size[0], _blocks(size[1])
    if not gated:
        return size[0], _blocks(size[1]), _blocks(size[2])
    if size[1] % 2:
        raise ValueError(f"{name} is gated and needs an even number of rows")
    return size[0], 2 * _blocks(size[1] // 2), _blocks(size[2])


class Blocks:
    """A matrix in blocks: codes float8_e4m3fn [M,K] (blocks of 1 x 128) or [E,N,K] (of 128 x
    128) and exponents uint8 [M,ceil(K/128)] or [E,ceil(N/128),ceil(K/128)]; gated: N = 2F and
    exponents [E,2 ceil(F/128),ceil(K/128)], the gate rows' before the up rows'.  The value
    of a code is code * 2^(e - 127), NaN where e = 255."""

    __slots__ = ("codes", "exponents", "gated")

    def __init__(self, codes: torch.Tensor, exponents: torch.Tensor, gated: bool = False):
        self.codes = codes
        self.exponents = exponents
        self.gated = bool(gated)

    def check(self, name: str, dim: int, gated: bool, device: int) -> None:
        c, e = self.codes, self.exponents
        if c.requires_grad and torch.is_grad_enabled():
            raise RuntimeError(f"the codes of {name} want a gradient, which the 8-bit experts do not have: call them "
                               "under torch.no_grad()")
        if (c.dtype is not _E4M3 or e.dtype is not _U8 or c.dim() != dim or device < 0
                or c.get_device() != device or e.get_device() != device
                or not (c.is_contiguous() and e.is_contiguous())):
            raise ValueError(f"{name} must be contiguous CUDA codes float8_e4m3fn of {dim} dimensions and "
                             "exponents uint8, all tensors on one device")
        if self.gated is not gated:
            raise ValueError(f"{name} must be {'' if gated else 'not '}gated")
        size = c.shape
        if e.shape != _exponent_shape(name, size, gated):
            raise ValueError(f"the exponents of {name} must be {list(_exponent_shape(name, size, gated))}, "
                             f"here {list(e.shape)}")

    def values(self) -> torch.Tensor:
        """do_block_values: the values it stands for, bf16, exact for what this module quantised."""
        c = self.codes
        dev = _device(c)
        dim = c.dim()
        if dim not in (2, 3):
            raise ValueError("codes are [M,K] or [E,N,K]")
        self.check("the matrix", dim, self.gated if dim == 3 else False, dev)
        out = torch.empty(c.shape, dtype=torch.bfloat16, device=c.device)
        if out.numel():
            K = c.shape[-1]
            planes, N, rows = 1, c.shape[0], 1
            if dim == 3:
                planes, N, rows = (2 * c.shape[0], c.shape[1] // 2, BLOCK) if self.gated else (*c.shape[:2], BLOCK)
            dl._check("do_block_values", dl.lib().do_block_values(
                c.data_ptr(), self.exponents.data_ptr(), planes, N, K, rows, out.data_ptr(), _raw_stream(dev)))
        return out


def _no_graph(name: str, x: torch.Tensor, combine: torch.Tensor | None = None) -> None:
    if fwd._current_level >= 0:
        _no_tangent(name, x, combine)
    if (x.requires_grad or (combine is not None and combine.requires_grad)) and torch.is_grad_enabled():
        raise RuntimeError(f"{name} is not differentiable: call it under torch.no_grad()")


@functools.lru_cache(maxsize=256)
def _ffn_bytes(T: int, k: int, H: int, F: int) -> int:
    return int(dl.lib().do_expert_ffn8_workspace_size(T, k, H, F))


def quantise_rows(x: torch.Tensor) -> Blocks:
    """do_quantise_rows: x [M,K] bf16 in blocks of 1 x 128."""
    _no_graph("quantise_rows", x)
    dev = _device(x)
    _bf16("x", x, 2, dev)
    M, K = x.shape
    device = x.device
    codes = torch.empty((M, K), dtype=_E4M3, device=device)
    exponents = torch.empty((M, (K + BLOCK - 1) // BLOCK), dtype=_U8, device=device)
    if M:
        st = (dl._lib or dl.lib()).do_quantise_rows(x.data_ptr(), M, K, codes.data_ptr(), exponents.data_ptr(),
                                                    _raw_stream(dev))
        if st:
            dl._check("do_quantise_rows", st)
    return Blocks(codes, exponents)


def quantise_weights(w: torch.Tensor, gated: bool = False) -> Blocks:
    """do_quantise_weights: w [E,N,K] bf16 in blocks of 128 x 128 (gated: the first and the
    second N/2 rows of an expert blocked apart)."""
    _no_graph("quantise_weights", w)
    dev = _device(w)
    _bf16("w", w, 3, dev)
    E, N, K = w.shape
    if gated and N % 2:
        raise ValueError("gated weights have an even number of rows")
    nb = 2 * _blocks(N // 2) if gated else _blocks(N)
    q = Blocks(torch.empty((E, N, K), dtype=torch.float8_e4m3fn, device=w.device),
               torch.empty((E, nb, _blocks(K)), dtype=torch.uint8, device=w.device), gated)
    if q.codes.numel():
        dl._check("do_quantise_weights", dl.lib().do_quantise_weights(
            w.data_ptr(), E, N, K, int(bool(gated)), q.codes.data_ptr(), q.exponents.data_ptr(), _raw_stream(dev)))
    return q


def _operands(a: Blocks, w: Blocks, gated: bool, offsets, rows, dev: int):
    if not isinstance(a, Blocks) or not isinstance(w, Blocks):
        raise ValueError("both operands must be Blocks (quantise_rows, quantise_weights)")
    a.check("the rows", 2, False, dev)
    w.check("the weights", 3, gated, dev)
    T, K = a.codes.shape
    E, N, Kw = w.codes.shape
    if Kw != K:
        raise ValueError("the weights must be [E, N, K] for rows [., K]")
    R = T
    if rows is not None:
        R = rows.numel()
        _index("rows", rows, R, dev)
    if offsets is not None:
        _index("offsets", offsets, E + 1, dev)
    elif E != 1:
        raise ValueError("offsets may be left out for a dense map, [1, N, K], only")
    return T, K, E, N, R


def matmul(a: Blocks, w: Blocks, offsets: torch.Tensor | None = None,
           rows: torch.Tensor | None = None) -> torch.Tensor:
    """do_grouped_matmul8: y [R,N] bf16, row r = a[rows[r]] (or a[r]) times the weights [E,N,K]
    of its expert; without offsets all rows go through the one map w [1,N,K]."""
    dev = _device(a.codes) if isinstance(a, Blocks) else -1
    T, K, E, N, R = _operands(a, w, False, offsets, rows, dev)
    codes = a.codes
    y = torch.empty((R, N), dtype=_BF16, device=codes.device)
    if R:
        st = (dl._lib or dl.lib()).do_grouped_matmul8(
            codes.data_ptr(), a.exponents.data_ptr(), w.codes.data_ptr(), w.exponents.data_ptr(),
            None if rows is None else rows.data_ptr(), None if offsets is None else offsets.data_ptr(), T, K, N, E, R,
            y.data_ptr(), _flag_ptrs.get(dev) or _status(dev), _raw_stream(dev))
        if st:
            dl._check("do_grouped_matmul8", st)
    return y


def expert_up(a: Blocks, w1: Blocks, offsets: torch.Tensor, rows: torch.Tensor | None = None) -> Blocks:
    """do_expert_up8: silu(z_gate) * z_up in blocks of 1 x 128, [R,F], with z = a[rows] w1^T of
    each row's expert (w1 gated)."""
    dev = _device(a.codes) if isinstance(a, Blocks) else -1
    if offsets is None:
        raise ValueError("expert_up needs the groups' offsets")
    T, H, E, F2, R = _operands(a, w1, True, offsets, rows, dev)
    F = F2 // 2
    act = Blocks(torch.empty((R, F), dtype=torch.float8_e4m3fn, device=a.codes.device),
                 torch.empty((R, _blocks(F)), dtype=torch.uint8, device=a.codes.device))
    if R:
        dl._check("do_expert_up8", dl.lib().do_expert_up8(
            a.codes.data_ptr(), a.exponents.data_ptr(), w1.codes.data_ptr(), w1.exponents.data_ptr(), dl._ptr(rows),
            offsets.data_ptr(), T, H, F, E, R, act.codes.data_ptr(), act.exponents.data_ptr(), _status(dev),
            _raw_stream(dev)))
    return act


def expert_ffn(x: torch.Tensor, w1: Blocks, w2: Blocks, combine: torch.Tensor, offsets: torch.Tensor,
               rows: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    """do_expert_ffn8: the experts of one MoE layer forward, as `experts.expert_ffn`, with weights
    w1 [E,2F,H] (gated) and w2 [E,H,F] in blocks; x [T,H] bf16 and the activations are
    quantised on the way.  out [T,H] bf16."""
    _no_graph("the 8-bit expert_ffn", x, combine)
    dev = _device(x)
    _bf16("x", x, 2, dev)
    if not isinstance(w1, Blocks) or not isinstance(w2, Blocks):
        raise ValueError("w1 and w2 must be Blocks (quantise_weights)")
    w1.check("w1", 3, True, dev)
    w2.check("w2", 3, False, dev)
    T, H = x.shape
    E, F2, Hw = w1.codes.shape
    F = F2 // 2
    if Hw != H or w2.codes.shape != (E, H, F) or combine.dim() != 2:
        raise ValueError("w1 must be [E, 2F, H], w2 [E, H, F] and combine [T, k] for x [T, H]")
    k = combine.shape[1]
    _fp32("combine", combine, (T, k), dev)
    _index("offsets", offsets, E + 1, dev)
    _index("rows", rows, T * k, dev)
    pos = _positions(pos, T, k, dev)
    if k == 0:
        return x.new_zeros((T, H))
    device = x.device
    out = torch.empty((T, H), dtype=_BF16, device=device)
    if T:
        n = _ffn_bytes(T, k, H, F)
        ws = torch.empty(n, dtype=_U8, device=device)
        st = (dl._lib or dl.lib()).do_expert_ffn8(
            x.data_ptr(), w1.codes.data_ptr(), w1.exponents.data_ptr(), w2.codes.data_ptr(), w2.exponents.data_ptr(),
            combine.data_ptr(), rows.data_ptr(), offsets.data_ptr(), pos.data_ptr(), T, k, H, F, E, out.data_ptr(),
            _flag_ptrs.get(dev) or _status(dev), ws.data_ptr(), n, _raw_stream(dev))
        if st:
            dl._check("do_expert_ffn8", st)
    return out
