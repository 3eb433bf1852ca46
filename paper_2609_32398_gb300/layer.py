"""A whole MoE layer forward for the few tokens of a decode step: router, Top-K, the
experts' two projections and their join, in two kernels (five where bf16 experts have
many tokens each).

Argument marshalling over libdoloss.so (include/doloss.h), by the rules of
`experts`: torch supplies device memory and the current stream, there is no CPU
fallback, the tensors of a call are on the current device, and what a call
records on the device is read by `experts.device_status`.

    out, ids, combine = moe_layer(x, wr, w1, w2, k)      # x [T,H] bf16, T <= 64

For more tokens, and where gradients are wanted, the same layer is
`doloss.route` on the logits and `experts.expert_ffn` (or `experts8.expert_ffn`).
"""
from __future__ import annotations

import functools

import torch
import torch.autograd.forward_ad as fwd

from . import doloss as dl
from .experts import _bf16, _device, _flag_ptrs, _no_tangent, _raw_stream, _status
from .experts8 import Blocks

MAX_TOKENS = 64


@functools.lru_cache(maxsize=256)
def _bytes(T: int, k: int, H: int, F: int) -> int:
    return int(dl.lib().do_moe_layer_workspace_size(T, k, H, F))


def moe_layer(x: torch.Tensor, wr: torch.Tensor, w1, w2, k: int, gate: int = dl.GATE_SIGMOID_NORM):
    """do_moe_layer: (out [T,H] bf16, expert ids [T,k] int32, combine [T,k] fp32) of tokens
    x [T,H] (at most 64), router weights wr [E,H] and expert weights w1 [E,2F,H], w2 [E,H,F],
    all bf16, or w1 and w2 both as `experts8.Blocks` (w1 gated).  out[t] = sum_q combine[t,q]
    W2_e (silu(g) * u) with (g, u) = W1_e x[t], e = ids[t,q] the k largest of wr x[t].
    Not differentiable."""
    eight = isinstance(w1, Blocks)
    if eight != isinstance(w2, Blocks):
        raise ValueError("w1 and w2 must both be bf16 tensors or both Blocks")
    c1, c2 = (w1.codes, w2.codes) if eight else (w1, w2)
    if fwd._current_level >= 0:
        _no_tangent("moe_layer", x, wr, *(() if eight else (w1, w2)))
    if ((x.requires_grad or wr.requires_grad or (not eight and (w1.requires_grad or w2.requires_grad)))
            and torch.is_grad_enabled()):
        raise RuntimeError("moe_layer is not differentiable: call it under torch.no_grad(), or take doloss.route "
                           "and experts.expert_ffn, whose gradients are")
    dev = _device(x)
    _bf16("x", x, 2, dev)
    _bf16("wr", wr, 2, dev)
    if eight:
        w1.check("w1", 3, True, dev)
        w2.check("w2", 3, False, dev)
    else:
        _bf16("w1", w1, 3, dev)
        _bf16("w2", w2, 3, dev)
    T, H = x.shape
    E, F2, Hw = c1.shape
    F = F2 // 2
    if Hw != H or F2 % 2 or c2.shape != (E, H, F) or wr.shape != (E, H):
        raise ValueError("wr must be [E, H], w1 [E, 2F, H] and w2 [E, H, F] for x [T, H]")
    k = int(k)
    if not 1 <= k <= E:
        raise ValueError("k must be between 1 and the number of experts")
    if T > MAX_TOKENS:
        raise ValueError(f"moe_layer takes {MAX_TOKENS} tokens at most: doloss.route and expert_ffn take any number")
    device = x.device
    out = torch.empty((T, H), dtype=torch.bfloat16, device=device)
    ids = torch.empty((T, k), dtype=torch.int32, device=device)
    combine = torch.empty((T, k), dtype=torch.float32, device=device)
    if T:
        n = _bytes(T, k, H, F)
        ws = torch.empty(n, dtype=torch.uint8, device=device)
        st = (dl._lib or dl.lib()).do_moe_layer(
            x.data_ptr(), wr.data_ptr(), c1.data_ptr(), w1.exponents.data_ptr() if eight else None, c2.data_ptr(),
            w2.exponents.data_ptr() if eight else None, T, H, F, E, k, gate, out.data_ptr(), ids.data_ptr(),
            combine.data_ptr(), _flag_ptrs.get(dev) or _status(dev), ws.data_ptr(), n, _raw_stream(dev))
        if st:
            dl._check("do_moe_layer", st)
    return out, ids, combine
