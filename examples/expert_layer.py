"""An MoE layer on the library: router, DO-loss and experts trained for a few steps
on synthetic tokens, then one token at a time through the trained layer.

    python examples/expert_layer.py [steps]

The router is a fp32 linear map; routing and combine weights come from `route`,
the DO-loss from `do_loss`, and the experts (bf16 weights, fp32 master copies and
gradients) from `expert_ffn`, whose backward pass works from 8-bit
pre-activations.  Prints the loss and the load's MaxVio per step, and the largest
difference between the layer's rows and the same tokens served one by one.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2609_32398_gb300 import doloss as dl  # noqa: E402
from paper_2609_32398_gb300 import experts as ex  # noqa: E402

T, H, F, E, k = 4096, 256, 128, 32, 4
DO_WEIGHT, LR = 1e-2, 0.3


def main(steps: int = 8) -> None:
    dl.lib()
    g = torch.Generator("cuda").manual_seed(0)

    def draw(*shape, scale):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    x = draw(T, H, scale=1.0).bfloat16()
    target = draw(T, H, scale=1.0).bfloat16()
    router = draw(E, H, scale=0.1).requires_grad_()
    master = [draw(E, 2 * F, H, scale=H ** -0.5), draw(E, H, F, scale=F ** -0.5)]
    grads = [torch.zeros_like(m) for m in master]
    ranks = (torch.arange(E, device="cuda") % 8).to(torch.int32)

    def layer(tokens):
        z = tokens.float() @ router.T
        _, combine, route = dl.route(z, k)
        return z, route, ex.expert_ffn(tokens, w1, w2, combine, *ex.dispatch_of(route), main_grads=tuple(grads))

    for step in range(steps):
        w1, w2 = (m.bfloat16().requires_grad_() for m in master)
        z, route, out = layer(x)
        loss = (out.float() - target.float()).square().mean()
        (loss + DO_WEIGHT * dl.do_loss(z, k)).backward()
        vio = dl.maxvio(route.counts, ranks, 8)
        print(f"step {step}: loss {float(loss.detach()):.5f}  MaxVio {float(vio[0]):.3f}")
        with torch.no_grad():
            for m, d in zip(master, grads):
                m -= LR * H * d
                d.zero_()
            router -= LR * router.grad
            router.grad = None
    if ex.device_status() != 0:
        raise RuntimeError("a device wait ran out")
    with torch.no_grad():
        w1, w2 = (m.bfloat16() for m in master)
        _, _, whole = layer(x[:64])
        single = torch.cat([layer(x[t:t + 1])[2] for t in range(64)])
    print(f"served one by one: largest difference {float((whole - single).abs().max()):.4f} "
          f"of {float(whole.abs().max()):.4f}")


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 8)
