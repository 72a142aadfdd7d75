"""A mixture-of-experts feed-forward layer on 4-bit weights: trained on a batch of tokens, then used for one token at a time.

    python examples/expert_layer.py

Every token goes to k of E experts, each a two-layer perceptron; weights and activations are multiplied as microscaled 4-bit
matrices.  Latent weights stay in float32 and are quantized again after each update; gradients pass the quantization straight
through, as the binary layers' training operators have it.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2306_08960_amd import binding as apb


class ExpertLayer:
    def __init__(self, experts, k, width, hidden, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda rows, cols: torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5
        self.E, self.k, self.K, self.H = experts, k, width, hidden
        self.router = new(experts, width)
        self.w1, self.w2 = new(experts * hidden, width), new(experts * width, hidden)       # latent, one expert after another
        self.quantize()

    def quantize(self):
        self.q1, self.q2 = apb.apb_mx4_quantize(self.w1), apb.apb_mx4_quantize(self.w2)

    def forward(self, x):
        """x [T, width] -> y [T, width], and what backward needs."""
        r = apb.apb_moe_route(x.float() @ self.router.t(), self.k)
        rows, off = r["row_token"].numel(), r["offsets"]
        x4 = apb.apb_mx4_quantize(x, rows_from=r["row_token"])
        h = apb.apb_mx4_gemm(x4, self.q1, rows, self.H, self.K, dtype=x.dtype, offsets=off)
        a4 = apb.apb_mx4_quantize(torch.relu(h))
        z = apb.apb_mx4_gemm(a4, self.q2, rows, self.K, self.H, dtype=x.dtype, offsets=off)
        return apb.apb_moe_combine(z, r["slot_row"], r["weight"]), (x, r, x4, h, a4, z)

    def backward(self, dy, saved):
        """Gradients of x, the router and both layers' latent weights."""
        x, r, x4, h, a4, z = saved
        off = r["offsets"]
        dz, dweight = apb.apb_moe_combine_backward(dy, z, r["slot_row"], r["weight"])
        dw2 = apb.apb_mx4_backward_weight(dz, a4, self.H, offsets=off)
        dh = apb.apb_mx4_backward_input(dz, self.q2, self.H, offsets=off) * (h > 0)
        dw1 = apb.apb_mx4_backward_weight(dh, x4, self.K, offsets=off)
        dx = apb.apb_moe_combine(apb.apb_mx4_backward_input(dh, self.q1, self.K, offsets=off), r["slot_row"])
        dlogits = apb.apb_moe_route_backward(r["expert"], r["weight"], dweight, self.E)
        return dx + (dlogits @ self.router).to(dx.dtype), dlogits.t() @ x.float(), dw1, dw2

    def serve(self, x):
        """The forward pass without anything kept: activations are quantized inside the products."""
        r = apb.apb_moe_route(x.float() @ self.router.t(), self.k)
        h = apb.apb_mx4_linear(x, self.q1, self.H, rows_from=r["row_token"], offsets=r["offsets"])
        z = apb.apb_mx4_linear(torch.relu(h), self.q2, self.K, offsets=r["offsets"])
        return apb.apb_moe_combine(z, r["slot_row"], r["weight"])


def main(tokens=2048, experts=8, k=2, width=256, hidden=512, steps=60, rate=0.1):
    layer, goal = ExpertLayer(experts, k, width, hidden, seed=1), ExpertLayer(experts, k, width, hidden, seed=2)
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(tokens, width, generator=g, device="cuda").bfloat16()
    want = goal.forward(x)[0].float()
    losses = []
    for step in range(steps):
        y, saved = layer.forward(x)
        error = y.float() - want
        losses.append(error.square().mean().item())
        _, dr, dw1, dw2 = layer.backward((error / tokens).to(x.dtype), saved)
        layer.router -= rate * dr
        layer.w1 -= rate * dw1
        layer.w2 -= rate * dw2
        layer.quantize()
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}  mean squared error {losses[-1]:.4f}", flush=True)
    batch, one = layer.forward(x)[0], torch.cat([layer.serve(x[t:t + 1]) for t in range(8)])
    print(f"one token at a time differs from the batch by {(one.float() - batch[:8].float()).abs().max().item():.4f}"
          f" of {batch.float().abs().max().item():.2f}")
    return losses, batch, one


if __name__ == "__main__":
    main()
