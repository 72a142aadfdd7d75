"""A gated feed-forward block on frozen 4-bit weights whose requests bring low-rank adapters: tuned on several sequences at once, with
its activations kept in 8 bits, then served a token of every request at a time.

    python examples/adapter_block.py

Y = W_d (act(G) * U), [G | U] = W_gu X; both products run on 4-bit weights and activations, and every sequence adds the low-rank
product of its own adapter to both.  The adapters are latent in float32 and cast for the kernels after each update.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2306_08960_amd import binding as apb


class AdapterBlock:
    def __init__(self, width, hidden, adapters, rank, activation="silu", dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        new = lambda *shape: torch.randn(*shape, generator=g, device="cuda") * shape[-1] ** -0.5
        self.K, self.H, self.L, self.activation, self.dtype = width, hidden, adapters, activation, dtype
        self.q_gu, self.q_d = apb.apb_mx4_quantize(new(2 * hidden, width)), apb.apb_mx4_quantize(new(width, hidden))
        # both sides of the two adapters; the second side starts at zero, so that the block starts as it is without them
        self.latent = {"a_gu": new(adapters, rank, width), "b_gu": torch.zeros(adapters, rank, 2 * hidden, device="cuda"),
                       "a_d": new(adapters, rank, hidden), "b_d": torch.zeros(adapters, rank, width, device="cuda")}
        self.scale = torch.full((adapters,), 2.0, device="cuda")
        self.cast()

    def cast(self):
        self.f = {name: w.to(self.dtype) for name, w in self.latent.items()}

    def forward(self, x, seg):
        """x [M, width], seg: the sequences' offsets and adapters -> y [M, width], and what backward needs."""
        M, f = x.shape[0], self.f
        gu = apb.apb_mx4_linear(x, self.q_gu, 2 * self.H)
        t_gu = apb.apb_adapter_down(x, f["a_gu"], scale=self.scale, **seg)
        apb.apb_adapter_up(t_gu, f["b_gu"], Y0=gu, Y=gu, **seg)
        saved = apb.alloc_mx8(2 * M, self.H)
        h = apb.apb_gated_forward(gu, self.activation, saved=saved)
        y = apb.apb_mx4_linear(h, self.q_d, self.K)
        t_d = apb.apb_adapter_down(h, f["a_d"], scale=self.scale, **seg)
        apb.apb_adapter_up(t_d, f["b_d"], Y0=y, Y=y, **seg)
        return y, (apb.apb_mx8_quantize(x), t_gu, saved, t_d, seg)

    def backward(self, dy, kept):
        """The gradients of x and of the adapters' sides; the 4-bit quantization is passed straight through."""
        x8, t_gu, saved, t_d, seg = kept
        f, grad = self.f, {}
        dt = apb.apb_adapter_down(dy, f["b_d"], scale=self.scale, **seg)
        dh = apb.apb_mx4_backward_input(dy, self.q_d, self.H)
        apb.apb_adapter_up(dt, f["a_d"], Y0=dh, Y=dh, **seg)
        h = torch.empty_like(dh)
        dgu = apb.apb_gated_backward(saved, dh, self.activation, Y=h)
        grad["b_d"] = apb.apb_adapter_gradient(t_d, dy, self.L, **seg)
        grad["a_d"] = apb.apb_adapter_gradient(dt, h, self.L, **seg)
        dt = apb.apb_adapter_down(dgu, f["b_gu"], scale=self.scale, **seg)
        dx = apb.apb_mx4_backward_input(dgu, self.q_gu, self.K)
        apb.apb_adapter_up(dt, f["a_gu"], Y0=dx, Y=dx, **seg)
        grad["b_gu"] = apb.apb_adapter_gradient(t_gu, dgu, self.L, **seg)
        grad["a_gu"] = apb.apb_adapter_gradient(dt, x8, self.L, K=self.K, **seg)
        return dx, grad

    def serve(self, x, seg=None):
        """The forward pass without anything kept.  seg None: nobody has an adapter, and both projections are one kernel."""
        if seg is None:
            return apb.apb_mx4_linear(apb.apb_mx4_gated_linear(x, self.q_gu, self.H, self.activation), self.q_d, self.K)
        f = self.f
        gu = apb.apb_mx4_linear(x, self.q_gu, 2 * self.H)
        apb.apb_adapter_up(apb.apb_adapter_down(x, f["a_gu"], scale=self.scale, **seg), f["b_gu"], Y0=gu, Y=gu, **seg)
        h = apb.apb_gated_forward(gu, self.activation)
        y = apb.apb_mx4_linear(h, self.q_d, self.K)
        apb.apb_adapter_up(apb.apb_adapter_down(h, f["a_d"], scale=self.scale, **seg), f["b_d"], Y0=y, Y=y, **seg)
        return y


def segments(lengths, adapters):
    """Sequences of these lengths, one after another, with these adapters (-1: none)."""
    off = [0]
    for n in lengths:
        off.append(off[-1] + n)
    return dict(offsets=torch.tensor(off, dtype=torch.int32, device="cuda"), adapter=torch.tensor(adapters, dtype=torch.int32, device="cuda"))


def main(width=256, hidden=512, rank=16, steps=60, rate=0.05):
    block, goal = AdapterBlock(width, hidden, 3, rank), AdapterBlock(width, hidden, 3, rank)
    g = torch.Generator(device="cuda").manual_seed(5)
    for name in ("b_gu", "b_d"):                                     # (what the adapters shall learn)
        goal.latent[name] = torch.randn(goal.latent[name].shape, generator=g, device="cuda") * 0.1
    goal.cast()
    lengths, adapters = [300, 150, 420, 80, 74], [0, 2, 1, 0, -1]
    seg = segments(lengths, adapters)
    x = torch.randn(sum(lengths), width, generator=g, device="cuda").bfloat16()
    want = goal.serve(x, seg).float()
    losses = []
    for step in range(steps):
        y, kept = block.forward(x, seg)
        error = y.float() - want
        losses.append(error.square().mean().item())
        _, grad = block.backward((error / x.shape[0]).to(x.dtype), kept)
        for name in ("b_gu", "b_d"):
            block.latent[name] -= rate * grad[name]
        block.cast()
        if step % 10 == 0 or step == steps - 1:
            print(f"step {step:3d}  mean squared error {losses[-1]:.5f}", flush=True)
    batch = block.serve(x, seg)
    first = seg["offsets"][:-1].long()                               # the first token of every request, all in one step
    step = block.serve(x[first], segments([1] * len(lengths), adapters))
    print(f"a token of every request at a time differs from the prompts by {(step.float() - batch[first].float()).abs().max().item():.4f}"
          f" of {batch.float().abs().max().item():.2f}")
    return losses, batch[first], step


if __name__ == "__main__":
    main()
