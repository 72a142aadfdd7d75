"""The expert layer of the examples: its pass and its gradients against the same layer in float64 with the quantization passed
straight through, the form for single tokens against the batch, and that training it works.

Tolerance, fixed before the first run: everything in the layer is float32 but the 4-bit values, which are the same on both sides
where float32 and float64 quantize the hidden values alike.  A hidden value near a decision boundary may go to the next level:
a few in 10^5, each changing a term of an output by a level.  So outputs are compared in the 2-norm, 1e-3 of the whole, with the
hidden activations' 4-bit form taken from the layer itself, whose own error is 1e-5."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    spec = importlib.util.spec_from_file_location("expert_layer", os.path.join(ROOT, "examples", "expert_layer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("T,E,k,K,H", [(1, 4, 2, 64, 96), (37, 5, 3, 100, 70), (300, 8, 2, 256, 320)])
def test_pass_and_gradients(ex, T, E, k, K, H):
    apb, layer = ex.apb, ex.ExpertLayer(E, k, K, H, seed=T)
    g = torch.Generator(device="cuda").manual_seed(T)
    x = torch.randn(T, K, generator=g, device="cuda")
    dy = torch.randn(T, K, generator=g, device="cuda")
    y, saved = layer.forward(x)
    got = dict(zip(("x", "router", "w1", "w2"), layer.backward(dy, saved)))
    r, x4, a4 = saved[1], saved[2], saved[4]
    R = T * k

    leaf = {"x": x, "router": layer.router, "w1": layer.w1, "w2": layer.w2}
    leaf = {n: v.double().cpu().requires_grad_() for n, v in leaf.items()}
    through = lambda v, q: v + (q.double().cpu() - v).detach()               # the value of q, the gradient of v
    xq, aq = apb.apb_mx4_dequantize(x4, R, K), apb.apb_mx4_dequantize(a4, R, H)
    w1 = through(leaf["w1"], apb.apb_mx4_dequantize(layer.q1, E * H, K))
    w2 = through(leaf["w2"], apb.apb_mx4_dequantize(layer.q2, E * K, H))
    token, off = r["row_token"].long().cpu(), r["offsets"].tolist()
    rows = through(leaf["x"][token], xq)
    z = []
    for e in range(E):
        part = slice(off[e], off[e + 1])
        h = rows[part] @ w1[e * H:(e + 1) * H].t()
        z.append(through(torch.relu(h), aq[part]) @ w2[e * K:(e + 1) * K].t())
    z = torch.cat(z)
    logits = leaf["x"] @ leaf["router"].t()
    weight = torch.softmax(logits.gather(1, r["expert"].long().cpu()), 1)
    want = (z[r["slot_row"].long().cpu()] * weight[:, :, None]).sum(1)
    (want * dy.double().cpu()).sum().backward()

    near = lambda a, b: (a.double().cpu() - b).norm() <= 1e-3 * b.norm()
    assert near(y, want.detach())
    for n in leaf:
        assert near(got[n], leaf[n].grad), n


def test_one_token_at_a_time_and_training(ex):
    losses, batch, one = ex.main(tokens=512, experts=4, width=128, hidden=128, steps=12)
    assert losses[-1] < 0.6 * losses[0] and batch.float().abs().max() > 0.5
    # bfloat16 outputs of bfloat16 hidden values: a rounding of each (2^-8) and few hidden values on another level
    assert (one.float() - batch[:8].float()).norm() <= 0.02 * batch[:8].float().norm()
