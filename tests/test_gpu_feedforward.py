"""examples/feedforward.py: what it computes, and its gradients against automatic differentiation of the same block in float32."""
import importlib.util
import os

import pytest
import torch

from paper_2104_08378_amd import sp24

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("feedforward", os.path.join(ROOT, "examples", "feedforward.py"))
feedforward = importlib.util.module_from_spec(spec)
spec.loader.exec_module(feedforward)


def test_decoding_in_8_bits():
    # two products on operands of 1 part in 127 of their largest (four standard deviations): 4 / 127 / sqrt(12) = 0.9 % each, four operands
    assert feedforward.decode(torch.Generator(device="cuda").manual_seed(1)) < 0.02


def test_fine_tuning_lowers_the_loss_and_keeps_the_pattern():
    losses = feedforward.fine_tune(torch.Generator(device="cuda").manual_seed(1))
    assert all(b < a for a, b in zip(losses, losses[1:])) and losses[-1] < 0.8 * losses[0]


def test_gradients_of_a_block():
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    E, H, F, N, topk = 4, 128, 192, 90, 2
    block = feedforward.ExpertBlock(1 + 0.1 * n(H), n(E * F, H) / H ** 0.5, n(E * H, F) / F ** 0.5, 0.1 * n(E * F), E)
    x, stream, dout = (n(N, H).to(torch.bfloat16) for _ in range(3))
    choice = n(N, E).topk(topk, dim=1)
    ids, weights = choice.indices.to(torch.int32), torch.softmax(choice.values, 1)
    ids[5:9] = -1                                                # tokens of no expert
    out, kept = block(x, stream, ids, weights)
    d = block.backward(dout, kept)

    leaves = dict(x=x.float(), norm=block.norm.clone(), up=block.up.master.to(torch.bfloat16).float(), down=block.down.master.to(torch.bfloat16).float(),
                  bias=block.bias.clone(), weights=weights.clone())
    leaves = {k: v.requires_grad_(True) for k, v in leaves.items()}
    with torch.enable_grad():
        h = leaves["x"] + stream.float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + 1e-6) * leaves["norm"]
        total = h
        for e in range(E):
            z = torch.nn.functional.gelu(y @ leaves["up"][e * F:(e + 1) * F].t() + leaves["bias"][e * F:(e + 1) * F], approximate="tanh")
            total = total + (z @ leaves["down"][e * H:(e + 1) * H].t()) * (leaves["weights"] * (ids == e)).sum(1, keepdim=True)
    total.backward(dout.float())
    # every value passes up to five roundings to 8 bits (2^-9 each on average); a gradient is a sum of many such
    assert float((out.float() - total.detach()).norm() / total.detach().norm()) < 0.01
    for k, v in d.items():
        want = leaves[k].grad
        if k in ("up", "down"):
            want = want * (leaves[k] != 0)
        assert float((v.float() - want).norm() / want.norm()) < 0.015, k
