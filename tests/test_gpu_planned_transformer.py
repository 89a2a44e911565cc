"""The example that trains a transformer stack by a plan: every budget gives the same numbers.

Matrix products are elementary here (products and sums in binary32), so that
nothing but the operators and the plan could make a difference: outputs and
gradients are compared bit for bit between plans, and with automatic
differentiation of the formulas in 64 bits.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

from conftest import ROOT
from oracle import nodes
from paper_1910_02653_amd import ckm

pytestmark = pytest.mark.gpu

spec = importlib.util.spec_from_file_location("planned_transformer", os.path.join(ROOT, "examples", "planned_transformer.py"))
example = importlib.util.module_from_spec(spec)
spec.loader.exec_module(example)


def matmul(a, b):
    return (a.float().unsqueeze(-1) * b.float().unsqueeze(-3)).sum(-2).to(a.dtype)


def small(dtype=torch.float32, **kw):
    return example.Stack(blocks=2, tokens=24, hidden=40, heads=4, p=0.2, seed=5, dtype=dtype, matmul=matmul, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_every_budget_gives_the_same_gradients(dtype):
    stack = small(dtype)
    size, cost = stack.measure()
    g, s = example.graph_of(stack, size, cost)
    try:
        total = int(size.sum()) + 4 * stack.input.numel() * stack.input.element_size() + 2 * sum(
            t.numel() * t.element_size() for t in stack.params.values())
        least = int(g.threshold_eval(s, np.arange(len(stack.nodes) + 1) / len(stack.nodes), 1 << 60)["peak"].min())
        seen, counts = None, []
        for budget in (total, (total + least) // 2, least):
            plan, mem, _ = example.choose(stack, g, s, size, budget)
            assert mem.max() <= budget
            stack.grads.clear()
            grads = stack.execute(plan)
            now = {k: v.clone() for k, v in grads.items()}
            now["loss"] = stack.loss.clone()
            counts.append(int((plan[:, 0] == ckm.OP_COMPUTE).sum()))
            if seen is None:
                seen = now
            assert now.keys() == seen.keys() and len(now) == 2 * 8 + 1
            for k in now:
                assert torch.equal(now[k], seen[k]), (budget, k)
        assert counts[0] == len(stack.nodes) < counts[-1]   # the smallest budget computes nodes again
    finally:
        g.close()
    # another step draws other masks
    other = small(dtype, step=1)
    other.execute([(ckm.OP_COMPUTE, k, k, k) for k in range(len(other.nodes))])
    assert not torch.equal(other.loss, seen["loss"])


def test_gradients_against_automatic_differentiation_in_64_bits():
    """Binary32 nodes against the formulas in 64 bits. Values are of order 1, a sum has at most 160 terms, a path some
    25 nodes: relative errors below 25 x 160 x 2^-24 = 2.4e-4 of a gradient's norm."""
    stack = small()
    stack.execute([(ckm.OP_COMPUTE, k, k, k) for k in range(len(stack.nodes))])
    S, H, heads = stack.tokens, stack.hidden, stack.heads
    P = {k: v.double().cpu().requires_grad_() for k, v in stack.params.items()}

    def factor(block, place, rows, cols):
        d = stack._drop(block, place)
        return torch.from_numpy(nodes.factors(rows, cols, d.seed, d.site, d.keep))

    x = stack.input.double().cpu()
    for b in range(stack.blocks):
        norm = torch.nn.functional.layer_norm
        y = norm(x, (H,), P[b, "ln1"], P[b, "ln1_bias"])
        q, k, v = (t.view(S, heads, -1).transpose(0, 1) for t in (y @ P[b, "qkv"]).chunk(3, 1))
        t = (q @ k.transpose(1, 2)) * (H // heads) ** -0.5
        t = t.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -float("inf"))
        p = t.softmax(-1) * factor(b, 0, heads * S, S).view(heads, S, S)
        a = (p @ v).transpose(0, 1).reshape(S, H) @ P[b, "proj"]
        h = x + a * factor(b, 1, S, H)
        y = norm(h, (H,), P[b, "ln2"], P[b, "ln2_bias"])
        x = h + (torch.nn.functional.gelu(y @ P[b, "up"]) @ P[b, "down"]) * factor(b, 2, S, H)
    loss = 0.5 * (x - stack.target.double().cpu()).square().mean()
    loss.backward()
    assert abs(float(stack.loss) - float(loss.detach())) < 2.4e-4 * float(loss.detach())
    for key, g in stack.grads.items():
        want = P[key].grad * 1024.0
        off = (g.double().cpu() - want).norm() / want.norm()
        assert off < 2.4e-4, (key, float(off))
