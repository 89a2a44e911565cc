"""The planned transformer with its gated feed-forward, its loss against a vocabulary and its gradients clipped: the
same bits at every budget, and gradients against automatic differentiation in 64 bits."""
import sys

import numpy as np
import pytest
import torch

from oracle import nodes
from paper_1910_02653_amd import ckm
from test_gpu_planned_transformer import example, matmul

pytestmark = pytest.mark.gpu


def small(dtype=torch.float32, **kw):
    return example.Stack(blocks=2, tokens=24, hidden=40, heads=4, p=0.2, seed=5, dtype=dtype, matmul=matmul, gated=True,
                         vocab=150, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
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
            stack.execute(plan)
            now = {"norm": stack.clip(0.1)}
            now.update({k: v.clone() for k, v in stack.grads.items()})
            now["loss"] = stack.loss.clone()
            counts.append(int((plan[:, 0] == ckm.OP_COMPUTE).sum()))
            seen = seen or now
            assert now.keys() == seen.keys() and len(now) == 2 * 9 + 1 + 2
            for k in now:
                assert torch.equal(now[k], seen[k]), (budget, k)
        assert counts[0] == len(stack.nodes) < counts[-1]
    finally:
        g.close()


def test_gradients_against_automatic_differentiation_in_64_bits():
    """Binary32 nodes: values of order 1, sums of at most 160 terms, paths of some 25 nodes: relative errors below 25 x
    160 x 2^-24 = 2.4e-4 of a gradient's norm, as for the stack without these operators; the norm's own no more."""
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
        g = y @ P[b, "gate"]
        x = h + ((g * torch.sigmoid(g) * (y @ P[b, "up"])) @ P[b, "down"]) * factor(b, 2, S, H)
    logits = x @ P[stack.blocks, "head"].t()
    loss = (torch.logsumexp(logits, 1) - logits.gather(1, stack.target.cpu()[:, None])[:, 0]).mean()
    loss.backward()
    assert abs(float(stack.loss) - float(loss.detach())) < 2.4e-4 * float(loss.detach())
    for key, g in stack.grads.items():
        want = P[key].grad * stack.LOSS_SCALE
        off = (g.double().cpu() - want).norm() / want.norm()
        assert off < 2.4e-4, (key, float(off))
    whole = torch.stack([P[k].grad.square().sum() for k in stack.grads]).sum().sqrt()
    before = {k: v.clone() for k, v in stack.grads.items()}
    norm = float(stack.clip(0.5 * float(whole)))
    assert abs(norm - float(whole)) < 2.4e-4 * float(whole)
    for k, v in stack.grads.items():   # the factor is off by as much, and rounded
        assert float((v - before[k] * 0.5).norm()) <= 2.5e-4 * float(before[k].norm())


def test_the_commands_that_the_example_names(monkeypatch, capsys):
    commands = [line.split()[1:] for line in example.__doc__.split("\n") if line.startswith("    python ")]
    assert any("--gated" in c for c in commands)
    for c in commands:
        print("%s" % c, flush=True)
        monkeypatch.setattr(sys, "argv", c)
        example.main()
    out = capsys.readouterr().out
    assert out.count("equal the first budget's") == 3 * len(commands), out
