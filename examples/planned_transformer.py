"""Train a transformer block stack within a memory budget, by a plan of the framework.

The forward and gradient nodes of a stack of pre-norm transformer blocks (the
block of the package's transformer workload, its elementwise nodes fused) are
numbered in topological order with their bytes and measured costs. The
threshold family rounds one score per value into candidate schedules, the
cheapest within the budget is chosen, Algorithm 1 turns it into statements,
and the statements are executed on the GPU: dropout, layer norm, attention
softmax and their gradients by the package's operators, matrix products by the
library. With --gated the feed-forward is the gated one, one node forward and
one for its gradient, which keeps no projection; with --vocab the loss is the
cross entropy against a vocabulary, whose logits never exist; with --clip the
gradients' norm is bounded at the end of the step. A node that a stage computes
again has the bits it had before (its dropout masks are functions of seed, site,
row and column), so a budget changes memory and time and no number.

    python examples/planned_transformer.py --blocks 4 --tokens 1024 --budgets 100 60 40
    python examples/planned_transformer.py --gated --vocab 32768 --clip 1.0 --budgets 100 60 50
"""
from __future__ import annotations

import argparse
import os
import sys
import time
from typing import NamedTuple

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1910_02653_amd import ckm, ops  # noqa: E402
from paper_1910_02653_amd import workloads as wl  # noqa: E402


class Node(NamedTuple):
    name: str
    deps: list      # node numbers
    run: object     # values of deps -> tuple of tensors


class Stack:
    """Parameters and nodes of a block stack, one training step long. gated: a gated feed-forward; vocab: the size of
    a vocabulary whose next tokens are the target (0: a squared error)."""

    LOSS_SCALE = 1024.0   # against underflow

    def __init__(self, blocks=2, tokens=512, hidden=512, heads=8, p=0.1, seed=1, step=0, dtype=torch.float16,
                 matmul=torch.matmul, gated=False, vocab=0):
        self.blocks, self.tokens, self.hidden, self.heads, self.p = blocks, tokens, hidden, heads, p
        self.seed, self.step, self.mm, self.gated, self.vocab = seed, step, matmul, gated, vocab
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape, gain=1.0):
            return (gain * torch.randn(shape, generator=gen, device="cuda")).to(dtype)

        h = hidden
        self.params, self.grads = {}, {}
        for b in range(blocks):
            for name, shape in (("qkv", (h, 3 * h)), ("proj", (h, h)), ("up", (h, 4 * h)), ("down", (4 * h, h)),
                                *((("gate", (h, 4 * h)),) if gated else ())):
                self.params[b, name] = normal(*shape, gain=shape[0] ** -0.5)
            for name in ("ln1", "ln2"):   # norms keep 32-bit weights
                self.params[b, name] = torch.ones(h, device="cuda")
                self.params[b, name + "_bias"] = torch.zeros(h, device="cuda")
        self.input, self.target = normal(tokens, h), normal(tokens, h)
        if vocab:
            self.params[blocks, "head"] = normal(vocab, h, gain=h ** -0.5)
            self.target = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
            self.d_loss = torch.full((tokens,), self.LOSS_SCALE / tokens, device="cuda")   # of the mean
        self.nodes = []
        self._build()

    def _drop(self, block, place):
        """Each dropout of each block and step has its own site."""
        return ops.Dropout(self.p, self.seed, (self.step << 32) | (block * 4 + place))

    def _add(self, name, deps, run):
        self.nodes.append(Node(name, deps, run))
        return len(self.nodes) - 1

    def _build(self):
        scale = (self.hidden // self.heads) ** -0.5
        place = []   # node numbers of each block
        x = None     # the stack's input is held outside the plan
        for b in range(self.blocks):
            n = {"x": x}
            self._forward(b, n, scale)
            place.append(n)
            x = n["out"]

        def loss(out):
            diff = out[0].float() - self.target.float()
            self.loss = 0.5 * diff.square().mean()
            return ((diff / diff.numel()).mul(self.LOSS_SCALE).to(out[0].dtype),)

        def token_loss(out):
            rows, lse = ops.cross_entropy(out[0], self.params[self.blocks, "head"], self.target)
            self.loss = rows.mean()
            return rows, lse

        def d_token_loss(out, loss):
            dx, self.grads[self.blocks, "head"] = ops.cross_entropy_backward(
                self.d_loss, out[0], self.params[self.blocks, "head"], self.target, loss[1])
            return (dx,)

        if self.vocab:
            grad = self._add("d_loss", [x, self._add("loss", [x], token_loss)], d_token_loss)
        else:
            grad = self._add("loss", [x], loss)
        for b in reversed(range(self.blocks)):
            grad = self._backward(b, place[b], grad, scale)

    def _heads(self, t):   # [tokens, hidden] -> [heads, tokens, hidden / heads]
        return t.view(self.tokens, self.heads, -1).transpose(0, 1).contiguous()

    def _merged(self, t):
        return t.transpose(0, 1).reshape(self.tokens, self.hidden)

    def _x(self, n, rest):
        """(the block's input, the other values): the first block's input is no node."""
        return (self.input, rest) if n["x"] is None else (rest[0][0], rest[1:])

    def _forward(self, b, n, scale):
        P, mm, drop = self.params, self.mm, self._drop
        xs = [] if n["x"] is None else [n["x"]]

        def ln1(*v):
            y, _, stats = ops.layer_norm(self._x(n, v)[0], P[b, "ln1"], P[b, "ln1_bias"])
            return y, stats

        def qkv(a):
            return tuple(self._heads(t) for t in mm(a[0], P[b, "qkv"]).chunk(3, 1))

        def ln2(*v):
            x, (a,) = self._x(n, v)
            return ops.layer_norm(a[0], P[b, "ln2"], P[b, "ln2_bias"], residual=x, drop=drop(b, 1))

        n["ln1"] = self._add("ln1", xs, ln1)
        n["qkv"] = self._add("qkv", [n["ln1"]], qkv)
        n["scores"] = self._add("scores", [n["qkv"]], lambda t: (mm(t[0], t[1].transpose(1, 2).contiguous()),))
        n["probs"] = self._add("probs", [n["scores"]],
                               lambda s: ops.softmax(s[0], scale, causal=True, drop=drop(b, 0)))
        n["context"] = self._add("context", [n["qkv"], n["probs"]], lambda t, p: (self._merged(mm(p[0], t[2])),))
        n["proj"] = self._add("proj", [n["context"]], lambda c: (mm(c[0], P[b, "proj"]),))
        n["ln2"] = self._add("ln2", xs + [n["proj"]], ln2)   # (y, h, statistics)
        if self.gated:
            n["act"] = self._add("gated", [n["ln2"]], lambda a: (ops.gated(a[0], P[b, "gate"], P[b, "up"]),))
        else:
            n["up"] = self._add("up", [n["ln2"]], lambda a: (mm(a[0], P[b, "up"]),))
            n["act"] = self._add("act", [n["up"]], lambda u: (torch.nn.functional.gelu(u[0]),))
        n["down"] = self._add("down", [n["act"]], lambda g: (mm(g[0], P[b, "down"]),))
        n["out"] = self._add("out", [n["ln2"], n["down"]],
                             lambda a, d: (ops.dropout(d[0], drop(b, 2), residual=a[1]),))

    def _backward(self, b, n, grad, scale):
        P, G, mm, drop = self.params, self.grads, self.mm, self._drop
        xs = [] if n["x"] is None else [n["x"]]

        def linear(name):
            """The gradient past a product, and its weight's."""
            def run(a, d):
                G[b, name] = mm(a[0].t(), d[0])
                return (mm(d[0], P[b, name].t()),)
            return run

        def d_act(u, d):
            with torch.enable_grad():
                v = u[0].detach().requires_grad_()
                return torch.autograd.grad(torch.nn.functional.gelu(v), v, d[0])

        def d_gated(a, d):
            dx, G[b, "gate"], G[b, "up"] = ops.gated_backward(d[0], a[0], P[b, "gate"], P[b, "up"])
            return (dx,)

        def d_ln2(a, past, d):
            dx, dh, G[b, "ln2"], G[b, "ln2_bias"] = ops.layer_norm_backward(
                d[0], a[1], a[2], P[b, "ln2"], dres=past[0], drop=drop(b, 1))
            return dx, dh

        def d_probs(t, p, d):
            g = self._heads(d[0])
            return (mm(g, t[2].transpose(1, 2).contiguous()), mm(p[0].transpose(1, 2).contiguous(), g))

        def d_qkv(t, d, s):
            dq, dk = mm(s[0], t[1]), mm(s[0].transpose(1, 2).contiguous(), t[0])
            return (torch.cat([self._merged(v) for v in (dq, dk, d[1])], 1),)

        def d_ln1(*v):
            x, (a, past, d) = self._x(n, v)
            dx, _, G[b, "ln1"], G[b, "ln1_bias"] = ops.layer_norm_backward(d[0], x, a[1], P[b, "ln1"], dres=past[1])
            return (dx,)

        down = self._add("d_out", [grad], lambda g: (ops.dropout_backward(g[0], drop(b, 2)),))
        act = self._add("d_down", [n["act"], down], linear("down"))
        if self.gated:
            ln2 = self._add("d_gated", [n["ln2"], act], d_gated)
        else:
            up = self._add("d_act", [n["up"], act], d_act)
            ln2 = self._add("d_up", [n["ln2"], up], linear("up"))
        both = self._add("d_ln2", [n["ln2"], grad, ln2], d_ln2)
        ctx = self._add("d_proj", [n["context"], both], linear("proj"))
        probs = self._add("d_context", [n["qkv"], n["probs"], ctx], d_probs)
        scores = self._add("d_probs", [n["scores"], n["probs"], probs], lambda s, p, d: (
            ops.softmax_backward(d[0], s[0], p[1], scale, causal=True, drop=drop(b, 0)),))
        qkv = self._add("d_scores", [n["qkv"], probs, scores], d_qkv)
        ln1 = self._add("d_qkv", [n["ln1"], qkv], linear("qkv"))
        return self._add("d_ln1", xs + [n["ln1"], both, ln1], d_ln1)

    # -- running -----------------------------------------------------------
    def execute(self, plan):
        """Algorithm 1's statements, one after another; returns the gradients by parameter."""
        regs, where = {}, {}
        for op, node, reg, _ in plan:
            if op == ckm.OP_COMPUTE:
                regs[reg] = self.nodes[node].run(*(regs[where[d]] for d in self.nodes[node].deps))
                where[node] = reg
            else:
                regs.pop(reg)
        return self.grads

    def clip(self, max_norm):
        """Bounds the norm of all gradients, which carry the loss scale, in place; returns it, without the scale."""
        norm, _ = ops.clip_gradients([self.grads[k] for k in sorted(self.grads)], max_norm * self.LOSS_SCALE)
        return norm / self.LOSS_SCALE

    def measure(self):
        """(bytes, cost in ns) of every node: one run that keeps everything, then each node timed."""
        values, size, cost = [], [], []
        for node in self.nodes:
            args = [values[d] for d in node.deps]
            values.append(node.run(*args))
            kept = {t.data_ptr(): t.numel() * t.element_size() for t in values[-1]}
            size.append(sum(kept.values()))
            begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            begin.record()
            for _ in range(3):
                node.run(*args)
            end.record()
            end.synchronize()
            cost.append(max(1, int(begin.elapsed_time(end) / 3 * 1e6)))
        return np.array(size, np.int64), np.array(cost, np.int64)


def graph_of(stack, size, cost):
    """The stack's nodes as a graph of the framework; S*: a value's share of the costliest byte's worth, while a
    later node still uses it."""
    ptr, idx = wl.csr_from_deps([n.deps for n in stack.nodes])
    held = sum(t.numel() * t.element_size() for t in stack.params.values())
    g = ckm.Graph(len(stack.nodes), ptr, idx, cost, size,
                  2 * stack.input.numel() * stack.input.element_size(), held)
    n = len(stack.nodes)
    last = np.zeros(n, np.int64)
    for j, node in enumerate(stack.nodes):
        for d in node.deps:
            last[d] = j
    worth = np.argsort(np.argsort(cost / size, kind="stable"), kind="stable")   # rank of cost saved by a byte
    s = np.zeros((n, n))
    for t in range(n):
        s[t, :t] = np.where(last[:t] >= t, (worth[:t] + 1.0) / n, 0.0)
    return g, s


def choose(stack, g, s, size, budget):
    """(statements, memory after each, cost) of the cheapest threshold schedule within the budget."""
    n = len(stack.nodes)
    thresholds = np.arange(n + 1) / n
    r = g.threshold_eval(s, thresholds, budget)
    if r["best_k"] < 0:
        raise SystemExit("no schedule fits %d bytes: the least peak is %d" % (budget, int(r["peak"].min())))
    plan, mem = g.plan(r["best_S"], r["best_R"], early=True)
    return plan, mem, int(r["cost"][r["best_k"]])


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--blocks", type=int, default=4)
    ap.add_argument("--tokens", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=16)
    ap.add_argument("--gated", action="store_true", help="a gated feed-forward")
    ap.add_argument("--vocab", type=int, default=0, help="cross entropy against a vocabulary of this size")
    ap.add_argument("--clip", type=float, default=0.0, help="the gradients' largest norm")
    ap.add_argument("--budgets", type=float, nargs="+", default=[100.0, 60.0, 40.0],
                    help="percent of the memory that keeping everything takes")
    a = ap.parse_args()
    stack = Stack(a.blocks, a.tokens, a.hidden, a.heads, gated=a.gated, vocab=a.vocab)
    size, cost = stack.measure()
    g, s = graph_of(stack, size, cost)
    base = 2 * stack.input.numel() * 2 + 2 * sum(t.numel() * t.element_size() for t in stack.params.values())
    first = None
    for pct in a.budgets:
        budget = int((base + size.sum()) * pct / 100)
        plan, mem, planned = choose(stack, g, s, size, budget)
        stack.execute(plan)                       # once before it is timed
        torch.cuda.synchronize()
        torch.cuda.reset_peak_memory_stats()
        held = torch.cuda.memory_allocated()
        begin = time.perf_counter()
        grads = stack.execute(plan)
        norm = stack.clip(a.clip) if a.clip else None
        torch.cuda.synchronize()
        took = time.perf_counter() - begin
        peak = torch.cuda.max_memory_allocated() - held
        now = [stack.loss.clone()] + [grads[k].clone() for k in sorted(grads)]
        first = first or now
        computed = int((plan[:, 0] == ckm.OP_COMPUTE).sum())
        print("budget %3.0f%%: %d nodes computed (%d in the graph), planned %.1f ms, took %.1f ms; planned peak of the "
              "values %.1f MiB, measured %.1f MiB; loss %.6f, gradients %s the first budget's"
              % (pct, computed, len(stack.nodes), planned / 1e6, took * 1e3, (mem.max() - base) / 2 ** 20, peak / 2 ** 20,
                 float(stack.loss), "equal" if all(torch.equal(p, q) for p, q in zip(now, first)) else "differ from")
              + ("" if norm is None else "; their norm %.4f" % float(norm)))
    g.close()


if __name__ == "__main__":
    main()
