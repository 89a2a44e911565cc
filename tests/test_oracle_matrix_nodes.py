"""The matrix operators without a GPU: the oracle's gradients against differences, every refusal of the C entry
points, and what calls on another stream wait for and hold."""
import ctypes as C

import numpy as np
import pytest

from oracle import nodes
from paper_1910_02653_amd import ckm, ops

RNG = np.random.default_rng(5)


def difference(f, x, dy, h=1e-6):
    """The gradient of sum(dy f(x)) by central differences."""
    g = np.zeros_like(x)
    for k in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[k] += h
        down[k] -= h
        g[k] = ((f(up) - f(down)) * dy).sum() / (2 * h)
    return g


@pytest.mark.parametrize("act", sorted(ops.ACTIVATIONS))
def test_gated_gradients_against_differences(act):
    x, wg, wu = RNG.normal(size=(4, 5)), RNG.normal(size=(5, 6)), RNG.normal(size=(5, 6))
    dh = RNG.normal(size=(4, 6))
    dx, dg, du = nodes.gated_backward(dh, x, wg, wu, act)
    # errors of central differences: h^2 of third derivatives, 1e-16 / h of rounding
    assert np.allclose(dx, difference(lambda v: nodes.gated(v, wg, wu, act), x, dh), rtol=1e-6, atol=1e-7)
    assert np.allclose(dg, difference(lambda v: nodes.gated(x, v, wu, act), wg, dh), rtol=1e-6, atol=1e-7)
    assert np.allclose(du, difference(lambda v: nodes.gated(x, wg, v, act), wu, dh), rtol=1e-6, atol=1e-7)


def test_cross_entropy_gradients_against_differences():
    x, w = RNG.normal(size=(5, 4)), RNG.normal(size=(7, 4))
    targets, dloss = np.array([2, -100, 6, 7, 0]), RNG.normal(size=5)
    loss, lse = nodes.cross_entropy(x, w, targets)
    assert np.all(loss[[1, 3]] == 0) and np.all(loss[[0, 2, 4]] > 0)
    assert np.allclose(np.exp(x @ w.T - lse[:, None]).sum(1), 1.0)
    dx, dw = nodes.cross_entropy_backward(dloss, x, w, targets, lse)
    assert np.allclose(dx, difference(lambda v: nodes.cross_entropy(v, w, targets)[0], x, dloss), rtol=1e-6, atol=1e-7)
    assert np.allclose(dw, difference(lambda v: nodes.cross_entropy(x, v, targets)[0], w, dloss), rtol=1e-6, atol=1e-7)


def test_known_values():
    assert np.allclose(nodes.activation(np.array([0.0, 1.0, -1.0]), "silu")[0], [0.0, 0.7310585786, -0.2689414214])
    assert np.allclose(nodes.activation(np.array([0.0, 1.0, -1.0]), "gelu")[0], [0.0, 0.8413447461, -0.1586552539])
    assert np.array_equal(nodes.activation(np.array([0.0, 2.0, -1.0]), "relu")[1], [0.0, 1.0, 0.0])
    assert nodes.norm([np.array([3.0]), np.array([[4.0]])]) == 5.0 and nodes.norm([]) == 0.0
    loss, lse = nodes.cross_entropy(np.zeros((1, 3)), np.ones((8, 3)), np.array([5]))
    assert np.isclose(loss[0], np.log(8)) and np.isclose(lse[0], np.log(8))


# pointers that are aligned and never followed: every call below is refused before a launch (operands from P on, far
# from one another, outputs from Q on)
P, Q = 1 << 20, 1 << 40


def gated(**kw):
    v = dict(rows=4, hidden=8, inner=8, act=0, d_x=P, ld_x=8, d_gate=2 * P, ld_gate=8, d_up=3 * P, ld_up=8)
    v.update(kw)
    return ops._Gated(*(v[n] for n, _ in ops._Gated._fields_))


BAD_GATED = [
    (dict(rows=-1), ckm.E_INVALID_ARG), (dict(hidden=0), ckm.E_INVALID_ARG), (dict(inner=0), ckm.E_INVALID_ARG),
    (dict(rows=(1 << 24) + 1), ckm.E_UNSUPPORTED), (dict(hidden=(1 << 20) + 1), ckm.E_UNSUPPORTED),
    (dict(inner=(1 << 20) + 1), ckm.E_UNSUPPORTED), (dict(act=3), ckm.E_INVALID_ARG), (dict(act=-1), ckm.E_INVALID_ARG),
    (dict(d_x=None), ckm.E_INVALID_ARG), (dict(d_gate=None), ckm.E_INVALID_ARG), (dict(d_up=None), ckm.E_INVALID_ARG),
    (dict(d_x=P + 1), ckm.E_INVALID_ARG), (dict(ld_x=-1), ckm.E_INVALID_ARG), (dict(ld_up=-8), ckm.E_INVALID_ARG),
    (dict(ld_x=1 << 60), ckm.E_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_GATED)
def test_gated_refusals(kw, status):
    L, c, n = ckm.lib(), gated(**kw), C.c_size_t()
    assert L.ckm_gated_async(ops.F16, C.byref(c), P, 8, P, 1 << 40, None) == status
    assert L.ckm_gated_backward_async(ops.F16, C.byref(c), P, 8, P, 8, P, 8, P, 8, P, 1 << 40, None) == status
    assert L.ckm_gated_workspace_size(ops.F16, C.byref(c), 1, C.byref(n)) == status
    assert L.ckm_last_error()


def test_gated_refuses_outputs_and_work():
    L, c, n = ckm.lib(), gated(), C.c_size_t()
    bad = ckm.E_INVALID_ARG
    assert L.ckm_gated_async(7, C.byref(c), P, 8, None, 0, None) == bad
    assert L.ckm_gated_async(ops.F16, None, P, 8, None, 0, None) == bad
    assert L.ckm_gated_async(ops.F16, C.byref(c), None, 8, None, 0, None) == bad
    assert L.ckm_gated_async(ops.F16, C.byref(c), P + 1, 8, None, 0, None) == bad
    assert L.ckm_gated_async(ops.F16, C.byref(c), P, 7, None, 0, None) == bad           # rows of h overlap
    assert L.ckm_gated_workspace_size(ops.F16, C.byref(c), 0, None) == bad
    assert L.ckm_gated_workspace_size(ops.F16, C.byref(c), 1, C.byref(n)) == ckm.OK and n.value >= 4 * 2 * 8 * 2
    back = lambda **kw: L.ckm_gated_backward_async(ops.F16, C.byref(c), *(   # noqa: E731
        {**dict(dh=4 * P, ldh=8, dx=Q, ldx=8, dg=2 * Q, ldg=8, du=3 * Q, ldu=8, work=P, n=n.value), **kw}).values(), None)
    for kw in (dict(dh=None), dict(ldx=7), dict(ldg=7), dict(ldu=7), dict(dg=None), dict(du=None), dict(dx=P + 1),
               dict(dg=P + 1), dict(work=None), dict(n=n.value - 1), dict(work=P + 8)):
        assert back(**kw) == bad, kw
    # rows that have to be copied need room; no rows need none
    ragged = gated(ld_x=(1 << 22) + 1)   # too far apart to be staged
    m = C.c_size_t()
    assert L.ckm_gated_workspace_size(ops.F16, C.byref(ragged), 0, C.byref(m)) == ckm.OK and m.value >= 4 * 8 * 2
    assert L.ckm_gated_async(ops.F16, C.byref(ragged), Q, 8, P, m.value - 1, None) == bad
    none = gated(rows=0, d_x=None)
    assert L.ckm_gated_workspace_size(ops.F16, C.byref(none), 1, C.byref(m)) == ckm.OK and m.value == 0
    assert L.ckm_gated_async(ops.F16, C.byref(none), None, 8, None, 0, None) == ckm.OK
    # more tiles than a launch counts
    vast = gated(rows=1 << 24, inner=1 << 20, hidden=1, ld_x=1, ld_gate=1 << 20, ld_up=1 << 20)
    assert L.ckm_gated_async(ops.F16, C.byref(vast), 1 << 60, 1 << 20, P, 1 << 62, None) == ckm.E_UNSUPPORTED
    # outputs over operands or one another, by an element; side by side in one matrix's rows they are apart
    for kw in (dict(dx=P), dict(dx=P + 62), dict(dx=P - 62), dict(dx=2 * P), dict(dg=3 * P), dict(du=2 * Q), dict(dg=Q, ldg=8),
               dict(dx=4 * P + 2), dict(du=2 * Q + 126)):
        assert back(**kw) == bad and b"overlaps" in L.ckm_last_error(), kw
    for kw in (dict(du=2 * Q + 16, ldg=16, ldu=16), dict(dx=P + 64)):
        assert back(**kw, n=0) == bad and b"work buffer" in L.ckm_last_error(), kw   # past the check
    for p in (P, 2 * P, 3 * P, 3 * P + 126):
        assert L.ckm_gated_async(ops.F16, C.byref(c), p, 8, P, 1 << 40, None) == bad and b"overlaps" in L.ckm_last_error()


def vocab(**kw):
    v = dict(rows=4, hidden=8, vocab=100, d_x=P, ld_x=8, d_weight=2 * P, ld_weight=8, d_targets=3 * P)
    v.update(kw)
    return ops._Vocab(*(v[n] for n, _ in ops._Vocab._fields_))


BAD_VOCAB = [
    (dict(rows=-1), ckm.E_INVALID_ARG), (dict(hidden=0), ckm.E_INVALID_ARG), (dict(vocab=0), ckm.E_INVALID_ARG),
    (dict(rows=(1 << 24) + 1), ckm.E_UNSUPPORTED), (dict(hidden=(1 << 20) + 1), ckm.E_UNSUPPORTED),
    (dict(vocab=(1 << 24) + 1), ckm.E_UNSUPPORTED), (dict(d_x=None), ckm.E_INVALID_ARG),
    (dict(d_weight=None), ckm.E_INVALID_ARG), (dict(d_targets=None), ckm.E_INVALID_ARG),
    (dict(d_weight=P + 1), ckm.E_INVALID_ARG), (dict(d_targets=P + 4), ckm.E_INVALID_ARG),
    (dict(ld_x=-1), ckm.E_INVALID_ARG), (dict(ld_weight=-8), ckm.E_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_VOCAB)
def test_cross_entropy_refusals(kw, status):
    L, c, n = ckm.lib(), vocab(**kw), C.c_size_t()
    assert L.ckm_cross_entropy_async(ops.F16, C.byref(c), P, P, P, 1 << 40, None) == status
    assert L.ckm_cross_entropy_backward_async(ops.F16, C.byref(c), P, P, P, 8, P, 8, P, 1 << 40, None) == status
    assert L.ckm_cross_entropy_workspace_size(ops.F16, C.byref(c), 1, C.byref(n)) == status


def test_cross_entropy_refuses_outputs_and_work():
    L, c, n, bad = ckm.lib(), vocab(), C.c_size_t(), ckm.E_INVALID_ARG
    assert L.ckm_cross_entropy_workspace_size(ops.BF16, C.byref(c), 0, C.byref(n)) == ckm.OK and n.value > 0
    assert L.ckm_cross_entropy_async(7, C.byref(c), Q, 2 * Q, P, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, None, Q, 2 * Q, P, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), Q + 2, 2 * Q, P, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), Q, 2 * Q + 2, P, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), Q, 2 * Q, None, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), Q, 2 * Q, P, n.value - 1, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), Q, 2 * Q, P + 8, n.value, None) == bad
    assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), None, None, None, 0, None) == ckm.OK   # nothing asked
    assert L.ckm_cross_entropy_workspace_size(ops.BF16, C.byref(c), 0, None) == bad
    assert L.ckm_cross_entropy_workspace_size(ops.BF16, C.byref(c), 1, C.byref(n)) == ckm.OK and n.value >= 4 * 100 * 2
    back = lambda **kw: L.ckm_cross_entropy_backward_async(ops.BF16, C.byref(c), *(   # noqa: E731
        {**dict(dl=4 * P, lse=5 * P, dx=Q, ldx=8, dw=2 * Q, ldw=8, work=P, n=n.value), **kw}).values(), None)
    for kw in (dict(dl=None), dict(dl=P + 2), dict(lse=None), dict(lse=P + 2), dict(ldx=7), dict(ldw=7), dict(dx=P + 1),
               dict(dw=P + 1), dict(work=None), dict(n=n.value - 1), dict(work=P + 8)):
        assert back(**kw) == bad, kw
    assert back(dx=None, dw=None) == ckm.OK
    for kw in (dict(dx=P), dict(dw=2 * P), dict(dx=3 * P), dict(dw=4 * P), dict(dx=5 * P), dict(dx=2 * Q), dict(dw=P + 62)):
        assert back(**kw) == bad and b"overlaps" in L.ckm_last_error(), kw
    assert L.ckm_cross_entropy_workspace_size(ops.BF16, C.byref(c), 0, C.byref(n)) == ckm.OK
    for loss, lse in ((P, Q), (Q, 2 * P), (Q, Q), (Q, Q + 12), (3 * P, Q)):
        assert L.ckm_cross_entropy_async(ops.BF16, C.byref(c), loss, lse, P, n.value, None) == bad
        assert b"overlaps" in L.ckm_last_error()
    # the work buffer holds a piece of the vocabulary at most, not its logits
    big = vocab(rows=1 << 16, hidden=64, vocab=1 << 18, ld_x=64, ld_weight=64)
    assert L.ckm_cross_entropy_workspace_size(ops.BF16, C.byref(big), 1, C.byref(n)) == ckm.OK
    assert n.value < (1 << 16) * (1 << 18) * 2 // 16


@pytest.mark.parametrize("dtype", [ops.F32, ops.F16, ops.BF16])
@pytest.mark.parametrize("rows", [1024, 8192, 16384, 65536, 1 << 20])
def test_cross_entropy_gradient_work_at_many_rows(dtype, rows):
    """x's copy, dx's sums, and d: 128 MB (its rows padded), or 8192 columns of it; each part is rounded up to 256 bytes, and
    a row of d has up to 384 more."""
    elt, hidden, words, L, n = 4 if dtype == ops.F32 else 2, 4096, 131072, ckm.lib(), C.c_size_t()
    c = vocab(rows=rows, hidden=hidden, vocab=words, ld_x=hidden, ld_weight=hidden, d_x=1 << 44, d_weight=1 << 45)
    assert L.ckm_cross_entropy_workspace_size(dtype, C.byref(c), 1, C.byref(n)) == ckm.OK
    d = max(128 << 20, rows * 8192 * elt)
    most = rows * hidden * elt + max(rows * hidden * 4, 512 << 20 if rows <= 8192 else 0) + d + rows * 384
    assert rows * hidden * (elt + 4) + rows * 8192 * elt // 2 <= n.value <= most + (1 << 20), (n.value >> 20, most >> 20)


def test_no_rows_refuse_outputs_over_the_weights():
    """Zero weight gradients are written without rows too, and so not over the weights or one another."""
    L, bad = ckm.lib(), ckm.E_INVALID_ARG
    c = gated(rows=0, d_x=None)
    for dg, du in ((2 * P, Q), (Q, 3 * P), (Q, 2 * P + 126), (Q, Q), (Q, Q + 64)):
        assert L.ckm_gated_backward_async(ops.F16, C.byref(c), None, 8, None, 8, dg, 8, du, 8, None, 0, None) == bad
        assert b"overlaps" in L.ckm_last_error(), (dg, du)
    v = vocab(rows=0, d_x=None, d_targets=None)
    for dw in (2 * P, 2 * P + 1598, 2 * P - 16):
        assert L.ckm_cross_entropy_backward_async(ops.F16, C.byref(v), None, None, None, 8, dw, 8, None, 0, None) == bad
        assert b"overlaps" in L.ckm_last_error(), dw


def tensors(*rows):
    return (C.c_int64 * (4 * len(rows)))(*(v for r in rows for v in r))


@pytest.mark.parametrize("rows,status", [
    ([(P, P, -1, 0)], ckm.E_INVALID_ARG), ([(P, P, 4, 3)], ckm.E_INVALID_ARG), ([(P, P, 4, -1)], ckm.E_INVALID_ARG),
    ([(P, P, 4, 1 << 32)], ckm.E_INVALID_ARG),
    ([(0, P, 4, 0)], ckm.E_INVALID_ARG), ([(P + 2, P, 4, 0)], ckm.E_INVALID_ARG), ([(P, P, 1 << 62, 0)], ckm.E_UNSUPPORTED),
    ([(P, P, 1 << 45, 0)], ckm.E_UNSUPPORTED), ([(P, P, 1 << 43, 0)] * 3, ckm.E_UNSUPPORTED),
])
def test_norm_refusals(rows, status):
    L, t = ckm.lib(), tensors(*rows)
    assert L.ckm_norm_async(len(rows), t, P, P, 1 << 40, None) == status
    assert L.ckm_clip_async(len(rows), t, 1.0, 0.0, P, P, 1 << 40, None) == status


@pytest.mark.parametrize("rows", [
    [(P, 0, 4, 0)], [(P, P + 2, 4, 0)],
    [(P, P, 4, 0), (P, P, 4, 0)],                              # twice
    [(P, 2 * P, 4, 0), (P + 64, 2 * P, 4, 0)],                 # two into one
    [(P, 2 * P, 4, 0), (P + 64, 2 * P + 12, 4, 0)],
    [(P, P + 4, 4, 0)],                                        # over its own input, not in its place
    [(P, P - 4, 4, 0)],
    [(P, P + 64, 4, 0), (P + 64, 2 * P, 4, 0)],                # over another's input
    [(P, 2 * P, 1000, 0), (P + 64, P + 128, 4, 0)],            # inside another's input
    [(P, 2 * P, 4, 0), (P + 16, 2 * P + 8, 4, 1)],
    [(P + 4 * k, P + 4 * k, 1, 0) for k in range(200)] + [(3 * P, P + 400, 1, 0)],
])
def test_clip_refuses_outputs_over_one_another(rows):
    assert ckm.lib().ckm_clip_async(len(rows), tensors(*rows), 1.0, 0.0, P, P, 1 << 40, None) == ckm.E_INVALID_ARG


def test_norm_may_not_lie_in_a_tensor():
    L, bad = ckm.lib(), ckm.E_INVALID_ARG
    t = tensors((P, 2 * P, 4, 0), (3 * P, 3 * P, 5, 2), (4 * P, 5 * P, 0, 0))
    for at in (P, P + 12, 3 * P, 3 * P + 8):
        assert L.ckm_norm_async(3, t, at, None, 0, None) == bad and b"norm overlaps" in L.ckm_last_error()
    for at in (P, P + 12, 2 * P, 2 * P + 12, 3 * P + 8):
        assert L.ckm_clip_async(3, t, 1.0, 0.0, at, None, 0, None) == bad and b"norm overlaps" in L.ckm_last_error()
    for at in (P + 16, P - 4, 3 * P + 12, 4 * P, 5 * P):   # beside them
        assert L.ckm_norm_async(3, t, at, None, 0, None) == bad and b"work buffer" in L.ckm_last_error()
        assert L.ckm_clip_async(3, t, 1.0, 0.0, at, None, 0, None) == bad and b"work buffer" in L.ckm_last_error()
    assert L.ckm_norm_async(3, t, 2 * P, None, 0, None) == bad and b"work buffer" in L.ckm_last_error()   # writes no output


def test_norm_refuses_the_rest():
    L, t, n, bad = ckm.lib(), tensors((P, P, 4, 0)), C.c_size_t(), ckm.E_INVALID_ARG
    assert L.ckm_norm_workspace_size(1, C.byref(n)) == ckm.OK and n.value > 0
    assert L.ckm_norm_workspace_size(-1, C.byref(n)) == bad and L.ckm_norm_workspace_size(1, None) == bad
    assert L.ckm_norm_workspace_size((1 << 20) + 1, C.byref(n)) == ckm.E_UNSUPPORTED
    assert L.ckm_norm_workspace_size(1, C.byref(n)) == ckm.OK
    assert L.ckm_norm_async((1 << 20) + 1, t, P, P, 1 << 40, None) == ckm.E_UNSUPPORTED
    for count, table, norm, work, size in ((-1, t, P, P, n.value), (1, None, P, P, n.value), (1, t, None, P, n.value),
                                           (1, t, P + 2, P, n.value), (1, t, P, None, n.value), (1, t, P, P, n.value - 1),
                                           (1, t, P, P + 4, n.value)):
        assert L.ckm_norm_async(count, table, norm, work, size, None) == bad
        assert L.ckm_clip_async(count, table, 1.0, 0.0, norm, work, size, None) == bad
    for most, eps in ((-1.0, 0.0), (float("nan"), 0.0), (1.0, -1.0), (1.0, float("nan")), (1.0, float("inf"))):
        assert L.ckm_clip_async(1, t, most, eps, P, P, n.value, None) == bad


def test_binding_refuses_host_tensors():
    import torch
    x, w, t = torch.zeros(4, 8), torch.zeros(8, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: ops.gated(x, w, w), lambda: ops.gated_backward(x, x, w, w), lambda: ops.cross_entropy(x, w, t),
                 lambda: ops.cross_entropy_backward(x[:, 0], x, w, t, x[:, 0]), lambda: ops.gated_workspace(x, w, w),
                 lambda: ops.cross_entropy_workspace(x, w, t)):
        with pytest.raises(ValueError):
            call()


def test_dense_tensors():
    import torch
    t = torch.zeros(4, 6, 8)
    for good in (t, t.transpose(0, 1), t.permute(2, 0, 1), t[1:3], t[2], t[:0], t[:, :0, :3], t[0, 0, 0], t.expand(1, 4, 6, 8)):
        assert ops._dense(good)
    for bad in (t[:, :3], t[:, :, 1:], t[::2], t[:1, :1, :1].expand(4, 6, 8), t[0, :, 0]):
        assert not ops._dense(bad)


def test_calls_on_another_stream_wait_for_the_current_one_and_hold_their_tensors(monkeypatch):
    """What happens to the streams and tensors before the calls' checks refuse the host tensors."""
    import contextlib

    import torch
    events, current = [], []

    class Stream:
        device = torch.device("cpu")

        def wait_stream(self, other):
            events.append(("wait", self, other))

    class Held(torch.Tensor):
        def record_stream(self, stream):
            events.append(("hold", id(self), stream))

    @contextlib.contextmanager
    def use(stream):
        current.append(stream)
        try:
            yield
        finally:
            current.pop()

    here, there = Stream(), Stream()
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current[-1] if current else here)
    monkeypatch.setattr(torch.cuda, "stream", use)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(ops, "_current_device", lambda: 0)
    t = [torch.zeros(4, 8).as_subclass(Held) for _ in range(7)]
    calls = [
        (lambda q: ops.gated(t[0], t[1], t[2], out=t[3], work=t[4], stream=q), range(5)),
        (lambda q: ops.gated_backward(t[0], t[1], t[2], t[3], work=t[4], stream=q), range(5)),
        (lambda q: ops.cross_entropy(t[0], t[1], t[2], work=t[3], stream=q), range(4)),
        (lambda q: ops.cross_entropy_backward(t[0], t[1], t[2], t[3], t[4], work=t[5], stream=q), range(6)),
        (lambda q: ops.gradient_norm([t[0], t[1]], work=t[2], stream=q), range(3)),
        (lambda q: ops.gradient_norm((v for v in t[:2]), work=t[2], stream=q), range(3)),
        (lambda q: ops.clip_gradients([t[0], t[1]], 1.0, out=[t[2], t[3]], work=t[4], stream=q), range(5)),
        (lambda q: ops.clip_gradients((v for v in t[:2]), 1.0, work=t[4], stream=q), (0, 1, 4)),
    ]
    for call, held in calls:
        for stream in (there, here, None):
            events.clear()
            with pytest.raises(ValueError):
                call(stream)
            if stream is not there:
                assert not events
                continue
            assert [e for e in events if e[0] == "wait"] == [("wait", there, here)]
            assert sorted(e[1] for e in events if e[0] == "hold") == sorted(id(t[k]) for k in held)
            assert all(e[2] is there for e in events if e[0] == "hold")
