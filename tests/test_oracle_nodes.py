"""The 64-bit oracle of the training-node operators (oracle/nodes.py), and what
the entry points refuse before they touch the device. CPU only.

The draws are compared with the rounding oracle's own Philox, gradients with
central differences of the forward formulas.
"""
import ctypes as C

import numpy as np
import pytest

from oracle import nodes, ref
from paper_1910_02653_amd import ckm, ops


@pytest.mark.parametrize("rows,cols,seed,site", [(3, 21, 0x0123456789ABCDEF, (7 << 32) | 9), (1, 8, 5, 0), (4, 1, 1, 2)])
def test_draws_are_the_rounding_generators(rows, cols, seed, site):
    u = nodes.draws(rows, cols, seed, site)
    for r in range(rows):
        for c in range(cols):
            x = ref.philox4x32_10((seed & 0xFFFFFFFF, seed >> 32), (c // 8, r, site & 0xFFFFFFFF, site >> 32))
            assert u[r, c] == (int(x[c % 8 // 2]) >> (16 * (c % 2))) & 0xFFFF


def test_keep_probability():
    """The share of kept elements lies within 5 sigma of keep / 65536."""
    keep, n = 58982, 400 * 512
    f = nodes.factors(400, 512, 3, 4, keep)
    p = keep / 65536
    assert abs((f > 0).sum() - n * p) < 5 * np.sqrt(n * p * (1 - p))
    assert np.all(f[f > 0] == 65536 / keep)


def differences(fn, x, dy, step=1e-5):
    """Gradient of sum(dy * fn(x)) by central differences, element by element."""
    out = np.zeros_like(x)
    flat, o = x.reshape(-1), out.reshape(-1)
    for i in range(flat.size):
        keep = flat[i]
        flat[i] = keep + step
        hi = (dy * fn(x)).sum()
        flat[i] = keep - step
        lo = (dy * fn(x)).sum()
        flat[i] = keep
        o[i] = (hi - lo) / (2 * step)
    return out


def test_dropout_gradient_is_the_dropout_of_the_gradient():
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((2, 3, 11))
    f = nodes.factors(3, 11, 8, 1, 40000)
    assert np.allclose(differences(lambda v: nodes.dropout(v, f), x, dy), nodes.dropout(dy, f), atol=1e-8)


def test_layer_norm_gradient_by_differences():
    rng = np.random.default_rng(2)
    h, dy = rng.standard_normal((2, 4, 9)) + 0.5
    w, b = rng.standard_normal((2, 9))
    eps = 1e-3
    _, mean, rstd = nodes.layer_norm(h, w, b, eps)
    dh, dw, db = nodes.layer_norm_backward(dy, h, mean, rstd, w)
    # truncation error of the differences: step^2 times third derivatives, about 1e-9
    assert np.allclose(differences(lambda v: nodes.layer_norm(v, w, b, eps)[0], h, dy), dh, atol=1e-7)
    assert np.allclose(differences(lambda v: nodes.layer_norm(h, v, b, eps)[0], w, dy), dw, atol=1e-7)
    assert np.allclose(differences(lambda v: nodes.layer_norm(h, w, v, eps)[0], b, dy), db, atol=1e-7)


@pytest.mark.parametrize("causal", [False, True])
def test_softmax_gradient_by_differences(causal):
    rng = np.random.default_rng(3)
    shape = (2, 2, 4, 5)
    x, dy = rng.standard_normal((2,) + shape)
    mask = rng.random((1, 2, 4, 5)) < 0.7
    mask[0, 0, 1] = False
    seen = nodes.visible(shape, causal, [5, 2], mask)
    f = nodes.factors(16, 5, 6, 2, 50000).reshape(shape)
    scale = 0.7

    def forward(v):
        return nodes.softmax(nodes.logits(v, scale, seen, mask))[0] * f

    p = nodes.softmax(nodes.logits(x, scale, seen, mask))[0]
    dx = nodes.softmax_backward(nodes.dropout(dy, f), p, scale)
    assert np.allclose(differences(forward, x, dy), dx, atol=1e-8)
    assert np.all(dx[~seen] == 0) and np.all(p[0, 0, 1] == 0)


# ---------------------------------------------------------------------------
# refusals (no device is touched)
# ---------------------------------------------------------------------------

P = 4096   # a pointer that is never followed


def call_dropout(t=ops.F16, rows=2, cols=8, x=P, ldx=8, res=None, ldr=0, keep=100, drop=True, y=P, ldy=8, d_site=None):
    d = ops._Drop(1, 2, d_site, keep)
    return ckm.lib().ckm_dropout_async(t, rows, cols, x, ldx, res, ldr, C.byref(d) if drop else None, y, ldy, None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=3), ckm.E_INVALID_ARG), (dict(t=-1), ckm.E_INVALID_ARG), (dict(rows=-1), ckm.E_INVALID_ARG),
    (dict(cols=-1), ckm.E_INVALID_ARG), (dict(rows=1 << 31), ckm.E_UNSUPPORTED),
    (dict(cols=(1 << 30) + 1), ckm.E_UNSUPPORTED), (dict(x=None), ckm.E_INVALID_ARG),
    (dict(y=None), ckm.E_INVALID_ARG), (dict(drop=False), ckm.E_INVALID_ARG), (dict(keep=65537), ckm.E_INVALID_ARG),
    (dict(x=P + 1), ckm.E_INVALID_ARG), (dict(ldy=7), ckm.E_INVALID_ARG), (dict(ldx=-8), ckm.E_INVALID_ARG),
    (dict(res=P + 1), ckm.E_INVALID_ARG), (dict(ldx=1 << 62), ckm.E_INVALID_ARG), (dict(d_site=P + 4), ckm.E_INVALID_ARG),
    (dict(rows=0, x=None, y=None), ckm.OK), (dict(cols=0, x=None, y=None), ckm.OK),
])
def test_dropout_refusals(kw, status):
    assert call_dropout(**kw) == status, ckm.last_error()


def call_norm(t=ops.F16, wt=ops.F16, rows=2, cols=8, x=P, ldx=8, res=None, drop=False, w=P, b=P, eps=1e-5, h=None, y=P,
              ldy=8, stats=P):
    d = ops._Drop(1, 2, None, 100)
    return ckm.lib().ckm_layer_norm_async(t, wt, rows, cols, x, ldx, res, 8, C.byref(d) if drop else None, w, b, eps, h,
                                          8, y, ldy, stats, None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=9), ckm.E_INVALID_ARG), (dict(wt=ops.BF16), ckm.E_INVALID_ARG), (dict(t=ops.F32, wt=ops.F16), ckm.E_INVALID_ARG),
    (dict(cols=0), ckm.E_INVALID_ARG), (dict(rows=-2), ckm.E_INVALID_ARG), (dict(cols=32769), ckm.E_UNSUPPORTED),
    (dict(rows=1 << 31), ckm.E_UNSUPPORTED), (dict(x=None), ckm.E_INVALID_ARG), (dict(y=None), ckm.E_INVALID_ARG),
    (dict(eps=-1e-5), ckm.E_INVALID_ARG), (dict(eps=float("nan")), ckm.E_INVALID_ARG),
    (dict(eps=float("inf")), ckm.E_INVALID_ARG), (dict(h=P), ckm.E_INVALID_ARG), (dict(w=P + 1), ckm.E_INVALID_ARG),
    (dict(b=P + 1), ckm.E_INVALID_ARG), (dict(wt=ops.F32, w=P + 2), ckm.E_INVALID_ARG), (dict(stats=P + 2), ckm.E_INVALID_ARG),
    (dict(ldy=4), ckm.E_INVALID_ARG), (dict(rows=0, x=None, y=None), ckm.OK),
])
def test_layer_norm_refusals(kw, status):
    assert call_norm(**kw) == status, ckm.last_error()


def call_norm_backward(t=ops.F16, wt=ops.F32, rows=2000, cols=64, dy=P, h=P, stats=P, w=P, dres=None, drop=False, dh=P,
                       dx=None, dw=P, db=P, work=P, work_bytes=1 << 40, lddh=64):
    d = ops._Drop(1, 2, None, 100)
    return ckm.lib().ckm_layer_norm_backward_async(t, wt, rows, cols, dy, 64, h, 64, stats, w, dres, 64,
                                                   C.byref(d) if drop else None, dh, lddh, dx, 64, dw, db, work,
                                                   work_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(t=5), ckm.E_INVALID_ARG), (dict(wt=ops.BF16), ckm.E_INVALID_ARG), (dict(cols=0), ckm.E_INVALID_ARG),
    (dict(cols=40000), ckm.E_UNSUPPORTED), (dict(dy=None), ckm.E_INVALID_ARG), (dict(h=None), ckm.E_INVALID_ARG),
    (dict(stats=None), ckm.E_INVALID_ARG), (dict(dx=P), ckm.E_INVALID_ARG), (dict(work=None), ckm.E_INVALID_ARG),
    (dict(work_bytes=16), ckm.E_INVALID_ARG), (dict(work=P + 8), ckm.E_INVALID_ARG), (dict(lddh=63), ckm.E_INVALID_ARG),
    (dict(dw=P + 2), ckm.E_INVALID_ARG), (dict(db=P + 1), ckm.E_INVALID_ARG), (dict(dres=P + 1), ckm.E_INVALID_ARG),
])
def test_layer_norm_backward_refusals(kw, status):
    assert call_norm_backward(**kw) == status, ckm.last_error()


def call_softmax(back=False, t=ops.F16, shape=(2, 3, 4, 8), scale=1.0, flags=0, lengths=None, mask=None, kind=0,
                 mask_stride=(0, 0, 0), x=P, xs=(96, 32, 8), y=P, ys=(96, 32, 8), stats=P, work=P, work_bytes=1 << 40,
                 keep=None, scores=True, dy=P):
    c = ops._Scores(*shape)
    c.scale, c.flags, c.d_lengths, c.d_mask, c.mask_kind = scale, flags, lengths, mask, kind
    c.mask_stride = ops._Stride(*mask_stride)
    d = None if keep is None else C.byref(ops._Drop(1, 2, None, keep))
    cp = C.byref(c) if scores else None
    xs, ys = (None if s is None else ops._Stride(*s) for s in (xs, ys))
    if back:
        return ckm.lib().ckm_softmax_backward_async(t, cp, dy, xs, x, xs, stats, d, y, ys, work, work_bytes, None)
    return ckm.lib().ckm_softmax_async(t, cp, x, xs, d, y, ys, stats, work, work_bytes, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("kw,status", [
    (dict(t=7), ckm.E_INVALID_ARG), (dict(scores=False), ckm.E_INVALID_ARG), (dict(shape=(2, -1, 4, 8)), ckm.E_INVALID_ARG),
    (dict(shape=(1 << 20, 1 << 20, 1, 8)), ckm.E_UNSUPPORTED), (dict(shape=(1, 1, 1, (1 << 30) + 1)), ckm.E_UNSUPPORTED),
    (dict(scale=float("nan")), ckm.E_INVALID_ARG), (dict(scale=float("inf")), ckm.E_INVALID_ARG),
    (dict(flags=2), ckm.E_INVALID_ARG), (dict(kind=3), ckm.E_INVALID_ARG), (dict(kind=1), ckm.E_INVALID_ARG),
    (dict(kind=2, mask=P + 1), ckm.E_INVALID_ARG), (dict(kind=1, mask=P, mask_stride=(-1, 0, 0)), ckm.E_INVALID_ARG),
    (dict(x=None), ckm.E_INVALID_ARG), (dict(y=None), ckm.E_INVALID_ARG), (dict(x=P + 1), ckm.E_INVALID_ARG),
    (dict(xs=None), ckm.E_INVALID_ARG), (dict(ys=None), ckm.E_INVALID_ARG), (dict(xs=(96, -32, 8)), ckm.E_INVALID_ARG),
    (dict(ys=(96, 32, 7)), ckm.E_INVALID_ARG), (dict(ys=(96, 16, 8)), ckm.E_INVALID_ARG), (dict(ys=(0, 32, 8)), ckm.E_INVALID_ARG),
    (dict(xs=(1 << 62, 32, 8)), ckm.E_INVALID_ARG), (dict(stats=P + 1), ckm.E_INVALID_ARG), (dict(lengths=P + 2), ckm.E_INVALID_ARG),
    (dict(keep=70000), ckm.E_INVALID_ARG), (dict(shape=(1, 1, 1, 100000), work=None), ckm.E_INVALID_ARG),
    (dict(shape=(1, 1, 1, 100000), work_bytes=8), ckm.E_INVALID_ARG), (dict(shape=(1, 1, 1, 100000), work=P + 4), ckm.E_INVALID_ARG),
    (dict(shape=(0, 3, 4, 8), x=None, y=None), ckm.OK),
])
def test_softmax_refusals(back, kw, status):
    assert call_softmax(back=back, **kw) == status, ckm.last_error()


def test_softmax_backward_needs_statistics_and_gradient():
    assert call_softmax(back=True, stats=None) == ckm.E_INVALID_ARG
    assert call_softmax(back=True, dy=None) == ckm.E_INVALID_ARG


def test_workspace_sizes():
    assert ops.layer_norm_workspace(0, 64) == 0 and ops.layer_norm_workspace(1, 4096) == 0
    assert ops.layer_norm_workspace(5000, 1000) >= 2 * 1000 * 4
    with pytest.raises(ckm.CkmError):
        ops.layer_norm_workspace(10, 0)
    L, n = ckm.lib(), C.c_size_t()
    assert L.ckm_softmax_workspace_size(None, C.byref(n)) == ckm.E_INVALID_ARG
    assert L.ckm_softmax_workspace_size(C.byref(ops._Scores(1, 1, 1, 8)), None) == ckm.E_INVALID_ARG
    assert L.ckm_layer_norm_workspace_size(1, 1, None) == ckm.E_INVALID_ARG
    assert L.ckm_softmax_workspace_size(C.byref(ops._Scores(1, 1, 1, 1 << 20)), C.byref(n)) == ckm.OK and n.value > 0


def test_binding_refuses_host_tensors_and_bad_dropouts():
    import torch
    x = torch.zeros(4, 8)
    d = ops.Dropout(0.1, 1)
    for call in (lambda: ops.dropout(x, d), lambda: ops.layer_norm(x), lambda: ops.softmax(x),
                 lambda: ops.layer_norm_backward(x, x, x), lambda: ops.softmax_backward(x, x, x)):
        with pytest.raises(ValueError):
            call()
    for bad in (dict(p=-0.1), dict(p=1.5), dict(p=float("nan")), dict(p=0.1, seed=-1), dict(p=0.1, seed=1 << 64),
                dict(p=0.1, site=1 << 64), dict(p=0.1, d_site=torch.zeros(1, dtype=torch.int64))):
        with pytest.raises(ValueError):
            ops.Dropout(**{"seed": 1, **bad})
    assert ops.Dropout(0.0, 1).keep == 65536 and ops.Dropout(1.0, 1).keep == 0 and ops.Dropout(0.1, 1).keep == 58982


@pytest.mark.parametrize("within,captured,waits", [(False, False, True), (True, False, True), (True, True, True),
                                                   (False, True, False)])
def test_calls_on_another_stream_wait_for_the_current_one_and_hold_their_tensors(monkeypatch, within, captured, waits):
    """Every operator with stream=: what happens to the streams and tensors before the call's checks refuse the host
    tensors. within, captured: whether the current stream and the other one are being captured."""
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
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: captured if current else within)
    t = [torch.zeros(4, 8).as_subclass(Held) for _ in range(7)]
    drop = ops.Dropout(0.1, 1)
    drop._d_site = t[6]   # past the check that it is on a device
    calls = [
        (lambda q: ops.dropout(t[0], drop, residual=t[1], out=t[2], stream=q), (0, 1, 2, 6)),
        (lambda q: ops.dropout_backward(t[0], drop, out=t[1], stream=q), (0, 1, 6)),
        (lambda q: ops.layer_norm(t[0], t[1], t[2], residual=t[3], drop=drop, out=t[4], stream=q), (0, 1, 2, 3, 4, 6)),
        (lambda q: ops.layer_norm_backward(t[0], t[1], t[2], t[3], dres=t[4], out=t[5], work=t[6], stream=q), range(7)),
        (lambda q: ops.softmax(t[0], lengths=t[1], mask=t[2], drop=drop, out=t[3], work=t[4], stream=q),
         (0, 1, 2, 3, 4, 6)),
        (lambda q: ops.softmax_backward(t[0], t[1], t[2], lengths=t[3], mask=t[4], out=t[5], work=t[6], stream=q),
         range(7)),
    ]
    for call, held in calls:
        for stream in (there, here, None):
            events.clear()
            with pytest.raises(ValueError):
                call(stream)
            if stream is not there:
                assert not events
                continue
            assert [e for e in events if e[0] == "wait"] == ([("wait", there, here)] if waits else [])
            assert sorted(e[1] for e in events if e[0] == "hold") == sorted(id(t[k]) for k in held)
            assert all(e[2] is there for e in events if e[0] == "hold")


def test_a_dropout_goes_by_what_it_is_assigned():
    d = ops.Dropout(0.25, 3, 4)
    d.p, d.seed, d.site = 0.5, (1 << 64) - 1, 5
    d.site += 1
    assert (d.p, d.keep, d.seed, d.site, d.d_site) == (0.5, 32768, (1 << 64) - 1, 6, None)
    assert (d._c.keep, d._c.seed, d._c.site, d._c.d_site) == (32768, (1 << 64) - 1, 6, None)
    for name, value in (("p", 1.5), ("p", float("nan")), ("seed", -1), ("site", 1 << 64), ("d_site", 3)):
        with pytest.raises(ValueError):
            setattr(d, name, value)
    with pytest.raises(AttributeError):
        d.keep = 1
    assert (d._c.keep, d._c.seed, d._c.site, d._c.d_site) == (32768, (1 << 64) - 1, 6, None)


def test_wide_rows_of_one_block_are_few():
    """Rows of two groups a thread take a block's whole turn twice over: no more than two of them share one."""
    for cols in (8193, 16384):
        assert ops.layer_norm_workspace(2, cols) == 0
        assert ops.layer_norm_workspace(3, cols) >= 3 * 2 * cols * 4 and ops.layer_norm_workspace(4, cols) >= 4 * 2 * cols * 4
    assert ops.layer_norm_workspace(4, 8192) == 0


def test_a_copied_dropout_is_its_own():
    import copy
    import pickle
    d = ops.Dropout(0.25, 3, 4)
    for other in (copy.copy(d), copy.deepcopy(d), pickle.loads(pickle.dumps(d))):
        assert (other.p, other.seed, other.site, other.d_site, other.keep) == (0.25, 3, 4, None, d.keep)
        other.site = 9
        assert d.site == 4 and other.site == 9
