"""Gated feed-forward, vocabulary cross entropy, gradient norm and clipping against their definitions in 64 bits.

Tolerances are error bounds, stated before any run, with u = 2^-24 (binary32)
and v the result type's half unit in the last place:
  * a product's sum of N terms, in whatever order and width it is added: at
    most (N + 8) u sum |terms| (each of N additions rounds once);
  * an activation and its derivative: 16 u of the value and of the argument (a
    binary32 exponential, reciprocal or error function and a few products);
    both are Lipschitz with a constant below 1.2 in the argument, the derivative
    of relu apart, which is unknown within the argument's error of 0;
  * exp(l - lse): relative 8 u + the error of l and u |l - lse|;
  * each rounding to the result type: v |y|, and half the smallest subnormal.
"""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import nodes
from paper_1910_02653_amd import ckm, ops

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 2.0 ** -126, "f16": 2.0 ** -25, "bf16": 2.0 ** -126}
U = 2.0 ** -24
ACT = 16 * U
NAN = float("nan")


def log(msg):
    print(msg, flush=True)


def randn(shape, dtype, seed, gain=1.0, offset=0, pad=0):
    """A device tensor whose rows start `offset` elements into an allocation and lie `pad` elements apart, NaN between."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = int(np.prod(shape[:-1])), shape[-1]
    flat = torch.full((offset + rows * (cols + pad) + 16,), NAN, dtype=TYPES[dtype], device="cuda")
    view = flat[offset:offset + rows * (cols + pad)].view(tuple(shape[:-1]) + (cols + pad,))[..., :cols]
    view.copy_(torch.randn(shape, generator=gen, device="cuda") * gain)
    return view


def host(t):
    return t.double().cpu().numpy()


def check(got, want, tol, dtype, what):
    """|got - want| <= tol + the one rounding to the result's type."""
    got = host(got)
    bound = tol + HALF_ULP[dtype] * (np.abs(want) + tol) + TINY[dtype]
    assert np.all(np.isfinite(got)), what
    worst = np.max(np.abs(got - want) / bound) if got.size else 0.0
    assert worst <= 1.0, "%s: error %.3g times its bound" % (what, worst)


def product(a, b, da=0.0, db=0.0):
    """(a @ b, the bound of its error) with errors da, db of the factors."""
    x, y = np.abs(a), np.abs(b)
    return a @ b, (a.shape[1] + 8) * U * ((x + da) @ (y + db)) + (x + da) @ (np.zeros_like(y) + db) + (np.zeros_like(x) + da) @ y


# ---------------------------------------------------------------------------
# gated feed-forward
# ---------------------------------------------------------------------------

def gated_bounds(x, wg, wu, act):
    g, eg = product(x, wg)
    u, eu = product(x, wu)
    a, da = nodes.activation(g, act)
    ea = 1.2 * eg + ACT * (np.abs(a) + np.abs(g))
    eda = 1.2 * eg + ACT * (1.0 + np.abs(g))
    if act == "relu":
        eda = np.where(np.abs(g) <= eg, 1.0, 0.0)
    return g, u, a, da, eu, ea, eda


def check_gated(dtype, rows, hidden, inner, act, offset=0, pad=0, seed=1):
    x = randn((rows, hidden), dtype, seed, offset=offset, pad=pad)
    wg, wu = (randn((hidden, inner), dtype, seed + k, gain=hidden ** -0.5, offset=offset, pad=pad + k * (pad > 0)) for k in (1, 2))
    dh = randn((rows, inner), dtype, seed + 3, offset=offset, pad=pad)
    h = ops.gated(x, wg, wu, act=act)
    X, G, W, D = (host(t) for t in (x, wg, wu, dh))
    g, u, a, da, eu, ea, eda = gated_bounds(X, G, W, act)
    eh = ea * (np.abs(u) + eu) + np.abs(a) * eu + U * np.abs(a * u)
    check(h, a * u, eh, dtype, "h")
    dx, dg, du = ops.gated_backward(dh, x, wg, wu, act=act)
    v = HALF_ULP[dtype]
    pg, pu = D * u * da, D * a
    epg = np.abs(D) * (eda * (np.abs(u) + eu) + np.abs(da) * eu) + 3 * U * np.abs(pg)
    epu = np.abs(D) * ea + 2 * U * np.abs(pu)
    epg, epu = epg + v * (np.abs(pg) + epg) + TINY[dtype], epu + v * (np.abs(pu) + epu) + TINY[dtype]   # rounded once
    both, eboth = product(np.concatenate([pg, pu], 1), np.concatenate([G, W], 1).T, da=np.concatenate([epg, epu], 1))
    check(dx, both, eboth, dtype, "dx")
    for got, p, e, what in ((dg, pg, epg, "dw_gate"), (du, pu, epu, "dw_up")):
        want, bound = product(X.T, p, db=e)
        check(got, want, bound, dtype, what)
    return h, dx, dg, du


GATED_SIZES = [(1, 1, 1), (1, 64, 64), (2, 8, 3), (3, 7, 5), (16, 128, 256), (17, 65, 129), (1, 1000, 264), (5, 520, 1032),
               (64, 200, 72), (65, 72, 200), (129, 96, 257), (255, 130, 64), (300, 513, 264), (257, 264, 1030)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,hidden,inner", GATED_SIZES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 3), (8, 8)])
def test_gated(dtype, rows, hidden, inner, offset, pad):
    act = ("silu", "gelu", "relu")[(rows + inner + pad) % 3]
    log("gated %s %dx%dx%d %s offset=%d pad=%d" % (dtype, rows, hidden, inner, act, offset, pad))
    check_gated(dtype, rows, hidden, inner, act, offset, pad)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("act", sorted(ops.ACTIVATIONS))
def test_gated_activations(dtype, act):
    check_gated(dtype, 40, 72, 136, act, seed=11)


def test_gelu_keeps_its_lower_tail():
    """Exact pre-activations (one hidden element, 1), a bound relative to the value. Binary32: the lower side's factor is
    off by 1 / (1 + k |z|) (3 u), ten multiply-adds of falling weight (8 u), the exponential (4 u, its corrected argument
    none) and two products: below 24 u in all, the derivative's two terms as much each, and its constant and products 4 u.
    16 bits: a relative 4.3e-7 and the argument's three roundings of z^2 / 2, against half a unit v of the result."""
    z = -torch.arange(0, 12 * 16 + 1, device="cuda").double() / 16
    for dtype in sorted(TYPES):
        log("gelu tail %s" % dtype)
        w = z.to(TYPES[dtype])[None]
        one, ones = torch.ones((1, 1), dtype=TYPES[dtype], device="cuda"), torch.ones_like(w)
        assert torch.equal(w[0].double(), z)
        c, e = 0.5 * torch.erfc(-z / 2 ** 0.5), torch.exp(-0.5 * z * z) / (2 * np.pi) ** 0.5
        own = 28 * U if dtype == "f32" else 5e-7 + (1.5 * z * z + 16) * U
        dx, dg, du = ops.gated_backward(ones, one, w, ones, act="gelu")
        for got, want, size in ((ops.gated(one, w, ones, act="gelu"), z * c, (z * c).abs()), (du, z * c, (z * c).abs()),
                                (dg, c + z * e, c + (z * e).abs())):
            bound = own * size
            bound = bound + (HALF_ULP[dtype] * (want.abs() + bound) + TINY[dtype] if dtype != "f32" else 0.0)
            worst = ((got[0].double() - want).abs() - bound).max()
            assert worst <= 0, (dtype, float(worst))
    up = ops.gated(torch.ones((1, 1), device="cuda"), torch.tensor([[3.0, 20.0, 1e30, float("inf")]], device="cuda"),
                   torch.ones((1, 4), device="cuda"), act="gelu")[0].double().cpu()
    assert abs(float(up[0]) - 2.995950305904595) < 4 * U * 3 and torch.equal(up[1:], torch.tensor([20.0, 1e30, float("inf")]).double())


def check_gated_on_device(dtype, rows, hidden, inner, act="silu", seed=21):
    """Larger sizes: products of the reference in 64 bits on the device; norms of the differences, since the bounds'
    products cost as much again. Rounding errors are independent: each result is off by at most its own rounding and
    that of dg and du, v each, in norm, and the sums in binary32 by (N + 8) u of the norms' product over sqrt N, which
    is below v / 4 for 16-bit types here; binary32 by 16 (N + 8)^0.5 u."""
    x = randn((rows, hidden), dtype, seed)
    wg, wu = (randn((hidden, inner), dtype, seed + k, gain=hidden ** -0.5) for k in (1, 2))
    dh = randn((rows, inner), dtype, seed + 3)
    h = ops.gated(x, wg, wu, act=act)
    got = (h,) + ops.gated_backward(dh, x, wg, wu, act=act)
    X, G, W, D = (t.double() for t in (x, wg, wu, dh))
    g, u = X @ G, X @ W
    s = torch.sigmoid(g)
    a, da = g * s, s * (1 + g * (1 - s))
    dg, du = D * u * da, D * a
    want = (a * u, dg @ G.t() + du @ W.t(), X.t() @ dg, X.t() @ du)
    most = max(hidden, 2 * inner, rows)
    tol = 2.25 * HALF_ULP[dtype] if dtype != "f32" else 16 * (most + 8) ** 0.5 * U
    for y, w, what in zip(got, want, ("h", "dx", "dw_gate", "dw_up")):
        off = float((y.double() - w).norm() / w.norm())
        assert off < tol, (what, off)
        big = float(((y.double() - w).abs() / (w.abs() + w.square().mean().sqrt())).max())
        assert big < 8 * tol, (what, big)   # no element by itself


@pytest.mark.parametrize("dtype,rows,hidden,inner", [
    ("bf16", 2048, 1024, 4096), ("f16", 4096, 2048, 2048), ("f32", 2048, 512, 2048), ("f16", 1, 4096, 16384),
    ("bf16", 37, 2048, 8200), ("f16", 777, 1023, 2731), ("f32", 5, 4100, 4099), ("bf16", 20000, 72, 136),
    ("bf16", 70, 96, 20000), ("f16", 129, 8192, 160)])
def test_gated_large(dtype, rows, hidden, inner):
    log("gated %s %dx%dx%d" % (dtype, rows, hidden, inner))
    check_gated_on_device(dtype, rows, hidden, inner)


def check_held(rows, hidden, inner, gains, offset=0, pad=0, act="silu"):
    """binary16's dg and du past its range, with results inside it. They are rounded relative to the power of two that they
    are held times: with the largest M of them outside [2^-6, 65504], M is brought to at least 2^14, so that the smallest
    step's half is below 2^-25 2^-14 M; inside, it is 2^-25."""
    x, wg, wu, dh = (randn(s, "f16", 61 + k, gain=g, offset=offset, pad=pad) for k, (s, g) in enumerate(
        zip(((rows, hidden), (hidden, inner), (hidden, inner), (rows, inner)), gains)))
    X, G, W, D = (host(t) for t in (x, wg, wu, dh))
    g, u, a, da, eu, ea, eda = gated_bounds(X, G, W, act)
    pg, pu = D * u * da, D * a
    most = max(np.abs(pg).max(), np.abs(pu).max())
    tiny, v = TINY["f16"] if 2.0 ** -6 <= most <= 65504 else most * 2.0 ** -39, HALF_ULP["f16"]
    epg = np.abs(D) * (eda * (np.abs(u) + eu) + np.abs(da) * eu) + 3 * U * np.abs(pg)
    epu = np.abs(D) * ea + 2 * U * np.abs(pu)
    epg, epu = epg + v * (np.abs(pg) + epg) + tiny, epu + v * (np.abs(pu) + epu) + tiny
    dx, dg, du = ops.gated_backward(dh, x, wg, wu, act=act)
    both, eboth = product(np.concatenate([pg, pu], 1), np.concatenate([G, W], 1).T, da=np.concatenate([epg, epu], 1))
    wants = [(dx, both, eboth, "dx")]
    for got, p, e, what in ((dg, pg, epg, "dw_gate"), (du, pu, epu, "dw_up")):
        wants.append((got,) + product(X.T, p, db=e) + (what,))
    for got, want, bound, what in wants:
        assert np.abs(want).max() < 60000, (what, np.abs(want).max())
        check(got, want, bound, "f16", what)
    return most, (x, wg, wu, dh), (dx, dg, du)


@pytest.mark.parametrize("rows,hidden,inner,offset,pad", [
    (4, 64, 64, 0, 0), (4, 64, 72, 1, 3), (129, 64, 200, 0, 0), (129, 65, 201, 1, 3), (300, 72, 1032, 0, 0),
    (16, 1024, 64, 0, 0), (16, 1024, 65, 1, 1), (600, 64, 2048, 0, 0)])
def test_gated_gradient_past_the_range_of_binary16(rows, hidden, inner, offset, pad):
    """dg = dh u act'(g) vanishes with dh and u small; it overflows with both large, while x and Wg are small enough for dW
    and dx."""
    root, wide = hidden ** -0.5, inner ** -0.5
    for step in (10, 14, 20):
        log("gated gradient %dx%dx%d of about 2^-%d" % (rows, hidden, inner, 2 * step))
        most, _, got = check_held(rows, hidden, inner, (8.0, root / 8, 2.0 ** -step, 2.0 ** -step), offset, pad)
        assert most < 2.0 ** -6 and (step > 10 or float(got[1].abs().max()) > 0)
    # u is 2^9 / sqrt(rows), dg 2^16 to 2^18 and its largest several times that; act(g) is far below 1
    log("gated gradient %dx%dx%d of about 2^18" % (rows, hidden, inner))
    gains = (2.0 ** -6 * rows ** -0.5, 2.0 ** -6 * wide, 2.0 ** 15 * root, min(2.0 ** 12.5, 2.0 ** 10 * rows ** 0.5))
    most, args, got = check_held(rows, hidden, inner, gains, offset, pad)
    x, wg, wu, dh = args
    assert most > 65504
    dh = dh.clone()   # what is infinite stays in its row of dx
    dh[1, 3] = float("inf")
    again = ops.gated_backward(dh, x, wg, wu)
    rest = [k for k in range(rows) if k != 1]
    assert torch.equal(again[0][rest], got[0][rest]) and not torch.isfinite(again[0][1]).all()


def test_gated_extremes():
    x, wg, wu = randn((6, 40), "bf16", 1), randn((40, 24), "bf16", 2), randn((40, 24), "bf16", 3)
    h = ops.gated(x, wg, wu)
    assert torch.equal(ops.gated(x[0], wg, wu).view(1, -1), ops.gated(x[:1], wg, wu))          # one dimension
    assert torch.equal(ops.gated(x.view(2, 3, 40), wg, wu), h.view(2, 3, 24))
    # no rows
    assert ops.gated(x[:0], wg, wu).shape == (0, 24)
    dx, dg, du = ops.gated_backward(h[:0], x[:0], wg, wu)
    assert dx.shape == (0, 40) and torch.all(dg == 0) and torch.all(du == 0)
    # what one row or column holds stays in it
    y = x.clone()
    y[2, 5] = NAN
    z = ops.gated(y, wg, wu)
    assert torch.isnan(z[2]).all() and torch.equal(z[[0, 1, 3, 4, 5]], h[[0, 1, 3, 4, 5]])
    g = wg.clone()
    g[7, 3] = float("inf")
    z = ops.gated(x, g, wu)
    rest = [k for k in range(24) if k != 3]
    assert torch.equal(z[:, rest], h[:, rest]) and not torch.isfinite(z[:, 3]).all()
    # zeros give zeros, whatever the other factor
    assert torch.all(ops.gated(torch.zeros_like(x), wg, wu) == 0)
    # a broadcast row: stride 0
    row = x[:1].expand(6, 40)
    assert torch.equal(ops.gated(row, wg, wu), h[:1].expand(6, 24))
    dh = randn((6, 24), "bf16", 4)
    for p, q in zip(ops.gated_backward(dh, row, wg, wu), ops.gated_backward(dh, row.contiguous(), wg, wu)):
        assert torch.equal(p, q)
    for p, q in zip(ops.gated_backward(dh[:1].expand(6, 24), x, wg, wu),
                    ops.gated_backward(dh[:1].expand(6, 24).contiguous(), x, wg, wu)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_gated_into_strided_rows(dtype):
    """Halves of one fused weight, rows of a wider result; what lies between stays."""
    x, w = randn((33, 72), dtype, 1), randn((72, 2 * 56), dtype, 2)
    wide = torch.full((33, 70), 7.0, dtype=TYPES[dtype], device="cuda")
    h = ops.gated(x, w[:, :56], w[:, 56:], out=wide[:, 5:61])
    assert torch.equal(h, ops.gated(x, w[:, :56].contiguous(), w[:, 56:].contiguous()))
    assert torch.all(wide[:, :5] == 7.0) and torch.all(wide[:, 61:] == 7.0)


def test_gated_backward_parts_and_strides_of_the_c_entry():
    """Any of the gradients alone, and rows of gradients apart from one another."""
    x, wg, wu, dh = randn((40, 72), "f16", 1), randn((72, 88), "f16", 2), randn((72, 88), "f16", 3), randn((40, 88), "f16", 4)
    want = ops.gated_backward(dh, x, wg, wu)
    c, device, _, dtype = ops._gated(x, wg, wu, "silu")
    need = ops.gated_workspace(x, wg, wu, backward=True)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")

    def call(dx, ldx, dg, ldg, du, ldu, bytes_=need):
        return ckm.lib().ckm_gated_backward_async(
            ops.F16, C.byref(c), dh.data_ptr(), 88, None if dx is None else dx.data_ptr(), ldx,
            None if dg is None else dg.data_ptr(), ldg, None if du is None else du.data_ptr(), ldu, work.data_ptr(), bytes_,
            torch.cuda.current_stream().cuda_stream)

    dx = torch.full((40, 75), 3.0, dtype=torch.float16, device="cuda")
    dg, du = (torch.full((72, n), 3.0, dtype=torch.float16, device="cuda") for n in (90, 97))
    assert call(dx, 75, None, 0, None, 0) == ckm.OK
    assert torch.equal(dx[:, :72], want[0]) and torch.all(dx[:, 72:] == 3.0)
    assert call(None, 0, dg, 90, du, 97) == ckm.OK
    assert torch.equal(dg[:, :88], want[1]) and torch.equal(du[:, :88], want[2])
    assert torch.all(dg[:, 88:] == 3.0) and torch.all(du[:, 88:] == 3.0)
    assert call(dx, 75, dg, 90, None, 0) == ckm.E_INVALID_ARG
    assert call(dx, 71, None, 0, None, 0) == ckm.E_INVALID_ARG
    assert call(dx, 75, None, 0, None, 0, need - 1) == ckm.E_INVALID_ARG


# ---------------------------------------------------------------------------
# cross entropy
# ---------------------------------------------------------------------------

def check_loss(dtype, rows, hidden, vocab, offset=0, pad=0, gain=2.0, weights=None, seed=31):
    x = randn((rows, hidden), dtype, seed, offset=offset, pad=pad)
    w = randn((vocab, hidden), dtype, seed + 1, gain=gain * hidden ** -0.5, offset=offset, pad=pad)
    gen = torch.Generator().manual_seed(seed)
    targets = torch.randint(0, vocab, (rows,), generator=gen)
    targets[::5] = -100
    targets[1::7] = vocab                    # past the table
    targets[2::11] = vocab - 1
    targets = targets.cuda()
    loss, lse = ops.cross_entropy(x, w, targets)
    X, W, t = host(x), host(w), targets.cpu().numpy()
    logits, el = product(X, W.T)
    want, lse64 = nodes.cross_entropy(X, W, t)
    most = el.max(1)
    e_lse = most + (vocab / 64 + 32) * U + 2 * U * np.abs(lse64)
    check(lse, lse64, e_lse, "f32", "lse")
    some = (t >= 0) & (t < vocab)
    check(loss, want, np.where(some, e_lse + most + U * np.abs(want), 0.0), "f32", "loss")
    assert torch.all(loss[torch.from_numpy(~some).cuda()] == 0)
    dloss = torch.full((rows,), 3.0, device="cuda") if weights is None else weights(rows)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, targets, lse)
    L, D = host(lse), host(dloss)
    d = np.exp(logits - L[:, None])
    ed = d * (np.expm1(el + 8 * U + U * np.abs(logits - L[:, None])))
    d[np.arange(rows)[some], t[some]] -= 1.0
    by = np.where(some, D, 0.0)[:, None]
    d, ed = np.where(some[:, None], d * by, 0.0), np.abs(by) * (ed + 3 * U * np.abs(d))
    tiny = TINY[dtype] if dtype != "f16" else TINY[dtype] * np.abs(by).max() / 32768 * 2   # relative to the largest
    ed = np.where(some[:, None], ed + HALF_ULP[dtype] * (np.abs(d) + ed) + tiny, 0.0)   # rounded once
    y, e = product(d, W, da=ed)
    check(dx, y, e, dtype, "dx")
    y, e = product(d.T, X, da=ed.T)
    check(dw, y, e, dtype, "dweight")
    assert torch.all(dx[torch.from_numpy(~some).cuda()] == 0)
    return loss, lse, dx, dw


LOSS_SIZES = [(1, 1, 1), (1, 64, 300), (2, 8, 1), (3, 7, 5), (16, 128, 256), (17, 65, 129), (1, 1000, 2050), (40, 520, 700),
              (64, 200, 72), (129, 96, 257), (255, 130, 64), (300, 264, 1030), (7, 24, 9001)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,hidden,vocab", LOSS_SIZES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (1, 3), (8, 8)])
def test_cross_entropy(dtype, rows, hidden, vocab, offset, pad):
    log("cross entropy %s %dx%dx%d offset=%d pad=%d" % (dtype, rows, hidden, vocab, offset, pad))
    check_loss(dtype, rows, hidden, vocab, offset, pad)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_cross_entropy_weighted_rows_and_peaked_logits(dtype):
    ramp = lambda n: torch.linspace(-1.0, 2.0, n, device="cuda")   # noqa: E731  some negative, one near 0
    check_loss(dtype, 100, 72, 500, weights=ramp)
    check_loss(dtype, 100, 72, 500, gain=30.0)                     # probabilities of 1 and of nothing
    check_loss(dtype, 100, 72, 500, weights=lambda n: torch.zeros(n, device="cuda"))
    check_loss(dtype, 100, 72, 500, weights=lambda n: torch.full((n,), 1e-7, device="cuda") * (1 if dtype == "f32" else 1e5))


def test_cross_entropy_pieces():
    """More rows and a larger vocabulary than one piece of d holds, and a table that is copied piece by piece (odd rows);
    the reference in 64 bits on the device, norms as in check_gated_on_device."""
    for dtype, rows, hidden, vocab in (("bf16", 9000, 40, 20011), ("f32", 5000, 24, 9500), ("f16", 8200, 136, 24600),
                                       ("f16", 3000, 1001, 60001), ("bf16", 300, 1001, 60001), ("f32", 40, 2003, 30000)):
        log("cross entropy pieces %s" % dtype)
        x, w = randn((rows, hidden), dtype, 1), randn((vocab, hidden), dtype, 2, gain=2 * hidden ** -0.5)
        targets = torch.randint(-1, vocab, (rows,), generator=torch.Generator().manual_seed(3)).cuda()
        loss, lse = ops.cross_entropy(x, w, targets)
        t = x.double() @ w.double().t()
        some = targets >= 0
        want = torch.logsumexp(t, 1)
        # logits of order 10 from sums of up to 2003 terms, |x| |w| of order 100 in all: (N + 8) u of a random walk's
        # square root, and the logarithm's own
        assert float((lse - want).abs().max()) < 64 * U * 16
        at = t.gather(1, targets.clamp(min=0)[:, None])[:, 0]
        assert float((loss - torch.where(some, want - at, 0.0)).abs().max()) < 2 * 64 * U * 16
        dloss = torch.full((rows,), 0.5, device="cuda")
        dx, dw = ops.cross_entropy_backward(dloss, x, w, targets, lse)
        t.sub_(lse.double()[:, None]).exp_()
        t[some.nonzero()[:, 0], targets[some]] -= 1.0
        t *= (some * 0.5)[:, None]
        tol = 2.25 * HALF_ULP[dtype] if dtype != "f32" else 16 * (rows + 8) ** 0.5 * U
        for y, z in ((dx, t @ w.double()), (dw, t.t() @ x.double())):
            assert float((y.double() - z).norm() / z.norm()) < tol
            assert float(((y.double() - z).abs() / (z.abs() + z.square().mean().sqrt())).max()) < 8 * tol
        del t


@pytest.mark.parametrize("dtype,log_step", [("bf16", 12), ("bf16", 33), ("bf16", 100), ("f16", 10), ("f16", 28), ("f32", 12),
                                            ("f32", 33), ("f32", 100)])
def test_cross_entropy_of_vast_logits(dtype, log_step):
    """Exact logits, whole steps of 2^log_step apart: lse is the largest, a row's d 1 there and -1 at its target."""
    side, unit = 2.0 ** ((log_step + 2) // 2), 2.0 ** (log_step - 3 - (log_step + 2) // 2)   # 8 products of both are a step
    for rows, vocab in ((5, 300), (300, 1030)):
        log("cross entropy of vast logits %s 2^%d %dx%d" % (dtype, log_step, rows, vocab))
        gen = torch.Generator().manual_seed(rows)
        steps = torch.randint(-15, 16, (vocab,), generator=gen)
        steps[7], steps[11] = 31, -31
        targets = torch.randint(0, vocab, (rows,), generator=gen)
        targets[:3] = torch.tensor([7, 11, -1])
        x = torch.full((rows, 8), side, dtype=TYPES[dtype], device="cuda")
        w = (steps[:, None] * unit).expand(vocab, 8).to(TYPES[dtype]).contiguous().cuda()
        loss, lse = ops.cross_entropy(x, w, targets.cuda())
        some = targets >= 0
        assert torch.all(lse.cpu().double() == 31 * 2.0 ** log_step)
        assert torch.equal(loss.cpu().double(), torch.where(some, (31 - steps[targets.clamp(min=0)]) * 2.0 ** log_step, 0.0))
        by = 2.0 ** -10
        dx, dw = ops.cross_entropy_backward(torch.full((rows,), by, device="cuda"), x, w, targets.cuda(), lse)
        d = torch.zeros((rows, vocab), dtype=torch.float64)
        d[some, 7] = by
        d[some.nonzero()[:, 0], targets[some]] -= by
        for y, z in ((dx, d @ w.cpu().double()), (dw, d.t() @ x.cpu().double())):   # exact sums, rounded once
            assert torch.all((y.cpu().double() - z).abs() <= HALF_ULP[dtype] * z.abs())


def test_cross_entropy_extremes():
    x, w = randn((5, 40), "f16", 1), randn((70, 40), "f16", 2)
    targets = torch.tensor([3, -100, 69, 70, 0], device="cuda")
    loss, lse = ops.cross_entropy(x, w, targets)
    dl = torch.ones(5, device="cuda")
    dx, dw = ops.cross_entropy_backward(dl, x, w, targets, lse)
    assert loss[1] == 0 and loss[3] == 0 and torch.all(dx[[1, 3]] == 0)
    # no rows, one dimension, more dimensions
    none = ops.cross_entropy(x[:0], w, targets[:0])
    assert none[0].shape == (0,) and none[1].shape == (0,)
    none = ops.cross_entropy_backward(dl[:0], x[:0], w, targets[:0], lse[:0])
    assert none[0].shape == (0, 40) and torch.all(none[1] == 0)
    one = ops.cross_entropy(x[2], w, targets[2])
    assert one[0].shape == () and torch.equal(one[1], ops.cross_entropy(x[2:3], w, targets[2:3])[1][0])
    many = ops.cross_entropy(x[:4].view(2, 2, 40), w, targets[:4].view(2, 2))
    assert torch.equal(many[0], ops.cross_entropy(x[:4], w, targets[:4])[0].view(2, 2))
    # a row that nothing counts may hold anything, its loss gradient too
    y, d2 = x.clone(), dl.clone()
    y[1], d2[1], d2[3] = NAN, NAN, float("inf")
    l2, s2 = ops.cross_entropy(y, w, targets)
    assert torch.equal(l2, loss) and torch.isnan(s2[1])
    got = ops.cross_entropy_backward(d2, y, w, targets, s2)
    assert torch.equal(got[0], dx) and torch.equal(got[1], dw)
    # a row of NaN or of infinite logits is NaN by itself
    y = x.clone()
    y[0, 0] = float("inf")
    y[2] = NAN
    l2, s2 = ops.cross_entropy(y, w, targets)
    assert torch.isnan(s2[[0, 2]]).all() and torch.isnan(l2[[0, 2]]).all() and torch.equal(s2[[1, 3, 4]], lse[[1, 3, 4]])
    # every target outside: no gradient at all
    far = torch.full_like(targets, 1 << 40)
    l2, s2 = ops.cross_entropy(x, w, far)
    assert torch.all(l2 == 0) and torch.equal(s2, lse)
    assert all(torch.all(g == 0) for g in ops.cross_entropy_backward(dl, x, w, far, lse))
    # a vocabulary of one: loss and gradient 0
    one = torch.zeros(5, dtype=torch.int64, device="cuda")
    l1, s1 = ops.cross_entropy(x, w[:1], one)
    assert torch.all(l1 == 0)
    # rounded logits against themselves: at most a few units of the logits
    assert all(float(g.abs().max()) < 64 * U * float(s1.abs().max() + 1) * 40 for g in ops.cross_entropy_backward(dl, x, w[:1], one, s1))


def moved(t, offset, pad):
    """t's values in rows that start `offset` elements into an allocation, `pad` elements apart."""
    view = randn(tuple(t.shape), {v: k for k, v in TYPES.items()}[t.dtype], 0, offset=offset, pad=pad)
    view.copy_(t)
    return view


PLACES = [(0, 0), (1, 0), (1, 3), (8, 8), (0, 5)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,hidden,inner", [(16, 2048, 2048), (16, 4096, 1024), (3, 1040, 264), (64, 1024, 4096), (130, 2056, 520),
                                               (700, 264, 1032)])
def test_gated_bits_go_by_the_sizes(dtype, rows, hidden, inner):
    """The same values give the same bits wherever x's, the weights' or dh's rows lie."""
    x, dh = randn((rows, hidden), dtype, 1), randn((rows, inner), dtype, 2)
    wg, wu = (randn((hidden, inner), dtype, k, gain=hidden ** -0.5) for k in (3, 4))
    h, grads = ops.gated(x, wg, wu), ops.gated_backward(dh, x, wg, wu)
    for at in PLACES[1:]:
        for which in (1, 2, 3):
            log("gated bits %s %dx%dx%d %s %d" % (dtype, rows, hidden, inner, at, which))
            a = [moved(t, *at) if which & bit else t for t, bit in ((x, 1), (wg, 2), (wu, 2), (dh, 1))]
            assert torch.equal(ops.gated(*a[:3]), h)
            for p, q in zip(ops.gated_backward(a[3], *a[:3]), grads):
                assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,hidden,vocab", [(16, 2048, 2048), (16, 1040, 50000), (3, 4104, 9000), (100, 1032, 30000), (520, 264, 20000),
                                               (2000, 264, 10000), (9000, 64, 17000), (40, 2008, 60000)])
def test_cross_entropy_bits_go_by_the_sizes(dtype, rows, hidden, vocab):
    x, w = randn((rows, hidden), dtype, 1), randn((vocab, hidden), dtype, 2, gain=2 * hidden ** -0.5)
    targets = torch.randint(-1, vocab, (rows,), generator=torch.Generator().manual_seed(3)).cuda()
    dloss = torch.full((rows,), 0.5, device="cuda")
    want = ops.cross_entropy(x, w, targets)
    grads = ops.cross_entropy_backward(dloss, x, w, targets, want[1])
    for at in PLACES[1:4]:
        for which in (1, 2, 3):
            log("cross entropy bits %s %dx%dx%d %s %d" % (dtype, rows, hidden, vocab, at, which))
            a = [moved(t, *at) if which & bit else t for t, bit in ((x, 1), (w, 2))]
            for p, q in zip(ops.cross_entropy(*a, targets), want):
                assert torch.equal(p, q)
            for p, q in zip(ops.cross_entropy_backward(dloss, *a, targets, want[1]), grads):
                assert torch.equal(p, q)


def test_cross_entropy_gradient_of_a_vast_table_off_16_bytes():
    """Copied by shares of dx, past 4 GB: the bits of the table that need not be copied, within a bound of room."""
    rows, hidden, vocab = 8, 1000, 1250000
    x, dloss = randn((rows, hidden), "f32", 1), torch.ones(rows, device="cuda")
    flat = torch.empty(vocab * hidden + 1, dtype=torch.float32, device="cuda")
    w = flat[:-1].view(vocab, hidden).normal_(0.0, hidden ** -0.5, generator=torch.Generator(device="cuda").manual_seed(2))
    targets = torch.tensor([0, 1, vocab - 1, 1100000, 1073000, -1, 600000, vocab // 2], device="cuda")
    loss, lse = ops.cross_entropy(x, w, targets)
    dx, dw = ops.cross_entropy_backward(dloss, x, w, targets, lse)
    need = ops.cross_entropy_workspace(x, w, targets, backward=True)
    d = torch.exp(x.double() @ w[-2000:].double().t() - lse.double()[:, None])
    d[2, -1] -= 1.0
    d[5] = 0.0
    want = d.t() @ x.double()
    assert float((dw[-2000:].double() - want).norm() / want.norm()) < 16 * (rows + 8) ** 0.5 * U
    aside = torch.empty_like(flat)[1:].view(vocab, hidden)
    aside.copy_(w)
    assert need < ops.cross_entropy_workspace(x, aside, targets, backward=True) < need + (4 << 30) + (1 << 20)
    for p, q in zip(ops.cross_entropy_backward(dloss, x, aside, targets, lse), (dx, dw)):
        assert torch.equal(p, q)


def test_rows_further_apart_than_32_bits_count():
    ld = (1 << 31) + 24
    flat = torch.empty(2 * ld + 72, dtype=torch.float16, device="cuda")
    wide = flat.as_strided((3, 72), (ld, 1))
    x = randn((3, 72), "f16", 4)
    wide.copy_(x)
    wg, wu, dh = randn((72, 40), "f16", 5), randn((72, 40), "f16", 6), randn((3, 40), "f16", 7)
    assert torch.equal(ops.gated(wide, wg, wu), ops.gated(x, wg, wu))
    for p, q in zip(ops.gated_backward(dh, wide, wg, wu), ops.gated_backward(dh, x, wg, wu)):
        assert torch.equal(p, q)
    assert torch.equal(ops.gated(wg.t().contiguous()[:, :3].contiguous(), wide, wide), ops.gated(wg.t().contiguous()[:, :3].contiguous(), x, x))
    targets = torch.tensor([1, 2, 0], device="cuda")
    w = randn((50, 72), "f16", 8)
    loss, lse = ops.cross_entropy(x, w, targets)
    assert torch.equal(ops.cross_entropy(wide, w, targets)[0], loss)
    for p, q in zip(ops.cross_entropy_backward(loss, wide, w, targets, lse), ops.cross_entropy_backward(loss, x, w, targets, lse)):
        assert torch.equal(p, q)
    assert torch.equal(ops.cross_entropy(x, wide, targets)[1], ops.cross_entropy(x, x, targets)[1])


# ---------------------------------------------------------------------------
# norm and clipping
# ---------------------------------------------------------------------------

def grads(sizes, dtypes, seed=41, gain=1.0, offset=0):
    return [randn((n,), d, seed + k, gain=gain, offset=offset) for k, (n, d) in enumerate(zip(sizes, dtypes))]


def check_clip(g, max_norm, eps=1e-6):
    """Squares and sums are binary64: the norm is off by its rounding to binary32 (and 1e-12). An element by that of the
    factor, of the product and of its type."""
    want = nodes.norm([host(t) for t in g]) if sum(t.numel() for t in g) < 300000 else float(
        torch.stack([t.double().square().sum() for t in g]).sum().sqrt())
    norm = ops.gradient_norm(g)
    assert norm.shape == () and norm.dtype == torch.float32
    assert abs(float(norm) - want) <= (U + 1e-12) * want + TINY["f32"]
    factor = min(1.0, max_norm / (want + eps))
    out = [torch.full_like(t, 9.0) for t in g]
    same, got = ops.clip_gradients(g, max_norm, eps, out=out)
    assert torch.equal(same, norm) and all(p is q for p, q in zip(got, out))
    for t, y in zip(g, out):
        name = {v: k for k, v in TYPES.items()}[t.dtype]
        w = host(t) * factor
        check(y, w, 3 * U * np.abs(w), name, "clipped")
        if factor == 1.0:
            assert torch.equal(y, t)
    inplace = [t.clone() for t in g]
    n, got = ops.clip_gradients(inplace, max_norm, eps)
    assert torch.equal(n, norm) and all(p is q for p, q in zip(got, inplace))
    for y, z in zip(inplace, out):
        assert torch.equal(y, z)


@pytest.mark.parametrize("max_norm", [0.5, 1e4, 0.0])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_clip(max_norm, offset):
    sizes = [1, 7, 8, 4096, 8191, 8192, 8193, 100003, 3, 0, 16385]
    check_clip(grads(sizes, ["f32", "f16", "bf16", "f16", "f32", "bf16", "f16", "bf16", "f32", "f16", "f32"], offset=offset), max_norm)


@pytest.mark.parametrize("count", [0, 1, 111, 112, 113, 300, 1000])
def test_clip_of_many_tensors(count):
    check_clip(grads([1 + (37 * k) % 211 for k in range(count)], [("f32", "f16", "bf16")[k % 3] for k in range(count)]), 1.0)
    check_clip([torch.empty(0, device="cuda")] * min(count, 3), 1.0)


def test_clip_large_and_uneven():
    check_clip(grads([50_000_003, 5, 9_000_000], ["bf16", "f32", "f32"]), 10.0)
    check_clip(grads([2_000_000] * 8 + [10] * 200, ["f16"] * 208), 10.0)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_norm_of_equal_elements(dtype):
    """Where every group of squares rounds the same way: sums in binary64, so one rounding, of the result to binary32
    (u of the norm), and 1e-12 of the sums."""
    for value in (1.8017578125, 1.3330078125, 0.2998046875, 3.0517578125e-05):
        for n in (8, 100, 8000, 1 << 20):
            t = torch.full((n,), value, device="cuda").to(TYPES[dtype])
            want = float(t[0].double()) * n ** 0.5
            got = float(ops.gradient_norm([t]))
            assert abs(got - want) <= (U + 1e-12) * want, (value, n, (got / want - 1) / U)


def test_norm_extremes():
    big = torch.full((1000,), 1e30, device="cuda")          # squares past binary32's range
    small = torch.full((1000,), 1e-30, device="cuda")       # and below it
    for t in (big, small, big.bfloat16(), small.bfloat16()):
        want = float(t[0].double()) * 1000 ** 0.5
        assert abs(float(ops.gradient_norm([t])) - want) <= 2 * U * want
        _, (y,) = ops.clip_gradients([t], 1.0, eps=0.0, out=[torch.empty_like(t)])
        if float(t[0]) > 1:
            assert abs(float(y.double().norm()) - 1.0) < 2.0 ** -8
        else:
            assert torch.equal(y, t)
    assert float(ops.gradient_norm([])) == 0.0 and float(ops.gradient_norm([torch.zeros(5, device="cuda")])) == 0.0
    n, (y,) = ops.clip_gradients([torch.zeros(5, device="cuda")], 0.0, eps=0.0)   # 0 / 0
    assert float(n) == 0.0 and torch.isnan(y).all()
    n, (y,) = ops.clip_gradients([torch.tensor([1.0, float("inf"), -2.0], device="cuda")], 1.0)
    assert float(n) == float("inf") and torch.isnan(y[1]) and y[0] == 0 and y[2] == 0
    n, (y,) = ops.clip_gradients([torch.tensor([1.0, NAN], device="cuda")], 1.0)
    assert torch.isnan(n) and torch.isnan(y).all()
    n, (y,) = ops.clip_gradients([torch.tensor([1.0, 2.0], device="cuda")], float("inf"))
    assert torch.equal(y, torch.tensor([1.0, 2.0], device="cuda"))
    # any order of dimensions, as long as the elements fill one range
    t = randn((20, 30), "f32", 5)
    t = t.contiguous()
    assert torch.equal(ops.gradient_norm([t.t()]), ops.gradient_norm([t]))
    assert torch.equal(ops.gradient_norm([t, t]), ops.gradient_norm([torch.cat([t, t])]))   # listed twice: counted twice
    _, (y,) = ops.clip_gradients([t.t()], 0.1, out=[torch.empty_like(t.t())])
    assert torch.equal(y.t(), ops.clip_gradients([t], 0.1, out=[torch.empty_like(t)])[1][0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_clip_by_factors_below_the_normal_range(dtype):
    """Elements near binary32's largest against a small bound: the product is normal where the factor is not. One rounding in
    binary64 and one to binary32 (2 u), and the type's."""
    g = torch.tensor([3.0e38, -1.0e37, 2.0e30, 0.0] * 5000, device="cuda").to(TYPES[dtype])
    for most in (1e-2, 1e-6, 1e-9):
        norm, (y,) = ops.clip_gradients([g], most, eps=0.0, out=[torch.empty_like(g)])
        wide = g.double()
        want = wide * (most / float(wide.square().sum().sqrt()))
        assert torch.all((y.double() - want).abs() <= (HALF_ULP[dtype] + 2 * U) * want.abs() + TINY[dtype]), most
        assert abs(float(y.double().norm()) / most - 1) < 2.0 ** -8


def test_clip_with_bounds_of_infinity():
    """A bound of inf leaves every element, whatever the norm; a smaller one with a norm of inf gives 0."""
    g = torch.tensor([1.0, float("inf"), -2.0], device="cuda")
    n, (y,) = ops.clip_gradients([g], float("inf"), out=[torch.empty_like(g)])
    assert float(n) == float("inf") and torch.equal(y, g)
    n, (y,) = ops.clip_gradients([g.clone()], float("inf"))
    assert float(n) == float("inf") and torch.equal(y, g)
    n, (y,) = ops.clip_gradients([g.clone()], 1e30)
    assert float(n) == float("inf") and torch.isnan(y[1]) and y[0] == 0 and y[2] == 0


@pytest.mark.parametrize("count", [1792, 1793, 2000, 20000])
def test_clip_of_long_lists(count):
    """On both sides of the length from which the sums are added once; each tensor by its own values."""
    flat = randn((count * 5,), "f32", 7)
    g = list(flat.split([4, 6] * (count // 2) + [5] * (count % 2)))
    want = float(flat.double().square().sum().sqrt())
    out = torch.empty_like(flat)
    norm, _ = ops.clip_gradients(g, 0.25 * want, eps=0.0, out=list(out.split([t.numel() for t in g])))
    assert abs(float(norm) - want) <= (U + 1e-12) * want and torch.equal(norm, ops.gradient_norm(g))
    assert torch.all((out.double() - 0.25 * flat.double()).abs() <= 2 * U * flat.double().abs() + TINY["f32"])


# ---------------------------------------------------------------------------
# together: streams, graphs, work buffers
# ---------------------------------------------------------------------------

def step(x, wg, wu, wd, table, targets, dloss, stream=None):
    """A block and a loss, forward and gradient, and the clipping at the end, as a training step has them."""
    h = ops.gated(x, wg, wu, stream=stream)
    y = (h.float().unsqueeze(-1) * wd.float()).sum(1).to(x.dtype)   # elementary product: the same bits everywhere
    loss, lse = ops.cross_entropy(y, table, targets, stream=stream)
    dy, dt = ops.cross_entropy_backward(dloss, y, table, targets, lse, stream=stream)
    dwd = (h.float().unsqueeze(-1) * dy.float().unsqueeze(1)).sum(0).to(x.dtype)
    dh = (dy.float().unsqueeze(1) * wd.float()).sum(2).to(x.dtype)
    dx, dg, du = ops.gated_backward(dh, x, wg, wu, stream=stream)
    out = [torch.empty_like(t) for t in (dg, du, dwd, dt)]
    norm, out = ops.clip_gradients([dg, du, dwd, dt], 0.5, out=out, stream=stream)
    return [loss, dx, norm] + list(out)


def step_inputs(dtype="f16", rows=33, hidden=40, inner=72, vocab=300, seed=51):
    return [randn((rows, hidden), dtype, seed), randn((hidden, inner), dtype, seed + 1, gain=0.2),
            randn((hidden, inner), dtype, seed + 2, gain=0.2), randn((inner, hidden), dtype, seed + 3, gain=0.2),
            randn((vocab, hidden), dtype, seed + 4, gain=0.2), torch.arange(rows, device="cuda") * 7 % (vocab + 9) - 1,
            torch.full((rows,), 1.0 / rows, device="cuda")]


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_step_against_automatic_differentiation_in_64_bits(dtype):
    """Each value passes at most 8 roundings to the type on its way, in norm v each (sums in binary32 are below v / 4, for
    binary32 tensors 300 u, the longest sum)."""
    args = step_inputs(dtype)
    got = step(*args)
    x, wg, wu, wd, table = (t.double().requires_grad_() for t in args[:5])
    targets, dloss = args[5], args[6].double()
    g = x @ wg
    y = (g * torch.sigmoid(g) * (x @ wu)) @ wd
    some = (targets >= 0) & (targets < table.shape[0])
    t = y @ table.t()
    loss = torch.where(some, torch.logsumexp(t, 1) - t.gather(1, torch.where(some, targets, 0)[:, None])[:, 0], 0.0)
    (loss * dloss).sum().backward()
    params = [wg.grad, wu.grad, wd.grad, table.grad]
    norm = torch.stack([p.square().sum() for p in params]).sum().sqrt()
    factor = min(1.0, 0.5 / (float(norm) + 1e-6))
    tol = 8 * HALF_ULP[dtype] if dtype != "f32" else 300 * U
    for a, b in zip(got, [loss.detach(), x.grad, norm] + [p * factor for p in params]):
        assert float((a.double() - b).norm() / b.norm()) < tol


def test_calls_on_another_stream_and_overlapping():
    args = step_inputs("bf16", rows=300, hidden=136, inner=264, vocab=1000)
    want = step(*args)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    x, wg, wu, _, table, targets, dloss = args
    for _ in range(3):
        # temporaries of the current stream as arguments
        h = ops.gated(x + 0, wg + 0, wu + 0, stream=side)
        loss, lse = ops.cross_entropy(x + 0, table + 0, targets + 0, stream=other)
        both = ops.cross_entropy_backward(dloss + 0, x + 0, table + 0, targets + 0, lse, stream=other)
        back = ops.gated_backward(h, x + 0, wg + 0, wu + 0, stream=side)
        norm = ops.gradient_norm([x + 0, wg + 0], stream=side)
        clipped = ops.clip_gradients([x + 0, wg + 0], 0.5, stream=other)
        side.synchronize()
        other.synchronize()
        h0 = ops.gated(x, wg, wu)
        assert torch.equal(h, h0)
        for p, q in zip(back, ops.gated_backward(h0, x, wg, wu)):
            assert torch.equal(p, q)
        l0, s0 = ops.cross_entropy(x, table, targets)
        assert torch.equal(loss, l0) and torch.equal(lse, s0)
        for p, q in zip(both, ops.cross_entropy_backward(dloss, x, table, targets, s0)):
            assert torch.equal(p, q)
        assert torch.equal(norm, ops.gradient_norm([x, wg]))
        n0, c0 = ops.clip_gradients([x + 0, wg + 0], 0.5)
        assert torch.equal(clipped[0], n0) and all(torch.equal(p, q) for p, q in zip(clipped[1], c0))
    for p, q in zip(step(*args), want):   # again: the same bits
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", sorted(TYPES))
def test_captured_and_replayed(dtype):
    """A whole step in a graph, replayed on other inputs with eager work between; two graphs that live at once."""
    sets = [step_inputs(dtype, seed=s) for s in (51, 71, 91)]
    sets[2][0] = randn((33, 41), dtype, 5)[:, :40]   # rows that have to be copied
    graphs = []
    for args in (sets[0], sets[2]):
        held = [torch.empty_like(t) if t.is_contiguous() else torch.empty((33, 41), dtype=t.dtype, device="cuda")[:, :40]
                for t in args]
        for p, q in zip(held, args):
            p.copy_(q)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(*held)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*held)
        graphs.append((graph, held, out))
    for turn in range(4):
        for graph, held, out in graphs:
            args = sets[turn % 2]
            for p, q in zip(held, args):
                p.copy_(q)
            graph.replay()
            want = step(*args)
            torch.cuda.synchronize()
            for p, q in zip(out, want):
                assert torch.equal(p, q), turn


def test_own_work_buffers():
    x, wg, wu = randn((50, 71), "f16", 1), randn((71, 90), "f16", 2), randn((71, 90), "f16", 3)
    dh, table = randn((50, 90), "f16", 4), randn((300, 71), "f16", 5)
    targets, dloss = torch.arange(50, device="cuda"), torch.ones(50, device="cuda")
    loss, lse = ops.cross_entropy(x, table, targets)
    calls = [
        (lambda w: [ops.gated(x, wg, wu, work=w)], ops.gated_workspace(x, wg, wu)),
        (lambda w: ops.gated_backward(dh, x, wg, wu, work=w), ops.gated_workspace(x, wg, wu, backward=True)),
        (lambda w: ops.cross_entropy(x, table, targets, work=w), ops.cross_entropy_workspace(x, table, targets)),
        (lambda w: ops.cross_entropy_backward(dloss, x, table, targets, lse, work=w),
         ops.cross_entropy_workspace(x, table, targets, backward=True)),
        (lambda w: [ops.gradient_norm([x.contiguous(), wg], work=w)], ops.norm_workspace(2)),
    ]
    for k, (call, need) in enumerate(calls):
        assert need > 0 or k in (0, 2)   # a forward call of few rows may need none
        want = call(None)
        work = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")   # NaN wherever it is read unwritten
        for p, q in zip(call(work[:need]), want):
            assert torch.equal(p, q)
        assert torch.all(work[need:] == 255)
        if need:
            with pytest.raises(ckm.CkmError):
                call(work[:need - 1])
    need = ops.norm_workspace(1)
    with pytest.raises(ckm.CkmError):
        ops.clip_gradients([wg], 1.0, work=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))


def test_refusals():
    x, w = randn((6, 40), "f16", 1), randn((40, 24), "f16", 2)
    dh, table, square = randn((6, 24), "f16", 3), randn((50, 40), "f16", 4), randn((40, 40), "f16", 5)
    targets = torch.zeros(6, dtype=torch.int64, device="cuda")
    dloss = torch.ones(6, device="cuda")
    lse = torch.zeros(6, device="cuda")
    bad = [
        lambda: ops.gated(x.cpu(), w, w),
        lambda: ops.gated(x.double(), w, w),
        lambda: ops.gated(x, w.float(), w),
        lambda: ops.gated(x, w[:39], w[:39]),
        lambda: ops.gated(x, w, w[:, :23]),
        lambda: ops.gated(x, w, None),
        lambda: ops.gated(x, None, w),
        lambda: ops.gated(x, w.t().contiguous().t(), w),           # columns not contiguous
        lambda: ops.gated(x, w, w, act="tanh"),
        lambda: ops.gated(x, w, w, out=dh[:5]),
        lambda: ops.gated(x, w, w, out=dh.float()),
        lambda: ops.gated(x, square, square, out=x),               # over its own operands
        lambda: ops.gated(x, square, square, out=square[5:11]),
        lambda: ops.gated(x[:, :0], w[:0], w[:0]),
        lambda: ops.gated(x, w[:, :0], w[:, :0]),
        lambda: ops.gated_backward(dh[:, :23], x, w, w),
        lambda: ops.gated_backward(None, x, w, w),
        lambda: ops.gated_backward(dh, x, w, w, work=torch.empty(10, device="cuda")),
        lambda: ops.cross_entropy(x, table[:, :39], targets),
        lambda: ops.cross_entropy(x, table.float(), targets),
        lambda: ops.cross_entropy(x, table[:0], targets),
        lambda: ops.cross_entropy(x, table, targets.int()),
        lambda: ops.cross_entropy(x, table, targets[:5]),
        lambda: ops.cross_entropy(x, table, targets.cpu()),
        lambda: ops.cross_entropy(x, table, None),
        lambda: ops.cross_entropy_backward(dloss.half(), x, table, targets, lse),
        lambda: ops.cross_entropy_backward(dloss[:5], x, table, targets, lse),
        lambda: ops.cross_entropy_backward(dloss, x, table, targets, None),
        lambda: ops.gradient_norm([x, x.cpu()]),
        lambda: ops.gradient_norm([x.double()]),
        lambda: ops.gradient_norm([x[:, :20]]),                    # gaps between its rows
        lambda: ops.gradient_norm([x[:1].expand(6, 40)]),
        lambda: ops.gradient_norm([3.0]),
        lambda: ops.clip_gradients([x], -1.0),
        lambda: ops.clip_gradients([x], NAN),
        lambda: ops.clip_gradients([x], 1.0, eps=-1.0),
        lambda: ops.clip_gradients([x, x], 1.0),                   # scaled twice
        lambda: ops.clip_gradients([x, w], 1.0, out=[x, x]),
        lambda: ops.clip_gradients([x], 1.0, out=[]),
        lambda: ops.clip_gradients([x], 1.0, out=[torch.empty_like(x).t()]),
        lambda: ops.clip_gradients([x], 1.0, out=[torch.empty_like(x).float()]),
        lambda: ops.clip_gradients([x.view(-1)[:100]], 1.0, out=[x.view(-1)[50:150]]),
    ]
    for k, f in enumerate(bad):
        with pytest.raises((ValueError, ckm.CkmError)):
            f()
            print("not refused: %d" % k)
    # in the rows of its own operand's matrix, but past its columns
    both = torch.zeros((6, 80), dtype=torch.float16, device="cuda")
    both[:, :40] = x
    assert torch.equal(ops.gated(both[:, :40], square, square, out=both[:, 40:]), ops.gated(x, square, square))
    assert torch.equal(both[:, :40], x)
    # listed in another's place: the outputs swap
    a, b = torch.ones(4, device="cuda"), torch.full((4,), 2.0, device="cuda")
    with pytest.raises(ckm.CkmError):
        ops.clip_gradients([a, b], 1.0, out=[b, a])
