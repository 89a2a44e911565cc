"""The training-node operators against their definitions in 64 bits (oracle/nodes.py).

Tolerances are error bounds of binary32 arithmetic, stated before any run, with
u = 2^-24 (binary32) and v the result type's half unit in the last place:
  * a value that is rounded once to the result type: v |y| (and half the
    smallest subnormal);
  * a sum of N terms, added in the order thread, wave, block, blocks: at most
    DEPTH u sum |terms|, DEPTH = 128 bounding the longest chain of additions
    at these sizes (32 in a thread, 16 waves, rows of a block, blocks);
  * products and differences: u each.
"""
import numpy as np
import pytest
import torch

from oracle import nodes
from paper_1910_02653_amd import ckm, ops

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}
U = 2.0 ** -24
DEPTH = 128
SEED, SITE = 0x9E3779B97F4A7C15, (3 << 32) | 17


def log(msg):
    print(msg, flush=True)


def randn(shape, dtype, seed, gain=1.0, shift=0.0, offset=0, pad=0):
    """A device tensor whose rows start `offset` elements into an allocation and lie `pad` elements apart."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, cols = int(np.prod(shape[:-1])), shape[-1]
    flat = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=TYPES[dtype], device="cuda")
    view = flat[offset:].view(tuple(shape[:-1]) + (cols + pad,))[..., :cols]
    view.copy_(torch.randn(shape, generator=gen, device="cuda") * gain + shift)
    return view


def host(t):
    return t.double().cpu().numpy()


def check(got, want, tol, dtype, what):
    """|got - want| <= tol + the one rounding to the result's type."""
    got = host(got)
    bound = tol + HALF_ULP[dtype] * (np.abs(want) + tol) + TINY[dtype]
    off = np.abs(got - want)
    assert np.all(np.isfinite(got)), what
    worst = np.max(off / bound) if off.size else 0.0
    assert worst <= 1.0, "%s: error %.3g times its bound" % (what, worst)


# ---------------------------------------------------------------------------
# dropout
# ---------------------------------------------------------------------------

SIZES = [(1, 1), (3, 7), (5, 8), (2, 9), (70, 64), (7, 513), (4097, 3), (65537, 1), (33, 1000), (2, 16389), (3, 100000), (1, 1200003)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("residual,offset,pad", [(False, 0, 0), (True, 1, 3)])
def test_dropout(dtype, rows, cols, residual, offset, pad):
    log("dropout %s %dx%d residual=%s" % (dtype, rows, cols, residual))
    d = ops.Dropout(0.3, SEED, SITE)
    x = randn((rows, cols), dtype, 1, offset=offset, pad=pad)
    r = randn((rows, cols), dtype, 2, offset=offset, pad=pad + 1) if residual else None
    f = nodes.factors(rows, cols, SEED, SITE, d.keep)
    y = ops.dropout(x, d, residual=r)
    want = nodes.dropout(host(x), f, None if r is None else host(r))
    # the factor's rounding and the product, then the sum
    check(y, want, 2 * U * np.abs(host(x)) * f + U * np.abs(want), TYPES[dtype], "y")
    if r is None:
        assert np.array_equal(host(y) != 0, (f > 0) & (host(x) != 0))
    dx = ops.dropout_backward(x, d)
    assert torch.equal(dx, ops.dropout(x, d))
    y2 = x.clone()
    assert ops.dropout(y2, d, residual=r, out=y2) is y2 and torch.equal(y2, y)   # in place, same bits


def test_dropout_special_values_and_extremes():
    d = ops.Dropout(0.5, SEED, SITE)
    f = nodes.factors(16, 100, SEED, SITE, d.keep)
    for value in (float("nan"), float("inf"), -float("inf")):
        x = torch.full((16, 100), value, device="cuda")
        y = host(ops.dropout(x, d))
        assert np.all(y[f == 0] == 0)
        assert np.all(np.isnan(y[f > 0]) if np.isnan(value) else y[f > 0] == value)
    x = randn((16, 100), "f16", 3)
    assert torch.equal(ops.dropout(x, ops.Dropout(0.0, 1)), x)
    assert torch.all(ops.dropout(x, ops.Dropout(1.0, 1)) == 0)
    assert ops.dropout(x[:0], d).shape == (0, 100) and ops.dropout(x[:, :0], d).shape == (16, 0)
    assert torch.equal(ops.dropout(x[0], d), ops.dropout(x[:1], d)[0])   # one dimension
    # other sites and seeds are other masks; a site from the device is added to the number
    y = ops.dropout(x, d)
    assert not torch.equal(y, ops.dropout(x, ops.Dropout(0.5, SEED, SITE + 1)))
    assert not torch.equal(y, ops.dropout(x, ops.Dropout(0.5, SEED + 1, SITE)))
    step = torch.tensor([SITE - 5], device="cuda")
    assert torch.equal(y, ops.dropout(x, ops.Dropout(0.5, SEED, 5, step)))


def test_rows_further_apart_than_32_bits_count():
    """Row offsets past 2^32 elements, for every operator that takes a stride."""
    ld = (1 << 31) + 24
    wide = torch.empty(2 * ld + 72, dtype=torch.float16, device="cuda").as_strided((3, 72), (ld, 1))
    x = randn((3, 72), "f16", 4)
    wide.copy_(x)
    d = ops.Dropout(0.2, SEED, SITE)
    assert torch.equal(ops.dropout(wide, d, residual=wide), ops.dropout(x, d, residual=x))
    for a, b in zip(ops.layer_norm(wide, drop=d), ops.layer_norm(x, drop=d)):
        assert torch.equal(a, b)
    _, _, stats = ops.layer_norm(x)
    for a, b in zip(ops.layer_norm_backward(wide, wide, stats), ops.layer_norm_backward(x, x, stats)):
        assert torch.equal(a, b)
    y, st = ops.softmax(wide, drop=d)
    assert torch.equal(y, ops.softmax(x, drop=d)[0])
    assert torch.equal(ops.softmax_backward(wide, wide, st, drop=d), ops.softmax_backward(x, x, st, drop=d))
    assert torch.equal(ops.dropout(x, d, out=wide), ops.dropout(x, d))


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 2), (5, 7), (17, 64), (40, 128), (9, 129), (33, 512), (7, 1000), (130, 1023), (20, 2048),
              (11, 4095), (6, 8192), (3, 12345), (4, 16384), (3, 16385), (2, 32768), (2000, 96), (5000, 40)]


def norm_bounds(h, w, eps):
    """Bounds of the errors of mean, of rstd (relative) and of y before its rounding."""
    n = h.shape[1]
    mean, d_mean = h.mean(1), DEPTH * U * np.abs(h).mean(1)
    var = ((h - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    # the centred values carry d_mean, which enters the variance squared
    d_var = (DEPTH + 6) * U * var + d_mean ** 2 + 2 * d_mean * U * np.abs(h).mean(1)
    d_rstd = 0.5 * d_var / (var + eps) + 4 * U
    xh = (h - mean[:, None]) * rstd[:, None]
    d_y = np.abs(w) * (d_mean[:, None] * rstd[:, None] + np.abs(xh) * (d_rstd[:, None] + 4 * U)) + 4 * U * np.abs(xh * w)
    return d_mean + U * np.abs(mean), d_rstd, d_y


@pytest.mark.parametrize("dtype,wtype", [("f32", "f32"), ("f16", "f16"), ("f16", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows,cols", NORM_SIZES)
def test_layer_norm_and_gradient(dtype, wtype, rows, cols):
    log("layer norm %s weights %s %dx%d" % (dtype, wtype, rows, cols))
    T, W, eps = TYPES[dtype], TYPES[wtype], 1e-5
    odd = rows % 2
    x = randn((rows, cols), dtype, 5, gain=1.5, shift=0.7, offset=odd, pad=odd)
    r = randn((rows, cols), dtype, 6, offset=2 * odd, pad=5 * odd)
    w, b = randn((cols,), wtype, 7, shift=1.0), randn((cols,), wtype, 8)
    d = ops.Dropout(0.25, SEED, SITE)
    f = nodes.factors(rows, cols, SEED, SITE, d.keep)

    y, h, stats = ops.layer_norm(x, w, b, eps=eps, residual=r, drop=d)
    want_h = nodes.dropout(host(x), f, host(r))
    check(h, want_h, 2 * U * np.abs(host(x)) * f + U * np.abs(want_h), T, "h")
    # the norm is of the rounded h
    hh, ww, bb = host(h), host(w), host(b)
    want, mean, rstd = nodes.layer_norm(hh, ww, bb, eps)
    d_mean, d_rstd, d_y = norm_bounds(hh, ww, eps)
    check(stats[..., 0], mean, d_mean, torch.float32, "mean")
    check(stats[..., 1], rstd, d_rstd * rstd, torch.float32, "rstd")
    check(y, want, d_y + 2 * U * (np.abs(want) + np.abs(bb)), T, "y")
    # one pass gives the bits of the separate operators
    h2 = ops.dropout(x, d, residual=r)
    assert torch.equal(h, h2)
    y2, h3, stats2 = ops.layer_norm(h2, w, b, eps=eps)
    assert h3 is h2 and torch.equal(y, y2) and torch.equal(stats, stats2)

    # gradient, on the statistics that the forward pass left
    dy = randn((rows, cols), dtype, 9, offset=3 * odd, pad=7 * odd)
    past = randn((rows, cols), dtype, 10)
    mean, rstd = host(stats[..., 0]), host(stats[..., 1])
    dx, dh, dw, db = ops.layer_norm_backward(dy, h, stats, w, dres=past, drop=d)
    g, pp = host(dy), host(past)
    want, want_w, want_b = nodes.layer_norm_backward(g, hh, mean, rstd, ww)
    xh = (hh - mean[:, None]) * rstd[:, None]
    gw = np.abs(g * ww)
    s1, s2 = gw.mean(1, keepdims=True), (gw * np.abs(xh)).mean(1, keepdims=True)
    d_dh = rstd[:, None] * (8 * U * gw + (DEPTH + 8) * U * (s1 + np.abs(xh) * s2)) + U * np.abs(want + pp) + U * np.abs(pp)
    check(dh, want + pp, d_dh, T, "dh")
    d_full = d_dh + HALF_ULP[T] * (np.abs(want + pp) + d_dh) + TINY[T]
    check(dx, nodes.dropout(want + pp, f), (d_full + 2 * U * np.abs(want + pp)) * f, T, "dx")
    check(dw, want_w, (DEPTH + 8) * U * np.abs(g * xh).sum(0), W, "dweight")
    check(db, want_b, DEPTH * U * np.abs(g).sum(0), W, "dbias")
    # the parts are the whole's: same bits without the fused ends, and a second time
    dx0, dh0, dw0, db0 = ops.layer_norm_backward(dy, h, stats, w, dres=past)
    assert dx0 is dh0 and torch.equal(dh, dh0) and torch.equal(dw, dw0) and torch.equal(db, db0)
    assert torch.equal(dx, ops.dropout_backward(dh, d))
    again = dy.clone()
    got = ops.layer_norm_backward(again, h, stats, w, dres=past, drop=d, out=again)
    assert got[1] is again and all(torch.equal(p, q) for p, q in zip(got, (dx, dh, dw, db)))


def test_layer_norm_without_weights_and_edges():
    x = randn((6, 48), "f32", 11, shift=2.0)
    one, zero = torch.ones(48, device="cuda"), torch.zeros(48, device="cuda")
    y, h, stats = ops.layer_norm(x)
    assert h is x and torch.equal(y, ops.layer_norm(x, one, zero)[0])
    assert torch.equal(ops.layer_norm(x, bias=one)[0], ops.layer_norm(x, one, one)[0])
    for p, q in zip(ops.layer_norm_backward(x, x, stats), ops.layer_norm_backward(x, x, stats, one)):
        assert torch.equal(p, q)
    # a constant row: no variance, y is the bias, and the gradient stays finite
    c = torch.full((3, 100), 7.25, device="cuda")
    y, _, stats = ops.layer_norm(c, torch.ones(100, device="cuda"), torch.full((100,), 0.5, device="cuda"), eps=1e-5)
    assert torch.all(y == 0.5) and torch.all(stats[:, 0] == 7.25)
    assert torch.isfinite(ops.layer_norm_backward(c, c, stats)[0]).all()
    # a mean far from 0 costs no digits beyond its own rounding: variance of exact values
    big = torch.tensor([[4096.0, 4097.0, 4098.0, 4099.0]], device="cuda")
    _, _, stats = ops.layer_norm(big, eps=0.0)
    assert abs(float(stats[0, 1]) - 1.25 ** -0.5) < 1e-6
    # no rows: nothing for y, zero weight gradients; a row with a NaN leaves the others alone
    empty = x[:0]
    assert ops.layer_norm(empty)[0].shape == (0, 48)
    dx, dh, dw, db = ops.layer_norm_backward(empty, empty, stats[:0], one)
    assert dh.shape == (0, 48) and torch.all(dw == 0) and torch.all(db == 0)
    wide = torch.empty((0, 20000), device="cuda")
    assert torch.all(ops.layer_norm_backward(wide, wide, torch.empty((0, 2), device="cuda"))[2] == 0)
    bad = x.clone()
    bad[2, 5] = float("nan")
    y, _, _ = ops.layer_norm(bad)
    assert torch.isnan(y[2]).all() and torch.equal(y[[0, 1, 3, 4, 5]], ops.layer_norm(x)[0][[0, 1, 3, 4, 5]])
    # more dimensions, a shared (broadcast) residual
    x3 = randn((2, 3, 48), "f16", 12)
    r = randn((48,), "f16", 13).expand(2, 3, 48)
    y, h, stats = ops.layer_norm(x3, residual=r)
    assert torch.equal(h, x3 + r) and stats.shape == (2, 3, 2)


# ---------------------------------------------------------------------------
# softmax
# ---------------------------------------------------------------------------

def masks(kind, shape, dtype, seed):
    """(device mask, host array): truth values shared by the heads, or added values shared by the batches."""
    B, H, Q, K = shape
    rng = np.random.default_rng(seed)
    if kind == "none":
        return None, None
    if kind == "bool":
        m = rng.random((B, 1, Q, K)) < 0.7
        m[:, :, Q // 2] = False            # a row that sees nothing
        return torch.from_numpy(m).cuda(), m
    m = rng.standard_normal((1, H, Q, K)).astype(np.float32)
    m[rng.random(m.shape) < 0.2] = -np.inf
    low = rng.random(m.shape) < 0.2
    m[:, :, Q // 3] = -np.inf
    t = torch.from_numpy(m).to(TYPES[dtype])
    t[torch.from_numpy(low & (m > -np.inf))] = torch.finfo(TYPES[dtype]).min
    first = t[..., 0]                      # not lowest everywhere
    first[first > -np.inf] = 0.0
    return t.cuda(), t.double().numpy()


SCORES = [(1, 1, 1, 1), (2, 3, 5, 7), (1, 2, 33, 128), (2, 1, 9, 300), (1, 3, 7, 1000), (2, 2, 3, 1025), (1, 1, 6, 2048),
          (1, 1, 5, 4093), (1, 2, 2, 4097), (1, 1, 70, 8000), (1, 1, 66, 16384), (1, 65, 1, 30001), (1, 1, 2, 70001),
          (3, 1, 1, 262147), (2, 2, 50, 20)]


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("shape", SCORES)
@pytest.mark.parametrize("kind,causal,ragged", [("none", True, False), ("bool", False, True), ("add", True, True)])
def test_softmax_and_gradient(dtype, shape, kind, causal, ragged):
    log("softmax %s %s mask=%s causal=%s ragged=%s" % (dtype, shape, kind, causal, ragged))
    T = TYPES[dtype]
    B, H, Q, K = shape
    rng = np.random.default_rng(B + H + Q + K)
    scale = 0.3
    x = randn(shape, dtype, 14, gain=4.0, offset=K % 3, pad=K % 5)
    lens = rng.integers(0, K + 1, B) if ragged else None
    if lens is not None:
        lens[-1] = K
    lengths = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    mask, hmask = masks(kind, shape, dtype, 15)
    seen = nodes.visible(shape, causal, lens, hmask)
    x = torch.where(torch.from_numpy(seen).cuda(), x, float("nan"))   # what is not seen is not used
    d = ops.Dropout(0.2, SEED, SITE)
    f = nodes.factors(B * H * Q, K, SEED, SITE, d.keep).reshape(shape)
    kw = dict(scale=scale, causal=causal, lengths=lengths, mask=mask)

    t = nodes.logits(host(x), scale, seen, hmask)
    p, m, z = nodes.softmax(t)
    tt, xx = np.where(seen, t, 0.0), np.where(seen, host(x), 0.0)
    add = np.zeros(shape) if hmask is None or hmask.dtype.kind == "b" else np.where(seen, np.broadcast_to(hmask, shape), 0.0)
    # relative error of each exponential: the logit's roundings (the scale is binary32 too), the
    # difference to the maximum, the factor log2 e, the unit's last bit
    rel = 3 * U * np.abs(xx * scale) + 2 * U * (np.abs(tt) + np.abs(add)) + 4 * U * np.abs(tt - m[..., None]) + 8 * U
    rel = np.where(p > 0, rel, 0.0)
    rel_z = (p * rel).sum(-1) + 2 * U * np.abs(m) + (DEPTH + 4) * U
    y, stats = ops.softmax(x, drop=d, **kw)
    d_p = p * (rel + rel_z[..., None] + 4 * U) + 2.0 ** -126
    check(y, p * f, d_p * f + 2 * U * p * f, T, "y")
    assert np.all(host(y)[~seen] == 0)
    check(stats[..., 0], m, 4 * U * np.abs(m) + 3 * U * np.abs(xx * scale).max(-1, initial=0.0), torch.float32, "max")
    check(stats[..., 1], z, z * rel_z, torch.float32, "1 / sum")
    assert np.array_equal(host(stats[..., 1]) == 0, z == 0)
    # the dropout inside is the dropout after it (where no rounding lies between: binary32)
    plain, stats2 = ops.softmax(x, **kw)
    assert torch.equal(stats, stats2)
    check(plain, p, d_p, T, "no dropout")
    if dtype == "f32":
        assert torch.equal(y, ops.dropout(plain, d))

    dy = randn(shape, dtype, 16, offset=1, pad=2)
    dy = torch.where(torch.from_numpy(seen & (f > 0)).cuda(), dy, float("inf"))
    dx = ops.softmax_backward(dy, x, stats, drop=d, **kw)
    g = nodes.dropout(np.where(seen & (f > 0), host(dy), 0.0), f)
    hs = host(stats)
    with np.errstate(invalid="ignore"):
        p = np.where(seen, np.exp(t - hs[..., :1]) * hs[..., 1:], 0.0)
    want = nodes.softmax_backward(g, p, scale)
    s = (p * g).sum(-1, keepdims=True)
    d_s = (np.abs(p * g) * (rel + (DEPTH + 8) * U)).sum(-1, keepdims=True)
    tol = scale * p * (np.abs(g - s) * (rel + 8 * U) + d_s + 3 * U * np.abs(g)) + 2.0 ** -120
    check(dx, want, tol, T, "dx")
    assert np.all(host(dx)[~seen] == 0)
    # again, and in place: the same bits
    buf = dy.clone()
    assert ops.softmax_backward(buf, x, stats, drop=d, out=buf, **kw) is buf and torch.equal(buf, dx)
    buf = x.clone()
    got = ops.softmax(buf, drop=d, out=buf, **kw)
    assert got[0] is buf and torch.equal(buf, y) and torch.equal(got[1], stats)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("keys", [5, 600, 5000, 40000])
def test_softmax_rows_of_one_kind(dtype, keys):
    """Whole rows at the type's lowest value, at -inf, hidden, and with infinities and NaN."""
    T = TYPES[dtype]
    low = torch.finfo(T).min
    x = torch.zeros((6, keys), dtype=T, device="cuda")
    x[1] = low
    x[2] = -float("inf")
    x[3, 0] = float("nan")
    x[4, keys // 2] = float("inf")
    x[5, 1:] = -float("inf")
    y, stats = ops.softmax(x)
    v = torch.full((keys,), 1.0 / keys, dtype=T, device="cuda")
    assert torch.allclose(y[0].float(), v.float(), rtol=2.0 ** -7) and torch.equal(y[1], y[0])
    assert torch.all(y[2] == 0) and torch.all(stats[2] == 0)
    assert torch.isnan(y[3]).all() and torch.isnan(y[4]).any()
    assert y[5, 0] == 1 and torch.all(y[5, 1:] == 0)
    # a mask of the lowest value everywhere hides nothing: every key is as likely
    m = torch.full((1, keys), low, dtype=T, device="cuda")
    y, stats = ops.softmax(torch.zeros((1, keys), dtype=T, device="cuda"), mask=m)
    assert torch.allclose(y.float(), v.float(), rtol=2.0 ** -7)
    dx = ops.softmax_backward(torch.ones_like(y), torch.zeros_like(y), stats, mask=m)
    assert torch.isfinite(dx).all()
    # of -inf everywhere hides all
    m.fill_(-float("inf"))
    y, stats = ops.softmax(x[3:4], mask=m)
    assert torch.all(y == 0) and torch.all(stats == 0)
    assert torch.all(ops.softmax_backward(x[3:4], x[3:4], stats, mask=m) == 0)


def test_softmax_more_queries_than_keys_lengths_out_of_range_and_no_keys():
    x = randn((2, 2, 9, 4), "f32", 17)
    y, stats = ops.softmax(x, causal=True)
    assert torch.all(y[:, :, :5] == 0) and torch.all(stats[:, :, :5] == 0) and torch.all(y[:, :, 5, 0] == 1)
    lengths = torch.tensor([-3, 100], dtype=torch.int32, device="cuda")
    y, _ = ops.softmax(x, lengths=lengths)
    assert torch.all(y[0] == 0) and torch.equal(y[1], ops.softmax(x)[0][1])
    none = x[..., :0]
    y, stats = ops.softmax(none)
    assert y.shape == (2, 2, 9, 0) and torch.all(stats == 0)
    assert ops.softmax_backward(none, none, stats).shape == (2, 2, 9, 0)
    assert ops.softmax(x[:0])[0].shape == (0, 2, 9, 4)


def test_softmax_layouts():
    """Scores, outputs and masks in other orders than they are named in, fewer dimensions: the same bits."""
    x = randn((2, 3, 10, 77), "bf16", 18)
    d = ops.Dropout(0.1, SEED, SITE)
    want, stats = ops.softmax(x, drop=d, causal=True)
    other = x.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3)
    out = torch.empty_like(other)
    assert out.stride() == other.stride() != x.stride()
    got, st = ops.softmax(other, drop=d, causal=True, out=out)
    assert torch.equal(got, want) and torch.equal(st, stats)
    dx = ops.softmax_backward(x, x, stats, drop=d, causal=True)
    assert torch.equal(ops.softmax_backward(other, x, stats, drop=d, causal=True, out=out), dx)
    for k in (1, 2, 3):
        part = x[(1,) * k]
        assert torch.equal(ops.softmax(part, causal=True)[0],
                           ops.softmax(part.reshape((1,) * k + part.shape), causal=True)[0].reshape(part.shape))
    m = torch.rand((10, 77), device="cuda") < 0.5
    full = m.expand(2, 3, 10, 77).contiguous()
    assert torch.equal(ops.softmax(x, mask=m)[0], ops.softmax(x, mask=full)[0])
    assert torch.equal(ops.softmax(x, mask=m.to(torch.uint8) * 7)[0], ops.softmax(x, mask=full)[0])
    bias = torch.zeros_like(x).masked_fill_(~full, -float("inf"))
    assert torch.equal(ops.softmax(x, mask=bias)[0], ops.softmax(x, mask=full)[0])


# ---------------------------------------------------------------------------
# streams, graphs, repetition, refusals
# ---------------------------------------------------------------------------

def all_ops(x, s, d, stream=None):
    """Every operator once; x [rows, cols] and scores s, tensors of one type."""
    w, b = torch.ones_like(x[0]), torch.zeros_like(x[0])
    out = [ops.dropout(x, d, residual=x, stream=stream), ops.dropout_backward(x, d, stream=stream)]
    y, h, stats = ops.layer_norm(x, w, b, residual=x, drop=d, stream=stream)
    out += [y, h, stats, *ops.layer_norm_backward(x, h, stats, w, dres=x, drop=d, stream=stream)]
    p, st = ops.softmax(s, 0.5, causal=True, drop=d, stream=stream)
    return out + [p, st, ops.softmax_backward(s, s, st, 0.5, causal=True, drop=d, stream=stream)]


SHAPES = [((300, 1000), (1, 4, 60, 700)), ((2, 20000), (1, 1, 1, 50000)), ((16, 64), (2, 2, 8, 8))]


@pytest.mark.parametrize("rows,scores", SHAPES)
def test_other_streams_and_repetition_give_the_same_bits(rows, scores):
    x, s = randn(rows, "f16", 19), randn(scores, "f16", 20)
    d = ops.Dropout(0.1, SEED, SITE)
    want = all_ops(x, s, d)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    runs = [all_ops(x, s, d, stream=q) for q in streams for _ in range(3)]   # overlapping calls
    with torch.cuda.stream(streams[0]):
        runs.append(all_ops(x, s, d))
    torch.cuda.synchronize()
    for r in runs:
        assert all(torch.equal(p, q) for p, q in zip(r, want))


@pytest.mark.parametrize("rows,scores", SHAPES)
def test_graph_capture(rows, scores):
    """Captured once, replayed with eager work and synchronizations between; the device's step makes each replay's mask."""
    x, s = randn(rows, "bf16", 21), randn(scores, "bf16", 22)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = ops.Dropout(0.1, SEED, SITE, step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_ops(x, s, d)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_ops(x, s, d)
    for n in range(4):
        step.fill_(n)
        for t in got:
            t.fill_(3.0)
        x.copy_(randn(rows, "bf16", 23 + n))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = all_ops(x, s, ops.Dropout(0.1, SEED, SITE + n))
        assert all(torch.equal(p, q) for p, q in zip(got, want)), n


def test_binding_refusals():
    x = torch.zeros((4, 6, 8), device="cuda")
    d = ops.Dropout(0.1, 1)
    w = torch.ones(8, device="cuda")
    stats = torch.zeros((4, 6, 2), device="cuda")
    bad = [
        lambda: ops.dropout(x, None), lambda: ops.dropout(x, 0.1), lambda: ops.dropout(x.double(), d),
        lambda: ops.dropout(x.int(), d), lambda: ops.dropout(torch.zeros((), device="cuda"), d),
        lambda: ops.dropout(x, d, residual=x.half()), lambda: ops.dropout(x, d, residual=x[:2]),
        lambda: ops.dropout(x, d, residual=x.cpu()), lambda: ops.dropout(x[..., ::2], d),
        lambda: ops.dropout(x.transpose(0, 1), d), lambda: ops.dropout(x, d, out=x.half()),
        lambda: ops.layer_norm(x, w[:7]), lambda: ops.layer_norm(x, w.half()), lambda: ops.layer_norm(x, w, w.half()),
        lambda: ops.layer_norm(x.half(), w.bfloat16()), lambda: ops.layer_norm(x, w.repeat(2)[::2]),
        lambda: ops.layer_norm_backward(x, x, stats[..., 0]), lambda: ops.layer_norm_backward(x, x.half(), stats),
        lambda: ops.layer_norm_backward(x, x, stats.half()), lambda: ops.layer_norm_backward(x, x, stats, dres=x[0]),
        lambda: ops.layer_norm_backward(x, x, stats, work=torch.zeros(8, device="cuda")),
        lambda: ops.softmax(x[..., ::2]), lambda: ops.softmax(x[None, None]), lambda: ops.softmax(x, lengths=torch.ones(1, device="cuda")),
        lambda: ops.softmax(x, lengths=torch.ones(3, dtype=torch.int32, device="cuda")),
        lambda: ops.softmax(x, mask=torch.ones((5, 8), dtype=torch.bool, device="cuda")),
        lambda: ops.softmax(x, mask=torch.ones((6, 1), dtype=torch.bool, device="cuda")),
        lambda: ops.softmax(x, mask=torch.ones((6, 8), dtype=torch.float64, device="cuda")),
        lambda: ops.softmax(x, mask=torch.ones((6, 8), dtype=torch.bool)),
        lambda: ops.softmax(x, out=x.half()), lambda: ops.softmax_backward(x, x, stats[:3]),
        lambda: ops.softmax_backward(x[:3], x, stats),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    one = torch.zeros((1, 8), device="cuda")
    for call in (lambda: ops.layer_norm(torch.zeros((2, 32769), device="cuda")), lambda: ops.layer_norm(x, eps=-1.0),
                 lambda: ops.dropout(x, d, out=one.expand(4, 6, 8)), lambda: ops.softmax(x, out=one.expand(4, 6, 8)),
                 lambda: ops.layer_norm(x, out=one.expand(4, 6, 8)),
                 lambda: ops.softmax(x, scale=float("nan"))):
        with pytest.raises(ckm.CkmError) as e:
            call()
        assert e.value.status in (ckm.E_INVALID_ARG, ckm.E_UNSUPPORTED)


# ---------------------------------------------------------------------------
# both sides of each launch rule, and the largest calls
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("cols", [9, 127, 128, 129, 255, 256, 257, 511, 512, 513, 1024, 1025, 2047, 2049, 4096, 4097, 8191,
                                  8193, 16383, 32761])
def test_layer_norm_at_its_launch_rules(cols):
    test_layer_norm_and_gradient("f16", "f32", 5, cols)
    test_layer_norm_and_gradient("f32", "f32", 2, cols)


@pytest.mark.parametrize("keys", [8, 9, 127, 129, 256, 257, 511, 513, 1024, 1025, 2047, 2049, 4096, 8191, 8193, 16385, 32767,
                                  32768, 32769, 34817])
@pytest.mark.parametrize("kind,causal,ragged", [("none", False, False), ("none", True, True), ("bool", True, False),
                                                ("add", False, True)])
def test_softmax_at_its_launch_rules(keys, kind, causal, ragged):
    test_softmax_and_gradient("f16", (2, 1, 3, keys), kind, causal, ragged)
    test_softmax_and_gradient("f32", (1, 2, 2, keys), kind, causal, ragged)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("keys", [13, 2000, 40000])
@pytest.mark.parametrize("scale", [-0.25, 0.0, 1e-30])
def test_softmax_other_scales(dtype, keys, scale):
    T = TYPES[dtype]
    x, dy = randn((3, keys), dtype, 31, gain=3.0), randn((3, keys), dtype, 32)
    y, stats = ops.softmax(x, scale)
    t = host(x) * scale
    p, m, z = nodes.softmax(t)
    # as in test_softmax_and_gradient: the logit, the difference, the factor, the last bit
    rel = 5 * U * np.abs(t) + 4 * U * np.abs(t - m[:, None]) + 8 * U
    d_p = p * (rel + (p * rel).sum(-1, keepdims=True) + 2 * U * np.abs(m)[:, None] + (DEPTH + 8) * U)
    check(y, p, d_p + 2.0 ** -126, T, "y")
    g = host(dy)
    s = (p * g).sum(-1, keepdims=True)
    d_s = (np.abs(p * g) * (2 * d_p / p + (DEPTH + 8) * U)).sum(-1, keepdims=True)
    tol = np.abs(scale) * (2 * d_p * np.abs(g - s) + p * (d_s + 6 * U * np.abs(g) + 6 * U * np.abs(s))) + 2.0 ** -120
    check(ops.softmax_backward(dy, x, stats, scale), nodes.softmax_backward(g, p, scale), tol, T, "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keys", [30, 3000, 40000])
def test_softmax_logits_near_the_range(dtype, keys):
    """Scores of 1e38 and more: the largest takes all, equal ones share, and gradients stay finite."""
    x = torch.full((4, keys), -3e38, dtype=TYPES[dtype], device="cuda")
    x[0, 7] = 3e38
    x[1, 3], x[1, 20] = 2e38, 2e38
    x[2] = 3e38
    x[3] = 0.0
    y, stats = ops.softmax(x, 1.1)
    assert y[0, 7] == 1 and y[0].float().sum() == 1 and y[1, 3] == 0.5 and y[1, 20] == 0.5
    for r in (2, 3):
        assert torch.allclose(y[r].float(), torch.full((keys,), 1.0 / keys, device="cuda"), rtol=2.0 ** -7)
    assert torch.isfinite(ops.softmax_backward(torch.ones_like(x), x, stats, 1.1)).all()


def test_more_rows_than_a_launch_has_blocks_in_one_dimension():
    rows = (1 << 24) + 37
    x = torch.ones((rows, 2), dtype=torch.float16, device="cuda")
    d = ops.Dropout(0.5, SEED, SITE)
    y, stats = ops.softmax(x, drop=d)
    want = 0.5 * np.where(nodes.draws(100, 2, SEED, SITE, row0=rows - 100) < d.keep, 65536.0 / d.keep, 0.0)
    assert np.array_equal(host(y[-100:]), want) and torch.all(stats[:, 1] == 0.5)
    assert torch.isfinite(ops.softmax_backward(x, x, stats, drop=d)).all()
    y, _, stats = ops.layer_norm(x)
    assert torch.all(y == 0) and torch.all(stats[:, 0] == 1)
    dx, _, dw, db = ops.layer_norm_backward(x, x, stats, wtype=torch.float32)
    assert torch.all(dw == 0)
    # a sum of ones, exact in 32 bits up to 2^24, then off by the roundings of its few largest partial sums
    assert torch.all((db - rows).abs() <= rows * 256 * U)


def test_largest_dropouts():
    d = ops.Dropout(0.25, SEED, SITE)
    scale = 65536.0 / d.keep
    rows = (1 << 28) + 1003
    y = ops.dropout(torch.ones((rows, 1), dtype=torch.float16, device="cuda"), d)
    u = nodes.draws(2000, 1, SEED, SITE, row0=rows - 2000)
    assert np.array_equal(host(y[-2000:]) > 0, u < d.keep) and float(y.max()) == float(torch.tensor(scale).half())
    del y
    cols = 1 << 30
    y = ops.dropout(torch.ones((1, cols), dtype=torch.float16, device="cuda"), d)
    u = nodes.draws(1, 800, SEED, SITE, group0=cols // 8 - 100)
    assert np.array_equal(host(y[:, -800:]) > 0, u < d.keep)
    with pytest.raises(ckm.CkmError):
        ops.dropout(y.expand(2, cols).reshape(1, 2 * cols)[:, :cols + 8], d)


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("shape,kw", [((3, 2, 40, 1), {}), ((2, 3, 5, 300), {"lengths": [1, 1]}), ((1, 1, 1, 50000), {"lengths": [1]}),
                                      ((1, 2, 1, 7), {"mask": True}), ((2, 1, 3, 1), {"scale": -0.7})])
def test_softmax_of_one_seen_key_is_one_and_its_gradient_zero(dtype, shape, kw):
    """A row that sees one key: probability 1 and gradient 0, exactly, whatever the score."""
    B, H, Q, K = shape
    scale = kw.get("scale", 0.0883883)
    args = dict(scale=scale)
    if "lengths" in kw:
        args["lengths"] = torch.tensor(kw["lengths"], dtype=torch.int32, device="cuda")
    if "mask" in kw:
        args["mask"] = torch.arange(K, device="cuda").expand(Q, K) == 0
    x, dy = randn(shape, dtype, 41, gain=20.0), randn(shape, dtype, 42)
    d = ops.Dropout(0.25, SEED, SITE)
    for drop in (None, d):
        y, stats = ops.softmax(x, drop=drop, **args)
        if drop is None:
            assert torch.all(y[..., 0] == 1) and torch.all(y[..., 1:] == 0)
        assert torch.all(stats[..., 1] == 1)
        assert torch.all(ops.softmax_backward(dy, x, stats, drop=drop, **args) == 0)
        # statistics from elsewhere, their maximum rounded to binary32 once
        other = torch.stack([(x[..., 0].float() * scale), torch.ones_like(x[..., 0], dtype=torch.float32)], -1)
        assert torch.all(ops.softmax_backward(dy, x, other, drop=drop, **args) == 0)


@pytest.mark.parametrize("rows,cols", [(1, 500), (16, 500), (64, 500), (65, 500), (4, 8000), (5, 8000), (256, 100), (257, 100)])
def test_layer_norm_gradient_of_few_rows(rows, cols):
    """Both sides of the rule that gives few rows to one block, which has no sums to join."""
    assert (ops.layer_norm_workspace(rows, cols) == 0) == (rows not in (65, 5, 257))
    test_layer_norm_and_gradient("bf16", "f32", rows, cols)


def test_arguments_made_on_the_current_stream_and_dropped_after_the_call():
    """A call on another stream reads what the current stream has yet to make, from memory that is not given out again
    before it has."""
    q = torch.cuda.Stream()
    d = ops.Dropout(0.1, SEED, SITE)
    x, s = randn((512, 1024), "f16", 51), randn((2, 3, 256, 512), "f16", 52)
    want = ops.layer_norm(x, residual=x * 2.0, drop=d)[0], ops.softmax(s, mask=s > 0.0)[0]
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(20_000_000)   # the current stream is busy for some milliseconds
        got = [ops.layer_norm(x, residual=x * 2.0, drop=d, stream=q)[0]]
        torch.cuda._sleep(20_000_000)
        got.append(ops.softmax(s, mask=s > 0.0, stream=q)[0])
        junk = [torch.zeros_like(x) for _ in range(4)] + [torch.zeros_like(s, dtype=torch.bool) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del junk


@pytest.mark.parametrize("dtype", sorted(TYPES))
@pytest.mark.parametrize("cols", [5, 64, 300, 2048, 8193, 20000])
@pytest.mark.parametrize("p", [0.25, 0.0])
def test_a_kept_zero_keeps_its_sign(dtype, cols, p):
    """The norm with a dropout and no residual before it: the bits of the two calls, zeros of both signs among them."""
    x = randn((6, cols), dtype, 81)
    x[0], x[1], x[2, ::2] = -0.0, 0.0, -0.0
    d = ops.Dropout(p, SEED, SITE)
    h = ops.dropout(x, d)
    y, _, stats = ops.layer_norm(h)
    for got, want in zip(ops.layer_norm(x, drop=d), (y, h, stats)):
        bits = torch.int16 if got.element_size() == 2 else torch.int32
        assert torch.equal(got.view(bits), want.view(bits))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("keys", [30, 3000, 40000])
@pytest.mark.parametrize("form", ["none", "bool", "add", "negative"])
def test_softmax_logits_past_the_range(dtype, keys, form):
    """A logit that binary32 cannot hold is an infinite score, in every kernel and in both directions: below the range
    it counts for nothing, above it the row is NaN."""
    T = TYPES[dtype]
    x = torch.full((4, keys), -3e38, dtype=T, device="cuda")   # row 0: all below
    x[1, 7] = 1.0                                              # all below but one
    x[2] = 0.0
    x[2, :2] = 3e38                                            # two above
    x[3, 5], x[3, 6] = 1e38, 1e38                              # in range, two alike
    scale, kw = 2.0, {}
    if form == "negative":
        x, scale = -x, -2.0
    if form == "bool":
        kw["mask"] = torch.ones((4, keys), dtype=torch.bool, device="cuda")
    if form == "add":
        kw["mask"] = torch.zeros((4, keys), dtype=T, device="cuda")
    y, stats = ops.softmax(x, scale, **kw)
    assert torch.all(y[0] == 0) and torch.all(stats[0] == 0)
    assert y[1, 7] == 1 and torch.all(y[1, :7] == 0) and torch.all(y[1, 8:] == 0)
    assert stats[1, 0] == 2 and stats[1, 1] == 1
    assert torch.isnan(y[2]).all() and stats[2, 0] == float("inf") and torch.isnan(stats[2, 1])
    assert y[3, 5] == 0.5 and y[3, 6] == 0.5 and y[3].float().sum() == 1
    dy = torch.linspace(-1, 1, 4 * keys, device="cuda").view(4, keys).to(T)
    dy[3, 5], dy[3, 6] = 1.0, -1.0
    dx = ops.softmax_backward(dy, x, stats, scale, **kw)
    assert torch.all(dx[:2] == 0) and torch.isnan(dx[2]).all()
    assert torch.all(dx[3, 7:] == 0) and dx[3, 5] == scale / 2 and dx[3, 6] == -scale / 2


def test_layer_norm_in_place_of_its_only_input_has_no_h():
    """y in the place of x, which would have been h: the call says that there is none, and the gradient refuses."""
    x, dy = randn((6, 48), "f16", 82), randn((6, 48), "f16", 83)
    for out in (x, x.view(6, 48)):
        y, h, stats = ops.layer_norm(x, out=out)
        assert y is out and h is None
        with pytest.raises((ValueError, ckm.CkmError)):
            ops.layer_norm_backward(dy, h, stats)
    r = randn((6, 48), "f16", 84)
    assert ops.layer_norm(x, residual=r, out=x)[1] is not None and ops.layer_norm(r, out=x)[1] is r
    empty = x[:0]
    assert ops.layer_norm(empty)[1] is empty and ops.layer_norm(empty, out=empty)[1] is empty


def test_a_dropout_whose_site_is_assigned_draws_another_mask():
    x = randn((16, 100), "f16", 85)
    d = ops.Dropout(0.5, SEED, SITE)
    first = ops.dropout(x, d)
    d.site += 1
    assert torch.equal(ops.dropout(x, d), ops.dropout(x, ops.Dropout(0.5, SEED, SITE + 1)))
    d.site, d.d_site = 3, torch.tensor([SITE - 3], device="cuda")
    assert torch.equal(ops.dropout(x, d), first)
    d.d_site, d.p = None, 0.0
    assert torch.equal(ops.dropout(x, d), x)


@pytest.mark.parametrize("rows,cols,at", [(4000, 30, 1), (4000, 30, 64), (300, 100, 1), (60000, 2, 64), (64, 1000, 1),
                                          (2048, 2048, 4), (2048, 30, 64)])
def test_weight_gradients_are_summed_in_trees(rows, cols, at):
    """One large term and many small ones, every `at`-th row: a chain of additions past the large one would lose them
    all. Depth: the rows of a thread (4 at most), trees over a block's rows (6) and over 32 slots of the blocks' sums
    (5) of 8 blocks each, and the result's rounding: 24."""
    dy = torch.zeros((rows, cols), device="cuda")
    dy[::at] = 1.0
    dy[0] = 2.0 ** 24
    h = torch.ones((rows, cols), device="cuda")
    stats = torch.tensor([0.0, 1.0], device="cuda").expand(rows, 2).contiguous()   # xh = 1: both sums are of dy
    _, _, dw, db = ops.layer_norm_backward(dy, h, stats)
    want = host(dy[:, 0]).sum()
    for got in (dw, db):
        assert np.all(np.abs(host(got) - want) <= 24 * U * want), (float(got[0]) - want)


@pytest.mark.parametrize("keys", [500, 3000, 40000])
@pytest.mark.parametrize("form", ["none", "bool", "add"])
def test_small_probabilities_in_binary32(keys, form):
    """exp(v) for v down to -80, with the largest logit 0 and the sum 1, is right to the exponential unit's last place
    (2 U), the correction's rounding (U) and the product with 1 / sum: 4 U; the rounding of v log2 e alone would be up
    to 2^-18, 64 U. The gradient adds a difference and two products."""
    rng = np.random.default_rng(keys)
    v = np.float32(rng.uniform(-80.0, -45.0, (3, keys)))
    v[:, keys // 3] = 0.0
    x = torch.from_numpy(v).cuda()
    kw = {}
    if form == "bool":
        kw["mask"] = torch.ones((3, keys), dtype=torch.bool, device="cuda")
    if form == "add":
        kw["mask"] = torch.zeros((3, keys), device="cuda")
    y, stats = ops.softmax(x, **kw)
    assert torch.all(stats[:, 0] == 0) and torch.all(stats[:, 1] == 1)
    want = np.exp(v.astype(np.float64))
    off = np.abs(host(y) - want) / want
    assert off.max() <= 4 * U, off.max() / U
    dy = torch.from_numpy(np.float32(rng.uniform(1.0, 2.0, (3, keys)))).cuda()
    dy[:, keys // 3] = 0.0
    dx = host(ops.softmax_backward(dy, x, stats, **kw))
    g = host(dy)
    full = want * (g - (want * g).sum(1, keepdims=True))
    seen = g > 0
    off = np.abs(dx - full)[seen] / np.abs(full)[seen]
    assert off.max() <= 8 * U, off.max() / U


@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("dtype,cols", [("f16", 16384), ("f32", 8199)])
def test_layer_norm_gradient_of_few_wide_rows(dtype, rows, cols):
    test_layer_norm_and_gradient(dtype, "f32", rows, cols)


# ---------------------------------------------------------------------------
# rows and keys past what a launch takes in one turn
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,wtype,rows,cols", [("f16", "f32", 2500, 2048), ("bf16", "bf16", 1100, 4104),
                                                   ("f16", "f16", 600, 16384), ("f32", "f32", 40000, 72),
                                                   ("f16", "f32", 300, 16392), ("bf16", "f32", 2100, 16392)])
def test_layer_norm_rows_past_one_turn(dtype, wtype, rows, cols):
    """More rows than a launch's blocks take at once: each block goes on to other rows, and the blocks' column sums are
    joined. DEPTH holds: a thread sums 9 rows at most."""
    test_layer_norm_and_gradient(dtype, wtype, rows, cols)


@pytest.mark.parametrize("dtype,shape", [("f16", (2, 150, 1, 50001)), ("f32", (1, 260, 1, 33001)), ("bf16", (1, 1, 1, 1100003))])
@pytest.mark.parametrize("kind,causal,ragged", [("none", False, True), ("bool", False, False), ("add", True, False)])
def test_softmax_shares_past_one_turn(dtype, shape, kind, causal, ragged):
    """Shares of more keys than a block holds at a time. DEPTH holds: a thread sums 80 keys in groups of 16 at most."""
    test_softmax_and_gradient(dtype, shape, kind, causal, ragged)


def test_rows_past_one_dimension_of_a_launch_by_value():
    """Every row its own: none skipped, none taken for another, at the start, around the launch's dimensions, the end."""
    rows, cols = (1 << 24) + 37, 3
    place = torch.arange(rows, device="cuda")
    x = torch.stack([((place * k) % 251).half() / 64 for k in (1, 5, 7)], -1)
    dy = torch.stack([((place * k) % 241).half() / 64 for k in (11, 13, 3)], -1)
    d = ops.Dropout(0.5, SEED, SITE)
    parts = [(0, 200), ((1 << 20) - 100, 200), ((1 << 24) - 100, 137)]

    def filled():
        return torch.full_like(x, float("nan"))

    y, stats = ops.softmax(x, drop=d, out=filled())
    dx = ops.softmax_backward(dy, x, stats, drop=d, out=filled())
    ny, _, nstats = ops.layer_norm(x, out=filled())
    ndx, _, dw, db = ops.layer_norm_backward(dy, x, nstats, wtype=torch.float32, out=filled())
    drop = ops.dropout(x, d, out=filled())
    for t in (y, stats, dx, ny, nstats, ndx, drop):
        assert torch.isfinite(t).all()
    for at, n in parts:
        f = np.where(nodes.draws(n, cols, SEED, SITE, row0=at) < d.keep, 65536.0 / d.keep, 0.0)
        hx, hg = host(x[at:at + n]), host(dy[at:at + n])
        p, m, z = nodes.softmax(hx)
        rel = 4 * U * np.abs(hx - m[:, None]) + 32 * U
        check(y[at:at + n], p * f, p * f * 3 * rel, torch.float16, "y")
        check(stats[at:at + n, 0], m, 0.0, torch.float32, "max")
        g = nodes.dropout(hg, f)
        tol = p * (np.abs(g) + np.abs(p * g).sum(1, keepdims=True)) * 8 * rel
        check(dx[at:at + n], nodes.softmax_backward(g, p, 1.0), tol, torch.float16, "dx")
        check(drop[at:at + n], nodes.dropout(hx, f), 0.0, torch.float16, "dropout")
        want, mean, rstd = nodes.layer_norm(hx, 1.0, 0.0, 1e-5)
        _, d_rstd, d_y = norm_bounds(hx, np.ones(cols), 1e-5)
        check(ny[at:at + n], want, d_y, torch.float16, "norm")
        check(nstats[at:at + n, 1], rstd, d_rstd * rstd, torch.float32, "rstd")
        hs = host(nstats[at:at + n])
        want, _, _ = nodes.layer_norm_backward(hg, hx, hs[:, 0], hs[:, 1], 1.0)
        xh = np.abs(hx - hs[:, :1]) * hs[:, 1:]
        tol = hs[:, 1:] * (DEPTH + 16) * U * (np.abs(hg) + np.abs(hg).mean(1, keepdims=True)
                                              + xh * (np.abs(hg) * xh).mean(1, keepdims=True))
        check(ndx[at:at + n], want, tol, torch.float16, "norm dx")
    # a thread sums 1025 rows, one after another
    g, xh = dy.double(), (x.double() - nstats[:, :1].double()) * nstats[:, 1:].double()
    depth = (1025 + DEPTH) * U
    check(dw, host((g * xh).sum(0)), depth * host((g * xh).abs().sum(0)), torch.float32, "dweight")
    check(db, host(g.sum(0)), depth * host(g.abs().sum(0)), torch.float32, "dbias")


# ---------------------------------------------------------------------------
# outputs in place of inputs, the caller's work buffers
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [(70, 40), (300, 1000), (9, 4096), (5, 12345), (300, 16400), (4, 30001)])
def test_layer_norm_in_place_of_its_inputs(dtype, rows, cols):
    x, r, dy = (randn((rows, cols), dtype, k, offset=1, pad=2) for k in (61, 62, 63))
    w, b = randn((cols,), dtype, 64, shift=1.0), randn((cols,), dtype, 65)
    d = ops.Dropout(0.25, SEED, SITE)
    y, h, stats = ops.layer_norm(x, w, b, residual=r, drop=d)
    for which in (0, 1):
        a = [x.clone(), r.clone()]
        got = ops.layer_norm(a[0], w, b, residual=a[1], drop=d, out=a[which])
        assert got[0] is a[which] and all(torch.equal(p, q) for p, q in zip(got, (y, h, stats)))
    a = x.clone()
    got = ops.layer_norm(a, w, b, out=a)
    want = ops.layer_norm(x, w, b)
    assert got[0] is a and torch.equal(a, want[0]) and torch.equal(got[2], want[2])
    want = ops.layer_norm_backward(dy, h, stats, w, dres=r, drop=d)
    for which in (0, 1, 2):
        a = [dy.clone(), h.clone(), r.clone()]
        got = ops.layer_norm_backward(a[0], a[1], stats, w, dres=a[2], drop=d, out=a[which])
        assert got[1] is a[which] and all(torch.equal(p, q) for p, q in zip(got, want))
    a = r.clone()
    assert ops.dropout(x, d, residual=a, out=a) is a and torch.equal(a, h)


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("keys", [13, 300, 2048, 20001, 40001])
@pytest.mark.parametrize("kind", ["none", "bool", "add"])
def test_softmax_gradient_in_place_of_the_scores(dtype, keys, kind):
    shape = (1, 2, 5, keys)
    x, dy = randn(shape, dtype, 66, gain=3.0, offset=1, pad=2), randn(shape, dtype, 67)
    mask, _ = masks(kind, shape, dtype, 68)
    d = ops.Dropout(0.25, SEED, SITE)
    kw = dict(scale=0.5, causal=True, mask=mask, drop=d)
    _, stats = ops.softmax(x, **kw)
    want = ops.softmax_backward(dy, x, stats, **kw)
    a = x.clone()
    assert ops.softmax_backward(dy, a, stats, out=a, **kw) is a and torch.equal(a, want)


def test_work_buffers_of_the_caller():
    """The bits of the calls that make their own, whatever the buffer held; one that is too small is refused."""
    d = ops.Dropout(0.25, SEED, SITE)

    def buffers(need):
        assert need > 0
        return [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (need, need + 4096)]

    for rows, cols in ((300, 1000), (5000, 40), (9, 20000)):
        h, dy = randn((rows, cols), "f16", 71), randn((rows, cols), "f16", 72)
        _, _, stats = ops.layer_norm(h)
        want = ops.layer_norm_backward(dy, h, stats, drop=d)
        need = ops.layer_norm_workspace(rows, cols)
        for work in buffers(need):
            got = ops.layer_norm_backward(dy, h, stats, drop=d, work=work)
            assert all(torch.equal(p, q) for p, q in zip(got, want))
        with pytest.raises(ckm.CkmError):
            ops.layer_norm_backward(dy, h, stats, drop=d, work=work[:need - 1])
    shape = (1, 2, 3, 40001)
    x, dy = randn(shape, "bf16", 73), randn(shape, "bf16", 74)
    want, stats = ops.softmax(x, drop=d)
    dx = ops.softmax_backward(dy, x, stats, drop=d)
    need = ops.softmax_workspace(*shape)
    for work in buffers(need):
        got = ops.softmax(x, drop=d, work=work)
        assert torch.equal(got[0], want) and torch.equal(got[1], stats)
        work.fill_(255)
        assert torch.equal(ops.softmax_backward(dy, x, stats, drop=d, work=work), dx)
    for call in (lambda w: ops.softmax(x, work=w), lambda w: ops.softmax_backward(dy, x, stats, work=w)):
        with pytest.raises(ckm.CkmError):
            call(work[:need - 1])
    work = torch.zeros(16, dtype=torch.uint8, device="cuda")   # not needed: any will do
    assert torch.equal(ops.softmax(x[..., :100], work=work)[0], ops.softmax(x[..., :100])[0])


def test_a_mask_of_one_key_is_refused_by_its_name():
    x = torch.zeros((2, 3, 5, 8), device="cuda")
    for shape in ((), (1,), (5, 1), (2, 1, 1, 1)):
        for dtype in (torch.bool, torch.float32):
            with pytest.raises(ValueError, match="mask must have each of the 8 keys"):
                ops.softmax(x, mask=torch.ones(shape, dtype=dtype, device="cuda"))
    for shape in ((8,), (1, 8), (5, 8), (2, 1, 1, 8), (1, 3, 5, 8)):
        assert torch.all(ops.softmax(x, mask=torch.ones(shape, dtype=torch.bool, device="cuda"))[0] == 0.125)
    one = x[..., :1]   # one key: any mask has it
    assert torch.all(ops.softmax(one, mask=torch.ones((5, 1), dtype=torch.bool, device="cuda"))[0] == 1)


def test_calls_on_another_stream_in_a_capture():
    """A captured call on another stream joins the capture; the caller joins back. Replays give the eager bits."""
    x, s = randn((300, 1000), "f16", 91), randn((1, 4, 60, 700), "f16", 92)
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = ops.Dropout(0.1, SEED, SITE, step)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        all_ops(x, s, d)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = all_ops(x, s, d, stream=other)
        torch.cuda.current_stream().wait_stream(other)
    for n in range(3):
        step.fill_(n)
        for t in got:
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = all_ops(x, s, ops.Dropout(0.1, SEED, SITE + n))
        assert all(torch.equal(p, q) for p, q in zip(got, want)), n
