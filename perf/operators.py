"""Timed cases of the training-node operators: dropout, layer norm and the attention softmax.

A case names one pass through an operator, forward or gradient, with its types
and sizes. The plain forms below are elementary tensor operations in 32 bits;
with `own` true the same passes go through the package's entry points.

  dropout           y = residual + D(x)  (residual optional)
  layer_norm        h = residual + D(x) rounded to the tensors' type (fused
                    cases; else h = x), y = (h - mean) rstd w + b
  layer_norm_backward   dh, dx = D(dh), dw, db from dy, h and the statistics
  softmax           probabilities of scale x + mask over the visible keys,
                    with dropout; rows that see nothing are zero
  softmax_backward  the scores' gradient, the probabilities made again from
                    the scores and the row statistics

D drops by a counter: element (row, col) takes 16-bit draw col % 8 of
Philox4x32-10 with key `seed` and counter (col / 8, row, site low, site high),
is kept iff the draw is below keep = floor((1 - p) 65536), and is then scaled
by 65536 / keep.

`pad` is the number of unused elements after each row of the inputs (a view of
a wider tensor). Widths, tokens and heads of the first cases are those of the
package's transformer workload (2048 tokens, width 2048, 16 heads, 16-bit
tensors).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-5
SITE = (5 << 32) | 11


def _rows(name, op, dtype, rows, cols, p=0.0, residual=False, wtype=None, pad=0):
    return dict(name=name, op=op, dtype=dtype, rows=rows, cols=cols, p=p, residual=residual, wtype=wtype or dtype,
                pad=pad)


def _scores(name, op, dtype, batch, heads, queries, keys, p=0.0, causal=False, lengths=False, mask="none", pad=0):
    return dict(name=name, op=op, dtype=dtype, batch=batch, heads=heads, queries=queries, keys=keys, p=p,
                causal=causal, lengths=lengths, mask=mask, pad=pad)


def listed():
    return [
        # a few tokens: what counts is the call itself
        _rows("dropout add f16 16x2048", "dropout", "f16", 16, 2048, p=0.1, residual=True),
        # the block's output dropout and residual sum
        _rows("dropout add f16 2048x2048", "dropout", "f16", 2048, 2048, p=0.1, residual=True),
        # single precision, odd sizes, a column range of a wider tensor
        _rows("dropout f32 5003x1537 strided", "dropout", "f32", 5003, 1537, p=0.25, pad=6),
        # the block's first layer norm
        _rows("layer norm f16 2048x2048", "layer_norm", "f16", 2048, 2048),
        # dropout, residual sum and norm of a wide model in one pass, 32-bit weights
        _rows("layer norm fused bf16 8192x8192", "layer_norm", "bf16", 8192, 8192, p=0.1, residual=True, wtype="f32"),
        # a small odd one in single precision
        _rows("layer norm f32 777x1023", "layer_norm", "f32", 777, 1023),
        # the first layer norm's gradient
        _rows("layer norm backward f16 2048x2048", "layer_norm_backward", "f16", 2048, 2048),
        # many tokens: the weights' gradients sum over all of them
        _rows("layer norm backward fused bf16 16384x4096", "layer_norm_backward", "bf16", 16384, 4096, p=0.1,
              residual=True, wtype="f32"),
        # the block's scale, mask, softmax and attention dropout
        _scores("softmax f16 16x2048x2048 causal", "softmax", "f16", 1, 16, 2048, 2048, p=0.1, causal=True),
        # single queries against ragged long contexts, no dropout
        _scores("softmax bf16 8x16x1x32768 ragged", "softmax", "bf16", 8, 16, 1, 32768, lengths=True),
        # their gradient
        _scores("softmax backward f16 16x2048x2048 causal", "softmax_backward", "f16", 1, 16, 2048, 2048, p=0.1,
                causal=True),
        # odd sizes, a truth-value mask that leaves rows empty
        _scores("softmax backward f32 3x12x509x777 bool", "softmax_backward", "f32", 3, 12, 509, 777, p=0.1,
                mask="bool"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over their logarithm, every type, mask and direction; at most the largest listed bytes."""
    most = max(work(c)["bytes"] for c in listed())
    while True:
        op = rng.choice(["dropout", "layer_norm", "layer_norm_backward", "softmax", "softmax_backward"])
        dtype = rng.choice(["f32", "f16", "bf16"])
        p = rng.choice([0.0, 0.1, 0.25, 0.5])
        pad = rng.choice([0, 0, 0, 1, 8])
        if op in ("softmax", "softmax_backward"):
            one = rng.random() < 0.3   # single queries, long contexts
            case = _scores("", op, dtype, _log(rng, 1, 16), _log(rng, 1, 32), 1 if one else _log(rng, 1, 4096),
                           _log(rng, 1, 262144 if one else 8192), p=p, causal=rng.random() < 0.5,
                           lengths=rng.random() < 0.4, mask=rng.choice(["none", "none", "bool", "add"]), pad=pad)
        else:
            norm = op != "dropout"
            case = _rows("", op, dtype, _log(rng, 1, 65536), _log(rng, 1, 16384), p=p if norm or p else 0.1,
                         residual=rng.random() < 0.5, wtype=rng.choice([dtype, "f32"]) if norm else dtype, pad=pad)
        if work(case)["bytes"] <= most:
            del case["name"]
            return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _randn(gen, shape, dtype, pad=0, gain=1.0):
    wide = torch.randn(shape[:-1] + (shape[-1] + pad,), generator=gen, device="cuda").mul_(gain).to(TYPES[dtype])
    return wide[..., :shape[-1]] if pad else wide


def _visible(case, lengths, mask, shape):
    """Truth values [batch, heads, queries, keys]: what each row sees."""
    B, H, Q, K = shape
    j = torch.arange(K, device="cuda")
    seen = torch.ones((1, 1, 1, K), dtype=torch.bool, device="cuda")
    if case["causal"]:
        i = torch.arange(Q, device="cuda")[:, None]
        seen = seen & (j <= i + (K - Q))
    if lengths is not None:
        seen = seen & (j < lengths.long().view(B, 1, 1, 1))
    if mask is not None:
        seen = seen & (mask if mask.dtype == torch.bool else mask > -math.inf)
    return seen.expand(B, H, Q, K)


def _logits(case, scores, lengths, mask, scale, wide):
    t = scores.to(wide) * scale
    if mask is not None and mask.dtype != torch.bool:
        t = t + mask.to(wide)
    return torch.where(_visible(case, lengths, mask, scores.shape), t, -math.inf)


def _softmax_stats(t):
    """Per row: the largest logit and 1 / sum of exponentials; (0, 0) where nothing is visible."""
    m = t.amax(-1)
    m = torch.where(m > -math.inf, m, 0.0)
    z = torch.exp(t - m[..., None]).sum(-1)
    return torch.stack([m, torch.where(z > 0, 1.0 / z, 0.0)], -1)


def _mask(case, gen):
    B, H, Q, K = (case[k] for k in ("batch", "heads", "queries", "keys"))
    if case["mask"] == "none":
        return None
    empty = torch.rand((Q, 1), generator=gen, device="cuda") < 1 / 32
    if case["mask"] == "bool":   # one for each sequence, for all its heads
        seen = torch.rand((B, 1, Q, K), generator=gen, device="cuda") < 0.8
        seen[..., 0] = True
        return seen & ~empty
    # one for each head, for all sequences: a bias that falls with the distance,
    # some keys at the type's lowest value, some at -inf, some rows with nothing
    i, j = torch.arange(Q, device="cuda")[:, None], torch.arange(K, device="cuda")
    slope = torch.exp2(-8.0 * (torch.arange(H, device="cuda")[:, None, None] + 1) / H)
    bias = -slope * (i + (K - Q) - j).abs()
    roll = torch.rand((H, Q, K), generator=gen, device="cuda")
    roll[..., 0] = 1.0
    bias = bias.to(TYPES[case["dtype"]])
    bias[roll < 0.1] = torch.finfo(bias.dtype).min
    bias[roll < 0.05] = -math.inf
    bias[empty.expand(Q, K).expand(H, Q, K)] = -math.inf
    return bias[None]


def prepare(case, seed):
    gen = _generator(seed)
    op, dtype, pad = case["op"], case["dtype"], case["pad"]
    st = dict(case=case, seed=(int(seed) * 0x9E3779B97F4A7C15) & 0x7FFFFFFFFFFFFFFF)
    if op in ("softmax", "softmax_backward"):
        B, H, Q, K = shape = tuple(case[k] for k in ("batch", "heads", "queries", "keys"))
        st["scale"] = 128 ** -0.5
        st["scores"] = _randn(gen, shape, dtype, pad, gain=12.0)
        st["lengths"] = None
        if case["lengths"]:
            st["lengths"] = torch.randint(0, K + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        st["mask"] = _mask(case, gen)
        if op == "softmax_backward":
            st["stats"] = _softmax_stats(_logits(case, st["scores"], st["lengths"], st["mask"], st["scale"],
                                                 torch.float32))
            st["dy"] = _randn(gen, shape, dtype, pad)
        return st
    shape = (case["rows"], case["cols"])
    st["x"] = _randn(gen, shape, dtype, pad, gain=1.5)
    st["residual"] = _randn(gen, shape, dtype, pad) if case["residual"] else None
    if op != "dropout":
        st["w"] = (1.0 + 0.1 * torch.randn(shape[1], generator=gen, device="cuda")).to(TYPES[case["wtype"]])
        st["b"] = (0.1 * torch.randn(shape[1], generator=gen, device="cuda")).to(TYPES[case["wtype"]])
    if op == "layer_norm_backward":
        st["dy"] = _randn(gen, shape, dtype, pad)
        st["stats"] = _norm_stats(st["x"].float())
    return st


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _kept(rows, cols, seed, keep):
    """Truth values [rows, cols] of the counter-based generator."""
    low = 0xFFFFFFFF
    groups = (cols + 7) // 8
    c0 = torch.arange(groups, device="cuda").expand(rows, groups)
    c1 = torch.arange(rows, device="cuda")[:, None].expand(rows, groups)
    c2, c3 = torch.full_like(c0, SITE & low), torch.full_like(c0, SITE >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57   # the low 64 bits; the shifts below take their upper half
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    u = torch.stack([c0, c0 >> 16, c1, c1 >> 16, c2, c2 >> 16, c3, c3 >> 16], -1) & 0xFFFF
    return (u < keep).reshape(rows, 8 * groups)[:, :cols]


def _drop(x, p, seed):
    """D of a 32-bit tensor, rows by its last dimension."""
    keep = math.floor((1.0 - p) * 65536.0)
    kept = _kept(x[..., 0].numel(), x.shape[-1], seed, keep).view(x.shape)
    return torch.where(kept, x * (65536.0 / keep), 0.0)


def _norm_stats(h):
    mean = h.mean(-1)
    var = (h - mean[:, None]).square().mean(-1)
    return torch.stack([mean, torch.rsqrt(var + EPS)], -1)


def _plain(st):
    case = st["case"]
    op, dtype, p, seed = case["op"], TYPES[case["dtype"]], case["p"], st["seed"]
    if op in ("softmax", "softmax_backward"):
        t = _logits(case, st["scores"], st["lengths"], st["mask"], st["scale"], torch.float32)
        stats = st["stats"] if op == "softmax_backward" else _softmax_stats(t)
        prob = torch.exp(t - stats[..., :1]) * stats[..., 1:]
        if op == "softmax":
            return [(_drop(prob, p, seed) if p else prob).to(dtype), stats]
        g = st["dy"].float()
        g = _drop(g, p, seed) if p else g
        return [(st["scale"] * prob * (g - (prob * g).sum(-1, keepdim=True))).to(dtype)]
    x = st["x"].float()
    if op == "dropout":
        y = _drop(x, p, seed)
        return [(y if st["residual"] is None else st["residual"].float() + y).to(dtype)]
    w = st["w"].float()
    if op == "layer_norm":
        h = _drop(x, p, seed) if p else x
        h = (h if st["residual"] is None else st["residual"].float() + h).to(dtype)
        wide = h.float()
        stats = _norm_stats(wide)
        y = ((wide - stats[:, :1]) * stats[:, 1:] * w + st["b"].float()).to(dtype)
        return [y, h, stats] if p or case["residual"] else [y, stats]
    # here x is the norm's input h and residual the gradient that reaches h past the norm
    dy, mean, rstd = st["dy"].float(), st["stats"][:, :1], st["stats"][:, 1:]
    xh = (x - mean) * rstd
    g = dy * w
    dh = rstd * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    dh = (dh if st["residual"] is None else dh + st["residual"].float()).to(dtype)
    dw, db = (dy * xh).sum(0).to(st["w"].dtype), dy.sum(0).to(st["w"].dtype)
    return [dh, _drop(dh.float(), p, seed).to(dtype), dw, db] if p else [dh, dw, db]


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------

def _own(st):
    from paper_1910_02653_amd import ops

    case = st["case"]
    op = case["op"]
    drop = ops.Dropout(case["p"], st["seed"], SITE) if case["p"] else None
    if op == "softmax":
        return list(ops.softmax(st["scores"], st["scale"], causal=case["causal"], lengths=st["lengths"],
                                mask=st["mask"], drop=drop))
    if op == "softmax_backward":
        return [ops.softmax_backward(st["dy"], st["scores"], st["stats"], st["scale"], causal=case["causal"],
                                     lengths=st["lengths"], mask=st["mask"], drop=drop)]
    if op == "dropout":
        return [ops.dropout(st["x"], drop, residual=st["residual"])]
    if op == "layer_norm":
        y, h, stats = ops.layer_norm(st["x"], st["w"], st["b"], eps=EPS, residual=st["residual"], drop=drop)
        return [y, h, stats] if case["p"] or case["residual"] else [y, stats]
    dx, dh, dw, db = ops.layer_norm_backward(st["dy"], st["x"], st["stats"], st["w"], dres=st["residual"], drop=drop)
    return [dh, dx, dw, db] if case["p"] else [dh, dw, db]


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    """Each input and output once (scores and their gradients: where a row sees them; ragged lengths: their mean), and
    the arithmetic of the formulas with about eight integer operations an element for the draws."""
    e = 4 if case["dtype"] == "f32" else 2
    drawn = 8 if case["p"] else 0
    if case["op"] in ("softmax", "softmax_backward"):
        B, H, Q, K = (case[k] for k in ("batch", "heads", "queries", "keys"))
        full = Q * K
        if case["causal"]:
            first = max(0, Q - K)   # rows before it see nothing, then one key more for each
            n = Q - first
            full = n * (K - Q + first) + n * (n + 1) // 2
        seen = full // 2 if case["lengths"] else full
        back = case["op"] == "softmax_backward"
        mask = {"none": 0, "bool": B * seen, "add": H * seen * e}[case["mask"]]
        return dict(bytes=B * H * (seen * e * (2 if back else 1) + Q * K * e + 8 * Q) + mask + (4 * B if case["lengths"] else 0),
                    flops=B * H * seen * ((9 if back else 7) + drawn))
    E, we = case["rows"] * case["cols"], 4 if case["wtype"] == "f32" else 2
    res = 1 if case["residual"] else 0
    if case["op"] == "dropout":
        return dict(bytes=E * e * (2 + res), flops=E * (1 + res + drawn))
    if case["op"] == "layer_norm":
        fused = 1 if case["residual"] or case["p"] else 0
        return dict(bytes=E * e * (2 + res + fused) + 8 * case["rows"] + 2 * case["cols"] * we, flops=E * (8 + res + drawn))
    return dict(bytes=E * e * (3 + res + (1 if case["p"] else 0)) + 8 * case["rows"] + 3 * case["cols"] * we,
                flops=E * (14 + res + drawn))


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_keep(shape, seed, p):
    """Scale factors [shape] in 64 bits: 0 where dropped. The 32 x 32 bit products from 16-bit parts."""
    rows, cols = math.prod(shape[:-1]), shape[-1]
    keep = math.floor((1.0 - p) * 65536.0)
    cnt = (cols + 7) // 8

    def product(c, const):   # (high, low) 32 bits
        t = c * (const & 0xFFFF)
        u = c * (const >> 16) + (t >> 16)
        return u >> 16, ((u & 0xFFFF) << 16) | (t & 0xFFFF)

    at = torch.arange(rows * cnt, device="cuda")
    w = [at % cnt, at // cnt, torch.zeros_like(at) + SITE % (1 << 32), torch.zeros_like(at) + SITE // (1 << 32)]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for _ in range(10):
        hi0, lo0 = product(w[0], 0xD2511F53)
        hi1, lo1 = product(w[2], 0xCD9E8D57)
        w = [hi1.bitwise_xor(w[1]).bitwise_xor(key[0]), lo1, hi0.bitwise_xor(w[3]).bitwise_xor(key[1]), lo0]
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    f = torch.zeros((rows * cnt, 8), dtype=torch.float64, device="cuda")
    for n in range(8):
        half = w[n // 2] // 65536 if n % 2 else w[n // 2] % 65536
        f[:, n] = (half < keep).double() * (65536 / keep)
    return f.view(rows, 8 * cnt)[:, :cols].reshape(shape)


def exact(case, seed):
    st = prepare(case, seed)
    op, p = case["op"], case["p"]
    key = "scores" if op in ("softmax", "softmax_backward") else "x"
    x = st[key].double()
    f = _exact_keep(x.shape, st["seed"], p) if p else 1.0
    if key == "scores":
        B, H, Q, K = x.shape
        t = x * st["scale"]
        if case["mask"] == "add":
            t += st["mask"].double()
        if case["mask"] == "bool":
            t.masked_fill_(~st["mask"], -math.inf)
        if case["causal"]:
            t.masked_fill_(torch.ones((Q, K), dtype=torch.bool, device="cuda").triu_(K - Q + 1), -math.inf)
        if case["lengths"]:
            t.masked_fill_((torch.arange(K, device="cuda")[None] >= st["lengths"][:, None])[:, None, None], -math.inf)
        if op == "softmax":
            m = t.max(-1, keepdim=True).values
            m[m == -math.inf] = 0.0
            prob = (t - m).exp_()
            z = prob.sum(-1, keepdim=True)
            z[z > 0] = 1.0 / z[z > 0]
            prob *= z
            return [prob * f, torch.cat([m, z], -1)]
        prob = (t - st["stats"][..., :1].double()).exp_() * st["stats"][..., 1:].double()
        g = st["dy"].double() * f
        return [prob * (g - (prob * g).sum(-1, keepdim=True)) * st["scale"]]
    r = 0.0 if st["residual"] is None else st["residual"].double()
    if op == "dropout":
        return [x * f + r]
    w, b, n = st["w"].double(), st["b"].double(), x.shape[1]
    if op == "layer_norm":
        h = (x * f + r).to(TYPES[case["dtype"]]).double()
        centred = h - h.sum(1, keepdim=True) / n
        rstd = (centred.pow(2).sum(1, keepdim=True) / n + EPS).pow(-0.5)
        stats = torch.cat([h.sum(1, keepdim=True) / n, rstd], 1)
        y = centred * rstd * w + b
        return [y, h, stats] if p or case["residual"] else [y, stats]
    dy, s = st["dy"].double(), st["stats"].double()
    xh = (x - s[:, :1]) * s[:, 1:]
    g = dy * w
    dh = (g - g.sum(1, keepdim=True) / n - xh * ((g * xh).sum(1, keepdim=True) / n)) * s[:, 1:] + r
    dw, db = (dy * xh).sum(0), dy.sum(0)
    if p:
        return [dh, dh.to(TYPES[case["dtype"]]).double() * f, dw, db]
    return [dh, dw, db]
