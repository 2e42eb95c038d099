"""The layer operators of a feed-forward block in training and serving, as cases that can be timed and compared.

    linear     y = r + s drop(act(x W^T + b)), and its gradients
    gated      h = act(x Wg^T + bg) * (x Wu^T + bu), and its gradients
    norm       r' = r + s g * P(b), y = N(r'), P and N norms over a row, and its gradients
    dropout    y = r + s drop(x), and its gradient

drop(v) keeps element i of the dense (rows, columns) matrix, divided by the probability with which it is kept, unless
half-word i % 8 of Philox4x32-7 (counter i // 8 and the call's offset, key the call's seed) is below round(65536 p).

A case is one call.  ``own`` says which side runs: the plain form in elementary torch operations, computed in 32 bits, or the
package's kernels.  ``pad`` is what a row's stride has beyond its length.
"""
from __future__ import annotations

import math

import torch

own = False

_TORCH = {"fp16": torch.float16, "bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"fp16": 2, "bf16": 2, "fp32": 4}
_MOST_FLOPS = 2 * 8192 * 4096 * 10240   # of a drawn product in 16 bits; a quarter of it in 32
_MOST_CELLS = 16384 * 4096              # of a drawn row-wise case


def _linear(name, direction, dtype, rows, k, n, **kw):
    c = dict(op="linear", direction=direction, dtype=dtype, rows=rows, k=k, n=n, act="none", bias=True, residual=False, scale=1.0,
             p=0.0, pad=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _gated(name, direction, dtype, rows, k, n, **kw):
    c = dict(op="gated", direction=direction, dtype=dtype, rows=rows, k=k, n=n, act="silu", bias=False, save=True, pad=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _norm(name, direction, dtype, rows, n, **kw):
    c = dict(op="norm", direction=direction, dtype=dtype, rows=rows, n=n, kind="rms", post=True, gate=0, scale=1.0, weights="fp32",
             pad=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def _dropout(name, direction, dtype, rows, n, **kw):
    c = dict(op="dropout", direction=direction, dtype=dtype, rows=rows, n=n, p=0.1, residual=False, scale=1.0, pad=0)
    c.update(kw)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token served: the projection back to the model's width, added to the residual stream
        _linear("linear_token_bf16", "forward", "bf16", 1, 10240, 4096, bias=False, residual=True),
        # the first layer of the 784-128-10 perceptron, a batch of 96, parameters still stored in 32 bits
        _linear("linear_mlp_fp32", "forward", "fp32", 96, 784, 128, act="gelu"),
        # the projection back to the model's width in training, with dropout and a residual scale in its epilogue
        _linear("linear_train_bf16", "forward", "bf16", 8192, 10240, 4096, residual=True, scale=0.5, p=0.1),
        # an odd layer kept in 32 bits by the precision rule: rows, inputs and outputs that divide by nothing
        _linear("linear_grad_odd_fp32", "backward", "fp32", 1003, 777, 1531, act="gelu"),
        # four sequences served, one token each
        _gated("gated_tokens_fp16", "forward", "fp16", 4, 4096, 10240, save=False),
        # a large training batch: the heaviest product of a block
        _gated("gated_train_bf16", "forward", "bf16", 8192, 4096, 10240),
        # gradients of a gated block, with biases, in scaled 16-bit floats; a ragged number of rows
        _gated("gated_grad_fp16", "backward", "fp16", 4099, 2048, 5464, bias=True),
        # one token served: norm after the block, gate per channel, norm before the next
        _norm("norm_token_bf16", "forward", "bf16", 1, 4096, gate=-1),
        # a large training batch
        _norm("norm_train_bf16", "forward", "bf16", 16384, 4096, gate=-1, scale=0.7),
        # gradients with a gate per sequence of 2048 rows, centred norms, in all five of them
        _norm("norm_grad_bf16", "backward", "bf16", 8192, 4096, kind="layer", gate=2048),
        # a large training batch's block output, dropped out and added to the stream
        _dropout("dropout_train_bf16", "forward", "bf16", 16384, 4096, residual=True),
        # the gradient through a dropout of an odd shape whose rows lie apart
        _dropout("dropout_grad_odd_fp32", "backward", "fp32", 1537, 1023, p=0.25, pad=5),
    ]


def _size(rng, low, high):
    v = int(math.exp(rng.uniform(math.log(low), math.log(high + 1))))
    to = rng.choice((1, 1, 8, 64, 64, 64))
    v = max(low, min(high, v))
    v = max(low, v - v % to) if v >= to else v
    return v + 1 if v == 3072 else v


def draw(rng):
    op = rng.choice(("linear", "linear", "gated", "norm", "dropout"))
    direction, dtype = rng.choice(("forward", "backward")), rng.choice(("bf16", "bf16", "fp16", "fp32"))
    pad = rng.choice((0, 0, 0, 8, 5))
    if op in ("linear", "gated"):
        most = _MOST_FLOPS // (4 if dtype == "fp32" else 1) // (2 if op == "gated" else 1) // (2 if direction == "backward" else 1)
        while True:
            rows, k, n = _size(rng, 1, 8192), _size(rng, 16, 10240), _size(rng, 16, 10240)
            if 2 * rows * k * n <= most:
                break
        act = rng.choice(("relu", "silu", "gelu", "gelu_tanh"))
        if op == "gated":
            return _gated(None, direction, dtype, rows, k, n, act=act, bias=rng.random() < 0.5, save=rng.random() < 0.7, pad=pad)
        return _linear(None, direction, dtype, rows, k, n, act=rng.choice((act, "none")), bias=rng.random() < 0.7,
                       residual=rng.random() < 0.5, scale=rng.choice((1.0, 0.5)), p=rng.choice((0.0, 0.0, 0.1, 0.25)), pad=pad)
    while True:
        rows, n = _size(rng, 1, 16384), _size(rng, 16, 16384)
        if rows * n * (_BYTES[dtype] // 2) * (2 if direction == "backward" else 1) <= _MOST_CELLS:
            break
    if op == "dropout":
        return _dropout(None, direction, dtype, rows, n, p=rng.choice((0.05, 0.1, 0.5)), residual=rng.random() < 0.5,
                        scale=rng.choice((1.0, 0.5)), pad=pad)
    return _norm(None, direction, dtype, rows, n, kind=rng.choice(("rms", "layer")), post=rng.random() < 0.6,
                 gate=rng.choice((0, -1, -1, max(1, rows // 3))), scale=rng.choice((1.0, 0.7)),
                 weights=rng.choice(("fp32", dtype)), pad=pad)


def _randn(gen, rows, n, dtype, pad=0, scale=1.0):
    """A matrix of normal numbers whose rows are ``n + pad`` elements apart."""
    t = torch.empty(rows, n + pad, dtype=_TORCH[dtype], device=gen.device)
    t.copy_(torch.randn(rows, n + pad, generator=gen, device=gen.device).mul_(scale))
    return t[:, :n]


def _vec(gen, n, dtype, mean=0.0, scale=0.1):
    return (torch.randn(n, generator=gen, device=gen.device) * scale + mean).to(_TORCH[dtype])


def prepare(case, seed):
    c, gen = case, torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case=c, seed=int(seed) * 0x9E3779B97F4A7C15 % (1 << 63), offset=(1 << 33) + 7)
    dt, rows, n, pad, back = c["dtype"], c["rows"], c["n"], c["pad"], c["direction"] == "backward"
    if c["op"] == "linear":
        k = c["k"]
        s["x"] = _randn(gen, rows, k, dt, pad)
        s["w"] = _randn(gen, n, k, dt, scale=k ** -0.5)
        s["b"] = _vec(gen, n, dt) if c["bias"] else None
        s["r"] = _randn(gen, rows, n, dt, pad) if c["residual"] and not back else None
        if back:
            s["dy"] = _randn(gen, rows, n, dt, pad, 0.1)
            s["pre"] = _randn(gen, rows, n, dt) if c["act"] != "none" else None
    elif c["op"] == "gated":
        k = c["k"]
        s["x"] = _randn(gen, rows, k, dt, pad)
        s["wg"], s["wu"] = _randn(gen, n, k, dt, scale=k ** -0.5), _randn(gen, n, k, dt, scale=k ** -0.5)
        s["bg"], s["bu"] = (_vec(gen, n, dt), _vec(gen, n, dt)) if c["bias"] else (None, None)
        if back:
            s["dh"] = _randn(gen, rows, n, dt, pad, 0.1)
            s["g"], s["u"] = _randn(gen, rows, n, dt), _randn(gen, rows, n, dt)
    elif c["op"] == "norm":
        centred, w = c["kind"] == "layer", c["weights"]
        s["r"] = _randn(gen, rows, n, dt, pad, 2.0)
        s["b"] = _randn(gen, rows, n, dt, pad)
        s["gate"] = None if c["gate"] == 0 else _vec(gen, n, w, 0.5) if c["gate"] < 0 else _randn(gen, -(-rows // c["gate"]), n, w)
        s["pw"], s["pb"] = (_vec(gen, n, w, 1.0), _vec(gen, n, w) if centred else None) if c["post"] else (None, None)
        s["nw"], s["nb"] = _vec(gen, n, w, 1.0), _vec(gen, n, w) if centred else None
        if back:
            s["dr"], s["dy"] = _randn(gen, rows, n, dt, pad, 0.1), _randn(gen, rows, n, dt, pad, 0.1)
    else:
        s["x"] = _randn(gen, rows, n, dt, pad)
        s["r"] = _randn(gen, rows, n, dt, pad) if c["residual"] and not back else None
    return s


def work(case):
    c = case
    w, rows, n, back = _BYTES[c["dtype"]], c["rows"], c["n"], c["direction"] == "backward"
    cells = rows * n
    if c["op"] in ("linear", "gated"):
        k, mats = c["k"], 2 if c["op"] == "gated" else 1
        vectors = mats * n if c["bias"] else 0
        ins, weights = rows * k, mats * n * k
        if not back:
            kept = mats * cells if (c.get("save") or (c["op"] == "linear" and c["act"] != "none")) else 0
            elements = ins + weights + vectors + cells + kept + (cells if c.get("residual") else 0)
            return dict(bytes=w * elements, flops=2 * rows * k * n * mats)
        saved = mats * cells if c["op"] == "gated" or c["act"] != "none" else 0
        return dict(bytes=w * (2 * ins + 2 * weights + cells + saved) + 4 * vectors, flops=4 * rows * k * n * mats)
    if c["op"] == "norm":
        vectors = n * ((2 if c["post"] else 0) + 2) + (0 if c["gate"] == 0 else n if c["gate"] < 0 else n * -(-rows // c["gate"]))
        if back:   # reads both gradients, the stream and the block's output, writes two gradients
            return dict(bytes=6 * w * cells + vectors * (_BYTES[c["weights"]] + 4), flops=30 * cells)
        return dict(bytes=4 * w * cells + vectors * _BYTES[c["weights"]], flops=12 * cells)
    return dict(bytes=w * cells * (3 if c["residual"] and not back else 2), flops=4 * cells)


# ---- the plain form ------------------------------------------------------------------------------------------------------------


def _act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))


def _slope(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        t = 1 / (1 + torch.exp(-z))
        return t * (1 + z * (1 - t))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def _low_high(a, b):
    """The low and high 32 bits of the product of two 32-bit numbers, as int64."""
    v = a * b
    return v & 0xFFFFFFFF, (v >> 32) & 0xFFFFFFFF


def _kept(rows, n, p, seed, offset, device):
    """The dropout mask (rows, n) and what a kept element is multiplied by."""
    limit = min(65535, round(p * 65536))
    i = torch.arange((rows * n + 7) // 8, dtype=torch.int64, device=device)
    a, b = i & 0xFFFFFFFF, i >> 32
    c, d = torch.full_like(i, offset & 0xFFFFFFFF), torch.full_like(i, offset >> 32)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(7):
        (l0, h0), (l1, h1) = _low_high(a, 0xD2511F53), _low_high(c, 0xCD9E8D57)
        a, b, c, d = h1 ^ b ^ k0, l1, h0 ^ d ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    halves = torch.stack([v for w in (a, b, c, d) for v in (w & 0xFFFF, w >> 16)], dim=1).reshape(-1)
    return (halves[: rows * n] >= limit).reshape(rows, n), 65536 / (65536 - limit)


def _dropped(v, s, p, scale):
    if p > 0:
        keep, up = _kept(v.shape[0], v.shape[1], p, s["seed"], s["offset"], v.device)
        return torch.where(keep, v * (scale * up), torch.zeros_like(v))
    return v * scale


def _stats(x, kind):
    mean = x.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    d = x - mean
    return d * torch.rsqrt((d * d).mean(dim=1, keepdim=True) + 1e-6), torch.rsqrt((d * d).mean(dim=1, keepdim=True) + 1e-6)


def _affine(t, w, b):
    t = t * w.float()
    return t if b is None else t + b.float()


def _norm_grad(dn, t, rstd, kind):
    centre = dn.mean(dim=1, keepdim=True) if kind == "layer" else 0.0
    return rstd * (dn - centre - t * (dn * t).mean(dim=1, keepdim=True))


def _gate_rows(gate, c):
    if c["gate"] < 0:
        return gate.float()
    return gate.float().repeat_interleave(c["gate"], dim=0)[: c["rows"]]


def _plain_norm(s):
    c, dt = s["case"], s["r"].dtype
    r, b, kind = s["r"].float(), s["b"].float(), c["kind"]
    gate = 1.0 if c["gate"] == 0 else _gate_rows(s["gate"], c)
    bt, brstd = _stats(b, kind) if c["post"] else (b, None)
    t = _affine(bt, s["pw"], s["pb"]) if c["post"] else b
    if c["direction"] == "forward":
        r = r + c["scale"] * gate * t
        return dict(residual=r.to(dt), y=_affine(_stats(r, kind)[0], s["nw"], s["nb"]).to(dt))
    dy, out = s["dy"].float(), {}
    rt, rrstd = _stats(r, kind)
    out["norm_weight"] = (dy * rt).sum(dim=0)
    if kind == "layer":
        out["norm_bias"] = dy.sum(dim=0)
    d = s["dr"].float() + _norm_grad(dy * s["nw"].float(), rt, rrstd, kind)
    out["residual"] = d.to(dt)
    if c["gate"]:
        dg = c["scale"] * d * t
        if c["gate"] < 0:
            out["gate"] = dg.sum(dim=0)
        else:
            group = torch.arange(c["rows"], device=d.device) // c["gate"]
            out["gate"] = torch.zeros(s["gate"].shape, device=d.device).index_add_(0, group, dg)
    dt_ = c["scale"] * gate * d
    if c["post"]:
        out["post_weight"] = (dt_ * bt).sum(dim=0)
        if kind == "layer":
            out["post_bias"] = dt_.sum(dim=0)
        dt_ = _norm_grad(dt_ * s["pw"].float(), bt, brstd, kind)
    out["block"] = dt_.to(dt)
    return out


def _plain(s):
    c, out = s["case"], {}
    back = c["direction"] == "backward"
    if c["op"] == "norm":
        return _plain_norm(s)
    if c["op"] == "dropout":
        v = _dropped(s["x"].float(), s, c["p"], c["scale"])
        return dict(y=(v if s["r"] is None else v + s["r"].float()).to(s["x"].dtype))
    x, dt = s["x"].float(), s["x"].dtype
    if c["op"] == "linear":
        w = s["w"].float()
        if not back:
            z = x @ w.T
            z = z if s["b"] is None else z + s["b"].float()
            v = _dropped(_act(c["act"], z), s, c["p"], c["scale"])
            out["y"] = (v if s["r"] is None else v + s["r"].float()).to(dt)
            if c["act"] != "none":
                out["pre"] = z.to(dt)
            return out
        dz = _dropped(s["dy"].float(), s, c["p"], c["scale"])
        dz = dz if c["act"] == "none" else dz * _slope(c["act"], s["pre"].float())
        out["x"], out["weight"] = (dz @ w).to(dt), (dz.T @ x).to(dt)
        if c["bias"]:
            out["bias"] = dz.sum(dim=0)
        return out
    wg, wu = s["wg"].float(), s["wu"].float()
    if not back:
        g, u = x @ wg.T, x @ wu.T
        g, u = (g, u) if s["bg"] is None else (g + s["bg"].float(), u + s["bu"].float())
        out["h"] = (_act(c["act"], g) * u).to(dt)
        if c["save"]:
            out["gate"], out["up"] = g.to(dt), u.to(dt)
        return out
    dh, g, u = s["dh"].float(), s["g"].float(), s["u"].float()
    dg, du = dh * u * _slope(c["act"], g), dh * _act(c["act"], g)
    out["x"] = (dg @ wg + du @ wu).to(dt)
    out["gate_weight"], out["up_weight"] = (dg.T @ x).to(dt), (du.T @ x).to(dt)
    if c["bias"]:
        out["gate_bias"], out["up_bias"] = dg.sum(dim=0), du.sum(dim=0)
    return out


# ---- the package's kernels -----------------------------------------------------------------------------------------------------


def _kernels(s):
    import paper_2508_16905_amd as ta

    c = s["case"]
    back = c["direction"] == "backward"
    if c["op"] == "dropout":
        drop = ta.Dropout(c["p"], s["seed"], s["offset"])
        if back:
            return dict(y=ta.dropout_backward(s["x"], drop, scale=c["scale"]))
        return dict(y=ta.dropout(s["x"], drop, residual=s["r"], scale=c["scale"]))
    if c["op"] == "linear":
        drop = ta.Dropout(c["p"], s["seed"], s["offset"]) if c["p"] > 0 else None
        if not back:
            got = ta.linear(s["x"], s["w"], s["b"], residual=s["r"], act=c["act"], scale=c["scale"], dropout=drop, save=c["act"] != "none")
            return dict(y=got) if c["act"] == "none" else dict(y=got[0], pre=got[1])
        dx, dw, db = ta.linear_backward(s["dy"], s["x"], s["w"], s["pre"], act=c["act"], scale=c["scale"], dropout=drop, bias_grad=c["bias"])
        return dict(x=dx, weight=dw, **(dict(bias=db) if c["bias"] else {}))
    if c["op"] == "gated":
        if not back:
            got = ta.gated(s["x"], s["wg"], s["wu"], s["bg"], s["bu"], act=c["act"], save=c["save"])
            return dict(h=got[0], gate=got[1], up=got[2]) if c["save"] else dict(h=got)
        dx, dwg, dwu, dbg, dbu = ta.gated_backward(s["dh"], s["x"], s["wg"], s["wu"], s["g"], s["u"], act=c["act"], bias_grad=c["bias"])
        return dict(x=dx, gate_weight=dwg, up_weight=dwu, **(dict(gate_bias=dbg, up_bias=dbu) if c["bias"] else {}))
    post = ta.Norm(c["kind"], s["pw"], s["pb"], 1e-6) if c["post"] else None
    norm = ta.Norm(c["kind"], s["nw"], s["nb"], 1e-6)
    rows_per_gate = max(0, c["gate"])
    if not back:
        r, y = ta.residual_norm(s["r"], s["b"], gate=s["gate"], rows_per_gate=rows_per_gate, post=post, norm=norm, scale=c["scale"])
        return dict(residual=r, y=y)
    g = ta.residual_norm_backward(s["dr"], s["dy"], s["r"], s["b"], gate=s["gate"], rows_per_gate=rows_per_gate, post=post, norm=norm,
                                  scale=c["scale"])
    return {k: v for k, v in g._asdict().items() if v is not None}


def run(state):
    return _kernels(state) if own else _plain(state)


# ---- the definition in 64 bits -------------------------------------------------------------------------------------------------


def _normal_cdf(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))


def _value_and_slope(name, z):
    """act(z) and act'(z), in 64 bits."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp(min=0), torch.heaviside(z, torch.zeros((), dtype=z.dtype, device=z.device))
    if name == "silu":
        t = torch.sigmoid(z)
        return z * t, t + z * t * torch.sigmoid(-z)
    if name == "gelu":
        density = torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
        return z * _normal_cdf(z), _normal_cdf(z) + z * density
    # 1/2 (1 + tanh q) is the logistic function of 2 q
    q = 2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)
    t = torch.sigmoid(q)
    return z * t, t + z * t * torch.sigmoid(-q) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * z.square())


def _mulhilo16(m, v):
    """High and low words of m * v by 16-bit halves of m, so that nothing passes 63 bits."""
    low = (m & 0xFFFF) * v
    total = (m >> 16) * v + (low >> 16)
    return total >> 16, ((total & 0xFFFF) << 16) | (low & 0xFFFF)


def _factors(rows, n, p, seed, offset, device):
    """What each element is multiplied by: 0, or one over the probability of being kept."""
    index = torch.arange(rows * n, device=device, dtype=torch.int64)
    word = [v for v in ((index // 8) % (1 << 32), (index // 8) // (1 << 32), torch.full_like(index, offset % (1 << 32)),
                        torch.full_like(index, offset // (1 << 32)))]
    key = [seed % (1 << 32), seed // (1 << 32)]
    for step in range(7):
        hi0, lo0 = _mulhilo16(0xD2511F53, word[0])
        hi1, lo1 = _mulhilo16(0xCD9E8D57, word[2])
        bump = [(key[0] + step * 0x9E3779B9) % (1 << 32), (key[1] + step * 0xBB67AE85) % (1 << 32)]
        word = [hi1 ^ word[1] ^ bump[0], lo1, hi0 ^ word[3] ^ bump[1], lo0]
    lane = index % 8
    pick = torch.where(lane < 2, word[0], torch.where(lane < 4, word[1], torch.where(lane < 6, word[2], word[3])))
    half = (pick >> (16 * (lane % 2))) % 65536
    border = min(65535, round(p * 65536))
    return ((half >= border).double() / (1 - border / 65536)).reshape(rows, n)


def _standard(x, kind):
    if kind == "layer":
        var, mean = torch.var_mean(x, dim=1, unbiased=False, keepdim=True)
        return (x - mean) / torch.sqrt(var + 1e-6), 1 / torch.sqrt(var + 1e-6)
    rms = torch.sqrt(x.square().mean(dim=1, keepdim=True) + 1e-6)
    return x / rms, 1 / rms


def _through_norm(dn, t, inverse, kind):
    """The gradient of a row's input: what is left of dn without its part along t and, where the norm is centred, its mean."""
    n = t.shape[1]
    rest = dn - t * (torch.linalg.vecdot(dn, t).unsqueeze(1) / n)
    return inverse * (rest - (rest.mean(dim=1, keepdim=True) if kind == "layer" else 0.0))


def _exact_norm(s):
    c = s["case"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    one = torch.ones(c["n"], dtype=torch.float64, device="cuda")
    zero = torch.zeros_like(one)
    if c["gate"] > 0:
        gate = d["gate"][torch.div(torch.arange(c["rows"], device="cuda"), c["gate"], rounding_mode="floor")]
    else:
        gate = d.get("gate", one)
    unit, inverse = _standard(d["b"], c["kind"]) if c["post"] else (d["b"], 1.0)
    p = unit * d.get("pw", one) + d.get("pb", zero)
    if c["direction"] == "forward":
        r = torch.addcmul(d["r"], gate, p, value=c["scale"])
        return dict(residual=r, y=_standard(r, c["kind"])[0] * d["nw"] + d.get("nb", zero))
    t, rinv = _standard(d["r"], c["kind"])
    total = d["dr"] + _through_norm(d["dy"] * d["nw"], t, rinv, c["kind"])
    out = dict(residual=total, norm_weight=torch.linalg.vecdot(d["dy"], t, dim=0))
    dp = total * gate * c["scale"]
    if c["gate"] < 0:
        out["gate"] = torch.linalg.vecdot(total, p, dim=0) * c["scale"]
    elif c["gate"] > 0:
        out["gate"] = torch.stack([v.sum(dim=0) for v in torch.split(total * p * c["scale"], c["gate"])])
    if c["kind"] == "layer":
        out["norm_bias"] = d["dy"].sum(dim=0)
    if c["post"]:
        out["post_weight"] = torch.linalg.vecdot(dp, unit, dim=0)
        if c["kind"] == "layer":
            out["post_bias"] = dp.sum(dim=0)
        dp = _through_norm(dp * d["pw"], unit, inverse, c["kind"])
    out["block"] = dp
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c, back, out = case, case["direction"] == "backward", {}
    if c["op"] == "norm":
        return _exact_norm(s)
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    factors = _factors(c["rows"], c["n"], c["p"], s["seed"], s["offset"], "cuda") if c.get("p", 0.0) > 0 else 1.0
    if c["op"] == "dropout":
        return dict(y=d["x"] * factors * c["scale"] + d.get("r", 0.0))
    if c["op"] == "linear":
        if not back:
            z = torch.nn.functional.linear(d["x"], d["w"], d.get("b"))
            out["y"] = _value_and_slope(c["act"], z)[0] * factors * c["scale"] + d.get("r", 0.0)
            if c["act"] != "none":
                out["pre"] = z
            return out
        dz = d["dy"] * factors * c["scale"]
        if c["act"] != "none":
            dz = dz * _value_and_slope(c["act"], d["pre"])[1]
        out["x"], out["weight"] = torch.mm(dz, d["w"]), torch.mm(dz.t(), d["x"])
        if c["bias"]:
            out["bias"] = dz.sum(dim=0)
        return out
    if not back:
        g, u = torch.nn.functional.linear(d["x"], d["wg"], d.get("bg")), torch.nn.functional.linear(d["x"], d["wu"], d.get("bu"))
        out["h"] = _value_and_slope(c["act"], g)[0] * u
        if c["save"]:
            out["gate"], out["up"] = g, u
        return out
    value, slope = _value_and_slope(c["act"], d["g"])
    dg, du = d["dh"] * d["u"] * slope, d["dh"] * value
    out["x"] = torch.mm(dg, d["wg"]) + torch.mm(du, d["wu"])
    out["gate_weight"], out["up_weight"] = torch.mm(dg.t(), d["x"]), torch.mm(du.t(), d["x"])
    if c["bias"]:
        out["gate_bias"], out["up_bias"] = dg.sum(dim=0), du.sum(dim=0)
    return out
