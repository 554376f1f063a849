"""The operators of a layer that a worker computes on its weights, as cases to be timed and compared.

    op "norm"       layer norm of token rows, with the sum with the residual stream before it where there is one
       "norm_grad"  its gradients: of the rows, of the weight and of the bias
       "product"    rows quantized to 8 bits times 8-bit weights, a scale for each token and each channel
       "held"       the same with the packed weights that a worker holds; "norm" in the case: of the layer norm of the rows
       "held_grad"  the product's gradient towards its rows, with the packed weights
       "weight"     the product's gradient towards its weights, into a buffer, or added to what is there

`run` has each operator in its plain form (elementary torch operations), or, where `own` is true, as calls of this
repository's package.  `exact` restates it in 64 bits.

Layer norm, of a row h of C elements (h = x, or x + r rounded to the type of x):

    mean = sum h / C;  rstd = 1 / sqrt(sum (h - mean)^2 / C + eps);  xhat = (h - mean) rstd;  y = xhat w + b
    g = dy w;  dx = rstd (g - sum g / C - xhat sum(g xhat) / C) + ds;  dw = sum over rows of dy xhat;  db = sum over rows of dy

Rows in 8 bits: a = max(max |x|, 2^-100), q = x * (127 / a) rounded to the nearest whole number (ties to even; quotient and
product in binary32), worth q (a / 127).  Columns in 8 bits: the same along the other axis.

Products: y[m, n] = sa[m] sb[n] sum_k qa[m, k] qb[n, k] + bias[n].  Held weights: element (n, k) is the code of kx + 2 bits at
bits [(n K + k) (kx + 2), ...) of the stream, worth (code - 2^kx) / 2^(kx + 1).
"""
from __future__ import annotations

import random

import torch

own = False          # set from outside: the package's operators in place of the plain forms

EPS = 1e-12          # the layer norms of the transformer whose tensors are the "bert_base" set
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _norm(name, tokens, width, x, w, residual=False):
    c = dict(op="norm", tokens=tokens, width=width, x=x, w=w, residual=residual)
    return dict(c, name=name) if name else c


def _norm_grad(name, tokens, width, x, w, dw, ds=False, add=False):
    c = dict(op="norm_grad", tokens=tokens, width=width, x=x, w=w, dw=dw, ds=ds, add=add)
    return dict(c, name=name) if name else c


def _product(name, tokens, k, n, x, out, bias=False):
    c = dict(op="product", tokens=tokens, k=k, n=n, x=x, out=out, bias=bias)
    return dict(c, name=name) if name else c


def _held(name, tokens, k, n, kx, x, out, bias=False, norm=False):
    c = dict(op="held", tokens=tokens, k=k, n=n, kx=kx, x=x, out=out, bias=bias, norm=norm)
    return dict(c, name=name) if name else c


def _held_grad(name, tokens, k, n, kx, x, out):
    c = dict(op="held_grad", tokens=tokens, k=k, n=n, kx=kx, x=x, out=out, bias=False)
    return dict(c, name=name) if name else c


def _weight(name, tokens, k, n, x, out, add=False):
    c = dict(op="weight", tokens=tokens, k=k, n=n, x=x, out=out, bias=False, add=add)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One new token for each of 16 sequences; latency is all there is.
        _norm("norm_16_tokens", 16, 768, "bf16", "bf16"),
        # A worker's batch of 16 sequences of 512: the sum with the residual stream and its norm.
        _norm("norm_sum_8192", 8192, 768, "bf16", "f32", residual=True),
        # The same batch on the way back; the residual stream's own gradient is added.
        _norm_grad("norm_grad_8192", 8192, 768, "bf16", "f32", "f32", ds=True),
        # A long batch of odd sizes in full precision, added to gradients that are there already.
        _norm_grad("norm_grad_odd_30011", 30011, 2049, "f32", "f32", "f32", add=True),
        # A single token through a square layer of 8-bit weights.
        _product("token_4096", 1, 4096, 4096, "bf16", "bf16", bias=True),
        # Scores of the whole vocabulary for one token each of 16 sequences, from the packed embedding.
        _held("scores_16_held", 16, 768, 30522, 6, "bf16", "f32"),
        # An attention projection of the worker's batch, weights of one byte as they were broadcast.
        _held("held_8192", 8192, 768, 768, 6, "bf16", "bf16", bias=True),
        # Three projections in one, behind a layer norm whose output goes to the product in 8 bits.
        _held("norm_held_8192", 8192, 768, 2304, 6, "bf16", "bf16", bias=True, norm=True),
        # An odd batch, layer and code width.
        _held("held_narrow_5001", 5001, 1001, 1537, 2, "f32", "f32"),
        # Back through the three projections, towards their input.
        _held_grad("held_grad_8192", 8192, 768, 2304, 6, "bf16", "bf16"),
        # The gradient of the three projections' weights, into a worker's gradient.
        _weight("weight_grad_8192", 8192, 768, 2304, "bf16", "f32"),
        # A large batch through a large square layer.
        _product("product_16384", 16384, 8192, 8192, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng: random.Random):
    op = rng.choice(["norm", "norm_grad", "product", "held", "held", "held_grad", "weight"])
    x = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op in ("norm", "norm_grad"):
        tokens, width = _log(rng, 1, 65536), _log(rng, 64, 8192)
        tokens = max(1, min(tokens, (1 << 26) // width))
        if rng.random() < 0.7:
            width = -(-width // 8) * 8
        w = rng.choice(["f32", x])
        if op == "norm":
            return _norm(None, tokens, width, x, w, residual=rng.random() < 0.5)
        return _norm_grad(None, tokens, width, x, w, "f32", ds=rng.random() < 0.5, add=rng.random() < 0.5)
    tokens, k, n = _log(rng, 1, 16384), _log(rng, 64, 8192), _log(rng, 64, 16384)
    if rng.random() < 0.7:
        k, n = -(-k // 16) * 16, -(-n // 16) * 16
    out = rng.choice(["f32", x])
    tokens = max(1, min(tokens, (1 << 39) // (k * n)))
    if op == "product":
        return _product(None, tokens, k, n, x, out, bias=rng.random() < 0.5)
    if op == "weight":
        return _weight(None, tokens, k, n, x, "f32", add=rng.random() < 0.5)
    kx = rng.choice([6, 6, 6, 0, 2, 4])
    if op == "held_grad":
        return _held_grad(None, tokens, k, n, kx, x, out)
    norm = rng.random() < 0.3
    if norm and out == "f32":
        out = "bf16"          # which side of a border a normed value falls on is for its last bit to say
    return _held(None, tokens, k, n, kx, x, out, bias=rng.random() < 0.5, norm=norm)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, x_type = case["op"], TYPES[case["x"]]

    def randn(*shape):
        return torch.randn(*shape, device="cuda", generator=gen)

    tokens = case["tokens"]
    st = {"case": case}
    if op in ("norm", "norm_grad"):
        width, w_type = case["width"], TYPES[case["w"]]
        st["x"] = (randn(tokens, width) + 0.1 * randn(width)).to(x_type)
        st["w"] = (1 + 0.1 * randn(width)).to(w_type)
        st["b"] = (0.1 * randn(width)).to(w_type)
        if op == "norm":
            if case["residual"]:
                st["r"] = randn(tokens, width).to(x_type)
            return st
        h = st["x"].double()
        st["mean"] = h.mean(1).float()
        st["rstd"] = (h.var(1, correction=0) + EPS).rsqrt().float()
        del h
        st["dy"] = (1e-2 * randn(tokens, width)).to(x_type)
        if case["ds"]:
            st["ds"] = (1e-2 * randn(tokens, width)).to(x_type)
        if case["add"]:
            st["dw"], st["db"] = ((1e-2 * randn(width)).to(TYPES[case["dw"]]) for _ in range(2))
        return st
    k, n = case["k"], case["n"]
    # a token's size differs from the next one's
    x = randn(tokens, n if op == "held_grad" else k) * torch.exp2(randn(tokens, 1))
    st["x"] = x.to(x_type)
    del x
    if case["bias"]:
        st["bias"] = 0.1 * randn(n)
    if op == "weight":
        st["dy"] = (1e-2 * randn(tokens, n)).to(x_type)
        st["dw"] = (1e-2 * randn(n, k)).to(TYPES[case["out"]])
        return st
    if op == "product":
        # rows on 16 bytes, as a program that lays its weights out once has them
        q = torch.zeros(n, -(-k // 16) * 16, device="cuda", dtype=torch.int8)
        q[:, :k] = (randn(n, k) * 32).round().clamp(-127, 127).to(torch.int8)
        st["q"] = q[:, :k]
        st["scale"] = 1e-3 * torch.exp2(randn(n))
        return st
    if case.get("norm"):
        st["w"], st["b"] = 1 + 0.1 * randn(k), 0.1 * randn(k)
    kx = case["kx"]
    bits, total = kx + 2, -(-n * k // 128) * 128
    level = (randn(total) * (0.35 * 2 ** kx)).round().clamp(-2 ** kx, 2 ** kx).to(torch.int64)
    at = torch.arange(total, device="cuda") * bits
    words = torch.zeros(total * bits // 32 + 1, device="cuda", dtype=torch.int64)
    put = (level + 2 ** kx) << (at & 31)
    words.index_add_(0, at >> 5, put & 0xFFFFFFFF)
    words.index_add_(0, (at >> 5) + 1, put >> 32)
    words = words[:-1]
    st["codes"] = torch.stack([(words >> s) & 255 for s in (0, 8, 16, 24)], 1).reshape(-1).to(torch.uint8)
    return st


# ---------------------------------------------------------------- plain forms

def _eight_bits(x, dim):
    """-> whole numbers (binary32), what one is worth"""
    a = x.abs().amax(dim, keepdim=True).clamp(min=2.0 ** -100)
    top = torch.full_like(a, 127.0)              # (with a number in its place torch multiplies by a reciprocal)
    return (x * (top / a)).round(), a / top


def _normed(x, w, b):
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = 1.0 / (c.square().mean(1, keepdim=True) + EPS).sqrt()
    return c * rstd * w.float() + b.float(), mean[:, 0], rstd[:, 0]


def _levels(codes, kx, n, k):
    """The held weights' levels, binary32 [n, k]."""
    bits = kx + 2
    if bits == 8:
        code = codes[:n * k].to(torch.int32)
    else:
        at = torch.arange(n * k, device="cuda") * bits
        code = codes[at >> 3].to(torch.int32) | codes[((at >> 3) + 1).clamp(max=codes.numel() - 1)].to(torch.int32) << 8
        code = code >> (at & 7).to(torch.int32) & (1 << bits) - 1
    return (code - (1 << kx)).float().view(n, k)


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "norm":
        h = st["x"]
        if case["residual"]:
            h = (h.float() + st["r"].float()).to(h.dtype)
        y, mean, rstd = _normed(h.float(), st["w"], st["b"])
        y = y.to(h.dtype)
        return (y, h, mean, rstd) if case["residual"] else (y, mean, rstd)
    if op == "norm_grad":
        dy, rstd = st["dy"].float(), st["rstd"][:, None]
        xhat = (st["x"].float() - st["mean"][:, None]) * rstd
        g = dy * st["w"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if case["ds"]:
            dx = dx + st["ds"].float()
        dw, db = (dy * xhat).sum(0), dy.sum(0)
        if case["add"]:
            dw, db = st["dw"].float() + dw, st["db"].float() + db
        return dx.to(st["x"].dtype), dw.to(TYPES[case["dw"]]), db.to(TYPES[case["dw"]])
    out = TYPES[case["out"]]
    x = st["x"].float()
    if op == "weight":
        qd, sd = _eight_bits(st["dy"].float(), 0)
        qx, sx = _eight_bits(x, 0)
        dw = (qd.T @ qx) * sd.T * sx
        return (st["dw"].float() + dw if case["add"] else dw).to(out)
    if case.get("norm"):
        x = _normed(x, st["w"], st["b"])[0]
    qx, sx = _eight_bits(x, 1)
    if op == "product":
        y = (qx @ st["q"].float().T) * sx * st["scale"]
    else:
        w = _levels(st["codes"], case["kx"], case["n"], case["k"])
        y = (qx @ (w if op == "held_grad" else w.T)) * sx * 2.0 ** -(case["kx"] + 1)
    return (y + st["bias"] if case["bias"] else y).to(out)


# ---------------------------------------------------------------- the package's calls

def _own(st):
    import paper_2004_14180_b200 as qb
    case = st["case"]
    op = case["op"]
    if op == "norm":
        r = qb.layer_norm(st["x"], st["w"], st["b"], EPS, residual=st.get("r"))
        return (r.out, r.sum, r.mean, r.rstd) if case["residual"] else (r.out, r.mean, r.rstd)
    if op == "norm_grad":
        if case["add"]:
            dw, db = st["dw"].clone(), st["db"].clone()       # (the state's own would grow from pass to pass)
            return qb.layer_norm_grad(st["dy"], st["x"], st["mean"], st["rstd"], st["w"], dsum=st.get("ds"), dweight=dw, dbias=db,
                                      accumulate=True)
        return qb.layer_norm_grad(st["dy"], st["x"], st["mean"], st["rstd"], st["w"], dsum=st.get("ds"),
                                  grad_dtype=TYPES[case["dw"]])
    out = TYPES[case["out"]]
    if op == "weight":
        dw = st["dw"].clone() if case["add"] else st["dw"]
        return qb.int8_matmul(qb.quantize_columns(st["dy"]), qb.quantize_columns(st["x"]), out=dw, accumulate=case["add"])
    if op == "product":
        return qb.int8_matmul(qb.quantize_rows(st["x"]), qb.Int8Rows(st["q"], st["scale"]), bias=st.get("bias"), out_dtype=out)
    if case.get("norm"):
        a = qb.layer_norm(st["x"], st["w"], st["b"], EPS, dense=False, int8=True).rows
    else:
        a = qb.quantize_rows(st["x"])
    return qb.held_matmul(a, st["codes"], case["kx"], case["n"], case["k"], bias=st.get("bias"), transpose=op == "held_grad",
                          out_dtype=out)


def run(st):
    return _own(st) if own else _plain(st)


# ---------------------------------------------------------------- in 64 bits

def _exact_rows(x, dim):
    """The whole numbers go by values next to a border: quotient and product are rounded to binary32, as the definition has it
    (from 64 bits, which hold the product and decide the quotient's rounding)."""
    x = x.float().double()
    size = torch.maximum(x.abs().amax(dim, keepdim=True), torch.tensor(2.0 ** -100, dtype=torch.float64, device=x.device))
    per = (127.0 / size).float().double()
    return torch.round((x * per).float()).double(), size / 127.0


def _exact_product(p, q):
    """p q^T; whole numbers, in parts where all of q would be large."""
    return torch.cat([p @ part.double().T for part in q.split(4096)], 1)


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    x = st["x"].double()
    if op == "norm" or case.get("norm"):
        if case.get("residual"):
            x = (x + st["r"].double()).to(st["x"].dtype).double()
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        y = (x - mean) / torch.sqrt(var + EPS) * st["w"].double() + st["b"].double()
        if op == "norm":
            ends = (mean.flatten(), 1.0 / torch.sqrt(var + EPS).flatten())
            return (y, x) + ends if case["residual"] else (y,) + ends
        x = y
    if op == "norm_grad":
        r, dy = st["rstd"].double()[:, None], st["dy"].double()
        x -= st["mean"].double()[:, None]
        x *= r
        dw, db = torch.einsum("tc,tc->c", dy, x), dy.sum(0)
        dy *= st["w"].double()
        width = case["width"]
        along = torch.einsum("tc,tc->t", dy, x)[:, None] / width
        dx = (dy - dy.sum(1, keepdim=True) / width - along * x) * r
        if case["ds"]:
            dx += st["ds"].double()
        return dx, dw + (st["dw"].double() if case["add"] else 0), db + (st["db"].double() if case["add"] else 0)
    if op == "weight":
        a, sa = _exact_rows(st["dy"].double().T, 1)
        b, sb = _exact_rows(x.T, 1)
        dw = sa * sb.T * _exact_product(a, b)
        return st["dw"].double() + dw if case["add"] else dw
    q, size = _exact_rows(x, 1)
    if op == "product":
        y = _exact_product(q, st["q"]) * size * st["scale"].double()
    else:
        kx, n, k = case["kx"], case["n"], case["k"]
        weight = 2 ** torch.arange(kx + 2, device="cuda", dtype=torch.int16)
        bits = (st["codes"][:, None] >> torch.arange(8, device="cuda", dtype=torch.uint8) & 1).flatten()
        level = (bits[:n * k * (kx + 2)].view(n, k, kx + 2) * weight).sum(2, dtype=torch.int16) - 2 ** kx
        y = _exact_product(q, level.T if op == "held_grad" else level) * size / 2.0 ** (kx + 1)
    return y + st["bias"].double() if case["bias"] else y


def work(case):
    op, tokens = case["op"], case["tokens"]
    e = BYTES[case["x"]]
    if op in ("norm", "norm_grad"):
        width, ew = case["width"], BYTES[case["w"]]
        if op == "norm":
            return {"bytes": tokens * width * e * (4 if case["residual"] else 2) + 2 * width * ew + 8 * tokens,
                    "flops": 8 * tokens * width}
        edw = BYTES[case["dw"]] * (2 if case["add"] else 1)
        return {"bytes": tokens * width * e * (4 if case["ds"] else 3) + width * (ew + 2 * edw) + 8 * tokens,
                "flops": 14 * tokens * width}
    k, n, eo = case["k"], case["n"], BYTES[case["out"]]
    flops = 2 * tokens * k * n
    if op == "weight":
        return {"bytes": tokens * (k + n) * e + k * n * eo * (2 if case["add"] else 1), "flops": flops}
    rows, cols = (n, k) if op == "held_grad" else (k, n)
    weights = k * n + 4 * n if op == "product" else k * n * (case["kx"] + 2) // 8
    extra = (4 * n if case["bias"] else 0) + (8 * k if case.get("norm") else 0)
    return {"bytes": tokens * rows * e + weights + tokens * cols * eo + extra, "flops": flops}
