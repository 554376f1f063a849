"""The operators of a training step around the quantized step, as cases to be timed and compared.

    op "adamw"   one AdamW step over many tensors at once, moments in 32 or in 8 bits
       "norm"    the norm of all gradients, and the factor that clips it
       "lookup"  rows of the token embedding, scaled: dense weights, or the packed broadcast that a worker holds
       "grad"    the gradient of the token embedding, from the gradient of the looked-up rows

`run` has each operator in its plain form (elementary torch operations), or, where `own` is true, as the call of this
repository's package.  `exact` restates it in 64 bits.

AdamW, for gradient g, clipping factor c, moments m and v, weight x, at step t; one binary32 rounding per operation:

    g' = g c;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
    x  = x (1 - lr decay) - lr / (1 - b1^t) * (m / (sqrt(v) / sqrt(1 - b2^t) + eps))

With 8-bit moments a row of 128 elements has two binary32 scales, the largest |m| and the largest r = sqrt(v) of the row
(at least 2^-126).  y = |m| / scale becomes sign and 7 bits: floating point with 3 bits of mantissa, 1.0 the code 127, code 0
zero; r / scale becomes 8 bits with 4 bits of mantissa, 1.0 the code 255, and at least code 1 if r is not zero.  Both are
rounded at random: with h the element's 16 random bits, the mantissa's bits that are dropped get (2 (h mod 64) + 1) / 128 of a
step added (r: (2 (h div 64) + 1) / 2048), then are cut off.  Elements 128 apart share a Philox4x32-10 block: element i of a tensor that
starts at padded element o has half-word 4 ((i div 128) mod 2) + i mod 4 of the block with counter
((o + 256 (i div 256) + 4 ((i mod 128) div 4)) / 4, 0, t, 0) and key (seed, 0).
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False          # set from outside: the package's operators in place of the plain forms

BETA1, BETA2, EPS, LR = 0.9, 0.999, 1e-8, 1e-3
MAX_NORM = 1.0
DONE = 7             # steps a run in progress has behind it
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def _adamw(name, shape, bits, w, g, d=0, tensors=1, master=False, clip=False, packed=False, decay=0.01):
    c = dict(op="adamw", shape=shape, d=d, tensors=tensors, bits=bits, w=w, g=g, master=master, clip=clip, packed=packed,
             decay=decay)
    return dict(c, name=name) if name else c


def _norm(name, shape, g, d=0, tensors=1):
    c = dict(op="norm", shape=shape, d=d, tensors=tensors, g=g, packed=False)
    return dict(c, name=name) if name else c


def _lookup(name, tokens, rows, width, w, out, kx=-1, ids="i64"):
    c = dict(op="lookup", tokens=tokens, rows=rows, width=width, w=w, out=out, kx=kx, ids=ids)
    return dict(c, name=name) if name else c


def _grad(name, tokens, rows, width, dy, dw, add=False, ids="i64", pad=0.0):
    c = dict(op="grad", tokens=tokens, rows=rows, width=width, dy=dy, dw=dw, add=add, ids=ids, pad=pad)
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest set anyone steps: a few ragged tensors back to back in one bucket; latency is all there is.
        _adamw("adamw_ragged_13k", "tensors", 32, "f32", "f32", d=13290, tensors=3, packed=True),
        # A convolutional network's tensors in full precision, gradients clipped first.
        _adamw("adamw_resnet18_clip", "resnet18_qg", 32, "f32", "f32", clip=True),
        # A transformer's tensors in mixed precision: 16-bit weights and gradients, 32-bit master weights.
        _adamw("adamw_bert_master", "bert_base", 32, "bf16", "bf16", master=True),
        # The network of the second case with 8-bit moments.
        _adamw("adamw8_resnet18", "resnet18_qg", 8, "f32", "f32"),
        # The transformer with 8-bit moments and master weights.
        _adamw("adamw8_bert_master", "bert_base", 8, "bf16", "bf16", master=True),
        # What is looked at after every backward pass, on both sets of tensors.
        _norm("norm_resnet18", "resnet18_qg", "f32"),
        _norm("norm_bert", "bert_base", "bf16"),
        # One token each of 16 sequences.
        _lookup("lookup_16_tokens", 16, 30522, 768, "bf16", "bf16"),
        # A worker's batch of 16 sequences of 512, rows decoded from the 8-bit weights that it holds.
        _lookup("lookup_held_8192", 8192, 30522, 768, "held", "bf16", kx=6),
        # A short batch added to the gradient that the tied output layer has left there.
        _grad("grad_96_added", 96, 30522, 768, "bf16", "f32", add=True),
        # The batch of 16 x 512 with its padding, straight into an fp32 gradient.
        _grad("grad_bert_8192", 8192, 30522, 768, "bf16", "f32", pad=0.1),
        # A long batch, an odd number of tokens, a larger vocabulary, 16-bit gradients.
        _grad("grad_long_200001", 200001, 128256, 1024, "bf16", "bf16", ids="i32"),
    ]


def _log(rng, lo, hi):
    return int(lo * (hi / lo) ** rng.random())


def draw(rng):
    """Another case of the same ranges: sets of 10^4 to 10^8 elements, batches of 1 to 200 000 tokens, every type."""
    op = rng.choices(["adamw", "norm", "lookup", "grad"], [45, 15, 15, 25])[0]
    if op in ("adamw", "norm"):
        shape = rng.choices(["tensors", "resnet18_qg", "bert_base"], [70, 15, 15])[0]
        d, tensors = 0, 1
        if shape == "tensors":
            tensors = rng.choice([1, 1, 2, 5, rng.randint(3, 300), rng.randint(300, 1200)])
            d = max(60 * tensors, _log(rng, 10 ** 4, 10 ** 8))
        g = rng.choice(["f32", "bf16", "bf16", "f16"])
        if op == "norm":
            return _norm(None, shape, g, d=d, tensors=tensors)
        w = rng.choice(["f32", "f32", "bf16", "f16"])
        bits = rng.choice([32, 8])
        return _adamw(None, shape, bits, w, g, d=d, tensors=tensors, master=w != "f32" and rng.random() < 0.7,
                      clip=bits == 32 and rng.random() < 0.5, packed=shape == "tensors" and d < 4e6 and rng.random() < 0.4,
                      decay=rng.choice([0.0, 0.01, 0.1]))
    rows = rng.choice([2, 512, 30522, 30522, _log(rng, 1000, 131072)])
    width = rng.choice([768, 64 * rng.randint(1, 16), 64 * rng.randint(1, 32), rng.randint(1, 2000)])
    most = max(1, min(200000, 200000 * 1024 // width))
    tokens = _log(rng, 1, most)
    if op == "lookup":
        w = rng.choice(["f32", "bf16", "bf16", "f16", "held", "held"])
        return _lookup(None, tokens, rows, width, w, rng.choice(["f32", "bf16", "f16"]),
                       kx=rng.choice([0, 1, 2, 6, 14]) if w == "held" else -1, ids=rng.choice(["i64", "i32"]))
    return _grad(None, tokens, rows, width, rng.choice(["f32", "bf16", "bf16", "f16"]) if width * tokens < 10 ** 8 else "bf16",
                 rng.choice(["f32", "f32", "bf16"]), add=rng.random() < 0.3, ids=rng.choice(["i64", "i32"]),
                 pad=rng.choice([0.0, 0.1, 0.5]))


# ---------------------------------------------------------------- the tensors of a set

def _lengths(case):
    """Lengths of the set's tensors, and which of them decay (matrices)."""
    if case["shape"] == "tensors":
        rng = random.Random(case["d"] * 1000 + case["tensors"])
        parts = [10 ** (3 * rng.random()) for _ in range(case["tensors"])]
        lens = [max(1, int(case["d"] * p / sum(parts))) for p in parts]
        lens[-1] = max(1, lens[-1] + case["d"] - sum(lens))
        return lens, [n > 1000 for n in lens]
    from qadam_inputs import shapes
    every = shapes.bert_base_shapes() if case["shape"] == "bert_base" else shapes.resnet18_shapes()
    return [math.prod(s) for _, s, _ in every], [len(s) > 1 for _, s, _ in every]


class _Set:
    """Where the tensors lie: each begins at a multiple of 128 elements, or (packed) where the one before it ends."""

    def __init__(self, case, device):
        self.lens, self.decays = _lengths(case)
        pad = [-(-n // 128) * 128 for n in self.lens]
        self.off = [0]
        for n in pad:
            self.off.append(self.off[-1] + n)
        self.D, self.d = self.off.pop(), sum(self.lens)
        n = torch.tensor(self.lens, device=device)
        off = torch.tensor(self.off, device=device)
        rows = torch.tensor([p // 128 for p in pad], device=device)
        self.seg_of_row = torch.repeat_interleave(torch.arange(len(pad), device=device), rows)
        self.first_row = torch.repeat_interleave(off // 128, rows)               # of the row's tensor
        row = torch.arange(self.D // 128, device=device)
        left = torch.repeat_interleave(n, rows) - 128 * (row - self.first_row)
        self.live = torch.arange(128, device=device)[None, :] < left[:, None]    # not padding
        self.packed = case["packed"]
        self.at = self.live.reshape(-1).nonzero().reshape(-1) if self.packed else None   # padded place of each element

    def views(self, base):
        start = self.off
        if self.packed:
            start = [sum(self.lens[:i]) for i in range(len(self.lens))]
        return [base[o:o + n] for o, n in zip(start, self.lens)]

    def stored(self, padded):
        """A padded array as it lies in memory."""
        return padded.reshape(-1)[self.at] if self.packed else padded.reshape(-1)

    def padded(self, base):
        if not self.packed:
            return base
        out = torch.zeros(self.D, dtype=base.dtype, device=base.device)
        out[self.at] = base
        return out


def _sigma(s, gen):
    """A gradient scale for each tensor, log-uniform in [1e-4, 1e-1], by row."""
    per = 10.0 ** (3.0 * torch.rand(len(s.lens), device="cuda", generator=gen) - 4.0)
    return per[s.seg_of_row][:, None]


def _moments(s, sigma, gen):
    """m and v as some steps leave them."""
    m = torch.randn(s.D // 128, 128, device="cuda", generator=gen) * (0.3 * sigma) * s.live
    v = ((0.5 + torch.rand(s.D // 128, 128, device="cuda", generator=gen)) * sigma).square() * s.live
    return m, v


# ---------------------------------------------------------------- 8-bit moments, plain form

def _mul(a, x):
    """High and low word of the 64-bit products a x of 32-bit numbers held in 64 bits."""
    low = a * (x & 0xFFFF)
    high = a * (x >> 16) + (low >> 16)
    return high >> 16, ((high & 0xFFFF) << 16) | (low & 0xFFFF)


def _coins(s, seed, t):
    """16 random bits for each element, [rows, 128]."""
    row = torch.arange(s.D // 128, device="cuda") - s.first_row
    pair = s.first_row + 2 * (row // 2)                        # first row of the pair that shares its blocks
    c0 = pair[:, None] * 32 + torch.arange(32, device="cuda")[None, :]
    c1, c2, c3 = torch.zeros_like(c0), torch.full_like(c0, t), torch.zeros_like(c0)
    k0, k1 = seed & 0xFFFFFFFF, 0
    for _ in range(10):
        h0, l0 = _mul(0xD2511F53, c0)
        h1, l1 = _mul(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    odd = (row % 2 == 1)[:, None]
    a, b = torch.where(odd, c2, c0), torch.where(odd, c3, c1)
    return torch.stack([a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16], dim=2).reshape(-1, 128).int()


def _encode(x, bits_kept, offset):
    """Magnitudes of rows as codes (before the ends are seen to) and the rows' scales."""
    scale = x.abs().amax(dim=1, keepdim=True).clamp_min(2.0 ** -126)
    y = x.abs() * (1.0 / scale)
    drop = 23 - bits_kept
    return ((y.view(torch.int32) + offset) >> drop) - (127 << bits_kept), scale


def _encode_m(m, h):
    q, scale = _encode(m, 3, ((h & 63) << 14) + (1 << 13))
    code = (q + 127).clamp_min(0)
    return (code + 128 * ((m < 0) & (code > 0))).to(torch.uint8), scale


def _encode_r(r, h):
    q, scale = _encode(r, 4, ((h >> 6) << 9) + (1 << 8))
    return torch.where(r > 0, (q + 255).clamp_min(1), 0).to(torch.uint8), scale


def _decode_m(code, scale):
    c = code.int()
    y = (((c & 127) + 889) << 20).view(torch.float32)
    y = torch.where((c & 127) > 0, y, 0.0) * scale
    return torch.where(c > 127, -y, y)


def _decode_r(code, scale):
    y = ((code.int() + 1777) << 19).view(torch.float32)
    return torch.where(code > 0, y, 0.0) * scale


# ---------------------------------------------------------------- states

def _ids(case, gen):
    """Tokens as text has them: a few very frequent, most rare; some places are padding."""
    n = case["rows"]
    weight = 1.0 / (torch.arange(n, device="cuda", dtype=torch.float64) + 2.7)
    edges = torch.cumsum(weight / weight.sum(), 0)
    rank = torch.searchsorted(edges, torch.rand(case["tokens"], device="cuda", generator=gen, dtype=torch.float64))
    ids = torch.randperm(n, device="cuda", generator=gen)[rank.clamp_max(n - 1)]
    if case.get("pad"):
        ids = torch.where(torch.rand(ids.shape, device="cuda", generator=gen) < case["pad"], -1, ids)
    return ids.to(torch.int64 if case["ids"] == "i64" else torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    randn = lambda *n: torch.randn(*n, device="cuda", generator=gen)  # noqa: E731
    st = {"case": case}
    if case["op"] in ("adamw", "norm"):
        s = st["set"] = _Set(case, "cuda")
        sigma = _sigma(s, gen)
        g = s.stored(randn(s.D // 128, 128) * sigma * s.live).to(TYPES[case["g"]])
        st["g"] = g
        if case["op"] == "norm":
            if own:
                import paper_2004_14180_b200 as qb
                st["norm"] = qb.GradNorm(s.views(g))
            return st
        x = randn(s.D // 128, 128) * 0.05 * s.live
        w = s.stored(x).to(TYPES[case["w"]])
        m, v = _moments(s, sigma, gen)
        del x, sigma
        st.update(w=w, t=DONE, seed=int(seed) & 0x7FFFFFFF,
                  decay=[case["decay"] if yes else 0.0 for yes in s.decays])
        if case["master"]:
            st["master"] = s.padded(w).float() + randn(s.D) * 1e-5 * s.live.reshape(-1)
        if case["bits"] == 8:
            zero = torch.full((1, 128), 1 << 15, device="cuda", dtype=torch.int32)
            st["m"], st["ms"] = _encode_m(m, zero)
            st["r"], st["rs"] = _encode_r(v.sqrt(), zero)
        else:
            st["m"], st["v"] = m, v
        if own:
            import paper_2004_14180_b200 as qb
            opt = qb.AdamW(s.views(w), s.views(g), state_bits=case["bits"], master=case["master"], beta1=BETA1, beta2=BETA2,
                           eps=EPS, lr=LR, weight_decay=st["decay"], seed=st["seed"])
            if case["master"]:
                opt.master.copy_(st.pop("master"))
            if case["bits"] == 8:
                opt.m.copy_(st.pop("m").reshape(-1))
                opt.r.copy_(st.pop("r").reshape(-1))
                opt.m_scale.copy_(st.pop("ms").reshape(-1))
                opt.r_scale.copy_(st.pop("rs").reshape(-1))
                st["m32"], st["v32"] = torch.empty(s.D, device="cuda"), torch.empty(s.D, device="cuda")
            else:
                opt.m.copy_(st.pop("m").reshape(-1))
                opt.v.copy_(st.pop("v").reshape(-1))
            st["opt"] = opt
        return st
    st["ids"] = _ids(case, gen)
    n, width = case["rows"], case["width"]
    if case["op"] == "lookup":
        st["scale"] = math.sqrt(width)
        if case["w"] == "held":
            # the broadcast of a one-tensor problem: codes of kx + 2 bits, element j at bits [j b, (j + 1) b)
            bits = case["kx"] + 2
            total = -(-n * width // 128) * 128
            code = torch.randint(0, (2 << case["kx"]) + 1, (total,), device="cuda", generator=gen)
            at = torch.arange(total, device="cuda") * bits
            words = torch.zeros(total * bits // 32 + 1, device="cuda", dtype=torch.int64)
            put = (code << (at & 31))
            words.index_add_(0, at >> 5, put & 0xFFFFFFFF)
            words.index_add_(0, (at >> 5) + 1, put >> 32)
            words = words[:-1]
            st["w"] = torch.stack([(words >> k) & 255 for k in (0, 8, 16, 24)], 1).reshape(-1).to(torch.uint8)
        else:
            st["w"] = (randn(n, width) * 0.05).to(TYPES[case["w"]])
        return st
    st["scale"] = math.sqrt(width)
    st["dy"] = (randn(case["tokens"], width) * 1e-2).to(TYPES[case["dy"]])
    if case["add"]:
        st["dw"] = (randn(n, width) * 1e-3).to(TYPES[case["dw"]])
    return st


# ---------------------------------------------------------------- one pass

def _clip(g):
    norm = g.double().square().sum().sqrt().float()
    return norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))


def _plain_adamw(st):
    case, s, t = st["case"], st["set"], st["t"]
    g = s.padded(st["g"]).float().reshape(-1, 128)
    out = {}
    if case["clip"]:
        out["norm"], factor = _clip(st["g"])
        g = g * factor
    f = np.float32
    b1, b2 = f(BETA1), f(BETA2)
    c1, c2 = f(1) - b1, f(1) - b2
    lr = float(f(LR))
    a = float(f(lr / (1 - float(b1) ** t)))
    b = float(f(1 / math.sqrt(1 - float(b2) ** t)))
    keep = (1 - lr * torch.tensor(st["decay"], dtype=torch.float32).double()).float().to(g.device)[s.seg_of_row][:, None]
    if case["bits"] == 8:
        m, v = _decode_m(st["m"], st["ms"]), _decode_r(st["r"], st["rs"]).square()
    else:
        m, v = st["m"], st["v"]
    m = float(b1) * m + float(c1) * g
    v = float(b2) * v + float(c2) * (g * g)
    x = (st["master"] if case["master"] else s.padded(st["w"]).float()).reshape(-1, 128)
    x = x * keep - a * (m / (v.sqrt() * b + EPS))
    if case["master"]:
        st["master"].copy_(x.reshape(-1))
        out["master"] = st["master"]
    st["w"].copy_(s.stored(x))
    out["w"] = st["w"]
    if case["bits"] == 8:
        h = _coins(s, st["seed"], t)
        st["m"], st["ms"] = _encode_m(m, h)
        st["r"], st["rs"] = _encode_r(v.sqrt(), h)
        out["m"], out["v"] = _decode_m(st["m"], st["ms"]).reshape(-1), _decode_r(st["r"], st["rs"]).square().reshape(-1)
    else:
        st["m"].copy_(m)
        st["v"].copy_(v)
        out["m"], out["v"] = st["m"].reshape(-1), st["v"].reshape(-1)
    return out


def _own_adamw(st):
    case, opt, out = st["case"], st["opt"], {}
    factor = None
    if case["clip"]:
        out["norm"], factor = opt.grad_norm(MAX_NORM)
    opt.step(st["t"], grad_scale=factor)
    if case["master"]:
        out["master"] = opt.master
    out["w"] = st["w"]
    if case["bits"] == 8:
        out["m"], out["v"] = opt.moments(out=(st["m32"], st["v32"]))
    else:
        out["m"], out["v"] = opt.m, opt.v
    return out


def _plain_rows(st):
    """Rows of the table at the tokens, in 32 bits."""
    case, ids = st["case"], st["ids"].long()
    if case["w"] != "held":
        return st["w"][ids].float()
    bits, kx = case["kx"] + 2, case["kx"]
    at = (ids[:, None] * case["width"] + torch.arange(case["width"], device="cuda")[None, :]) * bits
    w = torch.cat([st["w"], st["w"].new_zeros(4)])
    byte = at >> 3
    word = w[byte].long() | (w[byte + 1].long() << 8) | (w[byte + 2].long() << 16)
    code = (word >> (at & 7)) & ((1 << bits) - 1)
    return (code - (1 << kx)).float() * 2.0 ** -(kx + 1)


def run(state):
    st, case = state, state["case"]
    if case["op"] == "adamw":
        st["t"] += 1
        return _own_adamw(st) if own else _plain_adamw(st)
    if case["op"] == "norm":
        return st["norm"](MAX_NORM) if own else _clip(st["g"])
    if case["op"] == "lookup":
        if own:
            import paper_2004_14180_b200 as qb
            if case["w"] == "held":
                return qb.held_lookup(st["w"], case["kx"], st["ids"], case["rows"], case["width"], scale=st["scale"],
                                      out_dtype=TYPES[case["out"]])
            return qb.embedding_lookup(st["w"], st["ids"], scale=st["scale"], out_dtype=TYPES[case["out"]])
        return (st["scale"] * _plain_rows(st)).to(TYPES[case["out"]])
    if own:
        import paper_2004_14180_b200 as qb
        if case["add"]:
            return qb.embedding_grad(st["ids"], st["dy"], case["rows"], scale=st["scale"], out=st["dw"], accumulate=True)
        return qb.embedding_grad(st["ids"], st["dy"], case["rows"], scale=st["scale"], dtype=TYPES[case["dw"]])
    ids = st["ids"].long()
    ids = torch.where(ids < 0, case["rows"], ids)              # padding adds to a row that is dropped
    total = torch.zeros(case["rows"] + 1, case["width"], device="cuda").index_add_(0, ids, st["dy"].float())[:-1] * st["scale"]
    return st["dw"].copy_(total + st["dw"].float()) if case["add"] else total.to(TYPES[case["dw"]])


# ---------------------------------------------------------------- what it costs, and what it is

def work(case):
    """Bytes: every input read once, every output written once.  8-bit moments are read and written, and then written out
    as the values they stand for."""
    if case["op"] in ("adamw", "norm"):
        lens, _ = _lengths(case)
        d, per = sum(lens), BYTES[case["g"]]
        if case["op"] == "norm":
            return {"bytes": float(d * per), "flops": float(2 * d)}
        per += 8 + BYTES[case["w"]] if case["master"] else 2 * BYTES[case["w"]]
        per += 16 if case["bits"] == 32 else 4 + 16 / 128 + 8
        return {"bytes": float(d * per), "flops": float(15 * d)}
    id_bytes = 8 if case["ids"] == "i64" else 4
    n, width, tokens = case["rows"], case["width"], case["tokens"]
    touched = _distinct(case)
    if case["op"] == "lookup":
        row = width * (case["kx"] + 2) / 8 if case["w"] == "held" else width * BYTES[case["w"]]
        return {"bytes": float(tokens * (id_bytes + width * BYTES[case["out"]]) + touched * row), "flops": float(tokens * width)}
    # written whole, or the rows of this batch read and written where it is added to
    dw = width * BYTES[case["dw"]] * (2 * touched if case["add"] else n)
    return {"bytes": float(tokens * (id_bytes + width * BYTES[case["dy"]] * (1 - case["pad"])) + dw),
            "flops": float(tokens * width)}


def _distinct(case):
    """Rows that a batch is expected to touch."""
    weight = 1.0 / (np.arange(case["rows"]) + 2.7)
    return float(np.sum(1 - (1 - weight / weight.sum()) ** case["tokens"]))


def _f32(x):
    """Rounded to binary32, held in 64 bits."""
    return x.to(torch.float32).double()


def _exact_coins(s, seed, t):
    row = np.arange(s.D // 128, dtype=np.int64)
    first = s.first_row.cpu().numpy()
    inside = row - first
    c = [((first + inside - inside % 2)[:, None] * 32 + np.arange(32)[None, :]).astype(np.uint64), np.uint64(0),
         np.uint64(t), np.uint64(0)]
    key = [seed & 0xFFFFFFFF, 0]
    word, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for k in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64((key[0] + k * 0x9E3779B9) & 0xFFFFFFFF), q & word,
             (p >> half) ^ c[3] ^ np.uint64((key[1] + k * 0xBB67AE85) & 0xFFFFFFFF), p & word]
    full = np.stack([np.broadcast_to(x, c[0].shape) for x in c], axis=2).astype("<u4")            # [rows, 32, 4]
    halves = np.ascontiguousarray(full).view("<u2").reshape(-1, 32, 2, 4)
    return torch.from_numpy(halves[row, :, inside % 2, :].reshape(-1, 128).astype(np.int32)).cuda().double()


def _exact_round(y, mantissa, add):
    """y = 2^e (1 + f): f to so many bits, `add` of a step added before the rest is cut off."""
    frac, e = torch.frexp(y)                                   # y = frac 2^e, frac in [1/2, 1)
    steps = 2.0 ** mantissa
    k = torch.floor((2 * frac - 1) * steps + add)
    return torch.ldexp(1 + k / steps, e - 1) * (y > 0)


def _exact_table(mantissa, top):
    """Magnitude of each code: floating point that ends at 1.0."""
    steps = 2 ** mantissa
    return torch.tensor([0.0] + [2.0 ** ((c - top) // steps) * (1 + (c - top) % steps / steps) for c in range(1, top + 1)],
                        dtype=torch.float64, device="cuda")


def _exact_adamw(case, st):
    s, t = st["set"], st["t"] + 1
    out = {}
    g = s.padded(st["g"]).double().reshape(-1, 128)
    if case["clip"]:
        norm = out["norm"] = torch.linalg.vector_norm(st["g"].double())
        g = g * min(1.0, MAX_NORM / float(norm))
    b1, b2, lr = (float(np.float32(h)) for h in (BETA1, BETA2, LR))
    eight = case["bits"] == 8
    if eight:
        c = st["m"].long()
        m = _exact_table(3, 127)[c & 127] * st["ms"].double() * torch.where(c > 127, -1.0, 1.0)
        r = _exact_table(4, 255)[st["r"].long()] * st["rs"].double()
        m32, v32 = _f32(m), _f32(_f32(r) * _f32(r))
        v = r * r
    else:
        m, v = st["m"].double(), st["v"].double()
    if eight:
        # which code a value gets is decided on the binary32 numbers of the definition: round where it rounds
        c1, c2 = float(np.float32(1) - np.float32(BETA1)), float(np.float32(1) - np.float32(BETA2))
        m32 = _f32(_f32(b1 * m32) + _f32(c1 * g))
        v32 = _f32(_f32(b2 * v32) + _f32(c2 * _f32(g * g)))
        h = _exact_coins(s, st["seed"], t)
        r32 = _f32(v32.sqrt())
        least = 2.0 ** -126
        sm = m32.abs().amax(1, keepdim=True).clamp_min(least)
        sr = r32.amax(1, keepdim=True).clamp_min(least)
        y = _exact_round(_f32(m32.abs() * _f32(1 / sm)), 3, (2 * torch.remainder(h, 64) + 1) / 128)
        y = torch.where(y < 1.25 * 2.0 ** -16, 0.0, y)
        out["m"] = (y * sm * torch.sign(m32)).reshape(-1)
        y = _exact_round(_f32(r32 * _f32(1 / sr)), 4, (2 * torch.div(h, 64, rounding_mode="floor") + 1) / 2048)
        y = torch.where(r32 > 0, y.clamp_min(1.125 * 2.0 ** -16), 0.0)
        out["v"] = (y * sr).square().reshape(-1)
        del h, r32, y, m32, v32
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    if not eight:
        out["m"], out["v"] = m.reshape(-1), v.reshape(-1)
    x = (st["master"] if case["master"] else s.padded(st["w"])).double().reshape(-1, 128)
    decay = torch.tensor(st["decay"], dtype=torch.float32, device="cuda").double()[s.seg_of_row][:, None]
    x = x - lr * decay * x - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + EPS)
    if case["master"]:
        out["master"] = x.reshape(-1)
    out["w"] = s.stored(x)
    return out


def exact(case, seed):
    global own
    before, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = before
    if case["op"] == "adamw":
        return _exact_adamw(case, st)
    if case["op"] == "norm":
        norm = torch.linalg.vector_norm(st["g"].double())
        return norm, torch.clamp(MAX_NORM / norm, max=1.0)
    ids, width, scale = st["ids"].long(), case["width"], float(np.float32(st["scale"]))
    if case["op"] == "lookup":
        if case["w"] != "held":
            return torch.index_select(st["w"], 0, ids).double() * scale
        bits = case["kx"] + 2
        every = np.unpackbits(st["w"].cpu().numpy(), bitorder="little")[: case["rows"] * width * bits].reshape(-1, bits)
        level = every.astype(np.int64) @ (1 << np.arange(bits)) - (1 << case["kx"])
        table = torch.from_numpy(level.reshape(case["rows"], width)).cuda().double() / (2 << case["kx"])
        return table[ids] * scale
    here = ids >= 0
    order = torch.argsort(ids[here], stable=True)
    dw = torch.zeros(case["rows"], width, dtype=torch.float64, device="cuda")
    dw.index_put_((ids[here][order],), st["dy"][here][order].double(), accumulate=True)
    dw *= scale
    return dw + st["dw"].double() if case["add"] else dw
