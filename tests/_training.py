"""Plain statements of the operators around the quantized step, in numpy: AdamW with its 8-bit moments, one
operation per binary32 rounding or in binary64; the gradient norm; embedding rows and their gradient."""
import numpy as np

F = np.float32


def adamw_constants(beta1, beta2, lr, decay, t):
    b1, b2, lr = F(beta1), F(beta2), float(F(lr))
    return dict(b1=b1, b2=b2, c1=F(1) - b1, c2=F(1) - b2, keep=F(1 - lr * float(F(decay))),
                a=F(lr / (1 - float(b1) ** t)), b=F(1 / np.sqrt(1 - float(b2) ** t)))


def adamw32(x, m, v, g, k, eps, scale=None):
    """One step in binary32, one rounding per operation.  -> x, m, v"""
    with np.errstate(all="ignore"):
        g = g.astype(F)
        if scale is not None:
            g = g * F(scale)
        m = k["b1"] * m + k["c1"] * g
        v = k["b2"] * v + k["c2"] * (g * g)
        return x * k["keep"] - k["a"] * (m / (np.sqrt(v) * k["b"] + F(eps))), m, v


def adamw64(x, m, v, g, beta1, beta2, lr, decay, t, eps, scale=1.0):
    """The same step in binary64 from the binary32 hyper-parameters, and how far binary32 may be from it: each output's
    error bound, from half a unit in the last place per operation."""
    b1, b2, lr, decay, eps = (float(F(h)) for h in (beta1, beta2, lr, decay, eps))
    x, m, v, g = (np.asarray(a, dtype=np.float64) for a in (x, m, v, g))
    u = 2.0 ** -24
    g = g * float(scale)
    # 1 - beta is rounded once (it is exact for beta >= 1/2), g c once, the products and the sum once each
    em = 4 * u * (np.abs(b1 * m) + np.abs((1 - b1) * g))
    m = b1 * m + (1 - b1) * g
    ev = 6 * u * (b2 * v + (1 - b2) * g * g)
    v = b2 * v + (1 - b2) * g * g
    root = np.sqrt(v)
    d = root / np.sqrt(1 - b2 ** t) + eps
    a = lr / (1 - b1 ** t)
    # d: root 3 + 1, b and its product 2, the sum 1: 7 u; the quotient, a and the product 3 u
    ex = 3 * u * np.abs(x) + a * em / d + 12 * u * a * np.abs(m) / d
    x = x - lr * decay * x - a * m / d
    return (x, m, v), (ex + 3 * u * np.abs(x) + 2.0 ** -148, em + 2.0 ** -148, ev + 2.0 ** -147)


# ---------------------------------------------------------------- 8-bit moments

def philox(c, key):
    """Philox4x32-10 (Salmon et al., SC 2011): c: four uint64 arrays of 32-bit words."""
    c = [np.asarray(w, dtype=np.uint64) for w in c]
    k0, k1 = int(key) & 0xFFFFFFFF, int(key) >> 32
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64(k0), q & low, (p >> half) ^ c[3] ^ np.uint64(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def coins(off, n, t, seed):
    """The 16 random bits of elements 0 .. n - 1 of a tensor at padded offset off."""
    i = np.arange(n, dtype=np.int64)
    q = (off + 256 * (i // 256) + 4 * ((i % 128) // 4)) // 4
    word = philox([q & 0xFFFFFFFF, q >> 32, np.full(n, t & 0xFFFFFFFF), np.full(n, t >> 32)], seed)
    h = 4 * ((i // 128) % 2) + i % 4
    w = np.choose(h // 2, [x.astype(np.int64) for x in word])
    return np.where(h % 2 == 0, w & 0xFFFF, w >> 16)


def code_values(mantissa):
    """Magnitude of each code."""
    top, steps = (127, 8) if mantissa == 3 else (255, 16)
    assert steps == 2 ** mantissa
    out = [0.0]
    for c in range(1, top + 1):
        e, k = divmod(c - top, steps)
        out.append(2.0 ** e * (1 + k / steps))
    return np.array(out)


def encode_rows(x, mantissa, add, keep_positive):
    """x: [rows, 128] binary32 magnitudes; add: share of a step added before cutting off, [rows, 128] -> codes, scales."""
    scale = np.maximum(x.max(axis=1, keepdims=True), F(2.0 ** -126))
    y = (x * (F(1) / scale)).astype(np.float64)
    frac, e = np.frexp(y)
    steps, top = 2 ** mantissa, 127 if mantissa == 3 else 255
    k = np.floor((2 * frac - 1) * steps + add)
    code = np.where(y > 0, (e - 1) * steps + k + top, 0)
    code = np.maximum(code, ((x > 0) * 1 if keep_positive else 0))
    return np.minimum(code, top).astype(np.uint8), scale[:, 0]


def decode_m(code, scale):
    y = (code_values(3)[code & 127].astype(F) * scale[:, None]).astype(F)
    return np.where(code > 127, -y, y)


def decode_r(code, scale):
    return (code_values(4)[code].astype(F) * scale[:, None]).astype(F)


def adamw8(x, cm, sm, cr, sr, g, k, eps, off, t, seed, scale=None):
    """One step with 8-bit moments; all arrays padded to rows of 128.  -> x, cm, sm, cr, sr"""
    shape = (-1, 128)
    m = decode_m(cm.reshape(shape), sm)
    v = decode_r(cr.reshape(shape), sr)
    x, m, v = adamw32(x.reshape(shape), m, v * v, g.reshape(shape), k, eps, scale)
    h = coins(off, x.size, t, seed).reshape(shape)
    nm, zm = encode_rows(np.abs(m), 3, (2 * (h % 64) + 1) / 128, False)
    nm = (nm + 128 * np.signbit(m)).astype(np.uint8)
    nr, zr = encode_rows(np.sqrt(v), 4, (2 * (h // 64) + 1) / 2048, True)
    return x.reshape(-1), nm.reshape(-1), zm, nr.reshape(-1), zr


# ---------------------------------------------------------------- packed weights, embedding

def held_rows(wcodes, kx, first, rows, width):
    """[rows, width] binary64: element j is the code of bits [j b, (j + 1) b), code q + 2^kx worth q 2^-(kx + 1)."""
    b = kx + 2
    bits = np.unpackbits(wcodes, bitorder="little")[first * b:(first + rows * width) * b].reshape(-1, b)
    q = bits.astype(np.int64) @ (1 << np.arange(b)) - (1 << kx)
    return (q / 2.0 ** (kx + 1)).reshape(rows, width)


def embedding_grad64(ids, dy, rows, padding=-1):
    """-> sums in binary64, sums of magnitudes, tokens of each row"""
    ids = np.asarray(ids).reshape(-1)
    dy = np.asarray(dy, dtype=np.float64).reshape(ids.size, -1)
    live = (ids >= 0) & (ids < rows) & (ids != padding)
    total, size, n = np.zeros((rows, dy.shape[1])), np.zeros((rows, dy.shape[1])), np.zeros(rows, dtype=np.int64)
    np.add.at(total, ids[live], dy[live])
    np.add.at(size, ids[live], np.abs(dy[live]))
    np.add.at(n, ids[live], 1)
    return total, size, n
