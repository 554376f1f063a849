"""Plain statements in binary64 of layer norm, its gradients and rows in 8 bits, with bounds of what binary32 may differ by."""
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # half a step, relative
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -25}   # half the smallest step, or more
U = 2.0 ** -24


def depth(width):
    """Additions one after the other in a sum over a row: at most 32 in a thread (a 1024th of a row wider than 32768), then a
    tree of 5 over the warp and 5 over the warps."""
    return max(32, -(-width // 1024)) + 10


def norm64(h, w, b, eps):
    """-> y, mean, rstd, and the bound of y's error, for h [rows, width] in binary64 (exact inputs)."""
    n = h.shape[1]
    mean = h.mean(1, keepdim=True)
    d = h - mean
    rstd = 1 / torch.sqrt(d.square().mean(1, keepdim=True) + eps)
    w = torch.ones(n, dtype=torch.float64, device=h.device) if w is None else w.double()
    b = torch.zeros(n, dtype=torch.float64, device=h.device) if b is None else b.double()
    xhat = d * rstd
    y = xhat * w + b
    k = depth(n) + 2
    mean_off = k * U * h.abs().mean(1, keepdim=True)              # sum, quotient
    # sum of squares: k roundings each side, and twice the difference's (U |d| + mean_off) on every d, which sums to 2 U and
    # the square of mean_off; a root halves what is relative; quotient, sum, root, reciprocal 4 more
    rstd_off = 0.5 * (k + 6) * U + (mean_off * rstd).square() + 4 * U
    off = (mean_off * rstd + xhat.abs() * (2 * U + rstd_off)) * w.abs() + U * y.abs()
    return y, mean[:, 0], rstd[:, 0], off * 1.01, mean_off[:, 0] * 1.01, rstd[:, 0] * rstd_off[:, 0] * 1.01


def grad64(dy, x, mean, rstd, w, ds):
    """-> dx, dw, db and their bounds before any rounding to a type (dw, db: of a sum in any order of at most `rows` additions
    is left to the caller: the sums of magnitudes are given)."""
    n = x.shape[1]
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    xhat = (x - mean) * rstd                                      # 2 roundings
    g = dy * w.double() if w is not None else dy                  # 1
    along, whole = (g * xhat).mean(1, keepdim=True), g.mean(1, keepdim=True)
    dx = rstd * (g - whole - xhat * along)
    k = depth(n) + 6
    off = rstd * U * (3 * g.abs() + k * g.abs().mean(1, keepdim=True) + xhat.abs() * k * (g * xhat).abs().mean(1, keepdim=True)
                      + 3 * (whole.abs() + (xhat * along).abs()))
    if ds is not None:
        dx = dx + ds.double()
    off = (off + U * dx.abs()) * 1.01
    return dx, (dy * xhat).sum(0), dy.sum(0), off, (dy * xhat).abs().sum(0), dy.abs().sum(0)


def rows8(x, columns=None):
    """q, scale by the definition: quotient and product rounded to binary32 (binary64 holds the product and decides the
    quotient's rounding), for x of any type."""
    x = x.double()
    if columns is not None:
        x = (x * columns.double()).float().double()
    a = x.abs().amax(1, keepdim=True).clamp(min=2.0 ** -100)
    per = (127.0 / a).float().double()
    q = torch.round((x * per).float()).double()
    scale = (a / 127.0).float()[:, 0]
    bad = ~torch.isfinite(x).all(1)
    q[bad] = 0
    scale[bad] = float("nan")
    return q.to(torch.int8), scale


def pack(level, kx):
    """Levels [any] as packed codes, padded to 128 elements."""
    b = kx + 2
    level = level.reshape(-1).to(torch.int64)
    code = torch.zeros(-(-level.numel() // 128) * 128, dtype=torch.int64, device=level.device)
    code[:level.numel()] = level + (1 << kx)
    bits = (code[:, None] >> torch.arange(b, device=level.device)) & 1
    return (bits.reshape(-1, 8) << torch.arange(8, device=level.device)).sum(1).to(torch.uint8)


def randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda")


def gen_of(*parts):
    return torch.Generator(device="cuda").manual_seed(sum((i + 1) * int(p) for i, p in enumerate(parts)))
