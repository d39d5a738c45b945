"""Plain 64-bit statements of the replica operators, and the roundings their stored values may carry."""
import numpy as np
import torch

# torch.finfo(t).eps / 2, the largest relative error of one rounding, and half of the smallest subnormal
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
EPS32 = 2.0 ** -24                     # one fp32 rounding
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def bound(exact, kind, compute):
    """How far a stored value may be from `exact`: `compute` (the fp32 arithmetic) and the rounding of the store, which
    is taken of the value that the arithmetic gave."""
    return compute + HALF_ULP[kind] * (exact.abs() + compute) + TINY[kind]


def check(got, exact, kind, compute, what=""):
    assert got.dtype == kind
    err = (got.double() - exact).abs()
    lim = bound(exact, kind, compute)
    assert torch.isfinite(got.double()).all(), what
    over = err - lim
    assert (over <= 0).all(), f"{what}: off by {err.max().item():.3g}, allowed {lim.flatten()[over.argmax()].item():.3g}, got {got.flatten()[over.argmax()].item()}"


def philox_words(seed, offset, worker, blocks):
    """Words of Philox4x32-10 for an array of block numbers: [len(blocks), 4] uint32 (numpy, unsigned 64-bit)."""
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    b = np.asarray(blocks, dtype=u)
    c = [b & low, (b >> half) + u(worker << 24), np.full_like(b, u(offset % 2 ** 32)), np.full_like(b, u(offset >> 32))]
    k0, k1 = seed % 2 ** 32, seed >> 32
    for _ in range(10):
        p, q = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ u(k0), q & low, (p >> half) ^ c[3] ^ u(k1), p & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    return np.stack(c, -1).astype(np.uint32)


def keep_mask(seed, offset, worker, n, p):
    words = philox_words(seed, offset, worker, np.arange((n + 3) // 4)).reshape(-1)[:n]
    p = float(np.float32(p))
    return torch.from_numpy(words.astype(np.int64) >= int(np.floor(p * 2.0 ** 32 + 0.5)))


def dropout64(x, r, keep, p):
    p = float(np.float32(p))
    y = torch.where(keep, x.double() / (1.0 - p), torch.zeros((), dtype=torch.float64, device=x.device))
    return y if r is None else y + r.double()


def layernorm64(x, gamma, beta, eps):
    """y, mean, rstd and the arithmetic's share of y's error."""
    x = x.double()
    cols = x.shape[-1]
    mean = x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + eps)
    g = torch.ones(cols, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    b = torch.zeros(cols, dtype=torch.float64, device=x.device) if beta is None else beta.double()
    h = (x - mean) * rstd
    # The mean of |x| carries at most (elements a thread + steps of the tree) <= 64 roundings; it moves every
    # deviation, and through the variance h by a share of itself; the rest is a handful of roundings of h g and b.
    dmean = 64 * EPS32 * x.abs().mean(-1, keepdim=True)
    compute = (dmean * rstd) * (1 + h.abs()) * g.abs() + 80 * EPS32 * (h * g).abs() + 4 * EPS32 * b.abs()
    return h * g + b, mean.squeeze(-1), rstd.squeeze(-1), compute, dmean.squeeze(-1)


def layernorm_backward64(dy, x, gamma, mean, rstd):
    """dx, dgamma, dbeta for given fp32 statistics, each with the arithmetic's share of its error."""
    dy, x, mean, rstd = dy.double(), x.double(), mean.double()[:, None], rstd.double()[:, None]
    rows, cols = x.shape
    g = torch.ones(cols, dtype=torch.float64, device=x.device) if gamma is None else gamma.double()
    h, t = (x - mean) * rstd, dy * g
    mt, mth = t.mean(-1, keepdim=True), (t * h).mean(-1, keepdim=True)
    dx = rstd * (t - mt - h * mth)
    # row means: at most 64 roundings of sums of absolute values; then a handful for each product and difference
    e = 64 * EPS32 * (t.abs().mean(-1, keepdim=True) + h.abs() * (t * h).abs().mean(-1, keepdim=True))
    e = e + 8 * EPS32 * (t.abs() + mt.abs() + (h * mth).abs())
    # column sums: at most rows + 64 additions, and four roundings of each term
    n = (rows + 68) * EPS32
    return (dx, rstd * e), ((dy * h).sum(0), n * (dy * h).abs().sum(0)), (dy.sum(0), n * dy.abs().sum(0))


def activation64(name, a):
    """Value and slope of the gate's activation."""
    if name == "silu":
        s = torch.sigmoid(a)
        return a * s, s * (1.0 + a * (1.0 - s))
    if name == "gelu":
        c = 0.5 * (1.0 + torch.erf(a * 0.5 ** 0.5))
        return a * c, c + a * torch.exp(-0.5 * a * a) / (2.0 * np.pi) ** 0.5
    return torch.clamp(a, min=0.0), (a > 0).double()


ACC = 2.0 ** -23          # one addition of the tensor cores' fp32 accumulation, which may truncate
FAST = 2.0 ** -20         # relative error of an activation of magnitude one: a few units of the fast exponential and quotient


def gated_ffn64(act, x, wg, wu):
    """(h, error), (a, error), (u, error) with the arithmetic's share of the errors."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    k = x.shape[1] * ACC
    a, u = x @ wg.T, x @ wu.T
    ea, eu = k * (x.abs() @ wg.abs().T), k * (x.abs() @ wu.abs().T)
    f, _ = activation64(act, a)
    # slopes are below 1.13; the exponential's relative error grows with its argument
    h = f * u
    return (h, 1.13 * ea * u.abs() + f.abs() * eu + 1.13 * ea * eu + FAST * (1 + a.abs()) * h.abs()), (a, ea), (u, eu)


def gated_ffn_backward64(act, dh, x, wg, wu, a, u, kind):
    """(dx, error), (dwg, error), (dwu, error) for given 16-bit a and u."""
    dh, x, wg, wu, a, u = (t.double() for t in (dh, x, wg, wu, a, u))
    f, slope = activation64(act, a)
    da, du = dh * u * slope, dh * f
    # each of da and du carries its fp32 arithmetic and one rounding to the storage type
    ea = HALF_ULP[kind] * da.abs() + FAST * (1 + a.abs()) * (dh * u).abs() * 1.13 + TINY[kind]
    eu = HALF_ULP[kind] * du.abs() + FAST * (1 + a.abs()) * du.abs() + TINY[kind]
    rows, hidden = dh.shape
    out = []
    out.append((da @ wg + du @ wu, ea @ wg.abs() + eu @ wu.abs() + 2 * hidden * ACC * (da.abs() @ wg.abs() + du.abs() @ wu.abs())))
    for d, e in ((da, ea), (du, eu)):
        out.append((d.T @ x, e.T @ x.abs() + rows * ACC * (d.abs().T @ x.abs())))
    return out
