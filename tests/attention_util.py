"""Plain 64-bit statements of the attention operators (head norms with rotation, attention within a window), and the share of
the kernels' 32-bit and tensor-core arithmetic in the errors of their results."""
import torch

from replica_util import ACC, EPS32, HALF_ULP, TINY


# ------------------------------------------------------------------ head norms with rotation

def pair_places(dim, rotary, pairing):
    """For each element its partner's place and the sign of the sine in its own turn, and the number of its pair (or -1)."""
    partner, sign, pair = torch.arange(dim), torch.zeros(dim, dtype=torch.float64), torch.full((dim,), -1)
    for i in range(rotary // 2):
        a, b = (i, i + rotary // 2) if pairing == "halves" else (2 * i, 2 * i + 1)
        partner[a], partner[b], sign[a], sign[b] = b, a, -1.0, 1.0
        pair[a] = pair[b] = i
    return partner, sign, pair


def turn64(x, positions, frequencies, pairing, back=False):
    """x [rows, heads, dim] turned by its rows' positions, and |x| + |partner| of the turned elements."""
    dim = x.shape[-1]
    rotary = 0 if frequencies is None else 2 * frequencies.numel()
    partner, sign, pair = (t.to(x.device) for t in pair_places(dim, rotary, pairing))
    if rotary == 0:
        return x, x.abs()
    angle = positions.double()[:, None] * frequencies.double()[pair.clamp(min=0)]
    cos = torch.where(pair >= 0, torch.cos(angle), 1.0)[:, None]
    sin = torch.where(pair >= 0, torch.sin(angle), 0.0)[:, None] * sign * (-1.0 if back else 1.0)
    other = x[..., partner]
    return x * cos + other * sin, torch.where(pair >= 0, x.abs() + other.abs(), x.abs())


def head_rotary64(x, w, positions, frequencies, pairing, eps):
    """y and the arithmetic's share of its error.  A mean of squares carries at most 24 roundings (16 terms a lane, 5 steps of
    the tree), half of which reach its root, the root's 4, two products; a turn 3 products and sums, and cosine and sine 6
    roundings of 1: the argument's pi, and theirs."""
    x = x.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    z = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w
    y, size = turn64(z, positions, frequencies, pairing)
    return y, 40 * EPS32 * size


def head_rotary_backward64(dy, x, w, positions, frequencies, pairing, eps):
    """(dx, error), (dw, error): the same roundings in dz = dy turned back and in h = x / norm; a mean of g h carries 24 more;
    the sum over rows and heads at most one rounding a term."""
    x, dy = x.double(), dy.double()
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    s = 1.0 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    dz, size = turn64(dy, positions, frequencies, pairing, back=True)
    h, g, most = x * s, dz * w, size * w.abs()
    dx = s * (g - h * (g * h).mean(-1, keepdim=True))
    e = 80 * EPS32 * s * (most + h.abs() * (most * h.abs()).mean(-1, keepdim=True))
    terms = x.shape[0] * x.shape[1]
    return (dx, e), ((dz * h).sum((0, 1)), (terms + 100) * EPS32 * (size * h.abs()).sum((0, 1)))


# ------------------------------------------------------------------ attention within a window

def visible(rows, bounds, left, right, sinks, device="cpu"):
    """[rows, rows] truth values: query i sees key j.  bounds: [(start, end), ...] of the sequences."""
    i, j = torch.arange(rows, device=device)[:, None], torch.arange(rows, device=device)[None]
    seen = torch.zeros(rows, rows, dtype=torch.bool, device=device)
    for start, end in bounds:
        inside = (i >= start) & (i < end) & (j >= start) & (j < end)
        seen |= inside & (j <= i + right) & ((j >= i - left) | (j < start + sinks))
    return seen


def _wide(t, heads):
    """[rows, some heads, dim] as [heads, rows, dim] in 64 bits."""
    return t.double().transpose(0, 1).repeat_interleave(heads // t.shape[1], 0)


def _hidden_as_zero(t):
    """Infinities and NaN, which only stand where nothing sees them, as zeros."""
    return torch.where(torch.isfinite(t), t, torch.zeros_like(t))


def attention64(q, k, v, seen, scale):
    """((out, error), (lse, error)), rows that see nothing as zeros.  A score's sum carries dim additions of the tensor cores; the
    exponential turns its error into a relative one and adds 2^-22 and, through its rounded argument, 2 roundings of the score's size;
    its result is rounded to the storage type (of a reference that makes the largest at least 1, so that half a subnormal
    weighs no more than that); sums over the keys add one addition a key."""
    heads, kind, n = q.shape[1], q.dtype, k.shape[0]
    q, k, v = (_hidden_as_zero(_wide(t, heads)) for t in (q, k, v))
    s = (scale * q @ k.mT).masked_fill(~seen, -torch.inf)
    some = seen.any(-1)[:, None]
    lse = torch.where(some, torch.logsumexp(s, -1, keepdim=True), 0.0)
    p = torch.where(seen, torch.exp(s - lse), 0.0)
    es = torch.where(seen, q.shape[-1] * ACC * scale * (q.abs() @ k.abs().mT) + 4 * EPS32 * (s.abs() + lse.abs()).nan_to_num(posinf=0.0), 0.0)
    out = p @ v
    rel = es + es.amax(-1, keepdim=True) + 2.0 ** -20 + n * ACC
    error = (p * (HALF_ULP[kind] + rel)) @ v.abs() + TINY[kind] * seen.double() @ v.abs()
    elog = es.amax(-1, keepdim=True) + (n + 8) * EPS32 + 4 * EPS32 * lse.abs()
    return (out.transpose(0, 1), error.transpose(0, 1)), (lse.squeeze(-1), elog.squeeze(-1))


def attention_backward64(dout, q, k, v, out, lse, seen, scale):
    """(dq, error), (dk, error), (dv, error) for given out and lse.  P and dS are rounded to the storage type; of half precision
    they carry powers of two: P 2^14, dS the one that takes its bound, twice the product of the longest rows of dout and v, to
    more than 2^14."""
    heads, kv_heads, kind, n = q.shape[1], k.shape[1], q.dtype, q.shape[0]
    longest = 2.0 * (_hidden_as_zero(dout).double().norm(dim=-1).max() * _hidden_as_zero(v).double().norm(dim=-1).max())
    dout, q, k, v, out = (_hidden_as_zero(_wide(t, heads)) for t in (dout, q, k, v, out))
    lse = lse.double()[..., None]
    s = scale * q @ k.mT
    p = torch.where(seen, torch.exp(s - lse), 0.0)
    dp, delta = dout @ v.mT, (dout * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    dim = q.shape[-1]
    rel = dim * ACC * scale * (q.abs() @ k.abs().mT) + 4 * EPS32 * (s.abs() + lse.abs()) + 2.0 ** -20
    most = dout.abs() @ v.abs().mT + (dout * out).abs().sum(-1, keepdim=True)
    eds = p * (dim * ACC * most + rel * (dp - delta).abs()) + HALF_ULP[kind] * ds.abs() + TINY[kind] * longest * 2.0 ** -14 * seen
    ep = p * (rel + HALF_ULP[kind]) + TINY[kind] * 2.0 ** -14 * seen

    def shared(t):
        return t.unflatten(0, (kv_heads, -1)).sum(1).transpose(0, 1)

    terms = n * (heads // kv_heads) * ACC
    dq = ((scale * ds @ k).transpose(0, 1), scale * (eds @ k.abs() + n * ACC * ds.abs() @ k.abs()).transpose(0, 1))
    dk = (shared(scale * ds.mT @ q), shared(scale * (eds.mT @ q.abs() + terms * ds.abs().mT @ q.abs())))
    dv = (shared(p.mT @ dout), shared(ep.mT @ dout.abs() + terms * p.mT @ dout.abs()))
    return dq, dk, dv
