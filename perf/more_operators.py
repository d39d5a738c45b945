"""Measured cases of the attention operators of the replicas: norms of the query and key heads with the position
rotation, and attention within a window, each of all M workers in one call and in both directions.

``run`` computes an operator in its plain form (elementary torch operations in fp32, angles in 64 bits, rounded
once), or, with ``own`` set, makes the library's call.  ``exact`` states the operators again in 64 bits.

A case holds, beside its operator: ``M`` workers, ``rows`` tokens a worker, ``heads`` of the queries and
``kv_heads`` of the keys and values, ``dim`` elements a head, the storage ``type``, and
  rotary     ``turned`` leading elements of a head that are rotated, in pairs of neighbours or of halves; the
             positions count the tokens of sequences of ``period`` rows, or are a tensor's (``far``: up to that)
  attention  sequences of ``period`` rows, or, with ``packed`` (about how many), of random lengths behind each other
             with a few rows left over; keys up to ``left`` places back (-1: all) and ``right`` places ahead (-1: all) and
             the first ``sinks`` of the sequence
"""
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def listed():
    def rotary(name, way, M, rows, heads, kv_heads, dim, kind, turned=None, pairing="halves", period=4096, far=0):
        return dict(name=name, op="rotary", way=way, M=M, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, type=kind,
                    turned=dim if turned is None else turned, pairing=pairing, period=period, far=far)

    def attention(name, way, M, rows, heads, kv_heads, dim, kind, left=-1, right=0, sinks=0, period=0, packed=0):
        return dict(name=name, op="attention", way=way, M=M, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, type=kind,
                    left=left, right=right, sinks=sinks, period=period or rows, packed=packed)

    return [
        # one token of width 768 in each of 4 replicas: the call's latency
        rotary("rotary fwd one token", "fwd", 4, 1, 12, 12, 64, "bf16"),
        # two sequences of 4096 tokens in each of 4 replicas, shared key heads
        rotary("rotary fwd large", "fwd", 4, 8192, 32, 8, 128, "bf16"),
        # an odd number of tokens and heads in fp32, half of a head turned, positions far into a long text
        rotary("rotary bwd odd fp32", "bwd", 3, 197, 7, 7, 80, "f32", turned=40, far=1_000_000),
        # two sequences, neighbours turned
        rotary("rotary bwd large", "bwd", 4, 8192, 16, 4, 128, "bf16", pairing="neighbours"),
        # five tokens: latency
        attention("attention fwd few tokens", "fwd", 4, 5, 12, 12, 64, "bf16"),
        # 32 images of 197 tokens, 12 heads, every token sees its whole image
        attention("attention fwd vit batch", "fwd", 4, 32 * 197, 12, 12, 64, "f16", right=-1, period=197),
        # texts of all lengths packed into a row of 16384 tokens, a window with a few first tokens
        attention("attention fwd packed window", "fwd", 2, 16384, 16, 4, 128, "bf16", left=1023, sinks=4, packed=6),
        # one long text, all tokens before a token visible
        attention("attention fwd long", "fwd", 2, 8192, 16, 8, 128, "bf16"),
        attention("attention bwd vit batch", "bwd", 4, 32 * 197, 12, 12, 64, "f16", right=-1, period=197),
        # ragged in everything: heads of 80, three queries' heads a key's, short texts, a short window
        attention("attention bwd ragged", "bwd", 3, 1001, 6, 2, 80, "f16", left=99, sinks=3, packed=5),
        attention("attention bwd packed window", "bwd", 2, 16384, 16, 4, 128, "bf16", left=1023, sinks=4, packed=6),
        attention("attention bwd long", "bwd", 2, 8192, 16, 8, 128, "bf16"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op, way, M = rng.choice(["rotary", "attention"]), rng.choice(["fwd", "bwd"]), _log(rng, 1, 8)
    kv_heads = _log(rng, 1, 16)
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    if op == "rotary":
        dim = rng.choice([64, 128, 64, 128, 32, 80, 96, 8 * rng.randint(1, 32), rng.randint(4, 256)])
        rows = _log(rng, 1, max(2, min(16384, 150_000_000 // (M * (heads + kv_heads) * dim))))
        return dict(op=op, way=way, M=M, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, type=rng.choice(["bf16", "f16", "f32"]),
                    turned=rng.choice([dim // 2 * 2, dim // 2 * 2, dim // 4 * 2, 0]), pairing=rng.choice(["halves", "neighbours"]),
                    period=_log(rng, 16, 8192), far=rng.choice([0, 0, 100_000, 4_000_000]))
    while True:
        # (where every query sees one key, its own, the gradients of queries and keys are zero but for roundings: not drawn)
        dim, rows = rng.choice([64, 128, 64, 128, 32, 80, 96, 112, 8]), _log(rng, 1 if way == "fwd" else 8, 16384)
        left = rng.choice([-1, rng.randint(1, 64), _log(rng, 64, 4096)])
        right = rng.choice([0, 0, 0, -1, rng.randint(1, 200)])
        packed = rng.choice([0, min(_log(rng, 1, 64), (rows + 3) // 4)])
        period = rows if rng.random() < 0.5 else max(_log(rng, 1, rows), rows // 64, 2)
        case = dict(op=op, way=way, M=M, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, type=rng.choice(["bf16", "f16"]), left=left,
                    right=right, sinks=rng.choice([0, 0, 1, 4, rng.randint(1, 64)]), period=period, packed=packed)
        longest = rows if packed else min(rows, period)
        seen = (longest if left < 0 else left) + (longest if right < 0 else right)      # at most; half of it where all tokens before are
        if M * rows * heads <= 2 * 16384 * 16 and M * heads * rows * min(longest, seen) <= 2 * 16 * 8192 * (4096 if right else 8192):
            return case


# ------------------------------------------------------------------ inputs

def _lengths(case, seed, worker):
    """The lengths of a worker's sequences: together at most `rows`."""
    rows = case["rows"]
    if not case["packed"]:
        return [min(case["period"], rows - at) for at in range(0, rows, case["period"])]
    rng = random.Random(f"{seed} {worker}")
    rows -= min(rows // 50, 7)                               # rows behind the last sequence
    cuts = sorted(rng.randint(0, rows) for _ in range(case["packed"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [rows])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, M, rows, heads, kv_heads, dim = TYPES[case["type"]], *(case[k] for k in ("M", "rows", "heads", "kv_heads", "dim"))

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).to(kind)

    def buffer(*shape, kind=kind):
        return torch.zeros(*shape, dtype=kind, device="cuda")

    s = dict(case)
    if case["op"] == "rotary":
        # queries, keys and values as one projection leaves them, side by side in a row
        qkv = normal(M, rows, heads + 2 * kv_heads, dim).mul_(torch.rand(M, rows, 1, 1, generator=gen, device="cuda").add_(0.5).to(kind))
        s["q"], s["k"] = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads]
        # the weights stand somewhere in the workers' flat parameter vectors
        flat = normal(M, 3 + 2 * dim, scale=0.1).add_(1.0)
        s["q_weight"], s["k_weight"] = flat[:, 3:3 + dim], flat[:, 3 + dim:]
        s["positions"] = torch.randint(0, case["far"], (M, rows), generator=gen, device="cuda") if case["far"] else None
        turned = case["turned"]
        s["frequencies"] = 10000.0 ** (-torch.arange(0, turned, 2, dtype=torch.float64, device="cuda") / turned) if turned else None
        if case["way"] == "fwd":
            s["q_out"], s["k_out"] = buffer(M, rows, heads, dim), buffer(M, rows, kv_heads, dim)
        else:
            s["dq_out"], s["dk_out"] = normal(M, rows, heads, dim, scale=1e-2), normal(M, rows, kv_heads, dim, scale=1e-2)
            grads = buffer(M, rows, heads + 2 * kv_heads, dim)
            s["dq"], s["dk"] = grads[:, :, :heads], grads[:, :, heads:heads + kv_heads]
            flat = buffer(M, 3 + 2 * dim)
            s["dq_weight"], s["dk_weight"] = flat[:, 3:3 + dim], flat[:, 3 + dim:]
    else:
        # queries and keys behind the norm and the rotation, values beside them in the projection's rows
        s["q"], s["k"] = normal(M, rows, heads, dim), normal(M, rows, kv_heads, dim)
        s["v"] = normal(M, rows, heads + 2 * kv_heads, dim)[:, :, heads + kv_heads:]
        s["lengths"] = [_lengths(case, seed, m) for m in range(M)]
        ends = torch.tensor([[0] + n for n in s["lengths"]], dtype=torch.int64).cumsum(1)
        s["offsets"] = ends.cuda() if case["packed"] else None
        s["out"], s["lse"] = buffer(M, rows, heads, dim), buffer(M, heads, rows, kind=torch.float32)
        if case["way"] == "bwd":
            s["dout"] = normal(M, rows, heads, dim, scale=1e-2)
            out, s["lse"] = _attention_plain(s)
            s["out"].copy_(out)
            s["dq"], s["dk"] = buffer(M, rows, heads, dim), buffer(M, rows, kv_heads, dim)
            s["dv"] = buffer(M, rows, heads + 2 * kv_heads, dim)[:, :, heads + kv_heads:]
    # the workers' own buffers, as the library takes them: one entry per worker
    s["each"] = {k: list(v.unbind(0)) for k, v in s.items() if isinstance(v, torch.Tensor) and k != "frequencies"}
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return _rotary(s) if s["op"] == "rotary" else _attention(s)


def _rotary(s):
    if own:
        import paper_2403_04206_b200 as grawa
        t = s["each"]
        where = dict(positions=t.get("positions"), period=s["period"], pairing=s["pairing"], eps=EPS)
        if s["way"] == "fwd":
            grawa.grawa_head_rotary_forward(t["q"], t["k"], t["q_weight"], t["k_weight"], t["q_out"], t["k_out"], s["frequencies"], **where)
            return s["q_out"], s["k_out"]
        grawa.grawa_head_rotary_backward(t["dq_out"], t["dk_out"], t["q"], t["k"], t["q_weight"], t["k_weight"], t["dq"], t["dk"],
                                         t["dq_weight"], t["dk_weight"], s["frequencies"], **where)
        return s["dq"], s["dk"], s["dq_weight"], s["dk_weight"]
    kind, turned = s["q"].dtype, s["turned"]
    cos = sin = None
    if turned:
        at = s["positions"] if s["positions"] is not None else torch.arange(s["rows"], device="cuda").remainder(s["period"])[None]
        angle = (at.double()[..., None] * s["frequencies"])[:, :, None]
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turn(x, sign):
        """The leading `turned` elements as pairs (x, y), turned by the angle, or back."""
        if not turned:
            return x
        lead = x[..., :turned]
        a, b = (lead[..., 0::2], lead[..., 1::2]) if s["pairing"] == "neighbours" else lead.chunk(2, -1)
        a, b = a * cos - sign * b * sin, b * cos + sign * a * sin
        lead = torch.stack([a, b], -1).flatten(-2) if s["pairing"] == "neighbours" else torch.cat([a, b], -1)
        return torch.cat([lead, x[..., turned:]], -1)

    outs, weights = [], []
    for name in ("q", "k"):
        x, w = s[name].float(), s[name + "_weight"].float()[:, None, None]
        rms = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
        if s["way"] == "fwd":
            outs.append(turn(x * rms * w, 1).to(kind))
            continue
        dz, xhat = turn(s["d" + name + "_out"].float(), -1), x * rms
        g = dz * w
        outs.append(((g - xhat * (g * xhat).mean(-1, keepdim=True)) * rms).to(kind))
        weights.append((dz * xhat).sum((1, 2)).to(kind))
    return tuple(outs + weights)


def _attention(s):
    if own:
        import paper_2403_04206_b200 as grawa
        t = s["each"]
        mask = dict(offsets=t.get("offsets"), period=s["period"], left=None if s["left"] < 0 else s["left"],
                    right=None if s["right"] < 0 else s["right"], sinks=s["sinks"])
        if s["way"] == "fwd":
            grawa.grawa_window_attention_forward(t["q"], t["k"], t["v"], t["out"], lse=t["lse"], **mask)
            return s["out"], s["lse"]
        grawa.grawa_window_attention_backward(t["dout"], t["q"], t["k"], t["v"], t["out"], t["lse"], t["dq"], t["dk"], t["dv"], **mask)
        return s["dq"], s["dk"], s["dv"]
    return _attention_plain(s) if s["way"] == "fwd" else _attention_plain_gradients(s)


def _blocks(s, m):
    """Blocks of a worker's query rows: (first, last + 1, rows of the keys that any of them sees, mask [queries, keys])."""
    lengths, rows = s["lengths"][m], s["rows"]
    left, right = (rows if s[k] < 0 else s[k] for k in ("left", "right"))
    at = 0
    for n in lengths:
        first, at = at, at + n
        size = max(128, min(1024, 2 ** 27 // (4 * s["heads"] * max(1, min(n, left + right + 1024)))))
        for a in range(first, at, size):
            b = min(a + size, at)
            low, high = max(first, a - left), min(at, b + right)
            sinks = min(first + s["sinks"], low)
            keys = torch.cat([torch.arange(first, sinks, device="cuda"), torch.arange(low, high, device="cuda")]) if sinks > first else \
                torch.arange(low, high, device="cuda")
            i = torch.arange(a, b, device="cuda")[:, None]
            yield a, b, keys, ((keys >= i - left) | (keys < first + s["sinks"])) & (keys <= i + right)


def _block(s, m, a, b, keys, name):
    """Rows of an operand in fp32, [kv_heads, queries' heads of each, rows, dim]: queries' rows a to b, or keys' rows."""
    x = s[name][m]
    if name in ("k", "v"):
        return (x[keys[0]:keys[0] + len(keys)] if not s["sinks"] else x[keys]).float().transpose(0, 1)[:, None]
    return x[a:b].float().transpose(0, 1).unflatten(0, (s["kv_heads"], -1))


def _scores(s, m, a, b, keys, mask):
    q, k = _block(s, m, a, b, keys, "q"), _block(s, m, a, b, keys, "k")
    return q, k, (q @ k.mT).mul_(s["dim"] ** -0.5).masked_fill_(~mask, -math.inf)


def _attention_plain(s):
    out, lse = torch.zeros_like(s["out"]), torch.zeros_like(s["lse"])
    for m in range(s["M"]):
        for a, b, keys, mask in _blocks(s, m):
            score = _scores(s, m, a, b, keys, mask)[2]
            top = score.amax(-1, keepdim=True)
            p = score.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            o = (p @ _block(s, m, a, b, keys, "v")) / total
            out[m, a:b] = o.flatten(0, 1).transpose(0, 1).to(out.dtype)
            lse[m, :, a:b] = (top + total.log()).flatten(0, 1).squeeze(-1)
    return out, lse


def _attention_plain_gradients(s):
    wide = {k: torch.zeros(s[k].shape, device="cuda") for k in ("dq", "dk", "dv")}
    for m in range(s["M"]):
        for a, b, keys, mask in _blocks(s, m):
            q, k, score = _scores(s, m, a, b, keys, mask)
            v, dout, out = (_block(s, m, a, b, keys, name) for name in ("v", "dout", "out"))
            p = score.sub_(s["lse"][m, :, a:b].unflatten(0, (s["kv_heads"], -1))[..., None]).exp_()
            ds = (dout @ v.mT).sub_((dout * out).sum(-1, keepdim=True)).mul_(p)
            scale = s["dim"] ** -0.5
            wide["dq"][m, a:b] = (ds @ k).mul_(scale).flatten(0, 1).transpose(0, 1)
            dk, dv = (ds.mT @ q).mul_(scale).sum(1), (p.mT @ dout).sum(1)
            wide["dk"][m].index_add_(0, keys, dk.transpose(0, 1))
            wide["dv"][m].index_add_(0, keys, dv.transpose(0, 1))
    return tuple(wide[k].to(s[k].dtype) for k in ("dq", "dk", "dv"))


# ------------------------------------------------------------------ what a pass cannot do without

def _pairs(case):
    """Pairs of a query and a key that it sees, in one head of one worker (of about equal lengths where they are random)."""
    rows = case["rows"]
    n = max(1, rows // case["packed"]) if case["packed"] else min(case["period"], rows)
    left, right = (n if case[k] < 0 else case[k] for k in ("left", "right"))
    back = sum(min(i, left) for i in range(n))
    ahead = sum(min(n - 1 - i, right) for i in range(n))
    far = sum(min(case["sinks"], max(0, i - left)) for i in range(n))
    return (n + back + ahead + far) * max(1, rows // n)


def work(case):
    M, rows, heads, kv_heads, dim = (case[k] for k in ("M", "rows", "heads", "kv_heads", "dim"))
    fwd, size = case["way"] == "fwd", 4 if case["type"] == "f32" else 2
    if case["op"] == "rotary":
        elems = M * rows * (heads + kv_heads) * dim
        weights = M * dim * (2 if fwd else 4)
        return {"bytes": size * (elems * (2 if fwd else 3) + weights) + (8 * M * rows if case["far"] else 0), "flops": elems * (7 if fwd else 14)}
    wide, narrow = M * rows * heads * dim, M * rows * kv_heads * dim
    moved = 2 * wide + 2 * narrow if fwd else 4 * wide + 4 * narrow
    return {"bytes": size * moved + 4 * M * rows * heads, "flops": (4 if fwd else 10) * M * heads * dim * _pairs(case)}


# ------------------------------------------------------------------ the operators in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rotary(s) if case["op"] == "rotary" else _exact_attention(s)


def _exact_rotary(s):
    """With complex numbers: a pair (x, y) is x + iy, and a turn is a product with exp(i angle)."""
    M, rows, dim, half = s["M"], s["rows"], s["dim"], s["turned"] // 2
    if half:
        position = s["positions"].double() if s["positions"] is not None else (torch.arange(rows, device="cuda") % s["period"]).double().expand(M, rows)
        factor = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.einsum("mr,f->mrf", position, s["frequencies"]))[:, :, None]
    index = torch.arange(2 * half, device="cuda")
    real, imag = (index[0::2], index[1::2]) if s["pairing"] == "neighbours" else (index[:half], index[half:])

    def turn(x, by):
        y = x.clone()
        if half:
            z = torch.complex(x[..., real], x[..., imag]) * by
            y[..., real], y[..., imag] = z.real, z.imag
        return y

    first, second = [], []
    for name in ("q", "k"):
        x, w = s[name].double(), s[name + "_weight"].double().view(M, 1, 1, dim)
        norm = torch.sqrt(torch.einsum("mrhd,mrhd->mrh", x, x) / dim + EPS).unsqueeze(3)
        if s["way"] == "fwd":
            first.append(turn(w * (x / norm), factor if half else None))
            continue
        dz = turn(s["d" + name + "_out"].double(), factor.conj() if half else None)
        along = torch.einsum("mrhd,mrhd->mrh", dz * w, x).unsqueeze(3)
        first.append(dz * w / norm - x * along / (dim * norm ** 3))
        second.append(torch.einsum("mrhd,mrhd->md", dz, x / norm))
    return tuple(first + second)


def _exact_attention(s):
    """Sequence by sequence, with the whole matrix of scores of a few heads at a time."""
    M, heads, dim, fwd = s["M"], s["heads"], s["dim"], s["way"] == "fwd"
    group = heads // s["kv_heads"]
    result = {k: torch.zeros(s[k].shape, dtype=torch.float64, device="cuda") for k in (("out", "lse") if fwd else ("dq", "dk", "dv"))}
    for m in range(M):
        start = 0
        for n in s["lengths"][m]:
            rows = slice(start, start + n)
            start += n
            if n == 0:
                continue
            place = torch.arange(n, device="cuda")
            back = place.unsqueeze(1) - place.unsqueeze(0)    # how far the key lies behind the query
            hidden = torch.zeros(n, n, dtype=torch.bool, device="cuda")
            if s["left"] >= 0:
                hidden |= (back > s["left"]) & (place >= s["sinks"]).unsqueeze(0)
            if s["right"] >= 0:
                hidden |= -back > s["right"]
            step = max(1, min(heads, 2 ** 26 // (n * n)))
            for h in range(0, heads, step):
                mine = torch.arange(h, min(h + step, heads), device="cuda")
                q = s["q"][m, rows][:, mine].double()
                k, v = (s[name][m, rows][:, mine // group].double() for name in ("k", "v"))
                score = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(dim)
                score[:, hidden] = -math.inf
                if fwd:
                    lse = torch.logsumexp(score, 2)
                    result["lse"][m, mine, rows] = lse
                    result["out"][m, rows, h:h + len(mine)] = torch.einsum("hij,jhd->ihd", torch.exp(score - lse.unsqueeze(2)), v)
                    continue
                dout, out = (s[name][m, rows][:, mine].double() for name in ("dout", "out"))
                p = torch.exp(score - s["lse"][m, mine, rows].double().unsqueeze(2))
                ds = p * (torch.einsum("ihd,jhd->hij", dout, v) - torch.einsum("ihd,ihd->hi", dout, out).unsqueeze(2))
                result["dq"][m, rows, h:h + len(mine)] = torch.einsum("hij,jhd->ihd", ds, k) / math.sqrt(dim)
                result["dk"][m, rows].index_add_(1, mine // group, torch.einsum("hij,ihd->jhd", ds, q) / math.sqrt(dim))
                result["dv"][m, rows].index_add_(1, mine // group, torch.einsum("hij,ihd->jhd", p, dout))
    return tuple(result.values())
