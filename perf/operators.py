"""Measured cases of the replica operators: dropout, layer norm and the gated feed-forward product of
all M workers in one call, each in both directions.

``run`` computes an operator in its plain form (elementary torch operations in fp32, rounded once), or,
with ``own`` set, makes the library's call.  ``exact`` states the operators again in 64 bits.

A case holds, beside its operator: ``M`` workers, the storage ``type``, and
  dropout    n elements a worker, probability p, the seed and the offset of its random numbers
  layernorm  rows x cols a worker; ``pad`` elements between the end of a row and the next one; ``lead``
             elements that stand in front of gamma and beta in the worker's flat parameter vector
  ffn        rows x d_in inputs, d_hidden columns, the activation; ``lead`` as above, for the weights
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5


# ------------------------------------------------------------------ the cases

def listed():
    def dropout(name, way, M, n, kind, p, **kw):
        return dict(name=name, op="dropout", way=way, M=M, n=n, type=kind, p=p, **kw)

    def norm(name, way, M, rows, cols, kind, pad=0, lead=0):
        return dict(name=name, op="layernorm", way=way, M=M, rows=rows, cols=cols, type=kind, pad=pad, lead=lead)

    def ffn(name, way, M, rows, d_in, d_hidden, kind, act, lead=0):
        return dict(name=name, op="ffn", way=way, M=M, rows=rows, d_in=d_in, d_hidden=d_hidden, type=kind, act=act, lead=lead)

    return [
        # one token of width 768 in each of 4 replicas: the call's latency
        dropout("dropout fwd one token", "fwd", 4, 768, "bf16", 0.1, residual=True),
        # 32 images of 197 tokens of width 768, 8 replicas: the end of a transformer sub-layer
        dropout("dropout fwd vit batch", "fwd", 8, 32 * 197 * 768, "bf16", 0.1, residual=True),
        # an odd length in fp32: a classifier head's features
        dropout("dropout bwd odd fp32", "bwd", 3, 1_000_003, "f32", 0.5),
        # the largest: 64 images, 16 replicas
        dropout("dropout bwd large", "bwd", 16, 64 * 197 * 768, "bf16", 0.1),
        # one token again
        norm("layernorm fwd one token", "fwd", 4, 1, 768, "bf16"),
        # long sequences of a wide model
        norm("layernorm fwd wide", "fwd", 4, 8192, 4096, "bf16"),
        # one image, rows of odd length inside a padded buffer, gamma and beta at an odd place of the vector
        norm("layernorm bwd odd fp32", "bwd", 3, 197, 1001, "f32", pad=6, lead=11),
        # 32 images, 8 replicas
        norm("layernorm bwd vit batch", "bwd", 8, 32 * 197, 768, "bf16"),
        # a few tokens against all weights: bound by the weights' bytes; weights at an odd place
        ffn("ffn fwd few tokens", "fwd", 4, 5, 768, 2048, "bf16", "silu", lead=3),
        # one micro-batch of a mid-sized model
        ffn("ffn fwd large", "fwd", 4, 4096, 2048, 5632, "bf16", "silu"),
        # 8 images in each of 2 replicas, a hidden width that is not a multiple of any tile
        ffn("ffn bwd ragged", "bwd", 2, 8 * 197, 768, 2050, "f16", "gelu"),
        ffn("ffn bwd large", "bwd", 4, 4096, 2048, 5632, "bf16", "silu"),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op, way = rng.choice(["dropout", "layernorm", "ffn"]), rng.choice(["fwd", "bwd"])
    M = _log(rng, 1, 16)
    if op == "dropout":
        case = dict(op=op, way=way, M=M, n=_log(rng, 1000, 50_000_000 // M), type=rng.choice(["bf16", "f16", "f32"]),
                    p=rng.choice([0.05, 0.1, 0.2, 0.5]))
        if way == "fwd":
            case["residual"] = rng.random() < 0.7
        return case
    if op == "layernorm":
        cols = _log(rng, 64, 16384)
        if rng.random() < 0.6:
            cols = cols // 8 * 8
        rows = _log(rng, 1, max(2, min(65536, 40_000_000 // (M * cols))))
        return dict(op=op, way=way, M=M, rows=rows, cols=cols, type=rng.choice(["bf16", "f16", "f32"]),
                    pad=rng.choice([0, 0, 8, 3]), lead=rng.choice([0, 0, 10, 64]))
    while True:
        M, rows, d_in, d_hidden = _log(rng, 1, 8), _log(rng, 1, 8192), _log(rng, 32, 4096), _log(rng, 64, 8192)
        if M * rows * d_in * d_hidden <= 4 * 4096 * 2048 * 5632 // 2:
            break
    if rng.random() < 0.7:
        d_in, d_hidden = d_in // 8 * 8, d_hidden // 8 * 8
    return dict(op=op, way=way, M=M, rows=rows, d_in=d_in, d_hidden=d_hidden, type=rng.choice(["bf16", "f16"]),
                act=rng.choice(["silu", "gelu", "relu"]), lead=rng.choice([0, 0, 0, 10]))


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind, M = TYPES[case["type"]], case["M"]

    def normal(*shape, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=gen, device="cuda").mul_(scale).add_(shift).to(kind)

    def buffer(*shape):
        return torch.zeros(*shape, dtype=kind, device="cuda")

    s = dict(case)
    if case["op"] == "dropout":
        # activations, or the gradient that comes back from the sub-layers behind
        s["x"] = normal(M, case["n"], scale=1.0 if case["way"] == "fwd" else 1e-2)
        s["r"] = normal(M, case["n"]) if case.get("residual") else None
        s["y"] = buffer(M, case["n"])
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 ^ seed, 12345 + seed
    elif case["op"] == "layernorm":
        rows, cols, pad, lead = (case[k] for k in ("rows", "cols", "pad", "lead"))
        # rows with their own offset and scale, as the residual stream has them
        x = normal(M, rows, cols + pad, scale=1.0, shift=0.25)
        s["x"] = x.mul_(torch.rand(M, rows, 1, generator=gen, device="cuda").add_(0.5).to(kind))[..., :cols]
        flat = torch.cat([normal(M, lead), normal(M, cols, scale=0.02, shift=1.0), normal(M, cols, scale=0.02)], 1)
        s["gamma"], s["beta"] = flat[:, lead:lead + cols], flat[:, lead + cols:]
        if case["way"] == "fwd":
            s["y"] = buffer(M, rows, cols + pad)[..., :cols]
            s["mean"], s["rstd"] = (torch.zeros(M, rows, device="cuda") for _ in range(2))
        else:
            s["dy"] = normal(M, rows, cols + pad, scale=1e-2)[..., :cols]
            wide = s["x"].float()
            s["mean"] = wide.mean(-1)
            s["rstd"] = (wide - s["mean"][..., None]).square().mean(-1).add(EPS).rsqrt()
            s["dx"] = buffer(M, rows, cols + pad)[..., :cols]
            grads = buffer(M, lead + 2 * cols)
            s["dgamma"], s["dbeta"] = grads[:, lead:lead + cols], grads[:, lead + cols:]
    else:
        rows, d_in, d_hidden, lead = (case[k] for k in ("rows", "d_in", "d_hidden", "lead"))
        size = d_in * d_hidden
        s["x"] = normal(M, rows, d_in)
        flat = normal(M, lead + 2 * size, scale=d_in ** -0.5)
        s["w_gate"], s["w_up"] = (flat[:, lead + k * size:lead + (k + 1) * size].unflatten(1, (d_hidden, d_in)) for k in (0, 1))
        if case["way"] == "fwd":
            s["h"], s["gate"], s["up"] = (buffer(M, rows, d_hidden) for _ in range(3))
        else:
            s["dh"], s["gate"], s["up"] = normal(M, rows, d_hidden, scale=0.1), normal(M, rows, d_hidden), normal(M, rows, d_hidden)
            s["dx"] = buffer(M, rows, d_in)
            grads = buffer(M, lead + 2 * size)
            s["dw_gate"], s["dw_up"] = (grads[:, lead + k * size:lead + (k + 1) * size].unflatten(1, (d_hidden, d_in)) for k in (0, 1))
    # the workers' own buffers, as the library takes them: one entry per worker
    s["each"] = {k: list(v.unbind(0)) for k, v in s.items() if isinstance(v, torch.Tensor)}
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return {"dropout": _dropout, "layernorm": _layernorm, "ffn": _ffn}[s["op"]](s)


def _philox(seed, offset, M, n):
    """Philox4x32-10: key = seed, counter = (block low, block high + (worker << 24), offset low, offset high);
    element j of a worker takes word j % 4 of block j // 4.  Returns [M, n] int64 of 32-bit words."""
    low = 0xFFFFFFFF
    block = torch.arange((n + 3) // 4, device="cuda")
    worker = torch.arange(M, device="cuda")[:, None]
    c0, c1 = (block & low).expand(M, -1), (block >> 32) + (worker << 24)
    c2, c3 = torch.full_like(c1, offset & low), torch.full_like(c1, offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57           # 64-bit products; the shifts below drop the sign
        c0, c1, c2, c3 = (b >> 32 & low) ^ c1 ^ k0, b & low, (a >> 32 & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack([c0, c1, c2, c3], -1).reshape(M, -1)[:, :n]


def _dropout(s):
    if own:
        import paper_2403_04206_b200 as grawa
        t = s["each"]
        if s["way"] == "fwd":
            grawa.grawa_dropout_forward(t["x"], t["y"], s["p"], s["seed"], s["offset"], residual=t.get("r"))
        else:
            grawa.grawa_dropout_backward(t["x"], t["y"], s["p"], s["seed"], s["offset"])
        return s["y"]
    p = float(np.float32(s["p"]))
    keep = _philox(s["seed"], s["offset"], s["M"], s["n"]) >= math.floor(p * 2.0 ** 32 + 0.5)
    out = torch.where(keep, s["x"].float() * (1.0 / (1.0 - p)), 0.0)
    if s["r"] is not None:
        out = out + s["r"].float()
    return out.to(s["x"].dtype)


def _layernorm(s):
    if own:
        import paper_2403_04206_b200 as grawa
        t = s["each"]
        if s["way"] == "fwd":
            grawa.grawa_layernorm_forward(t["x"], t["gamma"], t["beta"], t["y"], EPS, mean=t["mean"], rstd=t["rstd"])
            return s["y"], s["mean"], s["rstd"]
        grawa.grawa_layernorm_backward(t["dy"], t["x"], t["gamma"], t["mean"], t["rstd"], t["dx"], t["dgamma"], t["dbeta"])
        return s["dx"], s["dgamma"], s["dbeta"]
    x, gamma = s["x"].float(), s["gamma"].float()[:, None]
    if s["way"] == "fwd":
        mean = x.mean(-1)
        centred = x - mean[..., None]
        rstd = (centred.square().mean(-1) + EPS).rsqrt()
        return (centred * rstd[..., None] * gamma + s["beta"].float()[:, None]).to(s["x"].dtype), mean, rstd
    dy, rstd = s["dy"].float(), s["rstd"][..., None]
    xhat = (x - s["mean"][..., None]) * rstd
    g = dy * gamma
    dx = (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)) * rstd
    return tuple(v.to(s["x"].dtype) for v in (dx, (dy * xhat).sum(1), dy.sum(1)))


def _act(name, g, slope=False):
    """The activation of the gate, or its derivative."""
    if name == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return sig * (1.0 + g * (1.0 - sig)) if slope else g * sig
    if name == "gelu":
        cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return cdf + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5 if slope else g * cdf
    return (g > 0).to(g.dtype) if slope else g * (g > 0)


def _ffn(s):
    if own:
        import paper_2403_04206_b200 as grawa
        t = s["each"]
        if s["way"] == "fwd":
            grawa.grawa_gated_ffn_forward(t["x"], t["w_gate"], t["w_up"], t["h"], activation=s["act"], gate_out=t["gate"], up_out=t["up"])
            return s["h"], s["gate"], s["up"]
        grawa.grawa_gated_ffn_backward(t["dh"], t["x"], t["w_gate"], t["w_up"], t["gate"], t["up"], t["dx"], t["dw_gate"], t["dw_up"],
                                       activation=s["act"])
        return s["dx"], s["dw_gate"], s["dw_up"]
    x, w_gate, w_up = s["x"].float(), s["w_gate"].float(), s["w_up"].float()
    if s["way"] == "fwd":
        gate, up = x @ w_gate.mT, x @ w_up.mT
        return tuple(v.to(s["x"].dtype) for v in (_act(s["act"], gate) * up, gate, up))
    dh, gate = s["dh"].float(), s["gate"].float()
    d_gate, d_up = dh * s["up"].float() * _act(s["act"], gate, slope=True), dh * _act(s["act"], gate)
    return tuple(v.to(s["x"].dtype) for v in (d_gate @ w_gate + d_up @ w_up, d_gate.mT @ x, d_up.mT @ x))


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    M, size, fwd = case["M"], 4 if case["type"] == "f32" else 2, case["way"] == "fwd"
    if case["op"] == "dropout":
        return {"bytes": size * M * case["n"] * (3 if case.get("residual") else 2), "flops": 2 * M * case["n"]}
    if case["op"] == "layernorm":
        elems = M * case["rows"] * case["cols"]
        vectors = M * case["cols"] * (2 if fwd else 3)           # gamma and beta, or gamma and both gradients
        return {"bytes": size * (elems * (2 if fwd else 3) + vectors) + 8 * M * case["rows"], "flops": elems * (8 if fwd else 14)}
    rows, d_in, d_hidden = case["rows"], case["d_in"], case["d_hidden"]
    weights, narrow, hidden = 2 * d_in * d_hidden, rows * d_in, rows * d_hidden
    moved = weights + narrow + 3 * hidden if fwd else 2 * weights + 2 * narrow + 3 * hidden
    return {"bytes": size * M * moved, "flops": (4 if fwd else 8) * M * rows * d_in * d_hidden}


# ------------------------------------------------------------------ the operators in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    wide = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "dropout":
        p = np.float64(np.float32(case["p"]))
        y = wide["x"].div_(1.0 - p)
        for m in range(case["M"]):
            words = _words(s["seed"], s["offset"], m, case["n"])
            y[m].masked_fill_(torch.from_numpy(words < np.uint64(np.floor(p * 4294967296.0 + 0.5))).cuda(), 0.0)
        return y if s["r"] is None else y.add_(wide["r"])
    if case["op"] == "layernorm":
        n, x = case["cols"], wide["x"]
        if case["way"] == "fwd":
            mean = x.sum(2) / n
            var = torch.einsum("mrc,mrc->mr", x, x) / n - mean * mean
            y = torch.einsum("mrc,mr,mc->mrc", x - mean.unsqueeze(2), 1.0 / torch.sqrt(var + EPS), wide["gamma"])
            return y + wide["beta"].unsqueeze(1), mean, 1.0 / torch.sqrt(var + EPS)
        xhat = torch.einsum("mrc,mr->mrc", x - wide["mean"].unsqueeze(2), wide["rstd"])
        t = wide["dy"] * wide["gamma"].unsqueeze(1)
        along = torch.einsum("mrc,mrc->mr", t, xhat) / n
        dx = torch.einsum("mrc,mr->mrc", t - (t.sum(2) / n).unsqueeze(2) - torch.einsum("mrc,mr->mrc", xhat, along), wide["rstd"])
        return dx, torch.einsum("mrc,mrc->mc", wide["dy"], xhat), wide["dy"].sum(1)

    def value_and_slope(g):
        if case["act"] == "silu":
            sig = torch.sigmoid(g)
            return g * sig, sig + g * sig * torch.sigmoid(-g)
        if case["act"] == "gelu":
            cdf = torch.special.ndtr(g)
            return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return torch.clamp(g, min=0.0), torch.where(g > 0, 1.0, 0.0)

    if case["way"] == "fwd":
        gate = torch.einsum("mtk,mfk->mtf", wide["x"], wide["w_gate"])
        up = torch.einsum("mtk,mfk->mtf", wide["x"], wide["w_up"])
        return value_and_slope(gate)[0] * up, gate, up
    value, slope = value_and_slope(wide["gate"])
    d_gate, d_up = wide["dh"] * wide["up"] * slope, wide["dh"] * value
    dx = torch.einsum("mtf,mfk->mtk", d_gate, wide["w_gate"]) + torch.einsum("mtf,mfk->mtk", d_up, wide["w_up"])
    return dx, torch.einsum("mtf,mtk->mfk", d_gate, wide["x"]), torch.einsum("mtf,mtk->mfk", d_up, wide["x"])


def _words(seed, offset, worker, n):
    """The 32-bit random words of one worker's n elements, from Philox4x32-10's published rounds (numpy, unsigned 64-bit)."""
    u, half = np.uint64, np.uint64(32)
    low = u(0xFFFFFFFF)
    out = np.empty(((n + 3) // 4, 4), np.uint32)
    for at in range(0, out.shape[0], 1 << 14):             # pieces that stay in the processor's cache
        b = np.arange(at, min(out.shape[0], at + (1 << 14)), dtype=u)
        x0, x1 = b & low, (b >> half) + u(worker << 24)
        x2, x3 = np.full_like(b, u(offset % 2 ** 32)), np.full_like(b, u(offset // 2 ** 32))
        key = [seed % 2 ** 32, seed // 2 ** 32]
        for _ in range(10):
            left, right = x0 * u(0xD2511F53), x2 * u(0xCD9E8D57)
            x0, x1 = (right >> half) ^ x1 ^ u(key[0]), right & low
            x2, x3 = (left >> half) ^ x3 ^ u(key[1]), left & low
            key = [(key[0] + 0x9E3779B9) % 2 ** 32, (key[1] + 0xBB67AE85) % 2 ** 32]
        for k, v in enumerate((x0, x1, x2, x3)):
            out[at:at + len(b), k] = v
    return out.reshape(-1)[:n]
