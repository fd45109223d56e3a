"""Attention over packed texts in 64 bits, text by text, with a bound on what an implementation in a 16-bit type may be
off by, element by element.

With u = 2^-p the unit roundoff of the type, every operand that is rounded to it (the weights, dX, out) is off by u of its
own size, and every result by u of its own.  A product of length K summed in fp32 is wrong by at most K 2^-23 sum |a b|
(the tensor core truncates; one rounding per term is more than it does).  The exponent of a weight is then off by
  e = 2^-23 (dim + 8) |scale| sum |q k| + 2^-22 (|x| + 4) + what the cap's tanh adds, cap 2^-21,
a weight by the factor 1 +- e for itself and the same for the sum it is divided by.  To each rounding is added what
is lost at the lower end of the type: in fp16 half the smallest subnormal step, 2^-25; in bf16 2^-126, the smallest normal
value of fp32, below which an exponential is 0 (a key 100 nats below its row's maximum has such a weight, and its gradient,
which is a sum of terms of that size, nothing else).
"""
import math

import torch

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 2.0 ** -126, "f16": 2.0 ** -25}


def scores(q, k, scale, cap, slope, lk_minus_lq):
    """x [heads][lq][lk] from q [lq][heads][dim] and k [lk][heads][dim] (key heads repeated), and sum |q k| * scale."""
    raw = torch.einsum("ihd,jhd->hij", q, k) * scale
    size = torch.einsum("ihd,jhd->hij", q.abs(), k.abs()) * scale
    x = cap * torch.tanh(raw / cap) if cap else raw
    if slope is not None:
        i, j = torch.arange(q.shape[0], device=q.device)[:, None], torch.arange(k.shape[0], device=q.device)
        x = x - slope.double()[:, None, None] * (i + lk_minus_lq - j).abs()
    return raw, x, size


def visible(lq, lk, causal, prefix, device):
    if not causal:
        return torch.ones(lq, lk, dtype=torch.bool, device=device)
    i, j = torch.arange(lq, device=device)[:, None], torch.arange(lk, device=device)
    return (j <= i + lk - lq) | (j < prefix)


def text(q, k, v, dout, dtype, scale, cap, slope, causal, prefix):
    """Results and bounds for one text: dicts of [rows][heads][dim] tensors; out, lse and, with dout, dq, dk, dv."""
    q, k, v = q.double(), k.double(), v.double()
    (lq, h, d), (lk, kv, _) = q.shape, k.shape
    g, u, tiny = h // kv, U[dtype], TINY[dtype]
    kr, vr = k.repeat_interleave(g, 1), v.repeat_interleave(g, 1)
    raw, x, size = scores(q, kr, scale, cap, slope, lk - lq)
    see = visible(lq, lk, causal, prefix, q.device)
    some = see.any(1)
    x = torch.where(see, x, -math.inf)
    lse = torch.logsumexp(x, -1) if lk else torch.full((h, lq), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(see & some[:, None], torch.exp(x - torch.where(some, lse, 0.0)[..., None]), 0.0)
    e = 2.0 ** -23 * (d + 8) * size + 2.0 ** -22 * (torch.where(see, x, 0.0).abs() + 4) + (cap * 2.0 ** -21 if cap else 0.0)
    e = torch.where(see, e, 0.0).amax(-1, keepdim=True) if lk else torch.zeros(h, lq, 1, dtype=torch.float64, device=q.device)
    ep = torch.where(see, p * 2 * e + 2.0 ** -126, 0.0)               # error of a weight, which below 2^-126 is 0
    o = torch.einsum("hij,jhd->ihd", p, vr)
    pv = torch.einsum("hij,jhd->ihd", p, vr.abs())
    acc = 2.0 ** -23 * (lk + 8)
    eo = torch.einsum("hij,jhd->ihd", ep + u * p + tiny, vr.abs()) + acc * pv
    r, b = {"out": o, "lse": lse}, {"out": u * (o.abs() + eo) + eo + tiny, "lse": e[..., 0] * 2 + 2.0 ** -21 * (lse.abs() + 4)}
    if dout is None:
        return r, b
    do = dout.double()
    dp = torch.einsum("ihd,jhd->hij", do, vr)
    edp = 2.0 ** -23 * d * torch.einsum("ihd,jhd->hij", do.abs(), vr.abs())
    delta = (do * o).sum(-1).T[..., None]
    edelta = (do.abs() * (b["out"] + 2.0 ** -23 * d * o.abs())).sum(-1).T[..., None]
    slack = 1 - torch.tanh(raw / cap) ** 2 if cap else torch.ones_like(raw)
    eslack = 2.0 ** -20 + 2 * (2.0 ** -23 * (d + 8) * size / cap) if cap else 0.0
    dx = p * (dp - delta) * slack
    edx = ep * (dp - delta).abs() * slack + p * (edp + edelta) + p * (dp - delta).abs() * eslack
    edx = edx + u * (dx.abs() + edx) + tiny                          # its rounding

    def product(eq, a, ea, other, f, n):
        val = torch.einsum(eq, a, other) * f
        err = (torch.einsum(eq, ea, other.abs()) + 2.0 ** -23 * (n + 8) * torch.einsum(eq, a.abs() + ea, other.abs())) * f
        return val, err

    def shared(t):                                                    # the sum over the heads of a key head
        return t.view(lk, kv, g, d).sum(2)

    for name, (val, err) in {"dq": product("hij,jhd->ihd", dx, edx, kr, scale, lk),
                             "dk": product("hij,ihd->jhd", dx, edx, q, scale, lq * g),
                             "dv": product("hij,ihd->jhd", p, ep + u * p + tiny, do, 1.0, lq * g)}.items():
        if name != "dq":
            val, err = shared(val), shared(err)
        r[name], b[name] = val, u * (val.abs() + err) + err + tiny
    return r, b
