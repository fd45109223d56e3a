"""The operators of training and serving a text model, as cases that can be timed: token embedding with its gradient,
the gated feed-forward block with its backward pass, and the global gradient norm with clipping over many tensors.

`own` chooses what `run` computes with: elementary torch operations in 32 bits (False), or the library's entry points
(True).  Both take the same state.
"""
import math

import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ctx = None


def _lib():
    from paper_2310_05674_b200 import binding
    return binding


def _context():
    """One library context per process, as a program keeps it (its workspaces grow to the largest call)."""
    global _ctx
    if _ctx is None:
        _ctx = _lib().sama_create(0, 1 << 20, 0, None)
    return _ctx


# ----------------------------------------------------------------------------------------------------- the cases

def listed():
    return [
        # one decode step's lookup for a batch of 32 sequences: pure latency
        {"name": "embed-serve-32", "op": "embed", "tokens": 32, "vocab": 32768, "d": 1024, "dtype": "bf16",
         "grad": "none"},
        # a small fp32 classifier's training step: 16 texts of 128 tokens, odd vocabulary, gradient in fp32
        {"name": "embed-train-2k", "op": "embed", "tokens": 2048, "vocab": 8191, "d": 256, "dtype": "f32",
         "grad": "f32"},
        # a fine-tuning step of width 1024: 16k tokens, bf16 activations, gradient straight into the fp32 flat vector
        {"name": "embed-train-16k", "op": "embed", "tokens": 16384, "vocab": 50021, "d": 1024, "dtype": "bf16",
         "grad": "f32"},
        # a pretraining step's micro-batch: 131k tokens (ragged), wide rows, gradient in the parameters' type
        {"name": "embed-train-131k", "op": "embed", "tokens": 131007, "vocab": 65536, "d": 2048, "dtype": "bf16",
         "grad": "bf16"},
        # one token of one sequence: the weights are streamed once
        {"name": "ffn-serve-1", "op": "ffn", "tokens": 1, "d": 4096, "f": 8192, "dtype": "bf16", "act": "silu",
         "train": False},
        # a decode step of 45 sequences
        {"name": "ffn-serve-45", "op": "ffn", "tokens": 45, "d": 4096, "f": 8192, "dtype": "bf16", "act": "silu",
         "train": False},
        # the smallest training step: the tiny model's batch and width, half precision
        {"name": "ffn-train-128", "op": "ffn", "tokens": 128, "d": 256, "f": 688, "dtype": "f16", "act": "gelu",
         "train": True},
        # sizes that are a multiple of nothing: every row starts at another alignment
        {"name": "ffn-train-odd", "op": "ffn", "tokens": 1003, "d": 1001, "f": 2731, "dtype": "bf16",
         "act": "gelu_tanh", "train": True},
        # the widest model of the benchmark (width 4096) on 4096 tokens: bound by the tensor cores
        {"name": "ffn-train-4096", "op": "ffn", "tokens": 4096, "d": 4096, "f": 8192, "dtype": "bf16", "act": "silu",
         "train": True},
        # the tiny model's four gradient tensors (784-256-10): pure latency
        {"name": "clip-tiny", "op": "clip", "layers": 0, "width": 256, "vocab": 784, "matrix": "f32",
         "vector": "f32", "flat": True, "max_norm": 1.0},
        # 110 M elements, 16 layers: bf16 matrices and fp32 vectors gathered into the flat fp32 gradient
        {"name": "clip-110m", "op": "clip", "layers": 16, "width": 640, "vocab": 49001, "matrix": "bf16",
         "vector": "f32", "flat": True, "max_norm": 1.0},
        # 355 M elements, 24 layers, all fp32, every output in its tensor's own type
        {"name": "clip-355m", "op": "clip", "layers": 24, "width": 1024, "vocab": 51200, "matrix": "f32",
         "vector": "f32", "flat": False, "max_norm": 1.0},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["embed", "ffn", "clip"])
    if op == "embed":
        while True:
            c = {"op": op, "tokens": _log(rng, 1, 131072), "vocab": _log(rng, 50, 131072), "d": _log(rng, 8, 4096)}
            if rng.random() < 0.6:
                c["d"] = -(-c["d"] // 8) * 8
            if (2 * c["tokens"] + c["vocab"]) * c["d"] <= 2 * 131007 * 2048 and c["d"] != 3072:
                break
        c["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32"])
        c["grad"] = rng.choice(["none", "f32", c["dtype"], c["dtype"]])
        return c
    if op == "ffn":
        while True:
            d = _log(rng, 48, 4096)
            c = {"op": op, "tokens": _log(rng, 1, 4096), "d": d, "f": int(d * rng.uniform(1.5, 4.0))}
            if rng.random() < 0.6:
                c["d"], c["f"] = -(-c["d"] // 16) * 16, -(-c["f"] // 16) * 16
            if c["tokens"] * c["d"] * c["f"] <= 4096 * 4096 * 8192 and 3072 not in (c["d"], c["f"]):
                break
        c["dtype"] = rng.choice(["bf16", "bf16", "f16"])
        c["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"])
        c["train"] = rng.random() < 0.6
        return c
    while True:
        c = {"op": op, "layers": rng.randint(0, 24), "width": _log(rng, 17, 1024), "vocab": _log(rng, 50, 60000)}
        if sum(math.prod(s) for s in _shapes(c)) <= 353_000_000 and 768 != c["width"]:
            break
    c["matrix"] = rng.choice(["bf16", "f16", "f32"])
    c["vector"] = rng.choice([c["matrix"], "f32"])
    c["flat"] = rng.random() < 0.5
    c["max_norm"] = rng.choice([0.1, 1.0, 1.0, 1e4])
    return c


def _shapes(case):
    """Shapes of an encoder's parameters (or, with no layers, of a two-layer classifier), in registration order."""
    w, v = case["width"], case["vocab"]
    if case["layers"] == 0:
        return [(w, v), (w,), (10, w), (10,)]
    layer = [(w, w), (w,), (w, w), (w,), (w, w), (w,), (w, w), (w,), (w,), (w,), (4 * w, w), (4 * w,), (w, 4 * w), (w,),
             (w,), (w,)]
    return [(v, w)] + layer * case["layers"] + [(w,), (w,)]


def _kind(shape):
    return "matrix" if len(shape) == 2 else "vector"


# ------------------------------------------------------------------------------------------------- inputs and plan

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)


def prepare(case, seed):
    g = _gen(seed)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    if case["op"] == "embed":
        dt, t, v, d = _DT[case["dtype"]], case["tokens"], case["vocab"], case["d"]
        # token frequencies fall as 1 / rank, as in text: rank = V^u
        u = torch.rand(t, generator=g, device="cuda", dtype=torch.float64)
        st = {"ids": (torch.exp(u * math.log(v)) - 1.0).clamp(0, v - 1).to(torch.int32),
              "table": (0.02 * randn(v, d)).to(dt), "scale": math.sqrt(d)}
        if case["grad"] != "none":
            st["dout"] = (1e-2 * randn(t, d)).to(dt)
        if own:
            st["out"] = torch.empty(t, d, dtype=dt, device="cuda")
            if case["grad"] != "none":
                st["grad"] = torch.empty(v, d, dtype=_DT[case["grad"]], device="cuda")
    elif case["op"] == "ffn":
        dt, t, d, f = _DT[case["dtype"]], case["tokens"], case["d"], case["f"]
        st = {"x": randn(t, d).to(dt), "wg": (randn(f, d) / math.sqrt(d)).to(dt), "wu": (randn(f, d) / math.sqrt(d)).to(dt),
              "wd": (randn(d, f) / math.sqrt(f)).to(dt)}
        if case["train"]:
            st["dy"] = randn(t, d).to(dt)
        if own:
            st["y"] = torch.empty_like(st["x"])
            if case["train"]:
                st["gate"], st["up"] = (torch.empty(t, f, dtype=dt, device="cuda") for _ in range(2))
                st["dx"] = torch.empty_like(st["x"])
                st["dw"] = [torch.empty_like(st[k]) for k in ("wg", "wu", "wd")]
    else:
        shapes = _shapes(case)
        scale = [1e-3 * 10.0 ** (i % 3) for i in range(len(shapes))]
        kind = [_DT[case[_kind(s)]] for s in shapes]
        st = {"grads": [(a * randn(*s)).to(k) for s, a, k in zip(shapes, scale, kind)]}
        if own:
            if case["flat"]:
                st["flat"] = torch.empty(sum(x.numel() for x in st["grads"]), device="cuda")
                st["outs"] = [y.view(x.shape) for x, y in
                              zip(st["grads"], st["flat"].split([x.numel() for x in st["grads"]]))]
            else:
                # each tensor's output in its own type, packed by kind: the matrices in one buffer, the vectors in another
                for k in ("matrix", "vector"):
                    size = [x.numel() for x, s in zip(st["grads"], shapes) if _kind(s) == k]
                    st[k] = torch.empty(sum(size), dtype=_DT[case[k]], device="cuda")
                    st[k + "_parts"] = iter(st[k].split(size))
                st["outs"] = [next(st[_kind(s) + "_parts"]).view(s) for s in shapes]
            st["list"] = _lib().TensorList(st["grads"], st["outs"])
            st["norm"] = torch.empty((), device="cuda")
    st["case"] = case
    if own:
        st["ctx"] = _context()
    return st


# ------------------------------------------------------------------------------------------------------ one pass

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _embed_plain(st):
    dt = st["table"].dtype
    ids = st["ids"].long()
    out = (st["table"][ids].float() * st["scale"]).to(dt)
    if "dout" not in st:
        return {"out": out}
    grad = torch.zeros(st["table"].shape, device="cuda")
    grad.index_add_(0, ids, st["dout"].float() * st["scale"])
    return {"out": out, "grad": grad.to(_DT[st["case"]["grad"]])}


def _act(kind, g):
    """The activation and its derivative."""
    if kind == "relu":
        pos = (g > 0).to(g.dtype)
        return g * pos, pos
    if kind == "silu":
        s = 1.0 / (1.0 + torch.exp(-g))
        return g * s, s * (1.0 + g * (1.0 - s))
    if kind == "gelu":
        p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))
    a = math.sqrt(2.0 / math.pi)
    th = torch.tanh(a * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * g * (1.0 - th * th) * a * (1.0 + 0.134145 * g * g)


def _ffn_plain(st):
    dt = st["x"].dtype
    x, wg, wu, wd = (st[k].float() for k in ("x", "wg", "wu", "wd"))
    gate, up = x @ wg.T, x @ wu.T
    a, da = _act(st["case"]["act"], gate)
    h = a * up
    y = (h @ wd.T).to(dt)
    if "dy" not in st:
        return {"y": y}
    dy = st["dy"].float()
    dh = dy @ wd
    dgate, dup = dh * up * da, dh * a
    return {"y": y, "dx": (dgate @ wg + dup @ wu).to(dt), "dwg": (dgate.T @ x).to(dt), "dwu": (dup.T @ x).to(dt),
            "dwd": (dy.T @ h).to(dt)}


def _clip_plain(st):
    grads = [g.float() for g in st["grads"]]
    norm = torch.stack([(g * g).sum() for g in grads]).sum().sqrt()
    coef = torch.where(norm > st["case"]["max_norm"], st["case"]["max_norm"] / norm, 1.0)
    outs = [g * coef for g in grads]
    if st["case"]["flat"]:
        return {"flat": torch.cat([o.reshape(-1) for o in outs]), "norm": norm}
    packed = {k: torch.cat([o.reshape(-1) for o in outs if _kind(o.shape) == k]).to(_DT[st["case"][k]])
              for k in ("matrix", "vector")}
    return {**packed, "norm": norm}


_run_plain = {"embed": _embed_plain, "ffn": _ffn_plain, "clip": _clip_plain}


def _embed_own(st):
    S, c = _lib(), st["case"]
    t, v, d = c["tokens"], c["vocab"], c["d"]
    S.sama_embed(st["ctx"], S.DTYPES[c["dtype"]], t, v, d, st["table"], st["ids"], st["scale"], st["out"])
    if "dout" not in st:
        return {"out": st["out"]}
    S.sama_embed_grad(st["ctx"], S.DTYPES[c["dtype"]], t, v, d, st["ids"], st["dout"], st["scale"], -1,
                      S.DTYPES[c["grad"]], 0, st["grad"])
    return {"out": st["out"], "grad": st["grad"]}


def _ffn_own(st):
    S, c = _lib(), st["case"]
    dt, act = S.DTYPES[c["dtype"]], S.ACTS[c["act"]]
    t, d, f = c["tokens"], c["d"], c["f"]
    x, wg, wu, wd = st["x"], st["wg"], st["wu"], st["wd"]
    if not c["train"]:
        S.sama_gated_ffn(st["ctx"], dt, act, t, d, f, x, wg, wu, wd, st["y"])
        return {"y": st["y"]}
    S.sama_gated_ffn(st["ctx"], dt, act, t, d, f, x, wg, wu, wd, st["y"], st["gate"], st["up"])
    dwg, dwu, dwd = st["dw"]
    S.sama_gated_ffn_grad(st["ctx"], dt, act, t, d, f, x, wg, wu, wd, st["gate"], st["up"], st["dy"], st["dx"], dwg, dwu,
                          dwd)
    return {"y": st["y"], "dx": st["dx"], "dwg": dwg, "dwu": dwu, "dwd": dwd}


def _clip_own(st):
    S, c = _lib(), st["case"]
    S.sama_clip_grads(st["ctx"], st["list"], c["max_norm"], st["norm"])
    return {k: st[k] for k in (("flat",) if c["flat"] else ("matrix", "vector")) + ("norm",)}


_run_own = {"embed": _embed_own, "ffn": _ffn_own, "clip": _clip_own}


# ------------------------------------------------------------------------------------------- what a pass cannot avoid

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    if case["op"] == "embed":
        t, v, d, e = case["tokens"], case["vocab"], case["d"], size[case["dtype"]]
        b = 4 * t + 2 * t * d * e                        # ids, the rows looked up, the rows written
        if case["grad"] != "none":
            b += t * d * e + v * d * size[case["grad"]]   # the incoming gradient, every row of the table's gradient
        return {"bytes": b, "flops": t * d * (1 if case["grad"] == "none" else 2)}
    if case["op"] == "ffn":
        t, d, f = case["tokens"], case["d"], case["f"]
        b, n = 2 * (2 * t * d + 3 * d * f), 3             # x, y and the three weights; three products
        if case["train"]:
            b += 2 * (2 * t * d + 3 * d * f)              # dy, dx and the three weight gradients
            n += 6
        return {"bytes": b, "flops": 2 * n * t * d * f}
    b = n = 0
    for s in _shapes(case):
        e = size[case[_kind(s)]]
        n += math.prod(s)
        b += math.prod(s) * (e + (4 if case["flat"] else e))
    return {"bytes": b + 4, "flops": 3 * n}


# ------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "embed":
        ids, e = st["ids"].long(), st["table"].double()
        r = {"out": e.index_select(0, ids).mul_(st["scale"])}
        if case["grad"] != "none":
            r["grad"] = torch.zeros_like(e).index_put_((ids,), st["dout"].double(), accumulate=True).mul_(st["scale"])
        return r
    if case["op"] == "ffn":
        x, wg, wu, wd = (st[k].double() for k in ("x", "wg", "wu", "wd"))
        g = torch.einsum("td,fd->tf", x, wg)
        u = torch.einsum("td,fd->tf", x, wu)
        # activation a(g) and slope s(g), from the normal or logistic distribution function
        if case["act"] == "silu":
            cdf = torch.sigmoid(g)
            pdf = cdf * torch.sigmoid(-g)
        elif case["act"] == "relu":
            cdf, pdf = torch.heaviside(g, torch.zeros_like(g)), torch.zeros_like(g)
        elif case["act"] == "gelu":
            cdf = torch.special.ndtr(g)
            pdf = torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
        else:  # 0.5 (1 + tanh z) is the logistic function of 2 z
            z2 = 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
            cdf = torch.sigmoid(z2)
            pdf = cdf * torch.sigmoid(-z2) * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)
        a = g * cdf
        r = {"y": torch.einsum("tf,df->td", a * u, wd)}
        if case["train"]:
            dy = st["dy"].double()
            dh = torch.einsum("td,df->tf", dy, wd)
            dg, du = dh * u * (cdf + g * pdf), dh * a
            r["dx"] = torch.einsum("tf,fd->td", dg, wg) + torch.einsum("tf,fd->td", du, wu)
            r["dwg"] = torch.einsum("tf,td->fd", dg, x)
            r["dwu"] = torch.einsum("tf,td->fd", du, x)
            r["dwd"] = torch.einsum("td,tf->df", dy, a * u)
        return r
    flat = torch.cat([x.double().flatten() for x in st["grads"]])
    norm = torch.linalg.vector_norm(flat)
    flat *= min(1.0, case["max_norm"] / float(norm))
    if case["flat"]:
        return {"flat": flat, "norm": norm}
    parts = list(zip(st["grads"], flat.split([x.numel() for x in st["grads"]])))
    return {"matrix": torch.cat([p for x, p in parts if x.dim() == 2]),
            "vector": torch.cat([p for x, p in parts if x.dim() == 1]), "norm": norm}
