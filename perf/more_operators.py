"""The operators of a text model's attention and of learning from a teacher, as cases that can be timed: attention over
packed texts with its backward pass, attention of one new token over a paged cache, and distillation from a teacher's top
logits with its gradient.

`own` chooses what `run` computes with: elementary torch operations in 32 bits (False), or the library's entry points
(True).  Both take the same state.
"""
import math
import random

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
# attn: `texts` texts packed behind one another, the longest of `longest` tokens, the others' lengths by _lengths;
#   `earlier`: keys of earlier tokens that every text has in front of its own (a prompt's next chunk).
# paged: `seqs` sequences with caches of up to `longest` keys in pages of `page`.
# distill: `rows` rows of logits over `vocab`, the teacher's `k` largest.

def listed():
    return [
        # the text example's batch, 256 short texts of width 128: two small heads, latency and ragged ends
        {"name": "attn-short-train", "op": "attn", "texts": 256, "longest": 24, "mix": 1, "earlier": 0, "heads": 2,
         "kv": 2, "dim": 64, "dtype": "bf16", "causal": False, "prefix": False, "bias": False, "cap": 0.0, "train": True},
        # an encoder of width 1024 on a packed batch of texts of up to 512 tokens, with a bias by distance
        {"name": "attn-encoder-train", "op": "attn", "texts": 48, "longest": 512, "mix": 2, "earlier": 0, "heads": 16,
         "kv": 16, "dim": 64, "dtype": "bf16", "causal": False, "prefix": False, "bias": True, "cap": 0.0, "train": True},
        # instructions seen from everywhere, answers causal; a head size that is no power of two, half precision
        {"name": "attn-prefix-train", "op": "attn", "texts": 5, "longest": 2011, "mix": 3, "earlier": 0, "heads": 12,
         "kv": 4, "dim": 80, "dtype": "f16", "causal": True, "prefix": True, "bias": False, "cap": 0.0, "train": True},
        # one long document of a model of width 4096, shared key heads, capped scores: bound by the arithmetic
        {"name": "attn-long-train", "op": "attn", "texts": 1, "longest": 8192, "mix": 4, "earlier": 0, "heads": 32,
         "kv": 8, "dim": 128, "dtype": "bf16", "causal": True, "prefix": False, "bias": False, "cap": 30.0, "train": True},
        # serving: the next chunk of two prompts, behind the keys that are there already; forward only
        {"name": "attn-chunk", "op": "attn", "texts": 2, "longest": 1000, "mix": 5, "earlier": 7000, "heads": 32, "kv": 8,
         "dim": 128, "dtype": "bf16", "causal": True, "prefix": False, "bias": False, "cap": 0.0, "train": False},
        # the first tokens of a few answers: pure latency
        {"name": "paged-few", "op": "paged", "seqs": 4, "longest": 100, "mix": 6, "page": 16, "heads": 16, "kv": 16,
         "dim": 64, "dtype": "f16", "bias": True, "cap": 0.0},
        # one sequence with a long cache: there is work for the whole card only when the cache is split
        {"name": "paged-one-long", "op": "paged", "seqs": 1, "longest": 60001, "mix": 7, "page": 64, "heads": 32, "kv": 8,
         "dim": 128, "dtype": "bf16", "bias": False, "cap": 30.0},
        # a serving batch of ragged lengths
        {"name": "paged-batch", "op": "paged", "seqs": 96, "longest": 4096, "mix": 8, "page": 16, "heads": 32, "kv": 8,
         "dim": 128, "dtype": "bf16", "bias": False, "cap": 0.0},
        # a small student in fp32
        {"name": "distill-small", "op": "distill", "rows": 128, "vocab": 8191, "k": 16, "mix": 9, "dtype": "f32",
         "ragged": False, "grad": True},
        # evaluation on a validation batch: losses alone
        {"name": "distill-eval", "op": "distill", "rows": 1000, "vocab": 32768, "k": 100, "mix": 10, "dtype": "bf16",
         "ragged": True, "grad": False},
        # a fine-tuning step's rows: odd vocabulary, rows that start anywhere
        {"name": "distill-odd", "op": "distill", "rows": 4096, "vocab": 50021, "k": 64, "mix": 11, "dtype": "bf16",
         "ragged": False, "grad": True},
        # a large vocabulary: two passes over 1 GB of logits and as much gradient if rows are not kept on the chip
        {"name": "distill-large", "op": "distill", "rows": 4096, "vocab": 131072, "k": 128, "mix": 12, "dtype": "bf16",
         "ragged": True, "grad": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "paged", "distill"])
    mix = rng.randrange(1 << 20)
    if op == "distill":
        while True:
            c = {"op": op, "rows": _log(rng, 1, 16384), "vocab": _log(rng, 40, 200000)}
            if c["rows"] * c["vocab"] <= 4096 * 131072:
                break
        c["k"] = min(_log(rng, 1, 256), c["vocab"])
        c.update(mix=mix, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), ragged=rng.random() < 0.5,
                 grad=rng.random() < 0.75)
        if c["dtype"] == "f32":
            c["rows"] = -(-c["rows"] // 2)
        return c
    kv = rng.choice([1, 2, 4, 8, 16])
    c = {"op": op, "mix": mix, "kv": kv, "heads": kv * rng.choice([g for g in (1, 2, 3, 4, 7, 8) if g * kv <= 32]),
         "dim": rng.choice([64, 64, 128, 128, 8 * rng.randint(2, 16)]), "dtype": rng.choice(["bf16", "bf16", "f16"]),
         "bias": rng.random() < 0.3, "cap": rng.choice([0.0, 0.0, 0.0, 30.0, 50.0])}
    if op == "paged":
        c["page"] = rng.choice([8, 16, 16, 32, 64, 128, 48])
        while True:
            c["seqs"], c["longest"] = _log(rng, 1, 256), _log(rng, 1, 65536)
            if c["seqs"] * c["longest"] * c["kv"] * c["dim"] <= 96 * 4096 * 8 * 128:
                return c
    while True:
        c["texts"], c["longest"] = _log(rng, 1, 256), _log(rng, 1, 8192)
        c["earlier"] = _log(rng, 1, 8192) if rng.random() < 0.2 else 0
        c["causal"] = c["earlier"] > 0 or rng.random() < 0.6
        pairs = c["texts"] * c["longest"] * (c["longest"] + 2 * c["earlier"]) / (2 if c["causal"] else 1)
        tokens = c["texts"] * (c["longest"] + c["earlier"]) * c["heads"] * c["dim"]
        if pairs * c["heads"] * c["dim"] <= 8192 * 8192 // 2 * 32 * 128 and tokens <= 16384 * 4096:
            break
    c["prefix"] = c["causal"] and rng.random() < 0.3
    c["train"] = c["earlier"] == 0 and rng.random() < 0.7
    return c


def _lengths(case, n):
    """Lengths of n texts or caches, between a quarter of the longest and the longest itself."""
    rng = random.Random(case["mix"])
    return [case["longest"]] + [max(1, round(case["longest"] * rng.uniform(0.25, 1.0))) for _ in range(n - 1)]


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device="cuda")


# ------------------------------------------------------------------------------------------------- inputs and plan

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 13)


def _starts(lengths):
    out = [0]
    for n in lengths:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    g = _gen(seed)
    st = {"attn": _prepare_attn, "paged": _prepare_paged, "distill": _prepare_distill}[case["op"]](case, g)
    st["case"] = case
    if own:
        st["ctx"] = _context()
    return st


def _prepare_attn(case, g):
    dt, h, kv, d = _DT[case["dtype"]], case["heads"], case["kv"], case["dim"]
    lens = _lengths(case, case["texts"])
    qs, ks = _starts(lens), _starts([n + case["earlier"] for n in lens])
    nq, nk = qs[-1], ks[-1]
    st = {"lens": lens, "scale": 1.0 / math.sqrt(d)}
    if case["earlier"] == 0:
        # queries, keys and values side by side, as one projection gives them
        st["qkv"] = torch.randn(nq, h + 2 * kv, d, generator=g, device="cuda").to(dt)
        st["qkv"][:, :h] *= 2.5
        st["q"], st["k"], st["v"] = st["qkv"].split([h, kv, kv], dim=1)
    else:
        st["q"] = (2.5 * torch.randn(nq, h, d, generator=g, device="cuda")).to(dt)
        st["k"], st["v"] = (torch.randn(nk, kv, d, generator=g, device="cuda").to(dt) for _ in range(2))
    if case["train"]:
        st["dout"] = torch.randn(nq, h, d, generator=g, device="cuda").to(dt)
    if case["bias"]:
        st["slopes"] = _slopes(h)
    if case["prefix"]:
        st["prefix_host"] = [round(0.3 * n) for n in lens]
    if own:
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        S = _lib()
        st["out"] = torch.empty(nq, h, d, dtype=dt, device="cuda")
        st["lse"] = torch.empty(h, nq, device="cuda") if case["train"] else None
        if case["train"]:
            st["dqkv"] = torch.empty_like(st["qkv"])
            st["dq"], st["dk"], st["dv"] = st["dqkv"].split([h, kv, kv], dim=1)
        st["attn"] = S.Attn(S.DTYPES[case["dtype"]], h, kv, d, nq, nk, i32(qs), i32(ks) if case["earlier"] else None,
                            causal=case["causal"], prefix=i32(st["prefix_host"]) if case["prefix"] else None,
                            slopes=st.get("slopes"), scale=st["scale"], cap=case["cap"], q_stride=st["q"].stride(0),
                            k_stride=st["k"].stride(0), v_stride=st["v"].stride(0))
    return st


def _prepare_paged(case, g):
    dt, h, kv, d, page = _DT[case["dtype"]], case["heads"], case["kv"], case["dim"], case["page"]
    lens = _lengths(case, case["seqs"])
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)   # pages lie anywhere
    table = torch.full((case["seqs"], max(need)), -1, dtype=torch.int32, device="cuda")
    for s, (a, n) in enumerate(zip(_starts(need), need)):
        table[s, :n] = order[a:a + n]
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float32).to(dt)  # noqa: E731
    st = {"table": table, "lengths": torch.tensor(lens, dtype=torch.int32, device="cuda"), "scale": 1.0 / math.sqrt(d),
          "q": 2.5 * randn(case["seqs"], h, d), "k_new": randn(case["seqs"], kv, d), "v_new": randn(case["seqs"], kv, d),
          "k_cache": randn(n_pages, page, kv, d), "v_cache": randn(n_pages, page, kv, d), "longest": max(lens)}
    if case["bias"]:
        st["slopes"] = _slopes(h)
    if own:
        S = _lib()
        st["out"] = torch.empty_like(st["q"])
        st["paged"] = S.Paged(S.DTYPES[case["dtype"]], h, kv, d, page, n_pages, table, st["lengths"],
                              slopes=st.get("slopes"), scale=st["scale"], cap=case["cap"])
    return st


def _prepare_distill(case, g):
    dt, n, v, k = _DT[case["dtype"]], case["rows"], case["vocab"], case["k"]
    logits = (2.5 * torch.randn(n, v, generator=g, device="cuda")).to(dt)
    # the teacher agrees with the student in part
    teacher = torch.randn(n, v, generator=g, device="cuda").mul_(1.5).add_(logits, alpha=0.8)
    top, ids = teacher.topk(k, dim=1)
    ids = ids.to(torch.int32)
    if case["ragged"]:
        # rows for which fewer logits were kept (a cut by probability): the rest of the row is unused
        keep = torch.randint(1, k + 1, (n, 1), generator=g, device="cuda")
        ids = torch.where(torch.arange(k, device="cuda") < keep, ids, -1)
    st = {"logits": logits, "top": top, "ids": ids, "weight": torch.sigmoid(torch.randn(n, generator=g, device="cuda")),
          "temperature": 2.0, "grad_scale": (65536.0 if case["dtype"] == "f16" else 1.0) / n}
    if own:
        st["loss"] = torch.empty(n, device="cuda")
        st["grad"] = torch.empty_like(logits) if case["grad"] else None
    return st


# ------------------------------------------------------------------------------------------------------ one pass

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _attn_plain(st):
    """Texts of similar lengths in padded batches, a few key heads at a time, so that scores stay below 8 GB."""
    c = st["case"]
    h, kv, d, e = c["heads"], c["kv"], c["dim"], c["earlier"]
    grp, lens = h // kv, st["lens"]
    qs, ks = _starts(lens), _starts([n + e for n in lens])
    dt = st["q"].dtype
    r = {"out": torch.zeros(qs[-1], h, d, dtype=dt, device="cuda")}
    if c["train"]:
        r["dqkv"] = torch.zeros(qs[-1], h + 2 * kv, d, dtype=dt, device="cuda")
    order, at = sorted(range(len(lens)), key=lambda i: -lens[i]), 0
    while at < len(order):
        L = lens[order[at]]
        room = max(1, (1 << 31) // (L * (L + e) * grp))          # (texts, key heads) that fit together
        part = order[at:at + max(1, room // kv)]
        heads_at_once = min(kv, room)
        at += len(part)
        n = torch.tensor([lens[i] for i in part], device="cuda")[:, None]
        i, j = torch.arange(L, device="cuda"), torch.arange(L + e, device="cuda")
        q_real, k_real = i < n, j < n + e
        q_row = torch.where(q_real, torch.tensor([qs[t] for t in part], device="cuda")[:, None] + i, 0)
        k_row = torch.where(k_real, torch.tensor([ks[t] for t in part], device="cuda")[:, None] + j, 0)
        see = k_real[:, None, :].expand(-1, L, -1)
        if c["causal"]:
            past = j <= i[:, None] + e
            if c["prefix"]:
                past = past | (j < torch.tensor([st["prefix_host"][t] for t in part], device="cuda")[:, None, None])
            see = see & past
        see = see[:, None, None]                                  # [text][1][1][query][key]
        gap = (i[:, None] + e - j).abs().float()
        for k0 in range(0, kv, heads_at_once):
            k1 = min(kv, k0 + heads_at_once)
            hs = slice(k0 * grp, k1 * grp)

            def gather(x, row, real, a, b):                       # [text][key heads][queries of each][token][dim]
                y = x[row, a:b].float() * real[..., None, None]
                return y.transpose(1, 2).unflatten(1, (k1 - k0, -1))

            q = gather(st["q"], q_row, q_real, hs.start, hs.stop)
            k, v = (gather(st[x], k_row, k_real, k0, k1) for x in ("k", "v"))
            s = (q @ k.transpose(-1, -2)) * st["scale"]
            if c["cap"]:
                th = torch.tanh(s / c["cap"])
                s = c["cap"] * th
            if c["bias"]:
                s = s - st["slopes"][hs].view(k1 - k0, grp, 1, 1) * gap
            s = s.masked_fill(~see, -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            p = p / p.sum(-1, keepdim=True)
            del s
            o = p @ v

            def put(into, y, row, real, a):
                into[:, a:a + (k1 - k0) * y.shape[2]][row[real]] = y.flatten(1, 2).transpose(1, 2)[real].to(dt)

            put(r["out"], o, q_row, q_real, hs.start)
            if c["train"]:
                do = gather(st["dout"], q_row, q_real, hs.start, hs.stop)
                dv = (p.transpose(-1, -2) @ do).sum(2, keepdim=True)
                ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True))
                if c["cap"]:
                    ds = ds * (1.0 - th * th)
                ds = ds * st["scale"]
                put(r["dqkv"], ds @ k, q_row, q_real, hs.start)
                put(r["dqkv"], (ds.transpose(-1, -2) @ q).sum(2, keepdim=True), k_row, k_real, h + k0)
                put(r["dqkv"], dv, k_row, k_real, h + kv + k0)
    return r


def _paged_plain(st):
    c = st["case"]
    kv, d, page, grp = c["kv"], c["dim"], c["page"], c["heads"] // c["kv"]
    last = (st["lengths"] - 1).long()
    rows = torch.arange(c["seqs"], device="cuda")
    for cache, new in (("k_cache", "k_new"), ("v_cache", "v_new")):
        st[cache][st["table"][rows, last // page].long(), last % page] = st[new]
    j = torch.arange(st["longest"], device="cuda")
    out = torch.empty_like(st["q"])
    step = max(1, (1 << 30) // (st["longest"] * kv * d))          # sequences at a time
    for a in range(0, c["seqs"], step):
        b = min(c["seqs"], a + step)
        real = j <= last[a:b, None]
        at = st["table"][a:b, j // page].long().clamp(min=0)
        k, v = (st[x][at, j % page].float().transpose(1, 2) for x in ("k_cache", "v_cache"))   # [seq][head][key][dim]
        s = (st["q"][a:b].float().view(b - a, kv, grp, d) @ k.transpose(-1, -2)) * st["scale"]
        if c["cap"]:
            s = c["cap"] * torch.tanh(s / c["cap"])
        if c["bias"]:
            s = s - st["slopes"].view(kv, grp, 1) * (last[a:b, None] - j).float()[:, None, None]
        s = s.masked_fill(~real[:, None, None], -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        o = (p @ v) / p.sum(-1, keepdim=True)
        out[a:b] = o.reshape(b - a, c["heads"], d).to(out.dtype)
    return {"out": out, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _distill_plain(st):
    t = st["temperature"]
    z = st["logits"].float() / t
    used = st["ids"] >= 0
    ids = st["ids"].long().clamp(min=0)
    u = (st["top"] / t).masked_fill(~used, -math.inf)
    p = torch.exp(u - u.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    top = z.amax(1, keepdim=True)
    q = torch.exp(z - top)
    total = q.sum(1, keepdim=True)
    logq = z.gather(1, ids) - top - torch.log(total)
    logp = torch.log(torch.where(p > 0, p, 1.0))
    r = {"loss": t * t * (p * (logp - logq)).sum(1)}
    if st["case"]["grad"]:
        q = (q / total).scatter_add_(1, ids, -p)
        r["grad"] = (q * (t * st["grad_scale"] * st["weight"])[:, None]).to(st["logits"].dtype)
    return r


_run_plain = {"attn": _attn_plain, "paged": _paged_plain, "distill": _distill_plain}


def _attn_own(st):
    S = _lib()
    S.sama_attention(st["ctx"], st["attn"], st["q"], st["k"], st["v"], st["out"], st["lse"])
    if st["lse"] is None:
        return {"out": st["out"]}
    S.sama_attention_grad(st["ctx"], st["attn"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["dout"], st["dq"],
                          st["dk"], st["dv"])
    return {"out": st["out"], "dqkv": st["dqkv"]}


def _paged_own(st):
    S = _lib()
    S.sama_paged_attention(st["ctx"], st["paged"], st["q"], st["k_new"], st["v_new"], st["k_cache"], st["v_cache"],
                           st["out"])
    return {"out": st["out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}


def _distill_own(st):
    S, c = _lib(), st["case"]
    S.sama_distill(st["ctx"], S.DTYPES[c["dtype"]], c["rows"], c["vocab"], st["logits"], c["k"], S.SAMA_F32, st["top"],
                   st["ids"], st["temperature"], st["weight"], st["grad_scale"], st["loss"], st["grad"])
    return {"loss": st["loss"], "grad": st["grad"]} if c["grad"] else {"loss": st["loss"]}


_run_own = {"attn": _attn_own, "paged": _paged_own, "distill": _distill_own}


# ------------------------------------------------------------------------------------------- what a pass cannot avoid

def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["dtype"]]
    if case["op"] == "distill":
        n, v, k = case["rows"], case["vocab"], case["k"]
        b = n * v * size * (2 if case["grad"] else 1) + n * k * 8 + 8 * n
        return {"bytes": b, "flops": (6 if case["grad"] else 3) * n * v}
    h, kv, d = case["heads"], case["kv"], case["dim"]
    if case["op"] == "paged":
        lens = _lengths(case, case["seqs"])
        b = size * (2 * sum(lens) * kv * d + 2 * len(lens) * (h + kv) * d) + 4 * sum(-(-n // case["page"]) for n in lens)
        return {"bytes": b, "flops": 4 * sum(lens) * h * d}
    pairs = tokens = keys = 0
    for n in _lengths(case, case["texts"]):
        e = case["earlier"]
        tokens, keys = tokens + n, keys + n + e
        if not case["causal"]:
            pairs += n * (n + e)
        else:
            pairs += n * e + n * (n + 1) // 2
            if case["prefix"]:
                # query i sees i + e + 1 keys, or the prefix if that is longer
                p = round(0.3 * n)
                pairs += max(0, p - e) * max(0, p - e - 1) // 2 if p > e else 0
    b = size * d * (2 * tokens * h + 2 * keys * kv)
    f = 4 * pairs * h * d
    if case["train"]:
        b += size * d * (2 * tokens * h + 2 * keys * kv)          # the incoming gradient and three outgoing ones
        f += 10 * pairs * h * d                                   # five products
    return {"bytes": b, "flops": f}


# ------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    return {"attn": _attn_exact, "paged": _paged_exact, "distill": _distill_exact}[case["op"]](case, prepare(case, seed))


def _soft(score, visible):
    """Softmax over the last axis of the visible scores."""
    return torch.softmax(torch.where(visible, score, -torch.inf), dim=-1)


def _attn_exact(case, st):
    """Text by text and key head by key head; the gradients by differentiating the definition."""
    h, kv, d, e = case["heads"], case["kv"], case["dim"], case["earlier"]
    grp = h // kv
    nq = st["q"].shape[0]
    out = torch.zeros(nq, h, d, dtype=torch.float64, device="cuda")
    grad = torch.zeros(nq, h + 2 * kv, d, dtype=torch.float64, device="cuda") if case["train"] else None
    a = b = 0
    for t, n in enumerate(st["lens"]):
        pos_q, pos_k = torch.arange(e, e + n, device="cuda"), torch.arange(n + e, device="cuda")
        visible = torch.ones(n, n + e, dtype=torch.bool, device="cuda")
        if case["causal"]:
            visible = pos_k[None] <= pos_q[:, None]
            if case["prefix"]:
                visible = visible | (pos_k < st["prefix_host"][t])[None]
        dist = (pos_q[:, None] - pos_k[None]).abs().double()
        step = kv if n * (n + e) * h < 1 << 26 else 1             # key heads at a time
        for g in range(0, kv, step):
            hs, gs = slice(g * grp, (g + step) * grp), slice(g, g + step)
            q = st["q"][a:a + n, hs].double().requires_grad_(case["train"])
            k = st["k"][b:b + n + e, gs].double().requires_grad_(case["train"])
            v = st["v"][b:b + n + e, gs].double().requires_grad_(case["train"])
            score = torch.einsum("igxd,jgd->gxij", q.unflatten(1, (step, grp)), k) / math.sqrt(d)
            if case["cap"]:
                score = case["cap"] * torch.tanh(score / case["cap"])
            if case["bias"]:
                score = score - st["slopes"].double()[hs].view(step, grp, 1, 1) * dist
            o = torch.einsum("gxij,jgd->igxd", _soft(score, visible), v).flatten(1, 2)
            out[a:a + n, hs] = o.detach()
            if case["train"]:
                dq, dk, dv = torch.autograd.grad(o, (q, k, v), st["dout"][a:a + n, hs].double())
                grad[a:a + n, hs] = dq
                grad[b:b + n, h + g:h + g + step] = dk
                grad[b:b + n, h + kv + g:h + kv + g + step] = dv
            del o, score, q, k, v
        a, b = a + n, b + n + e
    return {"out": out, "dqkv": grad} if case["train"] else {"out": out}


def _paged_exact(case, st):
    kv, d, page = case["kv"], case["dim"], case["page"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device="cuda")
    for s, n in enumerate(st["lengths"].tolist()):
        pages = st["table"][s, :-(-n // page)].long()
        k, v = (st[c][pages].flatten(0, 1)[:n - 1].double() for c in ("k_cache", "v_cache"))
        k, v = torch.cat([k, st["k_new"][s:s + 1].double()]), torch.cat([v, st["v_new"][s:s + 1].double()])
        score = torch.einsum("gxd,jgd->gxj", st["q"][s].double().unflatten(0, (kv, -1)), k) / math.sqrt(d)
        if case["cap"]:
            score = case["cap"] * torch.tanh(score / case["cap"])
        if case["bias"]:
            away = torch.arange(n - 1, -1, -1, device="cuda").double()
            score = score - st["slopes"].double().view(kv, -1, 1) * away
        out[s] = torch.einsum("gxj,jgd->gxd", torch.softmax(score, -1), v).flatten(0, 1)
    return {"out": out, "k_cache": None, "v_cache": None}


def _distill_exact(case, st):
    n, t = case["rows"], st["temperature"]
    loss = torch.empty(n, dtype=torch.float64, device="cuda")
    grad = torch.empty(n, case["vocab"], dtype=torch.float64, device="cuda") if case["grad"] else None
    for a in range(0, n, 512):
        rows = slice(a, min(n, a + 512))
        logq = torch.log_softmax(st["logits"][rows].double() / t, dim=1)
        ids = st["ids"][rows].long()
        p = _soft(st["top"][rows].double() / t, ids >= 0)
        entry = torch.special.xlogy(p, p) - p * logq.gather(1, ids.clamp(min=0))
        loss[rows] = t * t * entry.sum(1)
        if case["grad"]:
            dense = torch.zeros_like(logq).scatter_add_(1, ids.clamp(min=0), p)
            grad[rows] = (torch.exp(logq) - dense) * (t * st["grad_scale"]) * st["weight"][rows, None].double()
    return {"loss": loss, "grad": grad} if case["grad"] else {"loss": loss}
