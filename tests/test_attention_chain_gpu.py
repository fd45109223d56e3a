"""Attention, the paged cache and distillation as a program uses them: a layer's training step with the other operators of
text models, eager and in a graph; a text read at once, in chunks, and token by token from the cache."""
import math

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1 << 16, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


VOCAB, D, HEADS, KV, F = 503, 128, 4, 2, 344
DIM = D // HEADS


class Student:
    """tokens -> embedding -> x + attention(x) -> h + feed-forward(h) -> logits, taught by a teacher's top logits; matrices
    between the operators are torch's.  One flat fp32 gradient at the end."""

    def __init__(self, lib, lens, seed=0):
        self.S, self.ctx = lib
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = sum(lens)
        self.n, self.lens = n, lens
        r = lambda *s, std=1.0: (std * torch.randn(*s, generator=g, device="cuda")).bfloat16()  # noqa: E731
        self.w = {"table": r(VOCAB, D), "wqkv": r((HEADS + 2 * KV) * DIM, D, std=D ** -0.5), "wo": r(D, HEADS * DIM, std=D ** -0.5),
                  "wg": r(F, D, std=D ** -0.5), "wu": r(F, D, std=D ** -0.5), "wd": r(D, F, std=F ** -0.5)}
        self.ids = torch.randint(VOCAB, (n,), generator=g, device="cuda", dtype=torch.int32)
        at = [0]
        for x in lens:
            at.append(at[-1] + x)
        self.starts = torch.tensor(at, dtype=torch.int32, device="cuda")
        self.top, ids = torch.randn(n, VOCAB, generator=g, device="cuda").topk(8, dim=1)
        self.top_ids = ids.to(torch.int32)
        self.weight = torch.sigmoid(torch.randn(n, generator=g, device="cuda"))
        S, width = self.S, (HEADS + 2 * KV) * DIM
        self.attn = S.Attn(S.SAMA_BF16, HEADS, KV, DIM, n, n, self.starts, causal=True, q_stride=width, k_stride=width, v_stride=width)
        e = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.x, self.y, self.dh, self.dx = (e(n, D) for _ in range(4))
        self.o, self.lse = e(n, HEADS, DIM), torch.empty(HEADS, n, device="cuda")
        self.dqkv = e(n, HEADS + 2 * KV, DIM)
        self.gate, self.up, self.loss, self.dz = e(n, F), e(n, F), torch.empty(n, device="cuda"), e(n, VOCAB)
        self.grad = {k: e(*v.shape) for k, v in self.w.items()}
        size = [v.numel() for v in self.grad.values()]
        self.flat, self.norm = torch.empty(sum(size), device="cuda"), torch.empty(1, device="cuda")
        self.tensors = S.TensorList(self.grad.values(), self.flat.split(size))

    def parts(self, t):
        return t.split([HEADS, KV, KV], 1)

    def step(self):
        S, c, n, w, b = self.S, self.ctx, self.n, self.w, self.S.SAMA_BF16
        S.sama_embed(c, b, n, VOCAB, D, w["table"], self.ids, 1.0, self.x)
        self.qkv = (self.x @ w["wqkv"].T).view(n, HEADS + 2 * KV, DIM)
        S.sama_attention(c, self.attn, *self.parts(self.qkv), self.o, self.lse)
        self.h = self.x + self.o.view(n, D) @ w["wo"].T
        S.sama_gated_ffn(c, b, S.SAMA_ACT_SILU, n, D, F, self.h, w["wg"], w["wu"], w["wd"], self.y, self.gate, self.up)
        out = self.h + self.y
        self.z = out @ w["table"].T
        S.sama_distill(c, b, n, VOCAB, self.z, 8, S.SAMA_F32, self.top, self.top_ids, 2.0, self.weight, 1.0, self.loss, self.dz)
        dout = self.dz @ w["table"]
        S.sama_gated_ffn_grad(c, b, S.SAMA_ACT_SILU, n, D, F, self.h, w["wg"], w["wu"], w["wd"], self.gate, self.up, dout, self.dh,
                              self.grad["wg"], self.grad["wu"], self.grad["wd"])
        dh = self.dh + dout
        torch.mm(dh.T, self.o.view(n, D), out=self.grad["wo"])
        self.do = (dh @ w["wo"]).view(n, HEADS, DIM)
        S.sama_attention_grad(c, self.attn, *self.parts(self.qkv), self.o, self.lse, self.do, *self.parts(self.dqkv))
        dq = self.dqkv.view(n, -1)
        torch.mm(dq.T, self.x, out=self.grad["wqkv"])
        torch.add(dh, dq @ w["wqkv"], out=self.dx)
        S.sama_embed_grad(c, b, n, VOCAB, D, self.ids, self.dx, 1.0, -1, b, 0, self.grad["table"])
        S.sama_clip_grads(c, self.tensors, math.inf, self.norm)

    def outputs(self):
        return [self.o, self.lse, self.dqkv, self.loss, self.dz, self.flat, self.norm]


def test_a_training_step_eager_and_in_a_graph(lib):
    """Every operator's results are those of its definition for the inputs that the step gave it, and a replay has the same bits."""
    m = Student(lib, [60, 1, 130, 33])
    m.step()
    torch.cuda.synchronize()
    at = m.starts.tolist()
    q, k, v = m.parts(m.qkv)
    dq, dk, dv = m.parts(m.dqkv)
    for a, b in zip(at, at[1:]):
        r = slice(a, b)
        want, bound = ref.text(q[r], k[r], v[r], m.do[r], "bf16", DIM ** -0.5, 0.0, None, True, 0)
        for name, x in (("out", m.o), ("dq", dq), ("dk", dk), ("dv", dv)):
            assert bool(((x[r].double() - want[name]).abs() <= bound[name]).all()), name
    z = m.z.double() / 2.0
    p, logq = torch.softmax(m.top.double() / 2.0, 1), torch.log_softmax(z, 1)
    loss = 4.0 * (p * (p.log() - logq.gather(1, m.top_ids.long()))).sum(1)
    assert torch.allclose(m.loss.double(), loss, rtol=2e-5, atol=2e-5)      # (fp32 sums of 503 terms; test_distill_gpu.py derives more)
    dz = (2.0 * m.weight.double())[:, None] * (logq.exp() - torch.zeros_like(z).scatter_add_(1, m.top_ids.long(), p))
    assert bool(((m.dz.double() - dz).abs() <= 2.0 ** -8 * dz.abs() + 1e-5).all())
    assert torch.allclose(m.norm.double(), m.flat.double().norm(), rtol=1e-6)
    want = [x.clone() for x in m.outputs()]
    assert m.S.sama_device_status(m.ctx) == 0
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        m.step()
    for _ in range(3):
        for x in (m.o, m.lse, m.dqkv, m.loss, m.dz, m.flat, m.norm):
            x.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(m.outputs(), want))


def test_two_students_on_two_streams(lib):
    S = lib[0]
    other = S.sama_create(0, 1 << 16, 0, None)
    a, b = Student(lib, [100, 77], 1), Student((S, other), [20] * 9, 2)
    for m in (a, b):
        m.step()
    torch.cuda.synchronize()
    want = [[x.clone() for x in m.outputs()] for m in (a, b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        for m, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                m.step()
    torch.cuda.synchronize()
    for m, w in zip((a, b), want):
        assert all(torch.equal(x, y) for x, y in zip(m.outputs(), w))
    S.sama_destroy(other)


@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, True)])
@pytest.mark.parametrize("dim", [64, 128])
def test_at_once_in_chunks_and_token_by_token(lib, cap, bias, dim):
    """Three ways of reading a text: all are the definition's values, within its bounds."""
    S, ctx = lib
    n, heads, kv, page, chunk = 150, 4, 2, 16, 61
    g = torch.Generator(device="cuda").manual_seed(dim)
    q, k, v = (torch.randn(n, h, dim, generator=g, device="cuda").bfloat16() for h in (heads, kv, kv))
    slopes = 0.5 ** torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) if bias else None
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    at_once = torch.empty_like(q)
    S.sama_attention(ctx, S.Attn(S.SAMA_BF16, heads, kv, dim, n, n, i32(0, n), causal=True, slopes=slopes, cap=cap), q, k, v, at_once)
    chunks = torch.empty_like(q)
    for a in range(0, n, chunk):
        b = min(n, a + chunk)
        t = S.Attn(S.SAMA_BF16, heads, kv, dim, b - a, b, i32(0, b - a), i32(0, b), causal=True, slopes=slopes, cap=cap)
        S.sama_attention(ctx, t, q[a:b], k[:b], v[:b], chunks[a:b])
    pages = -(-n // page)
    caches = [torch.full((pages + 2, page, kv, dim), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.randperm(pages + 2, generator=g, device="cuda").to(torch.int32)[None, :pages].contiguous()
    length = i32(0)
    p = S.Paged(S.SAMA_BF16, heads, kv, dim, page, pages + 2, table, length, slopes=slopes, cap=cap)
    tokens = torch.empty_like(q)
    for i in range(n):
        length.fill_(i + 1)
        S.sama_paged_attention(ctx, p, q[i:i + 1], k[i:i + 1], v[i:i + 1], *caches, tokens[i:i + 1])
    want, bound = ref.text(q, k, v, None, "bf16", dim ** -0.5, cap, slopes, True, 0)
    for x in (at_once, chunks, tokens):
        assert bool(((x.double() - want["out"]).abs() <= bound["out"]).all())
    at = torch.arange(n, device="cuda")
    assert torch.equal(caches[0][table[0, at // page].long(), at % page], k)
    assert S.sama_device_status(ctx) == 0


def test_first_calls_in_a_capture(lib):
    """Calls that need no workspace can be captured without one before them."""
    S, _ = lib
    ctx = S.sama_create(0, 1024, 0, None)
    q = torch.randn(70, 2, 48, device="cuda").half()
    out, starts = torch.empty_like(q), torch.tensor([0, 70], dtype=torch.int32, device="cuda")
    t = S.Attn(S.SAMA_F16, 2, 2, 48, 70, 70, starts, causal=True, cap=7.0)
    z = torch.randn(9, 40000, device="cuda").half()
    top, ids = z.float().topk(5, dim=1)
    ids, loss, grad = ids.to(torch.int32), torch.empty(9, device="cuda"), torch.empty_like(z)

    def run():
        S.sama_attention(ctx, t, q, q, q, out)
        S.sama_distill(ctx, S.SAMA_F16, 9, 40000, z, 5, S.SAMA_F32, top, ids, 1.0, None, 1.0, loss, grad)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    out.fill_(float("nan"))
    grad.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    got = [out.clone(), loss.clone(), grad.clone()]
    assert all(bool(torch.isfinite(x).all()) for x in got)
    run()
    assert all(torch.equal(x, y) for x, y in zip(got, (out, loss, grad)))
    S.sama_destroy(ctx)
