"""Attention over packed texts, forward and backward, against the definition in 64 bits (attention_reference.py, which
derives the tolerances)."""
import math

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def starts(lens, first=0):
    out = [first]
    for n in lens:
        out.append(out[-1] + n)
    return out


class Case:
    """Packed texts with `edge` rows of no text before and behind them, which hold NaN."""

    def __init__(self, lib, lq, lk=None, heads=2, kv=1, dim=64, dtype="bf16", causal=False, prefix=None, bias=False, cap=0.0,
                 fused=False, edge=5, seed=0, size=2.0, scale=None):
        self.S, self.ctx = lib
        S = self.S
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype, self.lq, self.lk = dtype, list(lq), list(lq if lk is None else lk)
        self.causal, self.prefix, self.cap = causal, prefix, cap
        self.qs, self.ks = starts(self.lq, edge), starts(self.lk, edge)
        self.nq, self.nk = self.qs[-1] + edge, self.ks[-1] + edge
        self.edge = edge
        dt = ref.DT[dtype]

        def rows(n, h, at, scale=1.0):
            x = torch.full((n, h, dim), NAN, device="cuda")
            x[edge:n - edge] = scale * torch.randn(n - 2 * edge, h, dim, generator=g, device="cuda")
            return x.to(dt)

        if fused:       # three parts of one projection's rows, with a gap behind them
            buf = torch.full((self.nq, heads + 2 * kv + 1, dim), NAN, dtype=dt, device="cuda")
            self.q, self.k, self.v, _ = buf.split([heads, kv, kv, 1], 1)
            grad = torch.full_like(buf, 7.0)
            self.grads = [grad[:, :heads], grad[:, heads:heads + kv], grad[:, heads + kv:heads + 2 * kv]]
            self.gap = grad[:, heads + 2 * kv:]
            for x, h, s in ((self.q, heads, size), (self.k, kv, 1.0), (self.v, kv, 1.0)):
                x.copy_(rows(self.nq, h, 0, s))
        else:
            self.q, self.k, self.v = rows(self.nq, heads, 0, size), rows(self.nk, kv, 0), rows(self.nk, kv, 0)
            self.grads = [torch.full_like(x, 7.0) for x in (self.q, self.k, self.v)]
            self.gap = None
        self.dout = rows(self.nq, heads, 0)
        self.out = torch.full((self.nq, heads, dim), 7.0, dtype=dt, device="cuda")
        self.lse = torch.full((heads, self.nq), 7.0, device="cuda")
        self.slopes = 0.5 ** torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) if bias else None
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.scale = dim ** -0.5 if scale is None else scale
        self.starts_q, self.starts_k = i32(self.qs), None if lk is None else i32(self.ks)
        self.attn = S.Attn(S.DTYPES[dtype], heads, kv, dim, self.nq, self.nk, self.starts_q, self.starts_k, causal=causal,
                           prefix=None if prefix is None else i32(prefix), slopes=self.slopes, scale=self.scale, cap=cap,
                           q_stride=self.q.stride(0), k_stride=self.k.stride(0), v_stride=self.v.stride(0))

    def forward(self, stream=None):
        self.S.sama_attention(self.ctx, self.attn, self.q, self.k, self.v, self.out, self.lse, stream)

    def run(self, stream=None):
        self.forward(stream)
        self.S.sama_attention_grad(self.ctx, self.attn, self.q, self.k, self.v, self.out, self.lse, self.dout, *self.grads, stream)

    def results(self):
        return [self.out, self.lse, *self.grads]

    def check(self, grad=True):
        inside_q, inside_k = torch.zeros(self.nq, dtype=torch.bool), torch.zeros(self.nk, dtype=torch.bool)
        for t, (nq, nk) in enumerate(zip(self.lq, self.lk)):
            a, b = slice(self.qs[t], self.qs[t] + nq), slice(self.ks[t], self.ks[t] + nk)
            inside_q[a], inside_k[b] = True, True
            want, bound = ref.text(self.q[a], self.k[b], self.v[b], self.dout[a] if grad else None, self.dtype, self.scale,
                                   self.cap, self.slopes, self.causal, self.prefix[t] if self.prefix else 0)
            got = {"out": self.out[a], "lse": self.lse[:, a]}
            if grad:
                got.update(dq=self.grads[0][a], dk=self.grads[1][b], dv=self.grads[2][b])
            for name, x in got.items():
                y = want[name]
                same = x.double() == y                                # infinities
                over = torch.where(same, -1.0, (x.double() - y).abs() - bound[name])
                assert bool((over <= 0).all()), (t, name, float(over.max()), float(y.abs().max()))
        # rows of no text are left alone
        for x, inside in ((self.out, inside_q), (self.lse.T, inside_q), *(((self.grads[0], inside_q), (self.grads[1], inside_k),
                                                                          (self.grads[2], inside_k)) if grad else ())):
            assert bool((x[~inside.cuda()] == 7.0).all())
        if self.gap is not None and grad:
            assert bool((self.gap == 7.0).all())


LENGTHS = [[1], [2, 1, 3], [63, 64, 65], [127, 128, 129], [0, 255, 0, 0, 256, 1, 257, 0], [24] * 9, [700, 5, 383]]


@pytest.mark.parametrize("lens", LENGTHS, ids=lambda v: "-".join(map(str, v)))
@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "bf16"), (64, "f16"), (128, "f16")])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(lib, lens, dim, dtype, causal):
    c = Case(lib, lens, dim=dim, dtype=dtype, causal=causal, seed=len(lens))
    c.run()
    c.check()
    assert c.S.sama_device_status(c.ctx) == 0


# How a call is worked on depends on its mean number of rows per text, those of no text among them: with many of them, texts
# of any length are worked on as long ones are.
MANY = 1024     # rows of no text, before and behind, per text


@pytest.mark.parametrize("lens", LENGTHS + [[2305]], ids=lambda v: "-".join(map(str, v)))
@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (128, "f16")])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths_among_many_rows(lib, lens, dim, dtype, causal):
    c = Case(lib, lens, dim=dim, dtype=dtype, causal=causal, edge=MANY * len(lens), seed=len(lens))
    c.run()
    c.check()
    assert c.S.sama_device_status(c.ctx) == 0


@pytest.mark.parametrize("dim", [40, 64, 72, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [0.0, 2.0, 30.0])
def test_capped_and_biased_scores_among_many_rows(lib, dim, dtype, bias, cap):
    for causal, fused in ((False, True), (True, False)):
        c = Case(lib, [300, 1, 77], heads=4, kv=2, dim=dim, dtype=dtype, causal=causal, bias=bias, cap=cap, fused=fused,
                 edge=3 * MANY, seed=3)
        c.run()
        c.check()


@pytest.mark.parametrize("cap", [0.0, 20.0])
@pytest.mark.parametrize("dim", [64, 128])
def test_masks_among_many_rows(lib, cap, dim):
    lq, lk, prefix = [3, 0, 200, 130, 1, 5, 300], [0, 40, 500, 30, 700, 5, 299], [5, 5, 0, 20, 3, 0, 2]
    for causal, prefix in ((False, None), (True, None), (True, prefix)):
        c = Case(lib, lq, lk, heads=4, kv=2, dim=dim, causal=causal, prefix=prefix, cap=cap, edge=7 * MANY, seed=5)
        c.run()
        c.check()
    for bad in (NAN, math.inf):
        plain, other = (Case(lib, [70, 61, 200], heads=2, kv=1, dim=dim, causal=True, edge=3 * MANY, seed=7) for _ in range(2))
        for x in (other.q, other.k, other.v, other.dout):
            x[other.qs[1]:other.qs[2]] = bad
        plain.run()
        other.run()
        for x, y in zip((plain.out, *plain.grads), (other.out, *other.grads)):
            for t in (0, 2):
                at = slice(plain.qs[t], plain.qs[t + 1])
                assert torch.equal(x[at], y[at]) and bool(torch.isfinite(x[at]).all())


def test_large_scores_among_many_rows(lib):
    c = Case(lib, [400, 130], heads=2, kv=2, dim=128, edge=2 * MANY, seed=8, size=60.0, scale=1.0)
    ramp = torch.linspace(0.1, 20.0, c.nk, device="cuda")[:, None, None]
    c.k.copy_((c.k.float() * ramp).to(c.k.dtype))
    c.run()
    c.check()


@pytest.mark.parametrize("dim", [8, 16, 24, 40, 56, 72, 80, 96, 104, 120])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (6, 2), (7, 1)])
def test_head_sizes_and_shared_heads(lib, dim, heads, kv):
    c = Case(lib, [130, 33], heads=heads, kv=kv, dim=dim, dtype="f16" if dim % 16 else "bf16", causal=heads != 3, seed=dim)
    c.run()
    c.check()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("cap", [0.0, 2.0, 30.0])
def test_capped_and_biased_scores(lib, dim, dtype, bias, cap):
    for causal, fused in ((False, True), (True, False)):
        c = Case(lib, [300, 1, 77], heads=4, kv=2, dim=dim, dtype=dtype, causal=causal, bias=bias, cap=cap, fused=fused, seed=3)
        c.run()
        c.check()


@pytest.mark.parametrize("prefix", [[0, 0, 0], [300, 1, 40], [129, 1000, 0], [64, -5, 77]])
@pytest.mark.parametrize("dim", [64, 128])
def test_prefixes(lib, prefix, dim):
    c = Case(lib, [300, 9, 77], heads=2, kv=2, dim=dim, causal=True, prefix=prefix, seed=4)
    c.run()
    c.prefix = [max(0, p) for p in prefix]
    c.check()


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_other_keys_than_queries(lib, causal, dim):
    """Texts without keys or queries, more keys than queries, and causal texts with fewer: rows that see nothing."""
    lq, lk = [3, 0, 200, 130, 1, 5, 300], [0, 40, 500, 30, 700, 5, 299]
    c = Case(lib, lq, lk, heads=4, kv=2, dim=dim, causal=causal, bias=True, seed=5)
    c.run()
    c.check()
    empty = c.out[c.qs[0]:c.qs[1]]
    assert bool((empty == 0).all()) and bool((c.lse[:, c.qs[0]:c.qs[1]] == -math.inf).all())
    # ... except for a prefix
    c = Case(lib, lq, lk, heads=4, kv=2, dim=dim, causal=True, prefix=[5, 5, 0, 20, 3, 0, 2], seed=6)
    c.run()
    c.check()


def test_no_keys_no_queries_no_texts(lib):
    for lq, lk in (([4, 3], [0, 0]), ([0, 0], [4, 3]), ([0], [0])):
        c = Case(lib, lq, lk, edge=0)
        c.run()
        c.check()
    c = Case(lib, [], edge=3)
    c.run()
    c.check()
    assert c.S.sama_device_status(c.ctx) == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [NAN, math.inf, -math.inf])
def test_texts_do_not_reach_one_another(lib, dim, bad):
    """Every row of the middle text is not finite; the others come out bit for bit as without it."""
    lens = [70, 61, 200]
    plain, other = (Case(lib, lens, heads=2, kv=1, dim=dim, causal=True, seed=7) for _ in range(2))
    rows = slice(other.qs[1], other.qs[2])
    for x in (other.q, other.k, other.v, other.dout):
        x[rows] = bad
    plain.run()
    other.run()
    for x, y in zip((plain.out, *plain.grads), (other.out, *other.grads)):
        for t in (0, 2):
            at = slice(plain.qs[t], plain.qs[t + 1])
            assert torch.equal(x[at], y[at]) and bool(torch.isfinite(x[at]).all())


@pytest.mark.parametrize("cap", [0.0, 50.0])
def test_large_scores(lib, cap):
    """Scores in the thousands: weights of one and zero, a maximum that rises along the row."""
    c = Case(lib, [400, 130], heads=2, kv=2, dim=64, cap=cap, seed=8, size=60.0, scale=1.0)
    ramp = torch.linspace(0.1, 3.0, c.nk, device="cuda")[:, None, None]
    c.k.copy_((c.k.float() * ramp).to(c.k.dtype))
    c.run()
    c.check()


def test_gradients_against_differences(lib):
    """The derivative of <dout, out> along random directions, by fourth-order differences of the definition in 64 bits."""
    for causal, cap, bias in ((False, 0.0, False), (True, 3.0, True)):
        c = Case(lib, [150], heads=4, kv=2, dim=32, dtype="f16", causal=causal, cap=cap, bias=bias, edge=0, seed=9)
        c.run()
        x = [t.double() for t in (c.q, c.k, c.v)]
        _, bound = ref.text(*x, c.dout, "f16", c.scale, cap, c.slopes, causal, 0)

        def f(parts):
            r, _ = ref.text(*parts, None, "f16", c.scale, cap, c.slopes, causal, 0)
            return float((c.dout.double() * r["out"]).sum())

        for i, name in enumerate(("dq", "dk", "dv")):
            g = torch.Generator(device="cuda").manual_seed(i)
            d = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
            h = 1e-3
            at = [f([t + k * h * d if j == i else t for j, t in enumerate(x)]) for k in (-2, -1, 1, 2)]
            want = (at[0] - 8 * at[1] + 8 * at[2] - at[3]) / (12 * h)
            got = float((c.grads[i].double() * d).sum())
            # (the differences themselves: fifth derivatives times h^4, and 1e-16 / h)
            assert abs(got - want) <= float((bound[name] * d.abs()).sum()) + 1e-6 * abs(want) + 1e-8, name


def test_the_same_bits_again_on_another_stream_and_context(lib):
    c = Case(lib, [513, 24, 24, 700], heads=4, kv=2, dim=128, causal=True, fused=True, seed=10)
    c.run()
    want = [x.clone() for x in c.results()]
    other = c.S.sama_create(0, 1024, 0, None)
    side = torch.cuda.Stream()
    for ctx, stream in ((c.ctx, None), (other, None), (c.ctx, side)):
        c.ctx = ctx
        for x in c.results():
            x.fill_(7.0)
        torch.cuda.synchronize()
        c.run(stream)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(c.results(), want))
    c.S.sama_destroy(other)


def test_two_contexts_on_two_streams_at_once(lib):
    cases = [Case(lib, [300, 200], heads=4, kv=4, dim=64, causal=True, seed=s) for s in (11, 12)]
    for c in cases:
        c.run()
    want = [[x.clone() for x in c.results()] for c in cases]
    cases[1].ctx = lib[0].sama_create(0, 1024, 0, None)
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            c.run(s)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert all(torch.equal(x, y) for x, y in zip(c.results(), w))
    lib[0].sama_destroy(cases[1].ctx)


def test_captured_and_replayed(lib):
    from paper_2310_05674_b200 import binding as S
    ctx = S.sama_create(0, 1024, 0, None)
    c = Case((S, ctx), [100, 180], heads=2, kv=1, dim=64, causal=True, seed=13)

    def capture(fn):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            fn()
        return g

    def refused():
        with pytest.raises(S.SamaError) as e:
            c.S.sama_attention_grad(ctx, c.attn, c.q, c.k, c.v, c.out, c.lse, c.dout, *c.grads)
        assert e.value.status == S.SAMA_ERR_NOMEM       # the workspace is not there yet

    capture(refused)
    c.run()
    want = [x.clone() for x in c.results()]
    graph = capture(c.run)
    for x in c.results():
        x.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(c.results(), want))
    # new texts in the same place
    c.lq = c.lk = [30, 250]
    c.qs = c.ks = starts(c.lq, c.edge)
    c.starts_q.copy_(torch.tensor(c.qs, dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    c.check()
    assert S.sama_device_status(ctx) == 0
    S.sama_destroy(ctx)


@pytest.mark.parametrize("bad", [[0, 50, 20, 90], [0, 50, 60, 1000], [-7, 50, 60, 90], [200, 300, 400, 500], [9, 8, 7, 6]])
def test_starts_out_of_order_or_range_are_reported(lib, bad):
    """They are taken as the nearest row, so that nothing outside the tensors is touched."""
    c = Case(lib, [30, 30, 30], edge=0)
    c.forward()
    assert c.S.sama_device_status(c.ctx) == 0
    c.starts_q.copy_(torch.tensor(bad, dtype=torch.int32))
    c.forward()
    assert c.S.sama_device_status(c.ctx) == c.S.SAMA_DEV_BAD_INDEX
    c.run()
    assert c.S.sama_device_status(c.ctx) == c.S.SAMA_DEV_BAD_INDEX


def test_many_texts(lib):
    """The search for a block's text, over more texts than one step of it covers, empty ones among them."""
    g = torch.Generator().manual_seed(1)
    lens = (torch.randint(0, 40, (3000,), generator=g) * (torch.rand(3000, generator=g) < 0.5)).tolist()
    c = Case(lib, lens, heads=1, kv=1, dim=16, seed=14)
    c.run()
    torch.cuda.synchronize()
    # a sample against the definition, all of them against one text at a time
    for t in [0, 1, 1499, 2998, 2999] + [i for i, n in enumerate(lens) if n > 36][:20]:
        a = slice(c.qs[t], c.qs[t + 1])
        want, bound = ref.text(c.q[a], c.k[a], c.v[a], c.dout[a], c.dtype, c.scale, 0.0, None, False, 0)
        for name, x in (("out", c.out[a]), ("dq", c.grads[0][a]), ("dk", c.grads[1][a]), ("dv", c.grads[2][a])):
            assert bool(((x.double() - want[name]).abs() <= bound[name]).all()), (t, name)
    assert bool(torch.isfinite(c.out[c.edge:-c.edge]).all()) and bool((c.out[:c.edge] == 7).all())


def test_rows_far_apart(lib):
    """Offsets that pass 32 bits: keys and values 2^29 elements apart."""
    S, ctx = lib
    stride, n, h, d = 1 << 29, 6, 2, 64
    big = torch.empty((n - 1) * stride + 2 * h * d, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(15)
    q, k0, v0, dout = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for _ in range(4))
    k, v = (big.as_strided((n, h, d), (stride, d, 1), at * h * d) for at in (0, 1))
    k.copy_(k0)
    v.copy_(v0)
    at = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(h, n, device="cuda")
    a = S.Attn(S.SAMA_BF16, h, h, d, n, n, at, causal=True, k_stride=stride, v_stride=stride)
    S.sama_attention(ctx, a, q, k, v, out, lse)
    want, bound = ref.text(q, k0, v0, dout, "bf16", d ** -0.5, 0.0, None, True, 0)
    assert bool(((out.double() - want["out"]).abs() <= bound["out"]).all())
    grads = [torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)]
    b = S.Attn(S.SAMA_BF16, h, h, d, n, n, at, causal=True)
    S.sama_attention_grad(ctx, b, q, k0, v0, out, lse, dout, *grads)
    for name, x in zip(("dq", "dk", "dv"), grads):
        assert bool(((x.double() - want[name]).abs() <= bound[name]).all()), name
