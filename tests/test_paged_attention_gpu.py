"""Attention of one new token over a paged cache, against the definition in 64 bits (attention_reference.py, which derives
the tolerances: a sequence is a text with one query)."""
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


class Case:
    """Caches in which everything that no sequence has is NaN: other pages, rows behind a sequence's last, and (with new
    tokens) the new token's place.  K and V of a page lie behind one another, so pages are twice as far apart."""

    def __init__(self, lib, lens, heads=4, kv=2, dim=64, dtype="bf16", page=16, cap=0.0, bias=False, new=True, columns=None,
                 seed=0, together=True):
        self.S, self.ctx = lib
        S = self.S
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.lens, self.dtype, self.cap, self.new, self.dim = lens, dtype, cap, new, dim
        dt, n = ref.DT[dtype], len(lens)
        need = [-(-x // page) for x in lens]
        n_pages = sum(need) + 5
        buf = torch.full((n_pages, 2, page, kv, dim), NAN, dtype=dt, device="cuda")
        self.caches = [buf[:, 0], buf[:, 1]] if together else [buf[:, 0].contiguous(), buf[:, 1].contiguous()]
        order = torch.randperm(n_pages, generator=g, device="cuda")[:sum(need)]
        self.table = torch.full((n, columns or max(need + [1])), -7, dtype=torch.int32, device="cuda")
        r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)  # noqa: E731
        self.q, self.fresh = 2 * r(n, heads, dim), [r(n, kv, dim), r(n, kv, dim)]
        self.rows, at = [], 0
        for s, (length, pages) in enumerate(zip(lens, need)):
            self.table[s, :pages] = order[at:at + pages].to(torch.int32)
            j = torch.arange(length, device="cuda")
            where = (order[at:at + pages][j // page], j % page) if length else None
            rows = [r(length, kv, dim), r(length, kv, dim)]
            if length:
                for x, f, cache in zip(rows, self.fresh, self.caches):
                    if new:
                        x[-1] = f[s]
                    cache[where] = x
                    if new:
                        cache[where[0][-1], where[1][-1]] = NAN
            self.rows.append((where, rows))
            at += pages
        self.slopes = 0.5 ** torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) if bias else None
        self.lengths = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.out = torch.full((n, heads, dim), 7.0, dtype=dt, device="cuda")
        self.before = [c.clone() for c in self.caches]
        self.paged = S.Paged(S.DTYPES[dtype], heads, kv, dim, page, n_pages, self.table, self.lengths, slopes=self.slopes, cap=cap,
                             page_stride=2 * page * kv * dim if together else 0)

    def run(self, stream=None):
        k, v = self.fresh if self.new else (None, None)
        self.S.sama_paged_attention(self.ctx, self.paged, self.q, k, v, *self.caches, self.out, stream)

    def check(self, skip=()):
        for s, (where, (k, v)) in enumerate(self.rows):
            if s in skip:
                continue
            if where is None:
                assert bool((self.out[s] == 0).all())
                continue
            want, bound = ref.text(self.q[s:s + 1], k, v, None, self.dtype, self.dim ** -0.5, self.cap, self.slopes, False, 0)
            over = (self.out[s:s + 1].double() - want["out"]).abs() - bound["out"]
            assert bool((over <= 0).all()), (s, self.lens[s], float(over.max()))
            for before, x in zip(self.before, (k, v)):
                if self.new:
                    before[where[0][-1], where[1][-1]] = x[-1]
        if not skip:
            for cache, want in zip(self.caches, self.before):     # the new token's rows, and nothing else
                assert torch.equal(cache.contiguous().view(torch.int16), want.contiguous().view(torch.int16))


LENGTHS = [1, 0, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 0, 1000]


@pytest.mark.parametrize("page", [1, 3, 7, 16, 48, 64, 128, 2000])
@pytest.mark.parametrize("new", [False, True])
@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16")])
def test_lengths_and_pages(lib, page, new, dim, dtype):
    c = Case(lib, LENGTHS, dim=dim, dtype=dtype, page=page, new=new, seed=page)
    c.run()
    c.check()
    assert c.S.sama_device_status(c.ctx) == 0


@pytest.mark.parametrize("dim", [8, 24, 40, 64, 72, 96, 120, 128])
@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 1), (7, 1), (8, 1), (9, 1), (40, 2), (6, 6)])
def test_head_sizes_and_shared_heads(lib, dim, heads, kv):
    c = Case(lib, [70, 200, 1, 0], heads=heads, kv=kv, dim=dim, dtype="bf16" if dim % 16 else "f16", seed=dim, together=dim != 64)
    c.run()
    c.check()


@pytest.mark.parametrize("cap", [0.0, 2.0, 30.0])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dim,dtype", [(64, "f16"), (128, "bf16")])
def test_capped_and_biased_scores(lib, cap, bias, dim, dtype):
    c = Case(lib, [333, 5, 90], heads=8, kv=2, dim=dim, dtype=dtype, cap=cap, bias=bias, seed=1)
    c.run()
    c.check()


@pytest.mark.parametrize("lens", [[100000], [30000, 5, 50001], [1] * 700, [3, 0] * 1000 + [9000], [2047] * 37],
                         ids=["one", "three", "ones", "many", "equal"])
def test_work_is_shared_whatever_the_lengths(lib, lens):
    c = Case(lib, lens, heads=2, kv=1, dim=64, seed=2, columns=8000)
    c.run()
    torch.cuda.synchronize()
    if len(lens) <= 100:
        c.check()
        return
    # a sample against the definition
    for s in [i for i, n in enumerate(lens) if n and (i % 97 < 2 or i > len(lens) - 4)]:
        want, bound = ref.text(c.q[s:s + 1], *c.rows[s][1], None, c.dtype, c.dim ** -0.5, 0.0, None, False, 0)
        assert bool(((c.out[s:s + 1].double() - want["out"]).abs() <= bound["out"]).all()), s
    zero = torch.tensor([x == 0 for x in lens], device="cuda")
    assert bool((c.out[zero] == 0).all()) and bool(torch.isfinite(c.out).all())


def test_the_same_bits_again(lib):
    c = Case(lib, [5000, 77, 0, 1200, 9000], heads=8, kv=2, dim=128, seed=3)
    c.run()
    want = c.out.clone()
    side = torch.cuda.Stream()
    other = c.S.sama_create(0, 1024, 0, None)
    for ctx, stream in ((c.ctx, None), (c.ctx, side), (other, None)):
        c.ctx = ctx
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):
            c.run(stream)
        torch.cuda.synchronize()
        assert torch.equal(c.out, want)
    c.S.sama_destroy(other)


def test_a_generation_step_by_step_in_a_graph(lib):
    """Captured once, replayed with lengths and tokens that change in place: every step appends a token and reads it."""
    from paper_2310_05674_b200 import binding as S
    ctx = S.sama_create(0, 1024, 0, None)
    heads, kv, dim, page, n = 4, 2, 64, 4, 3
    g = torch.Generator(device="cuda").manual_seed(4)
    caches = [torch.full((20, page, kv, dim), NAN, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.randperm(20, generator=g, device="cuda").to(torch.int32)[:18].view(n, 6).contiguous()
    lengths = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")       # sequences start one step apart
    q, k, v = (torch.zeros(n, h, dim, dtype=torch.bfloat16, device="cuda") for h in (heads, kv, kv))
    out = torch.empty_like(q)
    p = S.Paged(S.SAMA_BF16, heads, kv, dim, page, 20, table, lengths)
    history = [[], [], []]

    def step():
        S.sama_paged_attention(ctx, p, q, k, v, *caches, out)

    def refused():
        with pytest.raises(S.SamaError) as e:
            step()
        assert e.value.status == S.SAMA_ERR_NOMEM

    torch.cuda.synchronize()
    for what in ("refused", "eager", "captured"):
        if what == "eager":
            lengths.zero_()
            step()
            torch.cuda.synchronize()
            lengths.copy_(torch.tensor([0, 0, 0], dtype=torch.int32))
            continue
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            refused() if what == "refused" else step()
    for i in range(20):
        for x in (q, k, v):
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        lengths.copy_(torch.tensor([max(0, i + 1 - s) for s in range(n)], dtype=torch.int32))
        graph.replay()
        for s in range(n):
            if i >= s:
                history[s].append((k[s].clone(), v[s].clone()))
                ks, vs = (torch.stack([h[x] for h in history[s]]) for x in (0, 1))
                want, bound = ref.text(q[s:s + 1], ks, vs, None, "bf16", dim ** -0.5, 0.0, None, False, 0)
                assert bool(((out[s:s + 1].double() - want["out"]).abs() <= bound["out"]).all()), (i, s)
    torch.cuda.synchronize()
    assert S.sama_device_status(ctx) == 0
    S.sama_destroy(ctx)


def test_bad_pages_and_lengths_are_reported(lib):
    """Keys on pages that do not exist are left out; lengths are taken as the nearest that the table holds."""
    c = Case(lib, [100, 64, 33], page=16, new=False, seed=5)
    c.run()
    assert c.S.sama_device_status(c.ctx) == 0
    c.table[0, 2] = c.paged.a.n_pages
    c.table[0, 3] = -1
    c.run()
    assert c.S.sama_device_status(c.ctx) == c.S.SAMA_DEV_BAD_INDEX
    c.check(skip=(0,))
    keep = torch.ones(100, dtype=torch.bool, device="cuda")
    keep[32:64] = False
    k, v = (x[keep] for x in c.rows[0][1])
    want, bound = ref.text(c.q[:1], k, v, None, c.dtype, c.dim ** -0.5, 0.0, None, False, 0)
    assert bool(((c.out[:1].double() - want["out"]).abs() <= bound["out"]).all())
    c.table[0] = -1                                   # no page at all: nothing to attend to
    c.run()
    assert c.S.sama_device_status(c.ctx) == c.S.SAMA_DEV_BAD_INDEX and bool((c.out[0] == 0).all())
    d = Case(lib, [112, 64, 33], page=16, new=False, seed=6)
    want = (d.run(), d.out.clone())[1]
    d.lengths.copy_(torch.tensor([1 << 30, 64, -5], dtype=torch.int32))
    d.run()
    assert d.S.sama_device_status(d.ctx) == d.S.SAMA_DEV_BAD_INDEX
    assert torch.equal(d.out[:2], want[:2]) and bool((d.out[2] == 0).all())
    # a new token whose page does not exist is used, but not kept
    e = Case(lib, [17, 16], page=16, seed=7)
    e.table[0, 1] = 1 << 20
    e.run()
    assert e.S.sama_device_status(e.ctx) == e.S.SAMA_DEV_BAD_INDEX
    want, bound = ref.text(e.q[:1], *e.rows[0][1], None, e.dtype, e.dim ** -0.5, 0.0, None, False, 0)
    assert bool(((e.out[:1].double() - want["out"]).abs() <= bound["out"]).all())


def test_pages_far_apart(lib):
    """Offsets that pass 32 bits: pages 2^30 elements apart."""
    S, ctx = lib
    kv, dim, page, stride = 1, 64, 16, 1 << 30
    big = torch.empty(3 * stride + 2 * page * dim, dtype=torch.bfloat16, device="cuda")
    caches = [big.as_strided((4, page, kv, dim), (stride, kv * dim, dim, 1), at * page * dim) for at in (0, 1)]
    g = torch.Generator(device="cuda").manual_seed(8)
    k, v = (torch.randn(64, kv, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.tensor([[3, 0, 2, 1]], dtype=torch.int32, device="cuda")
    for cache, x in zip(caches, (k, v)):
        for j in range(4):
            cache[int(table[0, j])] = x[16 * j:16 * j + 16]
    q = torch.randn(1, 2, dim, generator=g, device="cuda").bfloat16()
    out, lengths = torch.empty_like(q), torch.tensor([64], dtype=torch.int32, device="cuda")
    p = S.Paged(S.SAMA_BF16, 2, kv, dim, page, 4, table, lengths, page_stride=stride)
    S.sama_paged_attention(ctx, p, q, None, None, *caches, out)
    want, bound = ref.text(q, k, v, None, "bf16", dim ** -0.5, 0.0, None, False, 0)
    assert bool(((out.double() - want["out"]).abs() <= bound["out"]).all())
