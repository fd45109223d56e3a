"""Distillation from a teacher's top logits against the definition in 64 bits.

Tolerances, with x = (z - max z) / T: an exponential's argument is off by a few units of 2^-24 of the terms it is made of,
(|z| + |max z|) / T, and the exponential itself by 2^-22, so each is off by a factor of at most 1 + E,
E = 2^-21 (max (|z| + |max z|) / T + 1); a sum of n terms, of which a thread adds m and then log2 n partial sums are
joined, by (m + 16) 2^-24 more.  A weight q or p is then off by twice that, a logarithm by as much plus 2^-22 of itself.
The gradient is rounded once, to half a unit in the last place (and half a subnormal step) of its type.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


class Case:
    def __init__(self, lib, n, vocab, k, dtype="f32", top="f32", T=2.0, ld=None, ld_grad=None, shift=0, shift_grad=None, ragged=False,
                 weighted=True, seed=0, size=2.5, grad_scale=1.0):
        self.S, self.ctx = lib
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.vocab, self.k, self.dtype, self.T, self.top_type, self.scale = n, vocab, k, dtype, T, top, grad_scale

        def rows(ld, shift):      # between rows, before and behind them: NaN
            buf = torch.full((n * ld + shift + 16,), NAN, dtype=DT[dtype], device="cuda")
            return buf, buf[shift:shift + n * ld].view(n, ld)[:, :vocab]

        self.z_buf, self.z = rows(ld or vocab, shift)
        self.z.copy_(size * torch.randn(n, vocab, generator=g, device="cuda"))
        self.g_buf, self.grad = rows(ld_grad or ld or vocab, shift if shift_grad is None else shift_grad)
        self.ids = torch.rand(n, vocab, generator=g, device="cuda").argsort(1)[:, :k].to(torch.int32).contiguous()
        self.top = (2 * torch.randn(n, k, generator=g, device="cuda")).to(DT[top])
        if ragged:
            keep = torch.randint(0, k + 1, (n, 1), generator=g, device="cuda")
            self.ids[torch.arange(k, device="cuda") >= keep] = -1
        self.weight = torch.sigmoid(torch.randn(n, generator=g, device="cuda")) if weighted else None
        self.loss = torch.full((n,), NAN, device="cuda")

    def run(self, loss=True, grad=True, stream=None):
        S = self.S
        S.sama_distill(self.ctx, S.DTYPES[self.dtype], self.n, self.vocab, self.z, self.k, S.DTYPES[self.top_type], self.top, self.ids,
                       self.T, self.weight, self.scale, self.loss if loss else None, self.grad if grad else None, stream=stream)

    def reference(self):
        z, T = self.z.double(), self.T
        used = (self.ids >= 0) & (self.ids < self.vocab)
        ids = torch.where(used, self.ids, 0).long()
        u = torch.where(used, self.top.double() / T, -math.inf)
        some = (u > -math.inf).any(1, keepdim=True)
        p = torch.where(some, torch.softmax(u, 1), 0.0)
        logq = torch.log_softmax(z / T, 1)
        size = (z.abs() + z.abs().amax(1, keepdim=True)).amax(1, keepdim=True) / T
        vec = max(64, self.vocab / 1024)
        e = 2.0 ** -21 * (size + 1) + (vec + 16) * 2.0 ** -24
        eu = 2.0 ** -21 * (2 * torch.where(u > -math.inf, self.top.double(), 0.0).abs().amax(1, keepdim=True) / T + 1) + 20 * 2.0 ** -24
        lq, lp = logq.gather(1, ids), torch.log(p)
        term = torch.where(p > 0, p * (lp - lq), 0.0)
        loss = T * T * term.sum(1)
        eterm = torch.where(p > 0, p * (2 * eu * (lp - lq).abs() + 2 * eu + 2 * e + 2.0 ** -22 * (lp.abs() + lq.abs() + size + 1)), 0.0)
        eloss = T * T * (eterm.sum(1) + 2.0 ** -23 * 32 * term.abs().sum(1)) + 2.0 ** -100
        w = torch.ones(self.n, device="cuda", dtype=torch.float64) if self.weight is None else self.weight.double()
        f = (self.scale * T * w)[:, None] * some
        q = torch.exp(logq)
        dense = torch.zeros_like(q).scatter_add_(1, ids, p)
        grad = f * (q - dense)
        eg = f.abs() * (2 * e * q + 2 * eu.amax(1, keepdim=True) * dense + 2.0 ** -22 * (q + dense))
        return loss, eloss, grad, U[self.dtype] * (grad.abs() + eg) + eg + TINY[self.dtype]

    def check(self, loss=True, grad=True):
        want, bound, g, bg = self.reference()
        if loss:
            over = (self.loss.double() - want).abs() - bound
            assert bool((over <= 0).all()), float(over.max())
        if grad:
            over = (self.grad.double() - g).abs() - bg
            assert bool((over <= 0).all()), (float(over.max()), int(over.argmax()))
            inside = torch.zeros_like(self.g_buf, dtype=torch.bool)
            inside.as_strided(self.grad.shape, self.grad.stride(), self.grad.storage_offset()).fill_(True)
            assert bool(torch.isnan(self.g_buf[~inside]).all())      # what lies between rows is left alone


# rows of each kind of team, at its limits: a warp up to 4 KB, a CTA up to 32, clusters of 2, 4, 8, of 8 larger CTAs up to 512
VOCABS = {"f32": [1, 2, 3, 5, 50, 1020, 1023, 1024, 1025, 8188, 8191, 8193, 16381, 20001, 40003, 65537, 131068, 131071, 140001],
          "bf16": [1, 7, 8, 9, 2039, 2048, 2050, 16371, 16383, 16385, 32768, 50021, 131055, 131072, 262143, 262145],
          "f16": [3, 100, 2041, 16384, 33333, 100001, 200003]}


@pytest.mark.parametrize("dtype,vocab", [(d, v) for d in VOCABS for v in VOCABS[d]])
def test_vocabularies(lib, dtype, vocab):
    for n, shift, seed in ((5, 0, 0), (3, 1, 1), (2, 3, 2)):
        c = Case(lib, n, vocab, min(vocab, 9), dtype, shift=shift, seed=seed)
        c.run()
        c.check()
    assert c.S.sama_device_status(c.ctx) == 0


@pytest.mark.parametrize("vocab", [37, 3001, 50021])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(lib, vocab, dtype):
    for ld, ld_grad, shift, shift_grad in ((vocab + 3, vocab + 3, 0, 0), (vocab + 11, vocab, 1, 5), (-(-vocab // 64) * 64, None, 8, 8), (vocab, vocab + 2, 2, 3)):
        c = Case(lib, 9, vocab, 7, dtype, ld=ld, ld_grad=ld_grad, shift=shift, shift_grad=shift_grad, seed=3)
        c.run()
        c.check()


@pytest.mark.parametrize("k,vocab", [(1, 1), (1, 5000), (127, 500), (128, 600), (129, 600), (500, 40000), (1024, 1024), (1024, 30000), (1000, 300000)])
@pytest.mark.parametrize("top", ["f32", "bf16", "f16"])
def test_numbers_of_entries(lib, k, vocab, top):
    for ragged in (False, True):
        c = Case(lib, 4, vocab, k, "bf16", top=top, ragged=ragged, seed=k)
        c.run()
        c.check()


@pytest.mark.parametrize("n", [1, 7, 295, 297, 2500])
@pytest.mark.parametrize("vocab,dtype", [(500, "bf16"), (9001, "f32"), (20000, "bf16")])
def test_numbers_of_rows(lib, n, vocab, dtype):
    c = Case(lib, n, vocab, 16, dtype, ragged=True, seed=n)
    c.run()
    c.check()


@pytest.mark.parametrize("vocab", [300, 9000, 70000, 300000])
def test_the_same_id_more_than_once(lib, vocab):
    c = Case(lib, 6, vocab, 40, "f32", seed=4)
    c.ids[1, 5] = c.ids[1, 30]
    c.ids[2, :] = 17
    c.ids[3, 10:] = c.ids[3, :10].repeat(3)
    c.ids[4, 39] = c.ids[4, 0]
    c.run()
    c.check()


@pytest.mark.parametrize("vocab", [300, 9000, 70000, 300000])
def test_rows_without_entries_or_weight(lib, vocab):
    c = Case(lib, 8, vocab, 12, "bf16", seed=5)
    c.ids[1] = -1                            # no entry
    c.top[2] = -math.inf                     # none above -infinity
    c.top[3, :11] = -math.inf                # one
    c.weight[4] = 0.0
    c.run()
    c.check()
    assert bool((c.grad[[1, 2, 4]] == 0).all()) and bool((c.loss[[1, 2]] == 0).all())
    # whatever the logits of such rows are
    for bad in (NAN, math.inf, -math.inf):
        c.z[[1, 2, 4]] = bad
        c.run()
        assert bool((c.grad[[1, 2, 4]] == 0).all()) and bool((c.loss[[1, 2]] == 0).all())
        assert bool(torch.isfinite(c.grad).all()) and bool(torch.isfinite(c.loss[[0, 3, 5, 6, 7]]).all())


@pytest.mark.parametrize("vocab", [300, 9000, 70000, 300000])
def test_masked_logits(lib, vocab):
    """Entries of the vocabulary at -infinity, and at the lowest value of the type, have no weight; a target there has an
    infinite loss, one without weight none."""
    c = Case(lib, 4, vocab, 8, "bf16", seed=6)
    masked = torch.arange(vocab, device="cuda") % 3 == 1
    c.ids.copy_(c.ids - c.ids % 3)           # targets that are not masked
    c.z[0, masked] = -math.inf
    c.z[1, masked] = torch.finfo(torch.bfloat16).min
    c.z[2, masked] = -math.inf
    c.ids[2, 3] = 1
    c.z[3, masked] = -math.inf
    c.ids[3, 3], c.top[3, 3] = 1, -math.inf
    c.run()
    assert float(c.loss[2]) == math.inf
    assert bool((c.grad[0, masked] == 0).all()) and bool((c.grad[1, masked] == 0).all())
    z = c.z.clone()
    c.z[:, masked] = -1e4                    # (with T = 2, a weight below any fp32 value)
    want, bound, g, bg = c.reference()
    # the bound of the finite stand-in is far too wide: that of the values that are left
    c.z.copy_(z)
    keep = [0, 1, 3]
    assert bool(((c.loss.double() - want).abs()[keep] <= 1e-4 * (1 + want.abs()[keep])).all())
    assert bool(((c.grad.double() - g).abs()[keep] <= 2.0 ** -8 * g.abs()[keep] + 1e-5).all())


@pytest.mark.parametrize("vocab", [300, 2500, 9000, 70000, 300001])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("T", [0.25, 1.0])
def test_rows_of_the_lowest_and_the_largest_value(lib, vocab, dtype, T):
    """Logits whose products with log2 e / T are beyond fp32, or have no digits left behind the point.  A row of one value is a row of zeros, and next to the largest
    value the lowest has no weight."""
    c = Case(lib, 4, vocab, 8, dtype, T=T, seed=9)
    low, high = torch.finfo(c.z.dtype).min, torch.finfo(c.z.dtype).max
    few = torch.arange(vocab, device="cuda") % 4 == 0
    c.ids.copy_(c.ids - c.ids % 4)           # targets among the few
    stand_in = torch.zeros_like(c.z)
    stand_in[2, ~few] = -200.0 * T           # (a weight below any fp32 value)
    c.z[0], c.z[1], c.z[2], c.z[3] = low, high, torch.where(few, high, low), -high / 2
    c.top[0], c.top[1] = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    c.run()
    z, top = c.z.clone(), c.top.clone()
    c.z.copy_(stand_in)
    c.top[:2] = 0.0
    want, bound, g, bg = c.reference()
    assert bool(((c.loss.double() - want).abs() <= bound).all())
    assert bool(((c.grad.double() - g).abs() <= bg).all())
    c.z.copy_(z)
    c.top.copy_(top)
    assert c.S.sama_device_status(c.ctx) == 0


def test_ids_out_of_range_are_reported(lib):
    for vocab in (300, 9000, 70000, 300000):
        c = Case(lib, 4, vocab, 6, "f32", seed=7)
        c.ids[1, 2] = -1
        c.run()
        assert c.S.sama_device_status(c.ctx) == 0
        c.ids[2, 1], c.ids[3, 5] = vocab, -2
        c.run()
        assert c.S.sama_device_status(c.ctx) == c.S.SAMA_DEV_BAD_INDEX
        c.check()


@pytest.mark.parametrize("vocab", [301, 9001, 70003, 300001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_in_parts(lib, vocab, dtype):
    c = Case(lib, 700, vocab, 5, dtype, seed=8) if vocab < 70000 else Case(lib, 50, vocab, 5, dtype, seed=8)
    c.run()
    loss, grad = c.loss.clone(), c.grad.clone()
    c.loss.fill_(NAN)
    c.run(grad=False)
    assert torch.equal(c.loss, loss)
    c.grad.fill_(NAN)
    c.run(loss=False)
    assert torch.equal(c.grad, grad)
    c.grad = c.z
    c.run()
    assert torch.equal(c.z, grad) and torch.equal(c.loss, loss)


@pytest.mark.parametrize("T", [0.25, 1.0, 20.0])
def test_temperatures(lib, T):
    for vocab in (300, 20000):
        c = Case(lib, 5, vocab, 10, "f32", T=T, weighted=False, seed=9, size=6.0, grad_scale=-0.5)
        c.run()
        # (a negative scale turns the gradient round)
        want, bound, g, bg = c.reference()
        assert bool(((c.loss.double() - want).abs() <= bound).all())
        assert bool(((c.grad.double() - g).abs() <= bg.abs()).all())


def test_gradient_against_differences(lib):
    c = Case(lib, 3, 50, 6, "f32", T=1.5, seed=10)
    c.run()
    z = c.z.double()

    def f(x):
        p = torch.softmax(c.top.double() / c.T, 1)
        lq = torch.log_softmax(x / c.T, 1).gather(1, c.ids.long())
        return float((c.weight.double() * c.T * c.T * (p * (torch.log(p) - lq)).sum(1)).sum())

    d = torch.randn(z.shape, dtype=torch.float64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    h = 1e-3
    want = (f(z - 2 * h * d) - 8 * f(z - h * d) + 8 * f(z + h * d) - f(z + 2 * h * d)) / (12 * h)
    _, _, _, bg = c.reference()
    assert abs(float((c.grad.double() * d).sum()) - want) <= float((bg * d.abs()).sum()) + 1e-8


def test_the_same_bits_again_captured_and_on_another_stream(lib):
    for vocab in (500, 9000, 50021, 140000):
        c = Case(lib, 40, vocab, 10, "f32", seed=11)
        c.run()
        want = [c.loss.clone(), c.grad.clone()]
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        for go in (lambda: c.run(stream=side), graph.replay):
            c.loss.fill_(NAN)
            c.grad.fill_(NAN)
            torch.cuda.synchronize()
            go()
            torch.cuda.synchronize()
            assert torch.equal(c.loss, want[0]) and torch.equal(c.grad, want[1])


def test_rows_far_apart(lib):
    """Offsets that pass 32 bits."""
    S, ctx = lib
    n, vocab, ld = 5, 5000, 1 << 29
    big = torch.empty((n - 1) * ld + vocab, dtype=torch.float32, device="cuda")
    c = Case(lib, n, vocab, 6, "f32", seed=12)
    c.run()
    z = big.as_strided((n, vocab), (ld, 1))
    z.copy_(c.z)
    loss = torch.empty_like(c.loss)
    S.sama_distill(ctx, S.SAMA_F32, n, vocab, z, c.k, S.SAMA_F32, c.top, c.ids, c.T, c.weight, 1.0, loss, z)
    assert torch.equal(loss, c.loss) and torch.equal(z, c.grad)
