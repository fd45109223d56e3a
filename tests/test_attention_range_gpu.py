"""fp16 holds 2^-14 to 65504 in full: gradients are as exact for small and large d_out, and many keys, as anywhere.

Bound: test_attention_offsets_gpu.py's, a relative one on the whole gradient, and what storing it in fp16 costs: half of the
smallest step, 2^-25, per element."""
import math

import pytest
import torch

import attention_reference as ref
from test_attention_offsets_gpu import run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


@pytest.mark.parametrize("dout", [1e-6, 1e-4, 1e-3, 1.0, 1e3])
@pytest.mark.parametrize("dim,lens,heads,kv", [(64, [2048], 2, 1), (64, [300, 1, 900], 4, 2), (128, [8192], 1, 1), (40, [700, 333], 2, 2)])
def test_size_of_the_incoming_gradient(lib, dout, dim, lens, heads, kv):
    for causal, cap in ((False, 0.0), (True, 20.0)):
        wrong, allowed, size = run(lib, lens, heads, kv, dim, "f16", causal, cap, False, 0.0, 0.0, dout_size=dout, seed=dim)
        for name, h, a, b, c in zip(("dq", "dk", "dv"), (heads, kv, kv), wrong, allowed, size):
            stored = math.sqrt(sum(lens) * h * dim) * 2.0 ** -25
            assert a <= math.sqrt(b * b + stored * stored), (name, causal, a / c, b / c, stored / c)


def gradients(lib, q, k, v, dout, causal):
    """For each gradient of one text of one head: the norm of what it is off by, and what it may be."""
    S, ctx = lib
    (n, _, dim), m = q.shape, k.shape[0]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    a = S.Attn(S.SAMA_F16, 1, 1, dim, n, m, i32(0, n), i32(0, m), causal=causal)
    out, lse = torch.empty_like(q), torch.empty(1, n, device="cuda")
    grads = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
    S.sama_attention(ctx, a, q, k, v, out, lse)
    S.sama_attention_grad(ctx, a, q, k, v, out, lse, dout, *grads)
    Q, K, V, D = (x[:, 0].double() for x in (q, k, v, dout))
    x = Q @ K.T * dim ** -0.5
    p = torch.softmax(torch.where(ref.visible(n, m, causal, 0, "cuda"), x, -math.inf), -1)
    o = p @ V
    dx = p * (D @ V.T - (D * o).sum(-1, keepdim=True)) * dim ** -0.5
    want = [dx @ K, dx.T @ Q, p.T @ D]
    # each rounded operand, and the result
    allowed = [(dx.square() @ K.square().sum(-1)).sum(), (dx.T.square() @ Q.square().sum(-1)).sum(), (p.T.square() @ D.square().sum(-1)).sum()]
    # beyond 65504 the right value is infinite (the values next to it, which rounding may take to either side, are left out)
    errors = []
    for g, w, e in zip(grads, want, allowed):
        g = g[:, 0].double()
        over, fits = w.abs() > 65504 * 1.01, w.abs() < 65504 * 0.99
        assert torch.equal(g[over], math.inf * w[over].sign())
        errors.append((float((g - w)[fits].norm()), math.sqrt(float(e + w.square().sum()) * 2.0 ** -22 + w.numel() * 2.0 ** -50)))
    return errors


def test_many_keys(lib):
    """Weights of 2^-18."""
    g = torch.Generator(device="cuda").manual_seed(0)
    r = lambda n: torch.randn(n, 1, 64, generator=g, device="cuda").half()  # noqa: E731
    errors = gradients(lib, r(70), r(200000), r(200000), (100 * r(70).float()).half(), False)
    for name, (wrong, allowed) in zip(("dq", "dk", "dv"), errors):
        assert wrong <= allowed, (name, wrong, allowed)


def test_queries_of_different_sizes(lib):
    """A gradient that comes to a text's last rows alone, or is far smaller there, as a weight per token makes it."""
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda n: torch.randn(n, 1, 64, generator=g, device="cuda").half()  # noqa: E731
    q, k, v, d = r(1000), r(1000), r(1000), r(1000)
    for factor in (1e-4, 0.0, 1e4):
        dout = d.clone()
        dout[:700] = (dout[:700].float() * factor).half()
        for causal in (False, True):
            for name, (wrong, allowed) in zip(("dq", "dk", "dv"), gradients(lib, q, k, v, dout, causal)):
                assert wrong <= allowed, (name, factor, causal, wrong, allowed)


def test_values_that_make_large_products(lib):
    """dX beyond 65504 (a few keys, which share the weights), of which dQ is not."""
    g = torch.Generator(device="cuda").manual_seed(2)
    r = lambda n, s=1.0: (s * torch.randn(n, 1, 128, generator=g, device="cuda")).half()  # noqa: E731
    k = r(500, 0.02)
    errors = gradients(lib, r(300, 50.0), k, r(500, 4.0), r(300, 8000.0), False)
    more = gradients(lib, r(300, 0.1), r(500, 0.1), r(500, 4.0), r(300, 8000.0), False)
    few = gradients(lib, r(300), r(4), r(4, 4.0), r(300, 8000.0), False)
    for name, (wrong, allowed) in zip(("dq", "dk", "dv") * 3, errors + more + few):
        assert wrong <= allowed, (name, wrong, allowed)


# Four keys with most of the weight (of each 16 that are worked on together among the first 64, one), whose values are zeros, and some
# 100,000 of one kind: each of those has 128.5 / 2^24 of a weight, which fp16 as it stands rounds by half a step of 2^-24, all of
# them to the same side.
KEYS, HEAVY, WEIGHT = 100001, [0, 16, 32, 48], 128.5 * 2.0 ** -24


def few_and_many(dim):
    g = torch.Generator(device="cuda").manual_seed(dim)
    k = torch.zeros(KEYS, 1, dim, dtype=torch.float16, device="cuda")
    k[HEAVY, 0, 0] = 1.0
    v = (1 + torch.rand(dim, generator=g, device="cuda").half()).repeat(KEYS, 1, 1)
    v[HEAVY] = 0.0
    total = (KEYS - 4) * WEIGHT
    return k, v, -math.log(WEIGHT), v[1, 0].double() * total / (4 + total)


def close(out, want):
    """A weight's rounding and the result's, 2^-11 each.  fp32: the score 12 is off by 2^-21.  The products of a row are added in
    order, 16 keys at a time, 6251 times, and the tensor core cuts the sum off, by 2^-23 of it at most; the weights' sum, by
    threads that add up 64 keys or more of each tile, is rounded 2 * 1563 + 64 times by 2^-24."""
    bound = 2.0 ** -10 + 2.0 ** -20 + 6251 * 2.0 ** -23 + 3190 * 2.0 ** -24
    assert bool(((out.double() - want).abs() <= bound * want).all()), float((out.double() / want - 1).abs().max())


@pytest.mark.parametrize("dim", [64, 128])
def test_many_small_weights_packed(lib, dim):
    S, ctx = lib
    k, v, scale, want = few_and_many(dim)
    q = torch.zeros(130, 1, dim, dtype=torch.float16, device="cuda")
    q[:, :, 0] = 1.0
    out, i32 = torch.empty_like(q), lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    S.sama_attention(ctx, S.Attn(S.SAMA_F16, 1, 1, dim, 130, len(k), i32(0, 130), i32(0, len(k)), scale=scale), q, k, v, out)
    close(out, want)


@pytest.mark.parametrize("dim", [64, 128])
def test_many_small_weights_cached(lib, dim):
    S, ctx = lib
    k, v, scale, want = few_and_many(dim)
    page = 11
    pages = len(k) // page                                            # (100,001 = 11 * 9091)
    seqs = 300                                                        # (so many that a CTA has a whole one)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").repeat(seqs, 1)
    q = torch.zeros(seqs, 1, dim, dtype=torch.float16, device="cuda")
    q[..., 0] = 1.0
    out, length = torch.empty_like(q), torch.full((seqs,), len(k), dtype=torch.int32, device="cuda")
    p = S.Paged(S.SAMA_F16, 1, 1, dim, page, pages, table, length, scale=scale)
    S.sama_paged_attention(ctx, p, q, None, None, k.view(pages, page, 1, dim), v.view(pages, page, 1, dim), out)
    close(out, want)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("texts", [1, 40])
def test_scores_without_places_behind_the_point(lib, dtype, dim, texts):
    """Scores of up to 10^9, far enough apart that a row's largest has all of the weight, rising along the keys: out is its value
    and lse, as far as 24 bits go, its score."""
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(dim)
    dt, n, m = ref.DT[dtype], 260, 400
    q, k = torch.zeros(texts * n, 1, dim, dtype=dt, device="cuda"), torch.zeros(texts * m, 1, dim, dtype=dt, device="cuda")
    q[:, 0, 0] = torch.exp(torch.rand(texts * n, generator=g, device="cuda") * 14 - 6).to(dt)
    k[:, 0, 0] = (100 + torch.arange(texts * m, device="cuda") % m).to(dt)       # (bf16: 100 .. 500 in steps of 1 to 4, some alike)
    v = torch.randn(texts * m, 1, dim, generator=g, device="cuda").to(dt)
    for t in range(texts):                                                      # the last keys of a text are alike: one value
        v[t * m:t * m + m] = v[t * m + m - 1]
    v[:, 0, 1] = (k[:, 0, 0] == k[-1, 0, 0]).to(dt)                             # 1 for the largest score, else 0
    i32 = lambda step: torch.arange(0, texts + 1, device="cuda", dtype=torch.int32) * step  # noqa: E731
    out, lse = torch.empty_like(q), torch.empty(1, texts * n, device="cuda")
    for scale in (1000.0, 500.123):
        S.sama_attention(ctx, S.Attn(S.DTYPES[dtype], 1, 1, dim, texts * n, texts * m, i32(n), i32(m), scale=scale), q, k, v, out, lse)
        x = scale * q[:, 0, 0].double() * float(k[-1, 0, 0])
        sure = scale * q[:, 0, 0].double() > 100                                # (the next key's score is that much less)
        assert int(sure.sum()) > 100 * texts and float(x.max()) > 5e8
        # (the weight is rounded, as it refers to a maximum that may be up to 2^8 less, and so is the result)
        off = (out[sure, 0, 1].double() - 1).abs()
        assert bool((off <= 2 * ref.U[dtype]).all()) and bool(torch.isfinite(out).all()), (float(off.max()), int((off > 0.5).sum()))
        alike = int((k[:m, 0, 0] == k[-1, 0, 0]).sum())
        assert bool(((lse[0, sure].double() - x[sure] - math.log(alike)).abs() <= 2.0 ** -21 * (x[sure] + 4)).all())
