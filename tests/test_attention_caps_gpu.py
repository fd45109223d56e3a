"""Caps far above the scores: cap tanh(x / cap) is x to within rounding, and has to be that for the kernels, too.

Bound: attention_reference's without a cap, in which the exponent of a weight is off by e = 2^-23 (dim + 8) |scale| sum |q k| + ..,
and beside it what tanh is off by, 7e-7 < 2^-20 of the score.  Since |x| <= |scale| sum |q k|, that is less than 8 / (dim + 8) of e, and
every bound grows by no more than its e does."""
import pytest
import torch

import attention_reference as ref
from test_attention_gpu import Case as Packed
from test_attention_gpu import MANY
from test_paged_attention_gpu import Case as Cached

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def within(name, got, want, bound, dim):
    over = (got.double() - want).abs() - bound * (1 + 8 / (dim + 8))
    assert bool((over <= 0).all()), (name, float(over.max()))


@pytest.mark.parametrize("cap", [1e4, 1e5, 1e6, 1e9])
@pytest.mark.parametrize("dim,among", [(64, 1), (64, MANY), (128, 1), (128, MANY)])
@pytest.mark.parametrize("causal", [False, True])
def test_packed(lib, cap, dim, among, causal):
    c = Packed(lib, [300, 9, 130], heads=4, kv=2, dim=dim, dtype="f16", causal=causal, cap=cap, edge=5 if among == 1 else 3 * MANY, seed=1)
    c.run()
    for lo, hi in zip(c.qs, c.qs[1:]):
        at = slice(lo, hi)
        args = (c.q[at], c.k[at], c.v[at], c.dout[at], "f16", c.scale)
        want, _ = ref.text(*args, cap, None, causal, 0)
        _, bound = ref.text(*args, 0.0, None, causal, 0)
        for name, x in (("out", c.out), ("lse", c.lse.T), ("dq", c.grads[0]), ("dk", c.grads[1]), ("dv", c.grads[2])):
            w, b = (r[name].T if name == "lse" else r[name] for r in (want, bound))
            within(name, x[at], w, b, dim)


@pytest.mark.parametrize("cap", [1e4, 1e5, 1e6, 1e9])
@pytest.mark.parametrize("dim", [64, 128])
def test_cached(lib, cap, dim):
    c = Cached(lib, [333, 5, 90], heads=8, kv=2, dim=dim, dtype="f16", cap=cap, seed=1)
    c.run()
    for s, (_, (k, v)) in enumerate(c.rows):
        want, _ = ref.text(c.q[s:s + 1], k, v, None, "f16", dim ** -0.5, cap, None, False, 0)
        _, bound = ref.text(c.q[s:s + 1], k, v, None, "f16", dim ** -0.5, 0.0, None, False, 0)
        within(s, c.out[s:s + 1], want["out"], bound["out"], dim)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", [0.0, 1e-4, 2.0])
@pytest.mark.parametrize("scale,cap", [(1.0, 2.0 ** -13), (2.0 ** -60, 2.0 ** -60), (2.0 ** -60, 2.0 ** 60), (0.125, 2.0 ** 60)])
def test_the_ends_of_the_range(lib, scale, cap, size, dim):
    """Queries of zeros among them, whose scores are all exactly 0."""
    for bias in (False, True):
        c = Packed(lib, [300, 9], heads=2, kv=1, dim=dim, dtype="bf16", causal=True, cap=cap, scale=scale, size=size, bias=bias, seed=2)
        c.run()
        for lo, hi in zip(c.qs, c.qs[1:]):
            at = slice(lo, hi)
            # (a large cap as none: the bounds have nothing for it)
            want, bound = ref.text(c.q[at], c.k[at], c.v[at], c.dout[at], "bf16", c.scale, 0.0 if cap > 1 else cap, c.slopes, True, 0)
            for name, x in (("out", c.out), ("lse", c.lse.T), ("dq", c.grads[0]), ("dk", c.grads[1]), ("dv", c.grads[2])):
                w, b = (r[name].T if name == "lse" else r[name] for r in (want, bound))
                within(name, x[at], w, b, dim)
    p = Cached(lib, [40, 3], heads=2, kv=1, dim=dim, cap=max(cap, dim ** -0.5 * 2.0 ** -13), seed=3)   # (its scale is dim ** -0.5)
    p.q *= size
    p.run()
    p.check()
