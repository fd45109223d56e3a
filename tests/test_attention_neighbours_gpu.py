"""Packed texts share tiles.  The results of a text are the same bits whatever finite values its neighbours have: values that
raise a running maximum, or leave the range of small scores, in one text and not in the other."""
import pytest
import torch

from test_attention_gpu import Case, MANY

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def same_bits(lib, lens, among=1, **kw):
    """Every second text a hundred times as large, or a hundredth, or as the others: the texts between come out the same."""
    results = []
    for factor in (1.0, 100.0, 0.01):
        c = Case(lib, lens, edge=MANY * len(lens) if among > 1 else 5, seed=21, **kw)
        for t in range(1, len(lens), 2):
            rows = slice(c.qs[t], c.qs[t + 1])
            for x in (c.q, c.k, c.v, c.dout):
                x[rows] *= factor
        c.run()
        results.append([[x[slice(c.qs[t], c.qs[t + 1])].clone() for t in range(0, len(lens), 2)]
                        for x in (c.out, c.lse.T, *c.grads)])
    for name, first, *others in zip(("out", "lse", "dq", "dk", "dv"), *results):
        for t, x in enumerate(first):
            assert bool(torch.isfinite(x).all())
            for y in others:
                assert torch.equal(x, y[t]), (name, 2 * t)


@pytest.mark.parametrize("among", [1, MANY])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_neighbours_do_not_raise_a_maximum(lib, dtype, causal, bias, dim, among):
    for lens in ([300, 61, 400, 30], [70, 500, 140], [129, 1, 385, 2]):
        same_bits(lib, lens, among, dim=dim, dtype=dtype, causal=causal, bias=bias)


@pytest.mark.parametrize("among", [1, MANY])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("causal,bias", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("cap", [20.0, 3.0])
def test_neighbours_do_not_choose_how_scores_are_capped(lib, cap, causal, bias, dim, among):
    """Scores within three quarters of a cap can do with less arithmetic than others.  (At a cap of 20 those of the texts
    looked at are, and their neighbours' are not.)"""
    for lens in ([300, 61, 400, 30], [70, 500, 140], [129, 1, 385, 2]):
        same_bits(lib, lens, among, dim=dim, causal=causal, bias=bias, cap=cap)


@pytest.mark.parametrize("among", [1, MANY])
@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16"), (40, "f16")])
@pytest.mark.parametrize("cap", [0.0, 20.0, 300.0])
@pytest.mark.parametrize("causal,bias", [(True, False), (False, True)])
def test_neighbours_that_are_not_finite(lib, causal, bias, cap, dim, dtype, among):
    lens = [70, 61, 300]
    for bad in (float("nan"), float("inf"), -float("inf")):
        plain, other = (Case(lib, lens, heads=2, kv=1, dim=dim, dtype=dtype, causal=causal, bias=bias, cap=cap, seed=7,
                             edge=MANY * len(lens) if among > 1 else 5) for _ in range(2))
        for x in (other.q, other.k, other.v, other.dout):
            x[other.qs[1]:other.qs[2]] = bad
        plain.run()
        other.run()
        for x, y in zip((plain.out, plain.lse.T, *plain.grads), (other.out, other.lse.T, *other.grads)):
            for t in (0, 2):
                at = slice(plain.qs[t], plain.qs[t + 1])
                assert torch.equal(x[at], y[at]) and bool(torch.isfinite(x[at]).all())
