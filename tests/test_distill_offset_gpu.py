"""Distillation of logits that lie far from zero, as a head with a bias or without any bound gives them: softmax does not depend on
where they lie, and neither may its errors.

Bounds: test_distill_gpu.py's, with |z - max z| in the place of |z| + |max z|: each exponential is off by a factor of at most 1 + E,
E = 2^-21 (max |z - max z| / T + 1)."""
import math

import pytest
import torch

from test_distill_gpu import Case, TINY, U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


@pytest.mark.parametrize("offset", [0.0, 100.0, -100.0, 690.0, -690.0, 1000.0])
@pytest.mark.parametrize("vocab", [300, 9000, 20001, 40003, 70000, 140001])
@pytest.mark.parametrize("T", [0.7, 1.0, 2.0])
def test_logits_far_from_zero(lib, offset, vocab, T):
    c = Case(lib, 6, vocab, 9, "f32", T=T, seed=21)
    c.z += offset * T
    if offset:
        c.z[:, ::2] -= 1.0        # (threads have other maxima than one another)
    c.run()
    z = c.z.double() / T
    away = (z.amax(1, keepdim=True) - z).amax(1, keepdim=True)
    u = c.top.double() / T
    p, logq = torch.softmax(u, 1), torch.log_softmax(z, 1)
    vec = max(64, vocab / 1024)
    e = 2.0 ** -21 * (away + 1) + (vec + 16) * 2.0 ** -24
    eu = 2.0 ** -21 * ((u.amax(1, keepdim=True) - u).amax(1, keepdim=True) + 1) + 20 * 2.0 ** -24
    lq, lp = logq.gather(1, c.ids.long()), torch.log(p)
    term = p * (lp - lq)
    loss = T * T * term.sum(1)
    eterm = p * (2 * eu * (lp - lq).abs() + 2 * eu + 2 * e + 2.0 ** -22 * (lp.abs() + lq.abs() + away + 1))
    bound = T * T * (eterm.sum(1) + 2.0 ** -23 * 32 * term.abs().sum(1))
    over = (c.loss.double() - loss).abs() - bound
    assert bool((over <= 0).all()), float(over.max())
    f = (c.scale * T * c.weight.double())[:, None]
    q, dense = torch.exp(logq), torch.zeros_like(z).scatter_add_(1, c.ids.long(), p)
    grad = f * (q - dense)
    eg = f.abs() * (2 * e * q + 2 * eu * dense + 2.0 ** -22 * (q + dense))
    over = (c.grad.double() - grad).abs() - (U["f32"] * (grad.abs() + eg) + eg + TINY["f32"])
    assert bool((over <= 0).all()), (float(over.max()), float(((c.grad.double() - grad).abs() / (eg + 1e-300)).max()))
    assert c.S.sama_device_status(c.ctx) == 0 and math.isfinite(float(c.loss.sum()))


@pytest.mark.parametrize("offset", [0.0, 123.4, -345.6, 567.8, 691.3, -701.9])
@pytest.mark.parametrize("vocab", [9000, 20001, 40003, 70000])
def test_shares_add_up(lib, offset, vocab):
    """The gradient's entries and the teacher's add up to the sum of q, which is 1: the exponentials are those that were summed, so
    only the sum's own roundings are left, of m + 16 terms with m of a thread, and 2^-24 of each entry's, 2^-21 with the scales'."""
    c = Case(lib, 20, vocab, 9, "f32", T=1.0, weighted=False, seed=22)
    c.z += offset
    c.z[:, ::2] -= 1.0
    c.run()
    off = c.grad.double().sum(1)                    # sum q - sum p
    bound = (max(64, vocab / 1024) + 16) * 2.0 ** -24 + 2.0 ** -21
    assert float(off.abs().max()) <= bound, float(off.abs().max()) / bound
