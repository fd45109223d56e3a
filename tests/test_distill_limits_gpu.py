"""Distillation at the ends of what it takes: the coldest and the hottest softmax."""
import math

import pytest
import torch

from test_distill_gpu import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


@pytest.mark.parametrize("vocab", [300, 9000, 70000, 300000])
def test_the_coldest_and_the_hottest(lib, vocab):
    for T, scale in ((2.0 ** -60, 2.0 ** 60), (2.0 ** 60, 2.0 ** -60)):
        c = Case(lib, 5, vocab, 8, "f32", T=T, weighted=False, grad_scale=scale, seed=23)
        c.run()
        if T < 1:       # all of the weight on the largest
            q = torch.zeros_like(c.z).scatter_(1, c.z.argmax(1, keepdim=True), 1.0)
            p = torch.zeros_like(c.z).scatter_(1, c.ids.long().gather(1, c.top.argmax(1, keepdim=True)), 1.0)
        else:           # uniform
            q = torch.full_like(c.z, 1 / vocab)
            p = torch.zeros_like(c.z).scatter_(1, c.ids.long(), 1 / 8)
        assert bool(((c.grad - (q - p)).abs() <= 1e-5 * (q + p)).all())
        # cold: T (largest z - z of the teacher's largest); hot: T^2 log(vocab / 8)
        want = T * (c.z.amax(1) - c.z.gather(1, c.ids.long().gather(1, c.top.argmax(1, keepdim=True)))[:, 0]) if T < 1 else \
            torch.full_like(c.loss, T * T * math.log(vocab / 8))
        assert bool(((c.loss - want).abs() <= 1e-5 * want.abs() + 2.0 ** -100).all())
