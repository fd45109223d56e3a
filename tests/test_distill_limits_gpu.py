"""Distillation at the ends of what it takes: rows on both sides of the sizes at which they are worked on in other ways, in
numbers that keep the device busy, with as many entries as there may be; the coldest and the hottest softmax."""
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


KB = 1024


# A row of up to 104 KB is a CTA's, with 512 entries beside it, longer ones a cluster's with 64 KB each, of 2 to 8 CTAs; rows that
# start between 16-byte groups need a group more.
@pytest.mark.parametrize("bytes_", [4 * KB, 16 * KB, 64 * KB, 104 * KB, 128 * KB, 192 * KB, 256 * KB, 448 * KB, 512 * KB])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_on_both_sides_of_a_limit(lib, dtype, bytes_):
    size = 4 if dtype == "f32" else 2
    for more in (-16 // size, -1, 0, 1, 16 // size):
        for shift in (0, 1):
            c = Case(lib, 90, bytes_ // size + more, 16, dtype, shift=shift, seed=bytes_ // KB + more)
            c.run()
            c.check()
    assert c.S.sama_device_status(c.ctx) == 0


@pytest.mark.parametrize("k", [511, 512, 513])
@pytest.mark.parametrize("vocab,dtype", [(53248, "bf16"), (53240, "bf16"), (26624, "f32"), (53256, "bf16"), (131072, "bf16"), (65536, "f32")])
def test_as_many_entries_as_there_may_be(lib, vocab, dtype, k):
    for n in (3, 90):
        c = Case(lib, n, vocab, k, dtype, ragged=True, seed=k)
        c.ids[0] = c.ids[0, 0]                       # one id, k times
        c.run()
        c.check()


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
