"""The text-model operators under stream capture, and the workspace that captured calls keep.

Results are compared bit for bit with the same calls made eagerly: a replay runs the same kernels on the same inputs, and
every sum has a fixed order.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def capture(fn):
    """A graph of fn's launches, captured on a stream of its own."""
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fn()
    return g


class Embedding:
    """One gradient call's tensors."""

    def __init__(self, lib, n, vocab=50021, d=1024, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.S, self.ctx = lib
        self.n, self.vocab, self.d = n, vocab, d
        u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
        self.ids = ((vocab + 1.0) ** u - 1).clamp(0, vocab - 1).to(torch.int32)
        self.dout = torch.randn(n, d, generator=g, device="cuda").bfloat16()
        self.grad = torch.empty(vocab, d, device="cuda")

    def run(self):
        self.S.sama_embed_grad(self.ctx, self.S.SAMA_BF16, self.n, self.vocab, self.d, self.ids, self.dout, 1.0, -1,
                               self.S.SAMA_F32, 0, self.grad)

    def eager(self):
        self.grad.fill_(float("nan"))
        self.run()
        return self.grad.clone()


def test_a_smaller_embedding_gradient_is_captured_after_a_larger_one(lib):
    Embedding(lib, 28416, seed=1).run()
    e = Embedding(lib, 14000, seed=2)      # more pieces than the 28,416 tokens had
    graph = capture(e.run)
    want = e.eager()
    for _ in range(3):                     # (from the second replay on, the sort's flag is found set)
        e.grad.fill_(float("nan"))
        graph.replay()
        assert torch.equal(e.grad, want)
    assert e.S.sama_device_status(e.ctx) == 0


def test_a_captured_embedding_gradient_outlives_smaller_calls(lib):
    large, small, few = Embedding(lib, 28416, seed=3), Embedding(lib, 14000, seed=4), Embedding(lib, 1500, seed=5)
    want = large.eager()
    graph = capture(large.run)
    for other in (small, few, small):
        other.run()
        large.grad.fill_(float("nan"))
        graph.replay()
        assert torch.equal(large.grad, want)
    large.ids.copy_(large.ids.flip(0))     # new tokens in the same place
    graph.replay()
    got = large.grad.clone()
    assert torch.equal(got, large.eager()) and not torch.equal(got, want)
