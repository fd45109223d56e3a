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


class Block:
    """A training step of the feed-forward block: both directions, on tensors `shift` elements past a 16-byte boundary."""

    def __init__(self, lib, M, d, f, seed=0, shift=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.S, self.ctx = lib
        self.sizes = (M, d, f)

        def r(rows, cols, scale):
            buf = torch.empty(rows * cols + 16, dtype=torch.bfloat16, device="cuda")
            return buf[shift:shift + rows * cols].view(rows, cols).copy_(scale * torch.randn(rows, cols, generator=g, device="cuda"))

        self.x, self.dy = r(M, d, 1.0), r(M, d, 1.0)
        self.w = [r(f, d, d ** -0.5), r(f, d, d ** -0.5), r(d, f, f ** -0.5)]
        self.gate, self.up = r(M, f, 1.0), r(M, f, 1.0)
        self.out = [torch.empty_like(v) for v in (self.x, self.x, *self.w)]

    def forward(self):
        self.S.sama_gated_ffn(self.ctx, self.S.SAMA_BF16, self.S.SAMA_ACT_SILU, *self.sizes, self.x, *self.w, self.out[0],
                              self.gate, self.up)

    def run(self):
        self.forward()
        self.S.sama_gated_ffn_grad(self.ctx, self.S.SAMA_BF16, self.S.SAMA_ACT_SILU, *self.sizes, self.x, *self.w, self.gate,
                                   self.up, self.dy, *self.out[1:])

    def clear(self):
        for v in self.out:
            v.fill_(float("nan"))

    def eager(self):
        self.clear()
        self.run()
        return [v.clone() for v in self.out]


@pytest.mark.parametrize("what", ["embedding", "block", "few tokens"])
def test_a_captured_call_that_would_have_to_allocate_is_refused(lib, what):
    S, ctx = lib
    call = {"embedding": lambda: Embedding(lib, 3000, 501, 64).run, "block": lambda: Block(lib, 64, 64, 96).run,
            "few tokens": lambda: Block(lib, 1, 64, 96).forward}[what]()
    x = torch.zeros(8, device="cuda")
    seen = []

    def captured():
        x.add_(1.0)
        with pytest.raises(S.SamaError) as e:
            call()
        seen.append(e.value.status)
        x.add_(1.0)

    graph = capture(captured)
    assert seen == [S.SAMA_ERR_NOMEM] and S.sama_launch_count(ctx) == 0
    graph.replay()                          # what was captured around it stands
    assert bool((x == 2.0).all())
    call()                                  # set up now: the same call can be captured
    capture(call).replay()
    torch.cuda.synchronize()
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("M,d,f,shift", [(1, 256, 344, 0), (16, 200, 333, 0), (64, 512, 1024, 0), (700, 256, 688, 0),
                                         (300, 129, 257, 0), (96, 128, 256, 3), (2305, 512, 1920, 0)])
def test_the_feed_forward_block_is_captured(lib, M, d, f, shift):
    b = Block(lib, M, d, f, 7, shift)
    want = b.eager()
    graph = capture(b.run)
    for _ in range(3):
        b.clear()
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(b.out, want))
    b.x.copy_(b.x.flip(0))                  # new inputs in the same place
    graph.replay()
    got = [v.clone() for v in b.out]
    assert all(torch.equal(p, q) for p, q in zip(got, b.eager()))
    assert b.S.sama_device_status(b.ctx) == 0


def test_a_captured_block_outlives_smaller_calls(lib):
    large, small = Block(lib, 700, 256, 688, 8), Block(lib, 40, 256, 344, 9)
    want = large.eager()
    graph = capture(large.run)
    small.run()
    large.clear()
    graph.replay()
    assert all(torch.equal(p, q) for p, q in zip(large.out, want))


def test_clipping_is_captured(lib):
    S, ctx = lib
    for sizes in ([600, 24, 400], [3_000_000, 17, 100_001]):
        ins = [torch.randn(n, device="cuda") for n in sizes]
        flat, norm = torch.empty(sum(sizes), device="cuda"), torch.empty(1, device="cuda")
        tensors = S.TensorList(ins, list(flat.split(sizes)))
        graph = capture(lambda: S.sama_clip_grads(ctx, tensors, 1.0, norm))
        for k in range(2):
            ins[0].mul_(3.0)
            graph.replay()
            got = [flat.clone(), norm.clone()]
            S.sama_clip_grads(ctx, tensors, 1.0, norm)
            assert torch.equal(got[0], flat) and torch.equal(got[1], norm)
    assert S.sama_device_status(ctx) == 0
