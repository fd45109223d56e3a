"""The text-model operators one behind the other, each launch starting while the one before it may still be running, and
two contexts on two streams at once.  Every result is compared bit for bit with that of the same call made alone, between
two synchronisations: sums have a fixed order, so that anything else is a value read too early or too late."""
import pytest
import torch

pytestmark = pytest.mark.gpu

VOCAB, D, F = 997, 256, 344


class Chain:
    """A small model on a context of its own, its inputs for `steps` steps, and one buffer for every intermediate."""

    def __init__(self, S, n, steps, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.S, self.n = S, n
        self.ctx = S.sama_create(0, 1024, 0, None)
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.table = torch.randn(VOCAB, D, generator=g, device="cuda").bfloat16()
        self.w = [(s * torch.randn(*shape, generator=g, device="cuda")).bfloat16()
                  for s, shape in ((D ** -0.5, (F, D)), (D ** -0.5, (F, D)), (F ** -0.5, (D, F)))]
        self.ids = torch.randint(VOCAB, (steps, n), generator=g, device="cuda").to(torch.int32)
        self.dy = torch.randn(steps, n, D, generator=g, device="cuda").bfloat16()
        self.x, self.dx, self.gate, self.up = bf(n, D), bf(n, D), bf(n, F), bf(n, F)
        self.dw, self.dtable = [bf(*w.shape) for w in self.w], bf(VOCAB, D)
        grads = [self.dtable, *self.dw]
        self.sizes = [t.numel() for t in grads]
        self.y = bf(steps, n, D)
        self.flat = torch.empty(steps, sum(self.sizes), device="cuda")
        self.lists = [S.TensorList(grads, list(row.split(self.sizes))) for row in self.flat]

    def forward(self, k):
        S = self.S
        S.sama_embed(self.ctx, S.SAMA_BF16, self.n, VOCAB, D, self.table, self.ids[k], 1.0, self.x)
        S.sama_gated_ffn(self.ctx, S.SAMA_BF16, S.SAMA_ACT_SILU, self.n, D, F, self.x, *self.w, self.y[k], self.gate, self.up)

    def step(self, k):
        S = self.S
        self.forward(k)
        S.sama_gated_ffn_grad(self.ctx, S.SAMA_BF16, S.SAMA_ACT_SILU, self.n, D, F, self.x, *self.w, self.gate, self.up,
                              self.dy[k], self.dx, *self.dw)
        S.sama_embed_grad(self.ctx, S.SAMA_BF16, self.n, VOCAB, D, self.ids[k], self.dx, 1.0, -1, S.SAMA_BF16, 0, self.dtable)
        S.sama_clip_grads(self.ctx, self.lists[k], 1.0)

    def results(self):
        torch.cuda.synchronize()
        return self.y.clone(), self.flat.clone()

    def alone(self, what):
        """Results of every call made between two synchronisations."""
        S = self.S
        names = ["sama_embed", "sama_gated_ffn", "sama_gated_ffn_grad", "sama_embed_grad", "sama_clip_grads"]

        class Waits:
            def __getattr__(self, name):
                f = getattr(S, name)
                if name not in names:
                    return f

                def call(*a):
                    torch.cuda.synchronize()
                    f(*a)
                    torch.cuda.synchronize()
                return call
        self.S = Waits()
        self.clear()
        for k in range(len(self.ids)):
            what(k)
        self.S = S
        return self.results()

    def clear(self):
        self.y.fill_(float("nan"))
        self.flat.fill_(float("nan"))
        torch.cuda.synchronize()

    def close(self):
        torch.cuda.synchronize()
        status = self.S.sama_device_status(self.ctx)
        self.S.sama_destroy(self.ctx)
        return status


@pytest.fixture(scope="module")
def S():
    from paper_2310_05674_b200 import binding
    return binding


def same(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("n", [1, 7, 16, 45, 300, 2500])
def test_steps_behind_one_another(S, n):
    c = Chain(S, n, 24, n)
    want = c.alone(c.step)
    assert bool(torch.isfinite(want[0]).all()) and bool(torch.isfinite(want[1]).all())
    for _ in range(4):
        c.clear()
        for k in range(24):
            c.step(k)
        assert same(c.results(), want)
    assert c.close() == 0


@pytest.mark.parametrize("n", [1, 16])
def test_decode_steps_behind_one_another(S, n):
    c = Chain(S, n, 100, n)
    want = c.alone(c.forward)[0]
    for _ in range(4):
        c.clear()
        for k in range(100):
            c.forward(k)
        assert torch.equal(c.results()[0], want)
    assert c.close() == 0


@pytest.mark.parametrize("n,m", [(16, 300), (300, 300), (2500, 40)])
def test_two_contexts_on_two_streams_at_once(S, n, m):
    chains = [Chain(S, n, 16, 1), Chain(S, m, 16, 2)]
    want = [c.alone(c.step) for c in chains]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for c in chains:
            c.clear()
        for k in range(16):
            for c, s in zip(chains, streams):
                with torch.cuda.stream(s):
                    c.step(k)
        assert all(same(c.results(), w) for c, w in zip(chains, want))
    assert [c.close() for c in chains] == [0, 0]


def test_the_workspace_grows_between_calls(S):
    """Small, large, small again: the workspace of the first is not that of the last, their results are the same."""
    small, large = Chain(S, 40, 1, 3), Chain(S, 4000, 1, 4)
    want = [c.alone(c.step) for c in (small, large)]
    for c in (small, large):
        c.close()
        c.ctx = None
    ctx = S.sama_create(0, 1024, 0, None)
    for c, w in [(small, want[0]), (large, want[1]), (small, want[0])]:
        c.ctx = ctx
        c.clear()
        c.step(0)
        assert same(c.results(), w)
    assert small.close() == 0
