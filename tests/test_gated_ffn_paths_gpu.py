"""Every way in which the gated feed-forward block works on a launch, against the plain implementation in 64 bits.

A launch's tiles go to single CTAs, to CTA pairs in one or several rounds, whole or with the contraction of the last tiles
split through the workspace, or to clusters of 2, 4 or 8 CTAs that share a tile's contraction; which, the library chooses
by the sizes.  The sizes here were searched for so that each of the five launches is worked on in each of these ways, and
the last test holds them to that: whoever changes the choice has to search again.  Bounds and inputs are those of the
block's other tests.
"""
import pytest
import torch

from test_gated_ffn_gpu import ACTS, backward, check_backward, check_forward, forward, lib, make  # noqa: F401

pytestmark = pytest.mark.gpu

SIZES = [(17, 24, 24), (18, 960, 968), (21, 2064, 920), (21, 4136, 9992), (45, 4096, 8192), (275, 1520, 6864),
         (300, 2048, 2048), (2305, 2048, 4096), (3505, 8696, 136), (3864, 1235, 1888), (4275, 2080, 1088), (4384, 1600, 24),
         (5255, 24, 1144), (10934, 136, 72), (19098, 272, 2040), (19568, 32, 1464)]
ODD = [(21, 4135, 9993), (275, 1521, 6865), (3505, 8699, 133), (19567, 31, 1461)]


def paths(lib):
    S, ctx = lib
    return [S.sama_last_ffn_path(ctx, k) for k in range(5)]


@pytest.mark.parametrize("M,d,f", SIZES + ODD)
def test_forward(lib, M, d, f):  # noqa: F811
    check_forward(lib, M, d, f, "bf16", "silu")
    assert lib[0].sama_device_status(lib[1]) == 0


@pytest.mark.parametrize("M,d,f", SIZES + ODD)
def test_backward(lib, M, d, f):  # noqa: F811
    check_backward(lib, M, d, f, "bf16", "silu")
    assert lib[0].sama_device_status(lib[1]) == 0


# gate-up and d-hidden, whose epilogues apply the activation: on pairs in several rounds, on pairs with a split contraction
# (d-hidden of the second, both of the third), on clusters
@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,d,f", [(275, 1520, 6864), (4275, 2080, 1088), (3505, 8696, 136), (18, 960, 968)])
def test_activations(lib, M, d, f, dtype, kind):  # noqa: F811
    check_forward(lib, M, d, f, dtype, kind)
    check_backward(lib, M, d, f, dtype, kind)


def test_the_sizes_reach_every_path(lib):  # noqa: F811
    reached = [set() for _ in range(5)]
    for M, d, f in SIZES:
        t = make(M, d, f, "bf16")
        forward(lib, t, "silu")
        backward(lib, t, "silu")
        for k, (kernel, parts) in enumerate(paths(lib)):
            reached[k].add((kernel, parts > 1 if kernel == "pairs" else parts))
    torch.cuda.synchronize()
    every = {("single", 1), ("pairs", False), ("pairs", True), ("clusters", 2), ("clusters", 4), ("clusters", 8)}
    assert reached == [every] * 5, [every - r for r in reached]
    t = make(16, 40, 264, "bf16")
    forward(lib, t, "silu")
    assert paths(lib)[:2] == [("few tokens", 1)] * 2 and paths(lib)[2][0] != "few tokens"
    assert lib[0].sama_last_ffn_path(lib[1], 5) is None and lib[0].sama_last_ffn_path(None, 0) is None
