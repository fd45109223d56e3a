"""The gated feed-forward block in fp16 at the ends of the type's range: what overflows is infinite and stays in its rows, and
small gradients lose no more than the type's subnormal step."""
import pytest
import torch

import test_gated_ffn_gpu as block
from test_gated_ffn_gpu import backward, check_backward, forward, lib, make  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [5, 200])
def test_hidden_values_beyond_the_range_are_infinite(lib, M):  # noqa: F811
    t = make(M, 64, 96, "f16", 3)
    t["x"].clamp_(-3.0, 3.0)
    clean, g, u = forward(lib, t, "relu", save=True)
    assert bool(torch.isfinite(clean).all())
    # row 1: G and U of some hundreds, finite in fp16, and products H beyond 65504
    t["x"][1] = torch.where(torch.arange(64, device="cuda") % 2 == 0, 200.0, -200.0)
    y, gate, up = forward(lib, t, "relu", save=True)
    h = gate.double().clamp(min=0) * up.double()
    assert bool(torch.isfinite(gate).all() and torch.isfinite(up).all()) and float(h[1].abs().max()) > 1.01 * 65504
    assert float(h[[0, *range(2, M)]].abs().max()) < 1e3
    # every output of the row has an infinite term (the weights are not zero); the other rows are as before
    assert bool((t["wd"] != 0).all()) and not bool(torch.isfinite(y[1]).any())
    keep = [0, *range(2, M)]
    assert torch.equal(y[keep], clean[keep]) and torch.equal(gate[keep], g[keep]) and torch.equal(up[keep], u[keep])


@pytest.mark.parametrize("M,d,f", [(3, 64, 96), (200, 192, 328), (40, 65, 130)])
@pytest.mark.parametrize("scale", [2.0 ** -10, 2.0 ** -16])
def test_small_gradients(lib, monkeypatch, M, d, f, scale):  # noqa: F811
    """dG and dU partly (2^-10) or all (2^-16) below 2^-14; the bounds count half a subnormal step per rounding."""
    def small(*a, **kw):
        t = make(*a, **kw)
        t["dy"].mul_(scale)
        return t

    monkeypatch.setattr(block, "make", small)
    check_backward(lib, M, d, f, "f16", "silu")
    t = small(M, d, f, "f16", M + f)
    assert any(bool(v.any()) for v in backward(lib, t, "silu"))
