"""Starts out of order or range, where a call has no queries: they are reported as anywhere, and nothing is written outside."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [[0, 50], [-1, 10], [7, 3]])
@pytest.mark.parametrize("dim", [64, 128])
def test_without_queries(bad, dim):
    from paper_2310_05674_b200 import binding as S
    ctx = S.sama_create(0, 1024, 0, None)
    k, v = (torch.randn(10, 2, dim, device="cuda").bfloat16() for _ in range(2))
    q, lse = torch.empty(0, 2, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(2, 0, device="cuda")
    buf = torch.full((2, 30, 2, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    dk, dv = buf[0, 10:20], buf[1, 10:20]
    starts, keys = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    a = S.Attn(S.SAMA_BF16, 2, 2, dim, 0, 10, starts, keys)

    def grad():
        S.sama_attention_grad(ctx, a, q, k, v, q, lse, q, q, dk, dv)
        return S.sama_device_status(ctx)

    assert grad() == 0
    assert bool((dk == 0).all()) and bool((dv == 0).all())
    keys.copy_(torch.tensor(bad, dtype=torch.int32))
    assert grad() == S.SAMA_DEV_BAD_INDEX
    assert bool((buf[:, :10] == 7).all()) and bool((buf[:, 20:] == 7).all())
    S.sama_destroy(ctx)
