"""Attention over a paged cache at the ends of what it takes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def test_the_longest_sequences(lib):
    """Every entry of the table names one page, which stands for 2^31 keys.  Keys of zeros: all weights are 1, and with values of
    0 to 2 sums are whole numbers that fp32 holds, a CTA's at least (2^31 / 296 of 2 at most); joining them rounds by 2^-24 each."""
    S, ctx = lib
    page, dim = 1 << 20, 8
    g = torch.Generator(device="cuda").manual_seed(0)
    k = torch.zeros(1, page, 1, dim, dtype=torch.bfloat16, device="cuda")
    v = torch.randint(0, 3, (1, page, 1, dim), generator=g, device="cuda").bfloat16()
    table = torch.zeros(1, 2049, dtype=torch.int32, device="cuda")
    q, length = torch.ones(1, 1, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    p = S.Paged(S.SAMA_BF16, 1, 1, dim, page, 1, table, length)
    want = v.double().mean(1)[0]
    for n, status in ((2 ** 31 - 64, 0), (2 ** 31 - 63, S.SAMA_DEV_BAD_INDEX), (2 ** 31 - 1, S.SAMA_DEV_BAD_INDEX)):
        length.fill_(n)
        out.fill_(7.0)
        S.sama_paged_attention(ctx, p, q, None, None, k, v, out)
        assert S.sama_device_status(ctx) == status, n
        # 64 keys of 2^31 less than the mean is over; 296 parts; the result's own rounding
        assert bool(((out[0].double() - want).abs() <= (2.0 ** -8 + 296 * 2.0 ** -23 + 2.0 ** -20) * want).all()), n
