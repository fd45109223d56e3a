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


@pytest.mark.parametrize("dim,dtype", [(64, "bf16"), (128, "f16")])
def test_sequences_that_share_pages(lib, dim, dtype):
    """A prompt's pages in several sequences, each with a last page of its own for its new token; and several tokens of one sequence
    at once, which are in the cache already."""
    import attention_reference as ref
    S, ctx = lib
    heads, kv, page, shared, n = 4, 2, 16, 9, 5
    g = torch.Generator(device="cuda").manual_seed(dim)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(ref.DT[dtype])  # noqa: E731
    k, v = r(shared + n, page, kv, dim), r(shared + n, page, kv, dim)
    table = torch.empty(n, shared + 1, dtype=torch.int32, device="cuda")
    table[:, :shared] = torch.arange(shared, device="cuda")
    table[:, shared] = shared + torch.arange(n, device="cuda")
    lengths = torch.tensor([shared * page + 1 + 3 * s for s in range(n)], dtype=torch.int32, device="cuda")
    q, k_new, v_new = r(n, heads, dim), r(n, kv, dim), r(n, kv, dim)
    out = torch.empty_like(q)

    def check(lengths, table):
        for s, length in enumerate(lengths.tolist()):
            K, V = (x[table[s].long()].flatten(0, 1)[:length] for x in (k, v))
            want, bound = ref.text(q[s:s + 1], K, V, None, dtype, dim ** -0.5, 0.0, None, False, 0)
            assert bool(((out[s:s + 1].double() - want["out"]).abs() <= bound["out"]).all()), s

    S.sama_paged_attention(ctx, S.Paged(S.DTYPES[dtype], heads, kv, dim, page, shared + n, table, lengths), q, k_new, v_new, k, v, out)
    torch.cuda.synchronize()
    check(lengths, table)
    at = lengths.long() - 1
    rows = (table[torch.arange(n, device="cuda"), at // page].long(), at % page)
    assert torch.equal(k[rows], k_new) and torch.equal(v[rows], v_new)
    # five tokens of the first sequence
    one, five = table[:1].repeat(n, 1), (shared * page + 2 + torch.arange(n, device="cuda")).to(torch.int32)
    S.sama_paged_attention(ctx, S.Paged(S.DTYPES[dtype], heads, kv, dim, page, shared + n, one, five), q, None, None, k, v, out)
    torch.cuda.synchronize()
    check(five, one)
    assert S.sama_device_status(ctx) == 0
