"""Token embedding and its gradient against a plain implementation in 64 bits.

Tolerances.  The forward is one fp32 product (relative error 2^-24 at most) and one rounding to the type, whose unit
roundoff for p significant bits is u = 2^-p: 2^-24 (fp32), 2^-8 (bf16) or 2^-11 (fp16).  The gradient adds k terms in
fp32, in any grouping: the error is at most k 2^-24 times the sum of the terms' magnitudes, then come the product and
the rounding.  fp16 adds half of its smallest subnormal step, 2^-25.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def place(x, shift):
    """A contiguous copy whose first element lies ``shift`` elements past a 16-byte boundary."""
    if shift == 0:
        return x.clone()
    buf = torch.empty(x.numel() + 16, dtype=x.dtype, device="cuda")
    v = buf[shift:shift + x.numel()].view(x.shape)
    return v.copy_(x)


def make_ids(kind, n, vocab, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        return torch.full((n,), vocab // 2, dtype=torch.int32)
    if kind == "spread":
        return (torch.arange(n) * 7919 % vocab).to(torch.int32)
    u = torch.rand(n, generator=g, dtype=torch.float64)
    return (torch.exp(u * np.log(vocab + 1.0)) - 1).clamp(0, vocab - 1).to(torch.int32)


def plain_grad(ids, dout, vocab, scale, skip, base=None):
    """(gradient, sum of the terms' magnitudes, number of terms) per row, in 64 bits."""
    ids, x = ids.long().cpu(), dout.double().cpu()
    keep = (ids >= 0) & (ids < vocab) & (ids != skip)
    g = torch.zeros(vocab, x.shape[1], dtype=torch.float64)
    m, k = torch.zeros_like(g), torch.zeros(vocab, 1, dtype=torch.float64)
    g.index_add_(0, ids[keep], x[keep])
    m.index_add_(0, ids[keep], x[keep].abs())
    k.index_add_(0, ids[keep], torch.ones(int(keep.sum()), 1, dtype=torch.float64))
    g, m = g * scale, m * abs(scale)
    if base is not None:
        g, m = g + base.double().cpu(), m + base.double().cpu().abs()
    return g, m, k


def check_grad(got, ref, mag, k, gt):
    got = got.double().cpu()
    bound = (k + 2) * 2.0 ** -24 * mag * 1.01 + 1.01 * U[gt] * ref.abs() + TINY[gt]
    assert bool(((got - ref).abs() <= bound).all()), float(((got - ref).abs() - bound).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,vocab,d", [(0, 5, 8), (1, 1, 1), (1, 9, 8), (33, 7, 3), (257, 1000, 40), (64, 300, 1024),
                                       (31, 50, 2100), (1000, 70001, 257)])
@pytest.mark.parametrize("shift", [0, 1])
def test_forward(lib, dtype, n, vocab, d, shift):
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(n + d)
    table = place(torch.randn(vocab, d, generator=g, device="cuda").to(DT[dtype]), shift)
    ids = make_ids("text", n, vocab, 3).cuda()
    scale = float(np.float32(np.sqrt(d)))
    out = place(torch.full((n, d), float("nan"), device="cuda").to(DT[dtype]), shift)
    S.sama_embed(ctx, S.DTYPES[dtype], n, vocab, d, table, ids, scale, out)
    ref = table.double()[ids.long()] * scale
    assert bool(((out.double() - ref).abs() <= 1.01 * U[dtype] * ref.abs() + TINY[dtype]).all())
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("dtype,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("kind", ["one", "spread", "text"])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 70001, 8), (2, 255, 5), (33, 256, 16), (1000, 257, 33),
                                       (5003, 300, 8), (20011, 70001, 24), (300, 40, 2100), (9001, 16777217, 2)])
def test_gradient(lib, dtype, gt, kind, n, vocab, d):
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(n + d)
    dout = torch.randn(n, d, generator=g, device="cuda").to(DT[dtype])
    ids = make_ids(kind, n, vocab, 5).cuda()
    scale = float(np.float32(-1.7))
    grad = torch.full((vocab, d), float("nan"), device="cuda").to(DT[gt])
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, scale, -1, S.DTYPES[gt], 0, grad)
    if vocab > 100000:   # only the rows that have tokens, and a count of the others
        used = torch.unique(ids.long())
        assert int((grad != 0).any(1).sum()) <= used.numel() and not bool(torch.isnan(grad).any())
        remap = torch.searchsorted(used, ids.long()).to(torch.int32)
        ref, mag, k = plain_grad(remap, dout, used.numel(), scale, -1)
        check_grad(grad[used], ref, mag, k, gt)
    else:
        check_grad(grad, *plain_grad(ids, dout, vocab, scale, -1), gt)
    again = torch.empty_like(grad)
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, scale, -1, S.DTYPES[gt], 0, again)
    assert torch.equal(grad, again)
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("dtype,gt,shift", [("f32", "f32", 0), ("bf16", "f32", 1), ("f16", "f16", 3)])
def test_accumulates_into_the_rows_that_have_tokens(lib, dtype, gt, shift):
    S, ctx = lib
    n, vocab, d = 3000, 777, 72
    dout = place(torch.randn(n, d, device="cuda").to(DT[dtype]), shift)
    ids = make_ids("text", n, vocab, 8).cuda()
    base = torch.randn(vocab, d, device="cuda").to(DT[gt])
    grad = place(base, shift)
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, 0.5, 3, S.DTYPES[gt], 1, grad)
    ref, mag, k = plain_grad(ids, dout, vocab, 0.5, 3, base)
    check_grad(grad, ref, mag, k, gt)
    untouched = torch.ones(vocab, dtype=torch.bool, device="cuda")
    untouched[ids.long()] = False
    untouched[3] = True
    assert int(untouched.sum()) > 1 and torch.equal(grad[untouched], base[untouched])


def test_ids_outside_the_vocabulary_and_the_skipped_id(lib):
    S, ctx = lib
    n, vocab, d = 500, 60, 16
    ids = make_ids("text", n, vocab, 2)
    ids[::7], ids[3::50], ids[5] = 4, -1, vocab
    ids[9], ids[10] = 2 ** 31 - 1, -2 ** 31
    ids = ids.cuda()
    table = torch.randn(vocab, d, device="cuda")
    out = torch.full((n, d), float("nan"), device="cuda")
    S.sama_embed(ctx, S.SAMA_F32, n, vocab, d, table, ids, 2.0, out)
    good = (ids >= 0) & (ids < vocab)
    assert torch.equal(out[good], table[ids[good].long()] * 2.0) and not bool(out[~good].any())
    assert S.sama_device_status(ctx) == S.SAMA_DEV_BAD_INDEX
    dout = torch.randn(n, d, device="cuda")
    dout[~good] = float("nan")            # what belongs to no row reaches none
    dout[ids == 4] = float("inf")
    grad = torch.empty(vocab, d, device="cuda")
    S.sama_embed_grad(ctx, S.SAMA_F32, n, vocab, d, ids, dout, 1.0, 4, S.SAMA_F32, 0, grad)
    assert S.sama_device_status(ctx) == S.SAMA_DEV_BAD_INDEX
    check_grad(grad, *plain_grad(ids, dout.nan_to_num(0.0, 0.0, 0.0), vocab, 1.0, 4), "f32")
    assert not bool(grad[4].any())
    # every token left out: a gradient of zeros
    S.sama_embed_grad(ctx, S.SAMA_F32, n, vocab, d, torch.full_like(ids, 4), dout, 1.0, 4, S.SAMA_F32, 0, grad.fill_(7))
    assert not bool(grad.any())
    S.sama_embed_grad(ctx, S.SAMA_F32, 0, vocab, d, None, None, 1.0, -1, S.SAMA_F32, 0, grad.fill_(7))
    assert not bool(grad.any())


def test_gradient_is_the_derivative(lib):
    """Differences of the forward in fp32: L = <dOut, out(E)> is linear in E, so a step of 1 has no truncation error."""
    S, ctx = lib
    n, vocab, d = 40, 9, 3
    ids = make_ids("text", n, vocab, 4).cuda()
    dout = torch.randint(-8, 9, (n, d), device="cuda").float()
    table = torch.randint(-8, 9, (vocab, d), device="cuda").float()
    grad, out = torch.empty_like(table), torch.empty_like(dout)

    def loss(e):
        S.sama_embed(ctx, S.SAMA_F32, n, vocab, d, e, ids, 0.5, out)
        return float((out.double() * dout.double()).sum())

    S.sama_embed_grad(ctx, S.SAMA_F32, n, vocab, d, ids, dout, 0.5, -1, S.SAMA_F32, 0, grad)
    for v in range(vocab):
        for c in range(d):
            e = table.clone()
            e[v, c] += 1
            assert loss(e) - loss(table) == float(grad[v, c])   # all values are exact in fp32


def test_offsets_beyond_32_bits(lib):
    S, ctx = lib
    n, vocab, d = 300, 2_200_000, 1024                           # 2.25e9 elements
    table = torch.zeros(vocab, d, dtype=torch.bfloat16, device="cuda")
    ids = (vocab - 1 - torch.arange(n, device="cuda") * 7333 % vocab).to(torch.int32)
    rows = torch.randn(n, d, device="cuda").bfloat16()
    table[ids.long()] = rows
    out = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    S.sama_embed(ctx, S.SAMA_BF16, n, vocab, d, table, ids, 1.0, out)
    assert torch.equal(out, rows)
    table.fill_(1.0)
    S.sama_embed_grad(ctx, S.SAMA_BF16, n, vocab, d, ids, rows, 1.0, -1, S.SAMA_BF16, 0, table)
    assert torch.equal(table[ids.long()], rows)
    table[ids.long()] = 0
    assert not bool(table.any())


def test_runs_on_the_callers_stream(lib):
    S, ctx = lib
    n, vocab, d = 4000, 500, 256
    s = torch.cuda.Stream()
    ids = make_ids("text", n, vocab, 1).cuda()
    dout, grad = torch.zeros(n, d, device="cuda"), torch.empty(vocab, d, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(20):
            dout.add_(0.25)      # the call must wait for this, and what follows for the call
        S.sama_embed_grad(ctx, S.SAMA_F32, n, vocab, d, ids, dout, 1.0, -1, S.SAMA_F32, 0, grad)
        copy = grad.clone()
    s.synchronize()
    count = torch.bincount(ids.long(), minlength=vocab).float()
    assert torch.equal(copy, (5.0 * count)[:, None].expand(-1, d))


def test_refusals(lib):
    S, ctx = lib
    t, i = torch.zeros(64, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    o = torch.zeros(64, device="cuda")
    a = t.data_ptr()

    def status(f, *args):
        with pytest.raises(S.SamaError) as e:
            f(*args)
        return e.value.status

    fw, bw = S.sama_embed, S.sama_embed_grad
    assert status(fw, None, 0, 4, 4, 4, a, i, 1.0, o) == S.SAMA_ERR_NULL
    assert status(fw, ctx, 0, 4, 4, 4, None, i, 1.0, o) == S.SAMA_ERR_NULL
    assert status(fw, ctx, 0, 4, 4, 4, t, None, 1.0, o) == S.SAMA_ERR_NULL
    assert status(fw, ctx, 3, 4, 4, 4, a, i, 1.0, o.data_ptr()) == S.SAMA_ERR_PARAM
    assert status(fw, ctx, 0, 4, 4, 4, t, i, float("nan"), o) == S.SAMA_ERR_PARAM
    assert status(fw, ctx, 0, -1, 4, 4, t, i, 1.0, o) == S.SAMA_ERR_SIZE
    assert status(fw, ctx, 0, 4, 0, 4, t, i, 1.0, o) == S.SAMA_ERR_SIZE
    assert status(fw, ctx, 0, 4, 4, 0, t, i, 1.0, o) == S.SAMA_ERR_SIZE
    assert status(fw, ctx, 0, 4, 4, 4, a + 2, i, 1.0, o) == S.SAMA_ERR_ALIGN
    assert status(fw, ctx, 0, 4, 4, 4, t, i, 1.0, a + 16) == S.SAMA_ERR_OVERLAP
    assert status(fw, ctx, 0, 40, 4, 4, t, i, 1.0, o) == S.SAMA_ERR_SIZE          # out is too small
    assert status(fw, ctx, 0, 4, 4, 4, t, i.long(), 1.0, o) == S.SAMA_ERR_PARAM     # ids of another type
    assert status(fw, ctx, 0, 2, 4, 4, t.view(8, 8)[:, :4], i, 1.0, o) == S.SAMA_ERR_PARAM  # not contiguous
    assert status(bw, ctx, 0, 4, 4, 4, i, None, 1.0, -1, 0, 0, o) == S.SAMA_ERR_NULL
    assert status(bw, ctx, 0, 4, 4, 4, i, t, 1.0, -1, 0, 0, None) == S.SAMA_ERR_NULL
    assert status(bw, ctx, 0, 4, 4, 4, i, a, 1.0, -1, 1, 0, o.data_ptr()) == S.SAMA_ERR_PARAM  # fp32 in, 16 bits out
    assert status(bw, ctx, 0, 4, 4, 4, i, t, 1.0, -1, 0, 2, o) == S.SAMA_ERR_PARAM
    assert status(bw, ctx, 0, 4, 4, 4, i, t, 1.0, -1, 0, 0, t) == S.SAMA_ERR_OVERLAP
    assert status(bw, ctx, 0, 4, 2 ** 31 - 1, 4, i, t, 1.0, -1, 0, 0, o) == S.SAMA_ERR_SIZE
    assert S.sama_device_status(ctx) == 0
