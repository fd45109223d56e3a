"""The token embedding's kernels on each side of the limits by which they are chosen, against 64 bits.

Lookup: one row per thread, and four (where the rows' threads are many), for rows of 16-byte groups, of pairs and of single
values.  Gradient: one launch (up to 2048 tokens) and two, the sort with and without its staging area (131,072 tokens),
rows of several slabs of columns, tables whose shares of the zeroing exceed what shared memory tracks (2^20 rows), large
tables with few tokens, and adding to a gradient in both forms.  Bounds are those of the embedding's other tests.
"""
import numpy as np
import pytest
import torch

from test_embed_gpu import DT, TINY, U, check_grad, lib, make_ids, place, plain_grad  # noqa: F401

pytestmark = pytest.mark.gpu


# On both sides of 404,139 tokens x threads of a row (groups: 128 and 256 threads for 1024 columns; up to 32 columns: 4 and
# 32 threads) and of 1,212,416 (chunks: 32 threads for 1030 columns in pairs, 8 for 34; 64 for 1030 and 1031 single values,
# 256 for 1024).
@pytest.mark.parametrize("dtype,n,d,shift", [
    ("bf16", 3001, 1024, 0), ("bf16", 3203, 1024, 0), ("f16", 9001, 1024, 0), ("f32", 1702, 1024, 0),   # groups
    ("bf16", 9301, 1030, 0), ("bf16", 40001, 1030, 0), ("f16", 40003, 1030, 0), ("bf16", 160001, 34, 0),  # pairs
    ("bf16", 9903, 1031, 0), ("bf16", 20003, 1031, 0), ("f32", 20003, 1030, 1), ("f16", 9903, 1024, 3),   # single values
    ("bf16", 90001, 3, 0), ("f32", 200003, 3, 0), ("f16", 50005, 31, 0)])                               # up to 32 columns
def test_lookups_of_many_rows(lib, dtype, n, d, shift):  # noqa: F811
    S, ctx = lib
    vocab = 3001
    g = torch.Generator(device="cuda").manual_seed(n + d)
    table = place(torch.randn(vocab, d, generator=g, device="cuda").to(DT[dtype]), shift)
    ids = make_ids("text", n, vocab, 3)
    ids[::101], ids[7::1009], ids[n - 1] = vocab, -1, 2 ** 31 - 1
    ids = ids.cuda()
    scale = float(np.float32(np.sqrt(d)))
    out = place(torch.full((n, d), float("nan"), device="cuda").to(DT[dtype]), shift)
    S.sama_embed(ctx, S.DTYPES[dtype], n, vocab, d, table, ids, scale, out)
    good = (ids >= 0) & (ids < vocab)
    ref = torch.where(good[:, None], table.double()[ids.long() * good] * scale, 0.0)
    assert bool(((out.double() - ref).abs() <= 1.01 * U[dtype] * ref.abs() + TINY[dtype]).all())
    assert S.sama_device_status(ctx) == S.SAMA_DEV_BAD_INDEX


@pytest.mark.parametrize("dtype,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("n,vocab,d", [(131072, 3001, 16), (131073, 3001, 16), (140001, 70001, 8), (300007, 257, 5),
                                       (5003, 700, 1030), (5003, 700, 1024), (5003, 700, 1031), (2048, 700, 1030),
                                       (2049, 700, 1030), (2048, 5, 264), (2049, 5, 264)])
@pytest.mark.parametrize("kind", ["text", "spread"])
def test_gradients(lib, dtype, gt, n, vocab, d, kind):  # noqa: F811
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(n + d)
    dout = torch.randn(n, d, generator=g, device="cuda").to(DT[dtype])
    ids = make_ids(kind, n, vocab, 5).cuda()
    scale = float(np.float32(0.3))
    grad = torch.full((vocab, d), float("nan"), device="cuda").to(DT[gt])
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, scale, 2, S.DTYPES[gt], 0, grad)
    check_grad(grad, *plain_grad(ids, dout, vocab, scale, 2), gt)
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("dtype,gt", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f16", "f16")])
@pytest.mark.parametrize("n,vocab,d,shift", [(1, 9, 8, 0), (40, 9, 72, 0), (1500, 777, 72, 0), (2048, 777, 70, 0), (2048, 60, 33, 1),
                                             (2049, 777, 70, 0), (700, 200003, 24, 0)])
def test_adding_to_a_gradient(lib, dtype, gt, n, vocab, d, shift):  # noqa: F811
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(n + d)
    dout = place(torch.randn(n, d, generator=g, device="cuda").to(DT[dtype]), shift)
    ids = make_ids("text", n, vocab, 8)
    ids[n // 2] = vocab                    # belongs to no row
    ids = ids.cuda()
    base = torch.randn(vocab, d, generator=g, device="cuda").to(DT[gt])
    grad = place(base, shift)
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, 0.5, 3, S.DTYPES[gt], 1, grad)
    assert S.sama_device_status(ctx) == S.SAMA_DEV_BAD_INDEX
    check_grad(grad, *plain_grad(ids, dout, vocab, 0.5, 3, base), gt)
    touched = torch.zeros(vocab + 1, dtype=torch.bool, device="cuda")
    touched[ids.long()] = True
    touched[3] = False
    assert torch.equal(grad[~touched[:vocab]], base[~touched[:vocab]])


# more rows per share of the zeroing than 2^20; a table too large for the one launch, with few tokens
@pytest.mark.parametrize("n,vocab,d,dtype,gt", [(3001, 120_000_007, 1, "bf16", "bf16"), (100, 20_000_003, 2, "bf16", "f32"),
                                                (1000, 19_000_000, 2, "f16", "f16")])
def test_large_tables(lib, n, vocab, d, dtype, gt):  # noqa: F811
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(n)
    dout = torch.randn(n, d, generator=g, device="cuda").to(DT[dtype])
    ids = torch.randint(vocab, (n,), generator=g, device="cuda").to(torch.int32)
    ids[0], ids[1], ids[2] = vocab - 1, 0, ids[3]
    grad = torch.full((vocab, d), float("nan"), dtype=DT[gt], device="cuda")
    S.sama_embed_grad(ctx, S.DTYPES[dtype], n, vocab, d, ids, dout, 1.0, -1, S.DTYPES[gt], 0, grad)
    used = torch.unique(ids.long())
    check_grad(grad[used], *plain_grad(torch.searchsorted(used, ids.long()).to(torch.int32), dout, used.numel(), 1.0, -1), gt)
    grad[used] = 0
    assert int(torch.count_nonzero(grad)) == 0      # (NaN counts)
    assert S.sama_device_status(ctx) == 0
