"""Host side of attention and distillation: what is refused, and how, before anything is launched.  No kernel runs."""
import ctypes
import math

import pytest

A, B, Q, K, V, O, L, D = (4096 * 1024 * i for i in range(1, 9))    # addresses, far enough apart
G = [4096 * 1024 * i for i in range(10, 13)]


@pytest.fixture(scope="module")
def S():
    from paper_2310_05674_b200 import build
    build.build()
    from paper_2310_05674_b200 import binding
    return binding


@pytest.fixture
def blank():
    """Zeroed memory in the place of a context, for checks that come before anything in a context is looked at."""
    memory = ctypes.create_string_buffer(1 << 16)
    yield ctypes.addressof(memory)


def attn(S, **change):
    a = dict(dtype=1, heads=4, kv_heads=2, head_dim=64, n_q=10, n_k=10, n_texts=1, causal=0, q_starts=A, k_starts=None, prefix=None,
             slopes=None, scale=0.125, cap=0.0, q_stride=0, k_stride=0, v_stride=0)
    a.update(change)
    return S.sama_attn_t(*(a[n] for n, _ in S.sama_attn_t._fields_))


def forward(S, ctx, a, q=Q, k=K, v=V, out=O, lse=L):
    return S.lib.sama_attention(ctx, ctypes.byref(a) if a else None, q, k, v, out, lse, None)


def backward(S, ctx, a, q=Q, k=K, v=V, out=O, lse=L, dout=D, dq=G[0], dk=G[1], dv=G[2]):
    return S.lib.sama_attention_grad(ctx, ctypes.byref(a) if a else None, q, k, v, out, lse, dout, dq, dk, dv, None)


WRONG = [("SIZE", dict(heads=0)), ("SIZE", dict(heads=3)), ("SIZE", dict(kv_heads=0)), ("SIZE", dict(head_dim=0)),
         ("SIZE", dict(head_dim=12)), ("SIZE", dict(head_dim=136)), ("SIZE", dict(heads=65536, kv_heads=1)), ("SIZE", dict(n_q=-1)),
         ("SIZE", dict(n_q=2 ** 30 + 1)), ("SIZE", dict(n_k=11)), ("SIZE", dict(n_texts=-1)), ("SIZE", dict(n_texts=2 ** 20 + 1)),
         ("SIZE", dict(q_stride=248)), ("SIZE", dict(q_stride=260)), ("SIZE", dict(k_stride=120)), ("SIZE", dict(v_stride=2 ** 32 + 8)),
         ("SIZE", dict(n_q=2 ** 30, n_k=2 ** 30, heads=1024)), ("PARAM", dict(dtype=0)), ("PARAM", dict(dtype=3)),
         ("PARAM", dict(causal=2)), ("PARAM", dict(scale=0.0)), ("PARAM", dict(scale=-1.0)), ("PARAM", dict(scale=math.inf)),
         ("PARAM", dict(scale=math.nan)), ("PARAM", dict(cap=-1.0)), ("PARAM", dict(cap=math.inf)), ("PARAM", dict(cap=math.nan)),
         ("NULL", dict(q_starts=None)), ("ALIGN", dict(q_starts=A + 2)), ("ALIGN", dict(prefix=B + 1)), ("ALIGN", dict(slopes=B + 2))]


@pytest.mark.parametrize("status,change", WRONG, ids=lambda v: v if isinstance(v, str) else "-".join("%s=%s" % i for i in v.items()))
def test_attention_arguments(S, blank, status, change):
    want = getattr(S, "SAMA_ERR_" + status)
    assert forward(S, blank, attn(S, **change)) == want
    assert backward(S, blank, attn(S, **change)) == want


def test_attention_pointers(S, blank):
    a = attn(S)
    assert forward(S, None, a) == forward(S, blank, None) == S.SAMA_ERR_NULL
    for name in ("q", "k", "v", "out"):
        assert forward(S, blank, a, **{name: None}) == S.SAMA_ERR_NULL, name
        assert forward(S, blank, a, **{name: 8}) == S.SAMA_ERR_ALIGN, name
    assert forward(S, blank, a, lse=L + 2) == S.SAMA_ERR_ALIGN
    for name in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        assert backward(S, blank, a, **{name: None}) == S.SAMA_ERR_NULL, name
        assert backward(S, blank, a, **{name: 8 if name != "lse" else 2}) == S.SAMA_ERR_ALIGN, name


def test_attention_without_texts_does_nothing(S, blank):
    a = attn(S, n_texts=0, q_starts=None)
    assert forward(S, blank, a) == backward(S, blank, a) == S.SAMA_OK
    a = attn(S, n_q=0, n_k=0)
    assert forward(S, blank, a, None, None, None, None, None) == S.SAMA_OK
    assert backward(S, blank, a, *[None] * 9) == S.SAMA_OK


def test_attention_overlaps(S, blank):
    a, wide = attn(S), 10 * 4 * 64 * 2
    for name, at in (("q", Q), ("k", K), ("v", V)):
        assert forward(S, blank, a, out=at + 16) == S.SAMA_ERR_OVERLAP, name
        assert forward(S, blank, a, lse=at + 4) == S.SAMA_ERR_OVERLAP, name
        assert backward(S, blank, a, dv=at) == S.SAMA_ERR_OVERLAP, name
    assert forward(S, blank, a, out=A - wide + 16) == S.SAMA_ERR_OVERLAP           # the last row, on the starts
    assert forward(S, blank, a, lse=O + wide - 4) == S.SAMA_ERR_OVERLAP
    for at in (O, D, L):
        assert backward(S, blank, a, dq=at) == S.SAMA_ERR_OVERLAP
    assert backward(S, blank, a, dk=G[2]) == backward(S, blank, a, dq=G[1] + 32) == S.SAMA_ERR_OVERLAP
    # (heads + 2 key heads) rows of one buffer lie in one another's gaps: not an overlap, unless they are too wide for it
    row, n = (4 + 2 + 2) * 64, 0
    a = attn(S, q_stride=row, k_stride=row, v_stride=row, n_texts=n)
    assert backward(S, blank, a, dq=G[0], dk=G[0] + 4 * 128, dv=G[0] + 6 * 128) == S.SAMA_OK
    assert backward(S, blank, a, dq=G[0], dk=G[0] + 4 * 128, dv=G[0] + 5 * 128) == S.SAMA_ERR_OVERLAP
    assert backward(S, blank, a, dq=G[0], dk=G[0] + 3 * 128, dv=G[0] + 6 * 128) == S.SAMA_ERR_OVERLAP
    assert backward(S, blank, a, dq=G[0], dk=G[0] + 4 * 128, dv=G[0] + 7 * 128) == S.SAMA_ERR_OVERLAP   # into the next row's dq
    b = attn(S, q_stride=row, k_stride=row + 64, v_stride=row, n_texts=n)
    assert backward(S, blank, b, dq=G[0], dk=G[0] + 4 * 128, dv=G[0] + 6 * 128) == S.SAMA_ERR_OVERLAP


def paged(S, **change):
    a = dict(dtype=1, heads=4, kv_heads=2, head_dim=64, page_size=16, n_seqs=3, max_pages=5, n_pages=20, page_stride=0, page_table=A,
             lengths=B, slopes=None, scale=0.125, cap=0.0)
    a.update(change)
    return S.sama_paged_t(*(a[n] for n, _ in S.sama_paged_t._fields_))


def decode(S, ctx, a, q=Q, k_new=G[0], v_new=G[1], k=K, v=V, out=O):
    return S.lib.sama_paged_attention(ctx, ctypes.byref(a) if a else None, q, k_new, v_new, k, v, out, None)


@pytest.mark.parametrize("status,change", [w for w in WRONG if set(w[1]) <= {"heads", "kv_heads", "head_dim", "dtype", "scale", "cap"}] + [
    ("SIZE", dict(page_size=0)), ("SIZE", dict(page_size=2 ** 20 + 1)), ("SIZE", dict(n_seqs=-1)), ("SIZE", dict(n_seqs=2 ** 20 + 1)),
    ("SIZE", dict(max_pages=0)), ("SIZE", dict(max_pages=2 ** 24 + 1)), ("SIZE", dict(n_pages=0)), ("SIZE", dict(n_pages=2 ** 31)),
    ("SIZE", dict(n_seqs=2 ** 20, max_pages=2 ** 20, page_size=64)), ("SIZE", dict(page_stride=2040)), ("SIZE", dict(page_stride=2052)), ("NULL", dict(page_table=None)), ("NULL", dict(lengths=None)),
    ("ALIGN", dict(page_table=A + 2)), ("ALIGN", dict(lengths=B + 1)), ("ALIGN", dict(slopes=D + 3))],
    ids=lambda v: v if isinstance(v, str) else "-".join("%s=%s" % i for i in v.items()))
def test_paged_arguments(S, blank, status, change):
    assert decode(S, blank, paged(S, **change)) == getattr(S, "SAMA_ERR_" + status)


def test_paged_pointers_and_overlaps(S, blank):
    a = paged(S)
    assert decode(S, None, a) == decode(S, blank, None) == S.SAMA_ERR_NULL
    for name in ("q", "k", "v", "out", "k_new", "v_new"):      # (one of the new rows without the other)
        assert decode(S, blank, a, **{name: None}) == S.SAMA_ERR_NULL, name
        assert decode(S, blank, a, **{name: 24}) == S.SAMA_ERR_ALIGN, name
    for at in (Q, K, V, G[0], A, B):
        assert decode(S, blank, a, out=at) == S.SAMA_ERR_OVERLAP, at
    assert decode(S, blank, a, k=V) == decode(S, blank, a, k_new=K + 32) == decode(S, blank, a, q=V) == S.SAMA_ERR_OVERLAP
    none = paged(S, n_seqs=0)
    assert decode(S, blank, none) == S.SAMA_OK
    page = 16 * 2 * 64
    apart = paged(S, page_stride=2 * page, n_seqs=0)           # keys and values of a page behind one another
    assert decode(S, blank, apart, k=K, v=K + 2 * page) == S.SAMA_OK
    assert decode(S, blank, apart, k=K, v=K + page) == S.SAMA_ERR_OVERLAP


def distill(S, ctx, dtype=1, n=4, vocab=100, logits=Q, ld=0, k=5, top_dtype=0, top=K, ids=V, T=1.0, weight=A, scale=1.0, loss=L, grad=O,
            ld_grad=0):
    return S.lib.sama_distill(ctx, dtype, n, vocab, logits, ld, k, top_dtype, top, ids, T, weight, scale, loss, grad, ld_grad, None)


@pytest.mark.parametrize("status,change", [
    ("SIZE", dict(n=-1)), ("SIZE", dict(n=2 ** 30 + 1)), ("SIZE", dict(vocab=0)), ("SIZE", dict(vocab=2 ** 24 + 1)), ("SIZE", dict(k=0)),
    ("SIZE", dict(k=1025)), ("SIZE", dict(ld=99)), ("SIZE", dict(ld_grad=99)), ("SIZE", dict(ld=2 ** 30 + 1)), ("PARAM", dict(dtype=3)),
    ("PARAM", dict(top_dtype=-1)), ("PARAM", dict(T=0.0)), ("PARAM", dict(T=-1.0)), ("PARAM", dict(T=math.inf)), ("PARAM", dict(T=math.nan)),
    ("PARAM", dict(scale=math.inf)), ("PARAM", dict(scale=math.nan)), ("NULL", dict(logits=None)), ("NULL", dict(top=None)),
    ("NULL", dict(ids=None)), ("ALIGN", dict(logits=Q + 1)), ("ALIGN", dict(grad=O + 1)), ("ALIGN", dict(top=K + 2)), ("ALIGN", dict(ids=V + 2)),
    ("ALIGN", dict(weight=A + 1)), ("ALIGN", dict(loss=L + 2)), ("OVERLAP", dict(grad=Q + 2)), ("OVERLAP", dict(grad=Q, ld_grad=104)),
    ("OVERLAP", dict(grad=K)), ("OVERLAP", dict(grad=V + 8)), ("OVERLAP", dict(grad=A - 790)), ("OVERLAP", dict(loss=Q + 796)),
    ("OVERLAP", dict(loss=O)), ("OVERLAP", dict(loss=A))], ids=lambda v: v if isinstance(v, str) else "-".join("%s=%s" % i for i in v.items()))
def test_distill_arguments(S, blank, status, change):
    assert distill(S, blank, **change) == getattr(S, "SAMA_ERR_" + status)


def test_distill_without_work(S, blank):
    assert distill(S, None) == S.SAMA_ERR_NULL
    assert distill(S, blank, n=0, logits=None, top=None, ids=None) == distill(S, blank, loss=None, grad=None) == S.SAMA_OK


class Tensor:
    """What the binding looks at, of a tensor."""

    def __init__(self, shape, dtype, device=0, stride=None, at=4096):
        self.shape, self.dtype, self.at, self.gpu, self.device = tuple(shape), dtype, at, device, "cuda:%d" % device
        self.strides = stride or [math.prod(shape[i + 1:]) for i in range(len(shape))]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def get_device(self):
        return self.gpu

    def stride(self, i=None):
        return tuple(self.strides) if i is None else self.strides[i]

    def is_contiguous(self):
        return list(self.strides) == [math.prod(self.shape[i + 1:]) for i in range(len(self.shape))]

    def data_ptr(self):
        return self.at

    def __getitem__(self, i):
        return Tensor(self.shape[1:], self.dtype, self.gpu, self.strides[1:])


def test_the_binding_checks_tensors(S, monkeypatch):
    import torch
    bf, i32, f32 = torch.bfloat16, torch.int32, torch.float32
    monkeypatch.setitem(S._device_of, 4096, 0)
    seen = []
    for name in ("sama_attention", "sama_paged_attention", "sama_distill"):
        monkeypatch.setattr(S.lib, name, lambda *a: seen.append(a) or 0)
    starts = Tensor([2], i32)

    def attend(q=None, k=None, v=None, out=None, lse=None, ctx=4096, **kw):
        a = S.Attn(1, 4, 2, 64, 10, 10, starts, **kw)
        S.sama_attention(ctx, a, q or Tensor([10, 4, 64], bf), k or Tensor([10, 2, 64], bf), v or Tensor([10, 2, 64], bf),
                         out or Tensor([10, 4, 64], bf), lse, stream=0)

    attend()
    attend(q=Tensor([10, 4, 64], bf, stride=[512, 64, 1]), q_stride=512)
    assert len(seen) == 2 and seen[1][1]._obj.q_stride == 512 and seen[0][1]._obj.n_texts == 1

    def refused(status, fn, **kw):
        with pytest.raises(S.SamaError) as e:
            fn(**kw)
        assert e.value.status == status, kw

    refused(S.SAMA_ERR_PARAM, attend, q=Tensor([10, 4, 64], bf, device=1))
    refused(S.SAMA_ERR_PARAM, attend, q=Tensor([10, 4, 64], torch.float16))
    refused(S.SAMA_ERR_PARAM, attend, q=Tensor([10, 4, 64], bf, stride=[512, 64, 1]))
    refused(S.SAMA_ERR_PARAM, attend, k=Tensor([10, 2, 64], bf, stride=[128, 1, 2]))
    refused(S.SAMA_ERR_SIZE, attend, q=Tensor([9, 4, 64], bf))
    refused(S.SAMA_ERR_SIZE, attend, k=Tensor([10, 4, 64], bf))
    refused(S.SAMA_ERR_SIZE, attend, out=Tensor([9, 4, 64], bf))
    refused(S.SAMA_ERR_SIZE, attend, lse=Tensor([39], f32))
    refused(S.SAMA_ERR_SIZE, attend, slopes=Tensor([3], f32))
    refused(S.SAMA_ERR_SIZE, attend, prefix=Tensor([0], i32))
    refused(S.SAMA_ERR_PARAM, attend, prefix=Tensor([1], f32))
    monkeypatch.setitem(S._device_of, 8192, 1)
    refused(S.SAMA_ERR_PARAM, attend, ctx=8192)

    def look(table=None, lengths=None, k=None, q=None, **kw):
        p = S.Paged(1, 4, 2, 64, 16, 20, table or Tensor([3, 5], i32), lengths or Tensor([3], i32), **kw)
        cache = Tensor([20, 16, 2, 64], bf)
        S.sama_paged_attention(4096, p, q or Tensor([3, 4, 64], bf), None, None, k or cache, cache, Tensor([3, 4, 64], bf), stream=0)

    look()
    refused(S.SAMA_ERR_SIZE, look, table=Tensor([15], i32))
    refused(S.SAMA_ERR_SIZE, look, lengths=Tensor([2], i32))
    refused(S.SAMA_ERR_SIZE, look, k=Tensor([19, 16, 2, 64], bf))
    refused(S.SAMA_ERR_SIZE, look, q=Tensor([2, 4, 64], bf))
    refused(S.SAMA_ERR_PARAM, look, k=Tensor([20, 16, 2, 64], bf, stride=[4096, 128, 64, 1]))
    refused(S.SAMA_ERR_PARAM, look, page_stride=4096)
    refused(S.SAMA_ERR_PARAM, look, k=Tensor([20, 16, 2, 64], bf, device=1))

    def learn(z=None, top=None, ids=None, grad=None, weight=None):
        S.sama_distill(4096, 1, 4, 100, z or Tensor([4, 100], bf), 5, 0, top or Tensor([4, 5], f32), ids or Tensor([4, 5], i32), 1.0, weight,
                       1.0, Tensor([4], f32), grad, stream=0)

    learn()
    learn(z=Tensor([4, 100], bf, stride=[128, 1]), grad=Tensor([4, 100], bf, stride=[104, 1]))
    assert seen[-1][5] == 128 and seen[-1][-2] == 104
    refused(S.SAMA_ERR_PARAM, learn, z=Tensor([4, 100], f32))
    refused(S.SAMA_ERR_PARAM, learn, z=Tensor([4, 100], bf, stride=[1, 4]))
    refused(S.SAMA_ERR_SIZE, learn, z=Tensor([4, 99], bf))
    refused(S.SAMA_ERR_SIZE, learn, grad=Tensor([3, 100], bf))
    refused(S.SAMA_ERR_SIZE, learn, ids=Tensor([4, 4], i32))
    refused(S.SAMA_ERR_PARAM, learn, ids=Tensor([4, 5], torch.int64))
    refused(S.SAMA_ERR_PARAM, learn, weight=Tensor([4], bf))
    refused(S.SAMA_ERR_PARAM, learn, top=Tensor([4, 5], f32, device=-1))


def test_data_that_may_change_is_not_read_through_the_read_only_path():
    """Kernels may start before the launch whose results they read has ended, and distillation may work in place."""
    import os
    import re
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_05674_b200", "csrc")
    for f in ("attention.h", "attention_fwd.cu", "attention_bwd.cu", "attention_paged.cu", "distill.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(csrc, f)).read())
        assert not re.search(r"__ldg\b|ld\.global\.nc|__restrict__", text), f
