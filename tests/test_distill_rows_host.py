"""Rows of a matrix that the binding hands to sama_distill: how far apart they lie, and what is refused.  No kernel runs."""
import math

import pytest


class Matrix:
    """What the binding looks at, of a tensor on the first GPU."""

    def __init__(self, shape, dtype, stride=None):
        self.shape, self.dtype, self.device = tuple(shape), dtype, "cuda:0"
        self.strides = tuple(stride or (math.prod(shape[i + 1:]) for i in range(len(shape))))

    def dim(self):
        return len(self.shape)

    def numel(self):
        return math.prod(self.shape)

    def get_device(self):
        return 0

    def stride(self, i=None):
        return self.strides if i is None else self.strides[i]

    def is_contiguous(self):
        return self.strides == tuple(math.prod(self.shape[i + 1:]) for i in range(len(self.shape)))

    def data_ptr(self):
        return 4096


@pytest.fixture
def distill(monkeypatch):
    """Calls sama_distill with a stand-in for the library; returns the row strides that it was given."""
    import torch
    from paper_2310_05674_b200 import build
    build.build()
    from paper_2310_05674_b200 import binding as S
    calls = []
    monkeypatch.setitem(S._device_of, 4096, 0)
    monkeypatch.setattr(S.lib, "sama_distill", lambda *a: calls.append(a) or 0)

    def call(n, vocab, z=None, grad=None, **kw):
        bf = torch.bfloat16
        z = Matrix((n, vocab), bf, z) if not isinstance(z, Matrix) else z
        S.sama_distill(4096, S.SAMA_BF16, n, vocab, z, 1, S.SAMA_F32, Matrix((n, 1), torch.float32), Matrix((n, 1), torch.int32), 1.0, None,
                       1.0, None, Matrix((n, vocab), bf, grad) if isinstance(grad, tuple) else grad, stream=0, **kw)
        return calls[-1][5], calls[-1][-2]

    call.S, call.bf, call.calls = S, torch.bfloat16, calls
    return call


@pytest.mark.parametrize("stride", [(0, 1), (1, 1), (999, 1)])
@pytest.mark.parametrize("n", [2, 64])
def test_rows_that_lie_in_one_another_are_refused(distill, n, stride):
    """One row that stands for many (`row.expand(n, -1)`) among them: to the library a stride of 0 means rows without gaps,
    and it would read, or write, n rows where there is one."""
    for kw in (dict(z=stride), dict(grad=stride)):
        with pytest.raises(distill.S.SamaError) as e:
            distill(n, 1000, **kw)
        assert e.value.status == distill.S.SAMA_ERR_PARAM
    assert not distill.calls


def test_one_column_that_stands_for_many_is_refused(distill):
    for kw in (dict(z=(0, 0)), dict(z=(0, 1)), dict(grad=(0, 1))):
        with pytest.raises(distill.S.SamaError):
            distill(5, 1, **kw)
    with pytest.raises(distill.S.SamaError):
        distill(5, 7, z=(7, 0))
    assert not distill.calls


def test_other_rows_are_handed_on(distill):
    assert distill(64, 1000, z=(1000, 1), grad=(1016, 1)) == (1000, 1016)
    # a single row has no stride, whatever the tensor says of it
    assert distill(1, 1000, z=(0, 1), grad=(0, 1)) == (0, 0)
    assert distill(1, 1000, z=Matrix((4, 1000), distill.bf, (0, 1)), ld=2000) == (2000, 0)


def test_a_ring_place_is_fenced_whatever_is_asked_for():
    """Rows that a warp each works on: what a thread has stored into a place of the ring (a row's ends) has to be ordered before
    the copy that takes the place next, for losses alone, too: once per row, after the stores, before that copy."""
    import os
    import re
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2310_05674_b200", "csrc", "distill.cu")
    text = re.sub(r"//[^\n]*", "", open(path).read())
    kernel = text[text.index("distill_few_kernel(const DistillParams P)"):text.index("distill_long_kernel(const DistillParams P)")]
    loop = kernel[kernel.index("[place] = edge"):kernel.index("fetch_row(after")]
    at = loop.index("if (P.grad) {")
    depth, end = 0, at
    for end in range(at, len(loop)):
        depth += {"{": 1, "}": -1}.get(loop[end], 0)
        if depth == 0 and loop[end] == "}":
            break
    with_gradient, without = loop[at:end], loop[:at] + loop[end:]
    assert "fence.proxy.async" in without
    last = max(m.start() for m in re.finditer(r"(chunk\)\[[^=]*\] = |store_n<)", with_gradient))
    assert "fence.proxy.async" in with_gradient[last:] or "fence.proxy.async" in loop[end:]
