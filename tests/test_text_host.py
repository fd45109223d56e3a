"""Host side of the text-model operators: what is refused, and how, before anything is launched.  No kernel runs."""
import ctypes

import pytest


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


@pytest.mark.parametrize("d", [2 ** 30 + 1, 2 ** 31 - 4, 2 ** 31 - 1])
def test_rows_that_32_bit_columns_cannot_step_through_are_refused(S, blank, d):
    assert S.lib.sama_embed(blank, S.SAMA_F32, 0, 1, d, 16, None, 1.0, None, None) == S.SAMA_ERR_SIZE
    assert S.lib.sama_embed_grad(blank, S.SAMA_F32, 0, 1, d, None, None, 1.0, -1, S.SAMA_F32, 1, 16, None) == S.SAMA_ERR_SIZE


def test_the_widest_row_is_accepted(S, blank):
    assert S.lib.sama_embed(blank, S.SAMA_F32, 0, 1, 2 ** 30, 16, None, 1.0, None, None) == S.SAMA_OK


def host_tensors(torch):
    """Every operand that is a tensor, by operator, on the host: each position is tried alone, beside plain addresses."""
    f, i, h = torch.zeros(64), torch.zeros(64, dtype=torch.int32), torch.zeros(64, dtype=torch.bfloat16)
    return {"sama_embed": ([0, 4, 4, 4], [f, i], [1.0], [f]),
            "sama_embed_grad": ([0, 4, 4, 4], [i, f], [1.0, -1, 0, 0], [f]),
            "sama_gated_ffn": ([1, 0, 4, 4, 4], [h] * 7, [], []),
            "sama_gated_ffn_grad": ([1, 0, 4, 4, 4], [h] * 11, [], [])}


@pytest.mark.parametrize("name,operands", [("sama_embed", 3), ("sama_embed_grad", 3), ("sama_gated_ffn", 7),
                                           ("sama_gated_ffn_grad", 11)])
def test_tensors_on_the_host_are_refused(S, name, operands):
    import torch
    for k in range(operands):
        n, a, between, b = host_tensors(torch)[name]
        a, b = ([t if at == k else 4096 * (at + 1) for at, t in part] for part in
                (list(enumerate(a)), list(enumerate(b, len(a)))))
        # (without a context, which is refused too, but later and with another status)
        with pytest.raises(S.SamaError) as e:
            getattr(S, name)(None, *n, *a, *between, *b, stream=0)
        assert e.value.status == S.SAMA_ERR_PARAM, k


def test_lists_of_tensors_on_the_host_are_refused(S):
    import torch
    for outs in (None, [None], [torch.zeros(8)]):
        with pytest.raises(S.SamaError) as e:
            S.TensorList([torch.zeros(8)], outs)
        assert e.value.status == S.SAMA_ERR_PARAM
    with pytest.raises(S.SamaError) as e:
        S.sama_clip_grads(None, S.TensorList([]), 1.0, torch.zeros(1), stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM


def test_tensors_on_another_gpu_than_the_context_are_refused(S, monkeypatch):
    class On:   # what the check looks at, of a tensor on GPU 1
        device = "cuda:1"

        def get_device(self):
            return 1

    monkeypatch.setitem(S._device_of, 4096, 0)
    with pytest.raises(S.SamaError) as e:
        S.sama_embed(4096, 0, 4, 4, 4, On(), 8192, 1.0, 16384, stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM
    tensors = S.TensorList([])
    tensors.device = 1
    with pytest.raises(S.SamaError) as e:
        S.sama_clip_grads(4096, tensors, 1.0, stream=0)
    assert e.value.status == S.SAMA_ERR_PARAM


def test_a_list_in_place_takes_any_iterable(S):
    class OnGpu:
        dtype = device = None

        def numel(self):
            return 8

        def get_device(self):
            return 0

        def is_contiguous(self):
            return True

        def data_ptr(self):
            return 4096

    import torch
    OnGpu.dtype = torch.float32
    x = OnGpu()
    tensors = S.TensorList(t for t in [x, x])
    assert tensors.ins == tensors.outs == [x, x] and tensors.c()[1].out == tensors.c()[1].in_ == 4096
