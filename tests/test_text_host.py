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
