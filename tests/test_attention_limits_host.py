"""The ranges of scale, cap and temperature: what is beyond them would pass fp32 inside the kernels.  No kernel runs."""
import pytest

from test_attention_host import attn, backward, blank, decode, distill, forward, paged, S  # noqa: F401  (fixtures among them)


@pytest.mark.parametrize("change", [dict(scale=2.0 ** -61), dict(scale=2.0 ** 61), dict(cap=2.0 ** -61), dict(cap=2.0 ** 61),
                                    dict(scale=1e-40), dict(cap=3e38), dict(cap=1e-30), dict(scale=1.0, cap=2.0 ** -14),
                                    dict(scale=2.0 ** 60, cap=1.0)], ids=str)
def test_scales_and_caps_beyond_the_range(S, blank, change):  # noqa: F811
    assert forward(S, blank, attn(S, **change)) == backward(S, blank, attn(S, **change)) == S.SAMA_ERR_PARAM
    assert decode(S, blank, paged(S, **change)) == S.SAMA_ERR_PARAM


@pytest.mark.parametrize("change", [dict(scale=2.0 ** -60), dict(scale=2.0 ** 60), dict(cap=2.0 ** 60), dict(scale=2.0 ** -60, cap=2.0 ** -60),
                                    dict(scale=1.0, cap=2.0 ** -13), dict(scale=2.0 ** -60, cap=2.0 ** 60)], ids=str)
def test_scales_and_caps_at_its_ends(S, blank, change):  # noqa: F811
    assert forward(S, blank, attn(S, n_texts=0, **change)) == backward(S, blank, attn(S, n_texts=0, **change)) == S.SAMA_OK
    assert decode(S, blank, paged(S, n_seqs=0, **change)) == S.SAMA_OK


@pytest.mark.parametrize("change", [dict(T=2.0 ** -61), dict(T=2.0 ** 61), dict(T=1e-40), dict(T=3e38), dict(T=2.0 ** 60, scale=2.0 ** 70),
                                    dict(T=4.0, scale=-3e38)], ids=str)
def test_temperatures(S, blank, change):  # noqa: F811
    assert distill(S, blank, **change) == S.SAMA_ERR_PARAM
    for T, scale in ((2.0 ** -60, 1.0), (2.0 ** 60, 2.0 ** 60), (0.5, 3e38)):
        assert distill(S, blank, n=0, T=T, scale=scale) == S.SAMA_OK
