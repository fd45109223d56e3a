"""Global gradient norm and clipping against a plain implementation in 64 bits.

Tolerances.  The squares of fp32 values are exact in double up to 2^-53 and their sum has a relative error of at most
(number of terms) 2^-53, far below fp32's 2^-24; the norm is then rounded once: 2^-24, and 1.1 of it leaves room.  The
factor is rounded to fp32 (2^-24), the product too (2^-24), then to the type (u = 2^-p: 2^-24, 2^-8, 2^-11 for fp32,
bf16, fp16): u + 2^-23 relative, and half of fp16's smallest subnormal step, 2^-25.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def plain(ins, max_norm):
    norm = math.sqrt(sum(float((x.double() ** 2).sum()) for x in ins))
    c = min(1.0, max_norm / norm) if norm > 0 else 1.0
    return norm, [x.double() * c for x in ins]


def close(got, ref):
    u = U[got.dtype]
    assert bool(((got.double() - ref).abs() <= (1.01 * u + 2.0 ** -23) * ref.abs() + TINY[got.dtype]).all())


def run(lib, ins, outs, max_norm):
    S, ctx = lib
    norm = torch.full((1,), -1.0, device="cuda")
    S.sama_clip_grads(ctx, S.TensorList(ins, outs), max_norm, norm)
    return float(norm)


def tensors(sizes, types, seed=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        t = DT[types[i % len(types)]]
        x = (10.0 ** (i % 4 - 2) * torch.randn(n + 16, generator=g, device="cuda")).to(t)
        out.append(x[shift:shift + n])
    return out


SIZES = {"none": [], "empty": [0], "one": [1], "small": [10, 0, 7, 8, 2047, 2048, 2049], "ragged": [100003, 5, 262144, 1, 40961],
         "many": [1 + 37 * i % 301 for i in range(400)], "launches": [1 + i % 5 for i in range(2500)],
         "large": [9_000_001, 3, 5_000_000]}


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16"], ["bf16", "f32", "f16"]])
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
@pytest.mark.parametrize("shift", [0, 3])
def test_separate_outputs(lib, sizes, types, max_norm, shift):
    ins = tensors(SIZES[sizes], types, 1, shift)
    keep = [x.clone() for x in ins]
    outs = [torch.full_like(x, 7.0) for x in ins]
    norm, ref = plain(ins, max_norm)
    got = run(lib, ins, outs, max_norm)
    assert abs(got - norm) <= 1.1 * 2.0 ** -24 * norm
    for y, r in zip(outs, ref):
        close(y, r)
    assert all(torch.equal(a, b) for a, b in zip(ins, keep))
    again = [torch.empty_like(x) for x in ins]
    assert run(lib, ins, again, max_norm) == got and all(torch.equal(a, b) for a, b in zip(outs, again))
    S, ctx = lib
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("count", [1, 100, 112, 113])
@pytest.mark.parametrize("total", [2 ** 18 + 1, 2 ** 19, 2 ** 19 + 1])
@pytest.mark.parametrize("types", [["f32"], ["bf16", "f32", "f16"]])
def test_where_one_launch_ends(lib, count, total, types):
    sizes = [total // count] * (count - 1)
    sizes.append(total - sum(sizes))
    ins = tensors(sizes, types, 4)
    outs = [torch.full_like(x, 7.0) for x in ins]
    norm, ref = plain(ins, 0.5)
    assert abs(run(lib, ins, outs, 0.5) - norm) <= 1.1 * 2.0 ** -24 * norm
    for y, r in zip(outs, ref):
        close(y, r)


@pytest.mark.parametrize("types", [["f32"], ["bf16"], ["f16", "f32"]])
@pytest.mark.parametrize("sizes", ["small", "ragged", "many"])
def test_into_the_flat_vector(lib, types, sizes):
    """Consecutive slices of one fp32 vector, most of them at an odd multiple of 4 bytes."""
    ins = tensors(SIZES[sizes], types, 2)
    flat = torch.full((sum(SIZES[sizes]) + 1,), float("nan"), device="cuda")
    outs = list(flat[:-1].split(SIZES[sizes]))
    norm, ref = plain(ins, 1.0)
    run(lib, ins, outs, 1.0)
    close(flat[:-1], torch.cat(ref))
    assert math.isnan(float(flat[-1]))


@pytest.mark.parametrize("types", [["f32"], ["bf16", "f32"], ["f16"]])
@pytest.mark.parametrize("shift", [0, 1])
def test_in_place(lib, types, shift):
    ins = tensors(SIZES["ragged"], types, 3, shift)
    keep = [x.clone() for x in ins]
    norm, ref = plain(ins, 1.0)
    run(lib, ins, None, 1e9)                       # nothing to clip: nothing is changed
    assert all(torch.equal(a, b) for a, b in zip(ins, keep))
    run(lib, ins, None, 1.0)
    for y, r in zip(ins, ref):
        close(y, r)
    new = run(lib, ins, None, 1.0)
    assert abs(new - 1.0) < 1e-2                   # (bf16 rounding of the clipped values moves their norm)


def test_norm_only_and_other_output_types(lib):
    S, ctx = lib
    ins = tensors([5000, 77, 3001], ["bf16", "f32"], 4)
    outs = [None, torch.empty(77, dtype=torch.float16, device="cuda"), torch.empty(3001, dtype=torch.float32, device="cuda")]
    norm, ref = plain(ins, 0.1)
    assert abs(run(lib, ins, outs, 0.1) - norm) <= 1.1 * 2.0 ** -24 * norm
    close(outs[1], ref[1])
    close(outs[2], ref[2])
    before = [x.clone() for x in ins]
    assert abs(run(lib, ins, [None] * 3, 0.1) - norm) <= 1.1 * 2.0 ** -24 * norm
    assert all(torch.equal(a, b) for a, b in zip(ins, before))
    S.sama_clip_grads(ctx, S.TensorList(ins, outs), float("inf"), None)   # no limit, no norm wanted
    close(outs[2], ins[2].double())


def test_zeros_and_values_whose_squares_leave_fp32(lib):
    S, ctx = lib
    z = [torch.zeros(1000, device="cuda")]
    o = [torch.ones(1000, device="cuda")]
    assert run(lib, z, o, 1.0) == 0.0 and not bool(o[0].any())
    for v in (3e38, 1e-38, 1e-44):
        x = [torch.full((3000,), v, device="cuda")]
        norm, ref = plain(x, 1e-30)
        out = [torch.empty_like(x[0])]
        got = run(lib, x, out, 1e-30)
        assert (math.isinf(got) and norm > 3.4e38) or abs(got - norm) <= 1.1 * 2.0 ** -24 * norm + 2.0 ** -150
        # subnormal results carry an absolute error of half a step, 2^-150, twice
        assert bool(((out[0].double() - ref[0]).abs() <= 2.0 ** -22 * ref[0].abs() + 2.0 ** -149).all())
    assert S.sama_device_status(ctx) == 0


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_a_gradient_that_is_not_finite_gives_zeros(lib, bad, dtype):
    S, ctx = lib
    ins = tensors([5000, 300000], [dtype], 6)
    ins[1][123457] = bad
    outs = [torch.ones_like(ins[0]), ins[1]]       # one separate, one in place
    got = run(lib, ins, outs, 1.0)
    assert not math.isfinite(got) and math.isnan(got) == math.isnan(bad)
    assert not bool(outs[0].any()) and not bool(ins[1].any())
    assert S.sama_device_status(ctx) == S.SAMA_DEV_NONFINITE_GRAD
    assert run(lib, ins, outs, 1.0) > 0 and S.sama_device_status(ctx) == 0


def test_feeds_the_adaptation(lib):
    """The clipped flat vector is what sama_adapt takes as the base gradient, on the same stream."""
    S, ctx = lib
    sizes = [600, 24, 400]
    ins = tensors(sizes, ["bf16", "f32"], 7)
    flat = torch.empty(1024, device="cuda")
    S.sama_clip_grads(ctx, S.TensorList(ins, list(flat.split(sizes))), 1.0)
    ss = torch.zeros(1, dtype=torch.float64, device="cuda")
    p = torch.empty(1024, device="cuda")
    S.sama_adapt(ctx, 1024, None, None, None, flat, S.Adam(identity=True), p, ss)
    assert abs(float(ss) - 1.0) < 1e-5 and torch.equal(p, flat)


def test_runs_on_the_callers_stream(lib):
    S, ctx = lib
    x = torch.zeros(1 << 20, device="cuda")
    out = torch.empty_like(x)
    lst = S.TensorList([x], [out])
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(16):
            x.add_(0.25)
        S.sama_clip_grads(ctx, lst, 1024.0)
        y = out.clone()
    s.synchronize()
    assert bool((y == 1.0).all())                  # norm 4 * 1024, clipped to 1024


def test_refusals(lib):
    S, ctx = lib
    x, y = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    norm = torch.zeros(1, device="cuda")

    def status(lst, max_norm=1.0, norm_out=norm, n=None, c=ctx):
        with pytest.raises(S.SamaError) as e:
            S._check(S.lib.sama_clip_grads(c, lst.c() if lst else None, len(lst.ins) if n is None else n, max_norm,
                                           S._ptr(norm_out), S._stream(None)), "sama_clip_grads")
        return e.value.status

    ok = S.TensorList([x], [y])
    assert status(ok, c=None) == S.SAMA_ERR_NULL
    assert status(None, n=1) == S.SAMA_ERR_NULL
    assert status(ok, n=-1) == S.SAMA_ERR_SIZE
    assert status(ok, n=65537) == S.SAMA_ERR_SIZE
    for m in (0.0, -1.0, float("nan")):
        assert status(ok, m) == S.SAMA_ERR_PARAM
    assert status(ok, norm_out=norm.data_ptr() + 2) == S.SAMA_ERR_ALIGN
    assert status(ok, norm_out=x) == S.SAMA_ERR_OVERLAP
    assert status(ok, norm_out=y) == S.SAMA_ERR_OVERLAP

    def broken(**kw):
        t = S.TensorList([x], [y])
        for k, v in kw.items():
            setattr(t.c()[0], k, v)
        return status(t)

    assert broken(in_=None) == S.SAMA_ERR_NULL
    assert broken(n=-1) == S.SAMA_ERR_SIZE
    assert broken(dtype=3) == S.SAMA_ERR_PARAM
    assert broken(out_dtype=-1) == S.SAMA_ERR_PARAM
    assert broken(in_=x.data_ptr() + 2) == S.SAMA_ERR_ALIGN
    assert broken(out=x.data_ptr() + 16, n=8) == S.SAMA_ERR_OVERLAP
    assert broken(out=x.data_ptr(), out_dtype=S.SAMA_BF16) == S.SAMA_ERR_OVERLAP
    with pytest.raises(S.SamaError):
        S.TensorList([x.view(8, 8)[:, :4]])
    with pytest.raises(S.SamaError):
        S.TensorList([x.double()])
    with pytest.raises(S.SamaError):
        S.TensorList([x], [y, y])
    with pytest.raises(S.SamaError):
        S.TensorList([x], [y[:5]])
    assert S.sama_device_status(ctx) == 0
