"""The gated feed-forward block and its backward pass against a plain implementation in 64 bits.

Tolerances are bounds, element by element, carried through the block's formulas.  With u = 2^-p the unit roundoff of the
type (2^-8 for bf16, 2^-11 for fp16, and half of fp16's smallest subnormal step, 2^-25, absolute), and a product of
length K summed in fp32 wrong by at most K 2^-23 sum |a b| (the tensor core truncates, one rounding per term is more than
it does), a value z computed from x with error dx has the error  |dz/dx| dx + rounding.  The activations are evaluated in
fp32 to 2^-20 (1 + |x|) absolute (exp and the quotient to a few units of 2^-23, times the factors that multiply them).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f16": torch.float16}
U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"bf16": 0.0, "f16": 2.0 ** -25}
ACC, FN = 2.0 ** -23, 2.0 ** -20
ACTS = ["silu", "gelu", "gelu_tanh", "relu"]
LIP = 1.13   # the largest slope of any of the activations


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def act(kind, g):
    if kind == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if kind == "silu":
        s = torch.sigmoid(g)
        return g * s, s + g * s * (1 - s)
    if kind == "gelu":
        p = torch.special.ndtr(g)
        return g * p, p + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def make(M, d, f, dtype, seed=0, shift=0):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def r(rows, cols, scale):
        buf = torch.empty(rows * cols + 16, dtype=DT[dtype], device="cuda")
        v = buf[shift:shift + rows * cols].view(rows, cols)
        return v.copy_(scale * torch.randn(rows, cols, generator=g, device="cuda"))

    return {"x": r(M, d, 1.0), "wg": r(f, d, 1.5 / math.sqrt(d)), "wu": r(f, d, 1 / math.sqrt(d)), "wd": r(d, f, 1 / math.sqrt(f)),
            "dy": r(M, d, 1.0), "gate": r(M, f, 1.5), "up": r(M, f, 1.0)}


def forward(lib, t, kind, save=False, stream=None):
    S, ctx = lib
    (M, d), f = t["x"].shape, t["wg"].shape[0]
    dt = S._dtype_of(t["x"])
    y = torch.full_like(t["x"], float("nan"))
    gate, up = (torch.full((M, f), float("nan"), dtype=t["x"].dtype, device="cuda") for _ in range(2)) if save else (None, None)
    S.sama_gated_ffn(ctx, dt, S.ACTS[kind], M, d, f, t["x"], t["wg"], t["wu"], t["wd"], y, gate, up, stream)
    return y, gate, up


def backward(lib, t, kind, want=(1, 1, 1, 1)):
    S, ctx = lib
    (M, d), f = t["x"].shape, t["wg"].shape[0]
    outs = [torch.full_like(t[k], float("nan")) if w else None for k, w in zip(("x", "wg", "wu", "wd"), want)]
    S.sama_gated_ffn_grad(ctx, S._dtype_of(t["x"]), S.ACTS[kind], M, d, f, t["x"], t["wg"], t["wu"], t["wd"], t["gate"],
                          t["up"], t["dy"], *outs)
    return outs


def within(got, ref, err, dtype):
    bound = U[dtype] * (ref.abs() + err) + err + TINY[dtype]
    over = (got.double() - ref).abs() - bound
    assert bool((over <= 0).all()), (float(over.max()), float((got.double() - ref).norm() / ref.norm()))


def check_forward(lib, M, d, f, dtype, kind, shift=0):
    t = make(M, d, f, dtype, M + d, shift)
    y, gate, up = forward(lib, t, kind, save=True)
    x, wg, wu, wd = (t[k].double() for k in ("x", "wg", "wu", "wd"))
    u, tiny = U[dtype], TINY[dtype]
    G, V = x @ wg.T, x @ wu.T
    eG, eV = d * ACC * (x.abs() @ wg.abs().T), d * ACC * (x.abs() @ wu.abs().T)
    within(gate, G, eG, dtype)
    within(up, V, eV, dtype)
    a, _ = act(kind, G)
    H = a * V
    ea = LIP * eG + FN * (1 + G.abs())
    eH = V.abs() * ea + a.abs() * eV + ea * eV
    eH = eH + u * (H.abs() + eH) + tiny
    eY = eH @ wd.abs().T + f * ACC * ((H.abs() + eH) @ wd.abs().T)
    within(y, H @ wd.T, eY, dtype)
    y2, _, _ = forward(lib, t, kind)     # without G and U: the same result
    assert torch.equal(y, y2)


def check_backward(lib, M, d, f, dtype, kind, shift=0):
    t = make(M, d, f, dtype, M + f, shift)
    got = backward(lib, t, kind)
    x, wg, wu, wd, dy, G, V = (t[k].double() for k in ("x", "wg", "wu", "wd", "dy", "gate", "up"))
    u, tiny = U[dtype], TINY[dtype]
    a, da = act(kind, G)
    dH, H = dy @ wd, a * V
    eF = FN * (1 + G.abs())
    eD = d * ACC * (dy.abs() @ wd.abs())
    dG, dV = dH * V * da, dH * a
    eG = (V * da).abs() * eD + (dH.abs() + eD) * V.abs() * eF
    eG = eG + u * (dG.abs() + eG) + tiny
    eV = a.abs() * eD + (dH.abs() + eD) * eF
    eV = eV + u * (dV.abs() + eV) + tiny
    eH = V.abs() * eF
    eH = eH + u * (H.abs() + eH) + tiny
    aG, aV, aH = dG.abs() + eG, dV.abs() + eV, H.abs() + eH
    within(got[0], dG @ wg + dV @ wu, eG @ wg.abs() + eV @ wu.abs() + 2 * f * ACC * (aG @ wg.abs() + aV @ wu.abs()), dtype)
    within(got[1], dG.T @ x, eG.T @ x.abs() + M * ACC * (aG.T @ x.abs()), dtype)
    within(got[2], dV.T @ x, eV.T @ x.abs() + M * ACC * (aV.T @ x.abs()), dtype)
    within(got[3], dy.T @ H, dy.abs().T @ eH + M * ACC * (dy.abs().T @ aH), dtype)
    assert all(torch.equal(p, q) for p, q in zip(got, backward(lib, t, kind)))
    only = backward(lib, t, kind, (0, 0, 1, 0))
    assert only[0] is None and torch.equal(only[2], got[2])


# tokens, d, f: one token, few tokens, tile edges on every side, odd sizes, both tile shapes (the last three have enough
# tiles for CTA pairs in every launch)
SIZES = [(1, 1, 1), (1, 8, 8), (1, 256, 688), (2, 64, 72), (3, 1001, 77), (5, 96, 1032), (8, 512, 256), (9, 40, 264),
         (16, 1024, 512), (17, 72, 136), (33, 100, 333), (64, 64, 64), (127, 136, 120), (129, 257, 65), (300, 320, 1000),
         (640, 128, 200), (1030, 2880, 1600), (1100, 2567, 1601), (2305, 2048, 1920)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,d,f", SIZES)
def test_forward(lib, M, d, f, dtype):
    check_forward(lib, M, d, f, dtype, "silu")
    assert lib[0].sama_device_status(lib[1]) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,d,f", SIZES)
def test_backward(lib, M, d, f, dtype):
    check_backward(lib, M, d, f, dtype, "silu")
    assert lib[0].sama_device_status(lib[1]) == 0


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("M,d,f,shift", [(1, 128, 256, 0), (7, 65, 130, 0), (200, 192, 328, 0), (40, 128, 256, 3)])
def test_activations_and_odd_addresses(lib, M, d, f, shift, dtype, kind):
    check_forward(lib, M, d, f, dtype, kind, shift)
    check_backward(lib, M, d, f, dtype, kind, shift)


@pytest.mark.parametrize("kind", ACTS)
def test_gradient_is_the_derivative(lib, kind):
    """Central differences, in 64 bits, of <dY, Y> along a random direction of each input."""
    M, d, f = 24, 40, 56
    t = make(M, d, f, "bf16", 9)
    p = {k: t[k].double() for k in ("x", "wg", "wu", "wd")}

    def loss(q):
        return float(((act(kind, q["x"] @ q["wg"].T)[0] * (q["x"] @ q["wu"].T)) @ q["wd"].T * t["dy"].double()).sum())

    _, t["gate"], t["up"] = forward(lib, t, kind, save=True)
    grads = dict(zip(("x", "wg", "wu", "wd"), backward(lib, t, kind)))
    g = torch.Generator(device="cuda").manual_seed(1)
    for k in p:
        v = torch.randn(p[k].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        diff = (loss({**p, k: p[k] + h * v}) - loss({**p, k: p[k] - h * v})) / (2 * h)
        # G and U are rounded, then H, dG and dU, then the result: four roundings of u at most on the way to any element,
        # independent of the direction; their sum over n elements stays below 4 u ||grad|| ||v|| (Cauchy-Schwarz), and the
        # ReLU's kink moves the difference by no more than that
        assert abs(float((grads[k].double() * v).sum()) - diff) <= 4 * U["bf16"] * float(grads[k].double().norm() * v.norm())


@pytest.mark.parametrize("M", [3, 200])
def test_values_that_are_not_finite_stay_in_their_rows(lib, M):
    t = make(M, 64, 96, "bf16", 3)
    clean, _, _ = forward(lib, t, "silu")
    t["x"][1, 5], t["x"][2, 6] = float("nan"), float("inf")
    y, _, _ = forward(lib, t, "silu")
    keep = [i for i in range(M) if i not in (1, 2)]
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[1]).all()) and not bool(torch.isfinite(y[2]).any())


@pytest.mark.parametrize("kind", ACTS)
def test_gates_whose_square_overflows(lib, kind):
    # a' is 1 to the right and 0 to the left of them, exactly, so dG is dH (rounded once) or 0
    M, d, f = 32, 64, 96
    t = make(M, d, f, "bf16", 5)
    t["gate"].copy_(torch.where(t["gate"] > 0, 2.0 ** 100, -2.0 ** 100))
    t["up"].fill_(1.0)
    _, dwg, _, _ = backward(lib, t, kind, want=(0, 1, 0, 0))
    x, wd, dy, G = (t[k].double() for k in ("x", "wd", "dy", "gate"))
    dH, eH = dy @ wd, d * ACC * (dy.abs() @ wd.abs())
    on = (G > 0).double()
    dG, eG = dH * on, (eH + U["bf16"] * (dH.abs() + eH)) * on
    err = eG.T @ x.abs() + M * ACC * ((dG.abs() + eG).T @ x.abs())
    within(dwg, dG.T @ x, err, "bf16")


def test_no_tokens(lib):
    S, ctx = lib
    t = make(4, 16, 24, "bf16")
    dw = [torch.full_like(t[k], 3.0) for k in ("wg", "wu", "wd")]
    S.sama_gated_ffn(ctx, S.SAMA_BF16, 0, 0, 16, 24, None, t["wg"], t["wu"], t["wd"], None)
    S.sama_gated_ffn_grad(ctx, S.SAMA_BF16, 0, 0, 16, 24, None, t["wg"], t["wu"], t["wd"], None, None, None, None, *dw)
    assert not any(bool(w.any()) for w in dw)


def test_runs_on_the_callers_stream(lib):
    t = make(256, 256, 512, "bf16", 5)
    ref, _, _ = forward(lib, t, "silu")
    x = t["x"].clone()
    s = torch.cuda.Stream()
    t["x"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        for _ in range(10):
            t["x"].add_(0.0)
        t["x"].copy_(x)
        y, _, _ = forward(lib, t, "silu")
        y = y.clone()
    s.synchronize()
    assert torch.equal(y, ref)


def test_refusals(lib):
    S, ctx = lib
    t = make(4, 16, 24, "bf16")
    y = torch.empty_like(t["x"])
    g = torch.empty_like(t["gate"])

    def status(f, *args):
        with pytest.raises(S.SamaError) as e:
            f(*args)
        return e.value.status

    w = [t["wg"], t["wu"], t["wd"]]
    f = S.sama_gated_ffn
    assert status(f, None, 1, 0, 4, 16, 24, t["x"], *w, y) == S.SAMA_ERR_NULL
    assert status(f, ctx, 1, 0, 4, 16, 24, None, *w, y) == S.SAMA_ERR_NULL
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"], *w, None) == S.SAMA_ERR_NULL
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"], *w, y, g) == S.SAMA_ERR_NULL              # G without U
    assert status(f, ctx, 0, 0, 4, 16, 24, *[v.data_ptr() for v in [t["x"], *w, y]]) == S.SAMA_ERR_PARAM
    assert status(f, ctx, 2, 0, 4, 16, 24, t["x"], *w, y) == S.SAMA_ERR_PARAM                # tensors are bf16
    assert status(f, ctx, 1, 4, 4, 16, 24, t["x"], *w, y) == S.SAMA_ERR_PARAM
    assert status(f, ctx, 1, 0, -1, 16, 24, t["x"], *w, y) == S.SAMA_ERR_SIZE
    assert status(f, ctx, 1, 0, 4, 0, 24, t["x"], *w, y) == S.SAMA_ERR_SIZE
    assert status(f, ctx, 1, 0, 4, 16, (1 << 20) + 1, *[v.data_ptr() for v in [t["x"], *w, y]]) == S.SAMA_ERR_SIZE
    assert status(f, ctx, 1, 0, 5, 16, 24, t["x"], *w, y) == S.SAMA_ERR_SIZE                 # x is too small
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"].data_ptr() + 1, *w, y) == S.SAMA_ERR_ALIGN
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"], *w, t["x"]) == S.SAMA_ERR_OVERLAP
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"], *w, y, g, g) == S.SAMA_ERR_OVERLAP
    assert status(f, ctx, 1, 0, 4, 16, 24, t["x"].t().contiguous().t(), *w, y) == S.SAMA_ERR_PARAM
    b = S.sama_gated_ffn_grad
    dw = [torch.empty_like(v) for v in w]
    a = [t["gate"], t["up"], t["dy"]]
    assert status(b, ctx, 1, 0, 4, 16, 24, t["x"], *w, None, t["up"], t["dy"], y, *dw) == S.SAMA_ERR_NULL
    assert status(b, ctx, 1, 0, 4, 16, 24, t["x"], *w, *a, t["dy"], *dw) == S.SAMA_ERR_OVERLAP
    assert status(b, ctx, 1, 0, 4, 16, 24, t["x"], *w, *a, y, dw[0], dw[0], dw[2]) == S.SAMA_ERR_OVERLAP
    assert S.sama_device_status(ctx) == 0
