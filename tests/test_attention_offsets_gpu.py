"""Gradients of attention whose keys and values have a common offset, against the definition in 64 bits, as a whole.

dQ = scale dX K does not grow with an offset of K (the rows of dX sum to nothing where scores are not capped) nor of V, but what
it is made from does.  Bound: each dX_ij is rounded once, by u of itself at most, and meets K_j; each element of dQ is rounded once.
These are independent of one another, so that the square of the error's norm is at most
  sum over i, j of (u scale dX_ij)^2 |K_j|^2  +  u^2 |dQ|^2,
with dX as it is formed before what out's rounding does to it is put right: with d_out . out of the stored out.  (A rounding is
off by u over the root of 3 or less on average: that leaves as much again for the products' own sums.)  Likewise dK and dV, with
the sums over a key's queries."""
import math

import pytest
import torch

import attention_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lib():
    from paper_2310_05674_b200 import binding
    ctx = binding.sama_create(0, 1024, 0, None)
    yield binding, ctx
    torch.cuda.synchronize()
    binding.sama_destroy(ctx)


def run(lib, lens, heads, kv, dim, dtype, causal, cap, bias, k_offset, v_offset, dout_size=1.0, seed=0):
    S, ctx = lib
    g = torch.Generator(device="cuda").manual_seed(seed)
    n, dt = sum(lens), ref.DT[dtype]
    at = [0]
    for x in lens:
        at.append(at[-1] + x)
    r = lambda h, size, offset: (size * torch.randn(n, h, dim, generator=g, device="cuda") + offset).to(dt)  # noqa: E731
    q, k, v, dout = r(heads, 2.0, 0.0), r(kv, 1.0, k_offset), r(kv, 1.0, v_offset), r(heads, dout_size, 0.0)
    slopes = 0.5 ** torch.arange(1, heads + 1, device="cuda", dtype=torch.float32) if bias else None
    starts = torch.tensor(at, dtype=torch.int32, device="cuda")
    a = S.Attn(S.DTYPES[dtype], heads, kv, dim, n, n, starts, causal=causal, slopes=slopes, cap=cap)
    out, lse = torch.empty_like(q), torch.empty(heads, n, device="cuda")
    grads = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)]
    S.sama_attention(ctx, a, q, k, v, out, lse)
    S.sama_attention_grad(ctx, a, q, k, v, out, lse, dout, *grads)
    u, scale, group = ref.U[dtype], dim ** -0.5, heads // kv
    wrong, allowed, size = [0.0] * 3, [0.0] * 3, [0.0] * 3
    for lo, hi in zip(at, at[1:]):
        Q, K, V, D, O = (x[lo:hi].double() for x in (q, k, v, dout, out))
        K, V = K.repeat_interleave(group, 1), V.repeat_interleave(group, 1)
        raw, x, _ = ref.scores(Q, K, scale, cap, slopes, 0)
        p = torch.softmax(torch.where(ref.visible(hi - lo, hi - lo, causal, 0, "cuda"), x, -math.inf), -1)
        slack = 1 - torch.tanh(raw / cap) ** 2 if cap else 1.0
        dp = torch.einsum("ihd,jhd->hij", D, V)
        exact, stored = ((D * o).sum(-1).T[..., None] for o in (torch.einsum("hij,jhd->ihd", p, V), O))
        dx, formed = p * (dp - exact) * slack, p * (dp - stored) * slack
        shared = lambda t: t.view(hi - lo, kv, group, dim).sum(2)  # noqa: E731
        want = [scale * torch.einsum("hij,jhd->ihd", dx, K), shared(scale * torch.einsum("hij,ihd->jhd", dx, Q)),
                shared(torch.einsum("hij,ihd->jhd", p, D))]
        k2, q2, d2 = ((t * t).sum(-1) for t in (K, Q, D))
        rounded = [torch.einsum("hij,jh->", (scale * formed) ** 2, k2), torch.einsum("hij,ih->", (scale * dx) ** 2, q2),
                   torch.einsum("hij,ih->", p ** 2, d2)]
        for i, (w, e, got) in enumerate(zip(want, rounded, grads)):
            wrong[i] += float((got[lo:hi].double() - w).square().sum())
            size[i] += float(w.square().sum())
            allowed[i] += u * u * (float(e) + float(w.square().sum()))
    return [math.sqrt(x) for x in wrong], [math.sqrt(x) for x in allowed], [math.sqrt(x) for x in size]


@pytest.mark.parametrize("k_offset,v_offset", [(0.0, 0.0), (1.0, 1.0), (3.0, 1.0), (0.0, 4.0), (4.0, 4.0)])
@pytest.mark.parametrize("dim,lens", [(64, [512]), (64, [1500]), (40, [300, 77, 401]), (128, [700, 5, 383]), (96, [2100])])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_offsets(lib, k_offset, v_offset, dim, lens, dtype):
    for causal, cap, bias in ((False, 0.0, False), (True, 5.0, False), (True, 0.0, True)):
        wrong, allowed, size = run(lib, lens, 4, 2, dim, dtype, causal, cap, bias, k_offset, v_offset, seed=dim)
        for name, a, b, c in zip(("dq", "dk", "dv"), wrong, allowed, size):
            assert a <= b, (name, causal, cap, a / c, b / c)
