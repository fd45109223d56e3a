"""The text example: its gradients against automatic differentiation in 64 bits, and what its training does.

Tolerance of the gradients: the encoder rounds its activations to bf16 (x, G, U, H, Y, dH, dG, dU, dx: nine roundings of
2^-8 at most on the way to any gradient), so each gradient is within 9 * 2^-8 of the exact one in the 2-norm.
"""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("text_reweight", os.path.join(ROOT, "examples", "text_reweight.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_gradients(ex):
    S = ex.S
    mlp = S.MLP((ex.D, ex.HIDDEN, ex.CLASSES))
    ctx = S.sama_create(0, S.sama_mlp_param_count(mlp), ex.BATCH, mlp)
    enc = ex.Encoder(ctx, 3)
    ids, _, y = ex.texts(ex.BATCH, 0.4, 5)
    theta = 0.2 * torch.randn(S.sama_mlp_param_count(mlp), device="cuda")
    weight = torch.rand(ex.BATCH, device="cuda")
    X = enc.features(ids)
    _, dX, gh = ex.head_gradients(theta, X, y, weight)
    enc.backward(ids, dX)

    w = {k: v.double().requires_grad_() for k, v in enc.w.items()}
    th = theta.double().requires_grad_()
    x = w["table"][ids.long()]
    h = x + (torch.nn.functional.silu(x @ w["wg"].T) * (x @ w["wu"].T)) @ w["wd"].T
    mask = (ids != ex.PAD).double().unsqueeze(-1)
    feat = (h * mask).sum(1) / mask.sum(1)
    loss, _, _ = ex.head_gradients(th, feat, y, weight.double())
    loss.backward()
    feat = feat.detach()
    assert float((X.double() - feat).norm() / feat.norm()) < 3 * 2.0 ** -8
    for k in w:
        assert float((enc.grad[k].double() - w[k].grad).norm() / w[k].grad.norm()) < 9 * 2.0 ** -8, k
    assert float((gh.double() - th.grad).norm() / th.grad.norm()) < 9 * 2.0 ** -8
    assert not bool(enc.grad["table"][ex.PAD].any())
    assert S.sama_device_status(ctx) == 0
    S.sama_destroy(ctx)


def test_training_lowers_the_weight_of_wrong_labels(ex):
    r = ex.train(steps=100, log=None)
    assert r["status"] == 0
    assert r["loss"] < 0.7 * 0.5 * math.log(ex.CLASSES)    # 0.7 of an untrained model's loss at weights of one half
    assert r["weight_wrong"] < r["weight_right"] - 0.1
