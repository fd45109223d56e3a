"""Data reweighting on a small text classifier, the setting of Sec. 4.1 with a token encoder in front of the head.

    tokens -> embedding -> x + gated feed-forward(x) -> mean over the text -> MLP head -> classes

The encoder is bf16 (sama_embed, sama_gated_ffn and their gradients), its master weights and the head are fp32.  Every
step: the base loss weights each text by sigmoid(lambda_i); the gradients of all tensors are clipped by their global norm
into one flat fp32 vector (sama_clip_grads), which Adam applies; then SAMA's meta gradient (sama_meta_grad on a clean
batch, sama_step on the base batch, both on the head's features) moves lambda, so that texts
with wrong labels lose weight.

    python examples/text_reweight.py --steps 200
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2310_05674_b200 import binding as S  # noqa: E402

VOCAB, D, F, HIDDEN, CLASSES, BATCH, LENGTH, TEXTS = 2003, 128, 344, 64, 4, 256, 24, 4096
PAD = 0


def texts(n, noise, seed):
    """Token ids [n][LENGTH] (padded at the end), clean labels, and labels of which a share `noise` is wrong."""
    g = torch.Generator().manual_seed(seed)
    y = torch.randint(CLASSES, (n,), generator=g)
    topic = 1 + (y[:, None] * 60 + torch.randint(60, (n, LENGTH), generator=g))       # a class's own words
    common = 1 + 60 * CLASSES + (torch.rand(n, LENGTH, generator=g) ** 3 * (VOCAB - 2 - 60 * CLASSES)).long()
    ids = torch.where(torch.rand(n, LENGTH, generator=g) < 0.25, topic, common)
    ids[torch.arange(LENGTH)[None, :] >= torch.randint(LENGTH // 2, LENGTH + 1, (n, 1), generator=g)] = PAD
    flip = torch.rand(n, generator=g) < noise
    wrong = (y + 1 + torch.randint(CLASSES - 1, (n,), generator=g)) % CLASSES
    return ids.to(torch.int32).cuda(), y.to(torch.int32).cuda(), torch.where(flip, wrong, y).to(torch.int32).cuda()


class Encoder:
    """Parameters and buffers of the encoder for BATCH texts."""

    SHAPES = {"table": (VOCAB, D), "wg": (F, D), "wu": (F, D), "wd": (D, F)}

    def __init__(self, ctx, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ctx, self.n = ctx, BATCH * LENGTH
        std = {"table": 1.0, "wg": D ** -0.5, "wu": D ** -0.5, "wd": F ** -0.5}
        self.sizes = [torch.Size(s).numel() for s in self.SHAPES.values()]
        self.master = torch.cat([std[k] * torch.randn(n, generator=g, device="cuda") for k, n in zip(self.SHAPES, self.sizes)])
        bf = lambda *s: torch.empty(*s, dtype=torch.bfloat16, device="cuda")  # noqa: E731
        self.w = {k: bf(*s) for k, s in self.SHAPES.items()}
        self.grad = {k: bf(*s) for k, s in self.SHAPES.items()}
        self.x, self.y, self.dx = (bf(self.n, D) for _ in range(3))
        self.gate, self.up = bf(self.n, F), bf(self.n, F)
        self.load()

    def load(self):
        """bf16 copies of the master weights."""
        for w, part in zip(self.w.values(), self.master.split(self.sizes)):
            w.copy_(part.view(w.shape))

    def features(self, ids):
        """fp32 [BATCH][D]: mean over each text's tokens of x + ffn(x)."""
        S.sama_embed(self.ctx, S.SAMA_BF16, self.n, VOCAB, D, self.w["table"], ids, 1.0, self.x)
        S.sama_gated_ffn(self.ctx, S.SAMA_BF16, S.SAMA_ACT_SILU, self.n, D, F, self.x, self.w["wg"], self.w["wu"],
                         self.w["wd"], self.y, self.gate, self.up)
        self.mask = (ids != PAD).float().unsqueeze(-1)
        self.count = self.mask.sum(1)
        h = (self.x.float() + self.y.float()).view(BATCH, LENGTH, D)
        return (h * self.mask).sum(1) / self.count

    def backward(self, ids, dfeat):
        """Fills self.grad from the gradient of the features of the last call."""
        dh = (self.mask * (dfeat / self.count).unsqueeze(1)).reshape(self.n, D).bfloat16()
        S.sama_gated_ffn_grad(self.ctx, S.SAMA_BF16, S.SAMA_ACT_SILU, self.n, D, F, self.x, self.w["wg"], self.w["wu"],
                              self.w["wd"], self.gate, self.up, dh, self.dx, self.grad["wg"], self.grad["wu"], self.grad["wd"])
        self.dx += dh                                          # the residual path
        S.sama_embed_grad(self.ctx, S.SAMA_BF16, self.n, VOCAB, D, ids, self.dx, 1.0, PAD, S.SAMA_BF16, 0, self.grad["table"])


def head_gradients(theta, X, y, weight):
    """Mean weighted cross-entropy of the two-layer head, its gradients with respect to X and to the flat theta."""
    w1, b1, w2, b2 = theta.split([HIDDEN * D, HIDDEN, CLASSES * HIDDEN, CLASSES])
    w1, w2 = w1.view(HIDDEN, D), w2.view(CLASSES, HIDDEN)
    z1 = X @ w1.T + b1
    a1 = z1.clamp(min=0)
    z2 = a1 @ w2.T + b2
    logp = z2 - z2.logsumexp(1, keepdim=True)
    pick = torch.nn.functional.one_hot(y.long(), CLASSES).float()
    loss = -(weight * (logp * pick).sum(1)).mean()
    dz2 = weight[:, None] * (logp.exp() - pick) / len(X)
    dz1 = (dz2 @ w2) * (z1 > 0)
    return loss, dz1 @ w1, torch.cat([(dz1.T @ X).flatten(), dz1.sum(0), (dz2.T @ a1).flatten(), dz2.sum(0)])


def train(steps=200, noise=0.4, max_norm=0.25, lr=3e-4, meta_lr=0.3, log=print):
    mlp = S.MLP((D, HIDDEN, CLASSES))
    n_head = S.sama_mlp_param_count(mlp)
    ctx = S.sama_create(0, n_head, BATCH, mlp)
    enc = Encoder(ctx)
    g = torch.Generator(device="cuda").manual_seed(1)
    theta = 0.1 * torch.randn(n_head, generator=g, device="cuda")
    all_ids, clean, noisy = texts(TEXTS, noise, 1)
    meta_ids, meta_clean, _ = texts(TEXTS // 4, 0.0, 2)
    lam = torch.zeros(TEXTS, device="cuda")

    # one flat fp32 gradient: the encoder's tensors, then the head's vector
    n_enc = enc.master.numel()
    flat = torch.empty(n_enc + n_head, device="cuda")
    g_head, g_meta, p = (torch.empty(n_head, device="cuda") for _ in range(3))
    tensors = S.TensorList([*enc.grad.values(), g_head], flat.split([*enc.sizes, n_head]))
    norm, metagrad = torch.empty(1, device="cuda"), torch.empty(BATCH, device="cuda")
    m, v = torch.zeros_like(flat), torch.zeros_like(flat)
    loss = None
    for t in range(1, steps + 1):
        at = torch.arange(BATCH, device="cuda") + (t - 1) * BATCH % TEXTS
        ids, y, weight_logits = all_ids[at], noisy[at], lam[at]
        X = enc.features(ids)
        loss, dX, gh = head_gradients(theta, X, y, torch.sigmoid(weight_logits))
        enc.backward(ids, dX)
        g_head.copy_(gh)
        S.sama_clip_grads(ctx, tensors, max_norm, norm)
        # the meta step, with the moments before this update; lambda moves by a fixed length on average
        mat = torch.arange(BATCH, device="cuda") + (t - 1) * BATCH % len(meta_ids)
        S.sama_meta_grad(ctx, mlp, theta, enc.features(meta_ids[mat]), meta_clean[mat], BATCH, g_meta)
        S.sama_step(ctx, mlp, n_head, theta, m[n_enc:].clone(), v[n_enc:].clone(), flat[n_enc:].clone(), g_meta,
                    S.Adam(lr=lr, step=t), 1.0, X, y, weight_logits, BATCH, p, None, None, metagrad)
        lam[at] -= meta_lr * metagrad / (metagrad.abs().mean() + 1e-30)
        m.mul_(0.9).add_(flat, alpha=0.1)
        v.mul_(0.999).addcmul_(flat, flat, value=0.001)
        update = lr * (m / (1 - 0.9 ** t)) / ((v / (1 - 0.999 ** t)).sqrt() + 1e-8)
        enc.master -= update[:n_enc]
        theta -= update[n_enc:]
        enc.load()
        if log and t % 25 == 0:
            w = torch.sigmoid(lam)
            log("step %4d  loss %.4f  gradient norm %.3f  mean weight: right labels %.3f, wrong labels %.3f"
                % (t, float(loss), float(norm), float(w[noisy == clean].mean()), float(w[noisy != clean].mean())))
    w = torch.sigmoid(lam)
    status = S.sama_device_status(ctx)
    S.sama_destroy(ctx)
    return {"loss": float(loss), "weight_right": float(w[noisy == clean].mean()),
            "weight_wrong": float(w[noisy != clean].mean()), "status": status}


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    a.add_argument("--steps", type=int, default=200)
    train(a.parse_args().steps)
