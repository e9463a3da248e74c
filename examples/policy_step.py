"""A round of policy training: workers that compute a language model's gradient bit for bit alike.

    python examples/policy_step.py

Seven workers, two of them adversaries, hold the 35 files of the subset assignment (r = 3).  A file
is a batch of tokens with the actions taken after them and their advantages.  Each of a file's three
workers computes the gradient by itself: the embedding of the tokens (aspis_embed), a layer behind a residual
connection with dropout (aspis_dropout), logits, the clipped policy loss with a KL term down to the logits'
gradient (aspis_policy_loss; log-probabilities before the step by aspis_token_logp), and the embedding's gradient
(aspis_embed_grad), written straight into the row of copies that the server gets.  Masks are functions of the file and the
step, and sums have a fixed order, so honest copies agree in every bit: aspis_round finds the adversaries, and AdamW
steps on the aggregate.  (The order of a row's sum depends on the row's address modulo 32: logits are tensors of their own here, so every
worker's begin at such a boundary.)"""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2108_02416_gb300 as ap  # noqa: E402

K, R, ADVERSARIES = 7, 3, (2, 5)
V, D, T = 203, 24, 96                                    # vocabulary, width, tokens of a file
SHAPES = [(V, D), (D, D), (V, D)]                        # embedding, layer, head
P, SCALE, CLIP, KL, SEED = 0.1, D ** 0.5, (0.2, 0.28), 0.05, 20_240_229


def cut(flat):
    """The model's tensors as views of a flat vector."""
    out, at = [], 0
    for shape in SHAPES:
        n = torch.Size(shape).numel()
        out.append(flat[at: at + n].view(shape))
        at += n
    return out


class Worker:
    """What a worker keeps: its buffers."""

    def __init__(self, device):
        self.h, self.x, self.du = (torch.empty(T, D, device=device) for _ in range(3))
        self.embed, self.policy = ap.EmbedBuffers(T, V, D, device), ap.PolicyBuffers(T, device)

    def logits(self, w, tokens, drops=(None, None)):
        ap.aspis_embed(w[0], tokens, self.h, scale=SCALE, drop=drops[0])
        u = torch.tanh(self.h @ w[1])
        ap.aspis_dropout(u, self.x, drops[1] or ap.Drop(0.0, 0), residual=self.h)
        return u, self.x @ w[2].T

    def logp(self, w, batch):
        """Log-probabilities of the actions, without dropout."""
        out = torch.empty(T, device=self.x.device)
        ap.aspis_token_logp(self.logits(w, batch["tokens"])[1], batch["actions"], out)
        return out

    def gradient(self, w, batch, drops, out):
        """The gradient of a file's loss into ``out`` (views as of :func:`cut`); the loss and its terms."""
        u, z = self.logits(w, batch["tokens"], drops)
        ap.aspis_policy_loss(z, batch["actions"], batch["old"], batch["advantages"], self.policy.sums, self.policy.work,
                             grad=z, ref_logp=batch["ref"], weights=batch["weights"], clip=CLIP, kl_coef=KL, scale=1 / T)
        torch.mm(z.T, self.x, out=out[2])
        dx = z @ w[2]
        ap.aspis_dropout(dx, self.du, drops[1])
        da = self.du * (1 - u * u)
        torch.mm(self.h.T, da, out=out[1])
        ap.aspis_embed_grad(dx + da @ w[1].T, batch["tokens"], out[0], self.embed.work, scale=SCALE, drop=drops[0])
        return self.policy.sums


def drops_of(file, step):
    """A file's masks: the same on each of its workers."""
    return [ap.Drop(P, SEED, stream=(step * 1000 + file) * 2 + layer) for layer in range(2)]


def make_batch(gen, dev):
    """Tokens, some of them padding; what came out of them is good where it equals the token's half."""
    tokens = torch.randint(0, V, (T,), device=dev, generator=gen)
    actions = torch.randint(0, V, (T,), device=dev, generator=gen)
    actions[::3] = tokens[::3] // 2
    tokens[5::17], actions[5::17] = -1, -1
    return {"tokens": tokens, "actions": actions, "advantages": torch.where(actions == tokens // 2, 1.0, -0.2),
            "weights": (torch.arange(T, device=dev) % 8 != 7).float()}


def train(steps=30, quiet=False, device="cuda:0"):
    dev = torch.device(device)
    gen = torch.Generator(dev).manual_seed(0)
    d = sum(torch.Size(s).numel() for s in SHAPES)
    a = ap.aspis_assign(K, R)
    holders = a.file_workers()
    workers = [Worker(dev) for _ in range(K)]
    buf, norms = ap.RoundBuffers(a, d, dev), ap.NormBuffers(dev)
    weights = [torch.randn(s, device=dev, generator=gen) * s[-1] ** -0.5 for s in SHAPES]
    first = [w.clone() for w in weights]                 # the reference policy
    m, v = ([torch.zeros_like(w) for w in weights] for _ in range(2))
    grads = cut(buf.out)
    plist = ap.ParamList(weights, grads, m, v)
    copies = torch.zeros((a.f, R, (d + 31) // 32 * 32), device=dev)
    history = []
    for step in range(1, steps + 1):
        loss = torch.zeros(4, device=dev)
        for i in range(a.f):
            batch = make_batch(gen, dev)
            batch["old"], batch["ref"] = workers[0].logp(weights, batch), workers[0].logp(first, batch)
            for s, k in enumerate(holders[i]):
                row = copies[i, s, :d]
                sums = workers[k].gradient(weights, batch, drops_of(i, step), cut(row))
                if k in ADVERSARIES:
                    row.mul_(-10.0)
            loss += sums / a.f
        ap.aspis_round(copies, d, a, buf.file_neq, buf.adj, buf.det, buf.sel, buf.out)
        ap.aspis_adamw(plist, step, 1e-2, max_norm=1.0, norm=norms.norm, work=norms.work)
        det = buf.detection()
        history.append({"sums": loss.tolist(), "norm": float(norms.norm), "clique": det.clique_mask, "weights": weights})
        if not quiet:
            s = history[-1]["sums"]
            print(f"step {step:3d}  loss {s[0]:+.4f}  policy {s[1]:+.4f}  KL {s[2]:.4f}  clipped {s[3]:.3f}  "
                  f"norm {history[-1]['norm']:.3f}  honest clique {det.clique_mask:#x}")
    return history


if __name__ == "__main__":
    train()
