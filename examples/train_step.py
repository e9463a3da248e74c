"""A parameter server's training loop: the round, then the end of the step over the model's tensors.

    python examples/train_step.py

Seven workers, two of them adversaries that return reversed gradients, hold the 35 files of the
subset assignment (r = 3).  Every round the server finds the honest clique and aggregates the files' gradients
into one flat vector (aspis_round).  Cut into the model's tensors, that vector is what AdamW steps on:
the tensors' addresses are whatever their lengths make them, the global norm is taken over
all of them (aspis_grad_norm, with every layer's own for the log), and gradients above the bound are clipped
inside the update (aspis_adamw), with fp32 master weights beside the bf16 ones that a server would hand out.
At the end the last gradients are clipped for the record, too (aspis_clip_grads)."""
from __future__ import annotations

import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2108_02416_gb300 as ap  # noqa: E402

K, R, ADVERSARIES = 7, 3, (0, 1)
LAYERS = [(33, 19), (33,), (33, 33), (33,), (1, 33), (1,)]          # odd sizes on purpose
LR, DECAY, MAX_NORM, BATCH = 1e-2, 0.01, 1.0, 64


def cut(flat):
    """The model's tensors as views of a flat vector."""
    out, at = [], 0
    for shape in LAYERS:
        n = torch.Size(shape).numel()
        out.append(flat[at: at + n].view(shape))
        at += n
    return out


def forward(w, x):
    h = torch.tanh(x @ w[0].T + w[1])
    h = torch.tanh(h @ w[2].T + w[3])
    return h @ w[4].T + w[5]


def gradient(masters, x, y):
    w = [t.detach().requires_grad_() for t in masters]
    loss = (forward(w, x) - y).square().mean()
    loss.backward()
    return loss.detach(), torch.cat([t.grad.reshape(-1) for t in w])


def train(steps=200, quiet=False, device="cuda:0"):
    dev = torch.device(device)
    gen = torch.Generator(dev).manual_seed(0)
    d = sum(torch.Size(s).numel() for s in LAYERS)
    a = ap.aspis_assign(K, R)
    workers = a.file_workers()

    # what a server keeps: the round's buffers, the weights with their moments, and the two lists
    buf, norms = ap.RoundBuffers(a, d, dev), ap.NormBuffers(dev)
    masters = [torch.randn(s, device=dev, generator=gen) / max(1, s[-1]) ** 0.5 for s in LAYERS]
    weights = [w.bfloat16() for w in masters]
    m, v = ([torch.zeros_like(w) for w in masters] for _ in range(2))
    grads = cut(buf.out)
    layer_norms = torch.zeros(len(LAYERS), device=dev)
    glist = ap.TensorList(grads)
    plist = ap.ParamList(weights, grads, m, v, masters=masters,
                         weight_decay=[DECAY if w.dim() > 1 else 0.0 for w in masters])

    target = [torch.randn(s, device=dev, generator=gen) / max(1, s[-1]) ** 0.5 for s in LAYERS]
    copies = torch.zeros((a.f, R, (d + 31) // 32 * 32), device=dev)
    history = []
    for step in range(1, steps + 1):
        loss = 0.0
        for i in range(a.f):                             # the workers: every file's gradient, r times
            x = torch.randn(BATCH, LAYERS[0][1], device=dev, generator=gen)
            one, g = gradient(masters, x, forward(target, x))
            loss += float(one) / a.f
            for s, worker in enumerate(workers[i]):
                copies[i, s, :d] = -10.0 * g if worker in ADVERSARIES else g
        # the server
        ap.aspis_round(copies, d, a, buf.file_neq, buf.adj, buf.det, buf.sel, buf.out)
        ap.aspis_grad_norm(glist, norms.norm, norms.work, tensor_norms=layer_norms)
        ap.aspis_adamw(plist, step, LR, (0.9, 0.95), max_norm=MAX_NORM, norm=norms.norm, skip_nonfinite=True)
        history.append({"loss": loss, "norm": float(norms.norm), "layers": layer_norms.tolist(),
                        "clique": buf.detection().omega})
        if not quiet and (step % 20 == 0 or step == 1):
            h = history[-1]
            print(f"step {step:4d}  loss {h['loss']:.4f}  norm {h['norm']:.3f}"
                  f"{' (clipped)' if h['norm'] > MAX_NORM else ''}  honest clique of {h['clique']}")
    clipped = [torch.empty_like(w) for w in weights]     # bf16, as they would be logged
    ap.aspis_clip_grads(ap.TensorList(grads, clipped), MAX_NORM, norms.norm, norms.work)
    if not quiet:
        total = sum(float(c.float().square().sum()) for c in clipped) ** 0.5
        print(f"last gradients: norm {float(norms.norm):.4f}, after clipping {total:.4f}")
    return history


if __name__ == "__main__":
    train()
