"""A pruned layer repaired without touching its kept weights: its layer norm and one low-rank adapter for each of several tasks are trained by AdamW, and the adapters are
served together beside the layer's 8-bit projection, every row of a batch with its own.

    python examples/repair_serve_adapters.py [--tokens 65536] [--d 128] [--f 192] [--tasks 4] [--rank 8] [--vocab 500] [--steps 200] [--bits 8]

The model is y = x + (silu(n Wg) * (n Wu)) Wd with n the layer norm of x, logits = y E; random weights, of which all but the norm's are frozen.  Each task answers with
a model of its own, whose Wd differs by a product of low rank.  Every step of the layer runs through the library; torch multiplies by Wd and E where it is trained."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2403_12983_amd as osscar  # noqa: E402


def make(tokens, d, f, tasks, rank, vocab, device):
    g = torch.Generator(device=device)
    g.manual_seed(0)

    def normal(*shape, scale):
        return (torch.randn(*shape, generator=g, device=device) * scale).to(torch.bfloat16)
    model = dict(w=torch.ones(d, device=device), b=torch.zeros(d, device=device), Wg=normal(d, f, scale=1 / math.sqrt(d)), Wu=normal(d, f, scale=1 / math.sqrt(d)),
                 Wd=normal(f, d, scale=1 / math.sqrt(f)), E=normal(d, vocab, scale=2 / math.sqrt(d)))
    X = normal(tokens, d, scale=1.0)
    index = torch.sort(torch.randint(0, tasks, (tokens,), generator=g, device=device)).values
    tutor = normal(tasks, rank, f, scale=1 / math.sqrt(f)), normal(tasks, rank, d, scale=1.0)
    targets = torch.multinomial(torch.softmax(forward(model, X, *tutor, index)["logits"].float(), 1), 1, generator=g)[:, 0]
    A, B = normal(tasks, rank, f, scale=1 / math.sqrt(f)), torch.zeros(tasks, rank, d, dtype=torch.bfloat16, device=device)
    return model, X, index, targets, A, B, g


def forward(model, X, A, B, index):
    """What each step leaves for the way back."""
    s = {}
    s["n"], s["stats"] = osscar.osscar_layernorm_forward(X, model["w"], model["b"], save=True)
    s["H"], s["G"], s["U"] = osscar.osscar_gated_forward(s["n"], model["Wg"], model["Wu"], save=True)
    y = X + s["H"] @ model["Wd"]
    s["y"], s["T"] = osscar.osscar_adapters_forward(s["H"], A, B, index=index, base=y, out=y, save=True)
    s["logits"] = s["y"] @ model["E"]
    return s


def gradients(model, X, A, B, index, targets):
    """(mean of -log p, gradients of the norm's gain and offset, of A and of B)"""
    s = forward(model, X, A, B, index)
    got = osscar.osscar_logprobs(s["logits"], targets)
    dlogits = osscar.osscar_logprobs_backward(s["logits"], targets, got.lse, torch.full_like(got.logp, -1.0 / X.shape[0]))
    dy = dlogits @ model["E"].t()
    dH = dy @ model["Wd"].t()
    dH, dA, dB = osscar.osscar_adapters_backward(s["H"], A, B, dy, T=s["T"], index=index, base=dH, out=dH)
    dn, _, _ = osscar.osscar_gated_backward(s["n"], model["Wg"], model["Wu"], dH, G=s["G"], U=s["U"], need_w=False)
    _, dw, db = osscar.osscar_layernorm_backward(X, model["w"], dn, s["stats"], need_x=False)
    return -got.logp.mean(), dw, db, dA, dB


def serve(model, X, A, B, index, rows):
    """Log probabilities are taken of these: a few rows at a time, the projection in 8 bits, any row any adapter."""
    Wq, w_scale = osscar.osscar_int_weights(model["Wd"])
    out = []
    for x, e in zip(X.split(rows), index.split(rows)):
        H = osscar.osscar_gated_forward(osscar.osscar_layernorm_forward(x, model["w"], model["b"]), model["Wg"], model["Wu"])
        y = x + osscar.osscar_int_product(H, Wq, w_scale)
        out.append(osscar.osscar_adapters_forward(H, A, B, index=e.contiguous(), base=y, out=y) @ model["E"])
    return torch.cat(out)


def run(tokens=65536, d=128, f=192, tasks=4, rank=8, vocab=500, steps=200, rate=2e-3, bits=8, device="cuda:0"):
    model, X, index, targets, A, B, g = make(tokens, d, f, tasks, rank, vocab, device)
    held = torch.rand(tokens, generator=g, device=device) < 0.25
    train = ~held
    losses = []
    plan = osscar.AdamW([model["w"], model["b"], A, B], bits=bits, masters=[None, None, A.float(), B.float()])
    for t in range(1, steps + 1):
        loss, *grads = gradients(model, X[train], A, B, index[train], targets[train])
        plan.osscar_adamw(rate, t, weight_decay=0.0, grads=grads, seed=t)
        losses.append(loss)
    order = torch.randperm(int(held.sum()), generator=g, device=device)      # requests of all tasks, mixed
    Xh, eh, th = X[held][order], index[held][order], targets[held][order]
    logits = serve(model, Xh, A, B, eh, 16)
    none = serve(model, Xh, A, B, torch.full_like(eh, -1), 1024)

    def perplexity(z):
        return math.exp(-osscar.osscar_logprobs(z, th).logp.double().mean().item())
    return dict(first=math.exp(losses[0].item()), last=math.exp(losses[-1].item()), served=perplexity(logits), without=perplexity(none))


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("tokens", 65536), ("d", 128), ("f", 192), ("tasks", 4), ("rank", 8), ("vocab", 500), ("steps", 200), ("bits", 8)):
        ap.add_argument("--" + name, type=int, default=value)
    got = run(**vars(ap.parse_args()))
    print("perplexity of the trained tokens {first:.2f} -> {last:.2f}; of others, served in 8 bits: {served:.2f} with the adapters, {without:.2f} without".format(**got))
