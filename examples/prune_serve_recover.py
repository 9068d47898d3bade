"""One gated feed-forward layer of a language model, from calibration to serving: prune it, narrow it, serve it in 8-bit integers, measure it by the
perplexity of its answers, and, for comparison, train the same kept neurons without the refit.

    python examples/prune_serve_recover.py [--tokens 32768] [--d 256] [--f 1024] [--keep 384] [--vocab 4000]

The model is a layer between an embedding and a vocabulary, y = x + (act(x Wg) * (x Wu)) Wd, logits = y E, with random weights; the tokens to be
predicted are drawn from the dense layer's own answers, so that its perplexity is the best there is.  Every step of the layer runs through the
library; torch multiplies by Wd and E where a float layer is trained."""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2403_12983_amd as osscar  # noqa: E402


def make(tokens, d, f, vocab, device):
    g = torch.Generator(device=device)
    g.manual_seed(0)

    def normal(*shape, scale):
        return torch.randn(*shape, generator=g, device=device) * scale
    r = max(4, d // 16)
    mix = normal(r, d, scale=1 / math.sqrt(r))      # hidden states live near a few of the dimensions
    X = (normal(tokens, r, scale=1.0) @ mix + normal(tokens, d, scale=0.02)).to(torch.bfloat16)
    Wg, Wu = (normal(d, f, scale=1 / math.sqrt(d)).to(torch.bfloat16) for _ in range(2))
    Wd = normal(f, d, scale=3 / math.sqrt(f)).to(torch.bfloat16)
    head = normal(d, vocab, scale=2 / math.sqrt(d)).to(torch.bfloat16)
    return X, Wg, Wu, Wd, head, g


def logits_of(X, layer, head):
    Wg, Wu, Wd = layer
    return (X + osscar.osscar_gated_forward(X, Wg, Wu) @ Wd) @ head


def perplexity(logits, targets):
    got = osscar.osscar_logprobs(logits, targets, top=1)
    return math.exp(-got.logp.double().mean().item()), (got.top_index[:, 0] == targets).double().mean().item()


def prune(X, layer, keep, swaps):
    """The kept neurons and the refitted rows of Wd, from the activations that enter it."""
    Wg, Wu, Wd = layer
    f, d = Wd.shape
    solver = osscar.Solver(f, d, f, 1, keep, swaps, torch.bfloat16, torch.bfloat16, X.device)
    segments = X.split(2048)
    for k, rows in enumerate(segments):
        H = osscar.osscar_gated_forward(rows, Wg, Wu)
        solver.osscar_gram(H, k + 1 == len(segments), Wd, 0.0, 1e-2)
    before = solver.osscar_init_support()
    found = solver.osscar_local_search(swaps)
    What, support, _ = solver.osscar_backsolve(torch.bfloat16)
    solver.close()
    kept = torch.from_numpy(support).long().to(X.device)
    return (Wg[:, kept].contiguous(), Wu[:, kept].contiguous(), What[kept].contiguous()), kept, before, found


def serve(X, layer, head, rows):
    """Logits of a few tokens at a time with Wd and the head in 8 bits."""
    Wg, Wu, Wd = layer
    Wq, w_scale = osscar.osscar_int_weights(Wd)
    Eq, e_scale = osscar.osscar_int_weights(head)
    out = []
    for x in X.split(rows):
        y = x + osscar.osscar_int_product(osscar.osscar_gated_forward(x, Wg, Wu), Wq, w_scale)
        out.append(osscar.osscar_int_product(y, Eq, e_scale))
    return torch.cat(out)


def recover(X, targets, layer, head, steps, rate):
    """Gradient steps on the kept neurons' weights, against the tokens' log probability."""
    Wg, Wu, Wd = layer
    masters = [w.float() for w in layer]
    n = X.shape[0]
    for _ in range(steps):
        H, G, U = osscar.osscar_gated_forward(X, Wg, Wu, save=True)
        logits = (X + H @ Wd) @ head
        got = osscar.osscar_logprobs(logits, targets)
        dlogp = torch.full_like(got.logp, -1.0 / n)
        dlogits = osscar.osscar_logprobs_backward(logits, targets, got.lse, dlogp, out=logits)
        dY = dlogits @ head.t()
        dWd = H.t() @ dY
        _, dWg, dWu = osscar.osscar_gated_backward(X, Wg, Wu, dY @ Wd.t(), G=G, U=U, need_x=False, dw_dtype=torch.float32)
        for w, m, dw in zip((Wg, Wu, Wd), masters, (dWg, dWu, dWd.float())):
            m -= rate * dw / (dw.norm() + 1e-12) * m.norm()
            w.copy_(m)
    return Wg, Wu, Wd


def run(tokens=32768, d=256, f=1024, keep=384, vocab=4000, swaps=200, steps=60, rate=0.004, device="cuda:0"):
    X, Wg, Wu, Wd, head, g = make(2 * tokens, d, f, vocab, device)
    dense = (Wg, Wu, Wd)
    logits = logits_of(X, dense, head)
    targets = torch.multinomial(torch.softmax(logits.float(), 1), 1, generator=g)[:, 0]
    train, held = slice(0, tokens), slice(tokens, None)
    result = {"dense": perplexity(logits[held], targets[held])}
    del logits
    pruned, kept, before, found = prune(X[train], dense, keep, swaps)
    result["search"] = (before, found["obj_final"], found["accepted"])
    naive = (Wg[:, kept].contiguous(), Wu[:, kept].contiguous(), Wd[kept].contiguous())
    result["pruned, not refitted"] = perplexity(logits_of(X[held], naive, head), targets[held])
    result["pruned"] = perplexity(logits_of(X[held], pruned, head), targets[held])
    result["pruned, 8 bits"] = perplexity(serve(X[held], pruned, head, 1024), targets[held])
    few = serve(X[held][:4], pruned, head, 1)      # token by token
    result["token by token"] = perplexity(few, targets[held][:4])[0]
    trained = recover(X[train], targets[train], naive, head, steps, rate)
    result["trained, not refitted"] = perplexity(logits_of(X[held], trained, head), targets[held])
    return result


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    for name, value in (("tokens", 32768), ("d", 256), ("f", 1024), ("keep", 384), ("vocab", 4000), ("swaps", 200), ("steps", 60)):
        ap.add_argument("--" + name, type=int, default=value)
    got = run(**vars(ap.parse_args()))
    before, after, accepted = got.pop("search")
    print(f"search: objective {before:.4g} -> {after:.4g} in {accepted} swaps")
    for name, value in got.items():
        print(f"{name:22s} perplexity {value[0]:8.3f}, its first choice right {100 * value[1]:5.1f} %" if isinstance(value, tuple) else f"{name:22s} perplexity {value:8.3f}")
