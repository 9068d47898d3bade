"""The operators that repair a pruned layer, run together: layer norm, gated layer, adapters, log probabilities, their gradients, a step of AdamW; and served in 8 bits."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("repair_serve_adapters", os.path.join(ROOT, "examples", "repair_serve_adapters.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _exact(model, X, A, B, index, targets):
    """Loss and gradients by autograd in float64 on the CPU."""
    m = {k: v.double().cpu() for k, v in model.items()}
    w, b, A, B = (t.double().cpu().requires_grad_() for t in (model["w"], model["b"], A, B))
    x, e = X.double().cpu(), index.cpu()
    c = x - x.mean(1, keepdim=True)
    n = c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * w + b
    g = n @ m["Wg"]
    H = g * torch.sigmoid(g) * (n @ m["Wu"])
    y = x + H @ m["Wd"] + ((A[e] * H[:, None]).sum(2)[:, :, None] * B[e]).sum(1)
    lp = torch.log_softmax(y @ m["E"], 1)
    loss = -lp[torch.arange(len(e)), targets.cpu()].mean()
    loss.backward()
    return loss.item(), w.grad, b.grad, A.grad, B.grad


def test_gradients_of_all_steps_together(ex):
    model, X, index, targets, A, B, g = ex.make(300, 96, 120, 3, 5, 200, DEV)
    B.copy_(torch.randn(B.shape, generator=g, device=DEV) * 0.3)
    model["w"].add_(torch.randn(96, generator=g, device=DEV) * 0.1)
    got = ex.gradients(model, X, A, B, index, targets)
    want = _exact(model, X, A, B, index, targets)
    # The way from X to a gradient rounds to bf16 (2^-8 of each number at most, a random 2^-8 / sqrt 3 of it on average) about ten times: n, H, y before and after the adapters, the logits, and back
    # dlogits, dy, dH, the gated layer's dg and du, dn; each goes on with a gain near one in the 2-norm, but for the logits, whose errors (sizes to about 8, so 8 times 2^-8 / sqrt 3)
    # are those of the probabilities.  In the 2-norm: sqrt(9 + 8^2) 2^-8 / sqrt 3 = 0.019, doubled for what is not random.
    assert abs(got[0].item() - want[0]) < 0.04 * abs(want[0])
    for x, y, name in zip(got[1:], want[1:], ("dw", "db", "dA", "dB")):
        off = torch.linalg.norm(x.double().cpu() - y) / torch.linalg.norm(y)
        assert off < 0.04, (name, off.item())


def test_a_step_is_the_sum_of_its_parts_captured_or_not(ex):
    import paper_2403_12983_amd as osscar

    def setup():
        model, X, index, targets, A, B, g = ex.make(256, 64, 80, 3, 4, 150, DEV)
        masters = [None, None, A.float(), B.float()]
        grads = [torch.zeros_like(t) for t in (model["w"], model["b"], A, B)]
        return model, X, index, targets, A, B, osscar.AdamW([model["w"], model["b"], A, B], grads, bits=8, masters=masters), grads

    def step(model, X, index, targets, A, B, plan, grads, lr, t):
        _, *new = ex.gradients(model, X, A, B, index, targets)
        for kept, x in zip(grads, new):
            kept.copy_(x)
        plan.osscar_adamw(lr, t)

    eager, graphed = setup(), setup()
    lr, t = torch.tensor(1e-2, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    step(*setup()[:8], 1e-2, 1)      # (libraries make their handles outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.add_(1)
        step(*graphed, lr, t)
    for k in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        step(*eager, lr, torch.tensor(k, device=DEV))
        torch.cuda.synchronize()
        for a, b in zip(eager[6].params, graphed[6].params):
            assert torch.equal(a, b), k
    assert t.item() == 3 and not torch.equal(eager[5], torch.zeros_like(eager[5]))


def test_example_runs_and_serves(ex):
    got = ex.run(tokens=2048, d=64, f=96, tasks=3, rank=4, vocab=300, steps=10)
    assert all(math.isfinite(v) and v > 1 for v in got.values())


def test_served_rows_in_any_grouping(ex):
    """Token by token, a few or many together, mixed or sorted: the same answers, but for the order of float32 sums and the rounding behind it."""
    model, X, index, targets, A, B, g = ex.make(700, 96, 120, 5, 6, 100, DEV)
    B.copy_(torch.randn(B.shape, generator=g, device=DEV) * 0.3)
    order = torch.randperm(700, generator=g, device=DEV)
    all_at_once = ex.serve(model, X, A, B, index, 700).float()
    for rows in (1, 16, 100, 300):
        few = ex.serve(model, X[order], A, B, index[order], rows).float()
        # y is bf16: where a sum falls on the other side of a border it is 2^-7 of itself off, and its logit as much of one of its 96 terms
        assert (few - all_at_once[order]).abs().max() <= 2.0 ** -5 * all_at_once.abs().max()
        assert ((few - all_at_once[order]).abs() > 2.0 ** -7 * all_at_once.abs().max()).float().mean() < 0.02
