"""osscar_adamw and osscar_adamw_values as plain calls, against the lists kept together (whose steps are checked against the definition elsewhere): the same bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
SHAPES = [(300,), (17, 33), (1,), (40, 70), (5000,), (0,), (3, 5, 7)]


@pytest.fixture(scope="module")
def osscar():
    import paper_2403_12983_amd as pkg
    pkg.load_library()
    return pkg


def _setup(kind):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    make = lambda s, scale: torch.randn(*s, generator=g, device=DEV) * scale  # noqa: E731
    params = [make(s, 0.3).to(F32 if kind == "f32" else BF16) for s in SHAPES]
    params[3] = params[3].t().contiguous().t()
    masters = [torch.empty_like(p, dtype=F32).copy_(p) for p in params] if kind == "master" else None
    return params, masters, [[torch.empty_like(p, dtype=(F32, BF16)[k % 2]).copy_(make(p.shape, 1e-2)) for k, p in enumerate(params)] for _ in range(3)]


def _same(a, b):
    return all(x is None and y is None or torch.equal(x.contiguous().view(-1).view(torch.uint8), y.contiguous().view(-1).view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("seed", [None, 7])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("kind", ["f32", "bf16", "master"])
def test_calls_are_the_steps_of_a_list(osscar, kind, bits, seed):
    params, masters, grads = _setup(kind)
    kept = osscar.AdamW([p.clone() for p in params], bits=bits, masters=None if masters is None else [m.clone() for m in masters])
    memory = [tuple(s) for s in osscar.AdamW(params, bits=bits).states]
    for t, g in enumerate(grads, 1):      # new gradients, and new tuples of the same states, each time
        states = [osscar.AdamWState(*s) for s in memory]
        osscar.osscar_adamw(params, g, states, 1e-3, t, 0.9, 0.99, 1e-6, 0.1, masters=masters, seed=seed)
        kept.osscar_adamw(1e-3, t, 0.9, 0.99, 1e-6, 0.1, grads=g, seed=seed)
        assert _same(params, kept.params) and (masters is None or _same(masters, kept.masters))
        assert all(_same(a, b) for a, b in zip(memory, kept.states))
        if bits == 8:
            for x, y, p in zip(osscar.osscar_adamw_values(states), kept.osscar_adamw_values(), params):
                assert x.m.shape == p.shape and x.m.stride() == p.stride() and torch.equal(x.m, y.m) and torch.equal(x.root, y.root)
    if bits == 8:      # a state that was not stepped: in the order of its memory
        x, p = osscar.osscar_adamw_values([osscar.AdamWState(*memory[3])])[0], params[3]
        assert torch.equal(x.root, osscar.osscar_adamw_values(states)[3].root.t().reshape(-1)) and not p.is_contiguous()


def test_calls_captured_and_on_another_stream(osscar):
    params, _, grads = _setup("bf16")
    eager = [p.clone() for p in params]
    a, b = osscar.AdamW(params, bits=8).states, osscar.AdamW(params, bits=8).states
    lr, step = torch.tensor(1e-3, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        osscar.osscar_adamw(params, grads[0], a, lr, step, seed=5)
        got = osscar.osscar_adamw_values(a)
    for t in range(1, 4):
        lr.fill_(1e-3 * t)
        graph.replay()
        torch.cuda.synchronize()
        osscar.osscar_adamw(eager, grads[0], b, lr, torch.tensor(t, device=DEV), seed=5, stream=side if t == 2 else None)
        torch.cuda.synchronize()
        assert _same(params, eager) and all(_same(x, y) for x, y in zip(a, b))
        assert all(torch.equal(x.root, y.root) and torch.equal(x.m, y.m) for x, y in zip(got, osscar.osscar_adamw_values(b)))


def test_a_parameter_moved_or_narrowed_between_steps(osscar):
    p, g = torch.ones(4000, device=DEV), torch.ones(4000, device=DEV)
    plan = osscar.AdamW([p], [g], bits=8)
    plan.osscar_adamw(1e-2, 1)
    p.data = p.data.clone()
    q = p.clone()
    plan.osscar_adamw(1e-2, 2)
    assert (p < q).all()      # where it is now
    before = p.clone()
    p.data = p.data[::2].clone()
    for call in (lambda: plan.osscar_adamw(1e-2, 3), lambda: plan.osscar_adamw(1e-2, 3, grads=[torch.ones(2000, device=DEV)]), lambda: plan.osscar_adamw_values()):
        with pytest.raises(osscar.OsscarError) as e:
            call()
        assert e.value.status == 1
    assert torch.equal(p, before[::2])
