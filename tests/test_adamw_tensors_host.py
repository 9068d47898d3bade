"""Where AdamW's tensors are, looked at on the CPU: what a step would hand to the library, which a stub stands in for."""
import contextlib

import pytest
import torch

import paper_2403_12983_amd as pkg
from paper_2403_12983_amd import layer_ops

F32, BF16 = torch.float32, torch.bfloat16


class _Library:
    """Takes down the rows of each call."""
    def __init__(self):
        self.rows = []

    def osscar_adamw(self, table, count, desc, handle):
        self.rows = [(r.n, r.p, r.master, r.g, r.m, r.v, r.m_scale, r.v_scale, r.p_dtype, r.g_dtype) for r in table[:count]]
        return 0

    def osscar_adamw_values(self, table, count, m_out, root_out, handle):
        self.rows = [(r.n, r.m, r.v, r.m_scale, r.v_scale) for r in table[:count]]
        return 0


@pytest.fixture
def library(monkeypatch):
    lib = _Library()
    monkeypatch.setattr(layer_ops, "_begin", lambda t, stream: (lib, t.get_device(), 0, contextlib.nullcontext()))
    return lib


def _address(t):
    return None if t is None or t.numel() == 0 else t.data_ptr()


def _rows(params, grads, masters, states):
    code = {F32: 0, BF16: 1}
    scales = [(s.m_scale, s.v_scale) for s in states]
    return [(p.numel(), _address(p), _address(q), _address(g), _address(s.m), _address(s.v), _address(a), _address(b), code[p.dtype], code[g.dtype])
            for p, q, g, s, (a, b) in zip(params, masters, grads, states, scales)]


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_goes_where_the_tensors_are(library, bits):
    params = [torch.zeros(1000), torch.zeros(30, 40).t(), torch.zeros(7, 5, dtype=BF16), torch.zeros(0), torch.zeros(3, dtype=BF16)]
    masters = [None, None, params[2].float(), None, None]
    grads = [torch.zeros_like(p, dtype=(BF16, F32)[k % 2]) for k, p in enumerate(params)]
    plan = pkg.AdamW(params, grads, bits=bits, masters=masters)
    plan.osscar_adamw(1e-3, 1)
    assert library.rows == _rows(params, grads, masters, plan.states)
    # memory that went elsewhere, of the same size
    params[0].data = torch.ones(1000)
    masters[2].data = torch.ones(7, 5)
    grads[1].data = torch.ones(30, 40).t()
    plan.osscar_adamw(1e-3, 2)
    assert library.rows == _rows(params, grads, masters, plan.states)
    if bits == 8:
        plan.osscar_adamw_values()
        assert library.rows == [(s.m.numel(), _address(s.m), _address(s.v), _address(s.m_scale), _address(s.v_scale)) for s in plan.states]
    plan.osscar_adamw(1e-3, 3, grads=[g.clone() for g in grads])
    assert library.rows == _rows(params, plan.grads, masters, plan.states) and plan.grads[0] is not grads[0]


@pytest.mark.parametrize("bits", [8, 32])
def test_a_parameter_that_was_narrowed_is_refused(library, bits):
    for narrow in (lambda t: t[::2].clone(), lambda t: t[:500], lambda t: torch.cat([t, t])):
        p, q = torch.zeros(300), torch.zeros(1000, 4)
        plan = pkg.AdamW([p, q], [torch.zeros(300), torch.zeros(1000, 4)], bits=bits)
        plan.osscar_adamw(1e-3, 1)
        library.rows = None
        q.data = narrow(q.data)
        for call in (lambda: plan.osscar_adamw(1e-3, 2), lambda: plan.osscar_adamw(1e-3, 2, grads=[torch.zeros(300), torch.zeros_like(q)]), lambda: plan.osscar_adamw_values()):
            with pytest.raises(pkg.OsscarError) as e:
                call()
            assert e.value.status == 1 and library.rows is None
    # its gradient or its master alone
    p, g = torch.zeros(1000, dtype=BF16), torch.zeros(1000)
    master = torch.zeros(1000)
    plan = pkg.AdamW([p], [g], bits=bits, masters=[master])
    for t in (g, master):
        whole = t.data
        t.data = t.data[:999]
        with pytest.raises(pkg.OsscarError):
            plan.osscar_adamw(1e-3, 2)
        t.data = whole
        plan.osscar_adamw(1e-3, 2)
    # another type, or memory that the next one has too
    p.data = torch.zeros(1000, dtype=torch.half)
    with pytest.raises(pkg.OsscarError):
        plan.osscar_adamw(1e-3, 3)
    both = [torch.zeros(8), torch.zeros(8)]
    plan = pkg.AdamW(both, [torch.zeros(8), torch.zeros(8)], bits=bits)
    both[1].data = both[0].data
    with pytest.raises(pkg.OsscarError):
        plan.osscar_adamw(1e-3, 1)


def test_what_is_no_list_of_tensors_is_refused(library):
    p = torch.zeros(4)
    for call in (lambda: pkg.AdamW([p, None]), lambda: pkg.AdamW([p], [None]), lambda: pkg.AdamW([p], masters=[3]), lambda: pkg.AdamW([p], states=[(p.clone(), None)]),
                 lambda: pkg.AdamW([torch.zeros(4, 4).to_sparse()]), lambda: pkg.AdamW([p], [torch.zeros(4).to_sparse()])):
        with pytest.raises((pkg.OsscarError, AttributeError)):
            call()


def test_the_call_without_a_list_kept(library):
    params, grads = [torch.zeros(300), torch.zeros(20, 30).t(), torch.zeros(5, dtype=BF16)], [torch.zeros(300), torch.zeros(20, 30).t(), torch.zeros(5, dtype=BF16)]
    masters = [None, None, torch.zeros(5)]
    for bits in (8, 32):
        states = pkg.AdamW(params, bits=bits).states
        fresh = [pkg.AdamWState(*s) for s in states]      # the same memory
        pkg.osscar_adamw(params, grads, fresh, 1e-3, 1, masters=masters)
        assert library.rows == _rows(params, grads, masters, states)
        pkg.osscar_adamw(tuple(params), tuple(grads), tuple(states), 1e-3, 1)
        assert library.rows == _rows(params, grads, [None] * 3, states)
        if bits == 8:
            values = pkg.osscar_adamw_values(fresh)
            assert [(x.m.shape, x.m.stride(), x.root.stride(), x.m.dtype) for x in values] == [(p.shape, p.stride(), p.stride(), BF16) for p in params]
            assert [x.m.shape for x in pkg.osscar_adamw_values([pkg.AdamWState(*s) for s in states])] == [(300,), (600,), (5,)]
            pkg.osscar_adamw([torch.zeros(600)], [torch.zeros(600)], fresh[1:2], 1e-3, 1)
            assert pkg.osscar_adamw_values(fresh[1:2])[0].root.shape == (600,)
    s32, s8 = pkg.AdamW(params).states, pkg.AdamW(params, bits=8).states
    library.rows = None
    for call in (lambda: pkg.osscar_adamw([], [], [], 1e-3, 1), lambda: pkg.osscar_adamw(params, grads[:2], s32, 1e-3, 1), lambda: pkg.osscar_adamw(params, grads, s32[:2], 1e-3, 1),
                 lambda: pkg.osscar_adamw(params, None, s32, 1e-3, 1), lambda: pkg.osscar_adamw(params, grads, s32, 1e-3, 1, masters=masters[:2]), lambda: pkg.osscar_adamw(params, grads, s8[:1] + s32[1:], 1e-3, 1),
                 lambda: pkg.osscar_adamw(params, grads, s32[:2] + s8[2:], 1e-3, 1), lambda: pkg.osscar_adamw([params[0]] * 2, [grads[0]] * 2, [s32[0], pkg.AdamWState(*(t.clone() for t in s32[0][:2]))], 1e-3, 1),
                 lambda: pkg.osscar_adamw(params, grads, s32, torch.tensor(1e-3, dtype=torch.double), 1), lambda: pkg.osscar_adamw(params, grads, s32, 1e-3, torch.tensor(1, dtype=torch.int32)),
                 lambda: pkg.osscar_adamw(params, grads, s32, 1e-3, 1, seed=1 << 32), lambda: pkg.osscar_adamw(params, grads, s32, 1e-3, 1, grad_scale=torch.ones(2)),
                 lambda: pkg.osscar_adamw_values(s32), lambda: pkg.osscar_adamw_values([]), lambda: pkg.osscar_adamw_values(s8[:1] + s32[1:])):
        with pytest.raises(pkg.OsscarError) as e:
            call()
        assert e.value.status == 1 and library.rows is None


def test_states_that_are_none_are_refused(library):
    p = [torch.zeros(4)]
    for states in (None, [], [None], [3], [(torch.zeros(4), torch.zeros(4))], [[torch.zeros(4), torch.zeros(4), None, None]], [(None, None, None, None)]):
        for call in (lambda: pkg.osscar_adamw(p, p, states, 1e-3, 1), lambda: pkg.osscar_adamw_values(states)):
            with pytest.raises(pkg.OsscarError) as e:
                call()
            assert e.value.status == 1 and not library.rows
    pkg.osscar_adamw(p, [torch.zeros(4)], [(torch.zeros(4), torch.zeros(4), None, None)], 1e-3, 1)      # a plain tuple of all four will do
    assert len(library.rows) == 1


def test_the_module_has_no_substitute(monkeypatch):
    import sys

    from paper_2403_12983_amd import binding
    assert pkg.load_tensors().adamw_rows
    monkeypatch.setattr(binding, "_TENSORS", None)
    monkeypatch.delattr(pkg, "_tensors", raising=False)
    monkeypatch.setitem(sys.modules, "paper_2403_12983_amd._tensors", None)
    with pytest.raises(FileNotFoundError, match="paper_2403_12983_amd.build"):
        binding.load_tensors()
