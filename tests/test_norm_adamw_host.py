"""CPU-only checks of layer norm's and AdamW's boundary: refusals come before any GPU work."""
import ctypes as C
import math
import os

import pytest
import torch


@pytest.fixture(scope="module")
def lib():
    import paper_2403_12983_amd as pkg
    if not os.path.exists(pkg.lib_path()):
        from paper_2403_12983_amd import build
        build.build()
    return pkg.load_library()


P, P2 = C.c_void_p(1 << 20), C.c_void_p(1 << 21)      # addresses that no refused call may touch
ODD = C.c_void_p((1 << 20) + 1)


def test_layernorm_calls_are_refused(lib):
    call = lambda **kw: lib.osscar_layernorm_forward(*{**dict(X=P, n=4, d=16, ldx=16, t=1, w=P, b=P, wt=0, eps=1e-5, Y=P2, ldy=16, st=P, s=None), **kw}.values())  # noqa: E731
    for kw in (dict(X=None), dict(X=ODD), dict(n=-1), dict(n=1 << 31), dict(d=0), dict(d=1 << 31, ldx=1 << 31, ldy=1 << 31), dict(ldx=15), dict(ldy=15), dict(t=2), dict(wt=2), dict(wt=-1), dict(w=ODD),
               dict(b=C.c_void_p((1 << 20) + 2)), dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-60), dict(Y=None), dict(Y=ODD), dict(st=ODD),
               dict(Y=P, ldy=20)):
        assert call(**kw) == 1, kw
        assert b"osscar_layernorm" in lib.osscar_last_error(None)
    assert call(n=0, X=None, Y=None) == 0      # no rows: nothing to do
    back = lambda **kw: lib.osscar_layernorm_backward(*{**dict(X=P, n=4, d=16, ldx=16, t=1, w=P, wt=0, dY=P, ldy=16, st=P, dX=P2, ldd=16, dw=P, db=P, dt=0, ws=P, size=1 << 30,  # noqa: E731
                                                               s=None), **kw}.values())
    for kw in (dict(X=None), dict(X=ODD), dict(n=-1), dict(d=0), dict(ldx=15), dict(t=2), dict(wt=3), dict(w=ODD), dict(dY=None), dict(dY=ODD), dict(ldy=15), dict(st=None), dict(st=ODD),
               dict(dX=ODD), dict(ldd=15), dict(dw=ODD), dict(db=ODD), dict(dt=2), dict(ws=C.c_void_p((1 << 20) + 64)), dict(dX=P, ldd=20)):
        assert back(**kw) == 1, kw
    assert back(ws=None) == 2 and back(size=100) == 2
    assert back(n=0, X=None, dY=None, st=None, dw=None, db=None) == 0 and back(dX=None, dw=None, db=None, ws=None, size=0) == 0
    for n, d in ((-1, 16), (4, 0), (1 << 31, 16), (4, 1 << 31)):
        assert lib.osscar_layernorm_workspace_bytes(n, d) == 0
    assert 2 * 16 * 4 <= lib.osscar_layernorm_workspace_bytes(1, 16) < 1024 and lib.osscar_layernorm_workspace_bytes(1 << 30, 7168) < 1 << 24


def test_adamw_calls_are_refused(lib):
    from paper_2403_12983_amd.binding import _AdamWDesc, _AdamWTensor

    def call(bits=32, count=1, tensor=None, null=False, **kw):
        t = _AdamWTensor(**{**dict(n=100, p=1 << 20, master=None, g=1 << 21, m=1 << 22, v=1 << 23, m_scale=1 << 24, v_scale=1 << 25, p_dtype=0, g_dtype=0), **(tensor or {})})
        d = _AdamWDesc(**{**dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=1, lr_dev=None, step_dev=None, grad_scale_dev=None, seed=0, stochastic=0, bits=bits), **kw})
        return lib.osscar_adamw(C.byref(t), count, None if null else C.byref(d), None)

    for kw in (dict(null=True), dict(count=-1), dict(bits=16), dict(bits=0), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=1e-60), dict(eps=math.inf),
               dict(eps=math.nan), dict(weight_decay=-1.0), dict(weight_decay=math.inf), dict(lr=-1.0), dict(lr=math.nan), dict(lr=1e300), dict(step=0), dict(lr_dev=2), dict(step_dev=4),
               dict(grad_scale_dev=1)):
        assert call(**kw) == 1, kw
        assert b"osscar_adamw" in lib.osscar_last_error(None)
    for t in (dict(n=-1), dict(n=1 << 31), dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(p=(1 << 20) + 2), dict(g=(1 << 21) + 1), dict(m=(1 << 22) + 2), dict(v=(1 << 23) + 1),
              dict(master=1 << 26), dict(master=(1 << 26) + 2, p_dtype=1), dict(p_dtype=2), dict(g_dtype=2), dict(p=(1 << 20) + 1, p_dtype=1)):
        assert call(tensor=t) == 1, t
    for t in (dict(m_scale=None), dict(v_scale=None), dict(m_scale=(1 << 24) + 1)):
        assert call(tensor=t, bits=8) == 1, t
    assert call(tensor=dict(n=0, p=None, g=None, m=None, v=None)) == 0 and lib.osscar_adamw(None, 0, C.byref(_AdamWDesc(1e-3, 0.9, 0.999, 1e-8, 0.1, 1, None, None, None, 0, 0, 8)), None) == 0
    t = _AdamWTensor(100, None, None, None, 1 << 22, 1 << 23, 1 << 24, 1 << 25, 0, 0)
    outs = lambda x: (C.c_void_p * 1)(x)  # noqa: E731
    for m, r in ((outs(None), outs(1 << 26)), (outs(1 << 26), outs(None)), (outs((1 << 26) + 1), outs(1 << 26))):
        assert lib.osscar_adamw_values(C.byref(t), 1, m, r, None) == 1
    assert lib.osscar_adamw_values(None, 1, outs(1 << 26), outs(1 << 26), None) == 1 and lib.osscar_adamw_values(None, 0, None, None, None) == 0


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    import paper_2403_12983_amd as pkg
    X = torch.zeros(2, 16)
    for call in (lambda: pkg.osscar_layernorm_forward(X), lambda: pkg.osscar_layernorm_backward(X, None, X, torch.zeros(2, 2)), lambda: pkg.AdamW([X], [X])):
        with pytest.raises(pkg.OsscarError) as e:
            call()
        assert e.value.status == 1
