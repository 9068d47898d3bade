"""CPU-only checks of the layer operators' boundary: refusals come before any GPU work, the workspace queries are host-only."""
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


P = C.c_void_p(1 << 20)      # an address that no refused call may touch
ODD = C.c_void_p((1 << 20) + 1)


def _desc(**kw):
    from paper_2403_12983_amd.binding import _GatedDesc
    v = dict(n=4, d=16, f=24, ldx=16, ldw=24, ldh=24, dtype=1, act=0, rows_out=0, unaligned=0)
    v.update(kw)
    return _GatedDesc(*v.values())


BAD_DESCS = [dict(n=-1), dict(d=0), dict(f=0), dict(n=1 << 31), dict(d=1 << 31, ldx=1 << 31), dict(ldx=15), dict(ldw=23), dict(rows_out=1, ldw=15), dict(ldh=23), dict(dtype=2), dict(dtype=-1),
             dict(act=4), dict(act=-1), dict(n=1 << 29, f=1 << 29, ldw=1 << 29, ldh=1 << 29)]


@pytest.mark.parametrize("change", BAD_DESCS)
def test_gated_descriptions_are_refused(lib, change):
    d = _desc(**change)
    assert lib.osscar_gated_workspace_bytes(C.byref(d), 0) == 0
    assert lib.osscar_gated_forward(C.byref(d), P, P, P, P, None, None, P, 1 << 40, None) == 1
    assert lib.osscar_gated_backward(C.byref(d), P, P, P, P, None, None, P, 16, P, P, 24, 1, P, 1 << 40, None) == 1
    assert b"osscar_gated" in lib.osscar_last_error(None)


def test_gated_buffers_are_refused(lib):
    d = C.byref(_desc())
    size = 1 << 30
    assert lib.osscar_gated_forward(None, P, P, P, P, None, None, P, size, None) == 1
    for k in range(4):
        a = [P, P, P, P]
        a[k] = None
        assert lib.osscar_gated_forward(d, *a, None, None, P, size, None) == 1, k
        a[k] = ODD
        assert lib.osscar_gated_forward(d, *a, None, None, P, size, None) == 1, k
    assert lib.osscar_gated_forward(d, C.c_void_p((1 << 20) + 2), P, P, P, None, None, P, size, None) == 1      # not declared unaligned
    assert lib.osscar_gated_forward(d, P, P, P, P, P, None, P, size, None) == 1                                 # G without U
    assert lib.osscar_gated_forward(d, P, P, P, P, None, None, C.c_void_p((1 << 20) + 128), size, None) == 1    # workspace
    b = lambda *a: lib.osscar_gated_backward(d, P, P, P, P, None, None, *a, P, size, None)  # noqa: E731
    assert b(P, 15, P, P, 24, 1) == 1 and b(P, 16, P, P, 23, 1) == 1 and b(P, 16, P, None, 24, 1) == 1 and b(P, 16, P, P, 24, 2) == 1 and b(ODD, 16, P, P, 24, 1) == 1
    # too little workspace is said, not written past
    q = _desc(n=300, ldx=17, d=17, ldw=25, f=25, ldh=25)
    need = lib.osscar_gated_workspace_bytes(C.byref(q), 2)
    assert need > 300 * 25 * 2 * 4
    assert lib.osscar_gated_backward(C.byref(q), P, P, P, P, None, None, P, 17, P, P, 25, 1, P, need // 2, None) == 2
    assert lib.osscar_gated_forward(C.byref(q), P, P, P, P, None, None, None, 0, None) == 2
    assert lib.osscar_gated_workspace_bytes(C.byref(q), 1) < need


def test_gated_forward_in_place_operands_need_next_to_no_workspace(lib):
    assert lib.osscar_gated_workspace_bytes(C.byref(_desc(n=16384, d=2048, f=8192, ldx=2048, ldw=8192, ldh=8192)), 0) <= 256
    assert lib.osscar_gated_workspace_bytes(C.byref(_desc(n=16384, d=2048, f=8192, ldx=2048, ldw=8192, ldh=8192, dtype=0)), 0) <= 256
    assert lib.osscar_gated_workspace_bytes(C.byref(_desc(n=16384, d=2048, f=8192, ldx=2048, ldw=8192, ldh=8192, unaligned=1)), 0) > 2 * 2048 * 8192 * 2


def test_int_calls_are_refused(lib):
    assert lib.osscar_int_workspace_bytes(4, 16, 8) > 0
    for n, d1, m in ((-1, 16, 8), (4, 0, 8), (4, 131072, 8), (4, 16, 0), (1 << 31, 16, 8), (1 << 30, 16, 1 << 30)):
        assert lib.osscar_int_workspace_bytes(n, d1, m) == 0
    call = lambda **kw: lib.osscar_int_product(*{**dict(X=P, n=4, d1=16, ldx=16, xt=1, xs=None, Wq=P, ldq=16, ws=P, m=8, bias=None, Y=P, ldy=8, yt=1, w=P, size=1 << 30,  # noqa: E731
                                                        s=None), **kw}.values())
    for kw in (dict(X=None), dict(X=ODD), dict(n=-1), dict(d1=0), dict(d1=131072, ldx=131072, ldq=131072), dict(ldx=15), dict(xt=3), dict(xs=P), dict(xt=2), dict(Wq=None),
               dict(Wq=C.c_void_p((1 << 20) + 8)), dict(ldq=24), dict(ldq=0), dict(ws=None), dict(m=0), dict(Y=None), dict(Y=ODD), dict(ldy=7), dict(yt=2), dict(w=C.c_void_p(64))):
        assert call(**kw) == 1, kw
    assert call(size=1) == 2 and call(w=None, size=0) == 2
    assert lib.osscar_int_rows(P, 4, 16, 16, 2, P, 16, P, None) == 1 and lib.osscar_int_rows(P, 4, 16, 15, 1, P, 16, P, None) == 1
    assert lib.osscar_int_rows(P, 4, 16, 16, 1, P, 17, P, None) == 1 and lib.osscar_int_rows(P, 4, 16, 16, 1, None, 16, P, None) == 1
    assert lib.osscar_int_weights(P, 16, 8, 7, 1, 0, P, 16, P, None) == 1 and lib.osscar_int_weights(P, 16, 8, 15, 1, 1, P, 16, P, None) == 1
    assert lib.osscar_int_weights(P, 16, 8, 8, 1, 0, P, 8, P, None) == 1 and lib.osscar_int_weights(P, 16, 8, 8, 1, 0, P, 16, None, None) == 1
    assert lib.osscar_int_product(None, 0, 16, 16, 1, None, P, 16, P, 8, None, None, 8, 1, None, 0, None) == 0      # no rows: nothing to do


def test_logprobs_calls_are_refused(lib):
    assert lib.osscar_logprobs_workspace_bytes(4, 100, 5) > 0
    for n, v, top in ((-1, 100, 5), (4, 0, 0), (4, 100, 65), (4, 3, 4), (4, 100, -1), (4, 1 << 31, 1)):
        assert lib.osscar_logprobs_workspace_bytes(n, v, top) == 0
    call = lambda **kw: lib.osscar_logprobs(*{**dict(L=P, n=600, v=100, ld=100, t=1, tg=P, scale=1.0, top=5, lp=P, en=P, lse=P, ti=P, tl=P, w=P, size=1 << 20, s=None), **kw}.values())  # noqa: E731
    for kw in (dict(L=None), dict(L=ODD), dict(n=-1), dict(v=0), dict(ld=99), dict(t=2), dict(tg=None), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(top=65),
               dict(top=101), dict(top=-1), dict(lp=None), dict(ti=None), dict(tl=None), dict(w=C.c_void_p(8))):
        assert call(**kw) == 1, kw
    assert call(n=4, v=100000, ld=100000, w=None, size=0) == 2
    back = lambda **kw: lib.osscar_logprobs_backward(*{**dict(L=P, n=4, v=100, ld=100, t=1, tg=P, scale=1.0, lse=P, dl=P, en=P, de=P, top=5, ti=P, dt=P, o=C.c_void_p(1 << 21), ldd=100, s=None),  # noqa: E731
                                                       **kw}.values())
    for kw in (dict(lse=None), dict(o=None), dict(o=ODD), dict(ldd=99), dict(en=None), dict(ti=None), dict(o=P, ldd=104), dict(scale=0.0), dict(ld=99)):
        assert back(**kw) == 1, kw


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    import paper_2403_12983_amd as pkg
    X, W = torch.zeros(2, 16), torch.zeros(16, 8)
    for call in (lambda: pkg.osscar_gated_forward(X, W, W), lambda: pkg.osscar_gated_backward(X, W, W, torch.zeros(2, 8)), lambda: pkg.osscar_int_weights(W), lambda: pkg.osscar_int_rows(X),
                 lambda: pkg.osscar_int_product(X, torch.zeros(8, 16, dtype=torch.int8), torch.zeros(8)), lambda: pkg.osscar_logprobs(X, torch.zeros(2, dtype=torch.int64)),
                 lambda: pkg.osscar_logprobs_backward(X, torch.zeros(2, dtype=torch.int64), torch.zeros(2, 2))):
        with pytest.raises(pkg.OsscarError) as e:
            call()
        assert e.value.status == 1
