"""CPU-only checks of the adapters' boundary: refusals come before any GPU work."""
import ctypes as C
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


def _desc(**kw):
    from paper_2403_12983_amd.binding import _AdaptersDesc
    return _AdaptersDesc(**{**dict(n=4, d=16, m=24, ldx=16, lda=16, next_a=48, ldb=24, next_b=72, count=2, rank=3, dtype=1, index=1), **kw})


def _forward(lib, desc=None, **kw):
    return lib.osscar_adapters_forward(*{**dict(d=C.byref(desc or _desc()), X=P, A=P, B=P, i=P, s=P, r=P, base=P2, ldb=24, Y=P2, ldy=24, T=P, w=P, size=1 << 40, st=None), **kw}.values())


def _backward(lib, desc=None, **kw):
    return lib.osscar_adapters_backward(*{**dict(d=C.byref(desc or _desc()), X=P, A=P, B=P, i=P, s=P, r=P, dY=P, ldy=24, T=P, base=P2, ldb=16, dX=P2, ldx=16, dA=P, dB=P, t=1, w=P, size=1 << 40,
                                                 st=None), **kw}.values())


@pytest.mark.parametrize("change", [dict(n=-1), dict(n=(1 << 22) + 1), dict(d=0), dict(m=0), dict(d=1 << 31, ldx=1 << 31, lda=1 << 31), dict(ldx=15), dict(lda=15), dict(ldb=23), dict(next_a=-1), dict(next_b=-1),
                                    dict(count=0), dict(count=4097), dict(rank=0), dict(rank=1025), dict(dtype=2), dict(n=1 << 22, m=1 << 15, ldb=1 << 15)])
def test_descriptions_are_refused(lib, change):
    d = _desc(**change)
    wide = dict(ldb=1 << 15, ldy=1 << 15) if "m" in change else {}
    assert lib.osscar_adapters_workspace_bytes(C.byref(d), 0) == 0 and lib.osscar_adapters_workspace_bytes(C.byref(d), 1) == 0
    assert _forward(lib, d, **wide) == 1 and _backward(lib, d, **({"ldy": 1 << 15} if wide else {})) == 1
    assert b"osscar_adapters" in lib.osscar_last_error(None)


def test_buffers_are_refused(lib):
    assert lib.osscar_adapters_workspace_bytes(None, 0) == 0 and _forward(lib, d=None) == 1 and _backward(lib, d=None) == 1
    two = C.c_void_p((1 << 20) + 2)
    for kw in (dict(X=None), dict(X=ODD), dict(A=None), dict(A=ODD), dict(B=None), dict(B=ODD), dict(i=None), dict(i=C.c_void_p((1 << 20) + 4)), dict(s=two), dict(r=two), dict(base=ODD), dict(ldb=23),
               dict(Y=None), dict(Y=ODD), dict(ldy=23), dict(ldy=30), dict(T=two), dict(w=C.c_void_p((1 << 20) + 128))):
        assert _forward(lib, **kw) == 1, kw
    assert _forward(lib, _desc(index=0)) == 1      # an index that the description does not speak of
    assert _forward(lib, w=None) == 2 and _forward(lib, size=100) == 2
    for kw in (dict(X=None), dict(X=ODD), dict(A=None), dict(B=None), dict(i=None), dict(dY=None), dict(dY=ODD), dict(ldy=23), dict(T=two), dict(base=ODD), dict(ldb=15), dict(dX=None), dict(dX=ODD),
               dict(ldx=15), dict(ldx=20), dict(dA=None), dict(dB=None), dict(dA=ODD), dict(t=2), dict(w=C.c_void_p((1 << 20) + 128))):
        assert _backward(lib, **kw) == 1, kw
    assert _backward(lib, w=None) == 2 and _backward(lib, size=2000) == 2
    # nothing to do
    assert _forward(lib, _desc(n=0), X=None, Y=None, base=None, w=None, size=0) == 0
    assert _backward(lib, _desc(n=0), X=None, dY=None, dA=None, dB=None, w=None, size=0) == 0 and _backward(lib, dX=None, base=None, dA=None, dB=None, w=None, size=0) == 0


def test_workspaces_hold_what_the_calls_take(lib):
    size = lambda **kw: (lib.osscar_adapters_workspace_bytes(C.byref(_desc(**kw)), 0), lib.osscar_adapters_workspace_bytes(C.byref(_desc(**kw)), 1))  # noqa: E731
    f, b = size(n=8192, d=7168, ldx=7168, lda=7168, m=14336, ldb=14336, rank=32, count=1, index=0)
    assert 8192 * 32 * 4 <= f < 8 * 8192 * 32 * 4 + 1024 and b < 16 * 32 * (7168 + 14336) * 4 + 16 * 8192 * 32 * 4      # (16 pieces of 512 rows of both gradients)
    f, b = size(n=0)
    assert 0 < f <= 256 and 0 < b <= 1024


def test_the_binding_refuses_tensors_that_are_not_on_a_gpu():
    import paper_2403_12983_amd as pkg
    X, A, B = torch.zeros(2, 16), torch.zeros(1, 3, 16), torch.zeros(1, 3, 8)
    for call in (lambda: pkg.osscar_adapters_forward(X, A, B), lambda: pkg.osscar_adapters_backward(X, A, B, torch.zeros(2, 8))):
        with pytest.raises(pkg.OsscarError) as e:
            call()
        assert e.value.status == 1


def test_a_call_without_gradients_of_the_weights_takes_no_space_for_them(lib):
    """Their partial sums alone (one for each adapter and component at least, of both widths) are 22 GB here."""
    wide = dict(d=7168, ldx=7168, lda=7168, m=14336, ldb=14336, rank=64)
    for n, count, index in ((16384, 4096, 1), (4096, 1024, 1), (300, 3, 1), (16, 32, 1), (8192, 1, 0)):
        d = _desc(n=n, count=count, index=index, **wide)
        full, less = (lib.osscar_adapters_workspace_bytes(C.byref(d), k) for k in (1, 2))
        assert full > min(n, count) * 64 * (7168 + 14336) * 4 and less <= 4 * n * 64 * 4 + 8 * n + 1024      # T in four parts at most, the order of the rows
        calls = dict(ldy=14336, ldb=7168, ldx=7168, i=P if index else None)
        assert _backward(lib, d, dA=None, dB=None, size=less - 257, **calls) == 2 and _backward(lib, d, size=less, **calls) == 2


def test_gradients_wider_than_a_launch_are_refused(lib):
    """Column blocks of 128 of both widths, 256 threads each: 2^32 threads of one launch, which HIP would cut off without an error."""
    big = 1 << 30
    for rank in (1, 64):
        wide = dict(n=1, d=big, ldx=big, lda=big, m=big, ldb=big, rank=rank, count=1, index=0, next_a=0, next_b=0)
        d = _desc(**wide)
        assert lib.osscar_adapters_workspace_bytes(C.byref(d), 1) == 0
        assert _backward(lib, d, i=None, ldy=big, ldb=big, ldx=big) == 1 and b"osscar_adapters_backward" in lib.osscar_last_error(None)
        # a block less, and calls without them
        assert lib.osscar_adapters_workspace_bytes(C.byref(_desc(**{**wide, "m": big - 128})), 1) > 0
        assert lib.osscar_adapters_workspace_bytes(C.byref(d), 0) > 0 and lib.osscar_adapters_workspace_bytes(C.byref(d), 2) > 0
