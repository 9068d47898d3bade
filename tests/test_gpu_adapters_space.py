"""The adapters' backward call in exactly the workspace that it asks for, with and without the gradients of A and B: the bits of a call in more, and nothing beside it touched."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def osscar():
    import paper_2403_12983_amd as pkg
    pkg.load_library()
    return pkg


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d,m,count,r", [(1, 64, 96, 1, 4), (5, 300, 7168, 3, 16), (40, 7168, 5000, 1, 64), (300, 264, 700, 3, 12), (900, 200, 300, 12, 8), (700, 64, 72, 2000, 2), (2100, 520, 136, 1, 32)])
def test_exact_workspaces(osscar, n, d, m, count, r, dtype):
    from paper_2403_12983_amd.binding import OSSCAR_BF16, OSSCAR_F32, _AdaptersDesc
    lib = osscar.load_library()
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    make = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)  # noqa: E731
    X, dY, A, B = make(n, d), make(n, m), make(count, r, d), make(count, r, m)
    index = None if count == 1 else torch.randint(-1, count, (n,), generator=g, device=DEV)
    code = OSSCAR_BF16 if dtype == torch.bfloat16 else OSSCAR_F32
    desc = _AdaptersDesc(n, d, m, d, d, r * d, m, r * m, count, r, code, 0 if index is None else 1)
    want = osscar.osscar_adapters_backward(X, A, B, dY, index=index)
    for need_w in (True, False):
        size = lib.osscar_adapters_workspace_bytes(C.byref(desc), 1 if need_w else 2) - 256      # (the query adds 256 to what is taken)
        space = torch.full((size + 512,), 255, dtype=torch.uint8, device=DEV)      # (NaN wherever something is read before it is written)
        begin = 256 - space.data_ptr() % 256
        dX, dA, dB = torch.empty_like(X), torch.empty_like(A), torch.empty_like(B)
        status = lib.osscar_adapters_backward(C.byref(desc), X.data_ptr(), A.data_ptr(), B.data_ptr(), None if index is None else index.data_ptr(), None, None, dY.data_ptr(), m, None, None, d,
                                              dX.data_ptr(), d, dA.data_ptr() if need_w else None, dB.data_ptr() if need_w else None, code, space.data_ptr() + begin, size,
                                              torch.cuda.current_stream().cuda_stream)
        assert status == 0 and torch.equal(dX, want[0])
        assert not need_w or torch.equal(dA, want[1]) and torch.equal(dB, want[2])
        assert (space[:begin] == 255).all() and (space[begin + size:] == 255).all()
    assert all(torch.equal(x, y) for x, y in zip(osscar.osscar_adapters_backward(X, A, B, dY, index=index, need_w=False)[:1], want))


def test_a_gradient_of_x_through_many_adapters_fits_a_small_space(osscar):
    """2000 adapters: the gradients of their weights take 5.3 GB of partial sums at these widths, a call without them 2 MB."""
    n, d, m, count, r = 2000, 7168, 14336, 2000, 16
    X, dY = (torch.ones(n, k, dtype=torch.bfloat16, device=DEV) for k in (d, m))
    A, B = (torch.ones(1, r, k, dtype=torch.bfloat16, device=DEV).expand(count, r, k) for k in (d, m))
    index = torch.arange(n, device=DEV).flip(0).contiguous()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    dX, _, _ = osscar.osscar_adapters_backward(X, A, B, dY, index=index, need_w=False)
    torch.cuda.synchronize()
    assert torch.cuda.max_memory_allocated() - before < (64 << 20) and (dX == r * m).all()
