"""Layer norm, adapters and AdamW where offsets pass 32 bits: the last rows and elements are those of a small call on them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -8      # of rounding to bf16


@pytest.fixture(scope="module")
def osscar():
    import paper_2403_12983_amd as pkg
    pkg.load_library()
    return pkg


def _rows(n, d, tail, seed):
    """n x d bf16, ones but for the last `tail` rows"""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    X = torch.ones(n, d, dtype=torch.bfloat16, device=DEV)
    X[-tail:] = torch.randn(tail, d, generator=g, device=DEV)
    return X


def test_layernorm_past_32_bits(osscar):
    n, d, tail = 300100, 7168, 130      # 2.15e9 elements
    X, dY = _rows(n, d, tail, 1), _rows(n, d, tail, 2)
    w, b = torch.randn(d, device=DEV), torch.randn(d, device=DEV)
    Y, stats = osscar.osscar_layernorm_forward(X, w, b, save=True)
    want, wstats = osscar.osscar_layernorm_forward(X[-tail:], w, b, save=True)
    assert torch.equal(Y[-tail:], want) and torch.equal(stats[-tail:], wstats)
    assert torch.equal(Y[:7], b.to(torch.bfloat16).expand(7, d))      # (rows of one value)
    dX, dw, db = osscar.osscar_layernorm_backward(X, w, dY, stats, out=Y)
    wX, ww, _ = osscar.osscar_layernorm_backward(X[-tail:], w, dY[-tail:], wstats)
    assert torch.equal(dX[-tail:], wX)
    # rows of one value have h = 0: dw is the last rows'; db counts the ones
    assert (dw - ww).abs().max() <= 1e-4 * ww.abs().max() and (db - (n - tail)).abs().max() < 0.01 * n
    del X, dY, Y, dX


def test_adapters_past_32_bits(osscar):
    n, d, m, count, r, tail = 300032, 7168, 72, 3, 8, 128
    X = _rows(n, d, tail, 3)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    A = (torch.randn(count, r, d, generator=g, device=DEV) / 85).to(torch.bfloat16)
    B = torch.randn(count, r, m, generator=g, device=DEV).to(torch.bfloat16)
    index = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    index[-tail:] = torch.randint(0, count, (tail,), generator=g, device=DEV)
    Y, T = osscar.osscar_adapters_forward(X, A, B, index=index, save=True)
    want, wT = osscar.osscar_adapters_forward(X[-tail:], A, B, index=index[-tail:], save=True)
    near = lambda a, b, e: (a.float() - b.float()).abs().max() <= e * b.float().abs().max()  # noqa: E731
    assert not Y[:-tail].any() and not T[:-tail].any() and near(T[-tail:], wT, 1e-5) and near(Y[-tail:], want, 2 * U)
    # the other way round: dX is the large one, and dA reads X
    dY = torch.randn(n, m, generator=g, device=DEV).to(torch.bfloat16)
    dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, index=index, dw_dtype=torch.float32)
    wX, wA, wB = osscar.osscar_adapters_backward(X[-tail:], A, B, dY[-tail:], T=wT, index=index[-tail:], dw_dtype=torch.float32)
    assert near(dX[-tail:], wX, 2 * U) and near(dA, wA, 1e-4) and near(dB, wB, 1e-4) and not dX[:1000].any()
    Yx = osscar.osscar_adapters_forward(dY, B, A, index=index, base=X, out=X)      # y of 7168 columns, in place
    wx = osscar.osscar_adapters_forward(dY[-tail:], B, A, index=index[-tail:], base=_rows(tail, d, tail, 3))
    assert near(Yx[-tail:], wx, 2 * U) and (Yx[:1000] == 1).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_past_32_bits(osscar, bits):
    n, tail = (1 << 29) + 1000, 1000      # 2^31 bytes of float32 and more
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    p, grad = torch.ones(n, device=DEV), torch.ones(n, device=DEV)
    p[-tail:] = torch.randn(tail, generator=g, device=DEV)
    grad[-tail:] = torch.randn(tail, generator=g, device=DEV)
    small, sgrad = p[-tail:].clone(), grad[-tail:].clone()
    plan, one = osscar.AdamW([p], [grad], bits=bits), osscar.AdamW([small], [sgrad], bits=bits)
    plan.osscar_adamw(1e-2, 1)
    one.osscar_adamw(1e-2, 1)
    assert torch.equal(p[-tail:], small) and (p[: 1 << 20] == p[0]).all() and p[0] < 1
    if bits == 8:
        s, t = plan.states[0], one.states[0]      # (the tail begins at a block)
        assert torch.equal(s.v[-tail:], t.v) and torch.equal(s.m[-tail:].view(torch.uint8), t.m.view(torch.uint8)) and torch.equal(s.m_scale[-4:], t.m_scale)
        assert torch.equal(plan.osscar_adamw_values()[0].root[-tail:], one.osscar_adamw_values()[0].root)
