"""The layer operators at the ends of their ranges, against float64 definitions: masks by large constants, scales far from 1, gradients that are whole numbers and
have to be met exactly, the most rows and the longest rows that a call takes."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def osscar():
    import paper_2403_12983_amd as pkg
    pkg.load_library()
    return pkg


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def _whole(g, low, high, *shape, dtype):
    return torch.randint(low, high + 1, shape, generator=g, device=DEV).to(dtype)


def _check_logprobs(osscar, L, t, top, scale=1.0):
    """logp, entropy, lse, alternatives and the gradient of all three.  A difference of scaled logits is off by 2 e = 2^-23 of its size, the sum of the exponentials and its
    logarithm by about 1e-6 together; the gradient by a few e times (1 + |log p|) of the terms it is made of, and half a unit of bf16's eight bits where it is
    rounded to them."""
    n, v = L.shape
    z = L.double() * scale
    lp = torch.log_softmax(z, 1)
    p = lp.exp()
    plogp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -plogp.sum(1)
    logp = lp.gather(1, t[:, None])[:, 0]
    r = osscar.osscar_logprobs(L, t, top, scale)
    bound = lambda x: 2e-6 * (1 + x.abs() / 2)  # noqa: E731
    fine = torch.isfinite(logp)
    assert torch.equal(torch.isfinite(r.logp), fine) and ((r.logp.double() - logp)[fine].abs() <= bound(logp[fine])).all()
    assert ((r.entropy.double() - entropy).abs() <= 5e-6 * (1 + entropy)).all()
    lse = torch.logsumexp(z, 1)
    assert (((r.lse[:, 0].double() * scale + r.lse[:, 1].double()) - lse).abs() <= 2e-6 * (1 + lse.abs())).all()
    if top:
        order = torch.sort(L.float() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(r.top_index, order)
        want = torch.gather(lp, 1, order)
        fine = torch.isfinite(want)
        assert torch.equal(torch.isfinite(r.top_logp), fine) and ((r.top_logp.double() - want)[fine].abs() <= bound(want[fine])).all()
    g = _gen(n + v)
    a, b = _randn(g, n), _randn(g, n)
    c = _randn(g, n, top) if top else None
    hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
    own, total, size = a.double()[:, None] * hot, a.double()[:, None], a.double().abs()[:, None] * (hot + p)
    if top:
        own = own.scatter_add(1, r.top_index, c.double())
        total = total + c.double().sum(1, keepdim=True)
        size = size + torch.zeros_like(hot).scatter_add(1, r.top_index, c.double().abs()) + p * c.double().abs().sum(1, keepdim=True)
    want = scale * (own - p * total - b.double()[:, None] * (plogp + p * entropy[:, None]))
    size = scale * (size + b.double().abs()[:, None] * (plogp.abs() + p * (1 + entropy[:, None])))
    got = osscar.osscar_logprobs_backward(L, t, r.lse, a, entropy=r.entropy, dentropy=b, top_index=r.top_index, dtop=c, scale=scale)
    tol = 8e-6 * (1 + torch.where(p > 0, lp.abs(), torch.zeros_like(lp))) * size + (2.0 ** -8 * want.abs() if L.dtype == torch.bfloat16 else 0)
    assert ((got.double() - want).abs() <= tol + 1e-30).all()


MASKS = [-1e9, -1e10, -1e12, -1e20, -1e30]


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,v", [(3, 70), (2, 8200), (40, 20000), (600, 9000), (2, 131072)])
def test_logprobs_of_rows_masked_with_a_constant(osscar, n, v, dtype, mask):
    """a large finite number where others write minus infinity: over whole packets, whole steps, all of a row, all but one"""
    g = _gen(v)
    for pattern in ("blocks of 8", "blocks of 64", "first half", "last half", "all", "all but one"):
        at = torch.arange(v, device=DEV)
        if pattern.startswith("blocks"):
            size = int(pattern.split()[-1])
            out = (torch.rand(n, -(-v // size), generator=g, device=DEV) < 0.5).repeat_interleave(size, 1)[:, :v]
        elif pattern.endswith("half"):
            out = (at < v // 2 if pattern[0] == "f" else at >= v // 2).expand(n, v)
        else:
            out = torch.ones(n, v, dtype=torch.bool, device=DEV)
            if pattern == "all but one":
                out.scatter_(1, torch.randint(0, v, (n, 1), generator=g, device=DEV), False)
        L = torch.where(out, torch.full((), mask, device=DEV), _randn(g, n, v, scale=2.5)).to(dtype)
        t = torch.randint(0, v, (n,), generator=g, device=DEV)
        for top, scale in ((0, 1.0), (5, 0.01), (33, 1.0)):
            _check_logprobs(osscar, L, t, top, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", [1e6, 1e8, 1e10, 1e20, 1e30])
def test_logprobs_of_large_logits(osscar, size, dtype):
    """equal ones and normal ones of that size, of either sign"""
    g = _gen(17)
    for n, v in ((3, 70), (2, 8200), (700, 9000), (2, 70000)):
        t = torch.randint(0, v, (n,), generator=g, device=DEV)
        for L in (torch.full((n, v), size, device=DEV), _randn(g, n, v, scale=size)):
            _check_logprobs(osscar, L.to(dtype), t, 5)


@pytest.mark.parametrize("scale", [0.01, 1e-3, 1e-10])
def test_logprobs_rows_of_the_lowest_value_at_small_scales(osscar, scale):
    """every logit the lowest float32: as likely as the others, however small the scale"""
    for n, v in ((3, 70), (700, 9000), (2, 70000)):
        L = torch.full((n, v), torch.finfo(torch.float32).min, device=DEV)
        _check_logprobs(osscar, L, torch.randint(0, v, (n,), generator=_gen(v), device=DEV), 5, scale)


def test_logprobs_rows_of_the_lowest_value_at_the_smallest_scales(osscar):
    """so small that the lowest float32 times the scale is an ordinary number: a row of it is the start of the running maximum"""
    for scale in (1e-34, 1e-36, 1e-38):
        for n, v in ((3, 70), (700, 9000), (2, 70000)):
            L = torch.full((n, v), torch.finfo(torch.float32).min, device=DEV)
            _check_logprobs(osscar, L, torch.randint(0, v, (n,), generator=_gen(v), device=DEV), 5, scale)
            L[:, ::7] = 0.0
            _check_logprobs(osscar, L, torch.randint(0, v, (n,), generator=_gen(v), device=DEV), 5, scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_gradient_of_a_target_outside_the_vocabulary(osscar, dtype):
    """the whole row is NaN, the columns of probability zero among them; no other row is touched; without dlogp the target does not matter"""
    n, v = 4, 9000
    L = _randn(_gen(1), n, v, dtype=dtype)
    L[:, 100:200] = -math.inf
    t = torch.tensor([5, v, v + 7, -1], device=DEV)
    r = osscar.osscar_logprobs(L, t)
    one = torch.ones(n, device=DEV)
    d = osscar.osscar_logprobs_backward(L, t, r.lse, one)
    assert d[1:3].isnan().all() and torch.isfinite(d[0]).all() and (d[0, 100:200] == 0).all() and (d[3] == 0).all()
    d = osscar.osscar_logprobs_backward(L, t, r.lse, None, entropy=r.entropy, dentropy=one)
    assert torch.isfinite(d).all()
    d = osscar.osscar_logprobs_backward(L, t, r.lse, torch.full((n,), math.nan, device=DEV))
    assert d[:3].isnan().all() and (d[3] == 0).all()


MANY = (1 << 24) + 5      # rows of a workgroup each, 256 threads: more than 2^32 of them


def test_logprobs_of_more_rows_than_a_launch_takes(osscar):
    g = _gen(4)
    L = _randn(g, MANY, 3, dtype=torch.bfloat16)
    t = torch.randint(0, 3, (MANY,), generator=g, device=DEV)
    r = osscar.osscar_logprobs(L, t, 1)
    lp = torch.log_softmax(L.float(), 1)
    assert ((r.logp - lp.gather(1, t[:, None])[:, 0]).abs() <= 1e-5).all()      # (both float32)
    assert ((r.entropy + (lp * lp.exp()).sum(1)).abs() <= 1e-5).all() and ((r.lse.sum(1) - torch.logsumexp(L.float(), 1)).abs() <= 1e-5).all()
    best = L.float().max(1)
    first = torch.where(L[:, 0] == best.values.to(L.dtype), 0, torch.where(L[:, 1] == best.values.to(L.dtype), 1, 2))
    assert torch.equal(r.top_index[:, 0], first) and ((r.top_logp[:, 0] - lp.max(1).values).abs() <= 1e-5).all()
    d = osscar.osscar_logprobs_backward(L, t, r.lse, torch.ones(MANY, device=DEV))
    want = torch.zeros_like(lp).scatter_(1, t[:, None], 1.0) - lp.exp()
    assert ((d.float() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()


def test_int_rows_and_channels_beyond_what_a_launch_takes(osscar):
    """a row of one number x has the scale |x| / 127 and the digit 127 or -127; so has a channel"""
    g = _gen(5)
    X = _randn(g, MANY, 1)
    X[X.abs() < 1e-3] = 1e-3
    sign = torch.where(X[:, 0] > 0, 127, -127)
    scale = X[:, 0].abs().double() / 127
    q, s = osscar.osscar_int_rows(X)
    assert torch.equal(q[:, 0].int(), sign.int()) and ((s.double() - scale).abs() <= 2.0 ** -24 * scale).all()
    wq, ws = osscar.osscar_int_weights(X.t())      # 1 x MANY, a channel's number beside the next
    assert torch.equal(wq[:, 0].int(), sign.int()) and torch.equal(ws, s)
    two = torch.stack([X[:, 0], X[:, 0] / 2], 1)      # MANY x 2 in memory, a channel's numbers side by side
    wq, ws = osscar.osscar_int_weights(two.t())
    half = np.rint(two[:, 1].cpu().numpy() / s.cpu().numpy())      # (63.5 but for the quotient's rounding: 63 or 64)
    assert torch.equal(wq[:, 0].int(), sign.int()) and torch.equal(ws, s) and np.array_equal(wq[:, 1].cpu().numpy(), half) and (wq[:, 2:] == 0).all()
    one, s1 = osscar.osscar_int_weights(torch.ones(1, 1, device=DEV))
    Y = osscar.osscar_int_product(X, one, s1, out_dtype=torch.float32)
    assert ((Y - X).abs() <= 4 * 2.0 ** -24 * X.abs()).all()


@pytest.mark.parametrize("rows", ["in", "out"])
def test_gated_longest_bf16_rows(osscar, rows):
    """rows of 4194296: the last row of a tile of 256 ends just below 2^31 bytes from its first.  Whole numbers, which have one right value."""
    relu, K, g = osscar.OSSCAR_ACT_RELU, 4194296, _gen(6)
    lay = lambda t: t.t().contiguous().t() if rows == "out" else t  # noqa: E731
    X = torch.zeros(300, K, dtype=torch.bfloat16, device=DEV)
    at = torch.cat([torch.arange(40), torch.arange(K - 40, K)]).to(DEV)      # both ends of every row
    X[:, at] = _whole(g, -1, 1, 300, 80, dtype=torch.bfloat16)
    Wg, Wu = (_whole(g, -1, 1, K, 8, dtype=torch.bfloat16) for _ in range(2))
    x, wg, wu = X[:, at].double(), Wg[at].double(), Wu[at].double()
    want = ((x @ wg).clamp_min(0) * (x @ wu)).to(torch.bfloat16)
    assert torch.equal(osscar.osscar_gated_forward(X, lay(Wg), lay(Wu), relu), want)
    del X
    X = _whole(g, -1, 1, 300, 8, dtype=torch.bfloat16)
    Wg, Wu = (_whole(g, -1, 1, 8, K, dtype=torch.bfloat16) for _ in range(2))
    dH = torch.zeros(300, K, dtype=torch.bfloat16, device=DEV)
    dH[:, at] = _whole(g, -2, 2, 300, 80, dtype=torch.bfloat16)
    x, wg, wu, dh = X.double(), Wg[:, at].double(), Wu[:, at].double(), dH[:, at].double()
    gate, up = x @ wg, x @ wu
    dg, du = dh * up * (gate > 0), dh * gate.clamp_min(0)
    dX, dWg, dWu = osscar.osscar_gated_backward(X, lay(Wg), lay(Wu), dH, relu, dw_dtype=torch.float32)
    assert torch.equal(dX.double(), (dg @ wg.t().contiguous() + du @ wu.t().contiguous()).to(torch.bfloat16).double())
    xt = x.t().contiguous()
    assert torch.equal(dWg[:, at].double(), xt @ dg) and torch.equal(dWu[:, at].double(), xt @ du) and (dWg[:, 40:K - 40] == 0).all() and (dWu[:, 40:K - 40] == 0).all()


def test_gated_weights_whose_strides_differ_where_a_dimension_is_one(osscar):
    """what the stride of a dimension of one says does not matter"""
    g = _gen(2)
    for dtype in (torch.bfloat16, torch.float32):
        X = _randn(g, 5, 1, dtype=dtype)
        both = _randn(g, 1, 48, dtype=dtype)
        Wg, Wu = both[:, :24], torch.as_strided(both, (1, 24), (1, 1), 24)
        assert torch.equal(osscar.osscar_gated_forward(X, Wg, Wu), osscar.osscar_gated_forward(X, Wg.clone(), Wu.clone()))
        X, Wg, Wu = _randn(g, 5, 24, dtype=dtype), _randn(g, 24, 1, dtype=dtype), _randn(g, 1, 24, dtype=dtype).t()
        assert Wg.stride() != torch.as_strided(Wu, (24, 1), (1, 24)).stride()
        want = osscar.osscar_gated_forward(X, Wg, Wu.clone())
        assert torch.equal(osscar.osscar_gated_forward(X, Wg, torch.as_strided(Wu, (24, 1), (1, 24))), want)
        dH = _randn(g, 5, 1, dtype=dtype)
        for a, b in zip(osscar.osscar_gated_backward(X, Wg, torch.as_strided(Wu, (24, 1), (1, 24)), dH), osscar.osscar_gated_backward(X, Wg, Wu.clone(), dH)):
            assert torch.equal(a, b)


def test_int_product_of_one_channel_without_its_padding(osscar):
    """Wq[:, :d1] is taken for one channel as for several"""
    g = _gen(3)
    for n in (1, 5, 40):
        X, W = _randn(g, n, 20), _randn(g, 20, 2)
        Wq, ws = osscar.osscar_int_weights(W)
        want = osscar.osscar_int_product(X, Wq[:, :20], ws, out_dtype=torch.float32)
        one, s1 = osscar.osscar_int_weights(W[:, :1].contiguous())
        assert torch.equal(osscar.osscar_int_product(X, one[:, :20], s1, out_dtype=torch.float32), want[:, :1])
        assert torch.equal(osscar.osscar_int_product(X, Wq[1:, :20], ws[1:], out_dtype=torch.float32), want[:, 1:])
        with pytest.raises(osscar.OsscarError):      # a tensor that ends there is no such view
            osscar.osscar_int_product(X, torch.zeros(1, 20, dtype=torch.int8, device=DEV), s1)


# sizes of every way that the products are dealt out in: large tiles, tiles past a full chip, parts of a contraction, many parts, with rows, columns and stages left over
WHOLE = [(40, 96, 136), (300, 512, 777), (513, 65, 1030), (2100, 328, 3000), (2100, 333, 3001), (3600, 3600, 136), (3601, 1000, 137), (137, 3601, 2603), (136, 3600, 2600), (2300, 3000, 4100),
         (2303, 1001, 1000), (1100, 2700, 1900), (150, 1500, 5000), (64, 3003, 4100)] + [(2048 + r, 520, 1024 + r) for r in range(1, 9)] + [(640 + 8 * r, 1024, 264) for r in range(1, 8)]


@pytest.mark.parametrize("rows", ["in", "out"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d,f", WHOLE)
def test_gated_whole_numbers_are_exact(osscar, n, d, f, dtype, rows):
    """X and the weights in {-1, 0, 1}, dH in {-2, ..., 2} and RELU: g and u are whole numbers up to 256, which bf16 holds, as it does dg and du; every sum is a whole number
    below 2^24.  So G, U and the gradients have one right value each, rounded once where they are bf16: a single product left out, or counted twice, shows."""
    g = _gen(n + f)
    X = _whole(g, -1, 1, n, d, dtype=dtype)
    Wg, Wu = (_whole(g, -1, 1, *((f, d) if rows == "out" else (d, f)), dtype=dtype) for _ in range(2))
    if rows == "out":
        Wg, Wu = Wg.t(), Wu.t()
    dH = _whole(g, -2, 2, n, f, dtype=dtype)
    dH[dH == 0] = 1
    X64, Wg64, Wu64, dh = X.double(), Wg.double().contiguous(), Wu.double().contiguous(), dH.double()
    g64, u64 = X64 @ Wg64, X64 @ Wu64
    assert max(g64.abs().max().item(), u64.abs().max().item()) <= 256
    relu = osscar.OSSCAR_ACT_RELU
    H, G, Up = osscar.osscar_gated_forward(X, Wg, Wu, relu, save=True)
    a = g64.clamp_min(0)
    assert torch.equal(G.double(), g64) and torch.equal(Up.double(), u64) and torch.equal(H, (a * u64).to(dtype))
    dg, du = dh * u64 * (g64 > 0), dh * a
    dX64, dWg64, dWu64 = dg @ Wg64.t().contiguous() + du @ Wu64.t().contiguous(), X64.t().contiguous() @ dg, X64.t().contiguous() @ du
    for kept in (True, False):
        more = dict(G=G, U=Up) if kept else {}
        for dw_dtype in (torch.float32, torch.bfloat16):
            dX, dWg, dWu = osscar.osscar_gated_backward(X, Wg, Wu, dH, relu, dw_dtype=dw_dtype, **more)
            assert torch.equal(dX, dX64.to(dtype)) and torch.equal(dWg, dWg64.to(dw_dtype)) and torch.equal(dWu, dWu64.to(dw_dtype))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d,f", [(1, 2048, 4096), (24, 1365, 700), (150, 1500, 5000), (2100, 333, 3001), (2300, 2100, 2100)])
def test_two_calls_give_the_same_bits(osscar, n, d, f, dtype):
    g = _gen(n)
    X, dH = _randn(g, n, d, dtype=dtype), _randn(g, n, f, dtype=dtype)
    Wg, Wu = (_randn(g, d, f, scale=1 / math.sqrt(d), dtype=dtype) for _ in range(2))
    Wq, ws = osscar.osscar_int_weights(_randn(g, d, f))
    t = torch.randint(0, f, (n,), generator=g, device=DEV)

    def all_of():
        H, G, Up = osscar.osscar_gated_forward(X, Wg, Wu, save=True)
        r = osscar.osscar_logprobs(H, t, 7)
        return [H, G, Up, *osscar.osscar_gated_backward(X, Wg, Wu, dH, G=G, U=Up), *osscar.osscar_gated_backward(X, Wg, Wu, dH), osscar.osscar_int_product(X, Wq, ws), *r,
                osscar.osscar_logprobs_backward(H, t, r.lse, torch.ones(n, device=DEV), entropy=r.entropy, dentropy=torch.ones(n, device=DEV))]
    first = all_of()
    for _ in range(3):
        for a, b in zip(first, all_of()):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,v", [(3, 70), (2, 8200), (600, 9000), (2, 131072)])
def test_logprobs_of_targets_and_alternatives_masked_with_the_lowest_value(osscar, n, v, dtype):
    """their log probability is the mask's value times the scale, as long as that is a float: not minus infinity"""
    g = _gen(v)
    low = torch.finfo(dtype).min
    L = torch.full((n, v), low, dtype=dtype, device=DEV)
    L[:, 2:7] = _randn(g, n, 5, scale=2.5, dtype=dtype)
    t = torch.randint(7, v, (n,), generator=g, device=DEV)
    for scale in (1.0, 0.75, 0.01, 4.0):
        lp = torch.log_softmax(L.double() * scale, 1)
        r = osscar.osscar_logprobs(L, t, 33, scale)
        order = torch.sort(L.float(), dim=1, descending=True, stable=True).indices[:, :33]
        assert torch.equal(r.top_index, order)
        for got, want in ((r.logp, lp.gather(1, t[:, None])[:, 0]), (r.top_logp, lp.gather(1, order))):
            fine = torch.isfinite(want.float())
            assert torch.equal(torch.isfinite(got), fine) and ((got.double() - want)[fine].abs() <= 2e-6 * (1 + want[fine].abs() / 2)).all()
            assert (got[~fine] == -math.inf).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprobs_of_logits_whose_difference_is_no_float(osscar, dtype):
    """logits from one end of the type to the other, at a scale that makes ordinary numbers of them; the gradient in units of the scale"""
    g = _gen(31)
    for n, v in ((3, 70), (2, 8200), (600, 9000), (2, 70000)):
        L = (torch.rand(n, v, generator=g, device=DEV) * 2 - 1).mul_(3.3e38).to(dtype)
        t = torch.randint(0, v, (n,), generator=g, device=DEV)
        scale = 2.0 ** -125
        lp = torch.log_softmax(L.double() * scale, 1)
        r = osscar.osscar_logprobs(L, t, 5, scale)
        want = lp.gather(1, t[:, None])[:, 0]
        assert ((r.logp.double() - want).abs() <= 2e-6 * (1 + want.abs() / 2)).all()
        entropy = -(lp * lp.exp()).sum(1)
        assert ((r.entropy.double() - entropy).abs() <= 5e-6 * (1 + entropy)).all()
        assert torch.equal(r.top_index, torch.sort(L.float(), dim=1, descending=True, stable=True).indices[:, :5])
        unit = 2.0 ** 100
        d = osscar.osscar_logprobs_backward(L, t, r.lse, torch.full((n,), unit, device=DEV), scale=scale)
        p = lp.exp()
        hot = torch.zeros_like(p).scatter_(1, t[:, None], 1.0)
        assert ((d.double() / (unit * scale) - (hot - p)).abs() <= 8e-6 * (1 + lp.abs()) * (hot + p) + 2.0 ** -8 * (hot - p).abs() * (dtype == torch.bfloat16)).all()


def test_logprobs_at_the_largest_scale(osscar):
    """one-hot rows, ties in halves"""
    L = torch.tensor([[1.0, 2.0, -3.0, 0.5], [2.0, 2.0, 1.0, -1.0], [0.0, -1e-3, -1e30, -math.inf]], device=DEV)
    t = torch.tensor([1, 0, 0], device=DEV)
    r = osscar.osscar_logprobs(L, t, 2, 2.3e38)
    half = math.log(0.5)
    assert torch.allclose(r.logp, torch.tensor([0.0, half, 0.0], device=DEV), atol=1e-6) and torch.allclose(r.entropy, torch.tensor([0.0, -half, 0.0], device=DEV), atol=1e-6)
    assert r.top_index.tolist() == [[1, 0], [0, 1], [0, 1]]


def test_results_are_constants_to_autograd(osscar):
    """also of arguments that require a gradient; torch's part of a loss goes on from a result, the layer's part is the backward call's"""
    g = _gen(8)
    X, Wg, Wu = (_randn(g, *s).requires_grad_() for s in ((20, 48), (48, 64), (48, 64)))
    Wd = _randn(g, 64, 90).requires_grad_()
    t = torch.randint(0, 90, (20,), generator=g, device=DEV)
    H, G, U = osscar.osscar_gated_forward(X, Wg, Wu, save=True)
    assert not (H.requires_grad or G.requires_grad or U.requires_grad)
    H.requires_grad_()
    logits = H @ Wd
    r = osscar.osscar_logprobs(logits, t)
    assert not (r.logp.requires_grad or r.entropy.requires_grad)
    logits.backward(osscar.osscar_logprobs_backward(logits, t, r.lse, torch.ones(20, device=DEV)))
    assert Wd.grad is not None and Wg.grad is None
    dX, dWg, dWu = osscar.osscar_gated_backward(X, Wg, Wu, H.grad, G=G, U=U)
    x, wg, wu = (a.detach().double().cpu().requires_grad_() for a in (X, Wg, Wu))
    h = torch.nn.functional.silu(x @ wg) * (x @ wu)
    torch.log_softmax(h @ Wd.detach().double().cpu(), 1).gather(1, t.cpu()[:, None]).sum().backward()
    for got, want in ((dX, x.grad), (dWg, wg.grad), (dWu, wu.grad)):
        assert (got.double().cpu() - want).norm() <= 1e-5 * want.norm()
