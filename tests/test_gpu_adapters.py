"""Low-rank adapters against a plain float64 implementation of their definition.

Tolerances, elementwise.  u = 2^-8 is the largest relative error of rounding to bf16, e = 2^-24 that of float32; a float32 sum of K products is off by a random walk of about e sqrt(K) of the sum of their
sizes, walk(K) = e (4 + 2 sqrt(K)) is allowed.  The float32 factor of a bf16 product goes in as two pieces of bf16 (2^-16 of it is left out; three pieces, 2^-24, for float32 gradients).  So
T is off by walk(d) |X||A|, Y by what that and the pieces do to each of its terms, by its own sum's walk and by its rounding; the gradients likewise."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, E = 2.0 ** -8, 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16


def walk(K):
    return E * (4 + 2 * math.sqrt(K))


@pytest.fixture(scope="module")
def osscar():
    import paper_2403_12983_amd as pkg
    pkg.load_library()
    return pkg


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape, scale=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device=DEV) * scale).to(dtype)


def _within(got, want, tolerance, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape and torch.equal(torch.isfinite(got), torch.isfinite(want)), what
    over = torch.where(torch.isfinite(want), (got - want).abs() - tolerance, torch.zeros_like(want))
    assert over.numel() == 0 or over.max().item() <= 0, (what, over.max().item(), (got - want).abs().max().item())


def _case(g, n, d, m, count, r, dtype, order, ragged=False):
    X, dY = _randn(g, n, d, dtype=dtype), _randn(g, n, m, dtype=dtype)
    A, B = _randn(g, count, r, d, scale=1 / math.sqrt(d), dtype=dtype), _randn(g, count, r, m, scale=0.3, dtype=dtype)
    index = None
    if order != "one":
        index = torch.randint(-1, count, (n,), generator=g, device=DEV)
        if order == "runs":
            index = torch.sort(index).values
    scale = 0.5 + torch.rand(count, generator=g, device=DEV) * 3
    ranks = torch.randint(0, r + 1, (count,), generator=g, device=DEV, dtype=torch.int32) if ragged else None
    return X, dY, A, B, dict(index=index, scale=scale, ranks=ranks)


def _exact(X, dY, A, B, index, scale, ranks, rounding, piece):
    """{name: (value, tolerance without the result's own rounding)}; rounding of T's factor by `piece`"""
    n, d, m, (count, r) = X.shape[0], X.shape[1], B.shape[2], A.shape[:2]
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=DEV)  # noqa: E731
    out = {k: [z(*s), z(*s)] for k, s in (("T", (n, r)), ("Y", (n, m)), ("dX", (n, d)), ("dA", A.shape), ("dB", B.shape))}
    for e in range(count):
        rows = torch.arange(n, device=DEV) if index is None else torch.nonzero(index == e)[:, 0]
        if index is None and e > 0:
            break
        k = r if ranks is None else int(ranks[e])
        a, b, s = A[e, :k].double(), B[e, :k].double(), 1.0 if scale is None else float(scale[e])
        x, dy, c = X[rows].double(), dY[rows].double(), len(rows)
        at, bt = a.t().contiguous(), b.t().contiguous()
        t, tm = x @ at, x.abs() @ at.abs()
        dt, dtm = s * (dy @ bt), s * (dy.abs() @ bt.abs())
        terr, dterr = walk(d) * tm + 3 * E * t.abs(), walk(m) * dtm + 3 * E * dt.abs()
        out["T"][0][rows, :k], out["T"][1][rows, :k] = t, terr
        out["Y"][0][rows], out["Y"][1][rows] = s * (t @ b), s * ((terr + (piece + walk(k)) * t.abs()) @ b.abs())
        out["dX"][0][rows], out["dX"][1][rows] = dt @ a, (dterr + (piece + walk(k)) * dt.abs()) @ a.abs()
        for name, p, perr, q in (("dA", dt, dterr, x), ("dB", s * t, s * terr, dy)):
            pt = p.t().contiguous()
            out[name][0][e, :k] = pt @ q
            out[name][1][e, :k] = (perr.t().contiguous() + (rounding + walk(c) + 2 * E) * pt.abs()) @ q.abs()
    return out


def _check(pkg, X, dY, A, B, more, base=None, dbase=None, dw_dtype=None, T_kept=True):
    dw_dtype = dw_dtype or X.dtype
    bf16 = X.dtype == BF16
    own = U if bf16 else E
    want = _exact(X, dY, A, B, **more, rounding=0.0 if not bf16 else 2.0 ** -16 if dw_dtype == BF16 else 2.0 ** -24, piece=2.0 ** -16 if bf16 else 0.0)
    Y, T = pkg.osscar_adapters_forward(X, A, B, base=base, save=True, **more)
    for name, add in (("Y", base), ("dX", dbase)):
        if add is not None:
            want[name][0] += add.double()
            want[name][1] += E * add.double().abs()
    _within(T, want["T"][0], want["T"][1], "T")
    _within(Y, want["Y"][0], want["Y"][1] + own * 1.01 * want["Y"][0].abs(), "Y")
    got = pkg.osscar_adapters_backward(X, A, B, dY, T=T if T_kept else None, base=dbase, dw_dtype=dw_dtype, **more)
    for name, x, o in zip(("dX", "dA", "dB"), got, (own, U if dw_dtype == BF16 else E, U if dw_dtype == BF16 else E)):
        _within(x, want[name][0], want[name][1] + o * 1.01 * want[name][0].abs(), name)
    assert got[0].dtype == X.dtype == Y.dtype and got[1].dtype == got[2].dtype == dw_dtype
    assert torch.equal(Y, pkg.osscar_adapters_forward(X, A, B, base=base, **more))      # without keeping, the same bits again
    again = pkg.osscar_adapters_backward(X, A, B, dY, T=T if T_kept else None, base=dbase, dw_dtype=dw_dtype, **more)
    assert all(torch.equal(x, y) for x, y in zip(got, again))
    return Y, T, got


SIZES = [(1, 1, 1, 1, 1), (1, 2048, 300, 4, 16), (3, 7, 9, 2, 3), (2, 64, 130, 3, 8), (16, 300, 520, 32, 16), (17, 136, 77, 5, 17), (31, 33, 640, 3, 4), (33, 513, 129, 40, 12), (64, 128, 256, 7, 32),
         (70, 1365, 200, 3, 33), (200, 512, 1030, 90, 5), (300, 257, 128, 2, 64), (513, 130, 300, 6, 65), (777, 96, 1365, 3, 12), (1500, 520, 136, 2, 130), (2100, 40, 48, 300, 2), (65, 600, 520, 2, 16), (256, 520, 640, 20, 20), (257, 520, 640, 20, 20), (2, 9000, 70, 2, 100)]


@pytest.mark.parametrize("order", ["one", "runs", "mixed"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,m,count,r", SIZES)
def test_adapters(osscar, n, d, m, count, r, dtype, order):
    g = _gen(n + d + m)
    X, dY, A, B, more = _case(g, n, d, m, 1 if order == "one" else count, r, dtype, order, ragged=order == "mixed" and n % 2 == 1)
    base, dbase = (_randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype)) if (n + r) % 3 else (None, None)
    _check(osscar, X, dY, A, B, more, base, dbase)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("order", ["runs", "mixed"])
def test_adapters_float32_gradients_and_without_kept_products(osscar, order, dtype):
    g = _gen(2)
    X, dY, A, B, more = _case(g, 610, 333, 270, 4, 24, dtype, order)
    Y, T, got = _check(osscar, X, dY, A, B, more, dw_dtype=F32, T_kept=False)
    kept = osscar.osscar_adapters_backward(X, A, B, dY, T=T, dw_dtype=F32, **more)
    assert torch.equal(kept[0], got[0]) and torch.equal(kept[1], got[1])
    only = osscar.osscar_adapters_backward(X, A, B, dY, T=T, need_w=False, **more)
    assert only[1] is None and only[2] is None and torch.equal(only[0], got[0])
    only = osscar.osscar_adapters_backward(X, A, B, dY, T=T, need_x=False, dw_dtype=F32, **more)
    assert only[0] is None
    want = _exact(X, dY, A, B, **more, rounding=2.0 ** -24, piece=2.0 ** -16)
    for name, x in (("dA", only[1]), ("dB", only[2])):
        _within(x, want[name][0], want[name][1] + E * 1.01 * want[name][0].abs(), name)
    more["scale"] = None
    _check(osscar, X, dY, A, B, more)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_adapters_long_contractions_in_parts(osscar, dtype):
    g = _gen(3)
    for n, d, m, count, r in ((5, 14336, 7161, 3, 16), (40, 7168, 9001, 2, 64)):
        X, dY, A, B, more = _case(g, n, d, m, count, r, dtype, "mixed")
        _check(osscar, X, dY, A, B, more, _randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype))


def _strided(t, pad, shift):
    n, d = t.shape
    flat = torch.full((shift + n * (d + pad),), 7.0, dtype=t.dtype, device=t.device)
    view = flat[shift:].view(n, d + pad)[:, :d]
    view.copy_(t)
    return view, flat


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,m,r", [(5, 33, 50, 3), (65, 264, 391, 16), (130, 129, 640, 40)])
def test_adapters_strides_alignments_and_places(osscar, n, d, m, r, dtype):
    g = _gen(n)
    X0, dY0, A0, B0, more = _case(g, n, d, m, 3, r, dtype, "mixed", ragged=True)
    base0, dbase0 = _randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype)
    Y0, T0, got0 = _check(osscar, X0, dY0, A0, B0, more, base0, dbase0)
    for pad, shift in ((0, 1), (3, 0), (5, 3), (8, 8)):
        X, dY = _strided(X0, pad, shift)[0], _strided(dY0, pad, shift)[0]
        A = _strided(A0.reshape(3 * r, d), pad, shift)[0].view(3, r, d)
        B = _strided(B0.reshape(3 * r, m), pad, shift)[0].view(3, r, m)
        (base, fb), (dbase, fd) = _strided(base0, pad, shift), _strided(dbase0, pad, shift)
        (out, fo), (dout, fdo) = _strided(torch.zeros_like(base0), pad, shift), _strided(torch.zeros_like(dbase0), pad, shift)
        Y, T = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, out=out, **more)
        got = osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase, out=dout, **more)
        assert Y is out and got[0] is dout and torch.equal(Y, Y0) and torch.equal(T, T0) and all(torch.equal(x, y) for x, y in zip(got, got0))
        for flat, value, width in ((fo, Y0, m), (fdo, got0[0], d)):      # nothing beside the rows
            want = torch.full_like(flat, 7.0)
            want[shift:].view(n, width + pad)[:, :width] = value
            assert torch.equal(flat, want)
        # in place; rows without an adapter stay as they are
        osscar.osscar_adapters_forward(X, A, B, base=base, out=base, **more)
        osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase, out=dbase, need_w=False, **more)
        assert torch.equal(base, Y0) and torch.equal(dbase, got0[0])
        none = more["index"] < 0
        assert torch.equal(base[none], base0[none])
        for flat, value, width in ((fb, Y0, m), (fd, got0[0], d)):
            want = torch.full_like(flat, 7.0)
            want[shift:].view(n, width + pad)[:, :width] = value
            assert torch.equal(flat, want)
    # one set of weights for all adapters, by a stride of zero
    one = dict(more, ranks=None)
    A, B = A0[:1].expand(3, r, d), B0[:1].expand(3, r, m)
    got = osscar.osscar_adapters_forward(X0, A, B, **one)
    assert torch.equal(got, osscar.osscar_adapters_forward(X0, A.contiguous(), B.contiguous(), **one))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_adapters_rows_without_adapters_and_wrong_ones(osscar, dtype):
    g = _gen(5)
    n, d, m, count, r = 90, 200, 300, 4, 8
    X, dY, A, B, more = _case(g, n, d, m, count, r, dtype, "mixed")
    base, dbase = _randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype)
    good = osscar.osscar_adapters_forward(X, A, B, base=base, **more)
    index = more["index"].clone()
    wrong = [3, 40, 89]
    index[wrong] = torch.tensor([count, 1 << 40, count + 1], device=DEV)
    Y, T = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, **dict(more, index=index))
    dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase, **dict(more, index=index))
    assert torch.isnan(Y[wrong]).all() and torch.isnan(dX[wrong]).all() and not T[wrong].any()
    rest = [k for k in range(n) if k not in wrong]
    assert torch.equal(Y[rest], good[rest]) and torch.isfinite(dX[rest]).all() and torch.isfinite(dA).all() and torch.isfinite(dB).all()
    # no row has an adapter
    index = torch.full_like(index, -7)
    Y, T = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, **dict(more, index=index))
    dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase, **dict(more, index=index))
    assert torch.equal(Y, base) and torch.equal(dX, dbase) and not T.any() and not dA.any() and not dB.any()
    assert not osscar.osscar_adapters_forward(X, A, B, **dict(more, index=index)).any()
    # no rows; rank 0
    none = dict(more, index=index[:0])
    Y, T = osscar.osscar_adapters_forward(X[:0], A, B, save=True, **none)
    dX, dA, dB = osscar.osscar_adapters_backward(X[:0], A, B, dY[:0], T=T, **none)
    assert Y.shape == (0, m) and dX.shape == (0, d) and not dA.any() and not dB.any()
    dX, dA, dB = osscar.osscar_adapters_backward(X[:0], A, B, dY[:0], scale=more["scale"])
    assert not dA.any() and not dB.any()
    zero = dict(more, ranks=torch.zeros(count, dtype=torch.int32, device=DEV))
    Y, T = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, **zero)
    got = osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase, **zero)
    assert torch.equal(Y, base) and not T.any() and torch.equal(got[0], dbase) and not got[1].any() and not got[2].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_adapters_keep_what_is_not_finite_to_itself(osscar, bad, dtype):
    g = _gen(6)
    n, d, m, count, r = 70, 100, 200, 5, 10
    X, dY, A, B, more = _case(g, n, d, m, count, r, dtype, "mixed")
    more["ranks"] = torch.tensor([10, 4, 7, 10, 10], dtype=torch.int32, device=DEV)
    index = more["index"]
    index[:3] = torch.tensor([0, 1, -1], device=DEV)
    base = _randn(g, n, m, dtype=dtype)
    Y0, T0 = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, **more)
    got0 = osscar.osscar_adapters_backward(X, A, B, dY, T=T0, **more)
    A2, B2, X2, dY2 = A.clone(), B.clone(), X.clone(), dY.clone()
    A2[2, 7:], B2[2, 7:] = bad, bad      # components that do not count
    A2[4, 3, 5], B2[3, 2, 9] = bad, bad  # an adapter of its own each
    X2[2], dY2[2] = bad, bad             # a row without an adapter
    Y, T = osscar.osscar_adapters_forward(X2, A2, B2, base=base, save=True, **more)
    dX, dA, dB = osscar.osscar_adapters_backward(X2, A2, B2, dY2, T=T, **more)
    fine = ~((index == 3) | (index == 4))
    assert torch.equal(Y[fine], Y0[fine]) and torch.equal(T[fine], T0[fine]) and torch.equal(dX[fine], got0[0][fine])
    assert torch.equal(dA[:3], got0[1][:3]) and torch.equal(dB[:3], got0[2][:3]) and torch.equal(dB[3], got0[2][3]) and torch.equal(dA[4], got0[1][4])
    assert not torch.isfinite(Y[index == 3][:, 9]).any() and torch.isfinite(Y[index == 3][:, :9]).all() and not torch.isfinite(Y[index == 4]).all(1).any()
    # a row of an adapter: its own results, and its adapter's gradients
    X2 = X.clone()
    X2[0, 4] = bad
    Y, T = osscar.osscar_adapters_forward(X2, A, B, base=base, save=True, **more)
    dX, dA, dB = osscar.osscar_adapters_backward(X2, A, B, dY, T=T, **more)
    assert not torch.isfinite(Y[0]).any() and torch.equal(Y[1:], Y0[1:]) and torch.equal(dX, got0[0])
    assert not torch.isfinite(dA[0, :, 4]).any() and torch.equal(dA[1:], got0[1][1:]) and torch.equal(dB[1:], got0[2][1:])


def test_adapters_many_adapters_and_rows(osscar):
    g = _gen(7)
    for n, count, order in ((9000, 4096, "mixed"), (70000, 3, "mixed"), (5000, 2049, "runs")):
        X, dY, A, B, more = _case(g, n, 24, 40, count, 2, BF16, order)
        Y, T = osscar.osscar_adapters_forward(X, A, B, save=True, **more)
        dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, dw_dtype=F32, **more)
        has = more["index"] >= 0
        at = more["index"].clamp_min(0)
        s = more["scale"].double()[at] * has
        a, b = A.double()[at], B.double()[at]
        t = (a * X.double()[:, None]).sum(2)
        dt = (b * dY.double()[:, None]).sum(2) * s[:, None]
        mass = lambda p, q, e: (p.abs()[:, :, None] * q.abs()[:, None]) * e  # noqa: E731
        y = ((t * s[:, None])[:, :, None] * b).sum(1)
        ymass = ((a.abs() * X.double().abs()[:, None]).sum(2) * s[:, None])[:, :, None] * b.abs()
        _within(Y, y, 2.0 ** -15 * ymass.sum(1) + U * 1.01 * y.abs(), "Y")
        for got, p, q, pm in ((dA, dt, X, (b.abs() * dY.double().abs()[:, None]).sum(2) * s[:, None]), (dB, t * s[:, None], dY, (a.abs() * X.double().abs()[:, None]).sum(2) * s[:, None])):
            want = torch.zeros(got.shape, dtype=torch.float64, device=DEV).index_add_(0, at, p[:, :, None] * q.double()[:, None])
            size = torch.zeros(got.shape, dtype=torch.float64, device=DEV).index_add_(0, at, mass(pm, q.double(), 1.0))
            _within(got, want, (2 * walk(40) + walk(n // count + 100) + 2.0 ** -23) * size, "gradient")


def test_adapters_gradients_against_differences(osscar):
    """The loss sum dY Y is linear in each of X, A and B: differences over a step of any size are its slope, but for float32's rounding of Y over the step."""
    g = _gen(8)
    n, d, m, count, r = 60, 90, 110, 3, 6
    X, dY, A, B, more = _case(g, n, d, m, count, r, F32, "mixed")
    got = osscar.osscar_adapters_backward(X, A, B, dY, **more)
    for k, (w, dw) in enumerate(zip((X, A, B), got)):
        V = _randn(g, *w.shape)
        f = []
        for sign in (1, -1):
            args = [X, A, B]
            args[k] = w + sign * V
            y = osscar.osscar_adapters_forward(*args, **more).double()
            f.append(((dY.double() * y).sum(), (dY.double() * y).abs().sum()))
        slope, size = (f[0][0] - f[1][0]).item() / 2, (f[0][1] + f[1][1]).item()
        assert abs((dw.double() * V.double()).sum().item() - slope) <= 4 * (walk(d) + walk(n)) * size


def test_adapters_captured_and_on_another_stream(osscar):
    g = _gen(9)
    X, dY, A, B, more = _case(g, 300, 400, 500, 6, 16, BF16, "mixed")
    base = _randn(g, 300, 500, dtype=BF16)

    def both(**kw):
        Y, T = osscar.osscar_adapters_forward(X, A, B, base=base, save=True, **more, **kw)
        return (Y, *osscar.osscar_adapters_backward(X, A, B, dY, T=T, **more, **kw))

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = both(stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, both()))
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):      # two graphs, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both()
        graphs.append((graph, out))
    for k in range(4):
        X.copy_(_randn(g, 300, 400, dtype=BF16))
        more["index"].copy_(torch.randint(-1, 6, (300,), generator=g, device=DEV))
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, both()))
        torch.cuda.synchronize()


# rows of many adapters are put in their order: sizes at both sides of that, most tiles with several adapters, more adapters than rows
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,d,m,count,r", [(511, 130, 264, 8, 12), (512, 130, 264, 8, 12), (512, 97, 300, 7, 16), (640, 2100, 391, 9, 33), (1100, 130, 1030, 40, 20), (700, 64, 72, 4096, 2), (3333, 264, 200, 17, 70)])
def test_adapters_rows_put_in_order(osscar, n, d, m, count, r, dtype):
    g = _gen(n + count)
    X, dY, A, B, more = _case(g, n, d, m, count, r, dtype, "mixed", ragged=True)
    base, dbase = _randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype)
    Y, T, got = _check(osscar, X, dY, A, B, more, base, dbase)
    # a row's result does not know where it lies, nor its neighbours'
    at = torch.randperm(n, generator=g, device=DEV)
    moved = dict(more, index=more["index"][at].contiguous())
    Y2, T2 = osscar.osscar_adapters_forward(X[at].contiguous(), A, B, base=base[at].contiguous(), save=True, **moved)
    dX2 = osscar.osscar_adapters_backward(X[at].contiguous(), A, B, dY[at].contiguous(), T=T2, base=dbase[at].contiguous(), **moved)[0]
    assert torch.equal(Y2, Y[at]) and torch.equal(T2, T[at]) and torch.equal(dX2, got[0][at])
    # in place
    out = base.clone()
    osscar.osscar_adapters_forward(X, A, B, base=out, out=out, **more)
    assert torch.equal(out, Y)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_adapters_rows_put_in_order_without_adapters_and_with_wrong_ones(osscar, dtype):
    g = _gen(15)
    n, d, m, count, r = 900, 200, 300, 12, 8
    X, dY, A, B, more = _case(g, n, d, m, count, r, dtype, "mixed")
    base, dbase = _randn(g, n, m, dtype=dtype), _randn(g, n, d, dtype=dtype)
    good = osscar.osscar_adapters_forward(X, A, B, base=base, **more)
    index = more["index"].clone()
    wrong = [0, 40, 64, 513, 899]
    index[wrong] = torch.tensor([count, 1 << 40, count + 1, 15, 1 << 32], device=DEV)
    index[700:790] = torch.tensor([-1, -5, -(1 << 40)], device=DEV).repeat(30)
    rest = torch.tensor([k for k in range(n) if k not in wrong and not 700 <= k < 790], device=DEV)
    for out, dout in ((None, None), (base.clone(), dbase.clone())):
        use = dict(more, index=index)
        Y, T = osscar.osscar_adapters_forward(X, A, B, base=base if out is None else out, out=out, save=True, **use)
        dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, base=dbase if dout is None else dout, out=dout, **use)
        assert torch.isnan(Y[wrong]).all() and torch.isnan(dX[wrong]).all() and not T[wrong].any()
        assert torch.equal(Y[700:790], base[700:790]) and torch.equal(dX[700:790], dbase[700:790]) and not T[700:790].any()
        assert torch.equal(Y[rest], good[rest]) and torch.isfinite(dX[rest]).all() and torch.isfinite(dA).all() and torch.isfinite(dB).all()
    none = dict(more, index=torch.full((n,), -1, device=DEV))
    Y, T = osscar.osscar_adapters_forward(X, A, B, save=True, **none)
    dX, dA, dB = osscar.osscar_adapters_backward(X, A, B, dY, T=T, **none)
    assert not Y.any() and not T.any() and not dX.any() and not dA.any() and not dB.any()
    X, A = X.clone(), A.clone()      # what is not finite stays with its rows
    X[5] = math.nan
    A[3] = math.inf
    clean = [k for k in rest.tolist() if k != 5 and index[k] != 3]
    assert torch.equal(osscar.osscar_adapters_forward(X, A, B, base=base, **dict(more, index=index))[clean], good[clean])


def test_adapters_rows_put_in_order_in_graphs(osscar):
    g = _gen(16)
    X, dY, A, B, more = _case(g, 600, 400, 264, 20, 16, BF16, "mixed")

    def both():
        Y, T = osscar.osscar_adapters_forward(X, A, B, save=True, **more)
        return (Y, T) + tuple(osscar.osscar_adapters_backward(X, A, B, dY, T=T, **more))

    both()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both()
        graphs.append((graph, out))
    for k in range(5):
        X.copy_(_randn(g, 600, 400, dtype=BF16))
        more["index"].copy_(torch.randint(-1, (22, 3, 20)[k % 3], (600,), generator=g, device=DEV))
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) and torch.equal(torch.isnan(x), torch.isnan(y)) for x, y in zip(out, both()))
        torch.cuda.synchronize()


def test_adapters_refusals(osscar):
    X, dY, base = torch.zeros(4, 16, device=DEV), torch.zeros(4, 24, device=DEV), torch.zeros(4, 24, device=DEV)
    A, B = torch.zeros(2, 3, 16, device=DEV), torch.zeros(2, 3, 24, device=DEV)
    index, scale, ranks = torch.zeros(4, dtype=torch.int64, device=DEV), torch.ones(2, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV)
    F, G = osscar.osscar_adapters_forward, osscar.osscar_adapters_backward
    T = torch.zeros(4, 3, device=DEV)
    bad = [lambda: F(X.half(), A.half(), B.half()), lambda: F(X, A.bfloat16(), B), lambda: F(X, A, B.bfloat16()), lambda: F(X[0], A, B), lambda: F(X, A[0], B), lambda: F(X, A[:, :, :8], B),
           lambda: F(X, A[:1], B), lambda: F(X, A[:, :2], B), lambda: F(X, A.transpose(1, 2), B), lambda: F(X.t(), A, B), lambda: F(X, A.cpu(), B), lambda: F(X, A, B, index=index[:3]),
           lambda: F(X, A, B, index=index.int()), lambda: F(X, A, B, index=index.cpu()), lambda: F(X, A, B, scale=scale[:1]), lambda: F(X, A, B, scale=scale.double()),
           lambda: F(X, A, B, ranks=ranks.long()), lambda: F(X, A, B, base=base[:3]), lambda: F(X, A, B, base=base.bfloat16()), lambda: F(X, A, B, out=base[:, :5]),
           lambda: F(X, A, B, out=base.cpu()), lambda: F(X, A[:, :0], B[:, :0]), lambda: F(X, A[:0], B[:0]),
           lambda: F(X, A[:1].expand(5000, 3, 16), B[:1].expand(5000, 3, 24)), lambda: F(X, A[:, :1].expand(2, 1025, 16), B[:, :1].expand(2, 1025, 24)),
           lambda: G(X, A, B, dY[:3]), lambda: G(X, A, B, dY.bfloat16()), lambda: G(X, A, B, dY, T=T[:, :2]), lambda: G(X, A, B, dY, T=T.double()), lambda: G(X, A, B, dY, base=base),
           lambda: G(X, A, B, dY, need_x=False, base=X), lambda: G(X, A, B, dY, need_x=False, out=X), lambda: G(X, A, B, dY, dw_dtype=torch.half), lambda: G(X, A, B, dY, out=base)]
    for k, call in enumerate(bad):
        with pytest.raises(osscar.OsscarError) as e:
            call()
        assert e.value.status == 1, k
